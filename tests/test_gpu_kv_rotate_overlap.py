"""Turned queries whose memory is read by others of the same call: refused where it can be seen, before anything is launched."""
import pytest
import torch

from test_gpu_kv_cache import Case, ints, lpq  # noqa: F401  (lpq is a fixture)

pytestmark = pytest.mark.gpu


def test_outputs_in_the_place_of_what_is_read_are_refused(lpq):
    c = Case(lpq, 2, 64, 16, [40, 20], "bf16")
    k, v = torch.cat(c.k).cuda(), torch.cat(c.v).cuda()
    cos = torch.ones(50, 32, device="cuda")
    before, k0, v0 = c.cache.k.clone(), k.clone(), v.clone()

    def code(q, out):
        with pytest.raises(lpq.LpqError) as e:
            c.cache.write_rotated(k, v, ints([0, 0]), c.table, cos, cos, starts=ints([0, 40, 60]), q=q, out=out)
        return e.value.code
    q = torch.randn(60, 2, 64, device="cuda").bfloat16()
    assert code(q, k) == lpq.EINVAL and code(q, v) == lpq.EINVAL and code(k, k) == lpq.EINVAL
    room = torch.zeros(60, 4, 64, dtype=torch.bfloat16, device="cuda")
    assert code(room[:, :2], room.view(-1, 64)[:120].view(60, 2, 64)) == lpq.EINVAL          # where the queries begin, with other strides
    assert code(room[:, ::2], room[:, :2]) == lpq.EINVAL
    assert torch.equal(c.cache.k, before) and torch.equal(k, k0) and torch.equal(v, v0) and not room.any()
    # in place, and beside the keys in one tensor
    packed = torch.cat([q, k, v], 1)
    want = c.cache.write_rotated(k, v, ints([0, 0]), c.table, cos, cos, starts=ints([0, 40, 60]), q=q)
    got = c.cache.write_rotated(packed[:, 2:4], packed[:, 4:], ints([0, 0]), c.table, cos, cos, starts=ints([0, 40, 60]), q=packed[:, :2], out=packed[:, :2])
    assert torch.equal(got, want) and torch.equal(packed[:, 2:4], k0)
