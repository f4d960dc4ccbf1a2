"""Calls of the decoder layer on codes that would drop a gradient refuse the input that asks for one, before they look at its memory: no device needed."""
import os
from types import SimpleNamespace

import pytest
import torch
from torch.autograd import forward_ad


@pytest.fixture(scope="module")
def lpq():
    from paper_2110_08919_amd import build, lpq as m
    if not os.path.exists(m.LIB_PATH):
        build.build()
    m.lib()
    return m


@pytest.mark.parametrize("which", ["k", "v", "q", "cos", "sin"])
def test_rotated_rows_and_angles(lpq, which, monkeypatch):
    monkeypatch.setattr(lpq, "_current_device", lambda: 0)
    cache = object.__new__(lpq.KVCache)
    cache._at = 0
    given = {name: torch.zeros(1, 1, 4) for name in ("k", "v", "q")} | {name: torch.ones(1, 2) for name in ("cos", "sin")}
    given[which].requires_grad_()
    ints = torch.zeros(1, dtype=torch.int32)
    with pytest.raises(AssertionError, match="gradient"):
        cache.write_rotated(first=ints, table=ints[None], **given)
    with torch.no_grad(), pytest.raises(AssertionError, match="device"):      # taken, and then refused for where it lies
        cache.write_rotated(first=ints, table=ints[None], **given)


def test_a_bias_of_products(lpq):
    codes = SimpleNamespace(d=64, n=3, blocks=torch.zeros(1))
    bias = torch.zeros(3, requires_grad=True)
    with pytest.raises(AssertionError, match="gradient"):
        lpq.matmul_i8(codes, codes, bias)
    with torch.no_grad(), pytest.raises(AssertionError, match="device"):
        lpq.matmul_i8(codes, codes, bias)


def test_tangents(lpq):
    """Forward-mode derivatives are refused too, also where gradients are off: they would be dropped."""
    ints = torch.zeros(1, dtype=torch.int32)
    cache, layer = object.__new__(lpq.KVCache), object.__new__(lpq.Linear8)
    with forward_ad.dual_level():
        dual = forward_ad.make_dual(torch.zeros(3, 4), torch.ones(3, 4))
        rows, bias = dual[:1, None], dual[:, 0]
        codes = SimpleNamespace(d=64, n=3, blocks=torch.zeros(1))
        plain = torch.zeros(1, 1, 4)
        calls = [lambda: lpq.encode_rows(dual), lambda: layer(dual), lambda: lpq.matmul_i8(codes, codes, bias),
                 lambda: cache.attend(dual[None, :1, None], ints, ints[None], window=3),
                 lambda: cache.write_rotated(rows, plain, ints, ints[None], plain[0, :, :2], plain[0, :, :2]),
                 lambda: cache.write_rotated(plain, plain, ints, ints[None], plain[0, :, :2], plain[0, :, :2], q=rows)]
        for call in calls:
            with pytest.raises(AssertionError, match="tangent"):
                call()
            with torch.no_grad(), pytest.raises(AssertionError, match="tangent"):
                call()
        with pytest.raises(AssertionError, match="device"):                    # without one: refused for where it lies
            lpq.encode_rows(torch.zeros(3, 4))
