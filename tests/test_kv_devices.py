"""Memory of another device than the cache's is refused before a kernel gets its address, and so are calls with another current device.  None of it needs one."""
import os
from types import SimpleNamespace

import pytest
import torch


@pytest.fixture(scope="module")
def lpq():
    from paper_2110_08919_amd import build, lpq as m
    if not os.path.exists(m.LIB_PATH):
        build.build()
    m.lib()
    return m


class On:
    """A tensor that says it lies on device `at`."""

    def __init__(self, t, at):
        self.t, self.at, self.is_cuda = t, at, at >= 0

    def get_device(self):
        return self.at

    @property
    def device(self):
        return torch.device("cuda", self.at)

    def __getattr__(self, name):
        return getattr(self.t, name)


@pytest.fixture
def cache(lpq, monkeypatch):
    c = object.__new__(lpq.KVCache)
    c.heads, c.dim, c.page, c.pages, c._at, c._h = 1, 4, 16, 1, 1, None
    calls = []
    names = [f"lpq_kv_{name}" for name in ("write", "write_rotated", "read", "select", "attend", "attend_masked")]
    functions = {name: (lambda *arguments, name=name: calls.append(name) or 0) for name in names}
    workspaces = {f"lpq_kv_{name}_workspace_bytes": lambda *arguments: 0 for name in ("select", "attend", "attend_masked")}
    monkeypatch.setattr(lpq, "_lib", SimpleNamespace(**functions, **workspaces))
    monkeypatch.setattr(lpq, "_current_device", lambda: 1)
    monkeypatch.setattr(lpq, "_stream_of", lambda t: 0)
    c.calls = calls
    return c


def test_each_argument_of_a_call(lpq, cache):
    rows, ints = torch.zeros(2, 1, 4), torch.zeros(2, dtype=torch.int32)
    angles, table = torch.ones(1, 2), torch.zeros(2, 1, dtype=torch.int32)
    queries, pages, tree = torch.zeros(2, 1, 1, 4), torch.zeros(2, 1, 1, dtype=torch.int32), torch.ones(2, 1, 1, dtype=torch.bool)
    room = torch.zeros(256, dtype=torch.uint8)
    calls = {
        "write": dict(k=rows, v=rows, first=ints, table=table),
        "write_rotated": dict(k=rows, v=rows, first=ints, table=table, cos=angles, sin=angles, starts=torch.zeros(3, dtype=torch.int32), positions=ints,
                              q=rows, out=rows),
        "read": dict(first=ints, table=table, out=(rows, rows)),
        "select": dict(q=queries, lengths=ints, table=table, n_select=1, out=pages, workspace=room),
        "attend": dict(q=queries, lengths=ints, table=table, pages=pages, out=queries, workspace=room),
    }
    calls["masked"] = calls["attend"] | dict(tree=tree)
    for name, given in calls.items():
        method = getattr(cache, "attend" if name == "masked" else name)
        wrapped = lambda at: {k: (tuple(On(t, at) for t in v) if isinstance(v, tuple) else On(v, at) if isinstance(v, torch.Tensor) else v)
                              for k, v in given.items()}
        before = len(cache.calls)
        method(**wrapped(1))
        assert len(cache.calls) == before + 1
        for which in given:
            if not isinstance(given[which], int):
                with pytest.raises(AssertionError):
                    method(**(wrapped(1) | {which: wrapped(0)[which]}))
                with pytest.raises(AssertionError):
                    method(**(wrapped(1) | {which: given[which]}))
        assert len(cache.calls) == before + 1


def test_calls_with_another_current_device_are_refused(lpq, cache, monkeypatch):
    ints = On(torch.zeros(2, dtype=torch.int32), 1)
    out = tuple(On(torch.zeros(2, 1, 4), 1) for _ in range(2))
    table = On(torch.zeros(2, 1, dtype=torch.int32), 1)
    cache.read(ints, table, out=out)
    monkeypatch.setattr(lpq, "_current_device", lambda: 0)
    with pytest.raises(AssertionError, match="current"):
        cache.read(ints, table, out=out)
    assert len(cache.calls) == 1


def test_a_workspace_of_another_device(lpq):
    given = SimpleNamespace(is_cuda=True, is_contiguous=lambda: True, device=torch.device("cuda", 1), data_ptr=lambda: 0, numel=lambda: 512, element_size=lambda: 1)
    with pytest.raises(AssertionError):
        lpq.KVCache._workspace(given, 256, torch.device("cuda", 0))
    assert lpq.KVCache._workspace(given, 256, torch.device("cuda", 1))[1:] == (0, 512)
