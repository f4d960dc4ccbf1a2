"""Calls of the decoder layer on codes that would drop a gradient refuse the input that asks for one, before they look at its memory: no device needed."""
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


@pytest.mark.parametrize("which", ["k", "v", "q", "cos", "sin"])
def test_rotated_rows_and_angles(lpq, which):
    cache = object.__new__(lpq.KVCache)
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
