"""What KVCache refuses before it passes memory to a kernel: none of it needs a device."""
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


def test_storage_in_host_memory_is_refused(lpq):
    quantizer = SimpleNamespace(d=128, _h=None)
    with pytest.raises(AssertionError):
        lpq.KVCache(quantizer, quantizer, heads=2, page=16, pages=2, device="cpu")


@pytest.mark.parametrize("given", [torch.empty(4096, dtype=torch.uint8), torch.empty(64, dtype=torch.float32)])
def test_a_workspace_in_host_memory_is_refused(lpq, given):
    with pytest.raises(AssertionError):
        lpq.KVCache._workspace(given, 256, torch.device("cuda"))


def test_a_workspace_that_is_not_one_run_of_memory_is_refused(lpq):
    """A view of one byte with a stride of 0 says that it has as many bytes as one likes."""
    meta = SimpleNamespace(is_cuda=True)
    for t in (torch.empty(1, dtype=torch.uint8).expand(1 << 20), torch.empty(4096, dtype=torch.uint8)[::2]):
        view = SimpleNamespace(**vars(meta), is_contiguous=t.is_contiguous, data_ptr=t.data_ptr, numel=t.numel, element_size=t.element_size)
        with pytest.raises(AssertionError):
            lpq.KVCache._workspace(view, 256, torch.device("cuda"))
