"""What cache_attn takes as a workspace, on the host: the library's call is replaced by one that
records its arguments, and the checks that ask for GPU tensors by none."""
import pytest
import torch

import paper_2603_29494_amd as va
from paper_2603_29494_amd import _lib


@pytest.fixture
def calls(monkeypatch):
    seen = []
    monkeypatch.setattr(_lib, "_bf16_cuda", lambda t, name: None)
    monkeypatch.setattr(_lib, "_cache_args", lambda cache, table, lens, B, n_new=None:
                        cache.data.device)
    monkeypatch.setattr(_lib, "_call", lambda device, what, fn, *args: seen.append(args))
    return seen


def attend(workspace):
    c = va.Cache(torch.empty(va.cache_bytes(64, 1, 64), dtype=torch.uint8), 64, 1, 64, 64, 4)
    q = torch.zeros(1, 2, 1, 64, dtype=torch.bfloat16)
    table, lens = torch.zeros(1, 64, dtype=torch.int32), torch.zeros(1, dtype=torch.int32)
    need = va.cache_attn_workspace_bytes(q, c, 64)
    assert need > 0
    ws = workspace(need)
    va.cache_attn(q, c, table, lens, workspace=ws)
    return ws, need


@pytest.mark.parametrize("make", [
    lambda need: torch.empty(1, dtype=torch.uint8).expand(need),     # one byte behind them all
    lambda need: torch.empty(2 * need, dtype=torch.uint8)[::2],
    lambda need: torch.empty(need, 2, dtype=torch.uint8).t()])
def test_a_workspace_with_gaps_or_overlaps_is_refused(calls, make):
    with pytest.raises(ValueError):
        attend(make)
    assert not calls


@pytest.mark.parametrize("dtype", [torch.uint8, torch.float32])
def test_a_contiguous_workspace_counts_in_bytes(calls, dtype):
    ws, need = attend(lambda need: torch.empty(-(-need // dtype.itemsize), dtype=dtype))
    assert calls[0][-2:] == (ws.data_ptr(), ws.numel() * dtype.itemsize)
    assert calls[0][-1] >= need
