"""The host side of the paged cache's callers, on the CPU: what a pruning step
checks before it reserves."""
import ctypes
from types import SimpleNamespace

import pytest
import torch

from paper_2608_26806_amd import avtp as A
from paper_2608_26806_amd.progressive import ProgressivePruner
from paper_2608_26806_amd.workloads import build_layout


class Cache:
    """Stands for a PagedCache of two sequences; reserving is an error here."""

    def __init__(self):
        self.layers = [SimpleNamespace(Hkv=2, d=64, dtype=torch.bfloat16)]
        self.seq_len = torch.zeros(2, dtype=torch.int32)

    def reserve(self, *args, **kw):
        raise AssertionError("reserved before the rows were checked")

    def store(self, *args, **kw):
        pass


def _layouts_of_rows(n):
    """Rows [n, 2, 64] that no store takes, and the refusal."""
    flat = torch.zeros(n * 136 + 8, dtype=torch.bfloat16)
    return {
        "head-major": (torch.zeros(2, n, 64, dtype=torch.bfloat16).transpose(0, 1), "contiguous"),
        "value-major": (torch.zeros(n, 64, 2, dtype=torch.bfloat16).transpose(1, 2), "contiguous"),
        "one row for all": (torch.zeros(1, 2, 64, dtype=torch.bfloat16).expand(n, 2, 64), "overlap"),
        "a stride of 132": (flat[:n * 132].view(n, 132)[:, :128].unflatten(1, (2, 64)), "aligned"),
        "four values off": (flat[4:4 + n * 136].view(n, 136)[:, :128].unflatten(1, (2, 64)), "aligned"),
    }


@pytest.mark.parametrize("which", sorted(_layouts_of_rows(3)))
@pytest.mark.parametrize("name", ["k", "v"])
def test_a_pruning_step_checks_the_layout_of_k_and_v_before_it_reserves(monkeypatch, which, name):
    dl = A.DeviceLayout(build_layout([[9, 7], [5]], 2, 4, 50), host_only=True)
    monkeypatch.setattr(A, "_page_arg", lambda *args: 0)          # (the rows are in host memory)
    monkeypatch.setattr(A, "score_variation", lambda *args, **kw: (None, None))
    monkeypatch.setattr(A, "budget_select_compact", lambda *args, **kw: (None, None, None))
    good = torch.zeros(dl.N_tok, 2, 64, dtype=torch.bfloat16)
    bad, match = _layouts_of_rows(dl.N_tok)[which]
    kv = {"k": good, "v": good, name: bad}
    h = torch.zeros(dl.N_tok, 8)
    pruner = ProgressivePruner(dl, h)
    with pytest.raises(ValueError, match=f"{name}: .*{match}"):
        pruner.step(h, cache=Cache(), **kv)
    assert pruner.dl is dl


def test_a_pruning_step_refuses_rows_in_host_memory_before_it_reserves(monkeypatch):
    dl = A.DeviceLayout(build_layout([[9, 7], [5]], 2, 4, 50), host_only=True)
    monkeypatch.setattr(A, "score_variation", lambda *args, **kw: (None, None))
    monkeypatch.setattr(A, "budget_select_compact", lambda *args, **kw: (None, None, None))
    h, k = torch.zeros(dl.N_tok, 8), torch.zeros(dl.N_tok, 2, 64, dtype=torch.bfloat16)
    with pytest.raises(ValueError, match="k: a GPU tensor"):
        ProgressivePruner(dl, h).step(h, cache=Cache(), k=k, v=k)


BUF = torch.zeros(4096, dtype=torch.uint8)          # (never dereferenced: the calls are refused)
P, Q, R = (ctypes.c_void_p(BUF.data_ptr() + 64 * i) for i in range(3))
RESERVE = dict(stream=None, B=3, page_size=16, cu_new=P, seq_len=P, free_pages=P, n_pages=10, free_count=P,
               block_table=P, max_pages=4, slot_map=P, n_new=5, seq_len_out=Q, free_count_out=Q, kv_len=R,
               status=None)


@pytest.mark.parametrize("patch, rc", [
    (dict(kv_len=None), A.ERR_INVALID_ARG), (dict(kv_len=P), A.ERR_INVALID_ARG),
    (dict(kv_len=Q), A.ERR_INVALID_ARG),
    (dict(seq_len_out=P), A.ERR_INVALID_ARG), (dict(free_count_out=None), A.ERR_INVALID_ARG),
    (dict(cu_new=None), A.ERR_INVALID_ARG), (dict(B=0), A.ERR_INVALID_ARG), (dict(B=1 << 17), A.ERR_UNSUPPORTED),
    (dict(page_size=24), A.ERR_UNSUPPORTED), (dict(n_new=-1), A.ERR_INVALID_ARG)])
def test_reserve_refusals(patch, rc):
    assert A.lib().avtp_page_reserve(*{**RESERVE, **patch}.values()) == rc


def test_pages_on_another_device_than_the_current_one_are_refused(monkeypatch):
    # stand-ins for tensors on the second of two devices; the launch would be on the first
    def tensor(device):
        return SimpleNamespace(is_cuda=True, device=torch.device("cuda", device), dtype=torch.bfloat16, shape=(4, 2, 16, 64),
                               is_contiguous=lambda: True, numel=lambda: 8192, data_ptr=lambda: P.value, dim=lambda: 4)

    current = [1]
    monkeypatch.setattr(torch.cuda, "current_device", lambda: current[0])
    pages = A.Pages(tensor(1), tensor(1))
    assert A.page_attention_workspace_bytes(pages, 4, 1, 1, 5000) > 0
    current[0] = 0
    monkeypatch.setattr(A, "_page_rows", lambda t, name, heads, pages: (P, 128))    # (rows on device 0)
    rows, slots = SimpleNamespace(shape=(3, 2, 64)), tensor(0)
    slots.dtype, slots.numel = torch.int32, lambda: 3
    with pytest.raises(ValueError, match="pages: on cuda:1"):
        A.prepare_page_store(pages, rows, rows, slots, stream=ctypes.c_void_p(0))
    with pytest.raises(ValueError, match="pages: on cuda:1"):
        A.page_attention_workspace_bytes(pages, 4, 1, 1, 5000)
