"""Steps on the paged cache that go wrong: refused rows, requests without pages."""
import numpy as np
import pytest
import torch

from gpu_util import need_gpu, say
from paper_2608_26806_amd import avtp as A
from paper_2608_26806_amd.paged import PagedCache
from paper_2608_26806_amd.progressive import ProgressivePruner
from paper_2608_26806_amd.workloads import build_layout

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    need_gpu()
    A.lib()


def ints(x):
    return torch.tensor(np.asarray(x, dtype=np.int32), device="cuda")


def _normal(seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    return lambda *s: torch.randn(*s, generator=gen, device="cuda").to(torch.bfloat16)


def _state(cache):
    """Lengths, tables' pages in use and free pages (the stack's order aside)."""
    lens = cache.seq_len.tolist()
    held = [cache.block_table[b, :-(-n // cache.page_size)].tolist() for b, n in enumerate(lens)]
    return lens, held, sorted(cache.free_pages[:int(cache.free_count)].tolist())


def test_a_pruning_step_that_refuses_its_rows_leaves_the_cache_as_it_was():
    dl = A.DeviceLayout(build_layout([[40, 20], [30]], 3, 12, 50))
    rnd = _normal(4)
    cur, k = rnd(dl.N_tok, 64), rnd(dl.N_tok, 2, 64)
    pruner = ProgressivePruner(dl, rnd(dl.N_tok, 64))
    cache = PagedCache(dl.B, n_pages=20, max_pages=10, Hkv=2, d=64, page_size=16)
    cache.reserve(ints([0, 5, 22]), 22)
    before = _state(cache)
    say("[paged steps] refused rows")
    for bad, match in ((rnd(2, dl.N_tok, 64).transpose(0, 1), "contiguous"),
                       (rnd(dl.N_tok, 132)[:, :128].unflatten(1, (2, 64)), "aligned"), (k.cpu(), "GPU")):
        for kv in (dict(k=bad, v=k), dict(k=k, v=bad)):
            with pytest.raises(ValueError, match=match):
                pruner.step(cur, cache=cache, **kv)
            assert _state(cache) == before and pruner.dl is dl
    h, *_ = pruner.step(cur, cache=cache, k=k, v=k)
    assert sum(_state(cache)[0]) == 22 + h.shape[0]


def _short_of_pages(seed):
    """A pruning step of two sequences, 36 and 19 kept tokens, into a cache of
    six pages of 16 of which sequence 1 holds three: sequence 0 takes the rest and 1 has none."""
    dl = A.DeviceLayout(build_layout([[40, 20], [12]], 3, 12, 30))
    rnd = _normal(seed)
    cur, prior, k, v = rnd(dl.N_tok, 64), rnd(dl.N_tok, 64), rnd(dl.N_tok, 2, 64), rnd(dl.N_tok, 2, 64)
    cache = PagedCache(dl.B, n_pages=6, max_pages=6, Hkv=2, d=64, page_size=16)
    cache.reserve(ints([0, 0, 48]), 48)
    return dl, cur, prior, k, v, cache


def test_a_pruning_step_without_pages_raises_and_takes_its_places_back():
    dl, cur, prior, k, v, cache = _short_of_pages(6)
    pruner = ProgressivePruner(dl, prior)
    before, slots = _state(cache), cache.slots
    say("[paged steps] a shortage")
    for _ in range(2):
        with pytest.raises(RuntimeError, match=r"no pages .* sequences \[1\]"):
            pruner.step(cur, cache=cache, k=k, v=v)
        assert _state(cache) == before and cache.slots is slots and pruner.dl is dl and pruner.h_prior is prior
    cache.trim(ints([0, 16]))                                       # sequence 1 hands pages back
    h, _, keep, *_ = pruner.step(cur, cache=cache, k=k, v=v)
    n = pruner.dl.host["cu_seqlens"]
    assert cache.seq_len.tolist() == [int(n[1]), 16 + int(n[2] - n[1])] and h.shape[0] == int(n[2])
    s, P = cache.slots.long(), cache.layers[0]
    assert (s >= 0).all()
    assert torch.equal(P.k[s // 16, :, s % 16], k[keep.long()]) and torch.equal(P.v[s // 16, :, s % 16], v[keep.long()])


def test_a_pruning_step_with_a_status_flags_the_shortage():
    dl, cur, prior, k, v, cache = _short_of_pages(7)
    pruner = ProgressivePruner(dl, prior)
    status = torch.zeros(2, dtype=torch.int32, device="cuda")
    say("[paged steps] a shortage, flagged")
    _, _, keep, *_ = pruner.step(cur, cache=cache, k=k, v=v, status=status)
    n0 = int(pruner.dl.host["cu_seqlens"][1])
    assert status.tolist() == [0, A.FLAG_NO_PAGES] and cache.seq_len.tolist() == [n0, 48]
    s, P = cache.slots.long(), cache.layers[0]
    assert (s[:n0] >= 0).all() and (s[n0:] == -1).all()
    assert torch.equal(P.k[s[:n0] // 16, :, s[:n0] % 16], k[keep[:n0].long()])


def test_a_pruning_step_that_fails_behind_the_reservation_takes_its_places_back():
    dl, cur, prior, k, v, cache = _short_of_pages(8)
    cache.trim(ints([0, 0]))
    pruner = ProgressivePruner(dl, prior)
    before = _state(cache)
    say("[paged steps] a keep schedule that fails")
    with pytest.raises(TypeError):
        pruner.step(cur, cache=cache, k=k, v=v, keep_pct_next=None)
    assert _state(cache) == before and pruner.dl is dl
