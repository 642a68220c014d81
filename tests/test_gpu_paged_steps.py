"""Steps on the paged cache that go wrong: refused rows, requests without pages."""
import numpy as np
import pytest
import torch

from gpu_util import need_gpu, say
from paper_2608_26806_amd import avtp as A
from paper_2608_26806_amd.paged import PagedCache
from paper_2608_26806_amd.progressive import ProgressivePruner
from paper_2608_26806_amd.workloads import build_layout
from test_gpu_paged_cache import _check_rows

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


@pytest.mark.parametrize("B, high, free", [(1, 40, 9), (5, 300, 20), (64, 1, 30), (1500, 60, 2000), (3000, 1, 40)])
def test_lengths_for_attention(B, high, free):
    # the outputs of the call without them; 0 for the requests without a place (rows too short, pages, slots), as they
    # were for sequences without new tokens
    rng = np.random.default_rng(B)
    lens, new = rng.integers(0, 90, B), rng.integers(0, high + 1, B)
    cu = np.concatenate(([0], np.cumsum(new)))
    table = rng.integers(0, free, (B, 8))
    say(f"[paged steps] {B} requests, {free} free pages")
    got = []
    for kv in (None, ints([-7] * (B + 1))):
        t, status, n_new = ints(table), ints([0] * B), max(0, int(cu[-1]) - 3)
        slots, out, left = ints([5] * n_new), ints([5] * B), ints([5])
        A.prepare_page_tables(16, ints(cu), ints(lens), ints(range(free)), ints([free]), t, slots, out, left, status,
                              kv_len=kv)()
        got.append([x.tolist() for x in (t, status, slots, out, left)])
    assert got[0] == got[1]
    flags, out = got[0][1], got[0][3]
    assert kv.tolist() == [(0 if f & A.FLAG_NO_PAGES else n) if x else -7 for f, n, x in zip(flags, out, new)] + [-7]
    assert B == 1 or any(flags)


def _rows(rnd, n, Hq=4, Hkv=2, d=64):
    x = rnd(n, Hq + 2 * Hkv, d).clamp(-5, 5)
    return x[:, :Hq], x[:, Hq:Hq + Hkv], x[:, Hq + Hkv:]


def test_queries_of_a_request_without_a_place_see_nothing():
    rnd, scale = _normal(11), 0.125
    cache = PagedCache(3, n_pages=4, max_pages=4, Hkv=2, d=64, page_size=16)
    say("[paged steps] attention after a shortage")
    _, k0, v0 = _rows(rnd, 33)
    cache.reserve(ints([0, 16, 32, 33]), 33)                        # three of four pages
    cache.store(0, k0, v0)
    q, k, v = _rows(rnd, 19)
    cu = ints([0, 1, 18, 19])
    status = torch.zeros(3, dtype=torch.int32, device="cuda")
    cache.reserve(cu, 19, status=status)                            # request 0 takes the last page
    assert status.tolist() == [0, A.FLAG_NO_PAGES, 0] and cache.seq_len.tolist() == [17, 16, 2]
    cache.store(0, k, v)
    for bound in (17, None, 1 << 20):
        out, lse = cache.attend(0, q, cu, scale, max_kv_len=bound)
        assert not out[1:18].any() and (lse[:, 1:18] == -float("inf")).all()
        _check_rows(out[:1], lse[:, :1], torch.cat([k0[:16], k[:1]]), torch.cat([v0[:16], v[:1]]), q[:1], [17], scale)
        _check_rows(out[18:], lse[:, 18:], torch.cat([k0[32:], k[18:]]), torch.cat([v0[32:], v[18:]]), q[18:], [2], scale)
    # request 0 ends; 1 still has no place for its tokens, then it gets one
    cache.trim(ints([0, 100, 100]))
    out, lse = cache.attend(0, q, cu, scale)
    assert not out[:18].any() and (lse[:, :18] == -float("inf")).all() and out[18].any()
    status.zero_()
    cache.reserve(ints([0, 0, 17, 17]), 17, status=status)
    assert not status.any() and cache.seq_len.tolist() == [0, 33, 2]
    cache.store(0, k[1:18], v[1:18])
    out, lse = cache.attend(0, q[1:], ints([0, 0, 17, 18]), scale)
    _check_rows(out[:17], lse[:, :17], torch.cat([k0[16:32], k[1:18]]), torch.cat([v0[16:32], v[1:18]]), q[1:18],
                range(17, 34), scale)
    _check_rows(out[17:], lse[:, 17:], torch.cat([k0[32:], k[18:]]), torch.cat([v0[32:], v[18:]]), q[18:], [2], scale)


def test_a_captured_step_runs_into_a_shortage_and_out_of_it():
    B, page, scale = 3, 16, 0.125
    rnd = _normal(12)
    cu, slots = ints(range(B + 1)), torch.empty(B, dtype=torch.int32, device="cuda")
    q, k, v = _rows(rnd, B)
    out, lse = torch.empty(B, 4, 64, dtype=torch.bfloat16, device="cuda"), torch.empty(4, B, device="cuda")
    cache = PagedCache(B, n_pages=4, max_pages=4, Hkv=2, d=64, page_size=page)
    _, k0, v0 = _rows(rnd, 28)
    cache.store(0, k0, v0, cache.reserve(ints([0, 13, 14, 28]), 28))
    ws = A.alloc_workspace(A.page_attention_workspace_bytes(cache.layers[0], 4, B, B, 64))

    def step():
        cache.store(0, k, v, cache.reserve(cu, B, slot_map=slots))
        cache.attend(0, q, cu, scale, max_kv_len=64, out=out, lse=lse, ws=ws)

    ks, vs = ([t[a:b].clone() for a, b in ((0, 13), (13, 14), (14, 28))] for t in (k0, v0))
    stream = torch.cuda.Stream()
    say("[paged steps] a captured step through a shortage")
    with torch.cuda.stream(stream):
        warm = PagedCache(B, n_pages=4, max_pages=4, Hkv=2, d=64, page_size=page)   # (nothing is built in the capture)
        A.page_attention(warm.layers[0], q, cu, warm.seq_len, warm.block_table, scale, 64, out, lse, ws=ws)
        warm.reserve(cu, B)
        stream.synchronize()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=stream):
            step()
    refused = 0
    for r in range(9):
        if r == 7:
            cache.trim(ints([100, 0, 100]))                         # the short request ends and starts anew
            ks[1], vs[1] = ks[1][:0], vs[1][:0]
        k.copy_(rnd(B, 2, 64).clamp(-5, 5)), v.copy_(rnd(B, 2, 64).clamp(-5, 5))
        torch.cuda.synchronize()
        g.replay()
        torch.cuda.synchronize()
        for b, s in enumerate(slots.tolist()):
            if s < 0:
                refused += 1
                assert not out[b].any() and (lse[:, b] == -float("inf")).all(), (r, b)
                continue
            ks[b], vs[b] = torch.cat([ks[b], k[b:b + 1]]), torch.cat([vs[b], v[b:b + 1]])
            _check_rows(out[b:b + 1], lse[:, b:b + 1], ks[b], vs[b], q[b:b + 1], [len(ks[b])], scale)
        assert cache.seq_len.tolist() == [len(x) for x in ks]
    assert refused == 6                                             # request 0 four times, request 1 twice


def test_a_reservation_for_others_does_not_lift_a_refusal():
    # two reservations (say prompts, then single tokens) before one attention over both
    rnd, scale = _normal(13), 0.125
    cache = PagedCache(3, n_pages=4, max_pages=4, Hkv=2, d=64, page_size=16)
    say("[paged steps] two reservations, the first with a refusal")
    _, k0, v0 = _rows(rnd, 33)
    cache.store(0, k0, v0, cache.reserve(ints([0, 16, 32, 33]), 33))
    q, k, v = _rows(rnd, 41)
    status = torch.zeros(3, dtype=torch.int32, device="cuda")
    cache.store(0, k[:40], v[:40], cache.reserve(ints([0, 0, 40, 40]), 40, status=status))
    cache.store(0, k[40:], v[40:], cache.reserve(ints([0, 0, 0, 1]), 1, status=status))
    assert status.tolist() == [0, A.FLAG_NO_PAGES, 0] and cache.seq_len.tolist() == [16, 16, 2]
    out, lse = cache.attend(0, q, ints([0, 0, 40, 41]), scale)
    assert not out[:40].any() and (lse[:, :40] == -float("inf")).all()
    _check_rows(out[40:], lse[:, 40:], torch.cat([k0[32:], k[40:]]), torch.cat([v0[32:], v[40:]]), q[40:], [2], scale)
    # the untouched sequence's cached tokens are still seen
    out, lse = cache.attend(0, q[:1], ints([0, 1, 1, 1]), scale)
    _check_rows(out, lse, k0[:16], v0[:16], q[:1], [16], scale)
