"""The paged cache as a serving program uses it: a pruned prefill whose kept K
and V go into pages, chunks and decode steps over them, requests that end and
others that take their pages; and a captured decode step replayed."""
import numpy as np
import pytest
import torch

from gpu_util import need_gpu, say
from oracle import pages as P
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


def _attention(k, v, q, seen, scale):
    """One row over the first `seen` tokens, float64: out [Hq, d], lse [Hq]."""
    G = q.shape[0] // k.shape[1]
    kk, vv = (t[:seen].double().repeat_interleave(G, 1) for t in (k, v))
    z = (kk * q.double()[None]).sum(-1) * scale                       # [seen, Hq]
    return (torch.softmax(z, 0)[:, :, None] * vv).sum(0), torch.logsumexp(z, 0)


def _check_rows(got, lse, k, v, q, rows_seen, scale):
    # bf16: p and the result are rounded (2^-8 each, of sum p |v| and of the result); v is below 5
    for r, seen in enumerate(rows_seen):
        o, x = _attention(k, v, q[r], seen, scale)
        bound = 2.0 ** -8 * (o.abs() + 5.0) + 1e-4
        assert ((got[r].double() - o).abs() <= bound).all() and ((lse[:, r].double() - x).abs() < 1e-4).all()


@pytest.mark.parametrize("page", [16, 64])
def test_pruned_prefill_then_decode(page):
    Hq, Hkv, d, hidden, scale = 8, 2, 64, 256, 0.125
    lay = build_layout([[90, 140, 60], [75], [33, 200]], 3, 20, 40)
    dl = A.DeviceLayout(lay)
    gen = torch.Generator(device="cuda").manual_seed(page)
    rnd = lambda *s: torch.randn(*s, generator=gen, device="cuda").clamp(-5, 5).to(torch.bfloat16)  # noqa: E731
    prior, cur = rnd(dl.N_tok, hidden), rnd(dl.N_tok, hidden)
    qkv = rnd(dl.N_tok, Hq + 2 * Hkv, d)
    k, v = qkv[:, Hq:Hq + Hkv], qkv[:, Hq + Hkv:]
    cache = PagedCache(dl.B, n_pages=40, max_pages=20, Hkv=Hkv, d=d, page_size=page, layers=2)
    say(f"[paged cache] pruned prefill and decode, page {page}")
    # the step without a cache gives the same selection
    plain = ProgressivePruner(dl, prior)
    h0, _, keep0, *_ = plain.step(cur)
    pruner = ProgressivePruner(dl, prior)
    status = torch.zeros(dl.B, dtype=torch.int32, device="cuda")
    h, _, keep, *_ = pruner.step(cur, status=status, cache=cache, k=k, v=v, layer=1)
    assert torch.equal(h, h0) and torch.equal(keep, keep0) and not status.any()
    cu = pruner.dl.host["cu_seqlens"]
    lens = np.diff(cu)
    assert cache.seq_len.tolist() == lens.tolist()
    assert int(cache.free_count) == 40 - sum(-(-int(n) // page) for n in lens)
    kept = [keep[cu[b]:cu[b + 1]].long() for b in range(dl.B)]
    ks, vs = [k[i].clone() for i in kept], [v[i].clone() for i in kept]
    # a chunk of one, three and no new tokens, then single tokens
    for step, new in enumerate(([1, 3, 0], [1, 1, 1], [1, 1, 1], [2, 0, 17])):
        cu_q = ints(np.concatenate(([0], np.cumsum(new))))
        rows = rnd(sum(new) + 2, Hq + 2 * Hkv, d)                       # (two rows of padding)
        q, kn, vn = rows[:, :Hq], rows[:, Hq:Hq + Hkv], rows[:, Hq + Hkv:]
        slots = cache.reserve(cu_q, sum(new) + 2)
        assert slots.tolist()[-2:] == [-1, -1] and len(set(slots.tolist())) == sum(new) + 1
        cache.store(1, kn, vn, slots)
        out, lse = cache.attend(1, q, cu_q, scale)
        at = 0
        for b, n in enumerate(new):
            ks[b], vs[b] = torch.cat([ks[b], kn[at:at + n]]), torch.cat([vs[b], vn[at:at + n]])
            L = len(ks[b])
            _check_rows(out[at:at + n], lse[:, at:at + n], ks[b], vs[b], q[at:at + n],
                        range(L - n + 1, L + 1), scale)
            at += n
    # request 0 ends, request 2 takes back five tokens; a new request takes the pages
    before = int(cache.free_count)
    cache.trim(ints([0, 1 << 20, len(ks[2]) - 5]))
    assert cache.seq_len.tolist() == [0, len(ks[1]), len(ks[2]) - 5]
    assert int(cache.free_count) > before
    held = [int(x) for b in (1, 2) for x in cache.block_table[b, : -(-int(cache.seq_len[b]) // page)]]
    free = cache.free_pages[: int(cache.free_count)].tolist()
    assert sorted(held + free) == list(range(40))                     # every page once
    rows = rnd(70, Hq + 2 * Hkv, d)
    cu_q = ints([0, 70, 70, 70])
    slots = cache.reserve(cu_q, 70)
    cache.store(1, rows[:, Hq:Hq + Hkv], rows[:, Hq + Hkv:], slots)
    out, lse = cache.attend(1, rows[:, :Hq], cu_q, scale)
    _check_rows(out[::23], lse[:, ::23], rows[:, Hq:Hq + Hkv], rows[:, Hq + Hkv:], rows[::23, :Hq], [1, 24, 47, 70], scale)


def test_attention_lse_replaces_the_first_score_pass():
    # the row LSE that avtp_score takes, from the layer's own attention over its pages
    Hq, Hkv, d = 8, 2, 128
    lay = build_layout([[100, 260], [300]], 4, 30, 30)
    dl = A.DeviceLayout(lay)
    gen = torch.Generator(device="cuda").manual_seed(3)
    q, k, v = (torch.randn(dl.N_tok, h, d, generator=gen, device="cuda").to(torch.bfloat16) for h in (Hq, Hkv, Hkv))
    cache = PagedCache(dl.B, n_pages=64, max_pages=40, Hkv=Hkv, d=d, page_size=16)
    cu = dl.device_array("cu_seqlens")
    cache.store(0, k, v, cache.reserve(cu, dl.N_tok))
    _, lse = cache.attend(0, q, cu, d ** -0.5)
    text = dl.device_array("text_pos").long()
    q_text = q[text].contiguous()
    say("[paged cache] scores from the attention's LSE")
    s0, i0 = A.score_attn(dl, q_text, k, d ** -0.5)
    s1, i1 = A.score_attn(dl, q_text, k, d ** -0.5, row_lse=lse[:, text].contiguous())
    vis = torch.isfinite(s0)
    # (an LSE error e scales a row's probabilities by exp(e))
    assert torch.equal(vis, torch.isfinite(s1)) and ((s1 - s0).abs()[vis] <= 2e-5 * s0[vis]).all()
    assert torch.allclose(i0, i1, rtol=2e-5, atol=0)


def test_shortage_is_flagged_and_changes_nothing():
    cache = PagedCache(3, n_pages=4, max_pages=4, Hkv=1, d=64, page_size=16)
    cache.reserve(ints([0, 16, 32, 33]), 33)
    state = [t.clone() for t in (cache.seq_len, cache.free_count, cache.block_table)]
    assert state[0].tolist() == [16, 16, 1] and int(state[1]) == 1
    status = torch.zeros(3, dtype=torch.int32, device="cuda")
    slots = cache.reserve(ints([0, 0, 17, 18]), 18, status=status)      # request 1 needs two pages of one
    assert slots.tolist() == [-1] * 17 + [int(state[2][2, 0]) * 16 + 1]
    assert status.tolist() == [0, A.FLAG_NO_PAGES, 0] and cache.seq_len.tolist() == [16, 16, 2]
    assert int(cache.free_count) == 1 and torch.equal(cache.block_table, state[2])


def test_a_pruning_step_refuses_before_it_reserves_and_its_slots_serve_the_next_layer():
    dl = A.DeviceLayout(build_layout([[40, 20], [30]], 3, 12, 50))
    gen = torch.Generator(device="cuda").manual_seed(2)
    rnd = lambda *s: torch.randn(*s, generator=gen, device="cuda").to(torch.bfloat16)  # noqa: E731
    cur, k, v = rnd(dl.N_tok, 64), rnd(dl.N_tok, 2, 64), rnd(dl.N_tok, 2, 64)
    pruner = ProgressivePruner(dl, rnd(dl.N_tok, 64))
    cache = PagedCache(dl.B, n_pages=20, max_pages=10, Hkv=2, d=64, page_size=16, layers=2)
    with pytest.raises(ValueError, match="reserved"):
        cache.store(0, k, v)
    for bad in (dict(k=k), dict(k=k, v=v[:-1]), dict(k=k.float(), v=v), dict(k=k[:, :1], v=v)):
        with pytest.raises(ValueError, match="needed"):
            pruner.step(cur, cache=cache, **bad)
    with pytest.raises(ValueError, match="sequences"):
        pruner.step(cur, cache=PagedCache(5, n_pages=20, max_pages=10, Hkv=2, d=64, page_size=16), k=k, v=v)
    assert pruner.dl is dl and not cache.seq_len.any() and cache.slots is None
    h, _, keep, *_ = pruner.step(cur, cache=cache, k=k, v=v)
    k1, v1 = rnd(h.shape[0], 2, 64), rnd(h.shape[0], 2, 64)
    cache.store(1, k1, v1)
    s = cache.slots.long()
    for layer, (a, b) in enumerate(((k[keep.long()], v[keep.long()]), (k1, v1))):
        P = cache.layers[layer]
        assert torch.equal(P.k[s // 16, :, s % 16], a) and torch.equal(P.v[s // 16, :, s % 16], b)


def test_captured_decode_step():
    # reserve, store, attend, captured once and replayed while the cache grows past page borders
    Hq, Hkv, d, B, page, scale = 28, 4, 128, 5, 16, 128 ** -0.5
    gen = torch.Generator(device="cuda").manual_seed(9)
    rnd = lambda *s: torch.randn(*s, generator=gen, device="cuda").clamp(-5, 5).to(torch.bfloat16)  # noqa: E731

    def build():
        cache = PagedCache(B, n_pages=60, max_pages=12, Hkv=Hkv, d=d, page_size=page)
        first = [40, 15, 100, 16, 3]
        cu = ints(np.concatenate(([0], np.cumsum(first))))
        g = torch.Generator(device="cuda").manual_seed(1)
        kv = torch.randn(sum(first), 2 * Hkv, d, generator=g, device="cuda").to(torch.bfloat16)
        cache.store(0, kv[:, :Hkv], kv[:, Hkv:], cache.reserve(cu, sum(first)))
        return cache

    cu_q = ints(range(B + 1))
    rows, out = rnd(B, Hq + 2 * Hkv, d), rnd(B, Hq, d)
    lse = torch.empty(Hq, B, device="cuda")
    slots = torch.empty(B, dtype=torch.int32, device="cuda")

    def step(cache):
        cache.reserve(cu_q, B, slot_map=slots)
        cache.store(0, rows[:, Hq:Hq + Hkv], rows[:, Hq + Hkv:], slots)
        cache.attend(0, rows[:, :Hq], cu_q, scale, out=out, lse=lse, ws=ws)

    captured, eager = build(), build()
    ws = A.alloc_workspace(A.page_attention_workspace_bytes(captured.layers[0], Hq, B, B, 12 * page))
    stream = torch.cuda.Stream()
    with torch.cuda.stream(stream):
        step(build())                                                # (nothing of a step is built later)
        stream.synchronize()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=stream):
            step(captured)
    say("[paged cache] captured decode step, 20 replays")
    for r in range(20):
        rows.copy_(rnd(B, Hq + 2 * Hkv, d))
        torch.cuda.synchronize()
        g.replay()
        torch.cuda.synchronize()
        got = [t.clone() for t in (out, lse, slots, captured.seq_len, captured.free_count, captured.block_table)]
        out.zero_(), lse.zero_()
        step(eager)
        torch.cuda.synchronize()
        ref = (out, lse, slots, eager.seq_len, eager.free_count, eager.block_table)
        assert all(torch.equal(a, b) for a, b in zip(got, ref)), r
    assert captured.seq_len.tolist() == [60, 35, 120, 36, 23]
    t, s, n, c, f = P.page_tables(page, [0, 60, 95, 215, 251, 274], [0] * B, list(range(59, -1, -1)), 60,
                                  np.full((B, 12), -1), 274)
    assert int(captured.free_count) == c and not f.any()
