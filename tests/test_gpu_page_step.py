"""A layer's step around the paged cache as a serving program makes it: rows
normalised, rotated and stored, questions forked off a prompt, attention over a
window, requests that end while others hold their pages; and a captured step."""
import numpy as np
import pytest
import torch

from gpu_util import need_gpu, say
from paper_2608_26806_amd import avtp as A
from paper_2608_26806_amd.paged import PagedCache
from paper_2608_26806_amd.progressive import ProgressivePruner
from paper_2608_26806_amd.rotary import Rotary
from paper_2608_26806_amd.workloads import build_layout

pytestmark = pytest.mark.gpu
Hq, Hkv, d, scale = 8, 2, 64, 0.125


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    need_gpu()
    A.lib()


def ints(x):
    return torch.tensor(np.asarray(x, dtype=np.int32), device="cuda")


class Serving:
    """A cache, and beside it every sequence's rotated K and V as plain rows."""

    def __init__(self, seed, requests, n_pages, page=16, layers=1, **kw):
        self.gen = torch.Generator(device="cuda").manual_seed(seed)
        self.cache = PagedCache(requests, n_pages, 64, Hkv, d, page, layers=layers, **kw)
        self.rotary = Rotary(d, base=1e5, planes=[i % 3 for i in range(d // 2)])
        self.wq, self.wk = (1 + 0.2 * torch.randn(d, generator=self.gen, device="cuda") for _ in range(2))
        self.page, self.layers, self.n_pages = page, layers, n_pages
        none = torch.empty(0, Hkv, d, dtype=torch.bfloat16, device="cuda")
        self.k = [[none for _ in range(requests)] for _ in range(layers)]
        self.v = [[none for _ in range(requests)] for _ in range(layers)]

    def rows(self, n):
        # clamped, so that |v| is at most 5
        return torch.randn(n, Hq + 2 * Hkv, d, generator=self.gen, device="cuda").clamp(-5, 5).bfloat16()

    def step(self, new):
        """New tokens for every sequence: stored and attended in every layer, checked."""
        cu = np.concatenate(([0], np.cumsum(new)))
        n = int(cu[-1])
        pos = torch.randint(0, 5000, (3, n), generator=self.gen, device="cuda")
        status = torch.zeros(len(new), dtype=torch.int32, device="cuda")
        self.cache.reserve(ints(cu), n, status=status)
        assert not status.any()
        for layer in range(self.layers):
            x = self.rows(n)
            q, k, v = x[:, :Hq], x[:, Hq:Hq + Hkv], x[:, Hq + Hkv:]
            qr = self.cache.store_rotary(layer, self.rotary, pos, q, k, v, self.wq, self.wk)
            want_q, kr = A.norm_rotary(self.rotary, pos, q, k, self.wq, self.wk)
            assert torch.equal(qr, want_q)
            for b in range(len(new)):
                self.k[layer][b] = torch.cat([self.k[layer][b], kr[cu[b]:cu[b + 1]]])
                self.v[layer][b] = torch.cat([self.v[layer][b], v[cu[b]:cu[b + 1]]])
            out, lse = self.cache.attend(layer, qr, ints(cu), scale, status=status)
            assert not status.any()
            for b in range(len(new)):
                self.check(layer, b, qr[cu[b]:cu[b + 1]], out[cu[b]:cu[b + 1]], lse[:, cu[b]:cu[b + 1]])

    def check(self, layer, b, q, out, lse):
        n, L = len(q), len(self.k[layer][b])
        if n == 0:
            return
        G = Hq // Hkv
        k, v = (t.double().repeat_interleave(G, 1).transpose(0, 1) for t in (self.k[layer][b], self.v[layer][b]))
        z = (q.double().transpose(0, 1)[:, :, None] * k[:, None]).sum(-1) * scale
        p, j = torch.arange(L - n, L, device="cuda")[:, None], torch.arange(L, device="cuda")
        hidden = j > p
        if self.cache.window:
            hidden = hidden | ((j <= p - self.cache.window) & (j >= self.cache.sinks))
        z = z.masked_fill(hidden, -torch.inf)
        o = (torch.softmax(z, -1)[..., None] * v[:, None]).sum(2).transpose(0, 1)
        # bf16: p and the result are rounded (2^-8 each, of sum p |v| <= 5 and of the result)
        assert ((out.double() - o).abs() <= 2.0 ** -8 * (o.abs() + 5.0) + 1e-4).all()
        assert ((lse.double() - torch.logsumexp(z, -1)).abs() < 1e-4).all()

    def cut(self, keep, flags=None):
        status = torch.zeros(len(keep), dtype=torch.int32, device="cuda")
        self.cache.trim(ints(keep), status)
        assert status.tolist() == (flags or [0] * len(keep))
        for layer in range(self.layers):
            for b, n in enumerate(keep):
                if not flags or not flags[b]:
                    self.k[layer][b], self.v[layer][b] = self.k[layer][b][:n], self.v[layer][b][:n]
        self.check_pages()

    def fork(self, parent, n=None):
        status = torch.zeros(len(parent), dtype=torch.int32, device="cuda")
        self.cache.fork(ints(parent), None if n is None else ints(n), status)
        assert not status.any()
        for layer in range(self.layers):
            for b, p in enumerate(parent):
                if p >= 0:
                    m = len(self.k[layer][p]) if n is None else n[b]
                    self.k[layer][b], self.v[layer][b] = self.k[layer][p][:m], self.v[layer][p][:m]
        self.check_pages()

    def check_pages(self):
        """Every page is held by some sequence or free, and none is both."""
        c, ps = self.cache, self.page
        held = set()
        lens = [len(k) for k in self.k[0]]
        assert c.seq_len.tolist() == lens
        for b, n in enumerate(lens):
            gone = int(c.gone[b]) // ps if c.sharing else 0
            first = -(-c.sinks // ps)
            held |= {int(c.block_table[b, j]) for j in range(-(-n // ps)) if j < first or j >= gone}
        free = c.free_pages[:int(c.free_count)].tolist()
        assert sorted(free + list(held)) == list(range(self.n_pages))


@pytest.mark.parametrize("page", [16, 32])
def test_questions_about_the_same_images(page):
    say(f"[page step] forked questions, page {page}")
    s = Serving(page, 7, 90, page, layers=2, sharing=True)
    s.step([130, 0, 0, 64, 0, 0, 0])
    s.fork([-1, 0, 0, -1, 3, 3, 0], [0, 130, 100, 0, 64, 63, 0])
    s.step([1, 20, 3, 40, 1, 0, 2])              # the prompts go on too
    for t in range(4):
        s.step([1] * 7)
    L = [len(k) for k in s.k[0]]
    s.cut([0, L[1] - 4, L[2], 0, L[4], L[5] - 1, 0])    # both prompts end, their pages stay with the questions
    s.step([50, 1, 1, 0, 1, 1, 9])               # others take the places
    s.cut([len(k) for k in s.k[0]][:2] + [97] + [len(k) for k in s.k[0]][3:])
    s.fork([-1, -1, -1, 1, -1, -1, -1])          # a question of a question
    s.step([1, 1, 1, 3, 1, 1, 1])
    s.cut([0] * 7)
    assert int(s.cache.free_count) == 90


def test_a_cut_in_a_shared_page_leaves_all_as_it_was():
    s = Serving(3, 3, 30, 16, sharing=True)
    s.step([100, 0, 0])
    s.fork([-1, 0, -1])
    s.step([2, 1, 0])
    s.cut([102, 50, 0], [0, A.FLAG_REFUSED, 0])
    s.step([1, 1, 0])
    # the documented way: the tokens to be kept to an empty row, the old one ended
    s.fork([-1, -1, 1], [0, 0, 50])
    s.cut([103, 0, 50])
    s.step([1, 0, 5])


@pytest.mark.parametrize("window, sinks, page", [(40, 4, 16), (1, 0, 16), (100, 33, 32), (7, 0, 16)])
def test_a_window_in_little_memory(window, sinks, page):
    say(f"[page step] window {window} sinks {sinks} page {page}")
    # far fewer pages than the sequences' tokens fill
    s = Serving(window, 4, 4 * (-(-(window + 60) // page) + -(-sinks // page) + 1), page, window=window, sinks=sinks)
    s.step([30, 55, 1, 0])
    s.cut([len(k) for k in s.k[0]])
    for t in range(12):
        s.step([[1, 17, 2, 1], [30, 1, 1, 40]][t % 2])
        L = [len(k) for k in s.k[0]]
        s.cut([L[0], L[1] - (t % 2), 0 if t == 6 else L[2], L[3]])
    if s.cache.gone[1] > 0:
        L = [len(k) for k in s.k[0]]
        s.cut([L[0], L[1] - 1, L[2], L[3]], [0, A.FLAG_REFUSED, 0, 0])
        s.cut([0, L[1], L[2], L[3]])
        s.fork([1, -1, -1, -1])                   # a fork behind the window: all of it
        s.step([1, 2, 1, 1])
        s.cut([len(k) for k in s.k[0]])
    s.cut([0] * 4)
    assert int(s.cache.free_count) == s.n_pages


def test_behind_a_pruning_layer():
    # the pruning layer's kept rows, rotated beforehand and scored, then the next layer's
    lay = build_layout([[90, 140], [75], [60]], 3, 20, 40)
    dl = A.DeviceLayout(lay)
    s = Serving(5, 6, 90, 16, layers=2, sharing=True)
    x, x1 = s.rows(dl.N_tok), s.rows(dl.N_tok)
    pos = torch.arange(dl.N_tok, device="cuda")[None].repeat(3, 1)
    _, k = A.norm_rotary(s.rotary, pos, None, x[:, Hq:Hq + Hkv], None, s.wk)
    h = torch.randn(dl.N_tok, 64, generator=s.gen, device="cuda").bfloat16()
    h2 = torch.randn(dl.N_tok, 64, generator=s.gen, device="cuda").bfloat16()
    inner = PagedCache(dl.B, 90, 64, Hkv, d, 16, layers=2, sharing=True)
    status = torch.zeros(dl.B, dtype=torch.int32, device="cuda")
    pruner = ProgressivePruner(dl, h)
    _, (pos_kept,), keep, *_ = pruner.step(h2, [(pos, 1)], status=status, cache=inner, k=k, v=x[:, Hq + Hkv:], layer=0)
    n = pruner.dl.N_tok
    rows = x1[:n]
    q = inner.store_rotary(1, s.rotary, pos_kept, rows[:, :Hq], rows[:, Hq:Hq + Hkv], rows[:, Hq + Hkv:], s.wq, s.wk)
    cu = pruner.dl.host["cu_seqlens"]
    out, lse = inner.attend(1, q, ints(cu), scale)
    want_q, kr = A.norm_rotary(s.rotary, pos[:, keep.long()], rows[:, :Hq], rows[:, Hq:Hq + Hkv], s.wq, s.wk)
    assert torch.equal(q, want_q) and not status.any()
    for b in range(dl.B):
        r = slice(int(cu[b]), int(cu[b + 1]))
        s.k[1][b], s.v[1][b] = kr[r], rows[r, Hq + Hkv:]
        s.check(1, b, q[r], out[r], lse[:, r])
        kept = keep[r].long()
        at = torch.arange(len(kept), device="cuda")
        page = inner.block_table[b, at // 16].long()
        assert torch.equal(inner.layers[0].k[page, :, at % 16], k[kept])


def test_captured_step():
    B, window, sinks = 5, 50, 4
    say("[page step] captured step behind a window")
    caches = [PagedCache(B, 60, 64, Hkv, d, 16, window=window, sinks=sinks) for _ in range(2)]
    gen = torch.Generator(device="cuda").manual_seed(9)
    rotary = Rotary(d, base=1e4)
    wq = 1 + 0.2 * torch.randn(d, generator=gen, device="cuda")
    rows = torch.randn(B, Hq + 2 * Hkv, d, generator=gen, device="cuda").bfloat16()
    pos = torch.randint(0, 1000, (1, B), generator=gen, device="cuda")
    cu = ints(range(B + 1))
    first = [5, 40, 90, 16, 33]
    for c in caches:
        c.reserve(ints(np.concatenate(([0], np.cumsum(first)))), sum(first))
        kv = torch.randn(sum(first), 2 * Hkv, d, generator=torch.Generator(device="cuda").manual_seed(1),
                         device="cuda").bfloat16()
        c.store(0, kv[:, :Hkv], kv[:, Hkv:])
        c.trim(c.seq_len.clone())
    slots = torch.empty(B, dtype=torch.int32, device="cuda")
    out, lse = torch.empty(B, Hq, d, dtype=torch.bfloat16, device="cuda"), torch.empty(Hq, B, device="cuda")
    keep = caches[0].seq_len.clone()
    ws = A.alloc_workspace(A.page_attention_workspace_bytes(caches[0].layers[0], Hq, B, B, 200, window, sinks))

    def step(c, out, lse, ws):
        c.reserve(cu, B, slot_map=slots)
        q = c.store_rotary(0, rotary, pos, rows[:, :Hq], rows[:, Hq:Hq + Hkv], rows[:, Hq + Hkv:], wq, None)
        c.attend(0, q, cu, scale, 200, out=out, lse=lse, ws=ws)
        keep.copy_(c.seq_len)
        c.trim(keep)

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        for c in caches:
            step(c, out, lse, ws)
        side.synchronize()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=side):
            step(caches[0], out, lse, ws)
    torch.cuda.current_stream().wait_stream(side)
    for i in range(70):                           # pages leave the window, others are taken
        rows.copy_(torch.randn(rows.shape, generator=gen, device="cuda").bfloat16())
        pos.add_(1)
        g.replay()
        want, x = torch.empty_like(out), torch.empty_like(lse)
        step(caches[1], want, x, ws)
        torch.cuda.synchronize()
        assert torch.equal(out, want) and torch.equal(lse, x)
        for name in ("seq_len", "free_count", "gone", "block_table", "free_pages"):
            a, b = getattr(caches[0], name), getattr(caches[1], name)
            if name == "free_pages":
                a, b = a[:int(caches[0].free_count)], b[:int(caches[0].free_count)]
            assert torch.equal(a, b), name
    assert int(caches[0].seq_len[0]) == 5 + 71 and int(caches[0].free_count) > 20


def test_captured_forks():
    # a graph that ends the questions and forks new ones off the same prompts
    B, page = 6, 16
    c = PagedCache(B, 60, 20, Hkv, d, page, layers=2, sharing=True)
    gen = torch.Generator(device="cuda").manual_seed(4)
    first = [75, 0, 0, 40, 0, 0]
    rows = torch.randn(2, sum(first), 2 * Hkv, d, generator=gen, device="cuda").bfloat16()
    c.reserve(ints(np.concatenate(([0], np.cumsum(first)))), sum(first))
    for layer in range(2):
        c.store(layer, rows[layer, :, :Hkv], rows[layer, :, Hkv:])
    parent, keep = ints([-1, 0, 0, -1, 3, 0]), ints([75, 0, 0, 40, 0, 0])
    status = torch.zeros(B, dtype=torch.int32, device="cuda")

    def step():
        c.trim(keep, status)
        c.fork(parent, None, status)

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
        side.synchronize()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=side):
            step()
    torch.cuda.current_stream().wait_stream(side)
    for i, p in enumerate(([-1, 0, 0, -1, 3, 0], [-1, 3, 3, -1, 0, -1], [-1, 0, -1, -1, 0, 3], [-1, -1, 3, -1, 3, 3])):
        parent.copy_(ints(p))
        g.replay()
        torch.cuda.synchronize()
        lens = [first[x] if x >= 0 else first[b] for b, x in enumerate(p)]
        assert c.seq_len.tolist() == lens and not status.any()
        held = {int(c.block_table[b, j]) for b in range(B) for j in range(-(-lens[b] // page))}
        assert sorted(list(held) + c.free_pages[:int(c.free_count)].tolist()) == list(range(60))
        for b, x in enumerate(p):
            src = x if x >= 0 else b
            at = torch.arange(lens[b], device="cuda")
            pg = c.block_table[b, at // page].long()
            r0 = 0 if src == 0 else 75
            for layer in range(2):
                got = c.layers[layer].k[pg, :, at % page]
                assert torch.equal(got, rows[layer, r0:r0 + lens[b], :Hkv]), (i, b, layer)


@pytest.mark.parametrize("seed, window, sinks", [(1, None, 0), (2, None, 0), (3, 45, 4), (4, 1, 0), (5, 130, 40), (6, 30, 17)])
def test_random_serving(seed, window, sinks):
    # requests that come, grow, fork, are cut, refused and end, every step checked
    rng = np.random.default_rng(seed)
    B, page = 9, int(rng.choice([16, 32]))
    s = Serving(seed, B, 170, page, sharing=True, window=window, sinks=sinks)
    say(f"[page step] random serving, seed {seed}, window {window}, sinks {sinks}, page {page}")
    refused = 0
    for t in range(40):
        L = np.array([len(k) for k in s.k[0]])
        new = np.where(L == 0, np.where(rng.random(B) < 0.4, rng.integers(1, 90, B), 0),
                       np.where(rng.random(B) < 0.8, rng.integers(1, 6, B), 0))
        room = int(s.cache.free_count) * page - B * page
        if L.max() + 100 < 64 * page and new.sum() < room:
            s.step(new.tolist())
        L = np.array([len(k) for k in s.k[0]])
        keep = np.where(rng.random(B) < 0.12, 0, np.where(rng.random(B) < 0.3, np.maximum(L - rng.integers(0, 40, B), 0), L))
        gone = s.cache.gone.tolist()
        holds = {}
        for b in range(B):
            for j in range(-(-int(L[b]) // page)):
                if j < -(-sinks // page) or j >= gone[b] // page:
                    holds.setdefault(int(s.cache.block_table[b, j]), []).append(b)
        flags = [0] * B
        for b in range(B):
            k = int(keep[b])
            if 0 < k < L[b]:
                shared = k % page and len(holds.get(int(s.cache.block_table[b, k // page]), [])) > 1
                behind = gone[b] > 0 and k - (window or 0) + 1 < gone[b]
                flags[b] = A.FLAG_REFUSED if shared or behind else 0
        refused += sum(1 for f in flags if f)
        s.cut(keep.tolist(), flags)
        L = np.array([len(k) for k in s.k[0]])
        empty, full = np.nonzero(L == 0)[0], np.nonzero(L > 0)[0]
        if len(empty) and len(full) and int(s.cache.free_count) > B:
            parent, n = np.full(B, -1), np.zeros(B, dtype=int)
            for b in empty:
                if rng.random() < 0.5:
                    p = int(rng.choice(full))
                    parent[b] = p
                    n[b] = L[p] if int(s.cache.gone[p]) > 0 or rng.random() < 0.5 else rng.integers(0, L[p] + 1)
            s.fork(parent.tolist(), n.tolist())
    s.cut([0] * B)
    assert int(s.cache.free_count) == 170
    say(f"{refused} cuts refused")
