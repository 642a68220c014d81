"""Attention over the paged cache against the oracle in 64 bits.

What the tolerances count.  A logit is a chain of d products accumulated in
fp32 and one scaling: its error is below (d + 4) 2^-24 c sum|q k| (`reach` is
the row's largest c sum|q k|), and the exponential adds 2^-22 of itself.  The
row sum adds one rounding a term of its lane's chain, n / 32 + 20 of them.  lse
moves by the logit's error and the sum's relative one, plus its own rounding.
An output is sum p v / sum p: p's relative errors count twice (numerator and
sum) on sum p |v| (`weight`); bf16 rounds p once more (2^-8 of it) and the
result once (2^-8 of it); the chain over the keys rounds n / 16 + 20 times."""
import ctypes
import math

import numpy as np
import pytest
import torch

from gpu_util import need_gpu, say
from oracle import pages as P
from paper_2608_26806_amd import avtp as A

pytestmark = pytest.mark.gpu
E = 2.0 ** -24


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    need_gpu()
    A.lib()


def ints(x):
    return torch.tensor(np.asarray(x, dtype=np.int32), device="cuda")


class Case:
    def __init__(self, seed, dtype, Hq, Hkv, d, ps, new, kv, extra_rows=3, scale=None, extra_pages=2):
        gen = torch.Generator(device="cuda").manual_seed(seed)
        rnd = lambda *s: torch.randn(*s, generator=gen, device="cuda")  # noqa: E731
        self.new, self.kv, self.ps, self.d = list(new), list(kv), ps, d
        self.cu = np.concatenate(([0], np.cumsum(new)))
        need = [-(-n // ps) for n in kv]
        n_pages = sum(need) + extra_pages
        width = max(1, max(need)) + 1
        order = np.random.default_rng(seed).permutation(n_pages)
        self.table = np.full((len(kv), width), -1)
        at = 0
        for b, n in enumerate(need):
            self.table[b, :n] = order[at:at + n]
            at += n
        self.pages = A.Pages((rnd(n_pages, Hkv, ps, d) * torch.exp(0.5 * rnd(n_pages, 1, 1, 1))).to(dtype),
                             rnd(n_pages, Hkv, ps, d).to(dtype))
        self.q = rnd(int(self.cu[-1]) + extra_rows, Hq, d).to(dtype)
        self.scale = d ** -0.5 if scale is None else scale
        self.status = torch.zeros(len(kv), dtype=torch.int32, device="cuda")

    def run(self, max_kv=None, q=None, out=None, **kw):
        q = self.q if q is None else q
        if out is None:
            out = torch.full(q.shape, 7.0, dtype=q.dtype, device="cuda")
        lse = torch.full((q.shape[1], q.shape[0]), 7.0, device="cuda")
        say(f"[page attention] {q.dtype} heads {q.shape[1]}/{self.pages.Hkv} d {self.d} page {self.ps} "
            f"new {self.new[:8]} kv {self.kv[:8]}")
        return A.page_attention(self.pages, q, ints(self.cu), ints(self.kv), ints(self.table), self.scale,
                                max(self.kv) if max_kv is None else max_kv, out=out, lse=lse, status=self.status, **kw)

    def oracle(self):
        f = lambda t: t.double().cpu().numpy()  # noqa: E731
        return P.page_attention(f(self.pages.k), f(self.pages.v), f(self.q), self.cu, self.kv, self.table, self.scale)

    def check(self, got, ref=None):
        out, lse = (t.double().cpu().numpy() for t in got)
        o, x, (weight, reach) = self.oracle() if ref is None else ref
        n_tok = int(self.cu[-1])
        assert (out[n_tok:] == 7.0).all() and (lse[:, n_tok:] == 7.0).all(), "rows of no sequence were written"
        out, o, weight = out[:n_tok], o[:n_tok], weight[:n_tok]
        lse, x, reach = lse[:, :n_tok], x[:, :n_tok], reach[:, :n_tok]
        n = max(self.kv)
        with np.errstate(all="ignore"):
            ez = (self.d + 4) * E * reach                        # a logit
            es = ez + 2.0 ** -22 + (n / 32 + 20) * E             # a probability before it is normalised, the sum
            tol_x = es + 2.0 ** -22 * np.abs(x)
            ep = (2 * es.T[:, :, None] + (n / 16 + 20) * E) * weight
            step = 2.0 ** -8 if self.pages.dtype == torch.bfloat16 else E
            tol_o = ep + step * np.abs(o) + (step * weight if self.pages.dtype == torch.bfloat16 else 0.0)
        for a, r, tol, what in ((lse, x, tol_x, "lse"), (out, o, tol_o * 1.01, "out")):
            fine = np.isfinite(r)
            assert np.array_equal(np.isnan(a), np.isnan(r)), f"{what}: NaN in other places"
            assert np.array_equal(a[~fine & ~np.isnan(r)], r[~fine & ~np.isnan(r)]), f"{what}: infinities"
            err = np.abs(a[fine] - r[fine])
            bound = np.broadcast_to(tol, r.shape)[fine] + 1e-30
            worst = int(np.argmax(err / bound)) if err.size else 0
            assert (err <= bound).all(), f"{what}: {err[worst]:.3e} where {bound[worst]:.3e} is allowed"


KINDS = [(torch.bfloat16, 4, 2, 64), (torch.bfloat16, 7, 1, 128), (torch.bfloat16, 8, 8, 128),
         (torch.float32, 4, 2, 64), (torch.float32, 3, 1, 128), (torch.bfloat16, 40, 1, 64)]


@pytest.mark.parametrize("dtype, Hq, Hkv, d", KINDS)
@pytest.mark.parametrize("ps", [16, 64])
def test_single_tokens(dtype, Hq, Hkv, d, ps):
    kv = [1, 2, 15, 16, 17, 31, 32, 33, 63, 65, 100, 127, 128, 129, 255, 257, 300, 513]
    c = Case(Hq + d + ps, dtype, Hq, Hkv, d, ps, [1] * len(kv), kv)
    ref = c.oracle()
    c.check(c.run(), ref)                     # a block per sequence and key head (bf16)
    c.check(c.run(max_kv=5000), ref)          # an even line of work over the chip
    assert not c.status.any()


@pytest.mark.parametrize("dtype, Hq, Hkv, d", KINDS)
@pytest.mark.parametrize("ps", [16, 128])
def test_chunks(dtype, Hq, Hkv, d, ps):
    for new, kv in (([1, 3, 0, 33, 130, 2], [1, 70, 40, 33, 200, 300]), ([64], [64]), ([65, 31], [130, 31]),
                    ([5, 1, 9], [5, 900, 64]), ([200], [777])):
        c = Case(sum(new) + d, dtype, Hq, Hkv, d, ps, new, kv)
        c.check(c.run())
        assert not c.status.any()


@pytest.mark.parametrize("dtype, Hq, Hkv, d", KINDS)
def test_rows_that_see_nothing(dtype, Hq, Hkv, d):
    # more new tokens than the cache holds, sequences without any token, single tokens over nothing
    for new, kv in (([5, 1, 1, 40], [2, 0, 1, 7]), ([1, 1, 1], [0, 0, 3]), ([200, 3], [150, 0]), ([2], [0])):
        c = Case(d + new[0], dtype, Hq, Hkv, d, 16, new, kv)
        c.check(c.run())
        c.check(c.run(max_kv=4096))                               # several key ranges, most of them empty


@pytest.mark.parametrize("dtype, Hq, Hkv, d", KINDS)
def test_key_ranges_are_joined(dtype, Hq, Hkv, d):
    for new, kv in (([1], [3001]), ([1, 1], [1500, 40]), ([3], [2048]), ([40], [1111])):
        c = Case(kv[0], dtype, Hq, Hkv, d, 32, new, kv)
        ref = c.oracle()
        assert A.page_attention_workspace_bytes(c.pages, Hq, len(kv), c.q.shape[0], kv[0]) > 0
        c.check(c.run(), ref)
        c.check(c.run(max_kv=1), ref)                             # a bound that is too low: one range takes it all
        c.check(c.run(max_kv=600), ref)
        c.check(c.run(max_kv=1 << 20), ref)
        c.check(c.run(max_kv=1 << 62), ref)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_many_requests(dtype):
    rng = np.random.default_rng(4)
    for B, top in ((64, 2), (65, 3), (200, 2), (4097, 2)):
        new = rng.integers(0, top, B)
        kv = new + rng.integers(0, 40, B)
        c = Case(B, dtype, 2, 1, 64, 16, new, kv)
        c.check(c.run())


@pytest.mark.parametrize("dtype, Hq, Hkv, d", KINDS[:5])
def test_hidden_and_left_over_values_do_not_matter(dtype, Hq, Hkv, d):
    # infinities and NaN behind the last token of a page, in pages of nobody,
    # and in tokens that the later rows of a chunk see and the earlier ones do not
    new, kv = [40, 1, 150], [100, 37, 150]
    c = Case(d, dtype, Hq, Hkv, d, 16, new, kv, extra_pages=4)
    clean = [t.clone() for t in c.run()]
    used = np.zeros((c.pages.n_pages, 16), dtype=bool)
    for b, n in enumerate(kv):
        for t in range(n):
            used[c.table[b, t // 16], t % 16] = True
    free = torch.tensor(~used, device="cuda")
    bad = torch.tensor([float("nan"), float("inf"), -float("inf")], device="cuda").to(dtype)
    for t in (c.pages.k, c.pages.v):
        t.transpose(1, 2)[free] = bad[torch.arange(int(free.sum()), device="cuda") % 3][:, None, None]
    again = c.run()
    assert all(torch.equal(a, b) for a, b in zip(clean, again))
    # token 90 of sequence 0, 20 and 149 of sequence 2: hidden from the rows before them
    for b, t, val in ((0, 90, float("inf")), (2, 20, float("nan")), (2, 149, -float("inf")), (2, 70, float("inf"))):
        c.pages.v[c.table[b, t // 16], :, t % 16, (5 * t) % d] = val
    c.check(c.run())
    for b, t in ((0, 95), (2, 100)):
        c.pages.k[c.table[b, t // 16], :, t % 16, 3] = float("nan")
    c.check(c.run())
    c.check(c.run(max_kv=4096))


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_large_logits_and_rising_maxima(dtype):
    # logits up to the hundreds, the maximum rising from tile to tile and falling again
    c = Case(8, dtype, 4, 2, 64, 16, [1, 70], [500, 400], scale=1.0)
    for b in range(2):
        for p in range(25):
            s = 1.0 + (p if p < 15 else 30 - p) * 0.7
            c.pages.k[c.table[b, p]] = (c.pages.k[c.table[b, p]].float() * s).to(dtype)
    c.check(c.run())
    c.check(c.run(max_kv=4096))


def test_pages_outside_the_pool_count_as_zeros():
    c = Case(21, torch.bfloat16, 4, 2, 128, 16, [1, 20, 1], [200, 90, 64])
    c.table[0, 3], c.table[1, 0], c.table[0, 12] = -1, c.pages.n_pages, 2 ** 31 - 1
    c.check(c.run())
    assert c.status.tolist() == [A.FLAG_BAD_PAGE, A.FLAG_BAD_PAGE, 0]
    # entries behind a sequence's last token are not looked at
    c = Case(22, torch.bfloat16, 4, 2, 128, 16, [1, 2], [33, 16])
    c.table[0, 3:], c.table[1, 1:] = -9, 1 << 30
    c.check(c.run())
    assert not c.status.any()


def test_longer_than_its_table():
    c = Case(23, torch.float32, 4, 2, 64, 16, [1, 9], [200, 48])
    c.kv[1] = 60                                                 # the table holds four pages of nothing more
    c.table = c.table[:, :3].copy()
    c.kv[0] = 48
    c.check(c.run())
    assert c.status.tolist() == [0, A.FLAG_BAD_PAGE]


def test_strided_rows_and_a_pool_behind_4_gib():
    # q a slice of a fused projection, out a slice of a wider buffer, pages at the far end of 5.4 GB
    c = Case(31, torch.bfloat16, 32, 8, 128, 128, [1, 130], [700, 300])
    pool = A.Pages.empty(21000, 8, 128, 128)
    ids = np.array([20999, 16384, 8192, 16383, 12345, 20000, 19999, 17000, 16999])[: c.pages.n_pages - 2]
    move = np.unique(c.table[c.table >= 0])
    new_id = dict(zip(move.tolist(), ids.tolist()))
    for old, new in new_id.items():
        pool.k[new], pool.v[new] = c.pages.k[old], c.pages.v[old]
    ref = c.oracle()
    c.table = np.vectorize(lambda p: new_id.get(p, -1))(c.table)
    c.pages = pool
    wide = torch.randn(c.q.shape[0], 48, 128, device="cuda").to(torch.bfloat16)
    wide[:, 4:36] = c.q
    out = torch.full((c.q.shape[0], 40, 128), 7.0, dtype=torch.bfloat16, device="cuda")
    got = c.run(q=wide[:, 4:36], out=out[:, 2:34])
    c.check(got, ref)
    assert (out[:, :2] == 7.0).all() and (out[:, 34:] == 7.0).all()


def test_reruns_streams_and_two_calls_at_once():
    c = Case(41, torch.bfloat16, 28, 4, 128, 16, [1] * 6 + [30], [900, 33, 2000, 5, 128, 64, 70])
    e = Case(42, torch.bfloat16, 32, 8, 128, 64, [90, 3], [400, 1000])
    first, other = c.run(), e.run()
    for _ in range(3):
        assert all(torch.equal(a, b) for a, b in zip(first, c.run()))
    torch.cuda.synchronize()
    s1, s2 = torch.cuda.Stream(), torch.cuda.Stream()
    res = []
    for _ in range(3):
        with torch.cuda.stream(s1):
            res.append((first, c.run()))
        with torch.cuda.stream(s2):
            res.append((other, e.run()))
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for x, y in res for a, b in zip(x, y))


def test_a_workspace_belongs_to_the_stream_of_its_call(monkeypatch):
    # a stream named in the call: its workspace must not go to the current
    # stream's next allocation while the call may still be running
    c = Case(43, torch.bfloat16, 28, 4, 128, 16, [1, 1], [3000, 1500])
    args = (c.pages, c.q, ints(c.cu), ints(c.kv), ints(c.table), c.scale, 3000)
    first = A.page_attention(*args)
    torch.cuda.synchronize()
    s, alloc, spans = torch.cuda.Stream(), A.alloc_workspace, []

    def noted(*args):
        ws = alloc(*args)
        spans.append((ws.data_ptr(), ws.numel()))
        return ws

    monkeypatch.setattr(A, "alloc_workspace", noted)
    for stream in (s, ctypes.c_void_p(s.cuda_stream)):
        say(f"[page attention] on {stream}")
        got = A.page_attention(*args, stream=stream)
        ptr, n = spans[-1]
        assert not ptr <= alloc(n).data_ptr() < ptr + n
        torch.cuda.synchronize()
        n_tok = int(c.cu[-1])                                     # (other rows are left as they were)
        assert torch.equal(got[0][:n_tok], first[0][:n_tok]) and torch.equal(got[1][:, :n_tok], first[1][:, :n_tok])


def test_two_captured_graphs_with_growing_lengths():
    # one decode step of two batches as graphs that share a workspace; lengths
    # and pages change between the replays, eager work runs in between
    cases = [Case(51, torch.bfloat16, 32, 8, 128, 16, [1, 1, 1], [1900, 40, 300], extra_rows=0),
             Case(52, torch.bfloat16, 28, 4, 128, 16, [1, 1], [700, 1500], extra_rows=0)]
    calls = []
    ws = A.alloc_workspace(max(A.page_attention_workspace_bytes(c.pages, c.q.shape[1], len(c.kv), c.q.shape[0], 2048)
                               for c in cases))
    stream = torch.cuda.Stream()
    for c in cases:
        kv, out = ints(c.kv), torch.empty_like(c.q)
        lse = torch.empty(c.q.shape[1], c.q.shape[0], device="cuda")
        with torch.cuda.stream(stream):
            call = A.prepare_page_attention(c.pages, c.q, ints(c.cu), kv, ints(c.table), c.scale, 2048, out, ws, lse=lse)
            call()
            stream.synchronize()
            g = torch.cuda.CUDAGraph()
            with torch.cuda.graph(g, stream=stream):
                call()
        calls.append((c, g, kv, out, lse, call))
    for r in range(4):
        for c, g, kv, out, lse, call in calls:
            kv.sub_(17 * r)
            out.fill_(5.0)
            torch.cuda.synchronize()
            g.replay()
            torch.cuda.synchronize()
            got = [out.clone(), lse.clone()]
            call()
            torch.cuda.synchronize()
            assert torch.equal(got[0], out) and torch.equal(got[1], lse), (r, c.kv)
            c.kv = kv.tolist()
            c.check(got)


def test_refusals():
    c = Case(61, torch.bfloat16, 4, 2, 64, 16, [1], [3001])
    q = c.q
    with pytest.raises(TypeError, match="bfloat16"):
        c.run(q=q.float())
    with pytest.raises(ValueError, match="needed"):
        c.run(q=q[:, :, :32].contiguous())
    with pytest.raises(A.AvtpError):
        c.run(q=q[:, :3].contiguous())                            # 3 query heads on 2 key heads
    with pytest.raises(A.AvtpError, match="workspace"):
        c.run(ws=torch.empty(64, dtype=torch.uint8, device="cuda"))
    with pytest.raises(ValueError, match="GPU"):
        c.run(q=q.cpu(), out=torch.empty_like(q))
    c.scale = math.inf
    with pytest.raises(A.AvtpError):
        c.run()


def _reference(c):
    """out and lse of a large case in float64 on the GPU, a sequence and key head at a time."""
    N, Hq, d = c.q.shape
    Hkv, ps = c.pages.Hkv, c.ps
    out = torch.full((N, Hq, d), float("nan"), dtype=torch.float64, device="cuda")
    lse = torch.full((Hq, N), float("nan"), dtype=torch.float64, device="cuda")
    weight, reach = torch.zeros_like(out), torch.zeros_like(lse)
    for b, (n, L) in enumerate(zip(c.new, c.kv)):
        if n == 0:
            continue
        r0, G = int(c.cu[b]), Hq // Hkv
        ids = torch.tensor(c.table[b][: -(-L // ps)], device="cuda", dtype=torch.long)
        hidden = torch.arange(L, device="cuda")[None, :] >= L - n + 1 + torch.arange(n, device="cuda")[:, None]
        for g in range(Hkv):
            k, v = (t[ids, g].reshape(-1, d)[:L].double() for t in (c.pages.k, c.pages.v))
            for h in range(g * G, (g + 1) * G):
                qq = c.q[r0:r0 + n, h].double()
                z = (qq @ k.T.contiguous() * c.scale).masked_fill_(hidden, -math.inf)
                lse[h, r0:r0 + n] = torch.logsumexp(z, 1)
                p = torch.exp(z - lse[h, r0:r0 + n, None])
                out[r0:r0 + n, h], weight[r0:r0 + n, h] = p @ v, p @ v.abs()
                reach[h, r0:r0 + n] = (c.scale * (qq.abs() @ k.abs().T.contiguous())).masked_fill_(hidden, 0).amax(1)
    f = lambda t: t.cpu().numpy()  # noqa: E731
    return f(out), f(lse), (f(weight), f(reach))


@pytest.mark.parametrize("dtype, d", [(torch.bfloat16, 64), (torch.bfloat16, 128), (torch.float32, 64)])
def test_long_chunks_among_single_tokens(dtype, d):
    # sequences of one row tile beside some of 13 and of 80 tiles, and padding without tokens
    for B, long in ((65, {3: 100}), (100, {0: 640, 99: 37}), (64, {63: 90}), (1, {0: 9})):
        new = [long.get(b, b % 3 % 2) for b in range(B)]
        kv = [n + (53 * b) % 200 for b, n in enumerate(new)]
        c = Case(B + d, dtype, 4, 2, d, 16, new, kv)
        c.check(c.run(), _reference(c))


@pytest.mark.parametrize("dtype, Hq, Hkv, d", [(torch.bfloat16, 8, 2, 128), (torch.bfloat16, 4, 4, 64),
                                                (torch.float32, 6, 2, 64), (torch.float32, 4, 1, 128)])
def test_many_chunks(dtype, Hq, Hkv, d):
    rng = np.random.default_rng(Hq)
    for B, low, high, cached in ((70, 40, 60, 300), (64, 40, 60, 300), (7, 200, 500, 1500), (2, 1000, 1300, 0)):
        new = rng.integers(low, high, B)
        kv = new + rng.integers(0, cached + 1, B)
        if B > 60:
            new[5] = kv[5] = 0
        c = Case(B, dtype, Hq, Hkv, d, 32, new, kv)
        c.check(c.run(), _reference(c))


def test_long_caches():
    for new, kv in (([1, 1, 2], [40000, 70001, 513]), ([300], [20000]), ([1] * 9, [3001 + 777 * i for i in range(9)])):
        c = Case(len(kv), torch.bfloat16, 14, 2, 64, 64, new, kv)
        ref = _reference(c)
        c.check(c.run(), ref)
        c.check(c.run(max_kv=100), ref)


def test_first_row_is_not_row_zero():
    # a batch that starts behind other rows of q and out, few rows and many (more than 64 sequences among them)
    for B, n in ((3, 1), (3, 70), (66, 40)):
        c = Case(B, torch.bfloat16, 4, 2, 64, 16, [n] * B, [n + 30] * B, extra_rows=200)
        out, lse = (t.clone() for t in c.run())
        q = c.q.roll(150, 0)
        c.cu = c.cu + 150
        moved, mlse = c.run(q=q)
        m = n * B
        assert torch.equal(moved[150:150 + m], out[:m]) and torch.equal(mlse[:, 150:150 + m], lse[:, :m])
        assert (moved[:150] == 7.0).all() and (moved[150 + m:] == 7.0).all()


@pytest.mark.parametrize("dtype, Hq, Hkv, d", KINDS)
def test_chunks_in_every_form(dtype, Hq, Hkv, d):
    # short chunks as tiles of one block each (bf16), and with a bound that spreads them over blocks of 128 rows
    # and key ranges; tiles without keys, tiles of a few rows, more sequences than a wave has lanes
    for new, kv in (([1, 3, 0, 33, 130, 2], [1, 70, 40, 33, 200, 300]), ([70, 5, 130, 1], [300, 900, 130, 1]),
                    ([60, 60], [1000, 20]), ([12] * 66 + [0, 0, 40], [12 + 5 * i for i in range(66)] + [0, 90, 0])):
        c = Case(sum(new) + Hq, dtype, Hq, Hkv, d, 32, new, kv)
        ref = c.oracle()
        c.check(c.run(), ref)
        c.check(c.run(max_kv=1 << 20), ref)
        assert not c.status.any()


def test_chunks_over_bad_pages_in_every_form():
    c = Case(24, torch.bfloat16, 4, 2, 128, 16, [100, 40, 1], [200, 90, 64])
    c.table[0, 3], c.table[1, 0], c.table[0, 12] = -1, c.pages.n_pages, 2 ** 31 - 1
    for bound in (200, 4096):
        c.status.zero_()
        c.check(c.run(max_kv=bound))
        assert c.status.tolist() == [A.FLAG_BAD_PAGE, A.FLAG_BAD_PAGE, 0]
