"""Attention over a window of the paged cache and its first tokens, against the
oracle in 64 bits.

The tolerances are those of attention over all tokens, with the number of keys
that a row sees, n at most: a logit is a chain of d products and a scaling, (d + 4) E
of the row's largest c sum|q k| (E = 2^-24; `reach`); the exponential adds 2^-22 of
itself; the row sum rounds n / 32 + 20 times, the chain over the keys n / 16 + 20 times;
lse is rounded by 2^-22 of itself at most.  An output is sum p v / sum p: p's relative
errors count twice on sum p |v| (`weight`); bf16 rounds p once more (2^-8 of it) and the
result once (2^-8 of it)."""
import numpy as np
import pytest
import torch

from gpu_util import need_gpu, say
from oracle import pages as P
from paper_2608_26806_amd import avtp as A

pytestmark = pytest.mark.gpu
E = 2.0 ** -24
BF, F = torch.bfloat16, torch.float32


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    need_gpu()
    A.lib()


def ints(x):
    return torch.tensor(np.asarray(x, dtype=np.int32), device="cuda")


class Case:
    def __init__(self, seed, dtype, Hq, Hkv, d, ps, new, kv, window, sinks, extra_rows=3):
        gen = torch.Generator(device="cuda").manual_seed(seed)
        rnd = lambda *s: torch.randn(*s, generator=gen, device="cuda")  # noqa: E731
        self.new, self.kv, self.ps, self.d, self.window, self.sinks = list(new), list(kv), ps, d, window, sinks
        self.cu = np.concatenate(([0], np.cumsum(new)))
        need = [-(-n // ps) for n in kv]
        n_pages = sum(need) + 2
        order = np.random.default_rng(seed).permutation(n_pages)
        self.table = np.full((len(kv), max(1, max(need)) + 1), -1)
        at = 0
        for b, n in enumerate(need):
            self.table[b, :n] = order[at:at + n]
            at += n
        self.pages = A.Pages((rnd(n_pages, Hkv, ps, d) * torch.exp(0.5 * rnd(n_pages, 1, 1, 1))).to(dtype),
                             rnd(n_pages, Hkv, ps, d).to(dtype))
        self.q = rnd(int(self.cu[-1]) + extra_rows, Hq, d).to(dtype)
        self.scale = d ** -0.5
        self.status = torch.zeros(len(kv), dtype=torch.int32, device="cuda")

    def run(self, max_kv=None, table=None, **kw):
        out = torch.full(self.q.shape, 7.0, dtype=self.q.dtype, device="cuda")
        lse = torch.full((self.q.shape[1], self.q.shape[0]), 7.0, device="cuda")
        say(f"[window attention] {self.q.dtype} heads {self.q.shape[1]}/{self.pages.Hkv} d {self.d} page {self.ps} "
            f"window {self.window} sinks {self.sinks} new {self.new[:8]} kv {self.kv[:8]}")
        return A.page_attention(self.pages, self.q, ints(self.cu), ints(self.kv),
                                ints(self.table if table is None else table), self.scale,
                                max(self.kv) if max_kv is None else max_kv, out=out, lse=lse, status=self.status,
                                window=self.window, sinks=self.sinks, **kw)

    def oracle(self):
        f = lambda t: t.double().cpu().numpy()  # noqa: E731
        return P.page_attention_window(f(self.pages.k), f(self.pages.v), f(self.q), self.cu, self.kv, self.table,
                                       self.scale, self.window, self.sinks)

    def check(self, got, ref=None):
        out, lse = (t.double().cpu().numpy() for t in got)
        o, x, (weight, reach) = self.oracle() if ref is None else ref
        n_tok = int(self.cu[-1])
        assert (out[n_tok:] == 7.0).all() and (lse[:, n_tok:] == 7.0).all(), "rows of no sequence were written"
        out, o, weight = out[:n_tok], o[:n_tok], weight[:n_tok]
        lse, x, reach = lse[:, :n_tok], x[:, :n_tok], reach[:, :n_tok]
        n = min(max(self.kv), self.window + self.sinks)
        bf = self.pages.dtype == BF
        with np.errstate(all="ignore"):
            es = (self.d + 4) * E * reach + 2.0 ** -22 + (n / 32 + 20) * E
            tol_x = es + 2.0 ** -22 * np.abs(x)
            step = 2.0 ** -8 if bf else E
            tol_o = (2 * es.T[:, :, None] + (n / 16 + 20) * E + (step if bf else 0)) * weight + step * np.abs(o)
        for a, r, tol, what in ((lse, x, tol_x, "lse"), (out, o, tol_o * 1.01, "out")):
            fine = np.isfinite(r)
            assert np.array_equal(np.isnan(a), np.isnan(r)), f"{what}: NaN in other places"
            assert np.array_equal(a[~fine & ~np.isnan(r)], r[~fine & ~np.isnan(r)]), f"{what}: infinities"
            err, bound = np.abs(a[fine] - r[fine]), np.broadcast_to(tol, r.shape)[fine] + 1e-30
            worst = int(np.argmax(err / bound)) if err.size else 0
            assert (err <= bound).all(), f"{what}: {err[worst]:.3e} where {bound[worst]:.3e} is allowed"


KINDS = [(BF, 4, 2, 64), (BF, 7, 1, 128), (F, 4, 2, 64), (F, 3, 1, 128), (BF, 40, 1, 64)]
WINDOWS = [(1, 0), (1, 5), (16, 1), (31, 0), (33, 64), (100, 4), (64, 33), (129, 200), (5000, 3)]


@pytest.mark.parametrize("dtype, Hq, Hkv, d", KINDS)
@pytest.mark.parametrize("window, sinks", WINDOWS)
def test_single_tokens(dtype, Hq, Hkv, d, window, sinks):
    kv = [1, 2, 16, 17, 31, 32, 33, 65, 100, 128, 129, 257, 300, 513]
    c = Case(Hq + d + window, dtype, Hq, Hkv, d, 16 if sinks % 2 else 64, [1] * len(kv), kv, window, sinks)
    ref = c.oracle()
    c.check(c.run(), ref)                        # a block per sequence and key head (bf16)
    c.window, w = 1 << 20, c.window
    big = c.run(max_kv=5000)                     # everything is seen
    c.window = w
    c.check(c.run(max_kv=5000), ref)
    for t in big:
        assert torch.isfinite(t.float()).all()
    assert not c.status.any()


@pytest.mark.parametrize("dtype, Hq, Hkv, d", KINDS)
@pytest.mark.parametrize("window, sinks", WINDOWS)
def test_chunks(dtype, Hq, Hkv, d, window, sinks):
    for new, kv in (([1, 3, 0, 33, 130, 2], [1, 70, 40, 33, 200, 300]), ([65, 31], [130, 31]), ([5, 1, 9], [5, 900, 64]),
                    ([150], [400])):
        c = Case(sum(new) + d, dtype, Hq, Hkv, d, 16 if sinks % 2 else 128, new, kv, window, sinks)
        c.check(c.run())
        assert not c.status.any()


@pytest.mark.parametrize("dtype", [BF, F])
def test_many_keys_in_the_line(dtype):
    # windows that workers share and join (few rows), and ranges of a chunk's keys
    for new, kv, window, sinks in (([1, 1, 2], [3001, 2500, 1700], 2000, 7), ([1], [4000], 3500, 64), ([40], [3500], 3000, 5)):
        c = Case(sum(kv), dtype, 4, 2, 64, 32, new, kv, window, sinks)
        c.check(c.run())
        assert not c.status.any()


@pytest.mark.parametrize("ps", [32, 256, 1024])
def test_other_page_sizes(ps):
    for new, kv in (([1] * 4, [1100, 5, 2050, 700]), ([40, 130], [1500, 1030])):
        for window, sinks in ((300, 17), (1030, 0)):
            c = Case(ps + window, BF, 4, 2, 64, ps, new, kv, window, sinks)
            c.check(c.run())
            assert not c.status.any()


def test_more_than_64_sequences():
    rng = np.random.default_rng(3)
    for n in (130, 70):
        kv = rng.integers(1, 400, n)
        new = np.minimum(kv, rng.integers(0, 12 if n == 130 else 80, n))
        c = Case(n, BF, 4, 2, 64, 16, new.tolist(), kv.tolist(), 37, 18)
        c.check(c.run())
        assert not c.status.any()


@pytest.mark.parametrize("dtype, Hq, Hkv, d, B", [(BF, 8, 8, 128, 70), (BF, 14, 2, 128, 230), (BF, 8, 8, 64, 150),
                                                  (BF, 16, 8, 64, 80), (F, 8, 8, 128, 20), (F, 4, 4, 64, 50)])
def test_many_single_tokens_behind_a_window(dtype, Hq, Hkv, d, B):
    # blocks of two waves and of four, one round and several; some sequences are short
    rng = np.random.default_rng(B)
    kv = rng.integers(1, 700, B)
    for window, sinks in ((40, 4), (150, 0)):
        c = Case(B, dtype, Hq, Hkv, d, 16, [1] * B, kv.tolist(), window, sinks)
        ref = c.oracle()
        c.check(c.run(), ref)
        c.check(c.run(max_kv=100000), ref)
        assert not c.status.any()


@pytest.mark.parametrize("dtype", [BF, F])
@pytest.mark.parametrize("new, kv", [([1] * 5, [700, 300, 40, 1, 129]), ([50, 1, 200], [600, 500, 900])])
def test_pages_that_left_the_window_are_not_looked_at(dtype, new, kv):
    for window, sinks in ((100, 0), (64, 4), (97, 40)):
        c = Case(sum(kv) + window, dtype, 4, 2, 64, 16, new, kv, window, sinks)
        want = c.run()
        c.check(want)
        for stale in (-1, 10 ** 6, -2 ** 31):
            table = c.table.copy()
            for b, (n, L) in enumerate(zip(new, kv)):
                first, last = -(-sinks // 16), max(0, L - n - window + 1) // 16
                table[b, first:max(first, last)] = stale
            got = c.run(table=table)
            assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1]) and not c.status.any()


def test_a_page_in_the_window_that_is_not_there_is_flagged():
    c = Case(1, BF, 4, 2, 64, 16, [1, 1, 1], [200, 200, 200], 50, 20)
    c.table[1, 11] = -1
    c.table[2, 1] = 99999
    c.check(c.run())
    assert c.status.tolist() == [0, A.FLAG_BAD_PAGE, A.FLAG_BAD_PAGE]


@pytest.mark.parametrize("dtype", [BF, F])
@pytest.mark.parametrize("new, kv", [([1, 1, 1], [300, 170, 33]), ([90, 5], [400, 300])])
def test_values_behind_the_window_do_not_reach_a_row(dtype, new, kv):
    # everything outside the window and the sinks of the first row is NaN or infinite
    for window, sinks in ((40, 9), (33, 0), (1, 1)):
        c = Case(sum(kv) + window, dtype, 4, 2, 64, 16, new, kv, window, sinks)
        want = c.run()
        for b, (n, L) in enumerate(zip(new, kv)):
            for j in range(sinks, max(sinks, L - n - window + 1)):
                for t, x in ((c.pages.k, float("nan")), (c.pages.v, float("inf") if j % 2 else float("nan"))):
                    t[int(c.table[b, j // 16]), :, j % 16] = x
        got = c.run()
        assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
        assert not c.status.any()


@pytest.mark.parametrize("dtype", [BF, F])
def test_infinite_values_reach_the_rows_that_see_them_only(dtype):
    c = Case(8, dtype, 4, 2, 64, 16, [70], [150], 40, 6)
    for j, x in ((3, float("inf")), (90, float("-inf")), (100, float("nan")), (130, float("inf"))):
        c.pages.v[int(c.table[0, j // 16]), :, j % 16, j % 64] = x
    c.check(c.run())


def test_rows_that_see_nothing():
    c = Case(9, BF, 4, 2, 64, 16, [5, 3, 40], [2, 0, 30], 4, 2)
    got = c.run()
    c.check(got)
    assert (got[0][:3] == 0).all() and torch.isinf(got[1][:, :3]).all()


def test_a_table_that_ends_before_the_window():
    c = Case(10, BF, 4, 2, 64, 16, [2, 2], [40, 60], 10, 20)
    c.kv = [40, 200]                                   # the table has room for 80
    c.check(c.run(max_kv=200))
    assert c.status.tolist() == [0, A.FLAG_BAD_PAGE]


def test_a_bound_far_from_the_lengths():
    c = Case(11, BF, 7, 1, 128, 16, [1, 2, 1], [900, 33, 500], 300, 4)
    ref = c.oracle()
    for bound in (0, 1, 32, 300, 5000, 1 << 30, 1 << 40):
        c.check(c.run(max_kv=bound), ref)


def test_a_window_of_everything_is_attention_over_everything():
    for new, kv in (([1] * 3, [500, 40, 129]), ([100, 7], [300, 20])):
        c = Case(12, BF, 4, 2, 64, 16, new, kv, 1 << 40, 0)
        got = c.run()
        n = int(c.cu[-1])
        want = A.page_attention(c.pages, c.q, ints(c.cu), ints(c.kv), ints(c.table), c.scale, max(kv))
        assert torch.equal(got[0][:n], want[0][:n]) and torch.equal(got[1][:, :n], want[1][:, :n])


@pytest.mark.parametrize("Hq, Hkv, d, L, n, window, sinks", [(28, 4, 128, 131071, 1, 4096, 4), (8, 2, 64, 70001, 300, 1500, 64),
                                                          (32, 8, 128, 5000, 5000, 700, 16)])
def test_long(Hq, Hkv, d, L, n, window, sinks):
    c = Case(13, BF, Hq, Hkv, d, 64, [n], [L], window, sinks, extra_rows=0)
    out, lse = c.run()
    pos = torch.arange(L, device="cuda")
    page, within = ints(c.table)[0, pos // 64].long(), pos % 64
    some = sorted({0, 1, 130, n // 2, n - 1} & set(range(n)))
    for h in (0, Hq - 1):
        k, v = (t[page, h // (Hq // Hkv), within].double() for t in (c.pages.k, c.pages.v))
        for t in some:
            p = L - n + t
            j = (pos <= p) & ((pos > p - window) | (pos < sinks))
            q = c.q[t, h].double()
            z = (k[j] * q).sum(1) * c.scale
            x = torch.logsumexp(z, 0)
            w = torch.exp(z - x)
            o = (w[:, None] * v[j]).sum(0)
            weight, reach = (w[:, None] * v[j].abs()).sum(0), ((k[j] * q).abs().sum(1) * c.scale).max()
            m = window + sinks
            es = (d + 4) * E * reach + 2.0 ** -22 + (m / 32 + 20) * E
            assert abs(lse[h, t].double() - x) <= es + 2.0 ** -22 * abs(x)
            tol = (2 * es + (m / 16 + 20) * E + 2.0 ** -8) * weight + 2.0 ** -8 * o.abs()
            assert ((out[t, h].double() - o).abs() <= 1.01 * tol).all()
    assert not c.status.any()


def test_reruns_streams_and_graphs():
    c = Case(14, BF, 8, 2, 128, 16, [1] * 40, list(range(100, 4100, 100)), 1000, 4, extra_rows=0)
    want = c.run()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    got = A.page_attention(c.pages, c.q, ints(c.cu), ints(c.kv), ints(c.table), c.scale, 4000, stream=side,
                           window=1000, sinks=4)
    side.synchronize()
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
    kv, table, cu = ints(c.kv), ints(c.table), ints(c.cu)
    out, lse = torch.empty_like(want[0]), torch.empty_like(want[1])
    ws = A.alloc_workspace(A.page_attention_workspace_bytes(c.pages, 8, 40, 40, 4000, 1000, 4))
    call = A.prepare_page_attention(c.pages, c.q, cu, kv, table, c.scale, 4000, out, ws, lse,
                                    stream=side, window=1000, sinks=4)
    with torch.cuda.stream(side):
        call()
        side.synchronize()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=side):
            call()
    torch.cuda.current_stream().wait_stream(side)
    for i in range(4):
        kv.copy_(ints([max(1, x - 37 * i) for x in c.kv]))
        out.zero_()
        g.replay()
        eager = A.page_attention(c.pages, c.q, cu, kv, table, c.scale, 4000, window=1000, sinks=4)
        torch.cuda.synchronize()
        assert torch.equal(out, eager[0]) and torch.equal(lse, eager[1])


@pytest.mark.parametrize("seed", range(40))
def test_random_cases(seed):
    rng = np.random.default_rng(1000 + seed)
    dtype = BF if rng.random() < 0.7 else F
    d = int(rng.choice([64, 128]))
    Hkv = int(rng.choice([1, 2, 3]))
    Hq = Hkv * int(rng.choice([1, 2, 4, 7, 9]))
    B = int(rng.choice([1, 2, 5, 30, 70]))
    kv = np.exp(rng.uniform(0, np.log(1500 if B < 10 else 250), B)).astype(int)
    most = [1, 1, 4, 40, 150][rng.integers(5)] if B < 10 else [1, 1, 5, 20][rng.integers(4)]
    new = np.minimum(rng.integers(0 if rng.random() < 0.3 else 1, most + 1, B), kv + rng.integers(0, 2, B))
    if new.sum() == 0:
        new[0] = 1
    window = int(np.exp(rng.uniform(0, np.log(2000))))
    sinks = int(rng.choice([0, 1, 4, 31, 32, 33, 64, 100, 300]))
    c = Case(seed, dtype, Hq, Hkv, d, int(rng.choice([16, 32, 64, 256])), new.tolist(), kv.tolist(), window, sinks)
    ref = c.oracle()
    for bound in (int(kv.max()), int(rng.choice([1, 100, 4000, 100000]))):
        c.check(c.run(max_kv=bound), ref)
    assert not c.status.any()
