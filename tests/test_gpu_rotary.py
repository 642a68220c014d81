"""Norm and rotation of heads against the oracle in 64 bits.

What the tolerances count, in units of 2^-24 (E).  The square sum is a chain of up
to 16 fused terms and 4 additions, its relative error halves under the root; the
mean, eps, the root and the reciprocal round once each, and so do the two factors
of y: 10 + 4 + 2, 16 in all.  Sine and cosine: the angle's fraction is cut at 2^-32
turns (2^-29 rad), becomes a float and is multiplied (2 roundings of at most pi / 4),
the sums end in two roundings of at most 1: 4, one more for the scale.  A rotated
value is two products and a sum: 3 roundings of at most |a| + |b|.  So a value is off
by (16 + 5 + 3) E of the pair's |a| + |b| (of |y|, not rotated: 16), plus its own
rounding: half a step of the type, 2^-8 of it in bf16."""
import ctypes

import numpy as np
import pytest
import torch

from gpu_util import need_gpu, say, to_host_bits
from oracle import pages as P
from oracle import rotary as R
from paper_2608_26806_amd import avtp as A
from paper_2608_26806_amd.rotary import Rotary, rotary_frequencies

pytestmark = pytest.mark.gpu
E = 2.0 ** -24
BF, F = torch.bfloat16, torch.float32


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    need_gpu()
    A.lib()


def host(t):
    return t.double().cpu().numpy()


def turns_of(rotary):
    return rotary.turns.cpu().numpy().view(np.uint64)


def oracle(rotary, x, pos, weight, eps):
    planes = None if rotary.planes is None else rotary.planes.tolist()
    p = pos[None] if pos.dim() == 1 else pos
    return R.norm_rotary(host(x), p.cpu().numpy(), turns_of(rotary), rotary.pairs, planes, np.float32(rotary.scale),
                         None if weight is None else host(weight), np.float32(eps))


def check(got, ref, dtype, what):
    (o, bound), g = ref, host(got)
    tol = 24 * E * bound + (2.0 ** -8 if dtype == BF else E) * np.abs(o)
    fine = np.isfinite(o)
    assert np.array_equal(np.isnan(g), np.isnan(o)), f"{what}: NaN in other places"
    assert np.array_equal(g[~fine & ~np.isnan(o)], o[~fine & ~np.isnan(o)]), f"{what}: infinities"
    bad = np.abs(g - o)[fine] > tol[fine] + 1e-37
    assert not bad.any(), f"{what}: {bad.sum()} of {bad.size}, worst {np.max((np.abs(g - o) / (tol + 1e-37))[fine])}"


class Rows:
    """Rows of a fused projection: queries, keys and values side by side."""

    def __init__(self, seed, dtype, n, Hq, Hkv, d, planes=1, low=0, high=200000, pad=8):
        gen = torch.Generator(device="cuda").manual_seed(seed)
        self.all = torch.randn(n, (Hq + 2 * Hkv) * d + pad, generator=gen, device="cuda").to(dtype)
        heads = self.all[:, :(Hq + 2 * Hkv) * d].unflatten(1, (-1, d))
        self.q, self.k, self.v = heads[:, :Hq], heads[:, Hq:Hq + Hkv], heads[:, Hq + Hkv:]
        self.pos = torch.randint(low, high, (planes, n), generator=gen, device="cuda")
        self.wq, self.wk = (1 + 0.3 * torch.randn(d, generator=gen, device="cuda") for _ in range(2))
        say(f"[rotary] {dtype} n {n} heads {Hq}/{Hkv} d {d} planes {planes}")


SHAPES = [(4, 2, 64), (7, 1, 128), (3, 3, 64), (28, 4, 128), (1, 1, 128), (33, 11, 64)]


@pytest.mark.parametrize("dtype", [BF, F])
@pytest.mark.parametrize("pairs", ["half", "interleaved"])
@pytest.mark.parametrize("Hq, Hkv, d", SHAPES)
def test_rows(dtype, pairs, Hq, Hkv, d):
    for n, rot, planes, norm in ((1, d, 1, "qk"), (17, 16, 3, ""), (65, d // 2, 4, "q"), (130, d, 3, "k")):
        x = Rows(n + d, dtype, n, Hq, Hkv, d, planes)
        which = None if planes == 1 else [i * planes // (rot // 2) for i in range(rot // 2)]
        rotary = Rotary(rot, base=1e6, pairs=pairs, planes=which, scale=1.25)
        wq, wk = x.wq if "q" in norm else None, x.wk if "k" in norm else None
        q, k = A.norm_rotary(rotary, x.pos, x.q, x.k, wq, wk, eps=1e-5)
        check(q, oracle(rotary, x.q, x.pos, wq, 1e-5), dtype, "q")
        check(k, oracle(rotary, x.k, x.pos, wk, 1e-5), dtype, "k")


@pytest.mark.parametrize("dtype", [BF, F])
def test_many_rows_share_waves(dtype):
    # more tokens than waves: each wave takes several
    x = Rows(5, dtype, 9001, 4, 2, 64, 3)
    rotary = Rotary(64, base=1e4, planes=[0] * 8 + [1] * 12 + [2] * 12)
    q, k = A.norm_rotary(rotary, x.pos, x.q, x.k, x.wq, x.wk)
    some = torch.tensor([0, 1, 4095, 4096, 4097, 5000, 8191, 8192, 9000], device="cuda")
    check(q[some], oracle(rotary, x.q[some], x.pos[:, some], x.wq, 1e-6), dtype, "q")
    check(k[some], oracle(rotary, x.k[some], x.pos[:, some], x.wk, 1e-6), dtype, "k")
    one, _ = A.norm_rotary(rotary, x.pos[:, 8192:8193], x.q[8192:8193], x.k[8192:8193], x.wq, x.wk)
    assert torch.equal(one[0], q[8192])


@pytest.mark.parametrize("pairs", ["half", "interleaved"])
@pytest.mark.parametrize("low, high", [(-5000, 5000), (1 << 20, (1 << 20) + 100), (1 << 31, (1 << 31) + 9),
                                       (1 << 45, (1 << 45) + 9), (-(1 << 62), -(1 << 62) + 5)])
def test_far_and_negative_positions(pairs, low, high):
    x = Rows(3, F, 40, 2, 1, 128, 1, low, high)
    rotary = Rotary(128, base=5e5, pairs=pairs)
    q, _ = A.norm_rotary(rotary, x.pos, x.q, None)
    check(q, oracle(rotary, x.q, x.pos, None, 0.0), F, "q")


def test_turned_back_by_negated_frequencies():
    x = Rows(4, F, 50, 3, 1, 128)
    f = rotary_frequencies(128, 1e6, "parts", factor=4, trained=4096)[0]
    there, back = Rotary(128, f), Rotary(128, -f)
    q, _ = A.norm_rotary(there, x.pos, x.q, None)
    again, _ = A.norm_rotary(back, x.pos, q, None)
    # two rotations' roundings, 8 E of the pair's |a| + |b| each, once turned: at most sqrt(2) of it
    pair = x.q[..., :64].abs() + x.q[..., 64:].abs()
    assert ((again - x.q).abs() <= 2 * 8 * 1.5 * E * 1.5 * pair.repeat(1, 1, 2)).all()


@pytest.mark.parametrize("dtype", [BF, F])
def test_special_rows(dtype):
    x = Rows(6, dtype, 6, 2, 1, 64)
    q = x.q.contiguous()
    q[0] = 0.0
    q[1, 0, 3] = float("nan")
    q[2, 1, 40] = float("inf")
    q[3] *= 1e-20
    q[4] *= 1e15
    rotary = Rotary(32, base=1e4)
    x.pos[0, 5] = 0
    for weight in (None, x.wq):
        out, _ = A.norm_rotary(rotary, x.pos, q, None, weight, eps=1e-6)
        ref = oracle(rotary, q, x.pos, weight, 1e-6)
        # an infinity beside a sine that is not 0: the oracle's product decides
        check(out[[0, 3, 4, 5]], tuple(r[[0, 3, 4, 5]] for r in ref), dtype, "q")
        for r in (1, 2):
            g, o = host(out[r]), ref[0][r]
            assert np.array_equal(np.isfinite(g), np.isfinite(o))
    # values that are not rotated pass bit for bit without a norm
    out, _ = A.norm_rotary(rotary, x.pos, q, None)
    a, b = to_host_bits(out[..., 32:]), to_host_bits(q[..., 32:])
    assert np.array_equal(a, b)


def test_in_place_and_strides():
    for dtype in (BF, F):
        x = Rows(7, dtype, 33, 5, 5, 64, 3)
        rotary = Rotary(64, base=1e4, pairs="interleaved", planes=[0, 1, 2, 0] * 8)
        q, k = A.norm_rotary(rotary, x.pos, x.q, x.k, x.wq, x.wk)
        before = x.all.clone()
        A.prepare_norm_rotary(rotary, x.pos, x.q, x.q, x.k, x.k, x.wq, x.wk)()
        assert torch.equal(x.q, q) and torch.equal(x.k, k) and torch.equal(x.all[:, 640:], before[:, 640:])
        # positions that are a slice of longer planes
        more = torch.zeros(3, 50, dtype=torch.int64, device="cuda")
        more[:, :33] = x.pos
        q2, _ = A.norm_rotary(rotary, more, before[:, :320].unflatten(1, (5, 64)), None, x.wq)
        assert torch.equal(q2, q)


@pytest.mark.parametrize("dtype, Hq, Hkv, d", [(BF, 4, 2, 64), (BF, 28, 4, 128), (F, 3, 1, 128), (F, 16, 16, 64)])
@pytest.mark.parametrize("ps", [16, 128])
def test_pages(dtype, Hq, Hkv, d, ps):
    for n in (1, 70, 5000 if Hq == 4 else 300):
        x = Rows(n + ps, dtype, n, Hq, Hkv, d, 3)
        n_pages = n // ps + 3
        gen = torch.Generator(device="cuda").manual_seed(n)
        slots = torch.randperm(n_pages * ps, generator=gen, device="cuda")[:n].to(torch.int32)
        if n > 1:
            slots[1], slots[n // 2], slots[n - 1] = -1, n_pages * ps, 2 ** 31 - 1
        pages = A.Pages(*(torch.randn(n_pages, Hkv, ps, d, generator=gen, device="cuda").to(dtype) for _ in range(2)))
        rotary = Rotary(d, base=1e6, planes=[i % 3 for i in range(d // 2)])
        q, k = A.norm_rotary(rotary, x.pos, x.q, x.k, x.wq, x.wk)
        s = slots.cpu().numpy().astype(np.int64)
        want_k = P.page_store(to_host_bits(pages.k), to_host_bits(k), s)
        want_v = P.page_store(to_host_bits(pages.v), to_host_bits(x.v), s)
        got = A.page_store_rotary(pages, rotary, x.pos, x.q, x.k, x.v, slots, x.wq, x.wk)
        # the dense call's rows, bit for bit
        assert torch.equal(got, q)
        assert np.array_equal(to_host_bits(pages.k), want_k) and np.array_equal(to_host_bits(pages.v), want_v)


def test_keys_and_values_alone():
    x = Rows(15, BF, 40, 4, 2, 64)
    slots = torch.arange(40, dtype=torch.int32, device="cuda")
    one, two = A.Pages.empty(3, 2, 16, 64), A.Pages.empty(3, 2, 16, 64)
    for p in (one, two):
        p.k.zero_(), p.v.zero_()
    A.prepare_page_store_rotary(one, Rotary(64), x.pos, None, None, x.k, x.v, slots, None, x.wk)()
    A.page_store_rotary(two, Rotary(64), x.pos, x.q, x.k, x.v, slots, None, x.wk)
    assert torch.equal(one.k, two.k) and torch.equal(one.v, two.v)


def test_values_reach_the_pages_as_they_are():
    x = Rows(9, BF, 16, 2, 2, 64)
    bits = torch.arange(16 * 2 * 64, device="cuda", dtype=torch.int32).mul(37).to(torch.int16).view(16, 2, 64)
    bits[0, 0, :4] = torch.tensor([0x7F81, 0x7FC0, -0x7F, 0x7F80], dtype=torch.int16, device="cuda")  # NaN patterns
    pages = A.Pages.empty(1, 2, 16, 64)
    A.page_store_rotary(pages, Rotary(64), x.pos, x.q, x.k, bits.view(BF), torch.arange(16, dtype=torch.int32, device="cuda"),
                        x.wq, x.wk)
    assert torch.equal(pages.v[0].transpose(0, 1).contiguous().view(torch.int16), bits)


def test_slots_and_rows_behind_four_gigabytes():
    ps, Hkv, d = 64, 8, 128
    n_pages = (5 << 30) // (ps * Hkv * d * 2)
    pages = A.Pages.empty(n_pages, Hkv, ps, d)
    stride = 1 << 22                                  # 600 rows 8 MiB apart
    base = torch.empty(600 * stride, dtype=BF, device="cuda")
    rows = base.as_strided((600, 24, d), (stride, d, 1))
    gen = torch.Generator(device="cuda").manual_seed(3)
    rows.copy_(torch.randn(600, 24, d, generator=gen, device="cuda"))
    pos = torch.randint(0, 9999, (1, 600), generator=gen, device="cuda")
    slots = torch.arange(n_pages * ps - 600, n_pages * ps, dtype=torch.int32, device="cuda")
    rotary = Rotary(d, base=1e6)
    got = A.page_store_rotary(pages, rotary, pos, rows[:, :8], rows[:, 8:16], rows[:, 16:], slots)
    q, k = A.norm_rotary(rotary, pos, rows[:, :8].contiguous(), rows[:, 8:16].contiguous())
    at = slots.long()
    assert torch.equal(got, q) and torch.equal(pages.k[at // ps, :, at % ps], k)
    assert torch.equal(pages.v[at // ps, :, at % ps], rows[:, 16:])


def test_stream_and_graph():
    x = Rows(11, BF, 64, 8, 2, 128, 1)
    rotary = Rotary(128, base=1e6)
    want, want_k = A.norm_rotary(rotary, x.pos, x.q, x.k, x.wq, x.wk)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    got, _ = A.norm_rotary(rotary, x.pos, x.q, x.k, x.wq, x.wk, stream=side)
    side.synchronize()
    assert torch.equal(got, want)
    q, k = torch.zeros_like(want), torch.zeros_like(want_k)
    pos = x.pos.clone()
    call = lambda: A.prepare_norm_rotary(rotary, pos, x.q, q, x.k, k, x.wq, x.wk)()  # noqa: E731
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        call()
    side.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        call()
    for i in range(4):
        pos.copy_(x.pos + i)
        q.zero_()
        g.replay()
        eager, _ = A.norm_rotary(rotary, pos, x.q, x.k, x.wq, x.wk)
        torch.cuda.synchronize()
        assert torch.equal(q, eager)


@pytest.mark.parametrize("dtype, n", [(BF, 17001), (F, 8501)])
def test_large_outputs_past_the_caches(dtype, n):
    x = Rows(13, dtype, n, 32, 8, 128, 3)
    rotary = Rotary(128, base=1e6, planes=[i % 3 for i in range(64)])
    q, k = A.norm_rotary(rotary, x.pos, x.q, x.k, x.wq, x.wk)
    for r in (slice(0, n // 2), slice(n // 2, n)):       # each half below the border
        a, b = A.norm_rotary(rotary, x.pos[:, r], x.q[r], x.k[r], x.wq, x.wk)
        assert torch.equal(q[r], a) and torch.equal(k[r], b)
    some = torch.tensor([0, n // 2, n - 1], device="cuda")
    check(q[some], oracle(rotary, x.q[some], x.pos[:, some], x.wq, 1e-6), dtype, "q")


def test_nothing_to_do():
    rotary = Rotary(64)
    e = torch.empty(0, 2, 64, dtype=BF, device="cuda")
    q, k = A.norm_rotary(rotary, torch.empty(1, 0, dtype=torch.int64, device="cuda"), e, e)
    assert q.shape == k.shape == (0, 2, 64)


def test_refusals_on_the_device():
    x = Rows(12, BF, 8, 4, 2, 64)
    rotary = Rotary(64, planes=[0] * 16 + [1] * 16)
    with pytest.raises(ValueError, match="pos"):
        A.norm_rotary(rotary, x.pos, x.q, x.k)                       # one plane where two are named
    with pytest.raises(TypeError, match="pos"):
        A.norm_rotary(Rotary(64), x.pos.int(), x.q, x.k)
    with pytest.raises(ValueError, match="pos"):
        A.norm_rotary(Rotary(64), x.pos[:, :7], x.q, x.k)
    with pytest.raises(ValueError, match="rows"):
        A.norm_rotary(Rotary(64), x.pos, x.q, x.k[:5])
    with pytest.raises(ValueError, match="q_weight"):
        A.norm_rotary(Rotary(64), x.pos, x.q, x.k, x.wq[:32])
    with pytest.raises(TypeError, match="k_weight"):
        A.norm_rotary(Rotary(64), x.pos, x.q, x.k, None, x.wk.bfloat16())
    with pytest.raises(A.AvtpError):
        A.norm_rotary(Rotary(128), x.pos, x.q, x.k)                  # wider than the head
    with pytest.raises(A.AvtpError):
        A.norm_rotary(Rotary(64), x.pos, x.q, x.k, x.wq, x.wk, eps=-1.0)
    with pytest.raises(A.AvtpError):                                 # in place with another stride
        out = torch.as_strided(x.q, x.q.shape, (x.q.stride(0) - 8, 64, 1))
        A.prepare_norm_rotary(Rotary(64), x.pos, x.q, out, None, None)()
    assert ctypes.sizeof(A._Rotary) == 32
