"""Window attention where a row's reference has to rise behind its first tile.

In blocks of 128 rows a tile behind the first keeps the row's reference while the sum of
a lane's keys stays below 2^16, in tiles that all rows see and in those at a window's
ends; else the tile's largest logit becomes the reference.  The levels here rise by 20 to
60 (29 to 87 powers of two) and fall again every few dozen keys, so that as rows move on
each kind of tile does either: right behind the sinks, at both ends of the window, within."""
import numpy as np
import pytest
import torch

from gpu_util import need_gpu
from paper_2608_26806_amd import avtp as A
from test_gpu_page_window import BF, F, KINDS, Case

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    need_gpu()
    A.lib()


def _levels(kind, n, seed):
    t = np.arange(n)
    if kind == "rising":                    # to the end: every row's own tile holds its largest logits
        return 90.0 * t / n + 6.0 * (t // 16 % 2)
    if kind == "falling":                   # the sinks, then the window's first keys are the largest
        return 90.0 * (1 - t / n)
    if kind == "steps":                     # up by 20 or more and down again, at places that fit no tile
        at = np.cumsum(np.random.default_rng(seed).integers(7, 60, n))
        up = np.random.default_rng(seed + 1).uniform(0, 60, n)
        return up[np.searchsorted(at, t, side="right")]
    assert kind == "peaks"                  # single keys far above the rest
    return np.where(np.random.default_rng(seed).random(n) < 0.02, 70.0, 0.0)


def _case(kind, dtype, Hq, Hkv, d, new, kv, window, sinks):
    c = Case(sum(new) + d + window, dtype, Hq, Hkv, d, 32, new, kv, window, sinks)
    c.scale = 1.0
    c.pages.k.mul_(0.3)
    level = torch.tensor(_levels(kind, max(kv), window), device="cuda")
    for b, n in enumerate(kv):
        t = torch.arange(n, device="cuda")
        page = torch.tensor(c.table[b], device="cuda")[t // c.ps]
        c.pages.k[page, :, t % c.ps, 0] = level[:n].to(dtype)[:, None]
    c.q.mul_(0.5)
    # rows for which the levels are next to nothing beside rows for which they are all
    c.q[..., 0] = torch.linspace(0.02, 1.4, c.q[..., 0].numel(), device="cuda").reshape(c.q.shape[:2])[
        torch.randperm(c.q.shape[0], generator=torch.Generator().manual_seed(1)).cuda()].to(dtype)
    return c


def _reference(c):
    """The oracle's results, all rows of a sequence and head at once in 64 bits on the device."""
    N, Hq, d = c.q.shape
    G = Hq // c.pages.Hkv
    o, weight = (torch.zeros(N, Hq, d, dtype=torch.float64, device="cuda") for _ in range(2))
    x, reach = (torch.zeros(Hq, N, dtype=torch.float64, device="cuda") for _ in range(2))
    for b, (n, L) in enumerate(zip(c.new, c.kv)):
        j, r = torch.arange(L, device="cuda"), slice(int(c.cu[b]), int(c.cu[b + 1]))
        p = torch.arange(L - n, L, device="cuda")[:, None]
        hidden = (j > p) | ((j <= p - c.window) & (j >= c.sinks))
        page = torch.tensor(c.table[b], device="cuda")[j // c.ps]
        for h in range(Hq):
            k, v = (t[page, h // G, j % c.ps].double() for t in (c.pages.k, c.pages.v))
            q, kt = c.q[r, h].double(), k.T.contiguous()
            z = (torch.mm(q, kt) * c.scale).masked_fill(hidden, -torch.inf)
            x[h, r] = torch.logsumexp(z, 1)
            w = torch.exp(z - x[h, r, None])
            o[r, h], weight[r, h] = torch.mm(w, v), torch.mm(w, v.abs())
            reach[h, r] = (torch.mm(q.abs(), kt.abs()) * c.scale).masked_fill(hidden, 0.0).amax(1)
    return tuple(t.cpu().numpy() for t in (o, x)) + ((weight.cpu().numpy(), reach.cpu().numpy()),)


# more tiles of 32 rows than are joined in LDS (512), uncut in bf16 where the window is short; few tiles of
# many keys, in ranges
@pytest.mark.parametrize("kind", ["rising", "falling", "steps", "peaks"])
@pytest.mark.parametrize("dtype", [BF, F])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("Hq, Hkv, new, kv, window, sinks, cut", [
    (16, 8, [550, 550], [550, 700], 5, 0, False),          # windows within a wave's rows: some have no reference yet
    (16, 8, [550, 550], [700, 550], 90, 40, False),
    (16, 8, [300, 800], [900, 800], 333, 3, None),
    (16, 2, [130], [2600], 2100, 40, True)])
def test_references_rise_behind_the_first_tile(kind, dtype, d, Hq, Hkv, new, kv, window, sinks, cut):
    c = _case(kind, dtype, Hq, Hkv, d, new, kv, window, sinks)
    if cut is not None and dtype == BF:
        ws = A.page_attention_workspace_bytes(c.pages, Hq, len(new), c.q.shape[0], max(kv), window, sinks)
        assert (ws > 0) == cut
    c.check(c.run(), _reference(c))
    assert not c.status.any()


@pytest.mark.parametrize("dtype", [BF, F])
@pytest.mark.parametrize("kind", ["rising", "steps"])
def test_infinite_values_beside_references_that_rise(kind, dtype):
    # in the windows of some rows of a tile and not of others, where the levels rise
    c = _case(kind, dtype, 16, 8, 64, [550, 550], [700, 550], 60, 5)
    places = [(0, 3, "inf"), (0, 333, "-inf"), (0, 500, "nan"), (1, 80, "inf"), (1, 530, "nan")]
    for b, j, x in places:
        c.pages.v[int(c.table[b, j // 32]), j % 8, j % 32, j % 64] = float(x)
    out, lse = c.run()
    o, x, bound = c.oracle()
    # A weight below 2^-126 of the row's largest is zero in fp32 (exp2 flushes what is smaller), and so is the factor
    # that takes what was summed to a reference so much higher: infinity times it is NaN where the formula has infinity.
    # From 2^-125 of the row's sum on each factor on the way is at least that, and the infinity stays.
    for b, j, _ in places:
        g, e = j % 8, j % 64
        k = c.pages.k[int(c.table[b, j // 32]), g, j % 32].double()
        for h in (2 * g, 2 * g + 1):
            r = slice(int(c.cu[b]), int(c.cu[b + 1]))
            z = ((c.q[r, h].double() * k).sum(1) * c.scale).cpu().numpy()
            p = np.arange(c.kv[b] - c.new[b], c.kv[b])
            faint = (j <= p) & ((j > p - c.window) | (j < c.sinks)) & ((z - x[h, r]) / np.log(2) < -125)
            rows = np.arange(len(c.q))[r][faint]
            assert not np.isfinite(o[rows, h, e]).any() and not torch.isfinite(out[rows, h, e]).any()
            o[rows, h, e] = 0.0
            out[rows, h, e] = 0.0
    c.check((out, lse), (o, x, bound))


@pytest.mark.parametrize("dtype, Hq, Hkv, d", KINDS)
@pytest.mark.parametrize("sinks", [0, 5, 64])
def test_single_tokens_that_see_everything(dtype, Hq, Hkv, d, sinks):
    kv = [1, 2, 16, 17, 31, 32, 33, 65, 100, 128, 129, 257, 300, 513]
    c = Case(Hq + d, dtype, Hq, Hkv, d, 16, [1] * len(kv), kv, 1 << 20, sinks)
    ref = c.oracle()
    for bound in (513, 5000):
        c.check(c.run(max_kv=bound), ref)


@pytest.mark.parametrize("window, sinks", [(256, 5), (316, 4), (317, 4)])
def test_chunks_at_the_border_of_a_form(window, sinks):
    # 440 tiles: blocks that join their waves' parts up to 320 keys, two launches behind
    c = _case("steps", F, 14, 2, 64, [1000], [1700], window, sinks)
    ws = A.page_attention_workspace_bytes(c.pages, 14, 1, c.q.shape[0], 1700, window, sinks)
    assert (ws > 0) == (window + sinks > 320)
    c.check(c.run(), _reference(c))
