"""Attention over the pages where the running maximum lags or rises: sums near
the range of fp32 in long caches.

The maximum that a row's exponentials refer to is raised when their sum over a
lane's keys of a stage passes 2^16: 8 keys of a tile for 16-row tiles, 16 for
32-row ones, 32 where two tiles are looked at together (fp32, head size 64)."""
import math

import numpy as np
import pytest
import torch

from gpu_util import need_gpu
from paper_2608_26806_amd import avtp as A
from test_gpu_page_attention import E, Case, _reference

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    need_gpu()
    A.lib()


def _set_level(c, level):
    """The logit of token t, for a query whose first value is 1, is level[t] and what the other values add."""
    for b, n in enumerate(c.kv):
        t = torch.arange(n, device="cuda")
        page = torch.tensor(c.table[b], device="cuda")[t // c.ps]
        c.pages.k[page, :, t % c.ps, 0] = torch.as_tensor(level[:n], device="cuda").to(c.pages.dtype)[:, None]


# log2 of the weights behind the first tile, just below the limit of the form
@pytest.mark.parametrize("dtype, d, new, weight, bound", [
    (torch.float32, 64, 1, 12.9, 1), (torch.float32, 128, 1, 12.9, 1), (torch.float32, 128, 40, 11.9, 1),
    (torch.float32, 64, 40, 10.9, 1), (torch.bfloat16, 64, 1, 12.9, 1), (torch.bfloat16, 128, 1, 12.9, 131072),
    (torch.bfloat16, 128, 40, 11.9, 1), (torch.bfloat16, 64, 40, 11.9, 4096)])
def test_the_largest_values_over_a_long_cache(dtype, d, new, weight, bound):
    # 2^17 tokens, values of 2^96 to 2^97, weights of 2^13 a token that the maximum of the first tile leaves as they are
    n = 1 << 17
    c = Case(d + new, dtype, 4, 2, d, 128, [new], [n], scale=1.0)
    c.pages.k.zero_()
    level = np.full(n, weight * math.log(2) / 8)
    level[:32] = 0
    _set_level(c, level)
    c.q.zero_()
    c.q[..., 0] = 8.0
    sign = 1 - 2 * (torch.arange(d, device="cuda") % 2)
    c.pages.v.copy_((0.5 + 0.5 * torch.rand(c.pages.v.shape, device="cuda")) * 2.0 ** 97 * sign)
    out, lse = (t.double().cpu().numpy() for t in c.run(max_kv=bound))
    o, x, (size, reach) = (_reference(c))
    out, o, size, lse, x, reach = out[:new], o[:new], size[:new], lse[:, :new], x[:, :new], reach[:, :new]
    # a logit; the sum, a chain of n / 32 terms a lane; the products, a chain of n / 2 (fp32: two keys an MFMA) terms;
    # in bf16 the probabilities and the result are rounded (2^-8 each)
    es = (d + 4) * E * reach.max() + 2.0 ** -22 + (n / 32 + 20) * E
    step = 2.0 ** -8 if dtype == torch.bfloat16 else E
    assert np.isfinite(out).all() and (np.abs(out - o) <= (2 * es + (n / 2 + 20) * E + 2.02 * step) * size).all()
    assert (np.abs(lse - x) <= es + 2.0 ** -22 * np.abs(x)).all()


# levels that rise in the first and in the second tile of a stage of 64 keys, fall, and rise past all before
STEPS = ((0, 0.0), (96, 20.0), (128, 3.0), (256, 45.0), (288, 10.0), (416, 70.0), (430, 5.0), (704, 90.0), (740, 60.0))


def _rising(dtype, Hq, Hkv, d, new, kv):
    c = Case(sum(new) + d, dtype, Hq, Hkv, d, 32, new, kv, scale=1.0)
    c.pages.k.mul_(0.3)
    level = np.zeros(max(kv))
    for t, x in STEPS:
        level[t:] = x
    _set_level(c, level)
    c.q.mul_(0.5)
    # rows that rise at different steps: some hardly at all, some at each
    c.q[..., 0] = torch.linspace(0.02, 1.4, c.q[..., 0].numel(), device="cuda").reshape(c.q.shape[:2]).to(dtype)
    return c


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("Hq, Hkv, new, kv, bounds", [
    (8, 2, [1] * 5, [900, 97, 257, 430, 800], (900, 4096, 1)),            # 16-row tiles: short and few, in one piece too
    (4, 2, [12, 10, 14], [900, 300, 770], (900, 4096, 1)),                # 32-row tiles: short and few
    (4, 2, [70, 3], [900, 500], (900, 4096, 1)),                          # mixed, blocks of 128 rows in ranges
    (4, 2, [40 + i for i in range(30)], [300 + 20 * i for i in range(30)], (4096,)),   # blocks of 128 rows, uncut in bf16
    (40, 1, [1, 1], [900, 440], (900, 4096, 1))])                         # 40 rows of one token
def test_rising_and_falling_maxima_in_every_form(dtype, d, Hq, Hkv, new, kv, bounds):
    c = _rising(dtype, Hq, Hkv, d, new, kv)
    ref = _reference(c)
    for bound in bounds:
        c.check(c.run(max_kv=bound), ref)
