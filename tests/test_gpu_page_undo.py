"""A pruning step that fails leaves a cache with a window, or with forks, as it was:
lengths, what has left the windows, pages held and free, and the tokens that wait
for their attention."""
import numpy as np
import pytest
import torch

from gpu_util import need_gpu, say
from paper_2608_26806_amd import avtp as A
from paper_2608_26806_amd.paged import PagedCache
from paper_2608_26806_amd.progressive import ProgressivePruner
from paper_2608_26806_amd.workloads import build_layout

pytestmark = pytest.mark.gpu
PAGE = 16


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    need_gpu()
    A.lib()


def ints(x):
    return torch.tensor(np.asarray(x, dtype=np.int32), device="cuda")


def _normal(seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    return lambda *s: torch.randn(*s, generator=gen, device="cuda").to(torch.bfloat16)


def _state(c):
    """Everything but the order of the stack."""
    lens, gone = c.seq_len.tolist(), c.gone.tolist()
    first = -(-c.sinks // PAGE)
    held = [[int(c.block_table[b, j]) for j in range(-(-n // PAGE)) if j < first or j >= gone[b] // PAGE]
            for b, n in enumerate(lens)]
    free = sorted(c.free_pages[:int(c.free_count)].tolist())
    assert sorted(set(sum(held, []) + free)) == list(range(c.free_pages.numel())) and len(set(free)) == len(free)
    assert not set(sum(held, [])) & set(free)
    return lens, gone, held, free, c._seen.tolist()


def _step(seed):
    """A pruning step of two sequences, of 36 and 19 kept tokens."""
    dl = A.DeviceLayout(build_layout([[40, 20], [12]], 3, 12, 30))
    rnd = _normal(seed)
    k, v = rnd(dl.N_tok, 2, 64), rnd(dl.N_tok, 2, 64)
    return dl, rnd, rnd(dl.N_tok, 64), k, v, ProgressivePruner(dl, rnd(dl.N_tok, 64))


FAILURES = [(dict(), RuntimeError, "no pages"), (dict(keep_pct_next=None), TypeError, None)]


@pytest.mark.parametrize("failure, error, match", FAILURES)
def test_behind_a_window(failure, error, match):
    dl, rnd, cur, k, v, pruner = _step(1)
    window, sinks, scale = 20, 4, 0.125
    say("[page undo] a failing step behind a window")
    # 9 pages: 8 for 90 and 30 tokens, of which three leave the window, then two for 12 more tokens each
    c = PagedCache(2, 9 if match else 30, 12, 2, 64, PAGE, window=window, sinks=sinks)
    c.store(0, rnd(120, 2, 64), rnd(120, 2, 64), c.reserve(ints([0, 90, 120]), 120))
    c.trim(c.seq_len.clone())
    assert c.gone.tolist() == [71, 11]
    cu = ints([0, 12, 24])
    c.store(0, rnd(24, 2, 64), rnd(24, 2, 64), c.reserve(cu, 24))
    q = rnd(24, 4, 64)
    want = c.attend(0, q, cu, scale)
    before, slots = _state(c), c.slots
    if match:
        assert len(before[3]) == 2                    # sequence 0 takes both, 1 gets none
    for _ in range(2):
        with pytest.raises(error, match=match):
            pruner.step(cur, cache=c, k=k, v=v, **failure)
        assert _state(c) == before and c.slots is slots and pruner.dl is dl
    # the tokens reserved before it see what they saw, whoever takes pages now
    status = torch.zeros(2, dtype=torch.int32, device="cuda")
    got = c.attend(0, q, cu, scale, status=status)
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1]) and not status.any()
    # and drafts are cut as they could be
    c.trim(ints([92, 33]), status)
    assert not status.any() and c.seq_len.tolist() == [92, 33] and c.gone.tolist() == [73, 14]
    _state(c)
    if not match:
        pruner.step(cur, cache=c, k=k, v=v)
        assert c.seq_len.tolist() == [92 + 36, 33 + 19]
        _state(c)
    c.trim(ints([0, 0]))
    assert int(c.free_count) == c.free_pages.numel()


@pytest.mark.parametrize("failure, error, match", FAILURES)
def test_among_forks(failure, error, match):
    dl, rnd, cur, k, v, pruner = _step(2)
    say("[page undo] a failing step among forks")
    c = PagedCache(2, 6 if match else 30, 12, 2, 64, PAGE, sharing=True)
    c.store(0, rnd(40, 2, 64), rnd(40, 2, 64), c.reserve(ints([0, 40, 40]), 40))
    c.fork(ints([-1, 0]))                             # two whole pages shared, the third copied
    before = _state(c)
    assert len(set(before[2][0]) & set(before[2][1])) == 2
    with pytest.raises(error, match=match):
        pruner.step(cur, cache=c, k=k, v=v, **failure)
    assert _state(c) == before and pruner.dl is dl
    c.trim(ints([0, 40]))
    c.trim(ints([0, 0]))
    assert int(c.free_count) == c.free_pages.numel()


def test_a_window_that_no_trim_has_moved_yet():
    # nothing has left the window on record: the step must not let go of it either
    dl, rnd, cur, k, v, pruner = _step(3)
    say("[page undo] a failing step before the first trim")
    c = PagedCache(2, 12, 12, 2, 64, PAGE, window=5, sinks=0)
    c.store(0, rnd(150, 2, 64), rnd(150, 2, 64), c.reserve(ints([0, 100, 150]), 150))
    before = _state(c)
    assert before[1] == [0, 0] and len(before[3]) == 1
    with pytest.raises(RuntimeError, match="no pages"):
        pruner.step(cur, cache=c, k=k, v=v)
    assert _state(c) == before
