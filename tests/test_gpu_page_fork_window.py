"""Forks of sequences that have left tokens behind their window, by the calls on
plain tensors: release, fork, release."""
import numpy as np
import pytest
import torch

from gpu_util import need_gpu, say
from oracle import pages as P
from paper_2608_26806_amd import avtp as A

pytestmark = pytest.mark.gpu
PS = 16


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    need_gpu()
    A.lib()


def ints(x):
    return torch.tensor(np.asarray(x, dtype=np.int32), device="cuda")


class State:
    """Two sequences of 160 tokens and two empty rows, 30 pages, a window of 32."""

    def __init__(self):
        order = np.random.default_rng(1).permutation(30)
        table = np.full((4, 12), -1)
        table[0, :10], table[1, :10] = order[:10], order[10:20]
        self.lens, self.table, self.gone = ints([160, 160, 0, 0]), ints(table), ints([0] * 4)
        self.free, self.count = ints(np.concatenate([order[20:], np.full(20, -1)])), ints([10])
        self.status = torch.zeros(4, dtype=torch.int32, device="cuda")

    def release(self, keep, sinks=0):
        self.lens, self.count, self.gone = A.page_release(PS, ints(keep), self.lens, self.table, self.free, self.count, 32,
                                                          sinks, self.gone, self.status)

    def fork(self, parent, n, **kw):
        want = P.page_fork(PS, parent, n, *(t.cpu().numpy() for t in (self.lens, self.free)), int(self.count),
                           self.table.cpu().numpy(), self.gone.cpu().numpy())
        self.lens, self.count, src, dst, self.gone = A.page_fork(PS, ints(parent), ints(n), self.lens, self.free, self.count,
                                                                 self.table, self.status, gone=self.gone, **kw)
        torch.cuda.synchronize()
        got = self.table, self.lens, self.count, src, dst, self.gone, self.status
        for g, w, name in zip(got, want, ("table", "seq_len", "free_count", "src", "dst", "gone", "flags")):
            assert np.array_equal(g.cpu().numpy(), np.asarray(w).reshape(g.shape)), name

    def free_pages(self):
        return self.free[:int(self.count)].tolist()


@pytest.mark.parametrize("sinks", [0, 4])
def test_no_page_comes_back_twice(sinks):
    say(f"[fork behind a window] sinks {sinks}")
    s = State()
    s.release([160, 160, 0, 0], sinks)
    assert s.gone.tolist() == [129, 129, 0, 0]
    first = s.free_pages()
    assert len(first) == 10 + 2 * (8 - (sinks > 0))   # eight of ten pages each have left, but for the sinks
    s.fork([-1, -1, 0, -1], [0, 0, 160, 0])
    assert s.gone.tolist() == [129, 129, 129, 0] and s.lens.tolist() == [160, 160, 160, 0] and not s.status.any()
    s.release([160, 160, 0, 0], sinks)                # the child ends: the parent holds its pages
    assert s.free_pages() == first
    s.fork([-1, -1, 1, -1], [0, 0, 160, 0], stream=torch.cuda.current_stream())
    s.release([160, 0, 160, 0], sinks)                # the parent ends: the child holds them
    assert s.free_pages() == first
    s.release([0, 0, 0, 0], sinks)
    assert sorted(s.free_pages()) == list(range(30)) and not s.status.any()


def test_a_fork_of_less_is_refused():
    s = State()
    s.release([160, 160, 0, 0])
    s.fork([-1, -1, 0, 1], [0, 0, 20, 160])
    assert s.status.tolist() == [0, 0, A.FLAG_REFUSED, 0] and s.lens.tolist() == [160, 160, 0, 160]


def test_without_a_window_nothing_changes():
    a, b = State(), State()
    a.fork([-1, -1, 0, 1], [0, 0, 20, 33])
    out = A.page_fork(PS, ints([-1, -1, 0, 1]), ints([0, 0, 20, 33]), b.lens, b.free, b.count, b.table, b.status)
    assert len(out) == 4
    for x, y in zip((a.lens, a.count, a.table), (out[0], out[1], b.table)):
        assert torch.equal(x, y)
