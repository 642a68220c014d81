"""Pins of the oracle of window attention, forks and releases, on the CPU."""
import numpy as np
import pytest
import torch

from oracle import pages as P


@pytest.mark.parametrize("window, sinks", [(1, 0), (5, 2), (16, 0), (3, 40), (1000, 0)])
def test_window_is_masked_softmax(window, sinks):
    rng = np.random.default_rng(window)
    k, v = rng.standard_normal((2, 4, 2, 16, 8))
    q = rng.standard_normal((7, 4, 8))
    table = np.array([[2, 0, 3, -1]])
    out, lse, _ = P.page_attention_window(k, v, q, [0, 7], [45], table, 0.3, window, sinks)
    kk = torch.from_numpy(k[[2, 0, 3]]).transpose(0, 1).reshape(2, 48, 8)[:, :45].repeat_interleave(2, 0)
    vv = torch.from_numpy(v[[2, 0, 3]]).transpose(0, 1).reshape(2, 48, 8)[:, :45].repeat_interleave(2, 0)
    z = torch.from_numpy(q).transpose(0, 1) @ kk.transpose(1, 2) * 0.3
    p, j = torch.arange(38, 45)[:, None], torch.arange(45)
    z = z.masked_fill((j > p) | ((j <= p - window) & (j >= sinks)), -torch.inf)
    assert np.allclose(out, (torch.softmax(z, -1) @ vv).transpose(0, 1).numpy(), atol=1e-12)
    assert np.allclose(lse, torch.logsumexp(z, -1).numpy(), atol=1e-12)
    if window == 1000:
        a, b, _ = P.page_attention(k, v, q, [0, 7], [45], table, 0.3)
        assert np.allclose(a, out, atol=1e-13) and np.allclose(b, lse, atol=1e-13)


def test_fork_by_hand():
    table = [[5, 3, 8], [-1, -1, -1], [-1, -1, -1], [-1, -1, -1]]
    got = P.page_fork(16, [-1, 0, 0, 0], [0, 40, 32, 0], [40, 0, 0, 0], [9, 7, 1, 0, 0, 0, 0, 0, 0, 0], 3, table)
    assert got[0].tolist() == [[5, 3, 8], [5, 3, 1], [5, 3, -1], [-1, -1, -1]]
    assert got[1].tolist() == [40, 40, 32, 0] and got[2] == 2
    assert got[3].tolist() == [-1, 8, -1, -1] and got[4].tolist() == [-1, 1, -1, -1] and not got[6].any()


def test_release_by_hand():
    table = [[5, 3, 8, 2], [5, 3, 1, -1], [4, 6, 7, 0]]
    free = [9] + [-1] * 9
    # row 0 ends: 5 and 3 stay with row 1
    free2, lens, n, _, _ = P.page_release(16, [0, 40, 64], [60, 40, 64], table, free, 1)
    assert free2[:n].tolist() == [9, 2, 8] and lens.tolist() == [0, 40, 64]
    # both end, row 2 is cut at 17
    free2, lens, n, _, _ = P.page_release(16, [0, 0, 17], [60, 40, 64], table, free, 1)
    assert free2[:n].tolist() == [9, 0, 1, 2, 3, 5, 7, 8] and lens.tolist() == [0, 0, 17]
    # a window of 20 behind 4 first tokens: tokens 45 and later stay, page 0 too
    free2, lens, n, gone, _ = P.page_release(16, [60, 40, 64], [60, 40, 64], table, free, 1, 20, 4, [0, 0, 0])
    assert gone.tolist() == [41, 21, 45] and free2[:n].tolist() == [9, 6]  # row 1 still holds 3
    # a cut in a page that another row holds, one behind the window
    assert P.page_release(16, [60, 10, 64], [60, 40, 64], table, free, 1)[4].tolist() == [0, 64, 0]
    got = P.page_release(16, [60, 40, 63], [60, 40, 64], table, free, 1, 20, 4, [41, 21, 45])
    assert got[4].tolist() == [0, 0, 64] and got[3].tolist() == [41, 21, 45]


def test_every_page_is_held_or_free():
    rng = np.random.default_rng(4)
    for t in range(50):
        B, ps = 6, 16
        lens = rng.integers(1, 90, 3).tolist() + [0, 0, 0]
        need = [-(-n // ps) for n in lens]
        n_pages = sum(need) + 6
        order = rng.permutation(n_pages)
        table, at = np.full((B, 9), -1), 0
        for b, n in enumerate(need):
            table[b, :n] = order[at:at + n]
            at += n
        free = np.concatenate([order[at:], np.full(at, -1)])
        parent = [-1, -1, -1] + rng.integers(0, 3, 3).tolist()
        n = [0, 0, 0] + [int(rng.integers(0, lens[p] + 1)) for p in parent[3:]]
        table, lens, count, src, dst, _, flags = P.page_fork(ps, parent, n, lens, free, 6, table)
        assert not flags.any()
        keep = np.where(rng.random(B) < 0.4, 0, np.maximum(lens - rng.integers(0, 20, B), 0))
        free, lens, count, _, _ = P.page_release(ps, keep, lens, table, free, count)
        held = {int(i) for b in range(B) for i in table[b, :-(-int(lens[b]) // ps)]}
        assert sorted(held | set(free[:count].tolist())) == list(range(n_pages)) and len(held) + count == n_pages
