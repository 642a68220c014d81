"""The paged cache's oracle against hand-worked tables, torch's softmax and
invariants; mistakes planted in the oracle's inputs are noticed."""
import numpy as np
import pytest
import torch

from oracle import pages as P


def test_tables_by_hand():
    # page size 4; sequence 0 holds 3 tokens and gets 2 (one new page), 1 holds 4 and gets 1
    # (one new page), 2 holds none and gets none
    table = np.full((3, 3), -1)
    table[0, 0], table[1, 0] = 7, 5
    t, slots, lens, count, flags = P.page_tables(4, [0, 2, 3, 3], [3, 4, 0], [9, 8, 6, 2, 0, 0, 0, 0, 0, 0], 4,
                                                 table, 4)
    assert t.tolist() == [[7, 2, -1], [5, 6, -1], [-1, -1, -1]]
    assert slots.tolist() == [7 * 4 + 3, 2 * 4, 6 * 4, -1]
    assert lens.tolist() == [5, 5, 0] and count == 2 and not flags.any()


def test_tables_shortage_and_short_rows_by_hand():
    table = np.full((4, 2), -1)
    table[0, 0] = 1
    # 0: fits its page; 1: wants two pages of one; 2: one page, but 1 went without; 3: row too short
    t, slots, lens, count, flags = P.page_tables(4, [0, 1, 9, 10, 19], [3, 0, 0, 0], [3] + [0] * 9, 1, table, 19)
    assert t[0].tolist() == [1, -1] and (t[1:] == -1).all()
    assert slots.tolist() == [7] + [-1] * 18
    assert lens.tolist() == [4, 0, 0, 0] and count == 1
    assert flags.tolist() == [0] + [P.FLAG_NO_PAGES] * 3


def test_trim_undoes_tables():
    rng = np.random.default_rng(3)
    for ps in (16, 32):
        lens = rng.integers(0, 200, 9)
        new = rng.integers(0, 90, 9)
        cu = np.concatenate(([0], np.cumsum(new)))
        free = rng.permutation(400)
        table = np.full((9, 20), -1)
        t0, _, l0, c0, _ = P.page_tables(ps, np.concatenate(([0], np.cumsum(lens))), np.zeros(9), free, 400, table,
                                         int(lens.sum()))
        t1, slots, l1, c1, f = P.page_tables(ps, cu, l0, free, c0, t0, int(new.sum()))
        assert not f.any() and len(set(slots.tolist())) == len(slots)       # no place twice
        f2, l2, c2, _ = P.page_trim(ps, l0, l1, t1, free, c1)
        assert np.array_equal(l2, l0) and c2 == c0
        assert sorted(f2[:c2]) == sorted(free[:c0])                         # the same pages are free
        f3, l3, c3, _ = P.page_trim(ps, np.zeros(9), l2, t1, f2, c2)
        assert c3 == 400 and sorted(f3) == list(range(400)) and not l3.any()


def _random(seed, Hq=4, Hkv=2, d=64, ps=16):
    rng = np.random.default_rng(seed)
    kv, n = [40, 17, 3], [5, 17, 4]
    k, v = rng.standard_normal((12, Hkv, ps, d)), rng.standard_normal((12, Hkv, ps, d))
    table = rng.permutation(12)[:9].reshape(3, 3)
    q = rng.standard_normal((sum(n) + 1, Hq, d))
    return k, v, q, np.concatenate(([0], np.cumsum(n))), kv, table


def _torch(k, v, q, cu, kv, table, scale):
    out = []
    for b, L in enumerate(kv):
        kk, vv = (torch.tensor(np.concatenate([t[p] for p in table[b]], axis=1)[:, :L]) for t in (k, v))
        n = int(cu[b + 1] - cu[b])
        for t in range(n):
            for h in range(q.shape[1]):
                seen = max(0, L - n + t + 1)
                z = torch.mv(kk[h // 2][:seen], torch.tensor(q[cu[b] + t, h])) * scale
                out.append((torch.softmax(z, 0) @ vv[h // 2][:seen]).numpy())
    return np.array(out).reshape(-1, q.shape[1], q.shape[2])


def test_attention_against_torch_and_empty_rows():
    k, v, q, cu, kv, table = _random(0)
    out, lse, _ = P.page_attention(k, v, q, cu, kv, table, 0.125)
    assert np.allclose(out[:-1], _torch(k, v, q, cu, kv, table, 0.125), rtol=1e-12, atol=1e-13)
    assert np.isnan(out[-1]).all() and np.isnan(lse[:, -1]).all()            # a row of no sequence
    first = int(cu[2])                                                       # 4 queries over 3 tokens
    assert (out[first] == 0).all() and (lse[:, first] == -np.inf).all() and np.isfinite(lse[:, first + 1]).all()


@pytest.mark.parametrize("mistake", ["head", "row", "page", "scale"])
def test_planted_mistakes_are_noticed(mistake):
    k, v, q, cu, kv, table = _random(1)
    good, lse, _ = P.page_attention(k, v, q, cu, kv, table, 0.125)
    if mistake == "head":
        q = q[:, ::-1]
    elif mistake == "row":
        kv = [x - 1 for x in kv]
    elif mistake == "page":
        table = table[:, ::-1]
    bad, lse2, _ = P.page_attention(k, v, q, cu, kv, table, 0.125 if mistake != "scale" else 0.126)
    assert np.nanmax(np.abs(bad - good)) > 1e-3 and not np.allclose(lse, lse2, rtol=1e-6, equal_nan=True)


def test_hidden_values_do_not_reach_a_row():
    k, v, q, cu, kv, table = _random(2)
    good, lse, _ = P.page_attention(k, v, q, cu, kv, table, 0.125)
    last = kv[0] - 1                                                 # seen by the last row of sequence 0 only
    v[table[0, last // 16], :, last % 16] = np.nan
    bad, lse2, _ = P.page_attention(k, v, q, cu, kv, table, 0.125)
    assert np.array_equal(bad[:cu[1] - 1], good[:cu[1] - 1]) and np.isnan(bad[cu[1] - 1]).all()
    assert np.array_equal(lse[:, :cu[3]], lse2[:, :cu[3]])


def test_store_by_hand():
    pages = np.zeros((3, 1, 16, 2))
    rows = np.arange(8.0).reshape(4, 1, 2)
    out = P.page_store(pages, rows, [17, -1, 48, 5], keep_idx=[3, 1, 2, 9])
    assert out[1, 0, 1].tolist() == [6.0, 7.0] and np.count_nonzero(out) == 2
    out = P.page_store(pages, rows, [0, 47])
    assert out[0, 0, 0].tolist() == [0.0, 1.0] and out[2, 0, 15].tolist() == [2.0, 3.0]
