"""The paged cache's block tables, slots, trimming and stores on the GPU,
against the oracle: whole numbers and copies, so everything is equal."""
import numpy as np
import pytest
import torch

from gpu_util import need_gpu, say
from oracle import pages as P
from paper_2608_26806_amd import avtp as A

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    need_gpu()
    A.lib()


def ints(x):
    return torch.tensor(np.asarray(x, dtype=np.int32), device="cuda")


def _tables_equal(ps, cu, lens, free, count, table, n_new, what):
    say(f"[page tables] {what}: B {len(lens)}, page {ps}, {n_new} new, {count} of {len(free)} free")
    t, status = ints(table), torch.zeros(len(lens), dtype=torch.int32, device="cuda")
    slots, out, left = A.page_tables(ps, ints(cu), ints(lens), ints(free), ints([count]), t, n_new, status=status)
    ref = P.page_tables(ps, cu, lens, free, count, table, n_new)
    for got, want, name in zip((t, slots, out, left, status), ref, ("table", "slots", "lengths", "count", "flags")):
        assert np.array_equal(got.cpu().numpy().reshape(-1), np.asarray(want).reshape(-1)), (what, name)
    return ref


def _held(rng, B, ps, max_pages, low, high, n_pages):
    """A running state: lengths, a table of pages taken from a shuffled pool, the rest free."""
    lens = rng.integers(low, high + 1, B)
    order = rng.permutation(n_pages)
    table, used = np.full((B, max_pages), -1), 0
    for b in range(B):
        k = -(-int(lens[b]) // ps)
        table[b, :k] = order[used:used + k]
        used += k
    return lens, table, np.concatenate([order[used:], np.full(used, -1)]), n_pages - used


@pytest.mark.parametrize("B", [1, 2, 63, 65, 255, 1023, 1024, 1025, 2500])
@pytest.mark.parametrize("ps", [16, 64, 1024])
def test_tables_decode_and_chunks(B, ps):
    rng = np.random.default_rng(B * 7 + ps)
    for new_high, short in ((1, False), (40, False), (40, True)):
        n_pages = B * 8 + 4
        lens, table, free, count = _held(rng, B, ps, 6, 0, 4 * ps, n_pages)
        new = rng.integers(0, new_high + 1, B)
        if short:
            count = min(count, B // 3)
        cu = np.concatenate(([0], np.cumsum(new)))
        _tables_equal(ps, cu, lens, free, count, table, int(cu[-1]) + 5, f"new 0..{new_high}, short {short}")


def test_tables_long_prompts_padding_and_refused_requests():
    rng = np.random.default_rng(5)
    # whole prompts into an empty cache, slots over many blocks; one prompt too long for its row
    new = [5000, 0, 12345, 1, 1023, 9000, 1024, 2049]
    cu = np.concatenate(([0], np.cumsum(new)))
    free = rng.permutation(2300)
    table = np.full((8, 600), -1)
    ref = _tables_equal(16, cu, [0] * 8, free, 2300, table, int(cu[-1]) + 3000, "prompts")
    assert ref[4][2] == P.FLAG_NO_PAGES and (ref[1][cu[-1]:] == -1).all()
    # nothing new at all, and a slot map that is too short for the last two requests
    _tables_equal(16, [0] * 9, [0, 5, 16, 17, 0, 0, 33, 1], free, 10, np.zeros((8, 600)), 0, "nothing new")
    _tables_equal(16, cu, [0] * 8, free, 2300, np.full((8, 1000), -1), int(cu[6]) + 7, "short slot map")
    # the stack runs out inside a request; empty; a count above the pool's size is read as the pool's size
    for count in (0, 1, 700, 2300):
        _tables_equal(16, cu, [3, 0, 0, 40, 0, 16, 1, 0], free, count, np.full((8, 1000), 7), int(cu[-1]), f"{count} free")


def test_tables_page_ids_outside_the_pool():
    table = np.full((3, 4), -1)
    table[0, 0], table[1, 0], table[2, 0] = -1, 500, 3            # started pages: two bad ones, a good one
    ref = _tables_equal(16, [0, 2, 4, 6], [5, 5, 5], list(range(9)), 9, table, 6, "bad started pages")
    assert ref[4].tolist() == [P.FLAG_BAD_PAGE, P.FLAG_BAD_PAGE, 0]
    _tables_equal(16, [0, 20, 40], [0, 0], [5, -7, 900, 1], 4, np.zeros((2, 4)), 40, "bad stack entries")


def test_tables_of_more_requests_than_a_chunk_with_slots_across():
    rng = np.random.default_rng(9)
    B = 3000                                                     # three chunks of sequences, slots in many blocks
    lens, table, free, count = _held(rng, B, 16, 12, 0, 90, B * 10)
    new = rng.integers(0, 60, B)
    new[1000:1100] = 0
    cu = np.concatenate(([0], np.cumsum(new)))
    for c in (count, 2500, 6000):
        _tables_equal(16, cu, lens, free, min(c, count), table, int(cu[-1]), f"three chunks, {c} free")


@pytest.mark.parametrize("B", [1, 4, 5, 64, 1000, 1500, 5000])
def test_trim(B):
    rng = np.random.default_rng(B)
    for ps, share in ((16, 0.0), (64, 0.3), (16, 1.0)):
        lens, table, free, count = _held(rng, B, ps, 9, 0, 8 * ps, B * 10)
        keep = np.where(rng.random(B) < share, 0, np.maximum(0, lens - rng.integers(-2, 9, B)))
        status = torch.zeros(B, dtype=torch.int32, device="cuda")
        f = ints(free)
        say(f"[page trim] B {B}, page {ps}, {share} ended")
        out, left = A.page_trim(ps, ints(keep), ints(lens), ints(table), f, ints([count]), status=status)
        rf, rl, rc, rs = P.page_trim(ps, keep, lens, table, free, count)
        assert np.array_equal(f.cpu().numpy(), rf) and np.array_equal(out.cpu().numpy(), rl)
        assert int(left) == rc and np.array_equal(status.cpu().numpy(), rs)


def test_trim_into_a_full_stack_flags():
    table = np.arange(24).reshape(3, 8)
    status = torch.zeros(3, dtype=torch.int32, device="cuda")
    f = ints(np.full(24, 77))
    out, left = A.page_trim(16, ints([0, 0, 0]), ints([128, 100, 20]), ints(table), f, ints([14]), status=status)
    rf, rl, rc, rs = P.page_trim(16, [0, 0, 0], [128, 100, 20], table, np.full(24, 77), 14)
    assert np.array_equal(f.cpu().numpy(), rf) and int(left) == rc == 24 and not out.any()
    assert status.tolist() == rs.tolist() == [0, P.FLAG_OUT_CAPACITY, P.FLAG_OUT_CAPACITY]


def test_trim_of_more_pages_than_31_bits():
    # the pages handed back and the stack together pass 2^31: 31 sequences of 2^30 tokens
    B, per, n_pages = 31, 1 << 26, (1 << 27) - 1
    say("[page trim] 31 x 2^26 pages")
    table = torch.zeros(B, per, dtype=torch.int32, device="cuda")
    table[0, :100] = torch.arange(100, device="cuda", dtype=torch.int32) + 7
    f = torch.full((n_pages,), -3, dtype=torch.int32, device="cuda")
    status = torch.zeros(B, dtype=torch.int32, device="cuda")
    out, left = A.page_trim(16, ints([0] * B), ints([1 << 30] * B), table, f, ints([n_pages - 100]), status=status)
    assert int(left) == n_pages and not out.any() and (status == A.FLAG_OUT_CAPACITY).all()
    assert torch.equal(f[-100:], table[0, :100]) and (f[:-100] == -3).all()


def _bits(t):
    return t.view(torch.int32 if t.element_size() == 4 else torch.int16).cpu().numpy()


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("Hkv, d", [(1, 64), (2, 64), (3, 128), (8, 128), (16, 64), (5, 64)])
def test_store_bit_exact(dtype, Hkv, d):
    rng = np.random.default_rng(Hkv * d)
    gen = torch.Generator(device="cuda").manual_seed(Hkv + d)
    for ps, n, n_src, fused in ((16, 1, 1, False), (16, 77, 77, True), (64, 130, 400, True), (128, 9, 33, False)):
        n_pages = 2 * n // ps + 3
        pages = A.Pages(*(torch.randn(n_pages, Hkv, ps, d, generator=gen, device="cuda").to(dtype) for _ in "kv"))
        src = torch.randn(n_src, 3 + 2 * Hkv, d, generator=gen, device="cuda").to(dtype)
        k, v = (src[:, 3:3 + Hkv], src[:, 3 + Hkv:]) if fused else (src[:, :Hkv].contiguous(), src[:, -Hkv:].contiguous())
        slots = rng.permutation(n_pages * ps)[:n]
        keep = np.sort(rng.choice(n_src, n, replace=False)) if n_src != n else None
        if n > 20:                                       # no place, outside the pool, no such row
            slots[3], slots[7], slots[8] = -1, n_pages * ps, 2 ** 31 - 1
            if keep is not None:
                keep[11], keep[12] = -5, n_src
        want = [P.page_store(_bits(t), _bits(r.contiguous()), slots, keep) for t, r in ((pages.k, k), (pages.v, v))]
        say(f"[page store] {dtype} {Hkv} x {d}, page {ps}, {n} of {n_src} rows, fused {fused}")
        A.page_store(pages, k, v, ints(slots), None if keep is None else ints(keep))
        assert np.array_equal(_bits(pages.k), want[0]) and np.array_equal(_bits(pages.v), want[1])


def test_store_behind_4_gib():
    # places whose byte offset passes 32 bits, in a pool of 5.4 GB a tensor
    pages = A.Pages.empty(21000, 8, 128, 128)
    rows = torch.randn(6, 8, 128, device="cuda").to(torch.bfloat16)
    at = [0, 16500 * 128 + 5, 16384 * 128, 20999 * 128 + 127, 8191 * 128 + 127, 8192 * 128]
    say("[page store] slots behind 4 GiB")
    A.page_store(pages, rows, rows * 2, ints(at))
    for r, s in enumerate(at):
        assert torch.equal(pages.k[s // 128, :, s % 128], rows[r])
        assert torch.equal(pages.v[s // 128, :, s % 128], rows[r] * 2)


def test_store_of_more_rows_than_one_axis_has():
    # a block per row: 2^24 + 100 of them, few with a place
    n = (1 << 24) + 100
    pages = A.Pages(*(torch.zeros(2, 16, 16, 128, dtype=torch.bfloat16, device="cuda") for _ in "kv"))
    rows = torch.randn(3, 16, 128, device="cuda").to(torch.bfloat16)
    slots = torch.full((n,), -1, dtype=torch.int32, device="cuda")
    keep = torch.zeros(n, dtype=torch.int32, device="cuda")
    at = [(0, 5, 1), ((1 << 20) + 3, 0, 2), (1 << 24, 31, 0), (n - 1, 16, 2)]   # row, slot, source
    for r, s, j in at:
        slots[r], keep[r] = s, j
    say(f"[page store] {n} rows")
    A.page_store(pages, rows, -rows, slots, keep)
    want = torch.zeros_like(pages.k)
    for _, s, j in at:
        want[s // 16, :, s % 16] = rows[j]
    assert torch.equal(pages.k, want) and torch.equal(pages.v, -want)


def test_binding_refuses_bad_tensors():
    pages = A.Pages.empty(4, 2, 16, 64)
    rows = torch.zeros(6, 2, 64, dtype=torch.bfloat16, device="cuda")
    slots = ints(range(6))
    with pytest.raises(TypeError, match="float32"):
        A.page_store(pages, rows.float(), rows.float(), slots)
    with pytest.raises(ValueError, match="rows"):
        A.page_store(pages, rows[:5], rows[:5], slots)
    with pytest.raises(ValueError, match="needed"):
        A.page_store(pages, rows[:, :1], rows[:, :1], slots)
    with pytest.raises(ValueError, match="contiguous"):
        t = torch.zeros(6, 64, 2, dtype=torch.bfloat16, device="cuda").transpose(1, 2)
        A.page_store(pages, t, t, slots)
    with pytest.raises(ValueError, match="overlap"):
        t = rows[:1].expand(6, 2, 64)
        A.page_store(pages, t, t, slots)
    with pytest.raises(ValueError, match="aligned"):
        t = torch.zeros(6 * 132 + 1, dtype=torch.bfloat16, device="cuda")[1:].view(6, 132)[:, :128].unflatten(1, (2, 64))
        A.page_store(pages, t, t, slots)
    with pytest.raises(TypeError, match="int32"):
        A.page_store(pages, rows, rows, slots.long())
    with pytest.raises(ValueError, match="at least"):
        A.page_tables(16, ints([0, 1]), ints([0, 0]), ints([1]), ints([1]), ints([[0], [0]]), 2)
    x = ints([0, 0])
    with pytest.raises(A.AvtpError):                             # outputs must not alias inputs
        A.prepare_page_tables(16, ints([0, 1, 2]), x, ints([1, 2]), ints([2]), ints([[0], [0]]), ints([0, 0]), x,
                              ints([0]))()
    with pytest.raises(A.AvtpError):
        A.page_trim(24, x, ints([1, 2]), ints([[0], [0]]), ints([1, 2]), ints([0]))
