"""GPU tests of what goes on around trees of drafted tokens in the pages: kept tokens moved together, forks and copies, free pages; and the operators together,
as a serving loop uses them."""
import numpy as np
import pytest
import torch

from paged_util import new_tables, rows_of, store
from test_gpu_paged import BF, DEV, F32, bits, ints, randn
from tree_util import ancestors, check_tree, compact, fork, free_pages, random_parents
from paper_2605_19726_amd import binding as bd

pytestmark = pytest.mark.gpu


def filled(pages, heads, page, d, dtype, layout, seed):
    x = store(pages, heads, page, d, dtype, layout, DEV)
    x.copy_(randn((pages, heads, page, d), seed, dtype))
    return x


def by_slot(x):
    return x.permute(0, 2, 1, 3).reshape(-1, x.shape[1], x.shape[3]).clone()


def moved(x, moves):
    """What a cache holds, by slot, after all rows were read and then written."""
    rows = by_slot(x)
    if moves:
        a, b = (torch.tensor(t, device=DEV) for t in zip(*moves))
        rows[b] = rows[a]
    return rows


# ---------------------------------------------------------------- kept tokens
def _compact_check(dtype, d, heads, page, layout, start, kept, seed, stride=0, table_edit=None, counts=None):
    """kept[i]: list of kept tokens behind start[i]."""
    rng = np.random.default_rng(seed)
    n = len(start)
    lens = [max(s, 0) + (max(k) + 1 if len(k) else 0) for s, k in zip(start, kept)]
    pages = sum(-(-x // page) for x in lens) + 2
    table = new_tables(lens, page, pages, rng)
    if table_edit:
        table_edit(table)
    most = max([1] + [len(k) for k in kept])
    keep = np.full((n, most + stride), -9, dtype=np.int32)
    for i, k in enumerate(kept):
        keep[i, :len(k)] = k
    count = [len(k) for k in kept] if counts is None else counts
    k, v = (filled(pages, heads, page, d, dtype, x, seed + i) for i, x in enumerate((layout, "head")))
    k[-1], v[-1] = float("nan"), float("inf")
    moves = compact(table, start, keep[:, :most], count, page, pages)
    want = [moved(x, moves) for x in (k, v)]
    bd.basa_cache_compact(bd.PagedCache(k, v), ints(table), ints(start), ints(keep)[:, :most], ints(count))
    for x, w in zip((k, v), want):
        assert torch.equal(bits(by_slot(x)), bits(w))


def subset(n, share, rng):
    return np.sort(rng.permutation(n)[:int(round(n * share))]).tolist()


@pytest.mark.parametrize("dtype,d", [(BF, 128), (BF, 64), (F32, 128), (F32, 64)])
@pytest.mark.parametrize("heads,page,layout", [(1, 1, "head"), (8, 16, "head"), (8, 64, "token"), (5, 100, "token"), (33, 20, "head")])
def test_kept_tokens_of_steps_are_moved_together(dtype, d, heads, page, layout):
    rng = np.random.default_rng(heads)
    start = [0, 700, 15, 16, 17, 333, 90]
    kept = [[0, 1, 2], [1, 2, 3, 9], [], [15], subset(40, 0.3, rng), subset(200, 0.9, rng), list(range(1, 30))]
    _compact_check(dtype, d, heads, page, layout, start, kept, 3, stride=3)


@pytest.mark.parametrize("dtype,d,heads,page,layout", [(BF, 128, 8, 16, "token"), (BF, 64, 2, 100, "head"), (F32, 64, 4, 64, "head"), (F32, 128, 3, 1, "token")])
@pytest.mark.parametrize("share", [0.05, 0.5, 0.97])
def test_long_contexts_of_which_tokens_are_dropped(dtype, d, heads, page, layout, share):
    rng = np.random.default_rng(int(share * 100))
    sizes = [5000, 1, 0, 2049, 300, 257]
    kept = [subset(n, share, rng) for n in sizes]
    kept[4] = list(range(43, 300))                              # all of them one way
    kept[5] = list(range(256)) + [256]                          # none
    _compact_check(dtype, d, heads, page, layout, [0, 0, 4, 3, 0, 0], kept, 7)


# both sides of where lists are long: 48 moves and one for every 48 lines of 128 bytes; of 200 sequences short lists go past a block of moves
@pytest.mark.parametrize("dtype,d,n,most", [(BF, 64, 1, 48), (BF, 64, 1, 49), (BF, 128, 8, 53), (BF, 128, 8, 54), (BF, 128, 64, 90), (BF, 128, 64, 91), (F32, 128, 200, 314),
                                            (F32, 128, 200, 315), (BF, 128, 16, 600), (BF, 128, 15, 600)])
def test_short_and_long_lists(dtype, d, n, most):
    rng = np.random.default_rng(n + most)
    kept = [subset(int(rng.integers(1, 2 * most)), 0.5, rng) for _ in range(n)]
    kept[n // 2] = subset(most + most // 3, 1.0, rng)[most // 3:][:most]
    _compact_check(dtype, d, 8, 16, "head", rng.integers(0, 40, n).tolist(), kept, n)


def test_one_long_context():
    rng = np.random.default_rng(1)
    for share in (0.3, 0.999):
        _compact_check(BF, 128, 8, 64, "head", [0], [subset(40000, share, rng)], 5)


def test_kept_tokens_without_a_page_and_lists_that_are_none_stay_in_bounds():
    def edit(table):
        table[0, 1], table[1, 0] = -1, 2 ** 30
    _compact_check(BF, 64, 2, 16, "head", [0, 8], [list(range(5, 60)), list(range(1, 40))], 4, table_edit=edit)
    _compact_check(BF, 64, 2, 16, "head", [0, 8, 3], [[5, 6], [7, 9], [1, 2]], 4, counts=[-4, 2 ** 31 - 1, 1])
    _compact_check(BF, 64, 2, 16, "head", [-5, 8], [[5, 6], [7, 9]], 4)
    # descending, repeated, far and negative entries: no telling which rows move, but none outside the cache, and none of other sequences
    k, v = (filled(8, 2, 16, 64, BF, "head", i) for i in range(2))
    before = by_slot(k)
    table = ints([[0, 1, 2], [3, 4, 5]])
    keep = ints([[40, 9, 9, -7, 2 ** 31 - 1, 3, -2 ** 31, 47], [0] * 8])
    for start in ([0, 0], [2 ** 31 - 1, 5], [40, -2 ** 31]):
        bd.basa_cache_compact(bd.PagedCache(k, v), table, ints(start), keep, ints([8, 8]))
    torch.cuda.synchronize()
    assert torch.equal(bits(by_slot(k)[48:]), bits(before[48:]))
    bd.basa_cache_compact(bd.PagedCache(k, v), table[:0], ints([]), keep[:0], ints([]))
    bd.basa_cache_compact(bd.PagedCache(k, v), table, ints([0, 0]), keep[:, :0], ints([8, 8]))


# short lists and long ones; lengths below zero, within the kept tokens, and beyond the row
@pytest.mark.parametrize("dtype,d", [(BF, 128), (F32, 64)])
@pytest.mark.parametrize("size", [30, 700])
def test_kept_tokens_within_what_a_sequence_holds(dtype, d, size):
    rng = np.random.default_rng(size)
    n, page, pages = 9, 16, 9 * (size + 40) // 16 + 12
    start = rng.integers(0, 30, n)
    table = new_tables([size + 40] * n, page, pages, rng)
    most = size * 2 // 3
    keep = np.array([np.sort(rng.permutation(size)[:most]) for _ in range(n)], dtype=np.int32)
    keep[4] = np.arange(1, most + 1)
    lens = start + rng.integers(0, size, n)
    lens[0], lens[1], lens[2], lens[3], lens[5] = -7, 0, start[2], 2 ** 31 - 1, start[5] + keep[5][most // 2]
    k, v = (filled(pages, 2, page, d, dtype, x, i) for i, x in enumerate(("head", "token")))
    within = np.where(start[:, None] + keep < lens[:, None], keep, -1)                   # an entry that is none moves nothing
    moves = compact(table, start, within, [most] * n, page, pages)
    assert len(moves) > most
    want = [moved(x, moves) for x in (k, v)]
    bd.basa_cache_compact(bd.PagedCache(k, v), ints(table), ints(start), ints(keep), ints([most] * n), ints(lens))
    for x, w in zip((k, v), want):
        assert torch.equal(bits(by_slot(x)), bits(w))


@pytest.mark.parametrize("taken", [20, 150])
def test_a_sequence_that_was_not_served_keeps_nothing_and_writes_into_no_page_of_others(taken):
    """Two sequences draft; the first is cut back, and its row keeps the ids of the pages behind its length.  They go to the second.  When pages run short
    the first is not served: none of its drafted tokens may move, least of all within the second's pages."""
    page, pages, heads, d = 16, 24, 2, 64
    k, v = (filled(pages, heads, page, d, BF, "head", i) for i in range(2))
    cache = bd.PagedCache(k, v)
    table = torch.full((2, 24), -1, dtype=torch.int32, device=DEV)
    free, count = bd.basa_page_free(table, ints([0, 0]), page, pages)
    step = bd.basa_page_tables(ints([0, 0]), ints([20 + taken, 10]), table, free[:int(count)], page, tokens=30 + taken)
    assert step.lens.tolist() == [20 + taken, 10]
    lens = ints([20, 10])                                            # the first is cut back
    stale = table[0, 2:-(-(20 + taken) // page)].tolist()
    free, count = bd.basa_page_free(table, lens, page, pages)
    need = pages * page - 32                                         # all that there is goes to the second
    step = bd.basa_page_tables(lens, ints([0, need - 10]), table, free[:int(count)], page, tokens=need)
    assert step.lens.tolist() == [20, need] and set(stale) & set(table[1].tolist())
    lens = step.lens
    free, count = bd.basa_page_free(table, lens, page, pages)
    assert int(count) == 0
    step = bd.basa_page_tables(lens, ints([taken, 0]), table, free[:0], page, tokens=taken)
    assert step.lens.tolist() == [20, need] and step.pages.tolist()[0] == 0 and (step.slots == -1).all()
    before = [x.clone() for x in (k, v)]
    keep = torch.arange(1, taken, 2, dtype=torch.int32, device=DEV).expand(2, -1).contiguous()
    kept = ints([keep.shape[1], 0])
    bd.basa_cache_compact(cache, table, lens, keep, kept, step.lens)
    for x, b in zip((k, v), before):
        assert torch.equal(bits(x), bits(b))
    assert torch.minimum(lens + kept, step.lens).tolist() == [20, need]


def test_lists_that_are_none_leave_other_sequences_alone_in_k_and_v():
    """Descending, repeated, far and negative entries, of short lists and of long ones: the pages of no sequence, and of one without entries, hold what they held."""
    rng = np.random.default_rng(7)
    for most in (8, 300):
        k, v = (filled(60, 2, 16, 64, BF, x, i) for i, x in enumerate(("head", "token")))
        before = [by_slot(x) for x in (k, v)]
        table = ints(np.arange(60).reshape(3, 20))[:2]
        keep = rng.choice([-2 ** 31, -7, 0, 3, 9, 40, 319, 320, 2 ** 31 - 1], (2, most))
        keep[:, most // 2:] = rng.integers(0, 400, (2, most - most // 2))
        for start in ([0, 0], [2 ** 31 - 1, 5], [300, -2 ** 31]):
            for lens in (None, ints([320, 320]), ints([2 ** 31 - 1, -2 ** 31])):
                bd.basa_cache_compact(bd.PagedCache(k, v), table, ints(start), ints(keep), ints([most, 0]), lens)
        for x, b in zip((k, v), before):
            assert torch.equal(bits(by_slot(x)[320:]), bits(b[320:]))


def test_lists_that_are_longer_than_a_row():
    """As many entries as a call can name, all of them counted: those that a row has room for matter, and no others are looked at."""
    page, pages, width = 16, 40, 20
    keep = torch.empty((1, 2 ** 31 - 1), dtype=torch.int32, device=DEV)
    room, rng = width * page, np.random.default_rng(3)
    table = rng.permutation(pages)[:width].reshape(1, width).astype(np.int32)
    first = np.sort(rng.permutation(room)[:200])
    first = np.concatenate([first, np.arange(room - 200) + room]).astype(np.int32)
    keep[0, :room] = ints(first)
    for start in (0, 7):
        k, v = (filled(pages, 2, page, 64, BF, x, i) for i, x in enumerate(("head", "token")))
        moves = compact(table, [start], first[None], [room], page, pages)
        assert len(moves) > 100
        want = [moved(x, moves) for x in (k, v)]
        bd.basa_cache_compact(bd.PagedCache(k, v), ints(table), ints([start]), keep, ints([2 ** 31 - 1]))
        for x, w in zip((k, v), want):
            assert torch.equal(bits(by_slot(x)), bits(w))


# ---------------------------------------------------------------- forks and copies
def _fork_check(lens, parents, n_free, page, seed, width=None):
    rng = np.random.default_rng(seed)
    real = [max(x, 0) for x in lens]
    pages = sum(-(-x // page) for x in real) + n_free + 2
    table = new_tables(real, page, pages, rng, width)
    free = np.setdiff1d(np.arange(pages), table.reshape(-1))
    free = rng.permutation(free)[:n_free]
    rows, new_lens, copies, given = fork(table, lens, parents, free, page)
    out = bd.PageFork(len(parents), table.shape[1], DEV)
    for t in (out.table, out.lens, out.copies, out.pages):
        t.fill_(-77)
    assert bd.basa_page_fork(ints(table.reshape(len(lens), -1)), ints(lens), ints(parents), ints(free), page, out=out) is out
    want = np.full(out.table.shape, -77)
    for i, r in enumerate(rows):
        want[i, :len(r)] = r
    assert np.array_equal(out.table.cpu().numpy(), want)
    assert out.lens.tolist() == new_lens and out.copies.tolist() == copies and out.pages.tolist() == given
    return given


@pytest.mark.parametrize("page", [1, 16, 20, 128])
@pytest.mark.parametrize("n,m", [(1, 1), (1, 9), (8, 64), (300, 257), (7, 1000)])
def test_fork(page, n, m):
    rng = np.random.default_rng(n + page)
    lens = rng.integers(0, 400, n)
    lens[rng.random(n) < 0.2] = page * 2
    parents = rng.integers(0, n, m)
    asked = _fork_check(lens.tolist(), parents.tolist(), m, page, 1)[1]
    _fork_check(lens.tolist(), parents.tolist(), asked, page, 2)                       # exactly enough
    _fork_check(lens.tolist(), parents.tolist(), asked // 2, page, 3)                  # pages run short
    parents[rng.random(m) < 0.2] = rng.choice([-1, n, 2 ** 31 - 1, -2 ** 31])
    _fork_check(lens.tolist(), parents.tolist(), m, page, 4, width=-(-400 // page) + 3)


def test_fork_of_the_most_sequences_of_none_and_of_lengths_beyond_their_row():
    rng = np.random.default_rng(0)
    _fork_check(rng.integers(0, 60, 8192).tolist(), rng.integers(0, 8192, 8192).tolist(), 8192, 16, 1)
    out = bd.basa_page_fork(ints(np.zeros((0, 4))), ints([]), ints([0, 1]), ints([]), 16)
    assert out.lens.tolist() == [0, 0] and out.copies.tolist() == [[-1, -1, 0]] * 2 and out.pages.tolist() == [0, 0]
    out = bd.basa_page_fork(ints([[1, 2]]), ints([20]), ints([]), ints([5]), 16)
    assert out.pages.tolist() == [0, 0]
    out = bd.basa_page_fork(ints([[1, 2], [3, 4]]), ints([10 ** 9, -4]), ints([0, 0, 1]), ints([5]), 16)
    assert out.lens.tolist() == [32, 32, 0] and out.table[:2].tolist() == [[1, 2], [1, 2]] and out.pages.tolist() == [0, 0]


@pytest.mark.parametrize("dtype,d", [(BF, 128), (BF, 64), (F32, 128), (F32, 64)])
@pytest.mark.parametrize("heads,page,layout", [(1, 1, "head"), (8, 64, "head"), (8, 16, "token"), (5, 100, "token"), (33, 20, "head"), (2, 300, "head")])
def test_copies_of_pages(dtype, d, heads, page, layout):
    rng = np.random.default_rng(page)
    pages = 40
    k, v = (filled(pages, heads, page, d, dtype, x, 3 + i) for i, x in enumerate((layout, "head")))
    ids = rng.permutation(pages)
    copies = [[int(ids[i % 7]), int(ids[10 + i]), int(rng.integers(1, page + 1))] for i in range(20)]
    copies[0][2], copies[1][2], copies[2][2], copies[3][2] = page, 10 ** 9, 0, -5
    copies += [[-1, -1, 0], [-1, int(ids[35]), page], [int(ids[0]), -1, page], [pages, int(ids[36]), page], [int(ids[0]), 2 ** 31 - 1, page], [int(ids[1]), int(ids[1]), page]]
    moves = [(a * page + t, b * page + t) for a, b, n in copies if 0 <= a < pages and 0 <= b < pages for t in range(min(max(n, 0), page))]
    want = [moved(x, moves) for x in (k, v)]
    bd.basa_cache_copy(bd.PagedCache(k, v), ints(copies))
    for x, w in zip((k, v), want):
        assert torch.equal(bits(by_slot(x)), bits(w))
    bd.basa_cache_copy(bd.PagedCache(k, v), ints(np.zeros((0, 3))))


def test_copies_of_the_largest_pages():
    """Pages of nearly 2^31 pieces of 16 bytes, so that a lane's next one lies beyond that.  (Of heads and tokens side by side on the same memory: a page is a strip of it.)"""
    heads, page, d = 65472, 1025, 128
    assert 0 < 2 ** 31 - page * heads * 32 < 64 * 256
    strip = (heads + page) * d
    k, v = (randn((3 * strip,), 3 + i, F32).as_strided((3, heads, page, d), (strip, d, d, 1)) for i in range(2))
    before = [torch.as_strided(x, (3 * strip,), (1,)).clone() for x in (k, v)]
    bd.basa_cache_copy(bd.PagedCache(k, v), ints([[0, 2, 3], [1, 1, page], [3, 0, 5]]))
    for x, b in zip((k, v), before):
        want = b.clone()
        want[2 * strip:2 * strip + (heads + 2) * d] = b[:(heads + 2) * d]
        assert torch.equal(torch.as_strided(x, (3 * strip,), (1,)), want)


# pages, or heads, more than 4 GiB apart in all
@pytest.mark.parametrize("strides", [(2 ** 28 + 8, 1000, 2 ** 15 + 24), (2 ** 13, 2 ** 31 + 64, 136)])
def test_moves_and_copies_of_pages_beyond_32_bits(strides):
    rng = np.random.default_rng(5)
    small = [filled(20, 3, 16, 64, BF, "head", i) for i in range(2)]
    size = sum((n - 1) * x for n, x in zip((20, 3, 16), strides)) + 64
    k, v = (torch.empty(size, dtype=BF, device=DEV).as_strided(x.shape, (*strides, 1)).copy_(x) for x in small)
    table = rng.permutation(20)[:18].reshape(2, 9).astype(np.int32)
    for most in (20, 100):
        keep = np.array([np.sort(rng.permutation(140)[:most]) for _ in range(2)], dtype=np.int32)
        moves = compact(table, [2, 0], keep, [most, most - 1], 16, 20)
        small = [moved(x, moves).view(20, 16, 3, 64).permute(0, 2, 1, 3) for x in small]
        bd.basa_cache_compact(bd.PagedCache(k, v), ints(table), ints([2, 0]), ints(keep), ints([most, most - 1]))
        assert all(torch.equal(bits(x.contiguous()), bits(y.contiguous())) for x, y in zip(small, (k, v)))
    bd.basa_cache_copy(bd.PagedCache(k, v), ints([[0, 19, 7], [18, 1, 16]]))
    for x in small:
        x[19, :, :7], x[1] = x[0, :, :7].clone(), x[18].clone()
    assert all(torch.equal(bits(x.contiguous()), bits(y.contiguous())) for x, y in zip(small, (k, v)))


# ---------------------------------------------------------------- free pages
def _free_check(table, lens, page, pages):
    want = free_pages(table, lens, page, pages)
    out = torch.full((pages,), -7, dtype=torch.int32, device=DEV), torch.full((1,), -7, dtype=torch.int32, device=DEV)
    free, count = bd.basa_page_free(ints(table), ints(lens), page, pages, out=out)
    assert int(count) == len(want)
    assert np.array_equal(free[:len(want)].cpu().numpy(), np.array(want, dtype=np.int32))
    assert (free[len(want):] == -7).all()
    return len(want)


@pytest.mark.parametrize("pages", [1, 31, 32, 33, 64, 1000, 5000])
@pytest.mark.parametrize("n,width", [(1, 1), (3, 40), (64, 9), (700, 3)])
def test_free(pages, n, width):
    rng = np.random.default_rng(pages + n)
    table = rng.integers(0, pages, (n, width)).astype(np.int32)                        # shared at random
    _free_check(table, rng.integers(0, 16 * width + 1, n), 16, pages)
    table[rng.random((n, width)) < 0.3] = rng.choice([-1, pages, 2 ** 31 - 1, -2 ** 31])
    _free_check(table, rng.integers(0, 16 * width + 1, n), 16, pages)
    _free_check(table, [0] * n, 16, pages)
    _free_check(table, [-3] + [2 ** 31 - 1] * (n - 1), 16, pages)


@pytest.mark.parametrize("n,width,page,pages", [(2000, 100, 16, 100000), (3, 30000, 1, 400001), (5000, 20, 20, 300000), (1, 1, 16, 2 ** 20 + 5), (100, 700, 64, 70000)])
def test_free_of_large_pools(n, width, page, pages):
    rng = np.random.default_rng(n)
    table = rng.permutation(max(pages, n * width))[:n * width].reshape(n, width).astype(np.int32)
    _free_check(table, rng.integers(0, page * width + 1, n), page, pages)


# rows from one entry to more than a wave has lanes, on both sides of one workgroup
@pytest.mark.parametrize("n,width", [(1, 1), (17, 1), (1000, 2), (5000, 1), (1500, 3), (1025, 32), (500, 33), (512, 63), (513, 64), (255, 65), (257, 65), (300, 129), (2, 9000)])
def test_free_of_narrow_and_wide_rows(n, width):
    rng = np.random.default_rng(n + width)
    pages = n * width + 77
    table = rng.integers(-2, pages + 2, (n, width)).astype(np.int32)                  # none, others' pages, pages twice
    _free_check(table, rng.integers(-1, 16 * width + 20, n), 16, pages)
    wide = np.full((n, width + 3), 5, dtype=np.int32)
    wide[:, :width] = table
    lens = rng.integers(0, 16 * width + 1, n)
    free, count = bd.basa_page_free(ints(wide)[:, :width], ints(lens), 16, pages)
    want = free_pages(table, lens, 16, pages)
    assert int(count) == len(want) and np.array_equal(free[:len(want)].cpu().numpy(), np.array(want, dtype=np.int32))


def test_free_without_sequences():
    for pages in (50, 2 ** 19):
        free, count = bd.basa_page_free(ints(np.zeros((0, 4))), ints([]), 16, pages)
        assert int(count) == pages and torch.equal(free, torch.arange(pages, dtype=torch.int32, device=DEV))


# ---------------------------------------------------------------- together
@pytest.mark.parametrize("dtype,d", [(BF, 128), (F32, 64)])
def test_a_serving_loop_with_drafted_trees_samples_and_freed_pages(dtype, d):
    """Prompts; every one goes on as samples; trees of drafted tokens are attended to, a path of each is kept; sequences end and others begin.  Every sequence's
    tokens are kept beside the cache, and every step's attention is checked on them."""
    hq, hk, page, pages, width = 8, 2, 16, 300, 30
    rng = np.random.default_rng(9)
    k_cache, v_cache = (store(pages, hk, page, d, dtype, "token", DEV) for _ in range(2))
    cache = bd.PagedCache(k_cache, v_cache)
    seed = [100]

    def rows(T):
        seed[0] += 3
        return (randn((T, h, d), seed[0] + i, dtype) for i, h in enumerate((hq, hk, hk)))

    def compare(out, lse, q, held, cu, seen):
        """The attention on a cache of the sequences' own tokens, one page of 512 each."""
        own = [torch.zeros(len(held), hk, 512, d, dtype=dtype, device=DEV) for _ in range(2)]
        for i, kv in enumerate(held):
            for c, x in zip(own, kv):
                c[i, :, :x.shape[0]] = x.transpose(0, 1)
        check_tree(out, lse, q, *own, np.arange(len(held))[:, None], [x[0].shape[0] for x in held], cu, seen)

    # prompts of two sequences into an empty cache, as chains of new tokens
    free, count = bd.basa_page_free(ints(np.zeros((0, width))), ints([]), page, pages)
    lens, add = [0, 0], [37, 100]
    table = torch.full((2, width), -1, dtype=torch.int32, device=DEV)
    step = bd.basa_page_tables(ints(lens), ints(add), table, free[:int(count)], page, tokens=sum(add))
    q, k, v = rows(sum(add))
    out, lse = bd.ba_att_tree(q, k, v, cache, table, step.lens, step.slots, step.cu, want_lse=True)
    held = [(k[:37], v[:37]), (k[37:], v[37:])]
    compare(out, lse, q, held, [0, 37, 137], [None, None])
    # five samples of the first, two of the second
    parents = [0, 1, 0, 0, 1, 0, 0]
    free, count = bd.basa_page_free(table, step.lens, page, pages)
    forked = bd.basa_page_fork(table, step.lens, ints(parents), free[:int(count)], page)
    bd.basa_cache_copy(cache, forked.copies)
    assert forked.pages.tolist() == [5, 5] and forked.lens.tolist() == [[37, 100][p] for p in parents]
    table, lens, held = forked.table, forked.lens, [held[p] for p in parents]
    for turn in range(4):
        free, count = bd.basa_page_free(table, lens, page, pages)
        n = len(held)
        add = rng.integers(0, 20, n)
        trees = [random_parents(x, rng) for x in add]
        step = bd.basa_page_tables(lens, ints(add), table, free[:int(count)], page, tokens=int(add.sum()) + 3)
        given, asked = step.pages.tolist()
        assert given == asked
        masks, depths = bd.basa_tree_masks(ints(np.concatenate(trees + [np.zeros(3)])), step.cu, 1)
        q, k, v = rows(int(add.sum()) + 3)
        out, lse = bd.ba_att_tree(q, k, v, cache, table, step.lens, step.slots, step.cu, masks, want_lse=True)
        cu = step.cu.tolist()
        compare(out, lse, q, [tuple(torch.cat([x, y[cu[i]:cu[i + 1]]]) for x, y in zip(held[i], (k, v))) for i in range(n)], cu, [ancestors(t) for t in trees])
        # the path to some token of each tree is kept
        paths = []
        for i, t in enumerate(trees):
            path = [] if len(t) == 0 else np.flatnonzero(ancestors(t)[int(rng.integers(len(t)))]).tolist()
            assert len(path) == 0 or int(depths[cu[i] + path[-1]]) == len(path) - 1
            paths.append(path)
            at = [cu[i] + r for r in path]
            held[i] = tuple(torch.cat([x, y[at]]) for x, y in zip(held[i], (k, v)))
        keep = np.zeros((n, max([1] + [len(p) for p in paths])), dtype=np.int32)
        for i, p in enumerate(paths):
            keep[i, :len(p)] = p
        taken = ints([len(p) for p in paths])
        bd.basa_cache_compact(cache, table, lens, ints(keep), taken)
        lens = lens + taken
        # sequence 1 ends in turn 1, sequence 0 goes on as two in turn 2
        if turn in (1, 2):
            parents = [i for i in range(n) if i != 1] if turn == 1 else [0, 0] + list(range(1, n))
            free, count = bd.basa_page_free(table, lens, page, pages)
            forked = bd.basa_page_fork(table, lens, ints(parents), free[:int(count)], page)
            bd.basa_cache_copy(cache, forked.copies)
            table, lens, held = forked.table, forked.lens, [held[p] for p in parents]
    # single tokens go on from there
    free, count = bd.basa_page_free(table, lens, page, pages)
    n = len(held)
    step = bd.basa_page_tables(lens, ints([1] * n), table, free[:int(count)], page, tokens=n)
    q, k, v = rows(n)
    out, lse = bd.ba_att_decode(q, k, v, cache, table, step.lens, step.slots, want_lse=True)
    compare(out, lse, q, [tuple(torch.cat([x, y[i:i + 1]]) for x, y in zip(held[i], (k, v))) for i in range(n)], list(range(n + 1)), [None] * n)
    # everyone ends
    free, count = bd.basa_page_free(table, torch.zeros_like(lens), page, pages)
    assert int(count) == pages


@pytest.mark.parametrize("back", [[100, 40], [33, 40], [100, 48], [48, 0], [40, 100, 40]])
def test_sequences_that_are_cut_back_into_pages_of_a_fork_go_on_with_copies(back):
    """Samples of one prompt share its whole pages; cut back to `back` tokens, some of them within those, they get new tokens.  Everyone's tokens are their own."""
    dtype, d, hq, hk, page, pages, prompt, n = BF, 64, 4, 2, 16, 60, 100, len(back)
    k_cache, v_cache = (store(pages, hk, page, d, dtype, "head", DEV) for _ in range(2))
    cache = bd.PagedCache(k_cache, v_cache)
    seed = [0]

    def rows(T):
        seed[0] += 3
        return (randn((T, h, d), seed[0] + i, dtype) for i, h in enumerate((hq, hk, hk)))

    def grow(table, lens, add, held):
        free, count = bd.basa_page_free(table, lens, page, pages)
        step = bd.basa_page_tables(lens, ints(add), table, free[:int(count)], page, tokens=sum(add))
        given, asked = step.pages.tolist()
        assert given == asked
        q, k, v = rows(sum(add))
        out, lse = bd.ba_att_tree(q, k, v, cache, table, step.lens, step.slots, step.cu, want_lse=True)
        cu = step.cu.tolist()
        held = [tuple(torch.cat([x, y[cu[i]:cu[i + 1]]]) for x, y in zip(held[i], (k, v))) for i in range(len(held))]
        own = [torch.zeros(len(held), hk, 512, d, dtype=dtype, device=DEV) for _ in range(2)]
        for i, kv in enumerate(held):
            for c, x in zip(own, kv):
                c[i, :, :x.shape[0]] = x.transpose(0, 1)
        check_tree(out, lse, q, *own, np.arange(len(held))[:, None], step.lens.tolist(), cu, [None] * len(held))
        return step.lens, held

    none = torch.empty(0, hk, d, dtype=dtype, device=DEV)
    table = torch.full((1, 20), -1, dtype=torch.int32, device=DEV)
    lens, held = grow(table, ints([0]), [prompt], [(none, none)])

    def fork(table, lens, parents, held):
        free, count = bd.basa_page_free(table, lens, page, pages)
        f = bd.basa_page_fork(table, lens, ints(parents), free[:int(count)], page)
        bd.basa_cache_copy(cache, f.copies)
        given, asked = f.pages.tolist()
        assert given == asked
        return f.table, f.lens, [held[p] for p in parents]
    table, lens, held = fork(table, lens, [0] * n, held)
    lens, held = grow(table, lens, [5 + i for i in range(n)], held)
    lens, held = ints(back), [tuple(x[:b] for x in kv) for b, kv in zip(back, held)]
    # within the whole pages of the prompt and not at the end of one: named twice, the first of the two is dropped
    parents = [i for i, b in enumerate(back) for _ in range(1 + (b < prompt // page * page and b % page > 0))]
    table, lens, held = fork(table, lens, parents, held)
    left = [j for j, p in enumerate(parents) if p not in parents[j + 1:]]
    table, lens, held = table[left].contiguous(), lens[left].contiguous(), [held[j] for j in left]
    for add in ([1] * n, [3, 30, 17][:n], [20] * n):
        lens, held = grow(table, lens, add, held)
    assert lens.tolist() == [len(x[0]) for x in held]


def test_a_captured_step_of_all_operators():
    hq, hk, d, page, pages, width, n = 8, 2, 64, 16, 200, 20, 3
    k_cache, v_cache = (filled(pages, hk, page, d, BF, "head", i) for i in range(2))
    cache = bd.PagedCache(k_cache, v_cache)
    rng = np.random.default_rng(3)
    lens0 = [40, 133, 7]
    table0 = new_tables(lens0, page, 60, rng, width)
    table, lens, add, T = ints(table0), ints(lens0), ints([9, 9, 9]), 27
    parents, keep, taken = ints(np.concatenate([random_parents(9, rng) for _ in range(n)])), ints([[0, 2, 5], [1, 3, 4], [2, 6, 8]]), ints([3, 3, 3])
    q, k, v = (randn((T, h, d), h, BF) for h in (hq, hk, hk))
    q2 = q.clone()
    forks, free_out = bd.PageFork(5, width, DEV), (torch.zeros(pages, dtype=torch.int32, device=DEV), torch.zeros(1, dtype=torch.int32, device=DEV))
    forks.table.zero_()

    def step():
        free, count = bd.basa_page_free(table, lens, page, pages, out=free_out)
        s = bd.basa_page_tables(lens, add, table, free[:20], page, tokens=T)
        masks, depths = bd.basa_tree_masks(parents, s.cu, 1)
        out, lse = bd.ba_att_tree(q, k, v, cache, table, s.lens, s.slots, s.cu, masks, want_lse=True)
        bd.basa_cache_compact(cache, table, lens, keep, taken)
        lens.add_(taken)
        f = bd.basa_page_fork(table, lens, ints_of_parents, free[20:40], page, out=forks)
        bd.basa_cache_copy(cache, f.copies)
        return out, lse, depths, f.table, f.lens, f.copies

    ints_of_parents = ints([0, 0, 1, 2, 1])
    state = (table, lens, k_cache, v_cache, forks.table)
    start = [x.clone() for x in state]

    def restore():
        for x, y in zip(state, start):
            x.copy_(y)
    step()
    restore()
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        got = step()
    restore()
    eager = []
    for turn in range(4):
        q.copy_(q2 * (turn + 1))
        eager.append([x.clone() for x in step()] + [x.clone() for x in state] + [free_out[1].clone()])
    restore()
    for turn in range(4):
        q.copy_(q2 * (turn + 1))
        g.replay()
        torch.cuda.synchronize()
        for a, b in zip(eager[turn], list(got) + list(state) + [free_out[1]]):
            assert torch.equal(a if not a.is_floating_point() else bits(a), b if not b.is_floating_point() else bits(b)), turn
