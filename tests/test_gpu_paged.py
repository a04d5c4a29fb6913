"""GPU tests of the paged key-value cache and the single-token attention over it, against the plain statements of paged_util.py: whole
numbers and copies bit for bit, attention within the tolerance derived there."""
import numpy as np
import pytest
import torch

from paged_util import HALF_STEP, attention64, check_decode, decode_tolerance, new_tables, page_tables, rows_of, store
from paper_2605_19726_amd import binding as bd

pytestmark = pytest.mark.gpu
DEV = torch.device("cuda:0")
BF, F32 = torch.bfloat16, torch.float32


def ints(x, dtype=torch.int32):
    return torch.tensor(np.asarray(x), dtype=dtype, device=DEV)


def randn(shape, seed, dtype, scale=1.0):
    g = torch.Generator(device=DEV).manual_seed(seed)
    return (torch.empty(shape, dtype=F32, device=DEV).normal_(generator=g) * scale).to(dtype)


def bits(x):
    return x.contiguous().view(torch.int32 if x.dtype == F32 else torch.int16)


# ---------------------------------------------------------------- block tables and slot maps
def _tables_check(have, add, page, width, n_free, n_slots, stride=None, seed=0, bad_entry=False):
    rng = np.random.default_rng(seed)
    n = len(have)
    held = [-(-max(h, 0) // page) for h in have]
    ids = rng.permutation(sum(held) + n_free + 5).astype(np.int32)
    table = np.full((n, stride or width), -7, dtype=np.int32)
    at = 0
    for i, k in enumerate(held):
        k = min(k, width)
        table[i, :k] = ids[at:at + k]
        at += k
        if bad_entry and i % 3 == 0 and k:
            table[i, k - 1] = -1
    free = ids[at:at + n_free]
    want = page_tables(have, add, table[:, :width], free, page, n_slots)
    tab = ints(table.reshape(n, stride or width))
    out = bd.PageTables(n, n_slots, DEV)
    for t in (out.slots, out.lens, out.cu, out.pages):
        t.fill_(-99)
    got = bd.basa_page_tables(ints(have), ints(add), tab[:, :width], ints(free), page, n_slots, out=out)
    assert got is out
    after = tab.cpu().numpy()
    assert np.array_equal(after[:, :width], want[0])
    assert (after[:, width:] == -7).all()
    for name, a, b in zip(("slots", "lens", "cu", "pages"), (out.slots, out.lens, out.cu, out.pages), want[1:]):
        assert np.array_equal(a.cpu().numpy(), b), name
    return want


@pytest.mark.parametrize("page", [1, 2, 16, 20, 64, 100, 256])
@pytest.mark.parametrize("n", [1, 3, 64, 255, 257, 1000])
def test_page_tables_random(n, page):
    rng = np.random.default_rng(n * 1000 + page)
    have, add = rng.integers(0, 700, n), rng.integers(0, 40, n)
    add[rng.random(n) < 0.3] = 0
    have[rng.random(n) < 0.2] = 0
    width = -(-740 // page)
    need = sum(-(-(h + a) // page) - -(-h // page) for h, a in zip(have, add))
    total = int(add.sum())
    _tables_check(have, add, page, width, need, total, seed=1)                                    # exactly enough of everything
    _tables_check(have, add, page, width, need + 3, total + 77, stride=width + 5, seed=2)         # room, padded rows behind the last
    _tables_check(have, add, page, width, need // 2, total, seed=3)                               # pages run out
    _tables_check(have, add, page, max(1, width // 2), need, total - total // 3, seed=4, bad_entry=True)   # rows too narrow, slots cut


@pytest.mark.parametrize("have,add,page,width,n_free,n_slots", [
    ([0], [0], 16, 1, 0, 0), ([0], [1], 16, 1, 1, 1), ([0], [1], 16, 1, 0, 1), ([16], [1], 16, 2, 1, 1), ([15], [1], 16, 1, 0, 1),
    ([0], [70000], 16, 5000, 4375, 70000), ([5], [100000], 64, 2000, 1600, 100005), ([0, 0, 0], [0, 0, 0], 16, 3, 4, 9),
    ([-5, 7, 0], [3, -2, 4], 16, 3, 4, 20), ([2 ** 31 - 1, 3], [2 ** 31 - 1, 5], 16, 8, 9, 64), ([2 ** 30] * 3, [2 ** 31 - 1] * 3, 7, 8, 9, 64),
    ([100, 5, 90], [28, 2, 60], 16, 8, 9, 200)])
def test_page_tables_edges(have, add, page, width, n_free, n_slots):
    have_now = [min(h, width * page) if h > width * page else h for h in have]       # (the pages that it holds; more than a row's worth are no pages)
    if have_now != have:
        n = len(have)
        tab, out = ints(np.full((n, width), -7)), bd.PageTables(n, n_slots, DEV)
        bd.basa_page_tables(ints(have), ints(add), tab, ints(np.arange(n_free)), page, n_slots, out=out)
        want = page_tables(have, add, np.full((n, width), -7), np.arange(n_free), page, n_slots)
        for a, b in zip((tab, out.slots, out.lens, out.cu, out.pages), want):
            assert np.array_equal(a.cpu().numpy(), b)
        return
    _tables_check(have, add, page, width, n_free, n_slots)


def test_page_tables_of_the_largest_batch_and_of_none():
    rng = np.random.default_rng(5)
    n = 8192
    have, add = rng.integers(0, 300, n), rng.integers(0, 4, n)
    _tables_check(have, add, 16, 20, 4000, int(add.sum()) + 13)
    out = bd.PageTables(0, 6, DEV)
    bd.basa_page_tables(ints([]), ints([]), ints(np.zeros((0, 4))), ints([3, 4]), 16, 6, out=out)
    assert out.slots.tolist() == [-1] * 6 and out.cu.tolist() == [0] and out.pages.tolist() == [0, 0]


# ---------------------------------------------------------------- rows into the pages and out of them
@pytest.mark.parametrize("dtype,d", [(BF, 128), (BF, 64), (F32, 128), (F32, 64)])
@pytest.mark.parametrize("heads,page,layout,T", [(1, 1, "head", 1), (8, 16, "head", 257), (8, 16, "token", 1000), (5, 100, "token", 333),
                                                 (3, 20, "head", 2049), (33, 64, "token", 70), (16, 256, "head", 5000)])
def test_append_and_gather_are_exact_copies(dtype, d, heads, page, layout, T):
    rng = np.random.default_rng(T)
    pages = -(-T // page) + 4
    k_cache, v_cache = store(pages, heads, page, d, dtype, layout, DEV, 7.0), store(pages, heads, page, d, dtype, "head", DEV, 8.0)
    hq = 2 * heads
    qkv = randn((T, hq + 2 * heads, d), 11, dtype)                          # keys and values as slices of one projection
    k, v = qkv[:, hq:hq + heads], qkv[:, hq + heads:]
    k[T // 2] = float("nan")
    slots = rng.permutation(pages * page)[:T].astype(np.int64)
    off = rng.random(T) < 0.1
    slots[off] = rng.choice([-1, -2 ** 40, pages * page, pages * page + 5, 2 ** 31, 2 ** 40], off.sum())
    bd.basa_cache_append(k, v, ints(slots, torch.int64), bd.PagedCache(k_cache, v_cache))
    rows = torch.from_numpy(slots[~off]).to(DEV)
    for cache, x, fill in ((k_cache, k, 7.0), (v_cache, v, 8.0)):
        want = torch.full((pages * page, heads, d), fill, dtype=dtype, device=DEV)
        want[rows] = x[torch.from_numpy(~off).to(DEV)]
        assert torch.equal(bits(cache.permute(0, 2, 1, 3).reshape(-1, heads, d)), bits(want))
    # and back: four sequences, an empty one and pages that are none among them
    lens = [T // 2, 0, T // 3, 1]
    table = new_tables(lens, page, pages, rng, width=-(-T // page) + 1)
    where = table.copy()
    if table[0, 0] >= 0 and lens[0] > page:
        table[0, 0] = pages
        where[0, 0] = -1
    cu = np.concatenate([[2], 2 + np.cumsum(lens)])
    out = tuple(torch.full((int(cu[-1]) + 3, heads, d), 5.0, dtype=dtype, device=DEV) for _ in range(2))
    bd.basa_cache_gather(bd.PagedCache(k_cache, v_cache), ints(table), ints(cu), int(cu[-1]) + 3, out=out)
    for cache, got in ((k_cache, out[0]), (v_cache, out[1])):
        want = torch.full_like(got, 5.0)
        for i, n in enumerate(lens):
            at, place = rows_of(where[i], n, page)
            x = cache[at.clamp(min=0).to(DEV), :, place.to(DEV)].clone()
            x[(at < 0).to(DEV)] = 0.0
            want[int(cu[i]):int(cu[i]) + n] = x
        assert torch.equal(bits(got), bits(want))


def test_gather_of_offsets_that_do_not_ascend_stays_in_bounds():
    k_cache, v_cache = (store(6, 2, 16, 64, BF, "head", DEV, 1.0) for _ in range(2))
    table = ints(np.arange(6).reshape(2, 3))
    for cu in ([0, 90, 40], [50, 20, 90], [-5, 10, 30], [0, 2 ** 31 - 1, 2 ** 31 - 1], [-2 ** 31, 0, 60]):
        k, v = bd.basa_cache_gather(bd.PagedCache(k_cache, v_cache), table, ints(cu), 64)
        torch.cuda.synchronize()
        assert k.shape == (64, 2, 64) and v.shape == k.shape


def test_no_rows_is_no_work():
    cache = bd.PagedCache(*(store(2, 2, 16, 64, BF, "head", DEV, 1.0) for _ in range(2)))
    none = torch.empty(0, 2, 64, dtype=BF, device=DEV)
    bd.basa_cache_append(none, none, ints([], torch.int64), cache)
    k, v = bd.basa_cache_gather(cache, ints(np.zeros((1, 1))), ints([0, 0]), 0)
    assert k.shape == (0, 2, 64) and v.shape == (0, 2, 64)
    assert bd.basa_decode_attn(torch.empty(0, 4, 64, dtype=BF, device=DEV), cache, ints(np.zeros((0, 3))), ints([])).shape == (0, 4, 64)
    assert float(cache.k.float().min()) == 1.0 and float(cache.k.float().max()) == 1.0


# ---------------------------------------------------------------- attention of one token per sequence
def _decode_case(dtype, d, hq, hk, page, lens, seed, layout=("head", "head"), q_scale=2.0, spare=3, width=None):
    """Caches whose rows that no sequence holds are NaN, the table, and queries."""
    rng = np.random.default_rng(seed)
    pages = sum(-(-n // page) for n in lens) + spare
    table = new_tables(lens, page, pages, rng, width)
    k_cache, v_cache = store(pages, hk, page, d, dtype, layout[0], DEV), store(pages, hk, page, d, dtype, layout[1], DEV)
    for i, n in enumerate(lens):
        at, off = (x.to(DEV) for x in rows_of(table[i], n, page))
        k_cache[at, :, off] = randn((n, hk, d), seed * 100 + i, dtype)
        v_cache[at, :, off] = randn((n, hk, d), seed * 100 + 50 + i, dtype)
    return randn((len(lens), hq, d), seed + 7, dtype, q_scale), k_cache, v_cache, table


LENS = [1, 0, 31, 32, 33, 127, 128, 129, 500, 2, 1031]


@pytest.mark.parametrize("dtype,d", [(BF, 128), (BF, 64), (F32, 128), (F32, 64)])
@pytest.mark.parametrize("hq,hk,page,layout", [(4, 4, 16, "head"), (8, 1, 64, "token"), (8, 2, 1, "head"), (10, 2, 20, "token"),
                                               (32, 8, 128, "token"), (14, 2, 100, "head"), (16, 1, 3, "token"), (17, 1, 256, "head"),
                                               (40, 2, 32, "token"), (33, 1, 16, "head"), (66, 2, 50, "token")])
def test_decode_against_64_bits(dtype, d, hq, hk, page, layout):
    q, k, v, table = _decode_case(dtype, d, hq, hk, page, LENS, hq * 10 + page, (layout, "head"))
    out, lse = bd.basa_decode_attn(q, bd.PagedCache(k, v), ints(table), ints(LENS), want_lse=True)
    check_decode(out, lse, q, k, v, table, LENS, f"{dtype} d={d} {hq}/{hk} page={page}")
    assert not out[1].any() and (lse[1] == -float("inf")).all()


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("hq,hk,lens", [(4, 1, [70001]), (8, 2, [20000, 3, 9999]), (2, 2, [40000, 0, 1, 64, 33333]), (20, 1, [30011, 17]),
                                        (48, 1, [5000]), (128, 1, [20000, 5, 2000]), (68, 2, [1500] * 9)])
def test_long_sequences_are_split_and_joined(dtype, hq, hk, lens):
    q, k, v, table = _decode_case(dtype, 128, hq, hk, 64, lens, 3)
    cache = bd.PagedCache(k, v)
    out, lse = bd.basa_decode_attn(q, cache, ints(table), ints(lens), want_lse=True)
    check_decode(out, lse, q, k, v, table, lens)
    again, lse2 = bd.basa_decode_attn(q, cache, ints(table), ints(lens), want_lse=True)
    assert torch.equal(out, again) and torch.equal(lse, lse2)


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("n", [256, 512, 513, 700, 3001])
def test_many_short_sequences(dtype, n):
    lens = np.random.default_rng(n).integers(0, 70, n)
    lens[n // 2] = 3000
    q, k, v, table = _decode_case(dtype, 64, 4, 2, 16, [int(x) for x in lens], 5)
    out, lse = bd.basa_decode_attn(q, bd.PagedCache(k, v), ints(table), ints(lens), want_lse=True)
    some = sorted(set([0, 1, n // 2 - 1, n // 2, n // 2 + 1, n - 1]) | set(np.random.default_rng(1).integers(0, n, 40).tolist()))
    check_decode(out[some], lse[some], q[some], k, v, table[some], lens[some])
    assert torch.isfinite(out).all() and (torch.isfinite(lse).cpu().numpy() == (lens > 0)[:, None]).all()


def test_one_token_gives_its_value_exactly():
    for dtype in (BF, F32):
        q, k, v, table = _decode_case(dtype, 128, 8, 2, 16, [1, 1, 1], 9)
        out = bd.basa_decode_attn(q, bd.PagedCache(k, v), ints(table), ints([1, 1, 1]))
        for i in range(3):
            assert torch.equal(out[i], v[int(table[i, 0]), :, 0].repeat_interleave(4, 0))


@pytest.mark.parametrize("dtype", [BF, F32])
def test_pages_that_are_none_and_lengths_beyond_the_table_carry_no_weight(dtype):
    lens, page = [100, 300, 64, 50, 2000], 16
    q, k, v, table = _decode_case(dtype, 128, 8, 4, page, lens, 21)
    pages, width = k.shape[0], table.shape[1]
    table[0, 2] = -1                        # a hole
    table[1, ::2] = pages                   # every other page is none
    table[2, :4] = [-1, pages, 2 ** 31 - 1, -2 ** 31]        # none at all
    given = [100, 300, 64, -4, 2 ** 31 - 1]                  # below zero: none; beyond the row: all that it has room for
    used = [100, 300, 64, 0, width * page]
    k[torch.from_numpy(table[4, :125]).to(DEV)] = randn((125, 4, page, 128), 5, dtype)
    v[torch.from_numpy(table[4, :125]).to(DEV)] = randn((125, 4, page, 128), 6, dtype)
    out, lse = bd.basa_decode_attn(q, bd.PagedCache(k, v), ints(table), ints(given), want_lse=True)
    check_decode(out, lse, q, k, v, table, used)
    assert not out[2].any() and not out[3].any() and (lse[2:4] == -float("inf")).all()


@pytest.mark.parametrize("dtype", [BF, F32])
def test_infinite_scores(dtype):
    """-inf scores carry no weight, alone they leave the row empty; +inf and NaN scores make it NaN, as the formula does; other heads keep theirs."""
    lens = [90, 40, 70, 200]
    q, k, v, table = _decode_case(dtype, 64, 2, 2, 16, lens, 31)
    q[:, 0, 0] = 1.0
    at = [[x.to(DEV) for x in rows_of(table[i], lens[i], 16)] for i in range(4)]
    k[at[0][0][5:60], 0, at[0][1][5:60], 0] = -float("inf")
    k[at[1][0], 0, at[1][1], 0] = -float("inf")
    k[at[2][0][33], 0, at[2][1][33], 0] = float("inf")
    k[at[3][0][150], 0, at[3][1][150], 3] = float("nan")
    out, lse = bd.basa_decode_attn(q, bd.PagedCache(k, v), ints(table), ints(lens), want_lse=True)
    keep = torch.cat([torch.arange(5), torch.arange(60, 90)])
    ref, ref_lse, size = attention64(q[0, :1], k[at[0][0][keep], :1, at[0][1][keep]], v[at[0][0][keep], :1, at[0][1][keep]])
    tol, tol_lse = decode_tolerance(dtype, 90, 64, float(size[0]), 6.0)
    assert float(((out[0, 0].double() - ref[0]).abs() - HALF_STEP[dtype] * ref[0].abs()).max()) <= tol
    assert abs(float(lse[0, 0]) - float(ref_lse[0])) <= tol_lse
    assert not out[1, 0].any() and float(lse[1, 0]) == -float("inf")
    assert out[2, 0].isnan().all() and out[3, 0].isnan().all()
    for i in range(4):
        check_decode(out[i:i + 1, 1:], lse[i:i + 1, 1:], q[i:i + 1, 1:], k[:, 1:], v[:, 1:], table[i:i + 1], lens[i:i + 1], f"head 1 of {i}")


@pytest.mark.parametrize("dtype", [BF, F32])
def test_large_scores_and_tables_of_the_lowest_value(dtype):
    lens = [300, 90]
    q, k, v, table = _decode_case(dtype, 128, 4, 2, 16, lens, 41, q_scale=200.0)     # a few tokens carry everything, scores of some thousands
    at, off = (x.to(DEV) for x in rows_of(table[1], 90, 16))
    k[at, :, off] = 0.0
    k[at, :, off, 0] = torch.finfo(dtype).min / 4
    q[1] = 0.0
    q[1, :, 0] = 1.0                                                                  # every score the same huge negative number
    out, lse = bd.basa_decode_attn(q, bd.PagedCache(k, v), ints(table), ints(lens), want_lse=True)
    check_decode(out, lse, q, k, v, table, lens)


def test_strided_queries_and_outputs():
    lens = [77, 5, 1000]
    q, k, v, table = _decode_case(BF, 128, 8, 2, 16, lens, 51, ("token", "head"))
    qkv = randn((3, 12, 128), 1, BF)
    qkv[:, :8] = q
    buf = torch.full((3, 10, 136), 9.0, dtype=BF, device=DEV)
    wide = ints(np.concatenate([table, np.full((3, 9), 2 ** 30)], axis=1))
    out = bd.basa_decode_attn(qkv[:, :8], bd.PagedCache(k, v), wide[:, :table.shape[1]], ints(lens), out=buf[:, 1:9, :128])
    assert torch.equal(out, bd.basa_decode_attn(q, bd.PagedCache(k, v), ints(table), ints(lens)))
    buf[:, 1:9, :128] = 9.0
    assert (buf == 9.0).all()


def test_sequences_that_share_pages():
    lens = [200, 200, 130]
    q, k, v, table = _decode_case(BF, 64, 4, 2, 16, lens, 61)
    table[1, :10] = table[0, :10]
    table[2] = table[0]
    out, lse = bd.basa_decode_attn(q, bd.PagedCache(k, v), ints(table), ints(lens), want_lse=True)
    check_decode(out, lse, q, k, v, table, lens)


def test_offsets_beyond_32_bits():
    """A cache of more than 2^32 bytes and 2^31 elements per tensor: pages that lie 2^31 elements and more behind its start."""
    pages, hk, page, d, apart = 5, 2, 16, 128, 600 * 2 ** 20
    k, v = (torch.empty(apart * pages, dtype=BF, device=DEV).as_strided((pages, hk, page, d), (apart, page * d, d, 1)) for _ in range(2))
    T = 60
    rows_k, rows_v = randn((T, hk, d), 1, BF), randn((T, hk, d), 2, BF)
    table = np.array([[4, 0, 3, 1]], dtype=np.int32)
    slots = table[0, np.arange(T) // page].astype(np.int64) * page + np.arange(T) % page
    cache = bd.PagedCache(k, v)
    bd.basa_cache_append(rows_k, rows_v, ints(slots, torch.int64), cache)
    gk, gv = bd.basa_cache_gather(cache, ints(table), ints([0, T]), T)
    assert torch.equal(gk, rows_k) and torch.equal(gv, rows_v)
    q = randn((1, 4, d), 3, BF, 2.0)
    out, lse = bd.basa_decode_attn(q, cache, ints(table), ints([T]), want_lse=True)
    check_decode(out, lse, q, k, v, table, [T])


def test_slots_beyond_32_bits():
    """Pages of 2^20 tokens that all lie at the same place (stride 0): slot numbers pass 2^31 and 2^32."""
    page, hk, d = 2 ** 20, 1, 64
    k, v = (torch.zeros(page, d, dtype=BF, device=DEV).as_strided((5000, hk, page, d), (0, 0, d, 1)) for _ in range(2))
    slots = np.array([2 ** 31 - 1, 2 ** 31, 2 ** 32 + 5, 4999 * page + 77, 5000 * page], dtype=np.int64)
    rows = randn((5, hk, d), 1, BF)
    bd.basa_cache_append(rows, rows, ints(slots, torch.int64), bd.PagedCache(k, v))
    for t, s in enumerate(slots[:4]):
        assert torch.equal(k[0, :, int(s % page)], rows[t])
    assert int((k[0, 0].abs().sum(1) > 0).sum()) == 4


# ---------------------------------------------------------------- streams, graphs, and all of them together
@pytest.mark.parametrize("hq,hk", [(8, 2), (32, 1), (80, 2)])
def test_graphs_that_share_a_workspace_follow_changed_lengths(hq, hk):
    page, d = 16, 128
    lens = [500, 20, 9000]
    q, k, v, table = _decode_case(BF, d, hq, hk, page, lens, 71)
    cache, tab = bd.PagedCache(k, v), ints(table)
    now = ints(lens)
    ws = torch.empty(bd.decode_workspace_size(q, cache, tab), dtype=torch.uint8, device=DEV)
    q2 = randn(q.shape, 72, BF, 2.0)
    outs = [torch.empty_like(q) for _ in range(2)]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        for x, o in zip((q, q2), outs):
            bd.basa_decode_attn(x, cache, tab, now, ws=ws, out=o)
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    graphs = []
    for x, o in zip((q, q2), outs):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            bd.basa_decode_attn(x, cache, tab, now, ws=ws, out=o)
        graphs.append(g)
    for step in ([500, 20, 9000], [3, 0, 8999], [480, 17, 1], [0, 0, 0], [500, 20, 9000]):
        now.copy_(ints(step))
        for o in outs:
            o.fill_(7.0)
        for g in graphs:
            g.replay()
        torch.cuda.synchronize()
        for x, o in zip((q, q2), outs):
            assert torch.equal(o, bd.basa_decode_attn(x, cache, tab, now)), step
        check_decode(outs[1], None, q2, k, v, table, step)


def test_a_workspace_full_of_rubbish_changes_nothing():
    lens = [5000, 1, 0, 700]
    q, k, v, table = _decode_case(BF, 64, 8, 2, 16, lens, 81)
    cache, tab = bd.PagedCache(k, v), ints(table)
    want = bd.basa_decode_attn(q, cache, tab, ints(lens))
    size = bd.decode_workspace_size(q, cache, tab)
    for fill in (0, 255, 127):
        ws = torch.full((size + 512,), fill, dtype=torch.uint8, device=DEV)
        assert torch.equal(want, bd.basa_decode_attn(q, cache, tab, ints(lens), ws=ws[:size]))
        assert (ws[size:] == fill).all()


@pytest.mark.parametrize("dtype,d,hq,hk,page,layout", [(BF, 128, 8, 2, 16, "token"), (F32, 64, 4, 4, 20, "head")])
def test_prompts_then_steps_then_a_prompt_that_goes_on(dtype, d, hq, hk, page, layout):
    """A serving loop on the cache against the same attention on contiguous keys and values."""
    rng = np.random.default_rng(1)
    n, width, block = 4, 60, 64
    pool = rng.permutation(150).astype(np.int32)
    cache = bd.PagedCache(*(store(150, hk, page, d, dtype, layout, DEV) for _ in range(2)))
    table, lens, used = torch.full((n, width), -1, dtype=torch.int32, device=DEV), ints([0] * n), 0
    held = [[torch.empty(0, hk, d, dtype=dtype, device=DEV)] * 2 for _ in range(n)]
    seed = [100]

    def rows(count, heads):
        seed[0] += 1
        return randn((count, heads, d), seed[0], dtype)

    def step(add):
        nonlocal lens, used
        before = lens.tolist()
        total = sum(add)
        plan = bd.basa_page_tables(lens, ints(add), table, ints(pool[used:]), page, total)
        q, k, v = rows(total, hq), rows(total, hk), rows(total, hk)
        given, asked = plan.pages.tolist()
        assert given == asked and plan.lens.tolist() == [a + b for a, b in zip(before, add)]
        used += given
        lens = plan.lens
        cu = plan.cu.tolist()
        for i in range(n):
            held[i] = [torch.cat([x, y[cu[i]:cu[i + 1]]]) for x, y in zip(held[i], (k, v))]
        return plan, q, k, v, cu, before

    view = lambda x: x.permute(1, 0, 2).unsqueeze(0)
    # prompts
    plan, q, k, v, cu, _ = step([300, 1, 77, 129])
    out = bd.ba_att_cached(q, k, v, cu, cache, table, plan.slots, block=block, sparsity=0.25)
    assert torch.equal(out, bd.ba_att_varlen(q, k, v, cu, block, 0.25))
    # single tokens
    for _ in range(3):
        plan, q, k, v, cu, _ = step([1] * n)
        out, lse = bd.ba_att_decode(q, k, v, cache, table, plan.lens, plan.slots, want_lse=True)
        for i in range(n):
            ref, ref_lse, size = attention64(q[i], *held[i])
            for h in range(hq):
                tol, tol_lse = decode_tolerance(dtype, held[i][0].shape[0], d, float(size[h]), float(held[i][1].abs().max()))
                assert float(((out[i, h].double() - ref[h]).abs() - HALF_STEP[dtype] * ref[h].abs()).max()) <= tol
                assert abs(float(lse[i, h]) - float(ref_lse[h])) <= tol_lse
    # two sequences go on, one ends, one waits
    plan, q, k, v, cu, before = step([200, 0, 65, 0])
    out = bd.ba_att_cached(q, k, v, cu, cache, table, plan.slots, cached=before, block=block, sparsity=0.5, causal=True)
    for i in (0, 2):
        part = slice(cu[i], cu[i + 1])
        want, _ = bd.ba_att(view(q[part]), view(held[i][0]), view(held[i][1]), block, 0.5, causal=True)
        assert torch.equal(view(out[part]), want)
    assert table.max() < 150 and len(set(table[table >= 0].tolist())) == int((table >= 0).sum()) == used


@pytest.mark.parametrize("dtype", [BF, F32])
def test_a_captured_step_replays_on_its_own_results(dtype):
    """Tables, append and attention of a decode step in one graph that feeds its lengths and its free pages back to itself."""
    page, hk, hq, d, width, total = 16, 2, 8, 64, 80, 400
    start = [15, 0, 1000, 47]
    n = len(start)
    q, k_cache, v_cache, held = _decode_case(dtype, d, hq, hk, page, start, 91, spare=total - sum(-(-x // page) for x in start))
    table = np.full((n, width), -1, dtype=np.int32)
    table[:, :held.shape[1]] = held
    pool = np.setdiff1d(np.arange(total), table[table >= 0]).astype(np.int32)
    cache, tab, have, one = bd.PagedCache(k_cache, v_cache), ints(table), ints(start), ints([1] * n)
    pool_d, used = ints(pool), ints([0], torch.int64)
    free, ar = pool_d[:n].clone(), torch.arange(n, device=DEV)
    plan, out = bd.PageTables(n, n + 2, DEV), torch.empty_like(q)
    k, v = randn((n + 2, hk, d), 1, dtype), randn((n + 2, hk, d), 2, dtype)          # two rows of padding
    ws = torch.empty(bd.decode_workspace_size(q, cache, tab), dtype=torch.uint8, device=DEV)

    def step():
        bd.basa_page_tables(have, one, tab, free, page, n + 2, out=plan)
        bd.basa_cache_append(k, v, plan.slots, cache)
        bd.basa_decode_attn(q, cache, tab, plan.lens, ws=ws, out=out)
        have.copy_(plan.lens)
        used.add_(plan.pages[0])
        free.copy_(pool_d[used + ar])

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    state = [x.clone() for x in (tab, have, used, free, k_cache, v_cache)]
    with torch.cuda.stream(side):
        step()
    torch.cuda.current_stream().wait_stream(side)
    for x, y in zip((tab, have, used, free, k_cache, v_cache), state):
        x.copy_(y)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    lens, given = list(start), 0
    for it in range(20):
        for x, seed in ((q, 3), (k, 1), (v, 2)):
            x.copy_(randn(x.shape, 1000 * it + seed, dtype))
        out.fill_(9.0)
        graph.replay()
        torch.cuda.synchronize()
        want, slots, after, _, pages = page_tables(lens, [1] * n, table, pool[given:given + n], page, n + 2)
        given += int(pages[0])
        lens, table = after.tolist(), want
        assert np.array_equal(tab.cpu().numpy(), want) and np.array_equal(plan.slots.cpu().numpy(), slots) and have.tolist() == lens
        at, off = torch.from_numpy(slots[:n] // page).to(DEV), torch.from_numpy(slots[:n] % page).to(DEV)
        assert torch.equal(k_cache[at, :, off], k[:n]) and torch.equal(v_cache[at, :, off], v[:n])
        check_decode(out, None, q, k_cache, v_cache, want, lens, f"replay {it}")
        assert torch.equal(out, bd.basa_decode_attn(q, cache, tab, plan.lens))
    assert len(set(table[table >= 0].tolist())) == int((table >= 0).sum())


def test_calls_on_two_streams_with_workspaces_of_their_own():
    lens = [3000, 10, 0, 900]
    q, k, v, table = _decode_case(BF, 128, 8, 2, 16, lens, 95)
    cache, tab, now = bd.PagedCache(k, v), ints(table), ints(lens)
    want = bd.basa_decode_attn(q, cache, tab, now)
    streams = [torch.cuda.Stream() for _ in range(2)]
    outs = [[], []]
    for s in streams:
        s.wait_stream(torch.cuda.current_stream())
    for _ in range(10):
        for s, o in zip(streams, outs):
            with torch.cuda.stream(s):
                o.append(bd.basa_decode_attn(q, cache, tab, now))
    torch.cuda.synchronize()
    assert all(torch.equal(o, want) for side in outs for o in side)
