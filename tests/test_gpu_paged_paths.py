"""Every kernel that the paged cache's calls choose between, on both sides of the lines where the choice changes."""
import numpy as np
import pytest
import torch

from paged_util import check_decode, new_tables, store
from test_gpu_paged import BF, DEV, F32, _decode_case, bits, ints, randn
from paper_2605_19726_amd import binding as bd

pytestmark = pytest.mark.gpu
TYPES = [(BF, 128), (BF, 64), (F32, 128), (F32, 64)]
ONE_LAUNCH = 256                            # bytes of workspace that a call asks for which is one launch


def _attend(q, k, v, table, lens):
    """(out, lse, whether the call is one launch)"""
    cache, tab = bd.PagedCache(k, v), ints(table)
    out, lse = bd.basa_decode_attn(q, cache, tab, ints(lens), want_lse=True)
    return out, lse, bd.decode_workspace_size(q, cache, tab) == ONE_LAUNCH


@pytest.mark.parametrize("dtype,d", TYPES)
@pytest.mark.parametrize("hq,hk,page,layout", [(4, 4, 16, "head"), (8, 1, 64, "token"), (16, 1, 3, "token"), (17, 1, 25, "head"), (32, 8, 1, "head"),
                                               (40, 2, 32, "token"), (33, 1, 16, "head"), (66, 2, 50, "token"), (96, 1, 100, "head")])
def test_one_launch_for_rows_of_up_to_700_tokens(dtype, d, hq, hk, page, layout):
    lens = [1, 0, 31, 32, 33, 127, 128, 129, 500, 2, 700]
    q, k, v, table = _decode_case(dtype, d, hq, hk, page, lens, hq + page, (layout, "head"))
    out, lse, one = _attend(q, k, v, table, lens)
    assert one and not out[1].any() and (lse[1] == -float("inf")).all()
    check_decode(out, lse, q, k, v, table, lens)
    pages = k.shape[0]                      # and with pages that are none: one in between, all of a row, the last of the longest
    table[8, 0], table[4, :], table[10, (700 - 1) // page] = -1, pages, 2 ** 31 - 1
    out, lse, _ = _attend(q, k, v, table, lens)
    check_decode(out, lse, q, k, v, table, lens)
    assert not out[4].any() and (lse[4] == -float("inf")).all()


@pytest.mark.parametrize("dtype,d", TYPES)
@pytest.mark.parametrize("hq,hk,n", [(4, 1, 500), (1, 1, 131), (8, 4, 200), (17, 1, 300), (34, 2, 150), (40, 1, 260), (66, 2, 130)])
def test_many_short_rows_in_small_workgroups(dtype, d, hq, hk, n):
    rng = np.random.default_rng(n)
    lens = [int(x) for x in rng.integers(0, 61, n)]
    lens[:5] = [0, 1, 60, 33, 32]
    q, k, v, table = _decode_case(dtype, d, hq, hk, 16, lens, 5, width=4)
    table[5, 0], table[7, :], table[2, 2] = -1, k.shape[0], -2 ** 31
    out, lse, one = _attend(q, k, v, table, lens)
    some = sorted(set(range(10)) | set(rng.integers(0, n, 20).tolist()) | {n - 1})
    assert one and torch.isfinite(out).all()
    check_decode(out[some], lse[some], q[some], k, v, table[some], [lens[i] for i in some])
    assert not out[0].any() and not out[7].any()


@pytest.mark.parametrize("dtype,hq,hk,n,page,width,one", [
    (BF, 8, 2, 3, 3, 256, True), (BF, 8, 2, 3, 1, 769, False), (F32, 40, 2, 3, 3, 256, True), (F32, 40, 2, 3, 1, 769, False),        # 768 | 769 tokens
    (BF, 4, 1, 128, 16, 64, True), (BF, 4, 1, 127, 16, 64, False), (BF, 4, 1, 128, 25, 41, False), (BF, 40, 1, 64, 16, 64, True),   # 1024, 128 units
    (F32, 17, 1, 64, 16, 64, True), (F32, 17, 1, 63, 16, 64, False), (BF, 4, 1, 79, 20, 2, True), (BF, 4, 1, 80, 20, 2, True),
    (BF, 4, 1, 81, 20, 2, True), (BF, 33, 1, 39, 20, 2, True), (BF, 33, 1, 40, 20, 2, True), (F32, 4, 2, 39, 20, 2, True), (F32, 4, 2, 40, 20, 2, True)])
def test_both_sides_of_the_lines(dtype, hq, hk, n, page, width, one):
    """One launch or two: rows of 768 tokens, of 1024 where there are 128 units; 8 or 2 waves: twice as many units as tokens."""
    rng, most = np.random.default_rng(n), width * page
    lens = [int(x) for x in rng.integers(0, 40, n)]
    lens[0], lens[-1] = most, most - 1
    q, k, v, table = _decode_case(dtype, 128, hq, hk, page, lens, 9, width=width)
    out, lse, is_one = _attend(q, k, v, table, lens)
    assert is_one == one
    some = sorted({0, 1, n // 2, n - 2, n - 1})
    check_decode(out[some], lse[some], q[some], k, v, table[some], [lens[i] for i in some])
    assert torch.isfinite(out).all()


@pytest.mark.parametrize("T", [32767, 32768, 65536, 65537])
@pytest.mark.parametrize("layout", ["head", "token"])
def test_copies_on_both_sides_of_the_streaming_lines(T, layout):
    """8 heads of 128 in bf16, 4 KB a token: loads past the caches from 128 MB on, a gather's stores beyond 256 MB."""
    rng, heads, page, d = np.random.default_rng(T), 8, 64, 128
    pages = -(-T // page) + 3
    k_cache, v_cache = (store(pages, heads, page, d, BF, layout, DEV, x) for x in (7.0, 8.0))
    cache, k, v = bd.PagedCache(k_cache, v_cache), randn((T, heads, d), 1, BF), randn((T, heads, d), 2, BF)
    table = new_tables([T - 100, 100], page, pages, rng)
    slots = np.concatenate([table[i, np.arange(n) // page].astype(np.int64) * page + np.arange(n) % page for i, n in enumerate((T - 100, 100))])
    slots[17] = -1
    bd.basa_cache_append(k, v, ints(slots, torch.int64), cache)
    at = ints(np.delete(slots, 17), torch.int64)
    keep = torch.arange(T, device=DEV) != 17
    for x, rows, fill in ((k_cache, k, 7.0), (v_cache, v, 8.0)):
        want = torch.full((pages * page, heads, d), fill, dtype=BF, device=DEV)
        want[at] = rows[keep]
        assert torch.equal(bits(x.permute(0, 2, 1, 3).reshape(-1, heads, d)), bits(want))
    gk, gv = bd.basa_cache_gather(cache, ints(table), ints([0, T - 100, T]), T)
    for got, rows, fill in ((gk, k, 7.0), (gv, v, 8.0)):
        assert torch.equal(bits(got[keep]), bits(rows[keep])) and (got[17] == fill).all()


@pytest.mark.parametrize("cu", [[0, 90, 40], [50, 20, 90], [-5, 10, 30], [0, 2 ** 31 - 1, 2 ** 31 - 1], [-2 ** 31, 0, 60], [64, 0, 0], [3, 3, 61]])
def test_gather_takes_rows_of_the_named_pages_alone_whatever_the_offsets(cu):
    """Offsets that do not ascend, between guard rows and table entries that name other pages: rows outside [cu[0], cu[n]) stay as they were, every other
    one is a row of a page that the table names, or zero."""
    T, heads, page, d, pages, fill = 64, 2, 16, 64, 7, -3.0
    place = torch.arange(5 * page, device=DEV).reshape(5, 1, page, 1).float()
    caches = []
    for first in (1.0, 101.0):              # K's rows hold 1 .. 80, V's 101 .. 180; pages 5 and 6, which no entry of the table names, 250
        x = torch.full((pages, heads, page, d), 250.0, dtype=BF, device=DEV)
        x[:5] = (place + first).to(BF)
        caches.append(x)
    around = torch.full((4, 7), 5, dtype=torch.int32, device=DEV)
    around[3:], around[:, 5:] = 6, 6
    around[1:3, 2:5] = torch.tensor([[3, 0, 4], [1, 2, 0]], dtype=torch.int32, device=DEV)
    buffers = [torch.full((T + 40, heads, d), fill, dtype=BF, device=DEV) for _ in range(2)]
    out = tuple(b[20:20 + T] for b in buffers)
    bd.basa_cache_gather(bd.PagedCache(*caches), around[1:3, 2:5], ints(cu), T, out=out)
    for buffer, first in zip(buffers, (1.0, 101.0)):
        x = buffer.float()
        assert (x[:20] == fill).all() and (x[20 + T:] == fill).all()
        rows, inside = x[20:20 + T], torch.tensor([cu[0] <= t < cu[2] for t in range(T)], device=DEV)
        assert (rows[~inside] == fill).all()
        value = rows[inside][:, 0, 0]
        assert (rows[inside] == value[:, None, None]).all()              # a row in one piece
        assert ((value == 0) | ((value >= first) & (value < first + 5 * page))).all()
    k, v = (b[20:20 + T, 0, 0].float() for b in buffers)
    assert torch.equal(torch.where(k > 0, k + 100, k), v)                # K and V of the same place


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("width", [2, 70])
def test_batches_of_more_than_65535_rows(dtype, width):
    """70000 sequences that share eight pages, in small workgroups and cut by runs."""
    n, hq, hk, d, page, pages = 70000, 4, 2, 64, 16, 8
    rng = np.random.default_rng(width)
    k, v, q = randn((pages, hk, page, d), 1, dtype), randn((pages, hk, page, d), 2, dtype), randn((n, hq, d), 3, dtype, 2.0)
    table = rng.integers(0, pages, (n, width)).astype(np.int32)
    lens = [int(x) for x in rng.integers(0, 2 * page + 1, n)]
    lens[n - 1], lens[n // 2] = width * page, width * page - 7
    out, lse, one = _attend(q, k, v, table, lens)
    assert one == (width == 2) and torch.isfinite(out).all()
    some = [0, 1, 32767, 32768, n // 2 - 1, n // 2, 65535, 65536, n - 2, n - 1]
    check_decode(out[some], lse[some], q[some], k, v, table[some], [lens[i] for i in some])
    assert torch.equal(torch.isfinite(lse), (ints(lens) > 0)[:, None].expand(n, hq))
