"""Infinities and NaN among the cached values: what the formula makes of them in 64 bits, for every kernel of the single-token attention."""
import math

import numpy as np
import pytest
import torch

from paged_util import HALF_STEP, decode_tolerance, rows_of
from test_gpu_paged import BF, DEV, F32, _decode_case, ints
from paper_2605_19726_amd import binding as bd

pytestmark = pytest.mark.gpu
INF, NAN = float("inf"), float("nan")

# (query heads, KV heads, lengths, table width): 8 waves to a row, up to 16 heads and more, several units; 2 waves, the same; cut by runs, the same
PATHS = [(8, 2, [1, 40, 300, 700], 44), (34, 2, [1, 40, 300, 500], 44), (40, 1, [1, 40, 300, 500], 44),
         (8, 2, [1, 40, 30] + [7] * 125, 4), (34, 2, [1, 40, 30] + [7] * 125, 4), (68, 2, [1, 40, 30] + [7] * 125, 4),
         (8, 2, [1, 40, 3000, 700], 190), (34, 2, [1, 40, 3000, 700], 190), (68, 2, [1, 40, 3000, 700], 190)]


def _check(out, q, k, v, table, lens, rows):
    """Rows against sum p v / sum p in 64 bits: NaN and infinities where that has them, the others within the derived tolerance."""
    d = q.shape[2]
    for i in rows:
        at, off = (x.to(DEV) for x in rows_of(table[i], lens[i], k.shape[2]))
        ks, vs = k[at, :, off].double(), v[at, :, off].double()
        for h in range(q.shape[1]):
            g = h // (q.shape[1] // k.shape[1])
            s = torch.mv(ks[:, g], q[i, h].double()) / math.sqrt(d)
            p = torch.exp(s - s.max())
            want = (p[:, None] * vs[:, g]).sum(0) / p.sum()
            got, fine = out[i, h].double(), torch.isfinite(want)
            size = float(torch.mv(ks[:, g].abs(), q[i, h].double().abs()).max()) / math.sqrt(d)
            v_max = float(vs[vs.isfinite()].abs().max())
            tol, _ = decode_tolerance(q.dtype, lens[i], d, size, v_max)
            tol += 2.0 ** -16 * v_max        # the two positive numbers of a weight: 2^-15 of it
            assert torch.equal(got.isnan(), want.isnan()), f"sequence {i}, head {h}: NaN at {got.isnan().nonzero().flatten().tolist()}"
            assert torch.equal(got[~fine & ~want.isnan()], want[~fine & ~want.isnan()]), f"sequence {i}, head {h}: infinities"
            assert float(((got - want).abs() - HALF_STEP[q.dtype] * want.abs())[fine].max()) <= tol, f"sequence {i}, head {h}"


@pytest.mark.parametrize("dtype,d", [(BF, 128), (BF, 64), (F32, 128), (F32, 64)])
@pytest.mark.parametrize("hq,hk,lens,width", PATHS)
def test_infinite_values_stay_infinite(dtype, d, hq, hk, lens, width):
    """A value that is infinite makes its dimension infinite, whatever its token's weight: the only one, the largest, one that rounds up or down
    in 16 bits; both signs together, and NaN, make it NaN; other dimensions keep theirs."""
    q, k, v, table = _decode_case(dtype, d, hq, hk, 16, lens, 17, width=width)
    put = lambda i, t, dim, x: v.__setitem__((int(table[i, t // 16]), slice(None), t % 16, dim), x)
    put(0, 0, 3, INF), put(0, 0, 5, -INF), put(0, 0, 7, NAN)
    for dim in range(16):                   # tokens of all weights, half of which round up
        put(1, 2 * dim + 3, dim, INF if dim % 2 else -INF)
        put(2, (lens[2] - 1) * dim // 15, dim, -INF if dim % 2 else INF)
    put(1, 4, 40, INF), put(1, 30, 40, -INF), put(1, 39, 41, NAN)
    heavy = [x.to(DEV) for x in rows_of(table[2], lens[2], 16)]
    top = int(torch.mv(k[heavy[0], 0, heavy[1]].float(), q[2, 0].float()).argmax())
    put(2, top, 50, -INF)
    rows = [0, 1, 2, 3] if len(lens) == 4 else [0, 1, 2, 3, 100]
    out = bd.basa_decode_attn(q, bd.PagedCache(k, v), ints(table), ints(lens))
    _check(out, q, k, v, table, lens, rows)


@pytest.mark.parametrize("dtype,d", [(BF, 128), (BF, 64), (F32, 128), (F32, 64)])
@pytest.mark.parametrize("width", [8, 190])
def test_infinite_values_of_tiny_weight(dtype, d, width):
    """Weights from 2^-110 down to 2^-123, in the wave that has the largest score and in others."""
    lens = [100, 100]
    q, k, v, table = _decode_case(dtype, d, 4, 2, 16, lens, 19, width=width)
    q[:], k[:] = 0.0, 0.0
    q[:, :, 0] = 1.0
    for i, first in ((0, 3), (1, 65)):
        for j in range(10):
            t = first + 3 * j
            k[int(table[i, t // 16]), :, t % 16, 0] = -608.0 - 8 * j if d == 64 else -860.0 - 12 * j       # e^-76 to e^-85.6
            v[int(table[i, t // 16]), :, t % 16, 11 + j] = INF if j % 3 else -INF
    out = bd.basa_decode_attn(q, bd.PagedCache(k, v), ints(table), ints(lens))
    _check(out, q, k, v, table, lens, [0, 1])


@pytest.mark.parametrize("dtype,d", [(BF, 128), (BF, 64), (F32, 128), (F32, 64)])
@pytest.mark.parametrize("hq,hk,lens,width", PATHS)
def test_a_row_of_scores_of_minus_infinity_is_zero_whatever_its_values(dtype, d, hq, hk, lens, width):
    q, k, v, table = _decode_case(dtype, d, hq, hk, 16, lens, 23, width=width)
    q[:, :, 0] = 1.0
    for i in (0, 2):
        at, off = (x.to(DEV) for x in rows_of(table[i], lens[i], 16))
        k[at, :, off, 0] = -INF
        v[at, :, off, :3] = torch.tensor([INF, -INF, NAN], dtype=dtype, device=DEV)
    out, lse = bd.basa_decode_attn(q, bd.PagedCache(k, v), ints(table), ints(lens), want_lse=True)
    for i in (0, 2):
        assert not out[i].any() and (lse[i] == -INF).all()
    _check(out, q, k, v, table, lens, [1, 3])


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("hq,hk,lens,width", PATHS)
def test_captured_calls_follow_values_that_become_infinite_and_finite_again(dtype, hq, hk, lens, width):
    q, k, v, table = _decode_case(dtype, 128, hq, hk, 16, lens, 29, width=width)
    cache, tab, now = bd.PagedCache(k, v), ints(table), ints(lens)
    ws, out = torch.empty(bd.decode_workspace_size(q, cache, tab), dtype=torch.uint8, device=DEV), torch.empty_like(q)
    finite = bd.basa_decode_attn(q, cache, tab, now)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        bd.basa_decode_attn(q, cache, tab, now, ws=ws, out=out)
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        bd.basa_decode_attn(q, cache, tab, now, ws=ws, out=out)
    kept = v.clone()
    for x in (None, INF, NAN, None, -INF, None):
        v.copy_(kept)
        if x is not None:
            v[int(table[1, 2]), :, 5, 9] = x                   # token 37 of sequence 1
        out.fill_(7.0)
        graph.replay()
        torch.cuda.synchronize()
        eager = bd.basa_decode_attn(q, cache, tab, now)
        assert torch.equal(out.isnan(), eager.isnan()) and torch.equal(out.nan_to_num(nan=3.0), eager.nan_to_num(nan=3.0))
        if x is None:
            assert torch.equal(out, finite)
        else:
            assert not torch.isfinite(out[1, :, 9]).any() and torch.isfinite(out[1, :, :9]).all() and torch.equal(out[0], finite[0])
