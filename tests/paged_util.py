"""Plain statements of the paged-cache operators, in Python integers and 64-bit floats, and what their results may be off by."""
import math

import numpy as np
import torch

EPS32 = 2.0 ** -24
HALF_STEP = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8}


def page_tables(have, add, table, free, page, n_slots):
    """(table, slots, lens, cu, pages) of a step, one sequence after the other."""
    table, width = np.array(table, dtype=np.int64), np.shape(table)[1]
    slots, lens, cu, asked, given = [-1] * n_slots, [], [0], 0, 0
    for i, (h, a) in enumerate(zip(have, add)):
        h, a, begin = max(int(h), 0), max(int(a), 0), cu[-1]
        cu.append(begin + a)
        lens.append(h)
        if h + a > width * page or begin + a > n_slots:
            continue
        held, after = -(-h // page), -(-(h + a) // page)
        asked += after - held
        if asked > len(free):
            continue
        table[i, held:after] = free[asked - (after - held):asked]
        given, lens[i] = asked, h + a
        for t in range(a):
            entry = int(table[i, (h + t) // page])
            if entry >= 0:
                slots[begin + t] = entry * page + (h + t) % page
    top = 2 ** 31 - 1
    return table, np.array(slots, dtype=np.int64), np.array(lens), np.minimum(cu, top), np.array([given, min(asked, top)])


def new_tables(lens, page, n_pages, rng, width=None):
    """A block table whose sequences own pages of their own, in no order; entries that name no page are -1."""
    need = [-(-int(n) // page) for n in lens]
    width = max([1] + need) if width is None else width
    ids = rng.permutation(n_pages)
    assert sum(need) <= n_pages
    table, at = np.full((len(lens), width), -1, dtype=np.int32), 0
    for i, n in enumerate(need):
        table[i, :n] = ids[at:at + n]
        at += n
    return table


def store(pages, heads, page, d, dtype, layout, device, fill=float("nan")):
    """An empty cache of K or V as [pages, heads, page, d], stored head by head or token by token."""
    if layout == "head":
        return torch.full((pages, heads, page, d), fill, dtype=dtype, device=device)
    return torch.full((pages, page, heads, d), fill, dtype=dtype, device=device).permute(0, 2, 1, 3)


def rows_of(table_row, lens, page):
    """Page and place of the first `lens` tokens."""
    t = np.arange(lens)
    return torch.from_numpy(np.asarray(table_row, dtype=np.int64)[t // page]), torch.from_numpy(t % page)


def attention64(q, k, v):
    """One query of every head, q [heads, d], over k and v [tokens, kv heads, d]: (out, lse, bound on the scores' terms), 64 bits."""
    hq, d = q.shape
    n, hk, _ = k.shape
    q, k, v = q.double(), k.double(), v.double()
    out, lse = torch.zeros(hq, d, dtype=torch.float64, device=q.device), torch.full((hq,), -math.inf, dtype=torch.float64, device=q.device)
    size = torch.zeros(hq, dtype=torch.float64, device=q.device)
    if n == 0:
        return out, lse, size
    for h in range(hq):
        g = h // (hq // hk)
        s = torch.mv(k[:, g], q[h]) / math.sqrt(d)
        size[h] = torch.mv(k[:, g].abs(), q[h].abs()).max() / math.sqrt(d)
        lse[h] = torch.logsumexp(s, 0)
        if lse[h] != -math.inf:
            out[h] = torch.mv(v[:, g].t(), torch.exp(s - lse[h]))
    return out, lse, size


def decode_tolerance(dtype, n, d, size, v_max):
    """(what an output element may be off by beyond the rounding of its type, the same for lse) per query head.

    A score is a sum of d products: every term and partial sum, at most `size` = sum |q_i k_i| / sqrt(d), is rounded by up to 2^-24 of itself,
    the errors with either sign: 8 sqrt(d) 2^-24 size.  Its difference to the maximum (at most 2 size) and the product with log2 e / sqrt(d),
    whose factor is rounded too: 3 * 2 size * 2^-24.  The exponential: 2^-23.  A weight's relative error is their sum e_w; bf16 adds the
    two-part representation, 2^-16.  Numerator and denominator hold it once each.  Sums over n tokens: 8 sqrt(n + 64) 2^-24 of sum p |v|,
    which is at most v_max sum p.  lse: the error of the maximum's score, that of the sum, the logarithm and its last place."""
    e_w = EPS32 * (8 * math.sqrt(d) * size + 6 * size + 2)
    e_sum = 8 * math.sqrt(n + 64) * EPS32
    part = 2.0 ** -16 if dtype == torch.bfloat16 else 0.0
    return (2 * e_w + 2 * e_sum + part) * v_max + 1e-30, e_w + e_sum + EPS32 * (2 * size + 2 * math.log(n + 1) + 2)


def check_decode(out, lse, q, k_cache, v_cache, table, lens, what=""):
    """Every row of a decode call against 64 bits on the tokens whose page is one of the cache's."""
    pages, heads, page, d = k_cache.shape
    table = np.asarray(table)
    for i, n in enumerate(lens):
        n = max(0, min(int(n), table.shape[1] * page))
        at, off = rows_of(table[i], n, page)
        keep = (at >= 0) & (at < pages)
        at, off = at[keep].to(q.device), off[keep].to(q.device)
        k, v = k_cache[at, :, off], v_cache[at, :, off]              # [tokens, heads, d]
        ref, ref_lse, size = attention64(q[i], k, v)
        v_max = float(v.double().abs().max()) if len(at) else 0.0
        for h in range(q.shape[1]):
            tol, tol_lse = decode_tolerance(q.dtype, len(at), d, float(size[h]), v_max)
            err = (out[i, h].double() - ref[h]).abs() - HALF_STEP[q.dtype] * ref[h].abs()
            assert float(err.max()) <= tol, f"{what}: sequence {i} ({n} tokens), head {h}: off by {float(err.max()):.3e} beyond its type, {tol:.3e} allowed"
            if lse is not None:
                if math.isinf(float(ref_lse[h])):
                    assert float(lse[i, h]) == float(ref_lse[h]), f"{what}: lse of sequence {i}, head {h}: {float(lse[i, h])}"
                else:
                    off_by = abs(float(lse[i, h]) - float(ref_lse[h]))
                    assert off_by <= tol_lse, f"{what}: lse of sequence {i}, head {h}: off by {off_by:.3e}, {tol_lse:.3e} allowed"
