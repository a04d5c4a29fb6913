"""Plain statements of the operators for several new tokens per sequence and for the pages around them: Python integers and 64-bit floats."""
import math

import numpy as np
import torch

from paged_util import HALF_STEP, decode_tolerance, rows_of


def random_parents(n, rng, reach=8):
    """A tree: every token follows one of the `reach` before it, or the context."""
    return np.maximum(np.arange(n) - rng.integers(1, reach + 1, n), -1).astype(np.int32)


def ancestors(parents):
    """seen[r, j]: token r is token j or follows it, through however many others.  A parent that is not before its token is none."""
    n = len(parents)
    seen = np.zeros((n, n), dtype=bool)
    for r in range(n):
        at = r
        while True:
            seen[r, at] = True
            up = int(parents[at])
            if not 0 <= up < at:
                break
            at = up
    return seen


def mask_words(seen, words):
    """Rows of bits as int64 words; what does not fit is left out."""
    out = np.zeros((len(seen), words), dtype=np.uint64)
    for r, j in zip(*np.nonzero(seen)):
        if j < 64 * words:
            out[r, j // 64] |= np.uint64(1 << (int(j) % 64))
    return out.view(np.int64)


def check_tree(out, lse, q, k_cache, v_cache, table, lens, cu, seen, what="", only=None):
    """Every new token against 64 bits on the tokens that it sees and whose page is one of the cache's.  seen[i]: [n_i, n_i], None: a chain.  only: (sequence,
    its new tokens that are looked at)."""
    pages, heads, page, d = k_cache.shape
    hq, table = q.shape[1], np.asarray(table)
    group = hq // heads
    for i, n in enumerate(lens):
        a, b = cu[i], cu[i + 1]
        if b == a or (only and only[0] != i):
            continue
        new, n = b - a, max(0, min(int(n), table.shape[1] * page))
        at, off = rows_of(table[i], n, page)
        see = np.ones((new, n), dtype=bool)
        tree = np.tril(np.ones((new, new), dtype=bool)) if seen[i] is None else seen[i]
        first = max(new - n, 0)                                 # new tokens before it are in no page
        see[:, n - (new - first):] = tree[:, first:]
        see &= ((at >= 0) & (at < pages)).numpy()[None]
        pick = list(range(new)) if only is None else only[1]
        see, rows_at, new = see[pick], [a + r for r in pick], len(pick)
        see = torch.from_numpy(see).to(q.device)
        at, off = at.clamp(0, pages - 1).to(q.device), off.to(q.device)
        kept = see.any(0)
        for g in range(heads):
            # what no one sees may hold anything
            k, v = (x[at, g, off].double().masked_fill(~kept[:, None], 0.0) for x in (k_cache, v_cache))
            rows = q[rows_at, g * group:(g + 1) * group].double().reshape(new * group, d)
            hidden = ~see[:, None].expand(new, group, n).reshape(new * group, n)
            s = (rows @ k.t() / math.sqrt(d)).masked_fill(hidden, -math.inf)
            size = (rows.abs() @ k.abs().t() / math.sqrt(d)).masked_fill(hidden, 0.0).max(1).values if n else torch.zeros(new * group)
            ref_lse = torch.logsumexp(s, 1) if n else torch.full((new * group,), -math.inf, dtype=torch.float64, device=q.device)
            p = torch.exp(s - torch.where(ref_lse == -math.inf, 0.0, ref_lse)[:, None])
            ref = p @ v if n else torch.zeros(new * group, d, dtype=torch.float64, device=q.device)
            got = out[rows_at, g * group:(g + 1) * group].reshape(new * group, d).double()
            tol = [decode_tolerance(q.dtype, n, d, float(x), float(v.abs().max()) if n else 0.0) for x in size]
            room = torch.tensor([t[0] for t in tol], dtype=torch.float64, device=q.device)
            err = ((got - ref).abs() - HALF_STEP[q.dtype] * ref.abs()).max(1).values
            worst = int(torch.argmax(torch.nan_to_num(err - room, nan=math.inf)))
            assert bool((err <= room).all()), f"{what}: sequence {i} ({n} tokens, {new} new), KV head {g}, row {worst}: off by {float(err[worst]):.3e} " \
                f"beyond its type, {float(room[worst]):.3e} allowed"
            if lse is not None:
                e = lse[rows_at, g * group:(g + 1) * group].reshape(-1).double()
                assert torch.equal(torch.isinf(e), torch.isinf(ref_lse)), f"{what}: lse of sequence {i}: {e} / {ref_lse}"
                fin = torch.isfinite(ref_lse)
                room = torch.tensor([t[1] for t in tol], dtype=torch.float64, device=q.device)
                assert bool(((e - ref_lse).abs()[fin] <= room[fin]).all()), f"{what}: lse of sequence {i}, KV head {g}: {(e - ref_lse).abs()[fin].max()}"


def compact(table, start, keep, count, page, pages):
    """[(from slot, to slot)] of every move, in order."""
    moves, width = [], np.shape(table)[1]
    for i in range(len(start)):
        for j in range(max(0, min(int(count[i]), np.shape(keep)[1]))):
            a, b = int(start[i]) + int(keep[i][j]), int(start[i]) + j
            if int(keep[i][j]) <= j or int(start[i]) < 0 or a >= width * page:
                continue
            pa, pb = int(table[i][a // page]), int(table[i][b // page])
            if 0 <= pa < pages and 0 <= pb < pages:
                moves.append((pa * page + a % page, pb * page + b % page))
    return moves


def fork(table, lens, parents, free, page):
    """(rows of the new table as lists, lens, copies, pages), one new sequence after the other."""
    rows, new_lens, copies, asked, taken = [], [], [], 0, set()
    n, width = np.shape(table)
    for p in (int(p) for p in parents):
        length = max(0, min(int(lens[p]), width * page)) if 0 <= p < n else 0
        whole, rest = divmod(length, page)
        again = rest > 0 and p in taken
        if rest:
            taken.add(p)
        asked += again
        if again and asked > len(free):
            rows.append([])
            new_lens.append(0)
            copies.append([-1, -1, 0])
            continue
        row = [int(x) for x in table[p][:whole + (rest > 0)]] if length else []
        copies.append([row[whole], int(free[asked - 1]), rest] if again else [-1, -1, 0])
        if again:
            row[whole] = int(free[asked - 1])
        rows.append(row)
        new_lens.append(length)
    return rows, new_lens, copies, [min(asked, len(free)), asked]


def free_pages(table, lens, page, pages):
    used, width = set(), np.shape(table)[1]
    for row, n in zip(table, lens):
        used.update(int(x) for x in row[:-(-max(0, min(int(n), width * page)) // page)])
    return [p for p in range(pages) if p not in used]
