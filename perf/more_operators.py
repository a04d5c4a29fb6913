"""Operators for trees of drafted tokens over a paged key-value cache, and for the pages around them: listed cases, the ranges they stand
for, their plain forms and their values in 64 bits.

  op "masks"    who sees whom among drafted tokens, from the token that each follows (`basa_tree_masks`)
  op "tree"     attention of the drafted tokens of every sequence over its pages and over their ancestors (`basa_tree_attn`)
  op "compact"  kept tokens of every sequence moved together, in place (`basa_cache_compact`)
  op "fork"     block tables of sequences that go on from others, and the copies of the pages that are not full (`basa_page_fork`,
                `basa_cache_copy`)
  op "free"     the pages that no sequence holds (`basa_page_free`)

A cache of K or V is indexed [pages, heads_kv, page, d] and stored that way ("head" layout) or token-major, [pages, page, heads_kv, d]
("token" layout).  Sequence i owns the pages table[i, 0 .. ceil(len_i / page)); its token t lives in page table[i, t // page] at offset
t % page.  Lengths of a case are the same for every seed, in another order; which pages hold a sequence, trees, kept tokens and all
values go by the seed.
"""
import math
import random

import numpy as np
import torch

own = False

DEVICE = "cuda"
# len: tokens before the step; add: drafted tokens (tree, masks), tokens from `start` = len on of which `kept` stay (compact);
# chain: drafted tokens follow each other, no masks; new: sequences after the fork; spare: rows behind the last sequence
DEFAULTS = dict(op="tree", dtype="bf16", heads_q=32, heads_kv=8, d=128, page=64, layout="head", n_seq=1, len_lo=1, len_hi=1, add_lo=0,
                add_hi=0, chain=False, kept=0.5, new=1, spare=0, shape=1)


def _case(**kw):
    c = dict(DEFAULTS)
    c.update(kw)
    return c


def listed():
    return [
        # five drafted tokens on one short conversation: latency
        _case(name="tree_one_5", len_lo=700, len_hi=700, add_lo=5, add_hi=5, page=16),
        # fp32, a head of keys for every query head, heads of 64, ragged trees on lengths from a few tokens on, a page size that is no
        # power of two
        _case(name="tree_f32_mha_d64", dtype="f32", heads_q=16, heads_kv=16, d=64, page=100, n_seq=21, len_lo=3, len_hi=5000, add_lo=3,
              add_hi=31),
        # a batch of conversations of unequal lengths, small trees, pages stored token-major
        _case(name="tree_32_mid", n_seq=32, len_lo=1000, len_hi=16000, add_lo=8, add_hi=24, layout="token"),
        # a wide tree on one context of 128K tokens
        _case(name="tree_128k_64", len_lo=131072, len_hi=131072, add_lo=64, add_hi=64, page=128),
        # the masks of a small batch's step: latency
        _case(name="masks_step_8", op="masks", n_seq=8, add_lo=25, add_hi=25),
        # large ragged trees of a large batch, rows behind the last
        _case(name="masks_ragged_200", op="masks", n_seq=200, add_lo=1, add_hi=300, spare=50),
        # the accepted path of every sequence's tree, a third of 16 drafted tokens
        _case(name="compact_step_64", op="compact", n_seq=64, len_lo=500, len_hi=4000, add_lo=16, add_hi=16, kept=0.3),
        # long contexts of which a third is dropped, from the first token on, pages stored token-major
        _case(name="compact_evict_12", op="compact", n_seq=12, len_lo=0, len_hi=0, add_lo=2000, add_hi=16000, kept=0.67, page=16,
              layout="token"),
        # every prompt goes on as eight samples
        _case(name="fork_samples_64", op="fork", n_seq=8, new=64, len_lo=100, len_hi=3000),
        # a step of a beam search over many long sequences: some beams end, others go on several times
        _case(name="fork_beams_512", op="fork", n_seq=512, new=512, len_lo=2000, len_hi=9000, page=16, heads_q=4, heads_kv=2, d=64),
        # the pool of a small server
        _case(name="free_step_64", op="free", n_seq=64, len_lo=40, len_hi=8000, page=16),
        # the pool of a large one, short pages
        _case(name="free_large_2000", op="free", n_seq=2000, len_lo=0, len_hi=20000, page=16),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


MOST_ELEMENTS = 2.0e8        # of K in a drawn case's cache
MOST_FLOPS = 1.2e11          # of a drawn case's attention: below the largest listed one


def draw(rng):
    """One more case: sizes spread over their logarithm, most of them no multiple of anything."""
    op = rng.choice(["tree", "tree", "tree", "masks", "compact", "compact", "fork", "free"])
    hk, d = rng.choice([1, 2, 4, 5, 8, 16]), rng.choice([64, 128])
    group = rng.choice([1, 2, 4, 5, 7, 8, 16])
    while hk * group > 64:
        group //= 2
    c = _case(op=op, heads_kv=hk, heads_q=hk * group, d=d, page=rng.choice([1, 16, 20, 32, 64, 100, 128, 256]),
              dtype=rng.choice(["bf16", "bf16", "f32"]), layout=rng.choice(["head", "token"]), shape=rng.randint(1, 1 << 30))
    if op == "tree":
        n = _log(rng, 1, 200)
        add = _log(rng, 1, max(2, min(300, 4000 // n)))
        most = MOST_ELEMENTS / (hk * d) / n
        hi = _log(rng, 2, max(3, min(200000, int(most), int(MOST_FLOPS / (4 * d * hk * group * add * n)))))
        c.update(n_seq=n, add_lo=rng.choice([1, max(1, add // 3), add]), add_hi=add, len_lo=rng.choice([0, 1, max(1, hi // 3), hi]), len_hi=hi,
                 chain=rng.choice([True, False, False]))
    elif op == "masks":
        n = _log(rng, 1, 500)
        add = _log(rng, 1, max(2, min(1000, 40000 // n)))
        c.update(n_seq=n, add_lo=rng.choice([0, 1, add]), add_hi=add, spare=rng.randint(0, 100))
    elif op == "compact":
        n = _log(rng, 1, 200)
        add = _log(rng, 1, max(2, min(50000, int(MOST_ELEMENTS / (hk * d) / n / 2))))
        c.update(n_seq=n, len_lo=0, len_hi=rng.choice([0, _log(rng, 1, 1000)]), add_lo=rng.choice([0, 1, add]), add_hi=add,
                 kept=rng.choice([0.0, 0.2, 0.5, 0.9, 1.0]))
        if c["len_hi"] * n * hk * d > MOST_ELEMENTS:
            c["len_hi"] = 1
    elif op == "fork":
        n = _log(rng, 1, 300)
        hi = _log(rng, 1, max(2, min(20000, int(MOST_ELEMENTS / (hk * d) / n / 2))))
        c.update(n_seq=n, new=_log(rng, 1, 600), len_lo=rng.choice([0, 1, hi]), len_hi=hi)
    else:
        n = _log(rng, 1, 3000)
        c.update(n_seq=n, len_lo=0, len_hi=_log(rng, 1, 20000), page=rng.choice([16, 20, 32, 64, 100, 128, 256]))
    return c


def _lengths(c, what):
    """n_seq lengths between <what>_lo and <what>_hi, spread over their logarithm; one of them each bound."""
    lo, hi, n = c[what + "_lo"], c[what + "_hi"], c["n_seq"]
    rng = random.Random(c["shape"] * 2 + (what == "add"))
    lens = [max(lo, min(hi, int(math.exp(rng.uniform(math.log(lo + 0.5), math.log(hi + 0.999)))))) for _ in range(n)]
    lens[0] = hi
    if n > 1:
        lens[-1] = lo
    return lens


def _dtype(c):
    return torch.float32 if c["dtype"] == "f32" else torch.bfloat16


def _pages(n, page):
    return (n + page - 1) // page


def _ints(values, dtype=torch.int32):
    return torch.tensor(values, dtype=dtype, device=DEVICE)


def _cache(c, n_pages, gen):
    """One of K and V: [pages, heads_kv, page, d] in the case's layout."""
    hk, page, d = c["heads_kv"], c["page"], c["d"]
    shape = (n_pages, hk, page, d) if c["layout"] == "head" else (n_pages, page, hk, d)
    x = torch.empty(shape, dtype=_dtype(c), device=DEVICE).normal_(generator=gen)
    return x if c["layout"] == "head" else x.permute(0, 2, 1, 3)


def _words(c):
    return max(1, _pages(c["add_hi"], 64))


def _trees(rng, sizes):
    """Parents of every sequence's tokens: most of them one of the last few before it, some the cached context itself (-1)."""
    out = []
    for n in sizes:
        r = np.arange(n)
        back = rng.integers(1, 9, n)
        out.append(np.maximum(r - back, -1).astype(np.int32))
    return out


def _tree_bits(parents, words):
    """The masks of one tree, [n, words] as unsigned 64-bit numbers."""
    bits = np.zeros((len(parents), words), dtype=np.uint64)
    for r, p in enumerate(parents):
        if p >= 0:
            bits[r] = bits[p]
        bits[r, r // 64] |= np.uint64(1 << (r % 64))
    return bits


def prepare(case, seed):
    c = dict(case)
    op, page, n = c["op"], c["page"], c["n_seq"]
    gen = torch.Generator(device=DEVICE).manual_seed(int(seed))
    rng = np.random.default_rng(int(seed))
    base, add = _lengths(c, "len"), _lengths(c, "add")
    order = rng.permutation(n)
    base, add = [base[i] for i in order], [add[i] for i in order]
    total = [a + b for a, b in zip(base, add)]
    st = dict(c=c, base=base, add=add, total=total)
    if op in ("tree", "masks"):
        trees = _trees(rng, add)
        cu = np.concatenate([[0], np.cumsum(add)]).astype(np.int32)
        st.update(cu=_ints(cu), tokens=int(cu[-1]) + c["spare"], words=_words(c))
    if op == "masks":
        parents = np.full(st["tokens"], -1, dtype=np.int32)
        parents[:cu[-1]] = np.concatenate(trees)
        st.update(parents=_ints(parents), masks=torch.zeros(st["tokens"], st["words"], dtype=torch.int64, device=DEVICE),
                  depths=torch.zeros(st["tokens"], dtype=torch.int32, device=DEVICE))
        return st
    if op == "free":
        # every fourth sequence shares the first half of its pages with the one before it; rows name more pages than lengths need
        need = [_pages(x + 3 * page * (i % 3 == 0), page) for i, x in enumerate(total)]
        n_pages = sum(need) + sum(need) // 3 + 5
    else:
        need = [_pages(x, page) for x in total]
        n_pages = sum(need) + sum(need) // 8 + 3 + (c["new"] if op == "fork" else 0)
    ids = rng.permutation(n_pages).astype(np.int32)      # pages come from the pool in no order
    table = np.full((n, max(1, max(need))), -1, dtype=np.int32)
    at = 0
    for i, k in enumerate(need):
        table[i, :k] = ids[at:at + k]
        at += k
    if op == "free":
        for i in range(3, n, 4):
            half = min(need[i - 1], need[i]) // 2
            table[i, :half] = table[i - 1, :half]
    st.update(table=torch.from_numpy(table).to(DEVICE), lens=_ints(total), n_pages=n_pages)
    if op == "free":
        st.update(free=torch.full((n_pages,), -1, dtype=torch.int32, device=DEVICE), count=torch.zeros(1, dtype=torch.int32, device=DEVICE))
    else:
        st.update(k_cache=_cache(c, n_pages, gen), v_cache=_cache(c, n_pages, gen))
    if op == "tree":
        bits = np.concatenate([_tree_bits(p, st["words"]) for p in trees])
        # queries of up to four times the keys' size: from maps that look everywhere to ones with a few heavy tokens
        q = torch.empty((st["tokens"], c["heads_q"], c["d"]), dtype=torch.float32, device=DEVICE).normal_(generator=gen)
        q = q * (0.5 + 3.5 * torch.rand((st["tokens"], c["heads_q"], 1), device=DEVICE, generator=gen))
        st.update(q=q.to(_dtype(c)), trees=trees, masks=None if c["chain"] else torch.from_numpy(bits.view(np.int64)).to(DEVICE))
    elif op == "compact":
        most = max(1, max(int(round(a * c["kept"])) for a in add))
        keep, count = np.full((n, most), -1, dtype=np.int32), []
        for i, a in enumerate(add):
            k = int(round(a * c["kept"]))
            keep[i, :k] = np.sort(rng.permutation(a)[:k])
            count.append(k)
        st.update(start=_ints(base), keep=_ints(keep), count=_ints(count))
    elif op == "fork":
        m = c["new"]
        parents = rng.integers(0, n, m).astype(np.int32)
        st.update(parents=_ints(parents), free=_ints(rng.permutation(ids[at:])))
    if own:
        from paper_2605_19726_amd import binding as bd
        if op == "free":
            st["ws"] = torch.empty(bd.page_free_workspace_size(st["table"], n_pages), dtype=torch.uint8, device=DEVICE)
        else:
            st["cache"] = bd.PagedCache(st["k_cache"], st["v_cache"])
        if op == "tree":
            st["out"] = torch.empty_like(st["q"])
            st["ws"] = torch.empty(bd.tree_workspace_size(st["q"], st["cache"], st["table"]), dtype=torch.uint8, device=DEVICE)
        elif op == "fork":
            st["fork"] = bd.PageFork(c["new"], table.shape[1], DEVICE)
            st["fork"].table.fill_(-1)
    return st


# ---------------------------------------------------------------- plain forms
def _rounds(most):
    return max(1, int(most)).bit_length()


def _plain_masks(st):
    """Ancestors by doubling: after k rounds a token has its 2^k nearest."""
    T, W, cu, n = st["tokens"], st["words"], st["cu"].long(), st["c"]["n_seq"]
    t = torch.arange(T, device=DEVICE)
    seq = torch.searchsorted(cu[1:], t, right=True)
    inside = seq < n
    first = cu[seq.clamp(max=n - 1)]
    own_at, par = t - first, st["parents"].long()
    follows = inside & (par >= 0) & (par < own_at)
    up = torch.where(follows, first + par, T)                                # T: the root, which has no bits
    bit = torch.where((torch.arange(W, device=DEVICE) == (own_at // 64)[:, None]) & inside[:, None], 1 << (own_at % 64)[:, None], 0)
    bits = torch.cat([bit, torch.zeros(1, W, dtype=torch.int64, device=DEVICE)])
    depth = torch.cat([follows.long(), torch.zeros(1, dtype=torch.int64, device=DEVICE)])
    up = torch.cat([up, torch.full((1,), T, dtype=torch.int64, device=DEVICE)])
    for _ in range(_rounds(st["c"]["add_hi"])):
        bits, depth, up = bits | bits[up], depth + depth[up], up[up]
    st["masks"].copy_(torch.where(inside[:, None], bits[:T], st["masks"]))
    st["depths"].copy_(torch.where(inside, depth[:T], st["depths"].long()))
    return dict(masks=st["masks"], depths=st["depths"])


def _plain_tree(st):
    """Sequences padded to the longest, and the trees to the largest, of their part; parts of at most 2^29 scores."""
    c, q, table = st["c"], st["q"], st["table"]
    page, hk, hq, d, n = c["page"], c["heads_kv"], c["heads_q"], c["d"], c["n_seq"]
    group, masks, cu, lens = hq // hk, st["masks"], st["cu"].long(), st["lens"].long()
    out, lse = torch.empty_like(q), torch.empty(q.shape[:2], dtype=torch.float32, device=DEVICE)
    a = 0
    while a < n:
        b, most, wide = a + 1, st["total"][a], st["add"][a]
        while b < n and max(most, st["total"][b]) * max(wide, st["add"][b]) * (b - a + 1) * hq <= 2 ** 29 and \
                max(most, st["total"][b]) * (b - a + 1) * hk * d <= 2 ** 30:
            most, wide, b = max(most, st["total"][b]), max(wide, st["add"][b]), b + 1
        w, m = max(1, _pages(most, page)), b - a
        ids = table[a:b, :w].clamp(min=0).long()
        k, v = (x[ids].permute(0, 2, 1, 3, 4).reshape(m, hk, w * page, d).float() for x in (st["k_cache"], st["v_cache"]))
        r = torch.arange(wide, device=DEVICE)
        rows = (cu[a:b, None] + r).clamp(max=st["tokens"] - 1)                # [m, wide]; those behind a tree's end are not stored
        real = r < (cu[a + 1:b + 1] - cu[a:b])[:, None]
        pos = torch.arange(w * page, device=DEVICE)
        start = lens[a:b] - (cu[a + 1:b + 1] - cu[a:b])
        at = pos[None] - start[:, None]                                       # [m, L] place among the drafted tokens
        if masks is None:
            seen = at[:, None, :] <= r[None, :, None]
        else:
            word = torch.gather(masks[rows], 2, (at.clamp(min=0) // 64).clamp(max=masks.shape[1] - 1)[:, None, :].expand(m, wide, w * page))
            seen = (((word >> (at.clamp(min=0) % 64)[:, None, :]) & 1) == 1) | (at < 0)[:, None, :]
        seen = seen & (pos < lens[a:b, None])[:, None, :]
        qf = q[rows].float().reshape(m, wide, hk, group, d).permute(0, 2, 1, 3, 4).reshape(m, hk, wide * group, d)
        s = torch.matmul(qf, k.transpose(2, 3)) / math.sqrt(d)
        s = s.reshape(m, hk, wide, group, w * page).masked_fill(~seen[:, None, :, None, :], -math.inf).reshape(m, hk, wide * group, w * page)
        top = s.max(3, keepdim=True).values
        top = torch.where(top == -math.inf, 0.0, top)
        p = torch.exp(s - top)
        z = p.sum(3, keepdim=True)
        v = v.masked_fill((pos >= lens[a:b, None])[:, None, :, None], 0.0)
        o = torch.matmul(p, v) / torch.where(z == 0, 1.0, z)
        o = o.reshape(m, hk, wide, group, d).permute(0, 2, 1, 3, 4).reshape(m, wide, hq, d)
        e = (top + torch.log(z)).reshape(m, hk, wide, group).permute(0, 2, 1, 3).reshape(m, wide, hq)
        first, last = sum(st["add"][:a]), sum(st["add"][:b])
        out[first:last] = o[real].to(q.dtype)
        lse[first:last] = e[real]
        a = b
    return dict(out=out, lse=lse)


def _plain_compact(st):
    page, table, start, keep, count = st["c"]["page"], st["table"], st["start"].long(), st["keep"].long(), st["count"].long()
    j = torch.arange(keep.shape[1], device=DEVICE)
    used = j < count[:, None]
    seq = torch.arange(len(start), device=DEVICE)[:, None].expand_as(keep)[used]
    to, of = (start[:, None] + j).expand_as(keep)[used], (start[:, None] + keep)[used]
    k, v = (x[table[seq, of // page].long(), :, of % page] for x in (st["k_cache"], st["v_cache"]))
    at, off = table[seq, to // page].long(), to % page
    st["k_cache"][at, :, off] = k
    st["v_cache"][at, :, off] = v
    return dict(k_cache=st["k_cache"], v_cache=st["v_cache"])


def _plain_fork(st):
    page, table, parents, free = st["c"]["page"], st["table"], st["parents"].long(), st["free"]
    m, n = len(parents), len(table)
    lens = st["lens"].long()[parents]
    j = torch.arange(m, device=DEVICE)
    first = torch.full((n,), m, dtype=torch.int64, device=DEVICE).scatter_reduce(0, parents, j, "amin")
    rest = lens % page
    need = ((rest != 0) & (first[parents] != j)).long()
    asked = torch.cumsum(need, 0)
    served = (need == 0) | (asked <= free.numel())
    pool = torch.cat([free, torch.full((1,), -1, dtype=torch.int32, device=DEVICE)])
    fresh = pool[(asked - 1).clamp(0, free.numel())]
    copied = (need == 1) & served
    col = torch.arange(table.shape[1], device=DEVICE)
    rows = table[parents]
    last = (lens // page)[:, None]
    rows = torch.where((col == last) & copied[:, None], fresh[:, None], rows)
    used = (col < ((lens + page - 1) // page)[:, None]) & served[:, None]
    new_table = torch.where(used, rows, -1).int()
    source = torch.gather(table[parents], 1, last.clamp(max=table.shape[1] - 1))[:, 0]
    copies = torch.where(copied[:, None], torch.stack([source, fresh, rest.int()], 1), torch.tensor([-1, -1, 0], dtype=torch.int32, device=DEVICE))
    pages = torch.stack([torch.where(copied, asked, 0).max(), asked[-1]]).int()
    place = torch.arange(page, device=DEVICE)
    which, off = (copied[:, None] & (place < rest[:, None])).nonzero(as_tuple=True)
    for x in (st["k_cache"], st["v_cache"]):
        x[fresh[which].long(), :, off] = x[source[which].long(), :, off]
    return dict(table=new_table, lens=torch.where(served, lens, 0).int(), copies=copies, pages=pages, k_cache=st["k_cache"], v_cache=st["v_cache"])


def _plain_free(st):
    page, table, lens, n_pages = st["c"]["page"], st["table"], st["lens"], st["n_pages"]
    held = torch.arange(table.shape[1], device=DEVICE) < ((lens + page - 1) // page)[:, None]
    used = torch.zeros(n_pages + 1, dtype=torch.bool, device=DEVICE)
    used[torch.where(held & (table >= 0) & (table < n_pages), table, n_pages).long().reshape(-1)] = True
    free = ~used[:n_pages]
    place = torch.cumsum(free, 0)
    count = place[-1]
    ids = torch.cat([st["free"], st["free"][:1]])
    ids[torch.where(free, place - 1, n_pages)] = torch.arange(n_pages, device=DEVICE, dtype=torch.int32)
    st["free"].copy_(ids[:n_pages])
    return dict(free=st["free"], count=count.reshape(1).int())


def run(st):
    op = st["c"]["op"]
    if not own:
        return {"masks": _plain_masks, "tree": _plain_tree, "compact": _plain_compact, "fork": _plain_fork, "free": _plain_free}[op](st)
    from paper_2605_19726_amd import binding as bd
    if op == "masks":
        masks, depths = bd.basa_tree_masks(st["parents"], st["cu"], st["words"], out=(st["masks"], st["depths"]))
        return dict(masks=masks, depths=depths)
    if op == "tree":
        out, lse = bd.basa_tree_attn(st["q"], st["cache"], st["table"], st["lens"], st["cu"], st["masks"], want_lse=True, ws=st["ws"],
                                     out=st["out"])
        return dict(out=out, lse=lse)
    if op == "compact":
        bd.basa_cache_compact(st["cache"], st["table"], st["start"], st["keep"], st["count"])
        return dict(k_cache=st["k_cache"], v_cache=st["v_cache"])
    if op == "fork":
        f = bd.basa_page_fork(st["table"], st["lens"], st["parents"], st["free"], st["c"]["page"], out=st["fork"])
        bd.basa_cache_copy(st["cache"], f.copies)
        return dict(table=f.table, lens=f.lens, copies=f.copies, pages=f.pages, k_cache=st["k_cache"], v_cache=st["v_cache"])
    free, count = bd.basa_page_free(st["table"], st["lens"], st["c"]["page"], st["n_pages"], out=(st["free"], st["count"]), ws=st["ws"])
    return dict(free=free, count=count)


def work(case):
    """Every input that the operator needs read once, every output written once; 4 d flops for a query head and a token that it sees."""
    c = case
    page, e = c["page"], 4 if c["dtype"] == "f32" else 2
    n, hk, hq, d = c["n_seq"], c["heads_kv"], c["heads_q"], c["d"]
    base, add = _lengths(c, "len"), _lengths(c, "add")
    total = sum(base) + sum(add)
    row = 2.0 * hk * d * e                               # a token's K and V
    if c["op"] == "masks":
        return {"bytes": 8.0 * sum(add) + 8.0 * sum(add) * _words(c) + 4.0 * (n + 1), "flops": 0.0}
    if c["op"] == "tree":
        # (which length meets which tree goes by the seed: products on average; of the tree, every token itself)
        pairs = sum(base) * sum(add) / n + sum(add)
        masks = 0.0 if c["chain"] else 8.0 * sum(add) * _words(c)
        return {"bytes": total * row + 4.0 * total / page + 2.0 * sum(add) * hq * d * e + 4.0 * sum(add) * hq + masks + 8.0 * n, "flops": 4.0 * d * hq * pairs}
    if c["op"] == "compact":
        moved = sum(round(a * c["kept"]) * (c["kept"] < 1) for a in add)
        return {"bytes": 2.0 * moved * row + 4.0 * sum(round(a * c["kept"]) for a in add) + 12.0 * n, "flops": 0.0}
    if c["op"] == "fork":
        # (which are forked, and which of their pages are not full, goes by the seed: on average)
        m = c["new"]
        chosen = n * (1 - (1 - 1 / n) ** m)
        copied = max(0.0, m - chosen) * (1 - 1 / page)
        return {"bytes": 8.0 * m * total / n / page + 16.0 * m + 2.0 * copied * page / 2 * row, "flops": 0.0}
    held = total / page
    return {"bytes": 4.0 * held + 4.0 * n + 4.0 * held / 3, "flops": 0.0}


def exact(case, seed):
    """The operators' definitions, one sequence after the other: whole numbers and copies as they are, attention in 64 bits."""
    st = prepare(case, seed)
    c = st["c"]
    op, page, hk, hq, d, n = c["op"], c["page"], c["heads_kv"], c["heads_q"], c["d"], c["n_seq"]
    if op == "masks":
        parents, cu = st["parents"].cpu().numpy(), st["cu"].tolist()
        masks, depths = np.zeros((st["tokens"], st["words"]), dtype=np.uint64), np.zeros(st["tokens"], dtype=np.int32)
        for i in range(n):
            for r in range(cu[i + 1] - cu[i]):
                at, up = cu[i] + r, r
                while True:
                    masks[at, up // 64] |= np.uint64(1 << (up % 64))
                    nxt = int(parents[cu[i] + up])
                    if not 0 <= nxt < up:
                        break
                    up, depths[at] = nxt, depths[at] + 1
        return dict(masks=torch.from_numpy(masks.view(np.int64)), depths=torch.from_numpy(depths))
    table = st["table"].cpu().numpy().astype(np.int64)
    if op == "free":
        used = np.zeros(st["n_pages"], dtype=bool)
        for i, x in enumerate(st["total"]):
            used[table[i, :_pages(x, page)]] = True
        ids = np.flatnonzero(~used).astype(np.int32)
        free = np.full(st["n_pages"], -1, dtype=np.int32)
        free[:len(ids)] = ids
        return dict(free=torch.from_numpy(free), count=torch.tensor([len(ids)], dtype=torch.int32))
    k_rows, v_rows = (st[x].permute(0, 2, 1, 3).reshape(-1, hk, d) for x in ("k_cache", "v_cache"))    # by slot
    slots = lambda i, t: table[i, t // page] * page + t % page                  # noqa: E731
    paged = lambda x: x.reshape(-1, page, hk, d).permute(0, 2, 1, 3)            # noqa: E731
    if op == "compact":
        keep, count, src, dst = st["keep"].cpu().numpy(), st["count"].tolist(), [], []
        for i in range(n):
            src.append(slots(i, st["base"][i] + keep[i, :count[i]].astype(np.int64)))
            dst.append(slots(i, st["base"][i] + np.arange(count[i], dtype=np.int64)))
        src, dst = (torch.from_numpy(np.concatenate(x)).to(DEVICE) for x in (src, dst))
        return {name: paged(x.clone().index_copy_(0, dst, x.index_select(0, src))) for name, x in (("k_cache", k_rows), ("v_cache", v_rows))}
    if op == "fork":
        m, free, taken, seen, asked = c["new"], st["free"].tolist(), 0, set(), 0
        new_table, lens, copies = np.full((m, table.shape[1]), -1, dtype=np.int32), np.zeros(m, dtype=np.int32), np.full((m, 3), -1, dtype=np.int32)
        copies[:, 2] = 0
        src, dst = [np.zeros(0, dtype=np.int64)], [np.zeros(0, dtype=np.int64)]
        for j, p in enumerate(st["parents"].tolist()):
            L = st["total"][p]
            whole, rest = divmod(L, page)
            again = rest > 0 and p in seen
            seen.add(p)
            asked += again
            if again and asked > len(free):
                continue
            lens[j] = L
            new_table[j, :_pages(L, page)] = table[p, :_pages(L, page)]
            if again:
                taken = asked
                copies[j] = table[p, whole], free[asked - 1], rest
                new_table[j, whole] = free[asked - 1]
                src.append(table[p, whole] * page + np.arange(rest))
                dst.append(free[asked - 1] * page + np.arange(rest))
        src, dst = (torch.from_numpy(np.concatenate(x)).to(DEVICE) for x in (src, dst))
        k, v = (paged(x.clone().index_copy_(0, dst, x.index_select(0, src))) for x in (k_rows, v_rows))
        return dict(table=torch.from_numpy(new_table), lens=torch.from_numpy(lens), copies=torch.from_numpy(copies),
                    pages=torch.tensor([taken, asked], dtype=torch.int32), k_cache=k, v_cache=v)
    group, cu = hq // hk, st["cu"].tolist()
    out = torch.zeros(st["q"].shape, dtype=torch.float64, device=DEVICE)
    lse = torch.full(st["q"].shape[:2], -math.inf, dtype=torch.float64, device=DEVICE)
    for i in range(n):
        L, A = st["total"][i], st["add"][i]
        if A == 0:
            continue
        rows = torch.from_numpy(slots(i, np.arange(L, dtype=np.int64))).to(DEVICE)
        see = np.ones((A, L), dtype=bool)
        if c["chain"]:
            see[:, L - A:] = np.tril(np.ones((A, A), dtype=bool))
        else:
            see[:, L - A:] = False
            for r in range(A):
                up = r
                while up >= 0:
                    see[r, L - A + up] = True
                    up = int(st["trees"][i][up])
        hidden = ~torch.from_numpy(see).to(DEVICE)
        for g in range(hk):
            k, v = k_rows[:, g].index_select(0, rows).double(), v_rows[:, g].index_select(0, rows).double()
            heads = slice(g * group, (g + 1) * group)
            s = torch.mm(st["q"][cu[i]:cu[i] + A, heads].reshape(A * group, d).double(), k.t()) * d ** -0.5
            s = s.reshape(A, group, L).masked_fill(hidden[:, None], -math.inf).reshape(A * group, L)
            lse[cu[i]:cu[i] + A, heads] = torch.logsumexp(s, 1).reshape(A, group)
            out[cu[i]:cu[i] + A, heads] = torch.mm(torch.softmax(s, 1), v).reshape(A, group, d)
    return dict(out=out, lse=lse)
