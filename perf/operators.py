"""Operators of a paged key-value cache, as a serving loop around the block-sparse prefill uses them: listed cases, the ranges they
stand for, their plain forms and their values in 64 bits.

  op "tables"  block tables and slot maps of one step, built from the request lengths (`basa_page_tables`)
  op "append"  new tokens' keys and values written to their slots of the pages (`basa_cache_append`)
  op "gather"  cached keys and values read back from the pages into packed rows, for a prompt that goes on (`basa_cache_gather`)
  op "decode"  attention of one new token of every sequence over its pages (`basa_decode_attn`)

A cache of K or V is indexed [pages, heads_kv, page, d] and stored that way ("head" layout) or token-major, [pages, page, heads_kv, d]
("token" layout).  Sequence i owns the pages table[i, 0 .. ceil(len_i / page)); its token t lives in page table[i, t // page] at offset
t % page, slot number page id * page + offset.  Lengths of a case are the same for every seed, in another order; which pages hold a
sequence, and all values, go by the seed.
"""
import math
import random

import numpy as np
import torch

own = False

DEVICE = "cuda"
DEFAULTS = dict(op="decode", dtype="bf16", heads_q=32, heads_kv=8, d=128, page=64, layout="head", n_seq=1, len_lo=1, len_hi=1,
                add_lo=0, add_hi=0, spare=0, shape=1)


def _case(**kw):
    c = dict(DEFAULTS)
    c.update(kw)
    return c


def listed():
    return [
        # one decode step of a small batch: every sequence grows by one token, few need a page; latency
        _case(name="tables_step_8", op="tables", n_seq=8, page=16, len_lo=40, len_hi=8000, add_lo=1, add_hi=1),
        # prompts of very different lengths enter an empty cache, the slot map padded to the batch's capacity
        _case(name="tables_prompts_40", op="tables", n_seq=40, page=16, len_lo=0, len_hi=0, add_lo=60, add_hi=9000, spare=700),
        # a decode step of a large batch, as a mixed step: most sequences add one token, some a chunk of their prompt
        _case(name="tables_mixed_600", op="tables", n_seq=600, page=64, len_lo=0, len_hi=20000, add_lo=0, add_hi=150, spare=9),
        # the new tokens of a decode step
        _case(name="append_step_64", op="append", n_seq=64, add_lo=1, add_hi=1, len_lo=100, len_hi=4000, page=64),
        # a packed batch of prompts, keys and values as slices of one projection's output, pages stored token-major
        _case(name="append_prompts_41k", op="append", n_seq=12, add_lo=900, add_hi=9000, len_lo=0, len_hi=0, page=16, layout="token"),
        # fp32 heads of 64, a page size that is no power of two
        _case(name="append_f32_p100", op="append", dtype="f32", d=64, heads_kv=4, n_seq=7, add_lo=130, add_hi=2500, len_lo=0, len_hi=300,
              page=100),
        # the context of one long conversation, read back for the next block of its queries
        _case(name="gather_32k", op="gather", n_seq=1, len_lo=32768, len_hi=32768, page=64),
        # several of them, ragged, small pages stored token-major
        _case(name="gather_ragged_20", op="gather", n_seq=20, len_lo=37, len_hi=14000, page=16, layout="token", heads_kv=5, heads_q=5),
        # one short sequence: latency
        _case(name="decode_one_700", n_seq=1, len_lo=700, len_hi=700, page=16),
        # fp32, a head of keys for every query head, heads of 64, lengths from a few tokens on
        _case(name="decode_f32_mha_d64", dtype="f32", heads_q=16, heads_kv=16, d=64, page=100, n_seq=21, len_lo=3, len_hi=5000),
        # one sequence of 128K tokens: the length has to be split
        _case(name="decode_128k", n_seq=1, len_lo=131072, len_hi=131072, page=128),
        # a full batch of long contexts of unequal lengths, pages stored token-major
        _case(name="decode_64_long", n_seq=64, len_lo=8000, len_hi=60000, page=64, layout="token"),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


MOST_ELEMENTS = 1.6e9        # of K in a drawn case's cache: below the largest listed one


def draw(rng):
    """One more case: sizes spread over their logarithm, most of them no multiple of anything."""
    op = rng.choice(["tables", "append", "gather", "decode", "decode"])
    hk, d = rng.choice([1, 2, 4, 5, 8, 16, 32]), rng.choice([64, 128])
    group = rng.choice([1, 2, 4, 5, 7, 8, 16, 20, 40])
    while hk * group > 128:
        group //= 2
    c = _case(op=op, heads_kv=hk, heads_q=hk * group, d=d, page=rng.choice([1, 16, 20, 32, 64, 100, 128, 256]),
              dtype=rng.choice(["bf16", "bf16", "f32"]), layout=rng.choice(["head", "token"]), shape=rng.randint(1, 1 << 30))
    if op == "tables":
        n = _log(rng, 1, 2000)
        add = _log(rng, 1, max(2, min(20000, 200000 // n)))
        c.update(n_seq=n, len_lo=0, len_hi=_log(rng, 1, 20000), add_lo=rng.choice([0, 1, add]), add_hi=add, spare=rng.randint(0, 500),
                 page=rng.choice([16, 20, 32, 64, 100, 128, 256]))
    elif op == "append":
        n = _log(rng, 1, 256)
        add = _log(rng, 1, max(2, 80000 // n))
        c.update(n_seq=n, add_lo=rng.choice([0, 1, add]), add_hi=add, len_lo=0, len_hi=_log(rng, 1, 500))
    elif op == "gather":
        n = _log(rng, 1, 40)
        hi = _log(rng, 2, max(3, 120000 // n))
        c.update(n_seq=n, len_lo=rng.choice([0, 1, hi]), len_hi=hi)
    else:
        n = _log(rng, 1, 300)
        hi = _log(rng, 2, max(3, min(400000, int(MOST_ELEMENTS / (hk * d) / n))))
        c.update(n_seq=n, len_lo=rng.choice([0, 1, max(1, hi // 3), hi]), len_hi=hi)
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


def _cache(c, n_pages, gen, fill):
    """One of K and V: [pages, heads_kv, page, d] in the case's layout."""
    hk, page, d = c["heads_kv"], c["page"], c["d"]
    shape = (n_pages, hk, page, d) if c["layout"] == "head" else (n_pages, page, hk, d)
    x = torch.empty(shape, dtype=_dtype(c), device=DEVICE)
    if fill:
        x.normal_(generator=gen)
    else:
        x.zero_()
    return x if c["layout"] == "head" else x.permute(0, 2, 1, 3)


def prepare(case, seed):
    c = dict(case)
    page, n = c["page"], c["n_seq"]
    gen = torch.Generator(device=DEVICE).manual_seed(int(seed))
    rng = np.random.default_rng(int(seed))
    have, add = _lengths(c, "len"), _lengths(c, "add")
    order = rng.permutation(n)
    have, add = [have[i] for i in order], [add[i] for i in order]
    total = [a + b for a, b in zip(have, add)] if c["op"] != "decode" else have
    held = [_pages(x, page) for x in (have if c["op"] == "tables" else total)]
    taken = sum(_pages(x, page) for x in total)
    n_pages = taken + taken // 8 + 3
    ids = rng.permutation(n_pages).astype(np.int32)      # pages come from the pool in no order
    width = max(1, max(_pages(x, page) for x in total)) + (5 if c["op"] == "tables" else 0)
    table = np.full((n, width), -1, dtype=np.int32)
    at = 0
    for i, k in enumerate(held):
        table[i, :k] = ids[at:at + k]
        at += k
    st = dict(c=c, table=torch.from_numpy(table).to(DEVICE), have=have, add=add)
    if c["op"] == "tables":
        st.update(have=_ints(have), add=_ints(add), free=torch.from_numpy(ids[at:].copy()).to(DEVICE), tokens=sum(add) + c["spare"])
    elif c["op"] == "append":
        T = sum(add)
        slots = []
        for i in range(n):
            t = np.arange(have[i], total[i], dtype=np.int64)
            slots.append(table[i, t // page].astype(np.int64) * page + t % page)
        st.update(slots=torch.from_numpy(np.concatenate(slots)).to(DEVICE), k_cache=_cache(c, n_pages, gen, False),
                  v_cache=_cache(c, n_pages, gen, False))
        # a projection's output: query, key and value heads of a token side by side
        hq, hk = c["heads_q"], c["heads_kv"]
        qkv = torch.empty((max(1, T), hq + 2 * hk, c["d"]), dtype=_dtype(c), device=DEVICE).normal_(generator=gen)[:T]
        st.update(k=qkv[:, hq:hq + hk], v=qkv[:, hq + hk:])
    elif c["op"] == "gather":
        cu = np.concatenate([[0], np.cumsum(total)]).astype(np.int32)
        st.update(cu=torch.from_numpy(cu).to(DEVICE), tokens=int(cu[-1]), lens=_ints(total), k_cache=_cache(c, n_pages, gen, True),
                  v_cache=_cache(c, n_pages, gen, True))
    else:
        st.update(k_cache=_cache(c, n_pages, gen, True), v_cache=_cache(c, n_pages, gen, True), lens=_ints(have))
        # queries of up to four times the keys' size: from maps that look everywhere to ones with a few heavy tokens
        q = torch.empty((n, c["heads_q"], c["d"]), dtype=torch.float32, device=DEVICE).normal_(generator=gen)
        q = q * (0.5 + 3.5 * torch.rand((n, c["heads_q"], 1), device=DEVICE, generator=gen))
        st["q"] = q.to(_dtype(c))
    if own:
        from paper_2605_19726_amd import binding as bd
        if c["op"] == "tables":
            st["out"] = bd.PageTables(n, st["tokens"], DEVICE)
        else:
            st["cache"] = bd.PagedCache(st["k_cache"], st["v_cache"])
        if c["op"] == "decode":
            st["out"] = torch.empty_like(st["q"])
            st["ws"] = torch.empty(bd.decode_workspace_size(st["q"], st["cache"], st["table"]), dtype=torch.uint8, device=DEVICE)
    return st


# ---------------------------------------------------------------- plain forms
def _plain_tables(st):
    table, have, add, free, page, T = st["table"], st["have"], st["add"], st["free"], st["c"]["page"], st["tokens"]
    n, width = table.shape
    have64, add64 = have.long().clamp(min=0), add.long().clamp(min=0)
    ends = torch.cumsum(add64, 0)
    starts = ends - add64
    tot = have64 + add64
    held, after = (have64 + page - 1) // page, (tot + page - 1) // page
    fits = (tot <= width * page) & (ends <= T)
    need = torch.where(fits, after - held, 0)
    asked = torch.cumsum(need, 0)
    first = asked - need
    served = fits & (asked <= free.numel())
    pool = torch.cat([free.long(), torch.full((1,), -1, device=DEVICE, dtype=torch.int64)])
    j = torch.arange(width, device=DEVICE)
    opened = (j >= held[:, None]) & (j < after[:, None]) & served[:, None]
    table.copy_(torch.where(opened, pool[(first[:, None] + j - held[:, None]).clamp(0, free.numel())], table.long()))
    t = torch.arange(T, device=DEVICE)
    seq = torch.searchsorted(ends, t, right=True)
    inside = seq < n
    seq = seq.clamp(max=n - 1)
    pos = (have64[seq] + t - starts[seq]).clamp(min=0)
    entry = table[seq, (pos // page).clamp(max=width - 1)].long()
    slots = torch.where(inside & served[seq] & (entry >= 0), entry * page + pos % page, -1)
    lens = torch.where(served, tot, have64).int()
    cu = torch.cat([torch.zeros(1, device=DEVICE, dtype=torch.int64), ends]).int()
    pages = torch.stack([torch.where(served, asked, 0).max(), asked[-1]]).int()
    return dict(table=table, slots=slots, lens=lens, cu=cu, pages=pages)


def _plain_append(st):
    page, slots = st["c"]["page"], st["slots"]
    at, off = slots // page, slots % page
    st["k_cache"][at, :, off] = st["k"]
    st["v_cache"][at, :, off] = st["v"]
    return dict(k_cache=st["k_cache"], v_cache=st["v_cache"])


def _plain_gather(st):
    page, table, lens, T = st["c"]["page"], st["table"], st["lens"], st["tokens"]
    seq = torch.repeat_interleave(torch.arange(len(lens), device=DEVICE), lens.long(), output_size=T)
    pos = torch.arange(T, device=DEVICE) - st["cu"].long()[seq]
    at, off = table[seq, pos // page].long(), pos % page
    return dict(k=st["k_cache"][at, :, off], v=st["v_cache"][at, :, off])


def _plain_decode(st):
    """Sequences padded to the longest of their part; a part holds at most 2^31 padded elements of K."""
    c, q, lens, table = st["c"], st["q"], st["lens"], st["table"]
    page, hk, d, n = c["page"], c["heads_kv"], c["d"], c["n_seq"]
    group = c["heads_q"] // hk
    out, lse = torch.empty_like(q), torch.empty(q.shape[:2], dtype=torch.float32, device=DEVICE)
    a = 0
    while a < n:
        b, most = a, 0
        while b < n and max(most, st["have"][b], 1) * (b - a + 1) * hk * d <= max(2 ** 31, max(st["have"][a], 1) * hk * d):
            most = max(most, st["have"][b], 1)
            b += 1
        w = _pages(most, page)
        ids = table[a:b, :w].clamp(min=0).long()
        k, v = (x[ids].permute(0, 2, 1, 3, 4).reshape(b - a, hk, w * page, d).float() for x in (st["k_cache"], st["v_cache"]))
        dead = torch.arange(w * page, device=DEVICE) >= lens[a:b, None]
        qf = q[a:b].float().reshape(b - a, hk, group, d)
        s = torch.matmul(qf, k.transpose(2, 3)) / math.sqrt(d)
        s = s.masked_fill(dead[:, None, None, :], -math.inf)
        m = s.max(3, keepdim=True).values
        m0 = torch.where(m == -math.inf, 0.0, m)
        p = torch.exp(s - m0)
        z = p.sum(3, keepdim=True)
        v = v.masked_fill(dead[:, None, :, None], 0.0)
        o = torch.matmul(p, v) / torch.where(z == 0, 1.0, z)
        out[a:b] = o.reshape(b - a, hk * group, d).to(q.dtype)
        lse[a:b] = (m0 + torch.log(z)).reshape(b - a, hk * group)
        a = b
    return dict(out=out, lse=lse)


def run(st):
    op = st["c"]["op"]
    if not own:
        return {"tables": _plain_tables, "append": _plain_append, "gather": _plain_gather, "decode": _plain_decode}[op](st)
    from paper_2605_19726_amd import binding as bd
    if op == "tables":
        r = bd.basa_page_tables(st["have"], st["add"], st["table"], st["free"], st["c"]["page"], st["tokens"], out=st["out"])
        return dict(table=st["table"], slots=r.slots, lens=r.lens, cu=r.cu, pages=r.pages)
    if op == "append":
        bd.basa_cache_append(st["k"], st["v"], st["slots"], st["cache"])
        return dict(k_cache=st["k_cache"], v_cache=st["v_cache"])
    if op == "gather":
        k, v = bd.basa_cache_gather(st["cache"], st["table"], st["cu"], st["tokens"])
        return dict(k=k, v=v)
    out, lse = bd.basa_decode_attn(st["q"], st["cache"], st["table"], st["lens"], want_lse=True, ws=st["ws"], out=st["out"])
    return dict(out=out, lse=lse)


def work(case):
    """Every input that the operator needs read once, every output written once; 4 d flops for a query head and a cached token."""
    c = case
    page, e = c["page"], 4 if c["dtype"] == "f32" else 2
    n, hk, hq, d = c["n_seq"], c["heads_kv"], c["heads_q"], c["d"]
    have, add = _lengths(c, "len"), _lengths(c, "add")
    if c["op"] == "tables":                              # lengths and new tokens in, free pages in, table entries, slots, lengths, offsets out
        # (which lengths meet which additions goes by the seed: pages on average)
        opened = min(sum(add), sum(add) / page + n / 2)
        return {"bytes": 8.0 * n + 8.0 * opened + 4.0 * min(n, sum(add)) + 8.0 * (sum(add) + c["spare"]) + 8.0 * n + 12, "flops": 0.0}
    if c["op"] == "append":
        T = sum(add)
        return {"bytes": 4.0 * T * hk * d * e + 8.0 * T, "flops": 0.0}
    if c["op"] == "gather":
        T = sum(a + b for a, b in zip(have, add))
        return {"bytes": 4.0 * T * hk * d * e + 4.0 * T / page + 4.0 * (n + 1), "flops": 0.0}
    T = sum(have)
    return {"bytes": 2.0 * T * hk * d * e + 4.0 * T / page + 2.0 * n * hq * d * e + 8.0 * n * hq, "flops": 4.0 * T * hq * d}


def exact(case, seed):
    """The operators' definitions, one sequence after the other: whole numbers and copies as they are, attention in 64 bits."""
    st = prepare(case, seed)
    c = st["c"]
    page, hk, d = c["page"], c["heads_kv"], c["d"]
    if c["op"] == "tables":
        table = st["table"].cpu().numpy().copy()
        have, add, free = (st[x].cpu().tolist() for x in ("have", "add", "free"))
        slots, cu, lens, asked, given = np.full(st["tokens"], -1, dtype=np.int64), [0], [], 0, 0
        for i, (h, a) in enumerate(zip(have, add)):
            begin = cu[-1]
            cu.append(begin + a)
            lens.append(h)
            if h + a > table.shape[1] * page or begin + a > st["tokens"]:
                continue
            held, after = -(-h // page), -(-(h + a) // page)
            asked += after - held
            if asked > len(free):
                continue
            table[i, held:after] = free[asked - (after - held):asked]
            given = asked
            lens[i] = h + a
            for t in range(a):
                entry = int(table[i, (h + t) // page])
                if entry >= 0:
                    slots[begin + t] = entry * page + (h + t) % page
        return dict(table=torch.from_numpy(table), slots=torch.from_numpy(slots), lens=torch.tensor(lens, dtype=torch.int32),
                    cu=torch.tensor(cu, dtype=torch.int32), pages=torch.tensor([given, asked], dtype=torch.int32))
    k_rows, v_rows = (st[x].permute(0, 2, 1, 3).reshape(-1, hk, d) for x in ("k_cache", "v_cache"))    # by slot
    if c["op"] == "append":
        k_rows, v_rows = k_rows.clone(), v_rows.clone()
        k_rows.index_copy_(0, st["slots"], st["k"].contiguous())
        v_rows.index_copy_(0, st["slots"], st["v"].contiguous())
        return dict(k_cache=k_rows.reshape(-1, page, hk, d).permute(0, 2, 1, 3), v_cache=v_rows.reshape(-1, page, hk, d).permute(0, 2, 1, 3))
    lens, table = st["lens"].cpu().tolist(), st["table"].cpu().numpy().astype(np.int64)
    rows = []
    for i, L in enumerate(lens):
        rows.append(torch.from_numpy((table[i, :_pages(L, page), None] * page + np.arange(page)).reshape(-1)[:L]).to(DEVICE))
    if c["op"] == "gather":
        every = torch.cat(rows)
        return dict(k=k_rows.index_select(0, every), v=v_rows.index_select(0, every))
    group = c["heads_q"] // hk
    out = torch.zeros(st["q"].shape, dtype=torch.float64, device=DEVICE)
    lse = torch.full(st["q"].shape[:2], -math.inf, dtype=torch.float64, device=DEVICE)
    for i, L in enumerate(lens):
        if L == 0:
            continue
        for g in range(hk):
            heads = slice(g * group, (g + 1) * group)
            k, v = k_rows[:, g].index_select(0, rows[i]).double(), v_rows[:, g].index_select(0, rows[i]).double()
            s = torch.mm(st["q"][i, heads].double(), k.t()) * d ** -0.5
            lse[i, heads] = torch.logsumexp(s, 1)
            out[i, heads] = torch.mm(torch.softmax(s, 1), v)
    return dict(out=out, lse=lse)
