"""GPU tests of the attention of several new tokens per sequence over the pages, and of the masks of their trees, against the plain statements of tree_util.py."""
import math

import numpy as np
import pytest
import torch

from paged_util import HALF_STEP, decode_tolerance, new_tables, rows_of, store
from test_gpu_paged import BF, DEV, F32, bits, ints, randn
from tree_util import ancestors, check_tree, mask_words, random_parents
from paper_2605_19726_amd import binding as bd

pytestmark = pytest.mark.gpu
NAN, INF = float("nan"), float("inf")


def trees_of(new, seed):
    rng = np.random.default_rng(seed)
    return [random_parents(n, rng) for n in new]


# ---------------------------------------------------------------- masks
@pytest.mark.parametrize("sizes,words", [([1], 1), ([64], 1), ([65], 2), ([0, 7, 0, 0, 33, 0], 1), ([25] * 8, 1), ([200, 1, 63, 64, 65, 128, 129], 4), ([1000], 16),
                                         ([4096, 3], 64), ([300, 40], 3)])
def test_masks(sizes, words):
    rng = np.random.default_rng(sum(sizes))
    cu = np.concatenate([[3], 3 + np.cumsum(sizes)])
    T = int(cu[-1]) + 5
    parents = rng.integers(-2 ** 31, 2 ** 31 - 1, T).astype(np.int32)            # rows of no sequence: never looked at
    kinds = []
    for i, n in enumerate(sizes):
        p = [random_parents(n, rng), np.arange(n) - 1, random_parents(n, rng, 200), np.full(n, -5)][i % 4].astype(np.int32)
        if n > 5 and i % 2 == 0:                                                 # no parents: the token itself, one behind it, far ones
            p[n // 2], p[n // 3], p[n - 1] = n // 2, n - 1, 2 ** 31 - 1
        parents[cu[i]:cu[i + 1]] = p
        kinds.append(p)
    masks, depths = torch.full((T, words + 2), -7, dtype=torch.int64, device=DEV), torch.full((T,), -7, dtype=torch.int32, device=DEV)
    got, deep = bd.basa_tree_masks(ints(parents), ints(cu), words, out=(masks[:, :words], depths))
    want, want_depth = np.full((T, words + 2), -7, dtype=np.int64), np.full(T, -7)
    for i, p in enumerate(kinds):
        seen = ancestors(p)
        fit = min(len(p), 64 * words)
        want[cu[i]:cu[i] + fit, :words] = mask_words(seen[:fit], words)
        want[cu[i] + fit:cu[i + 1], :words] = 0
        want_depth[cu[i]:cu[i] + fit] = seen[:fit].sum(1) - 1
        want_depth[cu[i] + fit:cu[i + 1]] = -1
    assert np.array_equal(masks.cpu().numpy(), want) and np.array_equal(deep.cpu().numpy(), want_depth)
    a, b = bd.basa_tree_masks(ints(parents), ints(cu), words)                    # buffers of its own
    assert torch.equal(a[3:-5], got[3:-5]) and torch.equal(b[3:-5], deep[3:-5])


def test_masks_of_offsets_that_do_not_ascend_stay_in_bounds_and_of_no_tokens_are_none():
    parents = ints(np.arange(40) - 1)
    for cu in ([0, 30, 10], [50, 20, 90], [-5, 10, 30], [0, 2 ** 31 - 1, 2 ** 31 - 1], [-2 ** 31, 0, 60]):
        bd.basa_tree_masks(parents, ints(cu), 1)
        torch.cuda.synchronize()
    masks, depths = bd.basa_tree_masks(parents[:0], ints([0, 0]), 1)
    assert masks.shape == (0, 1) and depths.shape == (0,)
    bd.basa_tree_masks(parents, ints([0]), 1)


# ---------------------------------------------------------------- attention
class Case:
    """Caches whose rows that no sequence holds are NaN, the table, queries with rows of no sequence around them, masks."""

    def __init__(self, dtype, d, hq, hk, page, lens, new, seed, layout=("head", "head"), q_scale=2.0, width=None, chain=False, around=(2, 3), spare=3):
        rng = np.random.default_rng(seed)
        self.lens, self.new = list(lens), list(new)
        pages = sum(-(-n // page) for n in lens) + spare
        self.table = new_tables(lens, page, pages, rng, width)
        self.k, self.v = (store(pages, hk, page, d, dtype, x, DEV) for x in layout)
        for i, n in enumerate(lens):
            at, off = (x.to(DEV) for x in rows_of(self.table[i], n, page))
            self.k[at, :, off] = randn((n, hk, d), seed * 100 + 2 * i, dtype)
            self.v[at, :, off] = randn((n, hk, d), seed * 100 + 2 * i + 1, dtype)
        self.cu = np.concatenate([[around[0]], around[0] + np.cumsum(new)])
        self.T = int(self.cu[-1]) + around[1]
        self.q = randn((self.T, hq, d), seed + 7, dtype, q_scale)
        self.parents = [random_parents(n, rng) for n in new]
        self.seen = [None if chain else ancestors(p) for p in self.parents]
        self.set_masks()

    def set_masks(self, words=None):
        words = words or max(1, -(-max(self.new) // 64))
        if self.seen[0] is None:
            self.masks = None
            return
        rows = np.full((self.T, words), -1, dtype=np.int64)
        for i, s in enumerate(self.seen):
            rows[self.cu[i]:self.cu[i + 1]] = mask_words(s, words)
        self.masks = torch.from_numpy(rows).to(DEV)

    def cache(self):
        return bd.PagedCache(self.k, self.v)

    def run(self, **kw):
        return bd.basa_tree_attn(self.q, self.cache(), ints(self.table), ints(self.lens), ints(self.cu), self.masks, want_lse=True, **kw)

    def check(self, out, lse, what=""):
        check_tree(out, lse, self.q, self.k, self.v, self.table, self.lens, self.cu, self.seen, what)


LENS = [5, 0, 40, 33, 64, 128, 200, 700, 129, 1031, 17]
NEW = [5, 0, 1, 33, 8, 3, 70, 20, 0, 130, 16]                        # all of a sequence new; none; one; past a word


@pytest.mark.parametrize("dtype,d", [(BF, 128), (BF, 64), (F32, 128), (F32, 64)])
@pytest.mark.parametrize("hq,hk,page,layout,chain", [(4, 4, 16, "head", False), (8, 1, 64, "token", False), (8, 2, 1, "head", True), (10, 2, 20, "token", False),
                                                     (16, 8, 128, "token", True), (14, 2, 100, "head", False), (3, 1, 3, "token", False), (40, 2, 32, "token", False)])
def test_against_64_bits(dtype, d, hq, hk, page, layout, chain):
    c = Case(dtype, d, hq, hk, page, LENS, NEW, hq * 10 + page, (layout, "head"), chain=chain)
    c.check(*c.run(), f"{dtype} d={d} {hq}/{hk} page={page} chain={chain}")


# rows of a KV head per sequence up to 16, 32, 64 and beyond: each way of putting them together, in one launch and cut
@pytest.mark.parametrize("dtype,d", [(BF, 128), (BF, 64), (F32, 128), (F32, 64)])
@pytest.mark.parametrize("new", [1, 4, 7, 15, 33, 70])
@pytest.mark.parametrize("lens", [[500, 90, 71], [3000, 71, 900], [9000]])
def test_tiles_and_runs(dtype, d, new, lens):
    c = Case(dtype, d, 8, 2, 32, lens, [new] * len(lens), new + len(lens))
    out, lse = c.run()
    c.check(out, lse, f"{dtype} d={d} {new} new, {lens}")
    again, lse2 = c.run()
    rows = slice(int(c.cu[0]), int(c.cu[-1]))
    assert torch.equal(bits(out[rows]), bits(again[rows])) and torch.equal(lse[rows], lse2[rows])


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("hq,hk,lens,new,chain", [(4, 1, [70001], [5], False), (8, 2, [20000, 3, 9999], [64, 3, 1], False), (2, 2, [40000, 0, 64, 33333], [1, 0, 64, 9], True),
                                                  (20, 1, [30011, 17], [13, 17], False), (32, 4, [6000], [300], True), (16, 16, [1500] * 9, [31] * 9, False)])
def test_long_sequences_are_split_and_joined(dtype, hq, hk, lens, new, chain):
    c = Case(dtype, 128, hq, hk, 64, lens, new, 3, chain=chain)
    c.check(*c.run(), f"{dtype} {hq}/{hk} {lens}")


# rows of the table with room for 64 to 512 tokens: up to some number of them sequences are not cut, and few rows have rings of two steps
@pytest.mark.parametrize("dtype,d", [(BF, 128), (BF, 64), (F32, 128), (F32, 64)])
@pytest.mark.parametrize("room", [64, 80, 128, 144, 256, 272, 512, 528])
@pytest.mark.parametrize("n,new", [(1, 5), (3, 17), (70, 2)])
def test_short_sequences(dtype, d, room, n, new):
    rng = np.random.default_rng(room + n)
    lens = rng.integers(new, room + 1, n)
    lens[0] = room
    count = rng.integers(0, new + 1, n)
    count[0] = new
    c = Case(dtype, d, 10, 5, 16, lens.tolist(), count.tolist(), room + new, width=room // 16)
    c.check(*c.run(), f"{dtype} d={d} room for {room}, {n} sequences, {new} new")


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("n,width", [(513, 8), (700, 40)])
def test_many_sequences_in_a_mixed_step(dtype, n, width):
    rng = np.random.default_rng(n)
    new = rng.integers(0, 3, n)
    new[5], new[n - 1], new[n - 2] = 90, 40, 0
    lens = np.maximum(rng.integers(0, 120, n), new)
    c = Case(dtype, 64, 4, 2, 16, lens.tolist(), new.tolist(), 11, width=width)
    c.check(*c.run())


def test_one_new_token_agrees_with_the_single_token_attention():
    for dtype in (BF, F32):
        c = Case(dtype, 128, 16, 4, 16, [700, 33, 1, 5000], [1, 1, 1, 1], 5, around=(0, 0), chain=True)
        out, lse = c.run()
        one, lse1 = bd.basa_decode_attn(c.q, c.cache(), ints(c.table), ints(c.lens), want_lse=True)
        c.check(out, lse)
        c.check(one, lse1)


def test_rows_of_no_sequence_and_what_lies_between_strided_rows_stay_as_they_were():
    for dtype in (BF, F32):
        c = Case(dtype, 64, 6, 2, 20, [100, 900, 30], [10, 40, 0], 9, around=(3, 5))
        wide = torch.full((c.T, 11, 64 + 16), 5.0, dtype=dtype, device=DEV)
        out = wide[:, 2:8, :64]
        qkv = torch.full((c.T, 6 + 3, 64), NAN, dtype=dtype, device=DEV)               # queries as a slice of a projection
        qkv[:, 1:7] = c.q
        c.q = qkv[:, 1:7]
        masks = torch.full((c.T, c.masks.shape[1] + 3), -1, dtype=torch.int64, device=DEV)
        masks[:, 1:1 + c.masks.shape[1]] = c.masks
        c.masks = masks[:, 1:1 + c.masks.shape[1]]
        _, lse = c.run(out=out)
        c.check(out, lse)
        kept = torch.ones_like(wide, dtype=torch.bool)
        kept[3:53, 2:8, :64] = False
        assert (wide[kept] == 5.0).all()


def test_outputs_lie_in_no_other_tensor_but_may_lie_between_rows_of_the_queries():
    for dtype in (BF, F32):
        c = Case(dtype, 64, 8, 2, 16, [5000, 300, 30], [10, 40, 0], 9)
        out, lse = c.run()
        both = torch.full((c.T, 16, 64), 5.0, dtype=dtype, device=DEV)
        rows = slice(int(c.cu[0]), int(c.cu[-1]))
        for q, o in ((both[:, :8], both[:, 8:]), (both[:, ::2], both[:, 1::2])):
            q.copy_(c.q)
            _, lse2 = bd.basa_tree_attn(q, c.cache(), ints(c.table), ints(c.lens), ints(c.cu), c.masks, want_lse=True, out=o)
            assert torch.equal(bits(o[rows].contiguous()), bits(out[rows])) and torch.equal(lse2[rows], lse[rows]) and torch.equal(bits(q.contiguous()), bits(c.q))
        for o in (c.q, c.q.new_empty(1, 8, 64).expand(c.T, 8, 64), c.k.reshape(-1)[:c.q.numel()].view(c.q.shape)):
            with pytest.raises(RuntimeError, match="overlap|alias"):
                c.run(out=o)
        need = bd.tree_workspace_size(c.q, c.cache(), ints(c.table))
        ws = torch.empty(need + 2 ** 20, dtype=torch.uint8, device=DEV)
        with pytest.raises(RuntimeError, match="overlap"):
            c.run(ws=ws, out=ws[need // 256 * 256 - 256:][:c.q.numel() * c.q.element_size()].view(dtype).view(c.q.shape))
        behind = ws[-(-need // 256) * 256:][:c.q.numel() * c.q.element_size()].view(dtype).view(c.q.shape)
        c.run(ws=ws, out=behind)
        assert torch.equal(bits(behind[rows]), bits(out[rows]))


def test_masks_of_any_kind():
    """Bits that are no tree's: rows that see nothing at all, not themselves, later ones; bits behind the last new token; fewer words than tokens."""
    for dtype in (BF, F32):
        rng = np.random.default_rng(2)
        c = Case(dtype, 128, 4, 2, 16, [40, 100, 30, 1500], [40, 37, 30, 100], 4)
        c.seen = [rng.random((n, n)) < 0.3 for n in c.new]
        c.seen[0][3] = False
        c.seen[0][20:] = False
        c.seen[2][:] = False
        c.set_masks()
        for i, n in enumerate(c.new):                           # set bits of tokens that are not there
            if n % 64:
                c.masks[int(c.cu[i]):int(c.cu[i + 1]), n // 64] |= -1 << (n % 64)
            c.masks[int(c.cu[i]):int(c.cu[i + 1]), n // 64 + 1:] = -1
        out, lse = c.run()
        c.check(out, lse)
        a = int(c.cu[0])
        assert not out[a + 3].any() and (lse[a + 3] == -INF).all() and not out[a + 20:a + 40].any()
        assert not out[int(c.cu[2]):int(c.cu[3])].any() and (lse[int(c.cu[2]):int(c.cu[3])] == -INF).all()
        c.set_masks(words=1)
        for s in c.seen:
            s[:, 64:] = False
        c.check(*c.run())


def test_what_is_not_seen_may_hold_anything():
    """NaN and infinities in keys and values of new tokens that some rows do not see, in whole pages that are none, and behind the last token."""
    for dtype, d in ((BF, 128), (BF, 64), (F32, 128), (F32, 64)):
        for lens, new in (([300, 70], [40, 70]), ([5000, 70], [40, 70])):
            c = Case(dtype, d, 8, 2, 16, lens, new, 6)
            for i, (n, m) in enumerate(zip(lens, new)):
                at, off = (x.to(DEV) for x in rows_of(c.table[i], n, 16))
                # the last token is a leaf, and so are others: only they see themselves
                leaf = [r for r in range(m) if c.seen[i][:, r].sum() == 1]
                assert m - 1 in leaf
                for x, r in zip((NAN, INF, -INF, NAN), leaf[-4:]):
                    for cache in (c.k, c.v):
                        cache[at[n - m + r], :, off[n - m + r]] = x
            c.table[0, 2] = -1                                  # pages that are none, among the context
            c.table[0, 3] = 2 ** 30
            out, lse = c.run()
            for i, m in enumerate(new):
                a = int(c.cu[i])
                bad = [r for r in range(m) if c.seen[i][:, r].sum() == 1][-4:]
                rows = [r for r in range(m) if r not in bad]
                # every other row is right; these have keys of their own that are not finite
                check_tree(out, lse, c.q, c.k, c.v, c.table, c.lens, c.cu, c.seen, f"{dtype} {d} {lens}", only=(i, rows))
                assert torch.isnan(out[a + m - 1].float()).all()


def test_infinite_values_stay_infinite():
    for dtype, d in ((BF, 128), (F32, 64)):
        c = Case(dtype, d, 4, 1, 16, [200, 3000], [20, 20], 8, q_scale=0.5)
        at, off = (x.to(DEV) for x in rows_of(c.table[0], 200, 16))
        c.v[at[10], 0, off[10], 3] = INF                        # the context: every row
        c.v[at[180], 0, off[180], 5] = -INF                     # new token 0: those that follow it
        c.v[at[11], 0, off[11], 7], c.v[at[12], 0, off[12], 7] = INF, -INF
        out, _ = c.run()
        rows = out[int(c.cu[0]):int(c.cu[1])].float()
        assert (rows[:, :, 3] == INF).all() and torch.isnan(rows[:, :, 7]).all()
        follow = torch.from_numpy(c.seen[0][:, 0]).to(DEV)
        assert (rows[follow][:, :, 5] == -INF).all() and torch.isfinite(rows[~follow][:, :, 5]).all()
        others = [i for i in range(d) if i not in (3, 5, 7)]
        assert torch.isfinite(rows[:, :, others]).all()
        assert torch.isfinite(out[int(c.cu[1]):int(c.cu[2])].float()).all()


# few rows: waves take steps of the same rows side by side, and what is not finite stands in the steps of either
@pytest.mark.parametrize("dtype,d", [(BF, 128), (BF, 64), (F32, 128), (F32, 64)])
@pytest.mark.parametrize("lens", [[300, 40], [5000, 95], [31, 33]])
def test_values_that_are_not_finite_of_few_rows(dtype, d, lens):
    c = Case(dtype, d, 4, 2, 16, lens, [5, 7], 6, q_scale=0.5)
    out, lse = c.run()
    c.check(out, lse)
    for i, n in enumerate(lens):
        at, off = (x.to(DEV) for x in rows_of(c.table[i], n, 16))
        a, m = int(c.cu[i]), c.new[i]
        k, v = c.k.clone(), c.v.clone()
        for t in (0, 16, 33, 65, n - m):                        # of the context: every row; the first new one: those that follow it
            if t >= n:
                continue
            c.v[at[t], 1, off[t], 3] = INF
            got, _ = c.run()
            rows = got[a:a + m].float()
            sees = torch.from_numpy(c.seen[i][:, t - (n - m)]).to(DEV) if t >= n - m else torch.ones(m, dtype=torch.bool, device=DEV)
            assert (rows[sees][:, 2:, 3] == INF).all() and torch.isfinite(rows[~sees]).all()
            assert torch.equal(bits(got[a:a + m, :2]), bits(out[a:a + m, :2]))                     # the other KV head
            others = [x for x in range(d) if x != 3]
            assert (rows[:, :, others] - out[a:a + m].float()[:, :, others]).abs().max() <= 2.0 ** -6 * c.v[at, :, off].float().nan_to_num(0, 0, 0).abs().max()
            c.v.copy_(v)
        leaf = n - 1                                            # seen by itself alone
        c.k[at[leaf], :, off[leaf]], c.v[at[leaf], :, off[leaf]] = NAN, NAN
        got, _ = c.run()
        check_tree(got, None, c.q, c.k, c.v, c.table, c.lens, c.cu, c.seen, f"{dtype} {d} {lens}", only=(i, list(range(m - 1))))
        assert torch.isnan(got[a + m - 1].float()).all()
        c.k.copy_(k)
        c.v.copy_(v)


# in one launch and cut; few rows and many; scores that rise by less than 8 in units of the exponent of 2, and by more, from step to step
@pytest.mark.parametrize("dtype,d", [(BF, 128), (BF, 64), (F32, 128), (F32, 64)])
@pytest.mark.parametrize("n,new,room", [(120, 5, 128), (5000, 5, 5008), (5000, 60, 5008)])
@pytest.mark.parametrize("rise", [5.4375, 7.5])
def test_large_values_stay_finite(dtype, d, n, new, room, rise):
    """Values whose sum over all tokens is a number: of the whole call, and of one KV head with values that are not large beside it."""
    c = Case(dtype, d, 4, 2, 16, [n, 40], [new, 8], 17, width=room // 16, chain=True)
    at, off = (x.to(DEV) for x in rows_of(c.table[0], n, 16))
    c.q[:], c.k[at, :, off] = 0, 0
    c.q[:, :, 0] = d ** 0.5                                          # scores: what stands in the keys' first place
    scores = torch.linspace(0, rise, n, device=DEV)
    scores[torch.arange(n, device=DEV) % 64 >= 32] = rise * 0.99     # large ones in every second 32 tokens
    scores[:32] = 0
    c.k[at, :, off, 0] = scores[:, None].to(dtype)
    size = 3e38 / n
    c.v[at, 0, off] = (size * (0.5 + 0.5 * torch.rand(n, d, device=DEV, generator=torch.Generator(DEV).manual_seed(5)))).to(dtype)
    out, lse = c.run()
    assert torch.isfinite(out[int(c.cu[0]):int(c.cu[-1])].float()).all()
    c.check(out, lse, f"{dtype} d={d} {n} {rise}")


def test_parts_whose_sum_is_no_number_are_averaged():
    """Every part of a cut sequence has a sum, all of them together have not; with scores of equal size, and with most of the weight in few tokens."""
    for dtype in (BF, F32):
        for peak in (0.0, 6.0):
            c = Case(dtype, 64, 4, 2, 16, [20000], [7], 18, q_scale=0.1, chain=True)
            at, off = (x.to(DEV) for x in rows_of(c.table[0], 20000, 16))
            c.v[at, :, off] = (2e35 * (1 + c.v[at, :, off].float().clamp(-1, 1))).to(dtype)
            c.q[:, :, 0] = 8.0
            c.k[at, :, off, 0] = 0
            c.k[at[77::1000], :, off[77::1000], 0] = peak
            out, lse = c.run()
            assert torch.isfinite(out[int(c.cu[0]):int(c.cu[-1])].float()).all()
            c.check(out, lse, f"{dtype} {peak}")


def test_scores_that_are_minus_infinity():
    for dtype in (BF, F32):
        c = Case(dtype, 64, 2, 1, 16, [50], [4], 3, around=(0, 0))
        c.q[1] = torch.tensor([1.0] + [0.0] * 63, dtype=dtype, device=DEV)
        at, off = (x.to(DEV) for x in rows_of(c.table[0], 50, 16))
        c.q[:, :, 0] = 1.0
        c.k[at, 0, off, 0] = -INF
        out, lse = c.run()
        assert not out.any() and (lse == -INF).all()


def test_lengths_that_do_not_cover_the_new_tokens():
    """A length of less than the new tokens: the first of them are in no page.  Lengths below zero and beyond the table row."""
    for dtype in (BF, F32):
        c = Case(dtype, 64, 4, 2, 16, [30, 64, 5, 64], [10, 6, 5, 8], 5, width=4)
        c.lens = [4, -3, 2, 10 ** 9]
        out, lse = c.run()
        c.check(out, lse)
        rows = slice(int(c.cu[1]), int(c.cu[2]))
        assert not out[rows].any() and (lse[rows] == -INF).all()
        c.seen, c.masks = [None] * 4, None
        c.check(*c.run())


# in one launch and cut, of few rows and of many
@pytest.mark.parametrize("dtype,d", [(BF, 128), (BF, 64), (F32, 128), (F32, 64)])
@pytest.mark.parametrize("room,new", [(128, [5, 3, 9, 0, 2]), (4096, [5, 3, 9, 0, 2]), (4096, [40, 70, 8, 1, 90])])
def test_rows_of_sequences_that_were_not_served_are_zero(dtype, d, room, new):
    """Pages run short in the middle of a step: the sequences that were not served keep what they held, and their drafted tokens are in no page."""
    rng = np.random.default_rng(room + new[0])
    page, hq, hk, n, spare = 16, 8, 2, len(new), 3
    have = rng.integers(room // 8, room // 2, n)
    have[1] = have[1] // page * page                                 # this one and the third need more pages than there are
    have[2] = have[2] // page * page - 1
    pages = int(sum(-(-x // page) for x in have)) + 40
    table = new_tables(have, page, pages, rng, room // page)
    free = np.setdiff1d(np.arange(pages), table.reshape(-1))
    k, v = (store(pages, hk, page, d, dtype, "head", DEV, 0.0) for _ in range(2))
    for x in (k, v):
        x.copy_(randn(x.shape, 5 + (x is v), dtype))
    T = sum(new) + spare
    after = [-(-(h + a) // page) - -(-h // page) for h, a in zip(have, new)]
    dev_table = ints(table)
    step = bd.basa_page_tables(ints(have), ints(new), dev_table, ints(free[:after[0]]), page, tokens=T)
    cu, lens = step.cu.tolist(), step.lens.tolist()
    served = [x == h + a for x, h, a in zip(lens, have, new)]
    assert served[0] and not served[1] and not served[2]
    parents = [random_parents(x, rng) for x in new]
    seen = [ancestors(x) for x in parents]
    masks, _ = bd.basa_tree_masks(ints(np.concatenate(parents + [np.zeros(spare)])), step.cu, 2)
    q, kn, vn = (randn((T, h, d), 9 + i, dtype) for i, h in enumerate((hq, hk, hk)))
    cache = bd.PagedCache(k, v)
    for m, s in ((masks, seen), (None, [None] * n)):
        out, lse = bd.ba_att_tree(q, kn, vn, cache, dev_table, step.lens, step.slots, step.cu, m, want_lse=True)
        of_zero = torch.where(step.lens == ints(have) + ints(new), step.lens, 0)
        out0, lse0 = bd.basa_tree_attn(q, cache, dev_table, of_zero, step.cu, m, want_lse=True)
        for i in range(n):
            rows = slice(cu[i], cu[i + 1])
            if not served[i]:
                assert not out[rows].any() and (lse[rows] == -INF).all() and not out0[rows].any() and (lse0[rows] == -INF).all()
            else:
                check_tree(out, lse, q, k, v, dev_table.cpu().numpy(), lens, cu, s, f"{dtype} {d} {room}", only=(i, list(range(new[i]))))
                check_tree(out0, lse0, q, k, v, dev_table.cpu().numpy(), lens, cu, s, f"{dtype} {d} {room}", only=(i, list(range(new[i]))))


def test_slots_that_are_none():
    """Negative, and beyond the cache; the others' rows are what they are without slots."""
    for dtype, lens, new in ((BF, [100, 30], [20, 7]), (F32, [3000, 70], [20, 70])):
        c = Case(dtype, 128, 8, 2, 16, lens, new, 6)
        out, lse = c.run()
        all_slots = c.k.shape[0] * 16
        slots = torch.arange(c.T, dtype=torch.int64, device=DEV) % all_slots
        none = [int(c.cu[0]) + 3, int(c.cu[0]) + 11, int(c.cu[1]), int(c.cu[1]) + 6]
        for t, x in zip(none, (-1, all_slots, 2 ** 62, -2 ** 63)):
            slots[t] = x
        got, got_lse = c.run(slots=slots)
        assert not got[none].any() and (got_lse[none] == -INF).all()
        rest = [t for t in range(int(c.cu[0]), int(c.cu[-1])) if t not in none]
        assert torch.equal(bits(got[rest]), bits(out[rest])) and torch.equal(got_lse[rest], lse[rest])


def test_offsets_that_do_not_ascend_stay_in_bounds():
    c = Case(BF, 64, 4, 2, 16, [60, 40, 300], [8, 8, 8], 5)
    for cu in ([0, 20, 4, 24], [50, 20, 90, 7], [-5, 10, 30, 12], [0, 2 ** 31 - 1, 2 ** 31 - 1, 5], [-2 ** 31, 0, 60, -1]):
        for width in (4, 60):
            table = torch.full((3, width), -1, dtype=torch.int32, device=DEV)
            table[:, :4] = ints(c.table[:, :4])
            bd.basa_tree_attn(c.q, c.cache(), table, ints(c.lens), ints(cu), c.masks, want_lse=True)
            torch.cuda.synchronize()


class Guarded:
    """A tensor in the middle of a larger one, and whether what lies around it is as it was."""

    def __init__(self, shape, dtype, fill=0x5b, guard=2 ** 20):
        size = math.prod(shape) * torch.empty(0, dtype=dtype).element_size()
        self.all = torch.full((guard + size + guard,), fill, dtype=torch.uint8, device=DEV)
        self.guard, self.size, self.fill = guard, size, fill
        self.t = self.all[guard:guard + size].view(dtype).view(shape)

    def untouched(self):
        return bool((self.all[:self.guard] == self.fill).all()) and bool((self.all[self.guard + self.size:] == self.fill).all())


def _run_guarded(c, table, cu):
    """The C call on outputs and a workspace, of the size that it asks for, with guards around them, and on the inputs, which it leaves as they are."""
    cache, n = c.cache(), len(cu) - 1
    table, lens, cu = ints(table), ints(c.lens), ints(cu)
    need = bd.tree_workspace_size(c.q, cache, table)
    out, lse, ws = Guarded(c.q.shape, c.q.dtype), Guarded((c.T, c.q.shape[1]), F32), Guarded((need,), torch.uint8)
    inputs = (c.q, c.k, c.v, table, lens, cu) + (() if c.masks is None else (c.masks,))
    before = [x.clone() for x in inputs]
    words, stride = (0, 0) if c.masks is None else (c.masks.shape[1], c.masks.stride(0))
    hq, d = c.q.shape[1:]
    bd._launch(bd.load().basa_tree_attn, cache.device, bd._new_rows_desc(c.q, "q", cache), cache._kd, cache._vd, table.data_ptr(), table.shape[1], table.stride(0),
               lens.data_ptr(), cu.data_ptr(), n, None if c.masks is None else c.masks.data_ptr(), words, stride, out.t.data_ptr(), None, lse.t.data_ptr(), ws.t.data_ptr(), need)
    torch.cuda.synchronize()
    assert out.untouched() and lse.untouched() and ws.untouched()
    for x, b in zip(inputs, before):
        assert torch.equal(bits(x) if x.is_floating_point() else x, bits(b) if b.is_floating_point() else b)
    return out.t, lse.t


@pytest.mark.parametrize("dtype,d", [(BF, 128), (F32, 64)])
@pytest.mark.parametrize("n,new,width", [(3, 8, 4), (3, 8, 60), (3, 70, 300), (600, 3, 8), (600, 3, 40)])
def test_nothing_is_written_outside_the_outputs_and_the_workspace(dtype, d, n, new, width):
    """One launch and cut, offsets summed up by a wave and by a kernel; offsets that ascend, and ones that do not."""
    rng = np.random.default_rng(n + width)
    lens = rng.integers(new, min(16 * width, 1500) + 1, n).tolist()
    c = Case(dtype, d, 4, 2, 16, lens, [new] * n, 5, width=width, around=(0, 0))
    c.check(*_run_guarded(c, c.table, c.cu))
    T = c.T
    wild = [rng.integers(-2 ** 31, 2 ** 31 - 1, n + 1), rng.permutation(T + 50)[:n + 1] - 20 if T + 50 > n else rng.integers(-20, T + 30, n + 1), np.full(n + 1, T), np.full(n + 1, -5),
            np.arange(n + 1)[::-1] * new, np.where(np.arange(n + 1) % 2 == 0, 0, T), np.where(np.arange(n + 1) % 2 == 0, -2 ** 31, 2 ** 31 - 1)]
    masks = c.masks
    for cu in wild:
        for m in (masks, None):
            c.masks = m
            _run_guarded(c, c.table, cu)


def test_masks_are_written_in_their_rows_alone():
    for T, n, words in ((40, 2, 1), (300, 4, 3)):
        rng = np.random.default_rng(T)
        parents = ints(np.arange(T) - 1)
        for cu in ([0] + [T] * n, [T // 2] * (n + 1), np.sort(rng.integers(0, T, n + 1)), rng.integers(-2 ** 31, 2 ** 31 - 1, n + 1), np.arange(n + 1)[::-1] * (T // n), [-5] * n + [2 ** 31 - 1],
                   rng.integers(-T, 2 * T, n + 1), np.where(np.arange(n + 1) % 2 == 0, T // 2, -2 ** 31)):
            masks, depths = Guarded((T, words + 1), torch.int64), Guarded((T,), torch.int32)
            between = masks.t[:, words].clone()
            bd.basa_tree_masks(parents, ints(cu), words, out=(masks.t[:, :words], depths.t))
            torch.cuda.synchronize()
            assert masks.untouched() and depths.untouched() and torch.equal(masks.t[:, words], between)


# more sequences than a workgroup of the sum over them has threads, and than two rounds of the search tell apart; runs of empty ones, the last one without rows
@pytest.mark.parametrize("dtype,d,n,new,width", [(BF, 64, 1500, 3, 8), (F32, 64, 1500, 3, 40), (BF, 128, 5000, 2, 4), (BF, 128, 5000, 2, 40), (F32, 128, 5000, 2, 40), (BF, 128, 600, 80, 30),
                                                 (F32, 64, 600, 20, 30), (BF, 64, 600, 50, 8)])
def test_very_many_sequences(dtype, d, n, new, width):
    rng = np.random.default_rng(n + width)
    count = rng.integers(0, new + 1, n)
    for a in (0, n // 3, n - 70):
        count[a:a + 70] = 0
    count[-2] = new
    lens = np.maximum(rng.integers(0, 16 * min(width, 10) + 1, n), count)
    lens[rng.random(n) < 0.02] = 16 * width
    c = Case(dtype, d, 8, 2, 16, lens.tolist(), count.tolist(), 11, width=width)
    out, lse = c.run()
    table, cu = ints(c.table), c.cu
    # every row against calls of up to 256 sequences: either is off from 64 bits by what a call may be, and rounded once
    norm = lambda x: float(x.float().nan_to_num(0).norm(dim=-1).max())  # noqa: E731
    tol, tol_lse = decode_tolerance(dtype, int(lens.max()), d, norm(c.q) * norm(c.k) / math.sqrt(d), float(c.v.float().nan_to_num(0).abs().max()))
    for a in range(0, n, 256):
        b = min(a + 256, n)
        rows = slice(int(cu[a]), int(cu[b]))
        part, part_lse = bd.basa_tree_attn(c.q[rows], c.cache(), table[a:b], ints(lens[a:b]), ints(cu[a:b + 1] - cu[a]), c.masks[rows], want_lse=True)
        x, y, e, f = out[rows].double(), part.double(), lse[rows].double(), part_lse.double()
        assert bool(((x - y).abs() <= 2 * tol + HALF_STEP[dtype] * 1.01 * (x.abs() + y.abs())).all())
        assert torch.equal(torch.isinf(e), torch.isinf(f)) and bool(((e - f).abs()[torch.isfinite(e)] <= 2 * tol_lse).all())
    for i in sorted({70, n // 3 - 1, n // 3 + 70, n - 71, n - 2, *rng.integers(0, n, 40).tolist()}):
        check_tree(out, lse, c.q, c.k, c.v, c.table, c.lens, c.cu, c.seen, f"{dtype} {d} {n}", only=(i, list(range(c.new[i]))))


def _spread(x, stride_b, stride_h, stride_l):
    """The same pages far apart, in storage of which nothing else is ever written."""
    n, h, t, d = x.shape
    size = (n - 1) * stride_b + (h - 1) * stride_h + (t - 1) * stride_l + d
    y = torch.empty(size, dtype=x.dtype, device=DEV).as_strided(x.shape, (stride_b, stride_h, stride_l, 1))
    return y.copy_(x)


# pages, or heads, more than 4 GiB apart in all; strides that only 16 bytes divide
@pytest.mark.parametrize("dtype,d", [(BF, 128), (F32, 64)])
@pytest.mark.parametrize("stride_b,stride_h,stride_l", [(2 ** 27 + 8, 1000, 2 ** 15 + 24), (2 ** 13, 2 ** 31 + 64, 136), (2 ** 27, 2 ** 20, 256)])
def test_offsets_beyond_32_bits(dtype, d, stride_b, stride_h, stride_l):
    c = Case(dtype, d, 8, 2, 16, [300, 17, 120], [20, 3, 70], 13)
    assert c.k.shape[0] > 30
    c.k, c.v = _spread(c.k, stride_b, stride_h, stride_l), _spread(c.v, stride_b, stride_h, stride_l)
    c.check(*c.run(), f"{dtype} {stride_b} {stride_h}")


def test_no_tokens_or_no_sequences_is_no_work():
    cache = bd.PagedCache(*(store(2, 2, 16, 64, BF, "head", DEV, 1.0) for _ in range(2)))
    none = torch.empty(0, 4, 64, dtype=BF, device=DEV)
    assert bd.basa_tree_attn(none, cache, ints(np.zeros((1, 3))), ints([0]), ints([0, 0])).shape == (0, 4, 64)
    q, out = randn((3, 4, 64), 1, BF), torch.full((3, 4, 64), 7.0, dtype=BF, device=DEV)
    bd.basa_tree_attn(q, cache, ints(np.zeros((0, 3))), ints([]), ints([0]), out=out)
    bd.basa_tree_attn(q, cache, ints(np.zeros((2, 3))), ints([0, 5]), ints([1, 1, 1]), out=out)
    assert (out == 7.0).all()


def test_accuracy_is_that_of_32_bits():
    """The root of the mean square error against 64 bits is at most one and a half times what is left when the same attention is computed in 32 bits and rounded once."""
    for dtype, d in ((BF, 128), (BF, 64), (F32, 128), (F32, 64)):
        c = Case(dtype, d, 8, 2, 16, [3000], [40], 12, around=(0, 0), chain=True)
        out, lse = c.run()
        at, off = (x.to(DEV) for x in rows_of(c.table[0], 3000, 16))
        hidden = torch.ones(40, 3000, dtype=torch.bool, device=DEV).triu(2961)

        def plain(t):
            o, e = [], []
            for h in range(8):
                k, v = c.k[at, h // 4, off].to(t), c.v[at, h // 4, off].to(t)
                s = (c.q[:, h].to(t) @ k.t() / math.sqrt(d)).masked_fill(hidden, -INF)
                o.append(torch.softmax(s, 1) @ v)
                e.append(torch.logsumexp(s, 1))
            return torch.stack(o, 1), torch.stack(e, 1)
        (o64, e64), (o32, e32) = plain(torch.float64), plain(F32)
        rms = lambda x: float(x.double().square().mean().sqrt())                     # noqa: E731
        assert rms(out.double() - o64) <= 1.5 * rms(o32.to(dtype).double() - o64), (dtype, d)
        assert rms(lse.double() - e64) <= 2 * rms(e32.double() - e64) + 2.0 ** -24 * rms(e64), (dtype, d)


# ---------------------------------------------------------------- streams and graphs
def test_two_streams_with_workspaces_of_their_own():
    cases = [Case(BF, 128, 8, 2, 16, [4000, 700], [16, 5], 21), Case(F32, 64, 8, 8, 32, [2500], [31], 22)]
    want = [c.run() for c in cases]
    args = [(c.q, c.cache(), ints(c.table), ints(c.lens), ints(c.cu), c.masks) for c in cases]
    torch.cuda.synchronize()
    streams, got = [torch.cuda.Stream() for _ in cases], []
    for _ in range(5):
        got = []
        for s, a in zip(streams, args):
            with torch.cuda.stream(s):
                got.append(bd.basa_tree_attn(*a, want_lse=True))
    torch.cuda.synchronize()
    for c, (o, e), (o2, e2) in zip(cases, want, got):
        rows = slice(int(c.cu[0]), int(c.cu[-1]))
        assert torch.equal(bits(o[rows]), bits(o2[rows])) and torch.equal(e[rows], e2[rows])


def test_a_captured_call_follows_its_inputs():
    for dtype, lens, new in ((BF, [4000, 700], [16, 5]), (F32, [300, 100], [9, 30]), (BF, [500] * 600, [2] * 600)):
        c = Case(dtype, 64, 8, 2, 16, lens, new, 31, width=-(-max(lens) // 16) + 2, spare=4 * len(lens))
        cache, table, at, cu = c.cache(), ints(c.table), ints(c.lens), ints(c.cu)
        ws = torch.empty(bd.tree_workspace_size(c.q, cache, table), dtype=torch.uint8, device=DEV)
        out = torch.zeros_like(c.q)
        bd.basa_tree_attn(c.q, cache, table, at, cu, c.masks, ws=ws, out=out)
        torch.cuda.synchronize()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            _, lse = bd.basa_tree_attn(c.q, cache, table, at, cu, c.masks, want_lse=True, ws=ws, out=out)
        rows = slice(int(c.cu[0]), int(c.cu[-1]))
        for turn in range(4):
            at.copy_(ints([max(n - 7 * turn, m) for n, m in zip(lens, new)]))
            c.q.copy_(randn(c.q.shape, 50 + turn, dtype))
            ws.fill_(255)                                       # nothing is kept in it
            g.replay()
            torch.cuda.synchronize()
            o, e = bd.basa_tree_attn(c.q, cache, table, at, cu, c.masks, want_lse=True)
            assert torch.equal(bits(out[rows]), bits(o[rows])) and torch.equal(lse[rows], e[rows]), turn
