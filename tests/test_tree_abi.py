"""Refusals of the entry points for several new tokens per sequence and for the pages around them: on the host, before any launch (no GPU needed)."""
import ctypes as C

import pytest
import torch

from paper_2605_19726_amd import binding as bd
from test_abi import lib, status_of  # noqa: F401  (the fixture)
from test_paged_abi import INVALID, UNSUPPORTED, WORKSPACE, V, pages, tensor


def test_tree_masks(lib):  # noqa: F811
    good = dict(parents=0x1000, cu=0x2000, n=8, tokens=100, masks=0x10000, words=2, stride=3, depths=0x3000)

    def call(**kw):
        a = {**good, **kw}
        return status_of(lib, lib.basa_tree_masks, V(a["parents"]), V(a["cu"]), a["n"], a["tokens"], V(a["masks"]), a["words"], a["stride"],
                         V(a["depths"]), None)[0]
    for bad in (dict(parents=None), dict(cu=None), dict(masks=None), dict(n=-1), dict(tokens=-1), dict(words=0), dict(words=-3), dict(stride=1),
                dict(masks=0x10004), dict(masks=0x1000), dict(masks=0x2000 - 8 * (99 * 3 + 2) + 8), dict(depths=0x2000 - 396), dict(depths=0x10000)):
        assert call(**bad) == INVALID, bad
    for bad in (dict(words=65, stride=65), dict(tokens=2 ** 30 + 1, parents=2 ** 40, masks=2 ** 50, depths=None)):
        assert call(**bad) == UNSUPPORTED, bad
    assert call(tokens=0, parents=None, masks=None, depths=None) == "BASA_OK"


def _tree(lib, **kw):  # noqa: F811
    a = {**dict(q=tensor(heads=8, L=40), k=pages(), v=pages(ptr=0x4000000), table=0x1000, width=10, stride=12, lens=0x2000, cu=0x3000, n=4, masks=0x4000,
                words=1, mask_stride=1, out=0x5000, strides=None, ws=0x100000, ws_bytes=2 ** 40), **kw}
    r = C.byref
    strides = None if a["strides"] is None else (C.c_int64 * 2)(*a["strides"])
    return status_of(lib, lib.basa_tree_attn, r(a["q"]), r(a["k"]), r(a["v"]), V(a["table"]), a["width"], a["stride"], V(a["lens"]), V(a["cu"]), a["n"],
                     V(a["masks"]), a["words"], a["mask_stride"], V(a["out"]), strides, None, V(a["ws"]), a["ws_bytes"], None)[0]


def test_tree_attn(lib):  # noqa: F811
    good = tensor(heads=8, L=40)
    for bad in (dict(q=tensor(heads=8, batch=2)), dict(q=tensor(heads=8, dtype=bd.F32)), dict(q=tensor(heads=6)), dict(q=tensor(ptr=None, heads=8)),
                dict(q=tensor(ptr=0x10008, heads=8)), dict(q=tensor(heads=8, stride_l=130)), dict(v=pages(L=17)), dict(v=pages(batch=99)), dict(v=pages(dtype=bd.F32)),
                dict(table=None), dict(width=0), dict(stride=9), dict(lens=None), dict(cu=None), dict(n=-1), dict(out=None), dict(out=0x5008),
                dict(words=0), dict(mask_stride=0), dict(words=2), dict(masks=0x4004), dict(strides=(1024, 120)), dict(strides=(-8, 128)),
                dict(strides=(1024, 132)), dict(ws=0x100010)):
        assert _tree(lib, **bad) == INVALID, bad
    for bad in (dict(q=tensor(heads=8, d=96), k=pages(d=96), v=pages(d=96)), dict(q=tensor(heads=8, L=2 ** 21 + 1)), dict(width=2 ** 27, stride=2 ** 27),
                dict(k=pages(stride_b=2 ** 37)), dict(v=pages(stride_l=2 ** 40, ptr=0x4000000)), dict(k=pages(stride_b=2 ** 32 + 8)),
                dict(q=tensor(heads=8, L=200000), width=2 ** 26, stride=2 ** 26)):
        assert _tree(lib, **bad) == UNSUPPORTED, bad
    for bad in (dict(ws=None), dict(ws_bytes=0), dict(ws_bytes=lib.basa_tree_workspace_size(C.byref(good), C.byref(pages()), C.byref(pages()), 4, 10) - 1)):
        assert _tree(lib, **bad) == WORKSPACE, bad
    assert _tree(lib, n=0, table=None, lens=None) == "BASA_OK"
    size = lambda **kw: lib.basa_tree_workspace_size(C.byref(kw.get("q", good)), C.byref(pages()), C.byref(pages()), kw.get("n", 4), kw.get("width", 10))  # noqa: E731
    assert size() > 0 and size(n=-1) == 0 and size(width=0) == 0 and size(q=tensor(heads=7)) == 0


def test_tree_attn_of_slots(lib):  # noqa: F811
    def call(slots, q=tensor(heads=8, L=40), out=0x5000, ws_bytes=2 ** 40, n=4, lens=0x2000):
        k, v = pages(), pages(ptr=0x4000000)
        return status_of(lib, lib.basa_tree_attn_slots, C.byref(q), C.byref(k), C.byref(v), V(0x1000), 10, 12, V(lens), V(0x3000), n, V(0x4000), 1, 1, V(slots),
                         V(out), None, None, V(0x100000), ws_bytes, None)[0]
    assert call(0x6004) == INVALID and b"slots" in lib.basa_last_error()
    for slots in (None, 0x6000):
        assert call(slots, q=tensor(heads=6)) == INVALID and call(slots, out=None) == INVALID and call(slots, lens=None) == INVALID
        assert call(slots, ws_bytes=0) == WORKSPACE and call(slots, n=0, lens=None) == "BASA_OK"
    z = lambda *shape, dtype=torch.int32: torch.zeros(*shape, dtype=dtype)  # noqa: E731
    cache = bd.PagedCache(*(torch.zeros(6, 2, 16, 64, dtype=torch.bfloat16) for _ in range(2)))
    for slots in (z(5), z(4, dtype=torch.int64), z(10, dtype=torch.int64)[::2]):
        with pytest.raises(ValueError, match="slots"):
            bd.basa_tree_attn(torch.zeros(5, 4, 64, dtype=torch.bfloat16), cache, z(2, 4), z(2), z(3), slots=slots)


def test_tree_attn_refuses_outputs_in_other_tensors(lib):  # noqa: F811
    """One tensor is moved into another at a time, at its first and at its last bytes."""
    q, k, v = tensor(ptr=2 ** 33, heads=8, L=40, stride_l=3 * 1024, stride_h=128), pages(ptr=2 ** 34), pages(ptr=2 ** 35)
    need = lib.basa_tree_workspace_size(C.byref(q), C.byref(k), C.byref(v), 4, 10)
    at = dict(table=2 ** 36, lens=2 ** 37, cu=2 ** 38, masks=2 ** 39, slots=2 ** 40, out=2 ** 41, lse=2 ** 42, ws=2 ** 43)
    size = dict(q=40 * 3 * 2048 - 2 * 2048, k=100 * 16 * 4 * 256, v=100 * 16 * 4 * 256, table=4 * (3 * 12 + 10), lens=16, cu=20, masks=8 * (39 * 3 + 2), slots=320,
                out=39 * 2560 + 7 * 288 + 256, lse=40 * 8 * 4, ws=need)
    where = dict(at, q=2 ** 33, k=2 ** 34, v=2 ** 35)

    def call(**kw):
        a = dict(at, **kw)
        return status_of(lib, lib.basa_tree_attn_slots, C.byref(q), C.byref(k), C.byref(v), V(a["table"]), 10, 12, V(a["lens"]), V(a["cu"]), 4, V(a["masks"]), 2, 3,
                         V(a["slots"]), V(a["out"]), (C.c_int64 * 2)(1280, 144), V(a["lse"]), V(a["ws"]), need, None)[0]
    unit = dict(out=16, lse=4, ws=256)
    for o in ("out", "lse", "ws"):
        for other in where:
            if other == o:
                continue
            up = lambda x: -(-x // unit[o]) * unit[o]  # noqa: E731
            ends = [where[other], (where[other] + size[other] - 1) // unit[o] * unit[o]]          # its first unit and its last
            ends.append(up(where[other] - size[o] + 1))                                           # its first byte under the last of `o`
            for x in ends:
                assert call(**{o: x}) == INVALID, (o, other, x)
                assert b"overlap" in lib.basa_last_error()
    twice = (C.c_int64 * 2)(120, 128)
    assert status_of(lib, lib.basa_tree_attn_slots, C.byref(q), C.byref(k), C.byref(v), V(at["table"]), 10, 12, V(at["lens"]), V(at["cu"]), 4, None, 0, 0, None, V(at["out"]),
                     twice, None, V(at["ws"]), need, None)[0] == INVALID


def test_cache_compact(lib):  # noqa: F811
    good = dict(k=pages(), v=pages(ptr=0x4000000), table=0x1000, width=10, stride=12, start=0x2000, keep=0x3000, most=6, keep_stride=6, count=0x4000, n=4)

    def call(**kw):
        a = {**good, **kw}
        return status_of(lib, lib.basa_cache_compact, C.byref(a["k"]), C.byref(a["v"]), V(a["table"]), a["width"], a["stride"], V(a["start"]), V(a["keep"]), a["most"],
                         a["keep_stride"], V(a["count"]), a["n"], None)[0]
    for bad in (dict(v=pages(heads=5)), dict(v=pages(dtype=bd.F32)), dict(table=None), dict(width=0), dict(stride=9), dict(start=None), dict(keep=None),
                dict(count=None), dict(most=-1), dict(keep_stride=5), dict(n=-1)):
        assert call(**bad) == INVALID, bad
    assert call(width=2 ** 27, stride=2 ** 27) == UNSUPPORTED
    assert call(n=0, table=None, start=None, keep=None, count=None) == "BASA_OK"
    assert call(most=0, keep_stride=0, keep=None) == "BASA_OK"


def test_cache_compact_within_lengths(lib):  # noqa: F811
    def call(k=None, v=None, table=0x1000, n=4, width=10, most=6, start=0x2000, keep=0x3000, count=0x4000, lens=0x5000):
        k, v = k or pages(), v or pages(ptr=0x4000000)
        return status_of(lib, lib.basa_cache_compact_held, C.byref(k), C.byref(v), V(table), width, 12, V(lens), V(start), V(keep), most, 6, V(count), n, None)[0]
    for bad in (dict(v=pages(heads=5)), dict(table=None), dict(width=0), dict(start=None), dict(keep=None), dict(count=None), dict(most=7), dict(n=-1)):
        assert call(**bad) == INVALID, bad
    for lens in (0x5000, None):
        assert call(n=0, table=None, start=None, keep=None, count=None, lens=lens) == "BASA_OK"
        assert call(most=0, keep=None, lens=lens) == "BASA_OK"
    z = lambda *shape, dtype=torch.int32: torch.zeros(*shape, dtype=dtype)  # noqa: E731
    cache = bd.PagedCache(*(torch.zeros(6, 2, 16, 64, dtype=torch.bfloat16) for _ in range(2)))
    for lens in (z(3), z(2, dtype=torch.int64), z(4)[::2]):
        with pytest.raises(ValueError, match="lens"):
            bd.basa_cache_compact(cache, z(2, 4), z(2), z(2, 4), z(2), lens)


def test_page_fork(lib):  # noqa: F811
    good = dict(table=0x10000, width=20, stride=20, lens=0x1000, n=10, page=16, parents=0x2000, m=30, free=0x3000, n_free=50, new=0x20000, new_stride=24,
                new_lens=0x4000, copies=0x5000, pages=0x6000)

    def call(**kw):
        a = {**good, **kw}
        return status_of(lib, lib.basa_page_fork, V(a["table"]), a["width"], a["stride"], V(a["lens"]), a["n"], a["page"], V(a["parents"]), a["m"], V(a["free"]),
                         a["n_free"], V(a["new"]), a["new_stride"], V(a["new_lens"]), V(a["copies"]), V(a["pages"]), None)[0]
    for bad in (dict(table=None), dict(lens=None), dict(parents=None), dict(free=None), dict(new=None), dict(new_lens=None), dict(copies=None), dict(pages=None),
                dict(page=0), dict(width=0), dict(stride=19), dict(new_stride=19), dict(n=-1), dict(m=-1), dict(n_free=-1),
                dict(new=0x10000), dict(new=0x10000 + 4 * 199), dict(new_lens=0x1000), dict(new_lens=0x2000 + 116), dict(copies=0x3000 + 196),
                dict(pages=0x4000 + 116), dict(copies=0x6000 - 352)):
        assert call(**bad) == INVALID, bad
    far = dict(table=2 ** 40, new=2 ** 41, lens=2 ** 42, parents=2 ** 43, free=2 ** 44, new_lens=2 ** 45, copies=2 ** 46)
    for bad in (dict(n=8193, **far), dict(m=8193, **far), dict(width=2 ** 27, stride=2 ** 27, new_stride=2 ** 27)):
        assert call(**bad) == UNSUPPORTED, bad


def test_cache_copy(lib):  # noqa: F811
    call = lambda k, v, copies, n: status_of(lib, lib.basa_cache_copy, C.byref(k), C.byref(v), V(copies), n, None)[0]  # noqa: E731
    assert call(pages(), pages(heads=5), 0x1000, 3) == INVALID
    assert call(pages(), pages(), None, 3) == INVALID and call(pages(), pages(), 0x1000, -1) == INVALID
    assert call(pages(L=2 ** 20, heads=128), pages(L=2 ** 20, heads=128), 0x1000, 3) == UNSUPPORTED
    assert call(pages(), pages(), 0x1000, 2 ** 22 + 1) == UNSUPPORTED
    assert call(pages(), pages(), None, 0) == "BASA_OK"


def test_page_free(lib):  # noqa: F811
    good = dict(table=0x10000, width=20, stride=20, lens=0x1000, n=10, page=16, pages=300, free=0x2000, count=0x3000, ws=0x100000, ws_bytes=2 ** 30)

    def call(**kw):
        a = {**good, **kw}
        return status_of(lib, lib.basa_page_free, V(a["table"]), a["width"], a["stride"], V(a["lens"]), a["n"], a["page"], a["pages"], V(a["free"]), V(a["count"]),
                         V(a["ws"]), a["ws_bytes"], None)[0]
    for bad in (dict(table=None), dict(lens=None), dict(free=None), dict(count=None), dict(page=0), dict(width=0), dict(stride=19), dict(n=-1), dict(pages=0),
                dict(ws=0x100010), dict(free=0x10000), dict(free=0x1000 - 1196), dict(count=0x1000 + 36), dict(count=0x2000 + 1196), dict(ws=0x10000),
                dict(ws=0x2000)):
        assert call(**bad) == INVALID, bad
    for bad in (dict(ws=None), dict(ws_bytes=255), dict(pages=2 ** 20, free=2 ** 40, ws_bytes=2 ** 20 - 1)):
        assert call(**bad) == WORKSPACE, bad
    for bad in (dict(pages=2 ** 26 + 1, free=2 ** 40), dict(n=2 ** 22 + 1, table=2 ** 50, lens=2 ** 45), dict(width=2 ** 27, stride=2 ** 27)):
        assert call(**bad) == UNSUPPORTED, bad
    assert lib.basa_page_free_workspace_size(10, 20, 0) == 0 and lib.basa_page_free_workspace_size(0, 20, 2 ** 20) >= 2 ** 17


def test_more_sequences_than_a_launch_has_groups_for_are_refused(lib):  # noqa: F811
    many = 2 ** 22 + 1
    assert status_of(lib, lib.basa_tree_masks, V(2 ** 40), V(2 ** 41), many, 100, V(2 ** 42), 1, 1, None, None)[0] == UNSUPPORTED
    far = dict(table=2 ** 50, lens=2 ** 51, cu=2 ** 52, masks=None)
    assert _tree(lib, n=many, **far) == UNSUPPORTED
    compact = lambda k, n, most: status_of(lib, lib.basa_cache_compact, C.byref(k), C.byref(k), V(2 ** 40), 10, 10, V(2 ** 41), V(2 ** 42), most, most, V(2 ** 43), n, None)[0]  # noqa: E731
    assert compact(pages(), many, 6) == UNSUPPORTED and compact(pages(), many, 600) == UNSUPPORTED
    wide = pages(heads=2 ** 15, stride_l=2 ** 22, stride_h=128, stride_b=2 ** 26)
    assert compact(wide, 2 ** 16, 600) == UNSUPPORTED                  # 2^16 sequences of 2^16 lines of K and of V


def test_the_binding_refuses_what_the_kernels_would_misread():
    z = lambda *shape, dtype=torch.int32: torch.zeros(*shape, dtype=dtype)  # noqa: E731
    cache = bd.PagedCache(*(torch.zeros(6, 2, 16, 64, dtype=torch.bfloat16) for _ in range(2)))
    q = torch.zeros(5, 4, 64, dtype=torch.bfloat16)
    for bad in (dict(q=q.float()), dict(q=q[0]), dict(q=q.permute(0, 2, 1)), dict(lens=z(3)), dict(lens=z(2, dtype=torch.int64)), dict(cu=z(3, dtype=torch.int64)),
                dict(cu=z(6)[::2]), dict(masks=z(5, 1)), dict(masks=z(4, 1, dtype=torch.int64)), dict(masks=z(2, 5, dtype=torch.int64).t()), dict(table=z(3, 4)),
                dict(table=z(2, 4, dtype=torch.int64)), dict(out=q[:4]), dict(out=q.float()), dict(ws=torch.empty(1, dtype=torch.uint8).expand(10 ** 9))):
        a = {**dict(q=q, table=z(2, 4), lens=z(2), cu=z(3), masks=None, ws=None, out=None), **bad}
        with pytest.raises(ValueError):
            bd.basa_tree_attn(a["q"], cache, a["table"], a["lens"], a["cu"], a["masks"], ws=a["ws"], out=a["out"])
    for bad in (dict(parents=z(5, dtype=torch.int64)), dict(parents=z(10)[::2]), dict(cu=z(3, dtype=torch.int64)), dict(out=(z(5, 2, dtype=torch.int64), z(5))),
                dict(out=(z(5, 1), z(5))), dict(out=(z(5, 1, dtype=torch.int64), z(4)))):
        a = {**dict(parents=z(5), cu=z(3), out=None), **bad}
        with pytest.raises(ValueError):
            bd.basa_tree_masks(a["parents"], a["cu"], 1, out=a["out"])
    for bad in (dict(start=z(3)), dict(keep=z(3, 4)), dict(keep=z(4, 2).t()), dict(count=z(2, dtype=torch.int64)), dict(keep=z(2, 4, dtype=torch.int64))):
        a = {**dict(start=z(2), keep=z(2, 4), count=z(2)), **bad}
        with pytest.raises(ValueError):
            bd.basa_cache_compact(cache, z(2, 4), a["start"], a["keep"], a["count"])
    for bad in (dict(lens=z(3)), dict(parents=z(4, dtype=torch.int64)), dict(free=z(9)[::2]), dict(out=bd.PageFork(3, 4, "cpu")), dict(out=bd.PageFork(4, 5, "cpu"))):
        a = {**dict(lens=z(2), parents=z(4), free=z(9), out=None), **bad}
        with pytest.raises(ValueError):
            bd.basa_page_fork(z(2, 4), a["lens"], a["parents"], a["free"], 16, out=a["out"])
    for bad in (z(3, 2), z(3, 3, dtype=torch.int64), z(3, 6)[:, ::2]):
        with pytest.raises(ValueError):
            bd.basa_cache_copy(cache, bad)
    for bad in (dict(lens=z(3)), dict(out=(z(49), z(1))), dict(out=(z(50), z(2))), dict(out=(z(50, dtype=torch.int64), z(1)))):
        a = {**dict(lens=z(2), out=None), **bad}
        with pytest.raises(ValueError):
            bd.basa_page_free(z(2, 4), a["lens"], 16, 50, out=a["out"])
    # tensors that are not on a GPU
    with pytest.raises(ValueError):
        bd.basa_tree_attn(q, cache, z(2, 4), z(2), z(3))
    with pytest.raises(ValueError):
        bd.basa_page_free(z(2, 4), z(2), 16, 50)
