"""Refusals of the paged-cache entry points: on the host, before any launch (no GPU needed)."""
import ctypes as C

import pytest
import torch

from paper_2605_19726_amd import binding as bd
from test_abi import lib, status_of  # noqa: F401  (the fixture)

V = C.c_void_p
INVALID, UNSUPPORTED, WORKSPACE = "BASA_ERR_INVALID_ARG", "BASA_ERR_UNSUPPORTED", "BASA_ERR_WORKSPACE"


def tensor(ptr=0x10000, dtype=bd.BF16, batch=1, heads=4, L=50, d=128, **kw):
    s = dict(stride_b=heads * L * d, stride_h=L * d, stride_l=d)
    s.update(kw)
    return bd.BasaTensor(ptr, dtype, batch, heads, L, d, s["stride_b"], s["stride_h"], s["stride_l"])


def pages(**kw):
    return tensor(**{**dict(batch=100, L=16), **kw})


def test_page_tables(lib):  # noqa: F811
    good = dict(have=0x1000, add=0x2000, n_seq=8, page=16, table=0x10000, width=32, stride=40, free=0x3000, n_free=100, slots=0x20000,
                n_slots=64, lens=0x4000, cu=0x5000, pages=0x6000)

    def call(**kw):
        a = {**good, **kw}
        return status_of(lib, lib.basa_page_tables, V(a["have"]), V(a["add"]), a["n_seq"], a["page"], V(a["table"]), a["width"], a["stride"],
                         V(a["free"]), a["n_free"], V(a["slots"]), a["n_slots"], V(a["lens"]), V(a["cu"]), V(a["pages"]), None)[0]
    for bad in (dict(have=None), dict(add=None), dict(table=None), dict(free=None), dict(slots=None), dict(lens=None), dict(cu=None),
                dict(pages=None), dict(page=0), dict(page=-16), dict(width=0), dict(stride=31), dict(n_seq=-1), dict(n_free=-1),
                dict(n_slots=-1)):
        assert call(**bad) == INVALID, bad
    for bad in (dict(n_seq=8193, have=0x100000, add=0x200000), dict(width=2 ** 27, stride=2 ** 27), dict(n_slots=2 ** 30 + 1)):
        assert call(**bad) == UNSUPPORTED, bad
    # what every workgroup reads must not be what another one writes
    for bad in (dict(lens=0x1000), dict(lens=0x1000 + 28), dict(cu=0x2000 - 32), dict(pages=0x3000 + 396), dict(slots=0x1000 - 504),
                dict(table=0x3000 - 4 * 100), dict(lens=0x5000), dict(pages=0x20000 + 504), dict(lens=0x10000 + 4 * 40 * 7 + 124)):
        assert call(**bad) == INVALID, bad
        assert b"overlap" in lib.basa_last_error()


def test_append_and_gather(lib):  # noqa: F811
    some = V(0x8000)

    def append(k=None, v=None, kp=None, vp=None, slots=some):
        k, v, kp, vp = k or tensor(), v or tensor(), kp or pages(), vp or pages()
        return status_of(lib, lib.basa_cache_append, C.byref(k), C.byref(v), slots, C.byref(kp), C.byref(vp), None)[0]

    def gather(k=None, v=None, kp=None, vp=None, table=some, width=8, stride=8, cu=some, n=3):
        k, v, kp, vp = k or tensor(), v or tensor(), kp or pages(), vp or pages()
        return status_of(lib, lib.basa_cache_gather, C.byref(kp), C.byref(vp), table, width, stride, cu, n, C.byref(k), C.byref(v), None)[0]
    for f in (append, gather):
        for bad in (dict(k=tensor(ptr=0)), dict(v=tensor(ptr=0)), dict(kp=pages(ptr=0)), dict(vp=pages(ptr=0)), dict(k=tensor(dtype=bd.F32)),
                    dict(k=tensor(heads=2), v=tensor(heads=2)), dict(k=tensor(d=64), v=tensor(d=64)), dict(v=tensor(L=49)),
                    dict(vp=pages(batch=99)), dict(vp=pages(L=15)), dict(k=tensor(batch=2), v=tensor(batch=2)), dict(k=tensor(ptr=0x10008)),
                    dict(kp=pages(ptr=0x10008)), dict(k=tensor(stride_l=132)), dict(kp=pages(stride_b=-8)), dict(k=tensor(L=0), v=tensor(L=0)),
                    dict(kp=pages(L=0), vp=pages(L=0)), dict(k=tensor(dtype=7), v=tensor(dtype=7))):
            assert f(**bad) == INVALID, (f.__name__, bad)
        for bad in (dict(kp=pages(d=96), vp=pages(d=96)), dict(k=tensor(L=2 ** 30 + 1), v=tensor(L=2 ** 30 + 1)),
                    dict(kp=pages(heads=65536), vp=pages(heads=65536))):
            assert f(**bad) == UNSUPPORTED, (f.__name__, bad)
    assert append(slots=None) == INVALID
    for bad in (dict(table=None), dict(cu=None), dict(width=0), dict(stride=7), dict(n=-1)):
        assert gather(**bad) == INVALID, bad
    assert gather(width=2 ** 27, stride=2 ** 27) == UNSUPPORTED


def test_decode(lib):  # noqa: F811
    some = V(0x8000)
    strides = lambda *v: (C.c_int64 * 2)(*v)
    query = lambda **kw: tensor(**{**dict(batch=5, heads=8, L=1), **kw})

    def call(q=None, kp=None, vp=None, table=some, width=8, stride=8, lens=some, out=V(0x20000), ostr=None, ws=V(0x100000), n=1 << 40):
        q, kp, vp = q or query(), kp or pages(), vp or pages()
        return status_of(lib, lib.basa_decode_attn, C.byref(q), C.byref(kp), C.byref(vp), table, width, stride, lens, out, ostr, None, ws, n, None)[0]
    for bad in (dict(q=query(ptr=0)), dict(q=query(L=2)), dict(q=query(dtype=bd.F32)), dict(q=query(d=64)), dict(q=query(heads=6)), dict(table=None),
                dict(lens=None), dict(out=None), dict(out=V(0x20008)), dict(width=0), dict(stride=7), dict(ostr=strides(1024, 64)),
                dict(ostr=strides(1028, 128)), dict(ostr=strides(-1024, 128)), dict(vp=pages(heads=2)), dict(ws=V(0x100010))):
        assert call(**bad) == INVALID, bad
    assert call(q=query(d=96), kp=pages(d=96), vp=pages(d=96)) == UNSUPPORTED
    assert call(width=2 ** 27, stride=2 ** 27) == UNSUPPORTED
    assert call(q=query(batch=2 ** 19 + 1)) == UNSUPPORTED and b"batch*heads" in lib.basa_last_error()
    assert call(q=query(batch=100), width=2 ** 26, stride=2 ** 26) == UNSUPPORTED and b"steps" in lib.basa_last_error()
    size = lambda q, kp, w: lib.basa_decode_workspace_size(C.byref(q), C.byref(kp), C.byref(kp), w)
    need = size(query(), pages(), 8)
    assert need > 0 and call(n=need - 1) == WORKSPACE and call(ws=None) == WORKSPACE and b"need" in lib.basa_last_error()
    # more cached tokens never ask for less; a bad descriptor gives no size
    assert need <= size(query(), pages(), 800) <= size(query(), pages(), 80000)
    assert size(query(L=2), pages(), 8) == 0 and size(query(), pages(d=96), 8) == 0 and size(query(), pages(), 0) == 0


def test_the_binding_refuses_what_the_kernels_would_misread():
    bf = torch.bfloat16
    k, v = torch.zeros(9, 4, 16, 64, dtype=bf), torch.zeros(9, 4, 16, 64, dtype=bf)
    cache = bd.PagedCache(k, v)
    assert (cache.pages, cache.heads, cache.page, cache.d) == (9, 4, 16, 64)
    for a, b in ((k, v[:8]), (k, v.float()), (k[0], v[0]), (k.transpose(2, 3), v.transpose(2, 3)), (k.half(), v.half())):
        with pytest.raises(ValueError):
            bd.PagedCache(a, b)
    ints = lambda *shape: torch.zeros(shape, dtype=torch.int32)
    q, rows = torch.zeros(3, 8, 64, dtype=bf), torch.zeros(5, 4, 64, dtype=bf)
    slots, table = torch.zeros(5, dtype=torch.int64), ints(3, 7)
    for bad in (lambda: bd.basa_cache_append(rows, rows, slots[:4], cache), lambda: bd.basa_cache_append(rows, rows, slots.int(), cache),
                lambda: bd.basa_cache_append(rows.float(), rows.float(), slots, cache), lambda: bd.basa_cache_append(rows[:, :2], rows[:, :2], slots, cache),
                lambda: bd.basa_cache_append(rows, rows[:4], slots, cache), lambda: bd.basa_cache_append(rows[0], rows[0], slots, cache),
                lambda: bd.basa_cache_gather(cache, table, ints(3), 5), lambda: bd.basa_cache_gather(cache, table.long(), ints(4), 5),
                lambda: bd.basa_cache_gather(cache, table, ints(4), 5, out=(rows[:4], rows[:4])),
                lambda: bd.basa_decode_attn(q, cache, table[:2], ints(3)), lambda: bd.basa_decode_attn(q, cache, table, ints(4)),
                lambda: bd.basa_decode_attn(q, cache, table.t(), ints(3)), lambda: bd.basa_decode_attn(q.float(), cache, table, ints(3)),
                lambda: bd.basa_decode_attn(q, cache, table, ints(3).long()), lambda: bd.basa_decode_attn(q, cache, table, ints(6)[::2]),
                lambda: bd.basa_decode_attn(q, cache, table, ints(3), out=q[:2]),
                lambda: bd.basa_page_tables(ints(3), ints(2), table, ints(9), 16, 5), lambda: bd.basa_page_tables(ints(2), ints(2), table, ints(9), 16, 5),
                lambda: bd.basa_page_tables(ints(3), ints(3), table, ints(9).long(), 16, 5),
                lambda: bd.basa_page_tables(ints(3), ints(3), table, ints(9), 16, 5, out=bd.PageTables(3, 4, "cpu")),
                lambda: bd.ba_att_cached(rows, rows, rows, [0, 5], cache, table, slots, cached=[1, 2])):
        with pytest.raises(ValueError):
            bad()


def test_calls_go_to_the_device_of_their_tensors(monkeypatch):
    current, seen = [0], []

    class Device:
        def __init__(self, index):
            self.index = index

        def __enter__(self):
            current.append(self.index)

        def __exit__(self, *exc):
            current.pop()

    monkeypatch.setattr(bd, "_current_device", lambda: current[-1])
    monkeypatch.setattr(torch.cuda, "device", Device)
    monkeypatch.setattr(bd, "_raw_stream", lambda index: ("stream of", index))
    for index in (1, 0):
        bd._launch(lambda *args: seen.append((current[-1], args)) or 0, torch.device("cuda", index), 5)
    assert seen == [(1, (5, ("stream of", 1))), (0, (5, ("stream of", 0)))] and current == [0]


def test_strides_of_axes_of_one_do_not_count():
    one = torch.zeros(64, dtype=torch.bfloat16)
    x = one.as_strided((1, 1, 1, 64), (3, 5, 7, 1))
    cache = bd.PagedCache(x, x)
    assert (cache._kd.stride_b, cache._kd.stride_h, cache._kd.stride_l) == (0, 0, 64)
    row = one.as_strided((1, 1, 64), (3, 5, 1))
    desc = bd._packed_desc(row, "k", cache)
    assert desc.stride_h == 0 and desc.stride_l >= 64
    desc = bd._token_desc(row, "q", cache)
    assert (desc.stride_b, desc.stride_h, desc.stride_l) == (0, 0, 64)
