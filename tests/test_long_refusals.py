"""What the entry points for windows and 4-bit caches refuse before any launch, and the
sizes they ask for.  Host checks on made-up addresses."""
import ctypes

import pytest
import torch

from paper_2609_21827_gb300 import build, rheo


@pytest.fixture(scope="module")
def lib():
    build.build()
    return rheo.lib()


BASE = dict(batch=3, tokens=5, pages=64, page_size=16, max_pages=16, q_heads=4, kv_heads=2, head_dim=64, dtype="bf16")
A = 1 << 20


def _cfg(**kw):
    return rheo.CacheConfig(**{**BASE, **kw})


def _kv(**kw):
    d = dict(key=A, value=A, key_page=2048, key_head=1024, key_token=64, value_page=2048, value_head=1024, value_token=64)
    d.update(kw)
    return ctypes.byref(rheo._KV(**d))


def _io(**kw):
    d = dict(q=A, out=A, lse=0, q_batch=1280, q_token=256, q_head=64, out_batch=1280, out_token=256, out_head=64)
    d.update(kw)
    return ctypes.byref(rheo._AttendIO(**d))


def _p4(**kw):
    d = dict(data=A, page=2240, head=1120)
    d.update(kw)
    return ctypes.byref(rheo._Packed(**d))


@pytest.mark.parametrize("P,D,want", [(16, 64, 1120), (16, 128, 2240), (32, 128, 4352), (64, 128, 8704), (128, 64, 8704)])
def test_page_bytes(lib, P, D, want):
    assert rheo.packed_page_bytes(_cfg(page_size=P, head_dim=D)) == want


def test_fp32_caches_are_not_packed(lib):
    c = _cfg(dtype="f32")
    with pytest.raises(rheo.RheoError):
        rheo.packed_page_bytes(c)
    assert _packed_attend(lib, c=c, c4=c) == rheo.RHEO_EINVAL
    assert _pack(lib, c=c, c4=c) == rheo.RHEO_EINVAL
    assert _unpack(lib, c=c, c4=c) == rheo.RHEO_EINVAL


def _window_attend(lib, c=None, io=None, kv=None, table=A, ctx=A, window=None, scale=0.1, ws=A):
    c = c or _cfg()
    w = ctypes.byref(rheo._Window(4, 2, 0)) if window is None else window
    return lib.rheo_window_attend(c._ref, io or _io(), kv or _kv(), table, ctx, None, None, w, scale, ws, None)


@pytest.mark.parametrize("bad", [dict(io=_io(q=0)), dict(io=_io(out=A + 8)), dict(io=_io(out_token=192)), dict(io=_io(q_head=62)),
                                 dict(kv=_kv(key=0)), dict(kv=_kv(value_token=0)), dict(kv=_kv(key_page=2 ** 38)), dict(table=None),
                                 dict(ctx=None), dict(ws=None), dict(scale=float("nan")), dict(scale=float("inf")),
                                 dict(window=ctypes.byref(rheo._Window(-1, 0, 0))), dict(window=ctypes.byref(rheo._Window(1, -1, 0)))])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_window_attend_refuses(lib, bad, dtype):
    assert _window_attend(lib, c=_cfg(dtype=dtype), **bad) == rheo.RHEO_EINVAL


def test_window_attend_wants_a_window(lib):
    assert lib.rheo_window_attend(_cfg()._ref, _io(), _kv(), A, A, None, None, None, 0.1, A, None) == rheo.RHEO_EINVAL


def _packed_attend(lib, c=None, c4=None, io=None, kv=None, table=A, ctx=A, p4=None, table4=A, n4=A, window=None, scale=0.1, ws=A):
    c, c4 = c or _cfg(), c4 or _cfg(pages=9, max_pages=7)
    return lib.rheo_packed_attend(c._ref, c4._ref, io or _io(), kv or _kv(), table, ctx, None, p4 or _p4(), table4, n4, None,
                                  window, scale, ws, None)


BAD_PACKED = [dict(p4=_p4(data=0)), dict(p4=_p4(data=A + 8)), dict(p4=_p4(page=2248)), dict(p4=_p4(head=0)),
              dict(p4=_p4(head=-1120)), dict(p4=_p4(page=2 ** 39))]
OTHER = [dict(batch=2), dict(tokens=6), dict(page_size=32), dict(q_heads=2), dict(kv_heads=4), dict(head_dim=128), dict(dtype="f32"),
         dict(pages=0), dict(max_pages=0)]


@pytest.mark.parametrize("bad", BAD_PACKED + [dict(table4=None), dict(n4=None), dict(io=_io(q=0)), dict(kv=_kv(key_head=4)),
                                              dict(scale=float("nan")), dict(ws=None),
                                              dict(window=ctypes.byref(rheo._Window(-1, 0, 0)))])
def test_packed_attend_refuses(lib, bad):
    assert _packed_attend(lib, **bad) == rheo.RHEO_EINVAL


@pytest.mark.parametrize("other", OTHER)
def test_packed_pools_of_other_shapes_are_refused(lib, other):
    c4 = _cfg(**{**dict(pages=9, max_pages=7), **other})
    assert _packed_attend(lib, c4=c4) == rheo.RHEO_EINVAL
    assert _pack(lib, c4=c4) == rheo.RHEO_EINVAL
    assert _unpack(lib, c4=c4) == rheo.RHEO_EINVAL


def test_both_parts_together_stay_in_range(lib):
    half = 2 ** 25 + 1
    assert _packed_attend(lib, c=_cfg(batch=1, max_pages=half), c4=_cfg(batch=1, pages=9, max_pages=half)) == rheo.RHEO_EINVAL


# pointers of the nine tables, far apart
X = [A * (i + 1) for i in range(9)]
Y = [A * (i + 11) for i in range(9)]


def _pack(lib, c=None, c4=None, layers=1, kv=None, kl=131072, vl=131072, p4=None, pl=20160, keep=3, x=None, y=None, ws=A * 30):
    c, c4 = c or _cfg(), c4 or _cfg(pages=9, max_pages=7)
    x, y = x or X, y or Y
    pages = lambda v: ctypes.byref(rheo._Pages(*v))  # noqa: E731
    return lib.rheo_cache_pack(c._ref, c4._ref, layers, kv or _kv(), kl, vl, p4 or _p4(), pl, keep, pages(x[:4]), pages(x[4:8]),
                               x[8], pages(y[:4]), pages(y[4:8]), y[8], ws, None)


def _but(v, i, z):
    return v[:i] + [z] + v[i + 1:]


SIZES = [3 * 16, 3, 64, 1, 3 * 7, 3, 9, 1, 3]  # ints of each table


@pytest.mark.parametrize("bad", BAD_PACKED + [dict(layers=0), dict(layers=4097), dict(keep=-1), dict(ws=None), dict(kv=_kv(key=0)),
                                              dict(layers=2, kl=0), dict(layers=2, vl=-131072), dict(layers=2, kl=2 ** 38),
                                              dict(layers=2, pl=8), dict(layers=2, pl=20144), dict(p4=_p4(head=1104)),
                                              dict(p4=_p4(page=1120))])
def test_pack_refuses(lib, bad):
    assert _pack(lib, **bad) == rheo.RHEO_EINVAL


@pytest.mark.parametrize("i", range(9))
def test_pack_refuses_tables_that_share_memory(lib, i):
    assert _pack(lib, x=_but(X, i, 0)) == rheo.RHEO_EINVAL and _pack(lib, y=_but(Y, i, 0)) == rheo.RHEO_EINVAL
    assert _pack(lib, y=_but(X, i, Y[i])) == rheo.RHEO_EINVAL  # part in place, part not
    assert _pack(lib, y=_but(Y, i, X[i])) == rheo.RHEO_EINVAL
    for j in range(9):
        if i != j:
            into = Y[j] + 4 * (SIZES[j] - 1)  # its last element
            assert _pack(lib, y=_but(Y, i, into)) == rheo.RHEO_EINVAL
            assert _pack(lib, y=_but(Y, i, X[j] + 4 * (SIZES[j] - 1))) == rheo.RHEO_EINVAL
            z = _but(X, i, X[j] + 4 * (SIZES[j] - 1))
            assert _pack(lib, x=z, y=z) == rheo.RHEO_EINVAL


def _unpack(lib, c=None, c4=None, layers=1, kv=None, kl=131072, vl=131072, p4=None, pl=20160, n=2, src=A, dst=A, ws=A):
    c, c4 = c or _cfg(), c4 or _cfg(pages=9, max_pages=7)
    return lib.rheo_cache_unpack(c._ref, c4._ref, layers, p4 or _p4(), pl, kv or _kv(), kl, vl, n, src, dst, ws, None)


@pytest.mark.parametrize("bad", BAD_PACKED + [dict(layers=0), dict(n=-1), dict(src=None), dict(dst=None), dict(ws=None),
                                              dict(kv=_kv(key_token=56)), dict(kv=_kv(value_head=64)), dict(kv=_kv(key_page=1024)),
                                              dict(layers=2, kl=64), dict(layers=2, vl=0), dict(layers=2, pl=24)])
def test_unpack_refuses(lib, bad):
    assert _unpack(lib, **bad) == rheo.RHEO_EINVAL


def test_unpacking_nothing_is_done_at_once(lib):
    assert _unpack(lib, n=0, src=None, dst=None) == rheo.RHEO_OK


def test_what_is_not_refused(lib):
    """Layouts in any order reach the launch (which fails here: no GPU)."""
    if torch.cuda.is_available():
        pytest.skip("a launch would use made-up addresses")
    assert _pack(lib) == rheo.RHEO_ELAUNCH and _pack(lib, x=X, y=X) == rheo.RHEO_ELAUNCH
    assert _pack(lib, p4=_p4(page=1120, head=1120 * 9)) == rheo.RHEO_ELAUNCH
    assert _pack(lib, layers=2, p4=_p4(page=4480), pl=2240) == rheo.RHEO_ELAUNCH
    assert _unpack(lib, kv=_kv(key_page=2048, key_head=64, key_token=128)) == rheo.RHEO_ELAUNCH
    assert _unpack(lib, layers=2, kv=_kv(key_page=4096, value_page=4096), kl=2048, vl=2048) == rheo.RHEO_ELAUNCH
    assert _window_attend(lib, c=_cfg(dtype="f32")) == rheo.RHEO_ELAUNCH


def test_tensors_of_other_kinds_are_refused():
    """The binding wants CUDA tensors of the configurations' types and shapes."""
    c = _cfg()
    x, pool = torch.zeros((3, 5, 4, 64), dtype=torch.bfloat16), torch.zeros((1, 64, 2, 16, 64), dtype=torch.bfloat16)
    with pytest.raises(rheo.RheoError):
        rheo.window_attend(c, x, pool[0], pool[0], None, None, x, None, 4)
    with pytest.raises(rheo.RheoError):
        rheo.packed_attend(c, c, x, pool[0], pool[0], None, None, torch.zeros((64, 2, 1120), dtype=torch.uint8), None, x, None)
    with pytest.raises(rheo.RheoError):
        rheo.cache_pack(c, c, pool, pool, torch.zeros((1, 64, 2, 1120), dtype=torch.uint8), None, None, None, None)
    with pytest.raises(rheo.RheoError):
        rheo.cache_pack(c, c, pool[0], pool[0], torch.zeros((64, 2, 1120), dtype=torch.uint8), None, None, None, None)
    with pytest.raises(rheo.RheoError):
        rheo.cache_unpack(c, c, torch.zeros((1, 64, 2, 1120), dtype=torch.uint8), pool, pool, None, None, None)


@pytest.mark.parametrize("wrong", [-1, 2 ** 31, 2 ** 32, 2 ** 32 + 5, -2 ** 32])
def test_counts_past_32_bits(wrong):
    """The binding does not hand over what 32 bits would turn into another number."""
    c = _cfg()
    for call in (lambda: rheo._window(c, wrong, 0, None), lambda: rheo._window(c, 1, wrong, None),
                 lambda: rheo.cache_pack(c, c, None, None, None, None, None, None, None, keep=wrong)):
        with pytest.raises(rheo.RheoError, match="2\\^31"):
            call()
    assert rheo._window(c, 2 ** 31 - 1, 2 ** 31 - 1, None).window == 2 ** 31 - 1


@pytest.mark.parametrize("T,Hq,H,more", [(1, 4, 2, True), (5, 4, 2, True), (16, 4, 2, True), (17, 4, 2, False), (129, 32, 8, False)])
@pytest.mark.parametrize("D", [64, 128])
def test_scratch_sizes(lib, T, Hq, H, more, D):
    """Only the functions over packed pages ask for the parts of their small tiles; the others ask for no more than before, as
    buffers made for other configurations serve them."""
    c = _cfg(tokens=T, q_heads=Hq, kv_heads=H, head_dim=D)
    rows = min(-(-T * Hq // H // 8) * 8, 128 if T * Hq // H <= 128 else 256)
    parts = 2 * 152 * rows * (D + 2) * 4
    assert parts < c.scratch_bytes() < parts + 8192
    assert 4 * parts < c.packed_scratch_bytes() < 4 * parts + 16384 if more else c.packed_scratch_bytes() == c.scratch_bytes()
    ws = rheo.CacheWorkspace.__new__(rheo.CacheWorkspace)
    ws.nbytes, ws._ptr = c.scratch_bytes(), 1 << 20
    assert ws.of(c) == 1 << 20
    if more:
        with pytest.raises(rheo.RheoError, match="packed"):
            ws.of_packed(c)
    ws.nbytes = rheo.CacheWorkspace._size(c)
    assert ws.of(c) == ws.of_packed(c) == 1 << 20
    assert rheo.CacheWorkspace._size(_cfg(dtype="f32")) == _cfg(dtype="f32").scratch_bytes()
