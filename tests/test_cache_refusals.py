"""What the paged-cache entry points refuse before any launch: outputs over inputs that
other CTAs still read, outputs whose rows share memory, strides out of range.  Host
checks on made-up addresses."""
import ctypes

import pytest

from paper_2609_21827_gb300 import build, rheo


@pytest.fixture(scope="module")
def lib():
    build.build()
    return rheo.lib()


BASE = dict(batch=3, tokens=5, pages=64, page_size=16, max_pages=16, q_heads=4, kv_heads=2, head_dim=64, dtype="bf16")
A = 1 << 20


def _kv(**kw):
    d = dict(key=A, value=A, key_page=2048, key_head=1024, key_token=64, value_page=2048, value_head=1024, value_token=64)
    d.update(kw)
    return ctypes.byref(rheo._KV(**d))


# Refused where next_len lies in, or reaches into, a buffer that the call reads: 3 requests, depth 4, 16 pages each.
CTX, ACC, NODES, TABLE = A, 2 * A, 3 * A, 4 * A


@pytest.mark.parametrize("at", [CTX, CTX + 8, CTX - 8, ACC, ACC + 4, ACC - 4, NODES, NODES + 44, NODES - 8, TABLE, TABLE + 188,
                                TABLE - 4])
def test_commit_into_what_it_reads_is_rejected(lib, at):
    c = rheo.CacheConfig(**BASE)
    assert lib.rheo_cache_commit(c._ref, 1, _kv(), 64, 64, TABLE, CTX, ACC, NODES, 4, at, A, None) == rheo.RHEO_EINVAL


# (where no launch can follow: what is not refused would use the made-up addresses)
@pytest.mark.parametrize("at", [CTX + 12, CTX - 12, ACC + 12, NODES + 48, TABLE + 192, 5 * A])
def test_commit_beside_what_it_reads_is_not(lib, at):
    import torch
    if torch.cuda.is_available():
        pytest.skip("a launch would use made-up addresses")
    c = rheo.CacheConfig(**BASE)
    assert lib.rheo_cache_commit(c._ref, 1, _kv(), 64, 64, TABLE, CTX, ACC, NODES, 4, at, A, None) == rheo.RHEO_ELAUNCH


# [batch][token][head] strides of 3 requests, 5 tokens and 4 query heads of 64
APART = [(1280, 256, 64), (1280, 64, 320), (64, 768, 192), (8192, 1024, 64), (-1280, 256, 64), (1280, 256, -64)]
TOGETHER = [(1280, 256, 0), (1280, 0, 64), (0, 256, 64), (1280, 256, 56), (1280, 192, 64), (1216, 256, 64), (1280, 256, 320),
            (64, 64, 64)]
FAR = [(2 ** 38, 256, 64), (1280, -2 ** 38, 64), (1280, 256, 2 ** 62), (-2 ** 63, 256, 64)]


def _attend(lib, q, out, c):
    io = rheo._AttendIO(A, A, 0, *q, *out)
    return lib.rheo_tree_attend(c._ref, ctypes.byref(io), _kv(), A, A, None, None, 0.1, A, None)


def _rope(lib, q, k, out, c):
    x = rheo._QKV(A, A, A, *q, *k, *k)
    return lib.rheo_qk_norm_rope(c._ref, ctypes.byref(x), None, None, 1e-6, A, 9, 8, 0, A, A, _kv(), A, *out, A, None)


@pytest.mark.parametrize("s", TOGETHER + FAR)
def test_outputs_whose_rows_share_memory_are_rejected(lib, s):
    c = rheo.CacheConfig(**BASE)
    assert _attend(lib, APART[0], s, c) == rheo.RHEO_EINVAL
    assert _rope(lib, APART[0], (640, 128, 64), s, c) == rheo.RHEO_EINVAL


@pytest.mark.parametrize("s", FAR)
def test_strides_of_inputs_out_of_range_are_rejected(lib, s):
    c = rheo.CacheConfig(**BASE)
    assert _attend(lib, s, APART[0], c) == rheo.RHEO_EINVAL
    assert _rope(lib, s, (640, 128, 64), APART[0], c) == rheo.RHEO_EINVAL
    assert _rope(lib, APART[0], s, APART[0], c) == rheo.RHEO_EINVAL


@pytest.mark.parametrize("key,value", [(0, 65536), (65536, 0), (-65536, 65536), (65536, 2 ** 38), (2 ** 62, 65536)])
def test_layers_that_share_memory_are_rejected(lib, key, value):
    c = rheo.CacheConfig(**BASE)
    assert lib.rheo_cache_commit(c._ref, 2, _kv(), key, value, TABLE, CTX, ACC, NODES, 4, 5 * A, A, None) == rheo.RHEO_EINVAL


# (fp32 for the attention: its bf16 form asks the driver for a description of the cache first)
@pytest.mark.parametrize("s", APART)
def test_outputs_in_any_order_and_broadcast_inputs_are_not(lib, s):
    import torch
    if torch.cuda.is_available():
        pytest.skip("a launch would use made-up addresses")
    c = rheo.CacheConfig(**{**BASE, "dtype": "f32"})
    for q in (APART[0], (0, 256, 64), (1280, 0, 0), s):
        assert _attend(lib, q, s, c) == rheo.RHEO_ELAUNCH
        assert _rope(lib, q, (0, 128, 64), s, c) == rheo.RHEO_ELAUNCH
    one = rheo.CacheConfig(**{**BASE, "dtype": "f32", "batch": 1, "tokens": 1, "q_heads": 4})
    assert _attend(lib, (7, 5, 64), (0, 2 ** 60, 64), one) == rheo.RHEO_ELAUNCH
    for key in (0, -64, 65536):
        assert lib.rheo_cache_commit(c._ref, 1, _kv(), key, key, TABLE, CTX, ACC, NODES, 4, 5 * A, A, None) == rheo.RHEO_ELAUNCH
