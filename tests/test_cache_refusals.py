"""What the paged-cache entry points refuse before any launch: outputs over inputs that
other CTAs still read.  Host checks on made-up addresses."""
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
