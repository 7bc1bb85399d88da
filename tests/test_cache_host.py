"""Host checks of the paged-cache and log-probability entry points: what they
refuse before any launch, and the sizes they ask for."""
import ctypes

import pytest
import torch

from paper_2609_21827_gb300 import build, rheo


@pytest.fixture(scope="module")
def lib():
    build.build()
    return rheo.lib()


BASE = dict(batch=2, tokens=5, pages=64, page_size=16, max_pages=16, q_heads=4, kv_heads=2, head_dim=64, dtype="bf16")


@pytest.mark.parametrize("good", [dict(), dict(batch=4096), dict(tokens=4096), dict(page_size=128, head_dim=128),
                                  dict(q_heads=40, kv_heads=40), dict(dtype="f32"), dict(q_heads=1024, kv_heads=1)])
def test_sizes(lib, good):
    assert 0 < rheo.CacheConfig(**{**BASE, **good}).scratch_bytes() < 2 ** 28


@pytest.mark.parametrize("bad", [dict(batch=0), dict(batch=4097), dict(tokens=0), dict(tokens=4097), dict(page_size=8),
                                 dict(page_size=48), dict(page_size=256), dict(pages=0), dict(max_pages=0),
                                 dict(max_pages=2 ** 27), dict(head_dim=96), dict(head_dim=256), dict(kv_heads=0),
                                 dict(kv_heads=3), dict(q_heads=1), dict(q_heads=2048),
                                 dict(batch=4096, max_pages=2 ** 20)])
def test_invalid_cache_configurations_are_rejected(lib, bad):
    with pytest.raises(rheo.RheoError):
        rheo.CacheConfig(**{**BASE, **bad}).scratch_bytes()


@pytest.mark.parametrize("bad", [dict(rows=0), dict(rows=2 ** 20 + 1), dict(vocab=0), dict(vocab=262145), dict(top=-1),
                                 dict(top=33), dict(rows_per_temperature=0)])
def test_invalid_logprob_configurations_are_rejected(lib, bad):
    base = dict(rows=4, vocab=1000, top=5)
    assert rheo.LogprobConfig(**base).scratch_bytes() > 0
    with pytest.raises(rheo.RheoError):
        rheo.LogprobConfig(**{**base, **bad}).scratch_bytes()


def test_unknown_types_are_rejected():
    for cls, kw in ((rheo.CacheConfig, {**BASE, "dtype": "f16"}), (rheo.LogprobConfig, dict(rows=1, vocab=9, dtype="f64"))):
        with pytest.raises(rheo.RheoError):
            cls(**kw)


# Made-up addresses: every case is refused before any of them is used.
A = 4096


def _kv(**kw):
    d = dict(key=A, value=A, key_page=2048, key_head=1024, key_token=64, value_page=2048, value_head=1024, value_token=64)
    d.update(kw)
    return ctypes.byref(rheo._KV(**d))


BAD_KV = [dict(key=0), dict(value=0), dict(key=A + 8), dict(value=A + 2), dict(key_page=2044), dict(value_token=68),
          dict(key_head=1)]


@pytest.mark.parametrize("kw", BAD_KV)
def test_caches_without_alignment_are_rejected(lib, kw):
    c = rheo.CacheConfig(**BASE)
    io = rheo._AttendIO(A, A, 0, *[64] * 6)
    assert lib.rheo_tree_attend(c._ref, ctypes.byref(io), _kv(**kw), A, A, None, None, 0.1, A, None) == rheo.RHEO_EINVAL
    x = rheo._QKV(A, A, A, *[64] * 9)
    assert lib.rheo_qk_norm_rope(c._ref, ctypes.byref(x), None, None, 1e-6, A, 9, 8, 0, A, A, _kv(**kw), A, 64, 64, 64, A,
                                 None) == rheo.RHEO_EINVAL
    assert lib.rheo_cache_commit(c._ref, 1, _kv(**kw), 64, 64, A, A, A, A, 3, 2 * A, A, None) == rheo.RHEO_EINVAL


def test_attend_refusals(lib):
    c = rheo.CacheConfig(**BASE)
    good = dict(io=rheo._AttendIO(A, A, 0, *[64] * 6), table=A, ctx=A, scale=0.1, ws=A)
    for bad in (dict(io=rheo._AttendIO(0, A, 0, *[64] * 6)), dict(io=rheo._AttendIO(A, 0, 0, *[64] * 6)),
                dict(io=rheo._AttendIO(A + 4, A, 0, *[64] * 6)), dict(io=rheo._AttendIO(A, A, 0, 64, 64, 63, 64, 64, 64)),
                dict(table=0), dict(ctx=0), dict(ws=0), dict(scale=float("nan")), dict(scale=float("inf"))):
        x = {**good, **bad}
        assert lib.rheo_tree_attend(c._ref, ctypes.byref(x["io"]), _kv(), x["table"], x["ctx"], None, None, x["scale"],
                                    x["ws"], None) == rheo.RHEO_EINVAL
    assert lib.rheo_tree_attend(None, ctypes.byref(good["io"]), _kv(), A, A, None, None, 0.1, A, None) == rheo.RHEO_EINVAL


def test_rope_refusals(lib):
    c = rheo.CacheConfig(**BASE)
    base = dict(q=A, strides=[64] * 9, qw=None, eps=1e-6, cs=A, most=9, rot=8, inter=0, slot=A, pos=A, out=A, os=64, ws=A)
    for bad in (dict(q=0), dict(q=A + 8), dict(strides=[64] * 8 + [4]), dict(qw=A + 2), dict(eps=-1.0),
                dict(eps=float("nan")), dict(cs=None), dict(cs=A + 4), dict(most=0), dict(rot=-8), dict(rot=4), dict(rot=72),
                dict(inter=2), dict(slot=None), dict(pos=None), dict(out=None), dict(out=A + 6), dict(os=60), dict(ws=None)):
        x = {**base, **bad}
        qkv = rheo._QKV(x["q"], A, A, *x["strides"])
        assert lib.rheo_qk_norm_rope(c._ref, ctypes.byref(qkv), x["qw"], None, x["eps"], x["cs"], x["most"], x["rot"],
                                     x["inter"], x["slot"], x["pos"], _kv(), x["out"], 64, 64, x["os"], x["ws"],
                                     None) == rheo.RHEO_EINVAL, bad


def test_reserve_and_commit_refusals(lib):
    c = rheo.CacheConfig(**BASE)
    one, two = rheo._Pages(A, 2 * A, 3 * A, 4 * A), rheo._Pages(5 * A, 6 * A, 7 * A, 8 * A)
    half = rheo._Pages(A, 2 * A, 7 * A, 8 * A)  # part in place, part not
    gone = rheo._Pages(A, 0, 3 * A, 4 * A)
    for before, after, ctx, slot, ws in ((one, half, A, A, A), (gone, two, A, A, A), (one, gone, A, A, A),
                                         (one, two, None, A, A), (one, two, A, None, A), (one, two, A, A, None)):
        assert lib.rheo_cache_reserve(c._ref, ctx, None, None, ctypes.byref(before), ctypes.byref(after), slot, A, ws,
                                      None) == rheo.RHEO_EINVAL
    good = dict(layers=1, kl=64, vl=64, ctx=A, depth=3, nxt=2 * A)
    for bad in (dict(layers=0), dict(layers=5000), dict(kl=4), dict(vl=12), dict(ctx=None), dict(depth=0), dict(depth=129),
                dict(nxt=None), dict(nxt=A)):
        x = {**good, **bad}
        assert lib.rheo_cache_commit(c._ref, x["layers"], _kv(), x["kl"], x["vl"], A, x["ctx"], A, A, x["depth"], x["nxt"],
                                     A, None) == rheo.RHEO_EINVAL, bad


def test_logprob_refusals(lib):
    c = rheo.LogprobConfig(rows=4, vocab=1000, top=5)
    out = rheo._Logprobs(A, A, A, A, A)
    base = dict(logits=A, stride=1000, n=4, tok=A, out=out, ws=A)
    for bad in (dict(logits=None), dict(logits=A + 1), dict(stride=999), dict(n=0), dict(tok=None), dict(ws=None),
                dict(out=rheo._Logprobs(0, A, A, A, A)), dict(out=rheo._Logprobs(A, A, A, 0, A)),
                dict(out=rheo._Logprobs(A, A, A, A, 0))):
        x = {**base, **bad}
        assert lib.rheo_token_logprobs(c._ref, x["logits"], x["stride"], x["n"], None, x["tok"], None, ctypes.byref(x["out"]),
                                       x["ws"], None) == rheo.RHEO_EINVAL, bad


def test_tensors_on_the_host_are_refused():
    """The binding wants CUDA tensors of the configuration's types and shapes."""
    c = rheo.CacheConfig(**BASE)
    x = torch.zeros((2, 5, 4, 64), dtype=torch.bfloat16)
    with pytest.raises(rheo.RheoError):
        rheo.tree_attend(c, x, x, x, None, None, x, None)
    with pytest.raises(rheo.RheoError):
        rheo.qk_norm_rope(c, x, x, x, None, None, None, None, x, x, x, None)
    with pytest.raises(rheo.RheoError):
        rheo.cache_commit(c, x, x, None, None, None, x, None, None)
    lc = rheo.LogprobConfig(rows=2, vocab=10)
    with pytest.raises(rheo.RheoError):
        rheo.token_logprobs(lc, torch.zeros((2, 10)), torch.zeros(2, dtype=torch.int32), None, None)


@pytest.mark.parametrize("kw", [dict(key_head=0), dict(value_page=0), dict(key_token=-64), dict(value_head=2 ** 39)])
def test_cache_strides_out_of_range_are_rejected(lib, kw):
    """A head that is broadcast (stride 0), negative strides and strides past the range."""
    c = rheo.CacheConfig(**BASE)
    io = rheo._AttendIO(A, A, 0, *[64] * 6)
    assert lib.rheo_tree_attend(c._ref, ctypes.byref(io), _kv(**kw), A, A, None, None, 0.1, A, None) == rheo.RHEO_EINVAL
