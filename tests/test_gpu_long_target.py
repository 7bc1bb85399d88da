"""The operators for long contexts together: decoding cycles of a small transformer with
windowed layers and a cache that is packed into 4 bits between the cycles (target.py),
against the same model without a cache."""
import dataclasses

import pytest
import torch

from paper_2609_21827_gb300 import build, cycles, rheo, target
import cache_reference as ref
import long_reference as lr

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _lib():
    if not torch.cuda.is_available():
        pytest.skip("needs a CUDA GPU")
    build.build()


def _run(dtype, B, L, n_cycles, keep=None, **kw):
    V, g = 48, torch.Generator().manual_seed(3)
    shape = target.Shape(vocab=V, dtype=dtype, **kw)
    model = target.Target(shape, seed=1)
    draft = cycles.KGramLM.random(V, 1, 2.0, g)
    cfg = rheo.Config(batch=B, vocab=V, K=3, depth=3, budget=9, m=1, support=V, dtype=dtype)
    prompt = torch.randint(0, V, (B, L), generator=g).cuda()
    T = torch.full((B,), 0.9, device="cuda")
    seed = torch.arange(B, dtype=torch.int64, device="cuda") * 31 + 5
    return model, prompt, T, target.decode(cfg, draft, model, prompt, T, seed, n_cycles, keep=keep)


def _errors(model, prompt, T, got):
    """|reported - dense| of the log probability of every emitted token."""
    L, errors = prompt.shape[1], []
    for b in range(prompt.shape[0]):
        count = int(got.count[b])
        seq = torch.cat([prompt[b], got.tokens[b, :count]])
        y = torch.log_softmax(target.dense_logits(model, seq)[L - 1:L - 1 + count] / float(T[b]), -1)
        errors.append((got.logprobs[b, :count].double() - y.gather(1, got.tokens[b, :count, None])[:, 0]).abs())
    return torch.cat(errors)


@pytest.mark.parametrize("window,sinks", [(1, 0), (7, 2), (20, 0), (33, 5)])
def test_windowed_layers_are_the_dense_models(window, sinks):
    """fp32: log probabilities of every emitted token over many cycles of trees, windows shorter than the trees are
    deep among them.  fp32 errors through three layers stay below 1e-3; a place too many or too few moves a logit by tenths."""
    model, prompt, T, got = _run("f32", 4, 37, 12, layers=3, window=window, sinks=sinks)
    assert int(got.accepted.max()) >= 2
    assert _errors(model, prompt, T, got).max() < 1e-3


def test_the_window_counts():
    """The same tokens under another window have other log probabilities."""
    model, prompt, T, got = _run("f32", 2, 37, 6, layers=3, window=7, sinks=2)
    other = target.Target(dataclasses.replace(model.shape, window=9), seed=1)
    assert _errors(other, prompt, T, got).max() > 1e-2


@pytest.mark.parametrize("kw", [dict(), dict(window=24, sinks=3, layers=3)])
@pytest.mark.parametrize("keep", [0, 16, 40])
def test_packed_cycles_stay_near(keep, kw):
    """A cache in 4 bits but for the latest tokens, prompts of several pages: cycles run, and report log probabilities that
    are the model's own and not those of one with other weights."""
    model, prompt, T, got = _run("bf16", 3, 70, 10, keep=keep, head_dim=128, rot=128, q_heads=8, kv_heads=2, **kw)
    own, other = (_errors(m, prompt, T, got).mean() for m in (model, target.Target(model.shape, seed=9)))
    assert own < other / 4


def test_packed_forward_is_the_attention_over_unpacked_pages():
    """One forward over packed pages against the same forward over a 16-bit cache that holds the unpacked numbers:
    the same sums in another order."""
    shape = target.Shape(vocab=40, head_dim=64, layers=2, window=30, sinks=2)
    model = target.Target(shape, seed=2)
    g = torch.Generator().manual_seed(1)
    B, L, T, P = 2, 75, 6, 16
    tok = torch.randint(0, 40, (B, L + T), generator=g).to(torch.int32).cuda()
    first = target.Cached(model, B, L, 128, P, packed=True)
    first.forward(tok[:, :L].contiguous())
    first.ctx_len.fill_(L)
    first.pack(keep=10)
    assert rheo.scratch_status(first.ws) == 0
    n4 = int(first.packed_pages.n_pages[0])
    assert n4 == (L - 10) // P and first.packed_pages.n_pages.tolist() == [n4] * B
    near = first.ctx_len.clone()
    assert near.tolist() == [L - n4 * P] * B
    # a 16-bit cache with the numbers that the packed pages stand for, then those that were not packed
    plain = target.Cached(model, B, T, 128, P)
    plan, ws = rheo.CachePlan(plain.cfg), rheo.CacheWorkspace(plain.cfg)
    whole = dataclasses.replace(plain.cfg, tokens=L)
    rheo.cache_reserve(whole, plain.ctx_len, plain.pages, rheo.CachePlan(whole), rheo.CacheWorkspace(whole))
    src = first.packed_pages.block_table[:, :n4].reshape(-1).contiguous()
    dst = plain.pages.block_table[:, :n4].reshape(-1).contiguous()
    rheo.cache_unpack(plain.cfg, dataclasses.replace(first.cfg, tokens=T), first.data, plain.key, plain.value, src, dst, ws)
    for b in range(B):
        for x in range(n4 * P, L):
            p, r = ref.place(plain.pages.block_table[b], x, P)
            q, s = ref.place(first.pages.block_table[b], x - n4 * P, P)
            plain.key[:, p, :, r], plain.value[:, p, :, r] = first.key[:, q, :, s], first.value[:, q, :, s]
    plain.ctx_len.fill_(L)
    packed = target.Cached(model, B, T, 128, P, first)
    a, c = packed.forward(tok[:, L:].contiguous()), plain.forward(tok[:, L:].contiguous())
    for net in (packed, plain):
        assert rheo.scratch_status(net.ws) == 0
    # Two layers of at most ten roundings to bf16 each (norm, projections, weights, output, gate, sums), off by up to 2^-8 in
    # each forward; the sums and norms between them keep the 2-norm's order.
    def off(x):
        return float((x.double() - c.double()).norm() / c.double().norm())

    assert off(a) < 20 * 2.0 ** -8
    # and positions: the drafted tokens' keys are those at L ..
    assert torch.equal(packed.plan.position, plain.plan.position)
    # two pages in each other's place are further off than that
    t = first.packed_pages.block_table
    t[:, [n4 - 2, n4 - 1]] = t[:, [n4 - 1, n4 - 2]]
    assert off(packed.forward(tok[:, L:].contiguous())) > 20 * 2.0 ** -8


def test_packed_cycle_in_a_graph():
    """A step of a cycle (reserve, store, attend over packed pages, commit, pack), captured once and replayed, against the
    same calls one by one."""
    B, T, P, H, D = 2, 4, 16, 2, 64
    kw = dict(batch=B, tokens=T, page_size=P, q_heads=4, kv_heads=H, head_dim=D, pages=40, max_pages=20)
    g = torch.Generator(device="cuda").manual_seed(3)
    steps = [torch.randn((B, T, 4 + 2 * H, D), generator=g, device="cuda").bfloat16() for _ in range(40)]
    path = torch.tensor([[1, 2, 3]] * B, dtype=torch.int32, device="cuda")
    some = [torch.tensor([(i + b) % 4 for b in range(B)], dtype=torch.int32, device="cuda") for i in range(40)]

    class Side:
        def __init__(self):
            self.cfg = rheo.CacheConfig(**kw)
            self.key, self.value = rheo.make_cache(self.cfg)
            self.data = rheo.make_packed(self.cfg)
            self.pages, self.pages4, self.plan = rheo.Pages(self.cfg), rheo.Pages(self.cfg), rheo.CachePlan(self.cfg)
            self.ws = rheo.CacheWorkspace(self.cfg)
            self.ctx, self.next = (torch.zeros(B, dtype=torch.int32, device="cuda") for _ in range(2))
            self.qkv, self.take = torch.zeros_like(steps[0]), torch.zeros_like(some[0])
            self.out = torch.zeros((B, T, 4, D), dtype=torch.bfloat16, device="cuda")

        def step(self):
            c, ws = self.cfg, self.ws
            rheo.cache_reserve(c, self.ctx, self.pages, self.plan, ws)
            q, k, v = self.qkv[:, :, :4], self.qkv[:, :, 4:4 + H], self.qkv[:, :, 4 + H:]
            rheo.qk_norm_rope(c, q, k, v, None, None, None, self.plan, self.key[0], self.value[0], q, ws)
            rheo.packed_attend(c, c, q, self.key[0], self.value[0], self.pages, self.ctx, self.data[0], self.pages4, self.out, ws,
                               window=50, sinks=3)
            rheo.cache_commit(c, self.key, self.value, self.pages, self.ctx, self.take, path, self.next, ws)
            self.ctx.copy_(self.next)
            rheo.cache_pack(c, c, self.key, self.value, self.data, self.pages, self.pages4, self.ctx, ws, keep=5)

    a, b = Side(), Side()
    b.step()                                   # outside the graph first
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        b.step()
    # back to the start
    b.ctx.zero_()
    for x, y in ((b.pages, a.pages), (b.pages4, a.pages4)):
        for f in ("block_table", "n_pages", "free_list", "n_free"):
            getattr(x, f).copy_(getattr(y, f))
    for x in (b.key, b.value, b.data):
        x.zero_()
    for i in range(40):
        for s in (a, b):
            s.qkv.copy_(steps[i])
            s.take.copy_(some[i])
        a.step()
        graph.replay()
        assert torch.equal(a.out, b.out) and torch.equal(a.ctx, b.ctx)
        assert torch.equal(a.pages4.block_table, b.pages4.block_table) and torch.equal(a.data, b.data)
    assert int(a.pages4.n_pages.min()) >= 4
    assert rheo.scratch_status(a.ws) == 0 and rheo.scratch_status(b.ws) == 0
