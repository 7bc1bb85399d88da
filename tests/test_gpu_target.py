"""The cache operators together: decoding cycles whose target is a small transformer
with a paged cache (target.py), against the same model without a cache."""

import pytest
import torch

from paper_2609_21827_gb300 import build, cycles, rheo, target

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _lib():
    if not torch.cuda.is_available():
        pytest.skip("needs a CUDA GPU")
    build.build()


def _run(dtype, B, L, n_cycles, **kw):
    V, g = 48, torch.Generator().manual_seed(3)
    shape = target.Shape(vocab=V, dtype=dtype, **kw)
    model = target.Target(shape, seed=1)
    draft = cycles.KGramLM.random(V, 1, 2.0, g)
    cfg = rheo.Config(batch=B, vocab=V, K=3, depth=3, budget=9, m=1, support=V, dtype=dtype)
    prompt = torch.randint(0, V, (B, L), generator=g).cuda()
    T = torch.full((B,), 0.9, device="cuda")
    seed = torch.arange(B, dtype=torch.int64, device="cuda") * 31 + 5
    return model, prompt, T, target.decode(cfg, draft, model, prompt, T, seed, n_cycles)


@pytest.mark.parametrize("kw", [dict(), dict(q_heads=8, kv_heads=2, head_dim=128, rot=128), dict(rot=32)])
def test_cached_log_probabilities_are_the_dense_models(kw):
    """fp32: the reported log probabilities and entropies of every emitted token, over many cycles of reserve, store,
    attend, verify and commit, are those of the dense model on the emitted sequence.  fp32 errors through two layers
    stay below 1e-3 here; a line of the cache at a wrong place moves a logit by tenths."""
    B, L, n = 4, 21, 12
    model, prompt, T, got = _run("f32", B, L, n, **kw)
    assert int(got.accepted.max()) >= 2 and int(got.accepted.min()) == 0  # paths of several lengths were moved
    for b in range(B):
        count = int(got.count[b])
        toks = got.tokens[b, :count]
        assert (toks >= 0).all() and (got.tokens[b, count:] == -1).all()
        seq = torch.cat([prompt[b], toks])
        y = torch.log_softmax(target.dense_logits(model, seq)[L - 1:L - 1 + count] / float(T[b]), -1)
        lp = y.gather(1, toks[:, None])[:, 0]
        assert (got.logprobs[b, :count].double() - lp).abs().max() < 1e-3
        assert (got.entropy[b, :count].double() + (y.exp() * y).sum(-1)).abs().max() < 1e-3


def test_bf16_cycles_run_and_stay_near():
    """bf16: rounding differs between the two, so the log probabilities agree roughly; a misplaced line would not."""
    B, L, n = 3, 33, 10
    model, prompt, T, got = _run("bf16", B, L, n, head_dim=128, rot=128, q_heads=8, kv_heads=2)
    err = []
    for b in range(B):
        count = int(got.count[b])
        seq = torch.cat([prompt[b], got.tokens[b, :count]])
        y = torch.log_softmax(target.dense_logits(model, seq)[L - 1:L - 1 + count] / float(T[b]), -1)
        err.append((got.logprobs[b, :count].double() - y.gather(1, got.tokens[b, :count, None])[:, 0]).abs())
    assert torch.cat(err).mean() < 0.1


def test_prompt_in_one_pass_equals_token_by_token():
    """The cache after a chain of L tokens in one call is what L calls of one token leave, to rounding."""
    shape = target.Shape(vocab=40, dtype="f32", head_dim=64)
    model = target.Target(shape, seed=2)
    g = torch.Generator().manual_seed(1)
    tok = torch.randint(0, 40, (2, 19), generator=g).to(torch.int32).cuda()
    whole, step = target.Cached(model, 2, 19, 64), target.Cached(model, 2, 1, 64)
    a = whole.forward(tok)
    outs = []
    for t in range(19):
        outs.append(step.forward(tok[:, t:t + 1].contiguous()))
        step.ctx_len += 1
    b = torch.cat(outs, 1)
    assert (a - b).abs().max() < 1e-3
    for i in range(2):
        want = target.dense_logits(model, tok[i])
        assert (a[i].double() - want).abs().max() < 1e-3
    assert rheo.scratch_status(whole.ws) == 0 and rheo.scratch_status(step.ws) == 0
