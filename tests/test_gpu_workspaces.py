"""One scratch buffer serves every function and every configuration that it is large
enough for, in any order: what one call leaves behind reaches no other call."""
import pytest
import torch

from paper_2609_21827_gb300 import build, rheo
import cache_reference as ref

pytestmark = pytest.mark.gpu

V = 40000  # rows are cut, into two segments (bf16) or up to four (fp32), where there are at most 152


@pytest.fixture(scope="module", autouse=True)
def _lib():
    if not torch.cuda.is_available():
        pytest.skip("needs a CUDA GPU")
    build.build()


def _i32(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


def _logits(R, dtype, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return (4 * torch.randn((R, V), generator=g, device="cuda")).to(torch.bfloat16 if dtype == "bf16" else torch.float32)


def _check_rows(x, ws, dtype, top=4):
    """Every row's outputs, all of them poisoned beforehand.  Tolerance: the sum of V exponentials in fp32, some hundred a
    thread one after the other, is good to 4e-5; logits lie within 25 of 0, and each exponent's
    argument is off by a few roundings of up to 70."""
    R = x.shape[0]
    cfg = rheo.LogprobConfig(rows=R, vocab=V, top=top, dtype=dtype)
    out = rheo.Logprobs(cfg)
    for y in (out.logprob, out.rank, out.entropy, out.top_ids, out.top_logprobs):
        y.fill_(-77)
    tokens = torch.arange(R, dtype=torch.int32, device="cuda") * 7 + 3
    rheo.token_logprobs(cfg, x, tokens, out, ws)
    assert rheo.scratch_status(ws) == 0
    y = torch.log_softmax(x.double(), -1)
    lp = y.gather(1, tokens.long()[:, None])[:, 0]
    assert x.float().abs().max() < 25
    tol = 4e-5 + 24 * ref.U * 70
    assert ((out.logprob.double() - lp).abs() <= tol).all()
    own = x.float().gather(1, tokens.long()[:, None])
    ids = torch.arange(V, device="cuda")[None, :]
    rank = ((x.float() > own) | ((x.float() == own) & (ids < tokens.long()[:, None]))).sum(1)
    assert torch.equal(out.rank.long(), rank)
    H = -(y.exp() * y).sum(-1)
    assert ((out.entropy.double() - H).abs() <= tol * (1 + H)).all()
    want = torch.sort(x.float(), dim=1, descending=True, stable=True).indices[:, :top]
    assert torch.equal(out.top_ids.long(), want)
    assert ((out.top_logprobs.double() - y.gather(1, want)).abs() <= tol).all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("order", [(10, 100), (1, 152), (60, 30, 152, 3, 77), (40, 400, 120)])
def test_log_probabilities_of_fewer_rows_then_of_more(dtype, order):
    ws = rheo.LogprobWorkspace(rheo.LogprobConfig(rows=max(order), vocab=V, top=4, dtype=dtype))
    for i, R in enumerate(order):
        _check_rows(_logits(R, dtype, i), ws, dtype)


@pytest.mark.parametrize("first", [7, 152])
def test_a_workspace_of_one_configuration_is_large_enough_for_every_other(first):
    ws = rheo.LogprobWorkspace(rheo.LogprobConfig(rows=first, vocab=50, top=0, dtype="f32"))
    for R in (100, 2, 200):
        _check_rows(_logits(R, "bf16", R), ws, "bf16")


def _reserve(ws, ctx, T=5):
    cfg = rheo.CacheConfig(batch=len(ctx), tokens=T, pages=64, page_size=16, max_pages=16, q_heads=4, kv_heads=2, head_dim=64)
    pages, plan = rheo.Pages(cfg), rheo.CachePlan(cfg)
    table, owned = pages.block_table.tolist(), pages.n_pages.tolist()
    free, n_free = pages.free_list.tolist(), int(pages.n_free)
    rheo.cache_reserve(cfg, _i32(ctx), pages, plan, ws)
    assert rheo.scratch_status(ws) == 0
    want = ref.reserve(ctx, [T] * len(ctx), None, table, owned, free, n_free, 16, T, 16)
    assert pages.block_table.tolist() == want[0] and pages.n_pages.tolist() == want[1]
    assert pages.n_free.tolist() == [want[3]] and plan.slot.tolist() == want[4] and plan.position.tolist() == want[5]


def _attend(ws, dtype, ctx, T, seed):
    cfg = rheo.CacheConfig(batch=len(ctx), tokens=T, pages=160, page_size=64, max_pages=64, q_heads=4, kv_heads=2, head_dim=64,
                           dtype=dtype)
    g = torch.Generator(device="cuda").manual_seed(seed)
    rnd = lambda *s: torch.randn(s, generator=g, device="cuda").to(cfg.torch_dtype)  # noqa: E731
    key, value, q = rnd(160, 2, 64, 64), rnd(160, 2, 64, 64), rnd(len(ctx), T, 4, 64)
    table = torch.randperm(160, generator=torch.Generator().manual_seed(seed))[: len(ctx) * 64 if len(ctx) < 3 else 128]
    table = table.reshape(len(ctx), -1)
    table = torch.cat([table, torch.zeros((len(ctx), 64 - table.shape[1]), dtype=torch.int64)], 1).to(torch.int32).cuda()
    out = torch.full_like(q, 3.0)
    lse = torch.full((len(ctx), T, 4), 3.0, device="cuda")
    rheo.tree_attend(cfg, q, key, value, rheo.Pages(cfg, block_table=table), _i32(ctx), out, ws, lse=lse)
    assert rheo.scratch_status(ws) == 0
    o, w, A, S = ref.attend(q, key, value, table, ctx, [T] * len(ctx), None, 64 ** -0.5)
    e, el = ref.attend_bounds(o, w, A, S, 64, max(ctx) + T, dtype == "bf16")
    assert ((out.double() - o).abs() <= e).all() and ((lse.double() - w).abs() <= el).all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_the_functions_in_turn_on_one_buffer(dtype):
    """Tables, attention that leaves parts of split items, and log probabilities that leave parts of cut rows."""
    cfg = rheo.CacheConfig(batch=4, tokens=40, pages=160, page_size=64, max_pages=64, q_heads=4, kv_heads=2, head_dim=64, dtype=dtype)
    ws = rheo.CacheWorkspace(cfg)
    turns = [(10, [3000, 41], 40), (100, [1000, 900, 800, 700], 9), (152, [3500], 1), (3, [2000, 2], 17)]
    for i, (R, ctx, T) in enumerate(turns):
        _attend(ws, dtype, ctx, T, i)
        _check_rows(_logits(R, dtype, i), ws, dtype)
        _reserve(ws, [3, 40, 17, 90][: 1 + i])
        _check_rows(_logits(152 - R, dtype, i + 9) if R < 152 else _logits(20, dtype, 9), ws, dtype)
        _reserve(ws, [50, 4, 5])
