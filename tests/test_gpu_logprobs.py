"""Token log probabilities on the GPU against their definition in 64 bits."""
import math

import pytest
import torch

from paper_2609_21827_gb300 import build, rheo
import cache_reference as ref

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _lib():
    if not torch.cuda.is_available():
        pytest.skip("needs a CUDA GPU")
    build.build()


def _logits(R, V, dtype, kind, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    x = torch.rand((R, V), generator=g, device="cuda")
    if kind == "zipf":
        x = -1.2 * torch.log(1 + x * V) + 0.5 * torch.randn((R, V), generator=g, device="cuda")
    elif kind == "ties":
        x = (4 * x).floor()
    elif kind == "equal":
        x = torch.full_like(x, -2.5)
    elif kind == "rising":  # the largest logits side by side
        x = torch.arange(V, device="cuda").float()[None, :].expand(R, V) * 0.01
    elif kind == "masked":
        x = torch.where(x < 0.97, -math.inf, 3 * torch.randn((R, V), generator=g, device="cuda"))
        x[:, V // 2] = 0.5
    elif kind == "one":
        x = torch.full_like(x, -math.inf)
        x[:, V - 1] = -4.0
    elif kind == "zeros":  # negative and positive zeros are equal
        x = torch.where(x < 0.5, -0.0, 0.0)
    elif kind == "lowest":  # masks of the type's lowest value instead of -inf
        x = torch.where(x < 0.9, torch.finfo(dtype).min, torch.randn((R, V), generator=g, device="cuda"))
    elif kind == "stripes":  # one column in 512 vectors holds all large logits
        x = 0.1 * x
        vec = 8 if dtype == torch.bfloat16 else 4
        at = torch.arange(V, device="cuda") // vec % 512 == 77
        x = torch.where(at[None, :], 5 + torch.randn((R, V), generator=g, device="cuda"), x)
    return x.to(dtype)


def _check(logits, tokens, temps, k, rows, out, per):
    """Sums over V logits in fp32, a few hundred a thread one after the other: 4e-5 relatively; each exponent's
    argument is off by a few roundings of itself."""
    R = tokens.numel()
    n = logits.shape[0]
    for i in range(R):
        r = i if rows is None else int(rows[i])
        if r < 0 or r >= n:
            assert out.logprob[i] == 0 and out.rank[i] == -1 and out.entropy[i] == 0
            assert (out.top_ids[i] == -1).all() and (out.top_logprobs[i] == -math.inf).all()
            continue
        T = 1.0 if temps is None else float(temps[i // per])
        lp, rank, H, ids, lps = ref.logprobs(logits[r], int(tokens[i]), T, k)
        lp, *lps = torch.tensor([lp] + lps, dtype=torch.float64).float().tolist()  # -inf past the type's range
        assert int(out.rank[i]) == rank
        assert out.top_ids[i].tolist() == ids
        x = logits[r].double() / T
        fin = x[torch.isfinite(x) & (x >= x.max() - 200)]
        span = float((fin.max() - fin.min()).abs()) + float(x.max().abs())
        tol = 4e-5 + 16 * ref.U * span
        if lp == -math.inf:
            assert float(out.logprob[i]) == -math.inf
        else:
            assert abs(float(out.logprob[i]) - lp) <= tol + 8 * ref.U * abs(lp)
        assert abs(float(out.entropy[i]) - H) <= tol * (1 + H)
        for a, b in zip(out.top_logprobs[i].tolist(), lps):
            assert a == b if b == -math.inf else abs(a - b) <= tol + 8 * ref.U * abs(b)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("kind", ["zipf", "ties", "equal", "rising", "masked", "one", "zeros", "lowest", "stripes"])
@pytest.mark.parametrize("V,R,k", [(1, 2, 1), (7, 3, 32), (1000, 5, 5), (1003, 2, 32), (32000, 3, 20), (128256, 2, 32),
                                   (151936, 1, 0), (50257, 160, 3)])
def test_rows_of_every_kind(dtype, kind, V, R, k):
    dt = torch.bfloat16 if dtype == "bf16" else torch.float32
    x = _logits(R, V, dt, kind, V + R)
    cfg = rheo.LogprobConfig(rows=R, vocab=V, top=k, dtype=dtype, rows_per_temperature=2)
    g = torch.Generator().manual_seed(V)
    tokens = torch.randint(0, V, (R,), generator=g).to(torch.int32)
    tokens[0] = int(x[0].float().argmax())
    temps = 0.4 + torch.rand(-(-R // 2), generator=g)
    out, ws = rheo.Logprobs(cfg), rheo.LogprobWorkspace(cfg)
    picked = range(R) if R < 20 else range(0, R, 23)
    for t in (None, temps.cuda()):
        rheo.token_logprobs(cfg, x, tokens.cuda(), out, ws, temperature=t)
        assert rheo.scratch_status(ws) == 0
        sub = rheo.Logprobs(rheo.LogprobConfig(rows=len(picked), vocab=V, top=k, dtype=dtype))
        for name in ("logprob", "rank", "entropy", "top_ids", "top_logprobs"):
            setattr(sub, name, getattr(out, name)[list(picked)])
        tt = None if t is None else t[[i // 2 for i in picked]]
        _check(x[list(picked)], tokens[list(picked)], tt, k, None, sub, 1)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("offset,stride", [(0, 1003), (1, 1009), (3, 1016), (8, 1200)])
def test_strides_and_alignment(dtype, offset, stride):
    dt = torch.bfloat16 if dtype == "bf16" else torch.float32
    V, R = 1003, 6
    flat = torch.full((offset + R * stride,), 60.0, dtype=dt, device="cuda")
    x = torch.as_strided(flat, (R, V), (stride, 1), offset)
    x.copy_(_logits(R, V, dt, "zipf", 1))
    cfg = rheo.LogprobConfig(rows=R, vocab=V, top=7, dtype=dtype)
    tokens = torch.arange(0, 1003, 170)[:R].to(torch.int32)
    out, ws = rheo.Logprobs(cfg), rheo.LogprobWorkspace(cfg)
    rheo.token_logprobs(cfg, x, tokens.cuda(), out, ws)
    assert rheo.scratch_status(ws) == 0
    _check(x, tokens, None, 7, None, out, 1)


@pytest.mark.parametrize("V", [900, 60000])
def test_rows_and_tokens_left_out(V):
    x = _logits(10, V, torch.bfloat16, "zipf", 2)
    rows, tokens = [3, -1, 9, 0, 3, 10, -2, 5], [5, 6, -1, V - 1, 0, 1, 2, V]
    cfg = rheo.LogprobConfig(rows=8, vocab=V, top=4, rows_per_temperature=4)
    out, ws = rheo.Logprobs(cfg), rheo.LogprobWorkspace(cfg)
    temps = torch.tensor([0.7, 1.4], device="cuda")
    i32 = dict(dtype=torch.int32, device="cuda")
    for r, t, status in ((rows, tokens, rheo.STATUS_BAD_INDEX), (rows[:5] + [-1, -1, 5], tokens[:7] + [-1], 0)):
        rheo.token_logprobs(cfg, x, torch.tensor(t, **i32), out, ws, temperature=temps, rows=torch.tensor(r, **i32))
        assert rheo.scratch_status(ws) == status
        t = [y if 0 <= y < V else -1 for y in t]
        _check(x, torch.tensor(t), temps, 4, torch.tensor(r), out, 4)


@pytest.mark.parametrize("V", [500, 70000])
def test_faults_in_the_data_set_their_bits_and_stay_in_their_rows(V):
    x = _logits(6, V, torch.float32, "zipf", 3)
    x[1, V // 3], x[2, 5], x[3] = math.nan, math.inf, -math.inf
    cfg = rheo.LogprobConfig(rows=6, vocab=V, top=4, dtype="f32")
    out, ws = rheo.Logprobs(cfg), rheo.LogprobWorkspace(cfg)
    tokens = torch.arange(6, dtype=torch.int32, device="cuda")
    rheo.token_logprobs(cfg, x, tokens, out, ws)
    assert rheo.scratch_status(ws) == rheo.STATUS_BAD_LOGIT | rheo.STATUS_EMPTY_ROW
    good = [0, 4, 5]
    for i in good:
        lp, rank, H, ids, _ = ref.logprobs(x[i], i, 1.0, 4)
        assert int(out.rank[i]) == rank and out.top_ids[i].tolist() == ids
        assert abs(float(out.logprob[i]) - lp) <= 1e-4 and abs(float(out.entropy[i]) - H) <= 1e-3
    for bad in (0.0, -1.0, math.nan, math.inf):
        rheo.token_logprobs(cfg, x[good].repeat(2, 1), tokens, out, ws, temperature=torch.tensor([1, 1, 1, 1, 1, bad], device="cuda"))
        assert rheo.scratch_status(ws) == rheo.STATUS_BAD_TEMPERATURE


def test_the_emitted_path_of_a_verified_tree():
    """Rows and tokens as verification leaves them: the accepted path, the bonus token, then nothing."""
    B, N, V, D = 3, 6, 700, 4
    x = _logits(B * (N + 1), V, torch.bfloat16, "zipf", 5).reshape(B, N + 1, V)
    acc_len, nodes = torch.tensor([0, 2, 4]), torch.tensor([[-1] * 4, [2, 5, -1, -1], [1, 2, 4, 6]])
    toks, bonus = torch.tensor([[-1] * 4, [10, 20, -1, -1], [1, 2, 3, 4]]), torch.tensor([7, 8, 9])
    rows = torch.cat([torch.zeros((B, 1), dtype=torch.int64), nodes], 1)
    rows = torch.where(torch.arange(D + 1)[None, :] <= acc_len[:, None], rows + torch.arange(B)[:, None] * (N + 1), -1)
    t = torch.cat([toks, torch.full((B, 1), -1)], 1).scatter(1, acc_len[:, None], bonus[:, None])
    cfg = rheo.LogprobConfig(rows=B * (D + 1), vocab=V, top=3, rows_per_temperature=D + 1)
    out, ws = rheo.Logprobs(cfg), rheo.LogprobWorkspace(cfg)
    temps = torch.tensor([0.5, 1.0, 2.0], device="cuda")
    rows, t = rows.reshape(-1).to(torch.int32), t.reshape(-1).to(torch.int32)
    rheo.token_logprobs(cfg, x, t.cuda(), out, ws, temperature=temps, rows=rows.cuda())
    assert rheo.scratch_status(ws) == 0
    _check(x.reshape(-1, V), t, temps, 3, rows, out, D + 1)
