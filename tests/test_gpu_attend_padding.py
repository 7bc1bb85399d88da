"""Tokens past new_len in the attention over the paged cache: whatever their queries
hold, out is 0 and lse -infinity, in items that one CTA holds and in items that
several share, and the tokens beside them are as if the padding were not there."""
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


# contexts, new tokens, T, query heads, key/value heads: live and padded tokens share 32 rows in each
CASES = [([4000], [37], 61, 8, 2), ([9000], [3], 8, 4, 2), ([2500, 3100, 40], [5, 61, 0], 61, 4, 4),
         ([300 + 29 * b for b in range(70)], [b % 5 for b in range(70)], 5, 6, 2), ([5000, 60], [1, 20], 150, 2, 1)]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("case", range(len(CASES)))
def test_padded_tokens_of_any_content(dtype, case):
    ctx, new, T, Hq, H = CASES[case]
    B, D, P, scale = len(ctx), 128, 64, 128 ** -0.5
    need = [-(-(c + n) // P) for c, n in zip(ctx, new)]
    cfg = rheo.CacheConfig(batch=B, tokens=T, pages=sum(need), page_size=P, max_pages=max(need), q_heads=Hq, kv_heads=H,
                           head_dim=D, dtype=dtype)
    g = torch.Generator(device="cuda").manual_seed(case)
    rnd = lambda *s: torch.randn(s, generator=g, device="cuda").to(cfg.torch_dtype)  # noqa: E731
    key, value, q = rnd(cfg.pages, H, P, D), rnd(cfg.pages, H, P, D), rnd(B, T, Hq, D)
    order = torch.randperm(cfg.pages, generator=torch.Generator().manual_seed(case)).to(torch.int32)
    table, at = torch.full((B, cfg.max_pages), -1, dtype=torch.int32), 0
    for b, n in enumerate(need):
        table[b, :n] = order[at:at + n]
        at += n
    table = table.cuda()
    i32 = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")  # noqa: E731
    pages, ws = rheo.Pages(cfg, block_table=table), rheo.CacheWorkspace(cfg)
    pad = torch.arange(T, device="cuda")[None, :] >= i32(new)[:, None]
    o, w, A, S = ref.attend(q, key, value, table, ctx, new, None, scale)
    e, el = ref.attend_bounds(o, w, A, S, D, max(ctx) + T, dtype == "bf16")
    first = None
    for fill in (0.0, math.nan, math.inf, -math.inf, 3e38):
        q[pad] = fill
        out, lse = torch.full_like(q, 3.0), torch.full((B, T, Hq), 3.0, device="cuda")
        rheo.tree_attend(cfg, q, key, value, pages, i32(ctx), out, ws, new_len=i32(new), lse=lse)
        assert rheo.scratch_status(ws) == 0
        assert not torch.isnan(out).any() and not out[pad].any() and (lse[pad] == -math.inf).all()
        assert ((out.double() - o).abs() <= e).all()
        assert ((lse.double() - w).abs()[~pad] <= el[~pad]).all()
        first = first or (out, lse)
        assert torch.equal(out, first[0]) and torch.equal(lse, first[1])
