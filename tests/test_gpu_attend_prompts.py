"""Attention of hundreds to thousands of new tokens over the paged cache (a prompt, whole or
in stretches) against its definition in 64 bits."""
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


def _i32(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


class Prompt:
    def __init__(self, ctx, new, T, Hq, H, D, P, dtype, seed):
        need = [-(-(c + n) // P) for c, n in zip(ctx, new)]
        self.ctx, self.new, self.P, self.scale = ctx, new, P, D ** -0.5
        self.cfg = rheo.CacheConfig(batch=len(ctx), tokens=T, pages=sum(need) + 1, page_size=P, max_pages=max(need), q_heads=Hq,
                                    kv_heads=H, head_dim=D, dtype=dtype)
        g = torch.Generator(device="cuda").manual_seed(seed)
        rnd = lambda *s: torch.randn(s, generator=g, device="cuda").to(self.cfg.torch_dtype)  # noqa: E731
        self.key, self.value = rnd(self.cfg.pages, H, P, D), rnd(self.cfg.pages, H, P, D)
        self.q = rnd(len(ctx), T, Hq, D)
        order = torch.randperm(self.cfg.pages, generator=torch.Generator().manual_seed(seed)).to(torch.int32)
        table, at = torch.full((len(ctx), max(need)), -1, dtype=torch.int32), 0
        for b, n in enumerate(need):
            table[b, :n] = order[at:at + n]
            at += n
        self.table, self.ws = table.cuda(), rheo.CacheWorkspace(self.cfg)

    def run(self, mask=None):
        out, lse = torch.full_like(self.q, 3.0), torch.full(self.q.shape[:3], 3.0, device="cuda")
        rheo.tree_attend(self.cfg, self.q, self.key, self.value, rheo.Pages(self.cfg, block_table=self.table), _i32(self.ctx), out,
                         self.ws, new_len=_i32(self.new), mask=mask, lse=lse)
        assert rheo.scratch_status(self.ws) == 0
        return out, lse

    def check(self, mask=None):
        out, lse = self.run(mask)
        o, w, A, S = ref.attend(self.q, self.key, self.value, self.table, self.ctx, self.new, mask, self.scale)
        e, el = ref.attend_bounds(o, w, A, S, self.cfg.head_dim, max(c + n for c, n in zip(self.ctx, self.new)),
                                  self.cfg.dtype == "bf16")
        none = w == -math.inf
        assert torch.equal(lse == -math.inf, none) and not out[none].any()
        assert ((out.double() - o).abs() <= e).all() and ((lse.double() - w).abs()[~none] <= el[~none]).all()
        return out, lse


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("T,ctx,new,Hq,H,D,P", [(513, [0, 77], [513, 500], 4, 2, 64, 16), (1000, [0, 300, 5], [1000, 999, 1], 8, 2, 128, 64),
                                                (2048, [3000], [2048], 4, 1, 128, 128), (4096, [0], [4096], 2, 2, 64, 64),
                                                (4096, [33], [4001], 3, 1, 128, 32)])
def test_prompts_behind_any_context(dtype, T, ctx, new, Hq, H, D, P):
    Prompt(ctx, new, T, Hq, H, D, P, dtype, T + Hq).check()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_masks_of_a_thousand_tokens(dtype):
    """Every token sees a random seventh of the others, a few none at all."""
    T = 1000
    mask = (torch.rand((2, T, T), generator=torch.Generator().manual_seed(4)) < 1 / 7).to(torch.uint8)
    mask[0, 10:900:89] = 0
    out, lse = Prompt([0, 130], [T, 700], T, 4, 2, 64, 16, dtype, 5).check(mask.cuda())
    assert (lse[0, 10] == -math.inf).all() and not out[0, 10].any()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("bad", [math.nan, math.inf])
def test_late_tokens_that_are_not_finite_reach_no_earlier_ones(dtype, bad):
    """Values of a few tokens of a long chain are not finite in one column: tokens before them keep their bits, the others
    lose that column alone."""
    T, ctx, col = 1500, 90, 7
    p = Prompt([ctx], [T], T, 4, 2, 64, 16, dtype, 6)
    clean, clean_lse = p.check()
    nodes = [900, 901, 1333]
    for node in nodes:
        page, row = ref.place(p.table[0], ctx + node, 16)
        p.value[page, :, row, col] = bad
    out, lse = p.run()
    first = nodes[0]
    assert torch.equal(out[:, :first], clean[:, :first]) and torch.equal(lse, clean_lse)
    got = out[:, first:, :, col]
    assert torch.isnan(got).all() if math.isnan(bad) else (got == bad).all()
    keep = [d for d in range(64) if d != col]
    assert torch.equal(out[:, first:, :, keep], clean[:, first:, :, keep])
