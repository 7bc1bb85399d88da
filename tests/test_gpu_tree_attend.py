"""Attention of drafted tokens over the paged cache against its definition in 64
bits: types, head layouts, strides, page sizes, lengths from nothing to long,
masks that leave tokens without any place, and NaN and infinities in places
that a token does not see."""
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


def _tree_mask(B, T, g):
    """Ancestor masks of random trees."""
    m = torch.zeros((B, T, T), dtype=torch.uint8)
    for b in range(B):
        for i in range(T):
            if i:
                m[b, i] = m[b, int(torch.randint(max(0, i - 7), i, (1,), generator=g))]
            m[b, i, i] = 1
    return m.cuda()


class Problem:
    def __init__(self, ctx, new, T, Hq, H, D, P, dtype, mask=None, layout="heads", seed=0, extra_pages=3, spread=1.0):
        g = torch.Generator().manual_seed(1000 + seed)
        gd = torch.Generator(device="cuda").manual_seed(seed)
        B = len(ctx)
        new = [T] * B if new is None else new
        lens = [c + n for c, n in zip(ctx, new)]
        need = [-(-n // P) for n in lens]
        pages = sum(need) + extra_pages
        width = max(max(need), 1) + 2
        self.cfg = rheo.CacheConfig(batch=B, tokens=T, pages=pages, page_size=P, max_pages=width, q_heads=Hq, kv_heads=H,
                                    head_dim=D, dtype=dtype)
        dt = self.cfg.torch_dtype
        order = torch.randperm(pages, generator=g).tolist()
        table, at = torch.full((B, width), -2 ** 30, dtype=torch.int32), 0
        for b, n in enumerate(need):
            table[b, :n] = torch.tensor(order[at:at + n], dtype=torch.int32)
            at += n
        self.table = table.cuda()
        rnd = lambda *s: torch.randn(s, generator=gd, device="cuda").to(dt)  # noqa: E731
        if layout == "heads":
            self.key, self.value = rnd(pages, H, P, D), rnd(pages, H, P, D)
        elif layout == "tokens":
            self.key, self.value = rnd(pages, P, H, D).transpose(1, 2), rnd(pages, P, H, D).transpose(1, 2)
        else:  # keys and values of a token side by side, heads padded
            pool = rnd(pages, P, H, 2, D + 8 * (4 // dt.itemsize))
            self.key, self.value = (pool[:, :, :, i, :D].transpose(1, 2) for i in (0, 1))
        if layout == "heads":
            self.q = (spread * rnd(B, T, Hq, D)).to(dt)
            self.out = torch.full((B, T, Hq, D), 3.0, dtype=dt, device="cuda")
        else:
            self.q = (spread * rnd(B, T, Hq + 2 * H, D)).to(dt)[:, :, :Hq]
            self.out = torch.full((B, Hq, T, D), 3.0, dtype=dt, device="cuda").transpose(1, 2)
        self.ctx, self.new, self.T, self.mask = ctx, new, T, mask
        self.scale = D ** -0.5
        # what no request holds, and the rest of last pages: not a number
        held = torch.zeros((pages, P), dtype=torch.bool)
        for b, n in enumerate(lens):
            for x in range(n):
                page, row = ref.place(table[b], x, P)
                held[page, row] = True
        hole = ~held.cuda()
        for c in (self.key, self.value):
            c.transpose(1, 2)[hole] = math.nan
        self.lse = torch.full((B, T, Hq), 3.0, device="cuda")
        self.ws = rheo.CacheWorkspace(self.cfg)

    def run(self, new=True, stream=None):
        rheo.tree_attend(self.cfg, self.q, self.key, self.value, rheo.Pages(self.cfg, block_table=self.table),
                         _i32(self.ctx), self.out, self.ws, new_len=_i32(self.new) if new else None, mask=self.mask,
                         lse=self.lse, scale=self.scale, stream=stream)
        return self.out, self.lse

    def check(self, **kw):
        out, lse = self.run(**kw)
        assert rheo.scratch_status(self.ws) == 0
        o, w, A, S = ref.attend(self.q, self.key, self.value, self.table, self.ctx, self.new, self.mask, self.scale)
        L = max(c + n for c, n in zip(self.ctx, self.new))
        e, el = ref.attend_bounds(o, w, A, S, self.cfg.head_dim, L, self.cfg.dtype == "bf16")
        none = w == -math.inf
        assert torch.equal(lse == -math.inf, none) and not out[none].any()
        assert not torch.isnan(out).any()
        err = (out.double() - o).abs()
        assert (err <= e).all(), f"out: {float((err / e).max()):.3g} of the bound"
        err = (lse.double() - w).abs()[~none]
        assert (err <= el[~none]).all(), f"lse: {float((err / el[~none]).max()):.3g} of the bound"
        return out, lse


HEADS = [(4, 4, 64), (8, 2, 128), (5, 1, 64), (32, 8, 128), (40, 40, 128), (64, 8, 64), (7, 1, 128)]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("Hq,H,D", HEADS)
@pytest.mark.parametrize("T", [1, 2, 13, 49])
def test_trees_of_every_head_layout(dtype, Hq, H, D, T):
    g = torch.Generator().manual_seed(T)
    B = 4
    Problem([0, 17, 130, 301], None, T, Hq, H, D, 16, dtype, _tree_mask(B, T, g), seed=T + Hq).check(new=False)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("P", [16, 32, 64, 128])
@pytest.mark.parametrize("layout", ["heads", "tokens", "pairs"])
def test_pages_and_strides(dtype, P, layout):
    """Lengths around page and tile ends, chains (no mask), new tokens fewer than T."""
    ctx = [0, 0, P - 1, P, P + 1, 63, 64, 65, 126, 127, 128, 129, 255, 256]
    new = [0, 1, 1, 3, 9, 1, 9, 0, 2, 1, 4, 9, 1, 9]
    Problem(ctx, new, 9, 6, 3, 64, P, dtype, layout=layout, seed=P).check()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("T,Hq,H,D", [(129, 8, 2, 128), (61, 32, 8, 128), (300, 2, 2, 64), (33, 16, 1, 128), (128, 2, 1, 64)])
def test_more_rows_than_a_tile(dtype, T, Hq, H, D):
    g = torch.Generator().manual_seed(T)
    Problem([5, 0, 250], [T, T - 1, T // 2], T, Hq, H, D, 32, dtype, _tree_mask(3, T, g), seed=T).check()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("B,T,Hq,H,ctx", [(1, 1, 8, 1, 20011), (1, 17, 4, 1, 9001), (3, 1, 4, 2, 5003), (2, 49, 8, 2, 2000),
                                          (70, 1, 2, 2, 300), (200, 5, 4, 1, 40)])
def test_long_axes_are_split_and_joined(dtype, B, T, Hq, H, ctx):
    g = torch.Generator().manual_seed(B)
    lens = [max(0, ctx - 37 * b * (ctx // (40 * B) + 1)) for b in range(B)]
    Problem(lens, None, T, Hq, H, 128, 64, dtype, _tree_mask(B, T, g) if T > 1 else None, seed=B, spread=2.0).check()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_masks_that_leave_tokens_empty(dtype):
    """With nothing cached, a token whose mask row is 0 sees nothing: out 0, lse -inf."""
    T = 20
    g = torch.Generator().manual_seed(9)
    mask = (torch.rand((3, T, T), generator=g) < 0.15).to(torch.uint8)
    mask[0, 3], mask[0, 7], mask[1] = 0, 0, 0
    mask[2, :, 5] = 255  # any value but 0 counts
    p = Problem([0, 0, 70], [T, T, 11], T, 4, 2, 64, 16, dtype, mask.cuda(), seed=5)
    out, lse = p.check()
    assert (lse[0, 3] == -math.inf).all() and (lse[1] == -math.inf).all() and (lse[2, 11:] == -math.inf).all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("bad", [math.nan, math.inf, -math.inf])
def test_what_a_token_does_not_see_does_not_reach_it(dtype, bad):
    """One drafted token's key and value are not finite: tokens that do not see it are as if it were finite."""
    T, node = 30, 11
    g = torch.Generator().manual_seed(2)
    mask = _tree_mask(2, T, g)
    mask[:, :node, node] = 0
    ctx = [100, 9]
    p = Problem(ctx, None, T, 4, 2, 128, 16, dtype, mask, seed=3)
    clean, clean_lse = (x.clone() for x in p.check())
    for b in range(2):
        page, row = ref.place(p.table[b], ctx[b] + node, 16)
        p.key[page, :, row, ::3], p.value[page, :, row, 1::2] = bad, bad
    out, lse = p.run()
    sees = mask[:, :, node] != 0
    assert sees.any() and not sees.all()
    assert torch.equal(out[~sees], clean[~sees]) and torch.equal(lse[~sees], clean_lse[~sees])
    assert not torch.isfinite(out[sees][..., 1::2]).any()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("bad", [math.nan, math.inf, -math.inf])
def test_values_that_are_not_finite_stay_in_their_columns(dtype, bad):
    """Only the value of a drafted token is not finite: its columns alone are lost, for the tokens that see it."""
    T, node = 30, 4
    g = torch.Generator().manual_seed(2)
    mask = _tree_mask(1, T, g)
    p = Problem([100], None, T, 4, 2, 64, 16, dtype, mask, seed=3)
    clean = p.check()[0].clone()
    page, row = ref.place(p.table[0], 100 + node, 16)
    p.value[page, :, row, 5] = bad
    out, _ = p.run()
    sees = mask[:, :, node] != 0
    assert torch.equal(out[~sees], clean[~sees])
    col = out[sees][..., 5]
    assert torch.isnan(col).all() if math.isnan(bad) else (col == bad).all()
    keep = [d for d in range(64) if d != 5]
    assert torch.equal(out[sees][..., keep], clean[sees][..., keep])


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_large_scores_and_negative_scale(dtype):
    """Scores of hundreds: the maximum keeps the weights finite; the sign of the scale is the caller's."""
    p = Problem([200, 3], None, 7, 4, 2, 64, 32, dtype, seed=8, spread=20.0)
    p.check()
    p.scale = -0.05
    p.check()
    p.scale = 0.0
    p.check()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("T,G", [(1, 4), (9, 2), (61, 4)])
def test_scores_that_rise_along_the_context(dtype, T, G):
    """Each stretch of keys is larger than the one before: the running maximum moves again and again."""
    p = Problem([1500, 700, 40], None, T, 2 * G, 2, 128, 16, dtype, seed=12)
    for b, n in enumerate(p.ctx):
        for l in range(n + T):
            page, row = ref.place(p.table[b], l, 16)
            p.key[page, :, row] *= 1 + l // 100
    p.check()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("T,G", [(1, 4), (49, 4)])
def test_many_calls_one_after_the_other(dtype, T, G):
    """Calls that nothing waits between, each with its own tensors and workspace, many key tiles a CTA."""
    ps = [Problem([4000 - 500 * b for b in range(8)], None, T, 8 * G, 8, 128, 16, dtype, seed=20 + i) for i in range(3)]
    first = []
    for p in ps:
        first.append([x.clone() for x in p.run(new=False)])
        torch.cuda.synchronize()
    ctx, pages = _i32(ps[0].ctx), [rheo.Pages(p.cfg, block_table=p.table) for p in ps]
    for p in ps:
        p.out.fill_(1.0)
        p.lse.fill_(1.0)
    torch.cuda.synchronize()
    for i in range(60):
        p = ps[i % 3]
        rheo.tree_attend(p.cfg, p.q, p.key, p.value, pages[i % 3], ctx, p.out, p.ws, lse=p.lse, scale=p.scale)
    torch.cuda.synchronize()
    for p, (out, lse) in zip(ps, first):
        assert torch.equal(p.out, out) and torch.equal(p.lse, lse)
        assert rheo.scratch_status(p.ws) == 0
    ps[2].check(new=False)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("T,G", [(1, 4), (65, 2)])
def test_runs_of_short_items_between_long_ones(dtype, T, G):
    """Many items of one key tile in a row in every CTA, in calls that nothing waits between."""
    ctx = [(37 * b) % 60 for b in range(500)]
    ctx[100] = ctx[300] = 2000
    ps = [Problem(ctx, None, T, 8 * G, 8, 64, 16, dtype, seed=30 + i) for i in range(2)]
    for p in ps:
        p.run(new=False)
    for i in range(20):
        ps[i % 2].run(new=False)
    for p in ps:
        p.check(new=False)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_same_bits_every_time_and_on_another_stream(dtype):
    p = Problem([3000, 40, 1200], None, 17, 8, 2, 128, 16, dtype, seed=4)
    first = [x.clone() for x in p.check()]
    side = torch.cuda.Stream()
    for stream in (None, side, None):
        p.out.fill_(1.0)
        p.lse.fill_(1.0)
        torch.cuda.synchronize()
        p.run(stream=stream)
        torch.cuda.synchronize()
        assert torch.equal(p.out, first[0]) and torch.equal(p.lse, first[1])


def test_in_a_graph_with_lengths_that_change():
    """The lengths are read on the GPU: a captured call follows them."""
    p = Problem([500, 900], None, 5, 4, 2, 64, 16, "bf16", seed=6)
    ctx, pages = _i32([500, 900]), rheo.Pages(p.cfg, block_table=p.table)
    call = lambda: rheo.tree_attend(p.cfg, p.q, p.key, p.value, pages, ctx, p.out, p.ws, lse=p.lse)  # noqa: E731
    call()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call()
    for lens in ([500, 900], [3, 0], [129, 640]):
        ctx.copy_(_i32(lens))
        graph.replay()
        torch.cuda.synchronize()
        o, w, A, S = ref.attend(p.q, p.key, p.value, p.table, lens, [5, 5], None, p.scale)
        e, _ = ref.attend_bounds(o, w, A, S, 64, 905, True)
        assert ((p.out.double() - o).abs() <= e).all()
    assert rheo.scratch_status(p.ws) == 0


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_bad_lengths_and_pages_set_their_bits(dtype):
    p = Problem([40, 40, 40, 40], None, 3, 4, 2, 64, 16, dtype, seed=7)
    good = p.check()[0].clone()
    p.ctx = [40, -1, 10 ** 6, 40]
    out, lse = p.run()
    assert rheo.scratch_status(p.ws) == rheo.STATUS_BAD_LENGTH
    assert torch.equal(out[0], good[0]) and torch.equal(out[3], good[3])
    assert not out[1:3].any() and (lse[1:3] == -math.inf).all()
    p.ctx = [40] * 4
    for wrong in (p.cfg.pages, -1, 2 ** 31 - 1):
        table = p.table.clone()
        p.table[2, 1] = wrong
        out, _ = p.run()
        assert rheo.scratch_status(p.ws) == rheo.STATUS_BAD_INDEX
        assert torch.equal(out[0], good[0]) and torch.equal(out[1], good[1]) and torch.equal(out[3], good[3])
        p.table = table


def test_a_tree_of_the_pipeline():
    """Expand, prune, tree_attention and the attention under its mask."""
    from paper_2609_21827_gb300 import synth
    import dataclasses

    w = dataclasses.replace(synth.WORKLOADS["tiny"], name="tiny_b3", batch=3)
    cfg = rheo.Config(batch=3, vocab=w.vocab, K=w.K, depth=w.depth, budget=w.budget, m=w.m, dtype=w.dtype)
    draft = synth.make_draft_inputs(w, device="cuda")
    tree, pr, ws, ta = rheo.Tree(cfg), rheo.Pruned(cfg), rheo.Workspace(cfg), rheo.TreeAttn(cfg)
    for d in range(1, cfg.depth + 1):
        rheo.expand(cfg, d, draft.rows[d - 1], draft.temperature, draft.seed, draft.offset, tree, ws)
    rheo.prune(cfg, tree, pr, ws)
    rheo.tree_attention(cfg, pr, ta, ws)
    for dtype in ("bf16", "f32"):
        Problem([33, 0, 80], None, w.budget + 1, 4, 2, 64, 16, dtype, ta.mask, seed=1).check(new=False)
