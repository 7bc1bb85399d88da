"""Attention limited to a window, with first tokens that stay visible, against its
definition in 64 bits: windows from one place to more than there are, around page and
tile ends, chains and trees, pages outside every window that are gone, and numbers
that are not finite where a token does not see them."""
import math

import pytest
import torch

from paper_2609_21827_gb300 import build, rheo
import cache_reference as ref
import long_reference as lr

pytestmark = pytest.mark.gpu
i32 = lr.i32


@pytest.fixture(scope="module", autouse=True)
def _lib():
    if not torch.cuda.is_available():
        pytest.skip("needs a CUDA GPU")
    build.build()


def _problem(*a, **kw):
    return lr.Problem(rheo, *a, **kw)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("window,sinks", [(1, 0), (1, 5), (16, 0), (33, 1), (100, 70), (129, 4), (1000, 3), (2 ** 31 - 1, 2 ** 31 - 1)])
@pytest.mark.parametrize("T", [1, 3, 40])
def test_windows_around_page_and_tile_ends(dtype, window, sinks, T):
    near = [0, 1, 15, 16, 31, 63, 64, 65, 100, 127, 128, 129, 160, 200, 255, 256, 257, 400]
    _problem(near, None, T, 6, 3, 64, 16, dtype, window=window, sinks=sinks, tree=T == 40, seed=T + window % 97).check()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("Hq,H,D", [(4, 4, 64), (8, 2, 128), (5, 1, 64), (32, 8, 128), (64, 8, 64), (7, 1, 128), (16, 1, 128)])
@pytest.mark.parametrize("T", [1, 2, 49])
def test_head_layouts(dtype, Hq, H, D, T):
    _problem([0, 17, 530, 301], None, T, Hq, H, D, 32, dtype, window=150, sinks=2, tree=T > 2, seed=T + Hq, layout="pairs").check()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("P", [16, 32, 64, 128])
def test_ragged_new_tokens(dtype, P):
    near = [0, 0, P - 1, P, 300, 63, 64, 65, 126, 127, 128, 129, 255, 256]
    new = [0, 1, 1, 3, 9, 1, 9, 0, 2, 1, 4, 9, 1, 9]
    _problem(near, new, 9, 6, 3, 64, P, dtype, window=70, sinks=10, layout="pairs", seed=P).check()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("T,Hq,H,D,window,sinks", [(700, 4, 2, 64, 100, 5), (515, 4, 1, 128, 1, 0), (300, 8, 8, 64, 64, 300),
                                                   (129, 8, 2, 128, 1000, 0), (260, 3, 1, 64, 37, 1)])
def test_prompts(dtype, T, Hq, H, D, window, sinks):
    """Chains longer than the window, behind nothing and behind cached tokens."""
    _problem([0, 250, 33], [T, T - 1, T // 2], T, Hq, H, D, 32, dtype, window=window, sinks=sinks, seed=T).check()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("T,window,sinks", [(61, 3, 0), (61, 1, 2), (129, 2, 140), (30, 70, 0)])
def test_windows_within_a_tree(dtype, T, window, sinks):
    """A window shorter than the tree is deep hides ancestors, by their depth; sinks may lie among the drafted tokens."""
    _problem([0, 9, 140, 1], [T, T // 2, T, T], T, 8, 2, 64, 16, dtype, window=window, sinks=sinks, tree=True, seed=T).check()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_trees_by_place(dtype):
    """Without depths a tree's token has the depth of its place in the call."""
    _problem([5, 200, 40], None, 33, 4, 2, 64, 16, dtype, window=12, sinks=1, tree=True, with_depth=False, seed=1).check()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_depths_out_of_range_count_as_the_nearest(dtype):
    p = _problem([50, 300], None, 9, 4, 2, 64, 16, dtype, window=40, sinks=1, tree=True, seed=2)
    p.depth = i32([[0, -5, 3, 9, 100, 2 ** 31 - 1, -2 ** 31, 8, 1]] * 2)
    p.check()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("T,G", [(1, 4), (13, 4), (61, 4)])
def test_no_window_is_tree_attend(dtype, T, G):
    p = _problem([500, 3, 129], None, T, 2 * G, 2, 128, 16, dtype, window=0, sinks=7, tree=T > 1, seed=3)
    p.check()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("T", [1, 25, 80])
def test_pages_outside_every_window_may_be_gone(dtype, T):
    """Their entries of the table are out of range, or name pages of others that hold no numbers: nothing of it is read."""
    P, W, S = 16, 50, 20
    p = _problem([700, 90, 333], None, T, 4, 2, 64, P, dtype, window=W, sinks=S, tree=T == 25, seed=T)
    clean = [x.clone() for x in p.check()]
    for b, c in enumerate(p.near):
        first, last = -(-S // P), max(0, c - W + 1) // P   # pages wholly behind the sinks and before the first token's window
        for j in range(first, last):
            page = int(p.table[b, j])
            p.key[page], p.value[page] = math.nan, math.inf
            if j % 2:
                p.table[b, j] = (-1, p.cfg.pages, 2 ** 31 - 1)[j % 3]
    got = p.run()
    assert rheo.scratch_status(p.ws) == 0
    assert torch.equal(got[0], clean[0]) and torch.equal(got[1], clean[1])


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("bad", [math.nan, math.inf, -math.inf])
@pytest.mark.parametrize("T,G", [(6, 1), (6, 2), (40, 4)])
def test_what_is_outside_a_tokens_window_does_not_reach_it(dtype, bad, T, G):
    """Cached places that some tokens of the call see and others do not are not finite."""
    W, c = 90, 300
    p = _problem([c, 40], None, T, 2 * G, 2, 128, 16, dtype, window=W, sinks=2, seed=5)
    clean = [x.clone() for x in p.check()]
    places = [c - W + 3, c - W + 4, 10]        # seen by the first tokens only; by none
    for l in places:
        page, row = ref.place(p.table[0], l, 16)
        p.key[page, :, row, ::3], p.value[page, :, row, 1::2] = bad, bad
    out, lse = p.run()
    first = torch.arange(T) + c - W + 1
    sees = (first <= places[1]).cuda()         # token t sees places from first[t] on
    assert sees.any() and not sees.all()
    for b, clear in ((0, ~sees), (1, torch.ones(T, dtype=torch.bool, device="cuda"))):
        assert torch.equal(out[b][clear], clean[0][b][clear]) and torch.equal(lse[b][clear], clean[1][b][clear])
    assert not torch.isfinite(out[0][sees][..., 1::2]).any()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("bad", [math.nan, math.inf, -math.inf])
@pytest.mark.parametrize("T,G", [(5, 2), (30, 4)])
def test_values_that_are_not_finite_stay_in_their_columns(dtype, bad, T, G):
    """A cached value that only the first tokens' windows reach, and a drafted one."""
    W, c = 90, 300
    p = _problem([c], None, T, 2 * G, 2, 64, 16, dtype, window=W, seed=6)
    clean = p.check()[0].clone()
    for l, d in ((c - W + 2, 5), (c + 3, 9)):
        page, row = ref.place(p.table[0], l, 16)
        p.value[page, :, row, d] = bad
    out, _ = p.run()
    t = torch.arange(T, device="cuda")
    for d, sees in ((5, t <= 1), (9, t >= 3)):
        col = out[0, sees][..., d]
        assert torch.isnan(col).all() if math.isnan(bad) else (col == bad).all()
        assert torch.equal(out[0, ~sees][..., d], clean[0, ~sees][..., d])
    keep = [d for d in range(64) if d not in (5, 9)]
    assert torch.equal(out[..., keep], clean[..., keep])


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_masks_that_leave_tokens_empty(dtype):
    T = 20
    p = _problem([0, 0, 70], [T, T, 11], T, 4, 2, 64, 16, dtype, window=3, sinks=0, tree=True, seed=7)
    g = torch.Generator().manual_seed(9)
    p.mask = (torch.rand((3, T, T), generator=g) < 0.15).to(torch.uint8).cuda()
    p.mask[0, 3], p.mask[1], p.mask[2, :, 5] = 0, 0, 255
    p.check()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("B,T,Hq,H,ctx,window", [(1, 1, 8, 1, 20011, 9000), (3, 1, 4, 2, 5003, 4000), (2, 49, 8, 2, 4000, 1500),
                                                 (70, 1, 2, 2, 300, 100), (200, 5, 4, 1, 400, 30)])
def test_long_axes_and_many_requests(dtype, B, T, Hq, H, ctx, window):
    lens = [max(0, ctx - 37 * b * (ctx // (40 * B) + 1)) for b in range(B)]
    _problem(lens, None, T, Hq, H, 128, 64, dtype, window=window, sinks=5, tree=T == 49, seed=B, spread=2.0).check()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_large_scores_and_negative_scale(dtype):
    p = _problem([200, 3], None, 7, 4, 2, 64, 32, dtype, window=60, sinks=2, seed=8, spread=20.0)
    for scale in (p.scale, -0.05, 0.0):
        p.scale = scale
        p.check()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("T", [1, 61])
def test_same_bits_every_time_and_on_another_stream(dtype, T):
    p = _problem([3000, 40, 1200], None, T, 8, 2, 128, 16, dtype, window=700, sinks=4, tree=T > 1, seed=4)
    first = [x.clone() for x in p.check()]
    side = torch.cuda.Stream()
    for stream in (None, side, None):
        p.out.fill_(1.0)
        p.lse.fill_(1.0)
        torch.cuda.synchronize()
        p.run(stream=stream)
        torch.cuda.synchronize()
        assert torch.equal(p.out, first[0]) and torch.equal(p.lse, first[1])


@pytest.mark.parametrize("dtype,T", [("bf16", 1), ("bf16", 9), ("bf16", 40), ("f32", 5)])
def test_in_a_graph_with_lengths_that_change(dtype, T):
    p = _problem([500, 900], None, T, 4, 2, 64, 16, dtype, window=120, sinks=3, seed=6)
    near = i32([500, 900])
    call = lambda: rheo.window_attend(p.cfg, p.q, p.key, p.value, p.held, near, p.out, p.ws, window=120, sinks=3,  # noqa: E731
                                      lse=p.lse)
    call()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call()
    for lens in ([500, 900], [3, 0], [129, 640]):
        near.copy_(i32(lens))
        graph.replay()
        torch.cuda.synchronize()
        p.near = p.ctx = lens
        o, w, A, S = lr.attend(p.q, p.lines, lens, [T, T], None, None, 120, 3, p.scale)
        e, _ = ref.attend_bounds(o, w, A, S, 64, 1000, dtype == "bf16")
        assert ((p.out.double() - o).abs() <= e).all()
    assert rheo.scratch_status(p.ws) == 0


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("T", [3, 40])
def test_bad_lengths_and_pages_set_their_bits(dtype, T):
    p = _problem([60, 60, 60, 60], None, T, 4, 2, 64, 16, dtype, window=30, sinks=1, seed=7)
    good = p.check()[0].clone()
    p.near = [60, -1, 10 ** 6, 60]
    out, lse = p.run()
    assert rheo.scratch_status(p.ws) == rheo.STATUS_BAD_LENGTH
    assert torch.equal(out[0], good[0]) and torch.equal(out[3], good[3])
    assert not out[1:3].any() and (lse[1:3] == -math.inf).all()
    p.near = [60] * 4
    table = p.table.clone()
    for wrong in (p.cfg.pages, -1, 2 ** 31 - 1):
        p.table.copy_(table)
        p.table[2, 3] = wrong                   # places 48 to 63: in every window
        out, _ = p.run()
        assert rheo.scratch_status(p.ws) == rheo.STATUS_BAD_INDEX
        assert torch.equal(out[0], good[0]) and torch.equal(out[1], good[1]) and torch.equal(out[3], good[3])


@pytest.mark.parametrize("dtype,T,G", [("bf16", 1, 4), ("bf16", 49, 4), ("f32", 9, 2)])
def test_many_calls_one_after_the_other(dtype, T, G):
    """Calls that nothing waits between, each with its own tensors and workspace."""
    ps = [_problem([4000 - 500 * b for b in range(8)], None, T, 8 * G, 8, 128, 16, dtype, window=900, sinks=4, seed=20 + i)
          for i in range(3)]
    first = []
    for p in ps:
        first.append([x.clone() for x in p.run()])
        p.out.fill_(1.0)
    near = i32(ps[0].near)
    torch.cuda.synchronize()
    for i in range(60):
        p = ps[i % 3]
        rheo.window_attend(p.cfg, p.q, p.key, p.value, p.held, near, p.out, p.ws, window=900, sinks=4, lse=p.lse, scale=p.scale)
    torch.cuda.synchronize()
    for p, (out, lse) in zip(ps, first):
        assert torch.equal(p.out, out) and torch.equal(p.lse, lse) and rheo.scratch_status(p.ws) == 0
    ps[2].check()


@pytest.mark.parametrize("T", [30, 80])
@pytest.mark.parametrize("D", [64, 128])
def test_scales_below_zero_with_many_rows(T, D):
    p = _problem([500, 3, 129], None, T, 4, 2, D, 32, "bf16", window=150, sinks=5, tree=T == 30, seed=8, spread=8.0)
    for scale in (-0.05, -1.0, 0.05):
        p.scale = scale
        p.check()
