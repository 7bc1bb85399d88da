"""Windows over packed pages where they meet other things: numbers that are not finite
which some tokens see and others do not, trees of more than 64 tokens, tiles of one
half one behind the other, and lengths that change between the replays of a graph."""
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


def _expected(p):
    """out, lse and the bounds of their errors, of the numbers that p holds now."""
    o, w, A, S = lr.attend(p.q, p.lines, p.ctx, p.new, p.mask, p.depth, p.window, p.sinks, p.scale)
    e, el = ref.attend_bounds(o, w, A, S, p.cfg.head_dim, max(c + n for c, n in zip(p.ctx, p.new)), True)
    return o, w, e, el


def _rows_that_see(p, b, places):
    """[new tokens of request b]: whether one sees any of these places."""
    s = lr.seen(p.ctx[b], p.new[b], p.T, None if p.mask is None else p.mask[b], None if p.depth is None else p.depth[b],
                p.window, p.sinks, p.q.device)
    return s[:, places].any(1)


def _plant(p, b, place, key, value):
    """Writes into place's line of the 16-bit cache: {channels: number}."""
    page, row = ref.place(p.table[b], place - p.n4[b] * p.cfg.page_size, p.cfg.page_size)
    for cache, what in ((p.key, key), (p.value, value)):
        for channels, x in what.items():
            cache[page, :, row, channels] = x


def _near(got, want, bound):
    return ((got.double() - want).abs() <= bound).all()


# query rows of a head: the small tiles' one and two columns of eight, two groups of them, one stream, one, two
ROWS = [(6, 1), (6, 2), (7, 4), (40, 1), (9, 8), (40, 4)]


@pytest.mark.parametrize("bad", [math.nan, math.inf, -math.inf])
@pytest.mark.parametrize("T,G", ROWS)
@pytest.mark.parametrize("tree", [False, True])
def test_what_is_outside_a_tokens_window_does_not_reach_it(bad, T, G, tree):
    """Lines behind the packed pages: seen by no token, by the first ones' windows, by all, and a drafted one.  Rows that
    see none of them keep to the definition, the others are not finite."""
    W, near, n4 = 90, [300, 40], [5, 9]
    p = lr.Problem(rheo, near, None, T, 2 * G, 2, 128 if T % 2 else 64, 16, n4=n4, window=W, sinks=2, tree=tree, seed=T + G)
    p.check()
    o, w, e, el = _expected(p)
    c, pk = p.ctx[0], n4[0] * 16
    places = [pk + 3, c - W, c - W + 1, c - W + 2, c + T // 2]
    for l in places:
        _plant(p, 0, l, {slice(None, None, 3): bad}, {slice(1, None, 2): bad})
    out, lse = p.run()
    hit = _rows_that_see(p, 0, places)
    assert rheo.scratch_status(p.ws) == 0 and hit.any() and (tree or not hit.all())
    for b, clear in ((0, ~hit), (1, torch.ones_like(hit))):
        assert _near(out[b][clear], o[b][clear], e[b][clear]) and _near(lse[b][clear], w[b][clear], el[b][clear])
    assert not torch.isfinite(out[0][hit][..., 1::2]).any()


@pytest.mark.parametrize("bad", [math.nan, math.inf, -math.inf])
@pytest.mark.parametrize("T,G", ROWS)
@pytest.mark.parametrize("tree", [False, True])
def test_values_that_are_not_finite_stay_in_their_columns(bad, T, G, tree):
    """A cached value behind the packed pages that only the first tokens' windows reach, one that no token sees, and a
    drafted one."""
    W, n4 = 90, [5]
    p = lr.Problem(rheo, [300], None, T, 2 * G, 2, 64 if T % 2 else 128, 16, n4=n4, window=W, tree=tree, seed=T)
    p.check()
    o, w, e, el = _expected(p)
    c = p.ctx[0]
    planted = {5: c - W + 1, 7: n4[0] * 16 + 1, 9: c + T // 2}
    for d, l in planted.items():
        _plant(p, 0, l, {}, {d: bad})
    out, lse = p.run()
    assert rheo.scratch_status(p.ws) == 0 and _near(lse, w, el)
    for d, l in planted.items():
        hit = _rows_that_see(p, 0, [l])
        col = out[0][hit][..., d]
        assert torch.isnan(col).all() if math.isnan(bad) else (col == bad).all()
        assert _near(out[0][~hit][..., d], o[0][~hit][..., d], e[0][~hit][..., d])
        assert hit.any() == (d != 7) and not hit.all()
    keep = [d for d in range(p.cfg.head_dim) if d not in planted]
    assert _near(out[..., keep], o[..., keep], e[..., keep])


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("T,G", [(10, 4), (40, 2), (20, 8)])
def test_halves_of_tiles_one_behind_the_other(T, G, D):
    """Many items a CTA, whose sinks and whose packed pages end in the first half of a tile of 128: a stream of the second
    halves has no product there.  Behind them 16-bit tiles with drafted values that are not finite, in both halves; the
    columns of the others keep to the definition, and so do the rows that do not see them."""
    P, B = 16, 30
    n4 = [(9, 17, 1, 12, 0, 3)[b % 6] for b in range(B)]
    near = [(100, 60, 3, 127, 130, 64, 20)[b % 7] for b in range(B)]
    p = lr.Problem(rheo, near, None, T, 8 * G, 8, D, P, n4=n4, window=105, sinks=20, seed=T + D)
    p.check()
    o, w, e, el = _expected(p)
    for b in range(B):
        _plant(p, b, p.ctx[b] + T // 2, {}, {b % D: math.inf})
    out, lse = p.run()
    assert rheo.scratch_status(p.ws) == 0 and _near(lse, w, el)
    for b in range(B):
        keep = [d for d in range(D) if d != b % D]
        assert _near(out[b][..., keep], o[b][..., keep], e[b][..., keep])
        hit = _rows_that_see(p, b, [p.ctx[b] + T // 2])
        assert (out[b][hit][..., b % D] == math.inf).all() and hit.any()
        assert _near(out[b][~hit][..., b % D], o[b][~hit][..., b % D], e[b][~hit][..., b % D])


@pytest.mark.parametrize("T,G,D", [(65, 1, 128), (129, 1, 64), (129, 2, 128), (300, 1, 64)])
@pytest.mark.parametrize("window,sinks", [(3, 0), (1, 5), (70, 40), (6, 160), (200, 900), (5000, 2)])
@pytest.mark.parametrize("with_depth", [True, False])
def test_trees_of_more_than_64_tokens(T, G, D, window, sinks, with_depth):
    """Nothing packed, parts of any length, drafted tokens across the tiles' halves; sinks that end in the packed
    part, among the drafted tokens and behind them; positions by depth and by place."""
    near, n4 = [0, 1, 63, 130, 250, 5], [0, 1, 7, 0, 3, 25]
    p = lr.Problem(rheo, near, [T, T, T - 1, T, T // 2, 1], T, 2 * G, 2, D, 32 if T == 129 else 16, n4=n4, tree=True,
                   window=window, sinks=sinks, with_depth=with_depth, seed=T + window)
    p.check()


@pytest.mark.parametrize("T,tree", [(1, False), (7, True), (30, True), (80, True)])
def test_in_a_graph_with_lengths_that_change(T, tree):
    p = lr.Problem(rheo, [100, 90], None, T, 8, 2, 64, 16, n4=[30, 60], window=120, sinks=7, tree=tree, seed=6)
    near, held = i32(p.near), p.held4.n_pages
    call = lambda: rheo.packed_attend(p.cfg, p.cfg4, p.q, p.key, p.value, p.held, near, p.data, p.held4, p.out, p.ws,  # noqa: E731
                                      window=120, sinks=7, depth=p.depth, mask=p.mask, lse=p.lse, scale=p.scale)
    call()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call()
    for lens, packed in (([100, 90], [30, 60]), ([0, 3], [0, 1]), ([77, 0], [21, 59]), ([100, 90], [0, 60])):
        near.copy_(i32(lens))
        held.copy_(i32(packed))
        p.out.fill_(3.0)
        p.lse.fill_(3.0)
        graph.replay()
        torch.cuda.synchronize()
        p.near, p.n4, p.ctx = lens, packed, [c + 16 * n for c, n in zip(lens, packed)]
        o, w, e, el = _expected(p)
        assert _near(p.out, o, e) and _near(p.lse, w, el)
    assert rheo.scratch_status(p.ws) == 0
