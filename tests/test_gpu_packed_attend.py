"""Attention over pages in 4 bits and the 16-bit ones behind them, against its
definition in 64 bits on the numbers that the packed pages stand for."""
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


@pytest.mark.parametrize("Hq,H,D", [(4, 4, 64), (8, 2, 128), (5, 1, 64), (32, 8, 128), (40, 40, 128), (64, 8, 64), (7, 1, 128),
                                    (16, 1, 64), (20, 1, 128)])
@pytest.mark.parametrize("T", [1, 2, 13, 49])
def test_head_layouts(Hq, H, D, T):
    _problem([0, 17, 30, 1], None, T, Hq, H, D, 16, n4=[0, 1, 9, 20], tree=T > 2, seed=T + Hq).check()


@pytest.mark.parametrize("P", [16, 32, 64, 128])
@pytest.mark.parametrize("layout", ["heads", "pairs"])
@pytest.mark.parametrize("T", [1, 9, 33])
def test_parts_of_every_length(P, layout, T):
    """Nothing packed, nothing in 16 bits, both; odd numbers of pages; new tokens fewer than T."""
    n4 = [0, 0, 1, 1, 2, 3, 3, 4, 5, 7, 0, 6, 2, 9]
    near = [0, 5, 0, 1, P - 1, P, 0, 33, 31, 32, 70, 129, 2 * P, 64]
    new = [T, 1, T, 0, 1, T, 1, T, T // 2 + 1, 1, 0, T, T, 1]
    _problem(near, new, T, 6, 3, 64 if P == 32 else 128, P, n4=n4, layout=layout, seed=P + T).check()


@pytest.mark.parametrize("T,Hq,H,D", [(129, 8, 2, 128), (61, 32, 8, 128), (300, 2, 2, 64), (33, 16, 1, 128), (128, 2, 1, 64),
                                      (500, 4, 2, 128)])
@pytest.mark.parametrize("tree", [False, True])
def test_more_rows_than_an_item(T, Hq, H, D, tree):
    _problem([5, 0, 250], [T, T - 1, T // 2], T, Hq, H, D, 32, n4=[3, 7, 0], tree=tree, seed=T).check()


@pytest.mark.parametrize("T,Hq,H", [(8, 4, 2), (9, 2, 1), (5, 8, 2), (16, 4, 2), (17, 4, 2), (31, 1, 1), (32, 2, 2), (33, 1, 1), (4, 8, 1)])
@pytest.mark.parametrize("tree", [False, True])
@pytest.mark.parametrize("window", [0, 70])
def test_rows_where_the_tiles_change(T, Hq, H, tree, window):
    """16 to 34 query rows of a head: one group of the small tiles, two, the tensor cores' tiles."""
    _problem([5, 0, 250, 33], [T, T - 1, 1, T], T, Hq, H, 128 if T % 2 else 64, 32, n4=[3, 7, 0, 60], tree=tree, window=window,
             sinks=3, seed=T).check()


@pytest.mark.parametrize("window,sinks", [(1, 0), (1, 5), (16, 0), (33, 1), (100, 70), (129, 40), (300, 3), (2 ** 31 - 1, 9)])
@pytest.mark.parametrize("T", [1, 3, 40])
@pytest.mark.parametrize("P", [16, 64])
def test_windows_over_both_parts(window, sinks, T, P):
    near = [0, 1, 15, 40, 130, 33, 0, 64]
    n4 = [0, 1, 3, 5, 2, 0, 7, 4]
    _problem(near, None, T, 6, 3, 64, P, n4=n4, window=window, sinks=sinks, tree=T == 40, seed=T + window % 97).check()


@pytest.mark.parametrize("T", [1, 25])
def test_packed_pages_outside_every_window_may_be_gone(T):
    P, W, S = 16, 200, 20
    p = _problem([50, 9, 130], None, T, 4, 2, 64, P, n4=[40, 20, 9], window=W, sinks=S, tree=T == 25, seed=T)
    clean = [x.clone() for x in p.check()]
    for b, c in enumerate(p.ctx):
        for j in range(-(-S // P), min(p.n4[b], max(0, c - W + 1) // P)):
            p.table4[b, j] = (-1, p.cfg4.pages, 2 ** 31 - 1)[j % 3]
    got = p.run()
    assert rheo.scratch_status(p.ws) == 0
    assert torch.equal(got[0], clean[0]) and torch.equal(got[1], clean[1])


@pytest.mark.parametrize("B,T,Hq,H,n4", [(1, 1, 8, 1, 310), (1, 17, 4, 1, 140), (3, 1, 4, 2, 80), (2, 49, 8, 2, 31), (70, 1, 2, 2, 4),
                                         (200, 5, 4, 1, 1), (1, 1, 16, 1, 200), (1, 4, 8, 8, 100)])
def test_long_axes_are_split_and_joined(B, T, Hq, H, n4):
    _problem([(37 * b + 5) % 90 for b in range(B)], None, T, Hq, H, 128, 64, n4=[n4 - n4 * b // (2 * B) for b in range(B)],
             tree=T == 49, seed=B, spread=2.0).check()


def test_masks_that_leave_tokens_empty():
    T = 20
    p = _problem([0, 0, 70], [T, T, 11], T, 4, 2, 64, 16, n4=[0, 0, 2], tree=True, seed=5)
    g = torch.Generator().manual_seed(9)
    p.mask = (torch.rand((3, T, T), generator=g) < 0.15).to(torch.uint8).cuda()
    p.mask[0, 3], p.mask[1], p.mask[2, :, 5] = 0, 0, 255
    p.check()


@pytest.mark.parametrize("bad", [math.nan, math.inf, -math.inf])
@pytest.mark.parametrize("T,G", [(7, 2), (30, 4)])
def test_what_a_token_does_not_see_does_not_reach_it(bad, T, G):
    node = 5
    p = _problem([20, 9], None, T, 2 * G, 2, 128, 16, n4=[6, 0], tree=True, seed=3)
    p.mask[:, :node, node] = 0
    clean, clean_lse = (x.clone() for x in p.check())
    for b in range(2):
        page, row = ref.place(p.table[b], p.near[b] + node, 16)
        p.key[page, :, row, ::3], p.value[page, :, row, 1::2] = bad, bad
    out, lse = p.run()
    sees = p.mask[:, :, node] != 0
    assert sees.any() and not sees.all()
    assert torch.equal(out[~sees], clean[~sees]) and torch.equal(lse[~sees], clean_lse[~sees])
    assert not torch.isfinite(out[sees][..., 1::2]).any()


@pytest.mark.parametrize("bad", [math.nan, math.inf, -math.inf])
@pytest.mark.parametrize("T,G", [(5, 2), (30, 4)])
def test_values_that_are_not_finite_stay_in_their_columns(bad, T, G):
    p = _problem([40], None, T, 2 * G, 2, 64, 16, n4=[5], seed=6)
    clean = p.check()[0].clone()
    page, row = ref.place(p.table[0], 40 + 3, 16)
    p.value[page, :, row, 9] = bad
    out, _ = p.run()
    col = out[0, 3:][..., 9]
    assert torch.isnan(col).all() if math.isnan(bad) else (col == bad).all()
    keep = [d for d in range(64) if d != 9]
    assert torch.equal(out[0, :3], clean[0, :3]) and torch.equal(out[0, 3:][..., keep], clean[0, 3:][..., keep])


def test_large_scores_and_negative_scale():
    p = _problem([200, 3], None, 7, 4, 2, 64, 32, n4=[4, 1], seed=8, spread=20.0)
    for scale in (p.scale, -0.05, 0.0):
        p.scale = scale
        p.check()


@pytest.mark.parametrize("T", [40, 80])
@pytest.mark.parametrize("window", [0, 150])
@pytest.mark.parametrize("D", [64, 128])
def test_scales_below_zero_with_many_rows(T, window, D):
    """One stream of rows, and two."""
    p = _problem([200, 3], None, T, 4, 2, D, 32, n4=[4, 9], seed=8, spread=8.0, window=window, sinks=5, tree=T == 40)
    for scale in (-0.05, -1.0, 0.05):
        p.scale = scale
        p.check()


@pytest.mark.parametrize("T,G", [(1, 4), (4, 4), (61, 4)])
def test_scores_that_rise_along_the_context(T, G):
    """Scales grow page by page: the running maximum moves again and again."""
    p = _problem([100, 7], None, T, 2 * G, 2, 128, 16, n4=[60, 9], seed=12)
    N, D = 16, 128
    for b in range(2):
        for j in range(p.n4[b]):
            keys = p.data[int(p.table4[b, j]), :, N * D:N * D + D]
            keys += 8 * (j // 20)              # twice as much every 20 pages
    p.check()


@pytest.mark.parametrize("T", [1, 4, 17])
def test_same_bits_every_time_and_on_another_stream(T):
    p = _problem([30, 40, 0], None, T, 8, 2, 128, 16, n4=[190, 3, 77], tree=T > 1, seed=4)
    first = [x.clone() for x in p.check()]
    side = torch.cuda.Stream()
    for stream in (None, side, None):
        p.out.fill_(1.0)
        p.lse.fill_(1.0)
        torch.cuda.synchronize()
        p.run(stream=stream)
        torch.cuda.synchronize()
        assert torch.equal(p.out, first[0]) and torch.equal(p.lse, first[1])


@pytest.mark.parametrize("T", [1, 30])
def test_in_a_graph_with_lengths_that_change(T):
    p = _problem([100, 90], None, T, 8, 2, 64, 16, n4=[30, 60], seed=6)
    near, n4 = i32(p.near), p.held4.n_pages
    call = lambda: rheo.packed_attend(p.cfg, p.cfg4, p.q, p.key, p.value, p.held, near, p.data, p.held4, p.out, p.ws,  # noqa: E731
                                      lse=p.lse)
    call()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call()
    for lens, packed in (([100, 90], [30, 60]), ([0, 3], [0, 1]), ([77, 0], [21, 59])):
        near.copy_(i32(lens))
        n4.copy_(i32(packed))
        graph.replay()
        torch.cuda.synchronize()
        p.near, p.n4, p.ctx = lens, packed, [c + 16 * n for c, n in zip(lens, packed)]
        o, w, A, S = lr.attend(p.q, p.lines, p.ctx, [T, T], None, None, 0, 0, p.scale)
        e, _ = ref.attend_bounds(o, w, A, S, 64, 1100, True)
        assert ((p.out.double() - o).abs() <= e).all()
    assert rheo.scratch_status(p.ws) == 0


@pytest.mark.parametrize("T", [3, 40])
def test_bad_lengths_and_pages_set_their_bits(T):
    p = _problem([20, 20, 20, 20], None, T, 4, 2, 64, 16, n4=[5, 5, 5, 5], seed=7)
    good = p.check()[0].clone()
    for n4 in ([5, -1, p.cfg4.max_pages + 1, 5], [5, 2 ** 31 - 1, -2 ** 31, 5]):
        p.held4.n_pages.copy_(i32(n4))
        out, lse = p.run()
        assert rheo.scratch_status(p.ws) == rheo.STATUS_BAD_LENGTH
        assert torch.equal(out[0], good[0]) and torch.equal(out[3], good[3])
        assert not out[1:3].any() and (lse[1:3] == -math.inf).all()
    p.held4.n_pages.copy_(i32([5] * 4))
    table = p.table4.clone()
    for wrong in (p.cfg4.pages, -1, 2 ** 31 - 1):
        p.table4.copy_(table)
        p.table4[2, 3] = wrong
        out, lse = p.run()
        assert rheo.scratch_status(p.ws) == rheo.STATUS_BAD_INDEX
        assert torch.equal(out[0], good[0]) and torch.equal(out[1], good[1]) and torch.equal(out[3], good[3])
        assert torch.isfinite(out[2]).all()


@pytest.mark.parametrize("P,D", [(16, 64), (16, 128), (32, 128), (128, 64)])
@pytest.mark.parametrize("T", [1, 3, 40])
def test_bad_pages_read_as_zeros(T, P, D):
    """The same bits as over a page whose numbers are all 0 (n + 8 = 8: one bit of four, at bit 2 modulo 4)."""
    p = _problem([20, 20, 20], None, T, 8, 2, D, P, n4=[5, 6, 5], seed=9)
    table = p.table4.clone()
    spare = table[1, 5].item()
    zeros = p.data[spare].clone()
    p.data[spare] = 0x44
    p.held4.n_pages.copy_(i32([5, 5, 5]))
    for at in (0, 3, 4):
        p.table4.copy_(table)
        p.table4[2, at] = spare
        want = [x.clone() for x in p.run()]
        assert rheo.scratch_status(p.ws) == 0
        k, v = lr.unpack_pages(p.data[spare].cpu().numpy(), P, D)
        assert not k.any() and not v.any() and zeros.any()
        for wrong in (p.cfg4.pages, -1):
            p.table4[2, at] = wrong
            out, lse = p.run()
            assert rheo.scratch_status(p.ws) == rheo.STATUS_BAD_INDEX
            assert torch.equal(out, want[0]) and torch.equal(lse, want[1])


@pytest.mark.parametrize("T,G", [(1, 4), (49, 4)])
def test_many_calls_one_after_the_other(T, G):
    ps = [_problem([7 * b for b in range(8)], None, T, 8 * G, 8, 128, 16, n4=[250 - 30 * b for b in range(8)], seed=20 + i)
          for i in range(3)]
    first = []
    for p in ps:
        first.append([x.clone() for x in p.run()])
        p.out.fill_(1.0)
    near = i32(ps[0].near)
    torch.cuda.synchronize()
    for i in range(60):
        p = ps[i % 3]
        rheo.packed_attend(p.cfg, p.cfg4, p.q, p.key, p.value, p.held, near, p.data, p.held4, p.out, p.ws, lse=p.lse,
                           scale=p.scale)
    torch.cuda.synchronize()
    for p, (out, lse) in zip(ps, first):
        assert torch.equal(p.out, out) and torch.equal(p.lse, lse) and rheo.scratch_status(p.ws) == 0
    ps[2].check()


def test_packed_pages_past_32_bits():
    """A pool whose last pages lie more than 2^32 bytes from its first."""
    P, H, D = 128, 8, 128
    kw = dict(batch=1, tokens=1, page_size=P, q_heads=32, kv_heads=H, head_dim=D)
    p = _problem([3], None, 1, 32, H, D, P, n4=[4], seed=1)
    far = 2 ** 32 // (H * p.data.shape[-1]) + 2
    big = rheo.CacheConfig(pages=far + 4, max_pages=4, **kw)
    data = rheo.make_packed(big)[0]
    order = [far + 3, 0, far, far + 1]
    for j, to in enumerate(order):
        data[to] = p.data[int(p.table4[0, j])]
    want = [x.clone() for x in p.check()]
    held4 = rheo.Pages(big, block_table=i32([order]), n_pages=i32([4]))
    rheo.packed_attend(p.cfg, big, p.q, p.key, p.value, p.held, i32([3]), data, held4, p.out, p.ws, lse=p.lse, scale=p.scale)
    assert torch.equal(p.out, want[0]) and torch.equal(p.lse, want[1]) and rheo.scratch_status(p.ws) == 0
