"""Windows over packed pages where they meet other things: tiles of one half one behind the other."""
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
