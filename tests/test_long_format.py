"""The 4-bit format as the tests read it: every word's place once, pages there and back."""
import numpy as np
import pytest

import long_reference as lr


@pytest.mark.parametrize("P,D", [(16, 64), (16, 128), (32, 64), (64, 128), (128, 128)])
def test_pages_there_and_back(P, D):
    N = min(P, 32)
    key, value = lr.word_places(N, D)
    assert len(set(zip(*key.reshape(2, -1).tolist()))) == len(set(zip(*value.reshape(2, -1).tolist()))) == N * D
    g = np.random.RandomState(P + D)
    x = [g.randn(3, 2, P, D) * 10.0 ** g.uniform(-3, 3, (3, 2, 1, D)) for _ in range(2)]
    data = lr.pack_pages(*x)
    assert data.shape == (3, 2, P // N * (N * D + D + N * D // 32))
    k, v = lr.unpack_pages(data, P, D)
    # within half a step, of which seven reach the largest magnitude rounded up to four bits
    tk = np.abs(x[0]).reshape(3, 2, P // N, N, D).max(3, keepdims=True)
    tv = np.abs(x[1]).reshape(3, 2, P, D // 32, 32).max(4, keepdims=True)
    assert (np.abs(k - x[0]).reshape(3, 2, P // N, N, D) <= tk / 14 * 1.126).all()
    assert (np.abs(v - x[1]).reshape(3, 2, P, D // 32, 32) <= tv / 14 * 1.126).all()
    words = np.ascontiguousarray(data[..., :N * D]).view(np.uint32)
    assert (lr._words(lr._codes(words)) == words).all()


def test_scales_are_the_smallest_that_reach():
    top = np.concatenate([[0.0, 1e-9, lr.MOST], 7 * lr.STEPS, np.nextafter(7 * lr.STEPS[:-1], np.inf), 2.0 ** np.arange(-20, 15)])
    code = lr.scale_bytes(top).astype(int)
    assert (7 * lr.step(code) >= top).all()
    assert (code == 0)[:2].all() and all(c == 0 or 7 * lr.step(c - 1) < t for c, t in zip(code, top))


def test_halves_go_away_from_zero():
    assert lr.numbers(np.array([0.5, -0.5, 1.5, 2.5, -6.5, 7.0, 0.49]), 1.0).tolist() == [1, -1, 2, 3, -7, 7, 0]
