"""What the attention over packed pages leaves behind stays within the scratch that
rheo_packed_sizes asks for, at every number of rows of its small tiles and the first
ones of the larger."""
import pytest
import torch

from paper_2609_21827_gb300 import build, rheo
import long_reference as lr

pytestmark = pytest.mark.gpu
GUARD = 1 << 20


@pytest.fixture(scope="module", autouse=True)
def _lib():
    if not torch.cuda.is_available():
        pytest.skip("needs a CUDA GPU")
    build.build()


@pytest.mark.parametrize("T,G", [(1, 1), (8, 1), (9, 1), (4, 4), (17, 1), (3, 8), (32, 1), (33, 1)])
@pytest.mark.parametrize("D", [64, 128])
def test_nothing_is_written_behind_the_scratch(T, G, D):
    """Three requests of a head, whose tiles are cut over all CTAs, and 40 of them one behind the other on the line."""
    for n4 in ([120, 77, 90], [9] * 40):
        p = lr.Problem(rheo, [20] * len(n4), None, T, G, 1, D, 64, n4=n4, seed=T)
        n = p.cfg.packed_scratch_bytes()
        assert p.ws.nbytes == n
        whole = torch.full((n + 2 * GUARD,), 0xA5, dtype=torch.uint8, device="cuda")
        p.ws.buf = whole[GUARD:GUARD + n]
        p.ws._ptr = p.ws.buf.data_ptr()
        p.ws.init(None)
        p.check()
        assert (whole[:GUARD] == 0xA5).all() and (whole[GUARD + n:] == 0xA5).all()
