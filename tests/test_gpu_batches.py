"""Requests up to the most that a call takes: the shared memory that a launch asks for
passes the default limit on the way there."""
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


@pytest.mark.parametrize("B", [4080, 4088, 4089, 4095, 4096])
def test_reserve_of_the_most_requests(B):
    T, P, W = 3, 16, 4
    cfg = rheo.CacheConfig(batch=B, tokens=T, pages=3 * B, page_size=P, max_pages=W, q_heads=2, kv_heads=2, head_dim=64)
    pages, plan, ws = rheo.Pages(cfg), rheo.CachePlan(cfg), rheo.CacheWorkspace(cfg)
    ctx, new = [(13 * b) % 40 for b in range(B)], [b % 4 for b in range(B)]
    i32 = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")  # noqa: E731
    want = ref.reserve(ctx, new, None, pages.block_table.tolist(), [0] * B, pages.free_list.tolist(), 3 * B, P, T, W)
    rheo.cache_reserve(cfg, i32(ctx), pages, plan, ws, new_len=i32(new))
    assert rheo.scratch_status(ws) == 0
    assert pages.block_table.tolist() == want[0] and pages.n_pages.tolist() == want[1]
    assert pages.n_free.tolist() == [want[3]] and plan.slot.tolist() == want[4] and plan.position.tolist() == want[5]
