"""Trees whose prune asks for shared memory around the default limit, against the oracle."""
import pytest
import torch

from paper_2609_21827_gb300 import build, rheo, synth
import parity_harness as ph

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _lib():
    if not torch.cuda.is_available():
        pytest.skip("needs a CUDA GPU")
    build.build()
    import oracle
    oracle.build()


# 2,170, 2,242, 2,257, 2,314 nodes: 46.5, 48.1, 48.4 and 49.6 thousand bytes, of 49,152 with the kernel's static ones
@pytest.mark.parametrize("K,D", [(8, 31), (8, 32), (11, 18), (8, 33)])
def test_prune_around_the_default_limit(K, D):
    w = synth.Workload(name=f"K{K}_D{D}", batch=2, vocab=300, depth=D, K=K, budget=48, dtype="f32", zipf_s=1.1,
                       sigma_draft=0.6, sigma_target=0.6, temperatures=(0.8,), m=1, support=64, seed=1000 + D)
    cfg = rheo.Config(batch=w.batch, vocab=w.vocab, K=K, depth=D, budget=w.budget, m=w.m, support=w.support, dtype=w.dtype)
    draft = synth.make_draft_inputs(w, device="cuda")
    g = ph.run_gpu(w, draft, cfg)
    assert g.status == 0, f"device status {g.status}"
    rep = ph.compare(cfg, g, ph.run_oracle(w, draft, cfg, [0, 1]), [0, 1])
    assert rep.ok(), str(rep)
    assert len(rep.explained) <= 1, str(rep)
