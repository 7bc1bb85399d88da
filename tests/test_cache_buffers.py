"""The binding checks the tensors of Pages, CachePlan and Logprobs in every call, whatever
an earlier call has seen at their addresses.  Host tensors that claim to be CUDA tensors:
nothing is launched."""
import pytest
import torch

from paper_2609_21827_gb300 import rheo


class OnGpu(torch.Tensor):
    is_cuda = True


def _gpu(*shape, dtype=torch.int32):
    return torch.zeros(shape, dtype=dtype).as_subclass(OnGpu)


CFG = rheo.CacheConfig(batch=3, tokens=4, pages=12, page_size=16, max_pages=4, q_heads=4, kv_heads=2, head_dim=64)
LOG = rheo.LogprobConfig(rows=6, vocab=100, top=6)

# changes that keep the address: narrower, transposed, another type, resized
CHANGES = {
    "narrow": lambda x: setattr(x, "data", x[..., :-1]),
    "turned": lambda x: setattr(x, "data", x.t() if x.dim() == 2 else x[::2]),
    "type": lambda x: setattr(x, "data", x.view(torch.float32 if x.dtype != torch.float32 else torch.int32)),
    "resized": lambda x: x.resize_(x.numel() - 1),
}


def _pages():
    return rheo.Pages(CFG, block_table=_gpu(3, 4), n_pages=_gpu(3), free_list=_gpu(12), n_free=_gpu(1)), lambda p: p.c(CFG)


def _plan():
    return rheo.CachePlan(CFG, slot=_gpu(3, 4, dtype=torch.int64), position=_gpu(3, 4)), lambda p: p.ptrs(CFG)


def _logprobs():
    out = rheo.Logprobs(LOG, device="cpu")
    for name in ("logprob", "rank", "entropy", "top_ids", "top_logprobs"):
        x = getattr(out, name)
        setattr(out, name, _gpu(*x.shape, dtype=x.dtype))
    return out, lambda p: p.c(LOG)


FIELDS = [(_pages, n) for n in ("block_table", "n_pages", "free_list", "n_free")] + [(_plan, "slot"), (_plan, "position")] + [
    (_logprobs, n) for n in ("logprob", "rank", "entropy", "top_ids", "top_logprobs")]


@pytest.mark.parametrize("change", CHANGES)
@pytest.mark.parametrize("make,field", FIELDS)
def test_a_tensor_that_changed_at_its_address_is_refused(make, field, change):
    held, check = make()
    check(held)
    check(held)
    x = getattr(held, field)
    at, was = x.data_ptr(), (x.dtype, x.shape)
    CHANGES[change](x)
    if (x.dtype, x.shape) == was and x.is_contiguous():  # one element: its stride is not looked at
        pytest.skip("the change is none for this shape")
    assert x.data_ptr() == at or x.numel() == 0
    with pytest.raises(rheo.RheoError):
        check(held)
