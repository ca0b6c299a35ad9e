"""Refusals of the calls around the paged cache that need a GPU tensor to get that far."""
import pytest
import torch

from paper_2510_25739_b200 import binding

pytestmark = pytest.mark.gpu


def test_a_bias_under_an_rms_norm_is_refused():
    q = torch.zeros((3, 4, 64), dtype=torch.bfloat16, device="cuda")
    w = torch.ones(64, dtype=torch.bfloat16, device="cuda")
    out = torch.full_like(q, 7.0)
    with pytest.raises(ValueError, match="q_bias: goes with norm 'layer'"):
        binding.qk_norm_rope(q, None, None, None, norm="rms", q_weight=w, q_bias=w, q_out=out)
    pages = torch.full((2, 4, 16, 64), 7.0, dtype=torch.bfloat16, device="cuda")
    bt, rb, kv = (torch.zeros(s, dtype=torch.int32, device="cuda") for s in ((1, 2), (2,), (1,)))
    with pytest.raises(ValueError, match="k_bias: goes with norm 'layer'"):
        binding.rope_append(None, q, q, None, None, pages, pages, bt, rb, kv, norm="rms", k_weight=w, k_bias=w)
    torch.cuda.synchronize()
    assert (out == 7.0).all() and (pages == 7.0).all()
    binding.qk_norm_rope(q, None, None, None, norm="layer", q_weight=w, q_bias=w, q_out=out)
    assert (out == 1.0).all()


def test_running_out_of_memory_says_so():
    """A result or workspace that does not fit raises what torch raises for it, and nothing is launched."""
    q = torch.zeros((1, 1, 128), dtype=torch.bfloat16, device="cuda").expand(1 << 24, 128, 128)  # 512 GB as a result
    pages = torch.zeros((2, 128, 16, 128), dtype=torch.bfloat16, device="cuda")
    bt, rb, kv = (torch.zeros(s, dtype=torch.int32, device="cuda") for s in ((1, 2), (2,), (1,)))
    with pytest.raises(torch.OutOfMemoryError):
        binding.paged_attn(q, pages, pages, bt, rb, kv, 1, 16, 0.1)
    with pytest.raises(torch.OutOfMemoryError):
        binding.qk_norm_rope(q, None, None, None)
    x = torch.ones((1, 1, 128), dtype=torch.bfloat16, device="cuda")
    y, _ = binding.qk_norm_rope(x, None, None, None)
    assert torch.equal(x, y)
