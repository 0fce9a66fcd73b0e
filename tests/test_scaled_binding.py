"""What the binding of the scaled operators refuses by itself (CPU)."""
import pytest
import torch

import paper_2602_04870_amd as m

BIG = (1 << 32) + 64  # its low 32 bits are 64


def test_extents_past_32_bits_are_refused():
    """The C ABI takes d_model and the block rows as int: a wider value is not
    passed on by its low half, which would size a workspace for, or normalise,
    the first 64 columns alone."""
    x, w = torch.empty(0, BIG, dtype=torch.bfloat16), torch.empty(0)
    with pytest.raises(ValueError, match="d_model must fit"):
        m.mhlmoe_rmsnorm_backward_workspace(4, BIG)
    with pytest.raises(ValueError, match="d_model must fit"):
        m.mhlmoe_rmsnorm(x, w, 1e-6)
    with pytest.raises(ValueError, match="d_model must fit"):
        m.mhlmoe_rmsnorm_backward(x, w, 1e-6, x)
    good = dict(d_model=256, n_heads=2, d_head=64, n_experts=8, top_k=2, d_ff=64)
    assert m.mhlmoe_latent_layer_scaled_workspace(4, **good) > 0
    for name in good:
        with pytest.raises(ValueError, match=f"{name} must fit"):
            m.mhlmoe_latent_layer_scaled_workspace(4, **dict(good, **{name: (1 << 32) + good[name]}))
    y = torch.empty(16, 32, dtype=torch.bfloat16)
    with pytest.raises(ValueError, match="block_rows must fit"):
        m.mhlmoe_quantize(y, block_rows=(1 << 32) + 1)
    q, s = torch.empty(16, 32).to(m.E4M3), torch.empty(16, 1)
    with pytest.raises(ValueError, match="b_block_rows must fit"):
        m.mhlmoe_gemm_scaled(q, s, q, s, b_block_rows=(1 << 32) + 1)


def test_layer_extents_past_32_bits_are_refused():
    x = torch.empty(0, 256, dtype=torch.bfloat16)
    w = torch.empty(2, 8, 64, 64, dtype=torch.bfloat16)
    t = torch.empty(0)
    for n_heads, top_k, name in (((1 << 32) + 2, 2, "n_heads"), (2, (1 << 32) + 2, "top_k")):
        with pytest.raises(ValueError, match=f"{name} must fit"):
            m.mhlmoe_latent_layer_scaled(x, t, 1e-6, t, t, t, None, w, w, w, t, t, n_heads, top_k)
