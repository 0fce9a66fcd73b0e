"""The balance loss and its gradient where rows and weights are zero, tiny, huge or of
widely different size, in every form of the kernels, against the plain 64-bit reference
(tests/training_ref.py)."""
import numpy as np
import pytest
import torch

import paper_2602_04870_amd as mh
from tests import training_ref as ref
from tests.gpu_util import announce, needs_gpu
from tests.test_gpu_balance import _problem

pytestmark = [pytest.mark.gpu, needs_gpu]

BF16, F32 = torch.bfloat16, torch.float32

# T, Nh, dh, Ne: no number of experts is a multiple of 32
FEW = [(40, 1, 64, 1), (70, 2, 64, 6), (70, 2, 128, 33), (130, 3, 64, 100)]
# dX and dW together, dX by itself, one pass over a bf16 X
MANY = [(33100, 1, 64, 20), (16601, 1, 128, 50), (66000, 1, 128, 10), (4150, 2, 128, 300),
        (15001, 3, 128, 77)]


def _check(X, W, counts, m, dloss):
    """Loss, stats and gradient within the reference's bounds.  dW's terms are also off by
    the last step of its scaled fp16 values, 2^-25 times 2^15 over 2^60 each."""
    T, Nh, dh = X.shape
    loss, stats = mh.mhlmoe_balance_loss(X, W, counts, mask=m)
    dX, dW = mh.mhlmoe_balance_loss_backward(X, W, counts, stats, dloss, mask=m)
    b = ref.Balance(ref.host(X), ref.host(W), counts.cpu().numpy().astype(np.int64),
                    None if m is None else m.cpu().numpy())
    s, on = ref.host(stats)[:T], b.keep[:, None]
    assert np.all(np.abs(s[..., 0] - on * b.lse) <= on * b.e_lse)
    assert np.all(np.abs(s[..., 1] - on * b.u) <= on * (b.e_u + 2 * ref.U * np.abs(b.u)))
    assert np.all(np.abs(ref.host(loss) - b.loss) <= b.e_loss)
    wX, wW, x_off, w_off = b.backward(ref.host(dloss), None, None, X.dtype == BF16)
    half = ref.HALF[X.dtype]
    assert np.all(np.abs(ref.host(dX) - wX) <= x_off + half * (np.abs(wX) + x_off))
    assert np.all(np.abs(ref.host(dW) - wW) <= w_off + 2.0 ** -70 * ref.host(dloss)[:, None, None])


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("T,Nh,dh,Ne", FEW + MANY)
@pytest.mark.parametrize("rows,weights", [(0.0, 1.0), (0.0, 2.0 ** -13), (0.0, 0.0), (2.0 ** -12, 0.0),
                                          (2.0 ** -100, 2.0 ** -40)])
def test_balance_zero_and_tiny(T, Nh, dh, Ne, dtype, rows, weights):
    """Every third token's row times `rows`, some of them padded and the others not, before a
    router times `weights`: scores at or near zero are an even softmax, also where the
    experts end inside a block of 32."""
    announce(f"balance T={T} Nh={Nh} dh={dh} Ne={Ne} {dtype} rows={rows} weights={weights}")
    g, X, W, idx, m = _problem(T, Nh, dh, Ne, min(Ne, 3), dtype, "some", T + Ne)
    X[::3] *= rows  # (padded rows stay NaN)
    W = W * weights
    counts = mh.mhlmoe_expert_counts(idx, Ne, mask=m)
    _check(X, W, counts, m, 1 + 0.2 * torch.rand((Nh,), generator=g, device="cuda"))
