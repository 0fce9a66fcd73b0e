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
# the weights laid out first; dX and dW in one launch, or each by itself (66000 x 10, 300)
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


def _one_value(v):
    """v [n, ...] as single fp16 values of a power of two that all of them share."""
    k = 13 - np.floor(np.log2(np.abs(v).max()))
    return np.float16(v * 2.0 ** k).astype(np.float64) * 2.0 ** -k


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("T,Nh,dh,Ne", [(70, 2, 64, 6), (70, 2, 128, 33), (130, 3, 64, 100), (33100, 1, 64, 20),
                                        (16601, 1, 128, 50), (66000, 1, 128, 10), (15001, 3, 128, 77)])
def test_balance_dx_terms(T, Nh, dh, Ne, dtype):
    """dX is rounded once: where dX_add takes nearly all of it away, what is left shows its
    terms.  Rows of zeros have exact scores, so little else is off; terms of one fp16 value
    each, 2^-11 off, would be seen."""
    announce(f"balance dX T={T} Nh={Nh} dh={dh} Ne={Ne} {dtype}")
    g, X, W, _, _ = _problem(T, Nh, dh, Ne, 1, dtype, None, T + Ne)
    X.zero_()
    # an even load but for up to eight experts, whose terms are then most of dX
    counts = torch.full((Nh, Ne), 500, device="cuda", dtype=torch.int32)
    n = min(4, Ne // 2)
    at = torch.randperm(Ne, generator=g, device="cuda")[:2 * n]
    more = torch.randint(100, 500, (Nh, n), generator=g, device="cuda", dtype=torch.int32)
    counts[:, at[:n]] += more
    counts[:, at[n:]] -= more
    dloss = 1 + 0.2 * torch.rand((Nh,), generator=g, device="cuda")
    _, stats = mh.mhlmoe_balance_loss(X, W, counts)
    # a token is like all others: three of them, of which the reference has n = 3
    c64, dl = counts.cpu().numpy().astype(np.int64), ref.host(dloss) * 3 / T
    b = ref.Balance(ref.host(X[:3]), ref.host(W), c64, None)
    v, _, _, _ = b.backward(dl, None, None, False)
    add = torch.from_numpy(-v).to(dtype)
    w, _, off, _ = b.backward(dl, ref.host(add), None, False)
    ds = (b.p * (b.f - b.u[..., None]))[0] * (dl / 3)[:, None]
    one = np.einsum("he,hed->hd", np.stack([_one_value(d) for d in ds]),
                    np.stack([_one_value(h) for h in ref.host(W)]))
    half = ref.HALF[dtype]
    assert np.any(np.abs(one - v[0]) > 2 * off[0] + half * (np.abs(w[0]) + off[0]))
    dX, _ = mh.mhlmoe_balance_loss_backward(X, W, counts, stats, dloss,
                                            dX_add=add[:1].cuda().expand(T, Nh, dh).contiguous())
    err = np.abs(ref.host(dX) - w[0])
    assert np.all(err <= off[0] + half * (np.abs(w[0]) + off[0])), (err / off[0]).max()
