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


# every form of dW, by blocks of 32 experts to a workgroup: 1, 2, 4 for few tokens, 1, 2, 4, 8
DW = [(300, 2, 64, 20), (300, 2, 128, 40), (300, 1, 64, 100), (33100, 1, 64, 20), (16601, 1, 128, 50),
      (8200, 1, 128, 100), (4150, 2, 128, 300), (8200, 1, 64, 600)]


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("T,Nh,dh,Ne", DW)
def test_balance_dw_terms(T, Nh, dh, Ne, dtype):
    """Positive rows of some 60 tokens among T, scores of zero, an even load but for eight
    experts: a term of dW that were one fp16 value, 2^-11 off, would be seen."""
    announce(f"balance dW T={T} Nh={Nh} dh={dh} Ne={Ne} {dtype}")
    g, X, W, _, _ = _problem(T, Nh, dh, Ne, 1, dtype, None, T + Ne)
    X = (X.float().abs() + 0.5).to(dtype)
    W.zero_()
    m = torch.rand((T,), generator=g, device="cuda") < 60 / T
    m[T - 1] = True
    counts = torch.full((Nh, Ne), 500, device="cuda", dtype=torch.int32)
    at = torch.randperm(Ne, generator=g, device="cuda")[:8]
    more = torch.randint(100, 500, (Nh, 4), generator=g, device="cuda", dtype=torch.int32)
    counts[:, at[:4]] += more
    counts[:, at[4:]] -= more
    dloss = 1 + 0.2 * torch.rand((Nh,), generator=g, device="cuda")
    _, stats = mh.mhlmoe_balance_loss(X, W, counts, mask=m)
    _, dW = mh.mhlmoe_balance_loss_backward(X, W, counts, stats, dloss, mask=m)
    # the terms of the other tokens are zeros, exactly: n terms are added
    b = ref.Balance(ref.host(X[m]), ref.host(W), counts.cpu().numpy().astype(np.int64), None)
    _, want, _, off = b.backward(ref.host(dloss), None, None, False)
    ds = np.stack([_one_value(d) for d in (b.p * (b.f - b.u[..., None]))[0]])
    one = np.einsum("he,hd->hed", ds * (ref.host(dloss) / b.n)[:, None], b.X.sum(axis=0))
    assert np.any(np.abs(one - want) > 2 * off)
    err = np.abs(ref.host(dW) - want)
    assert np.all(err <= off), (err / np.maximum(off, 1e-300)).max()


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("T,Nh,dh,Ne", DW + FEW + [(66000, 1, 128, 10)])
def test_balance_score_products(T, Nh, dh, Ne, dtype):
    """Rows of one value: a score is one product, which has to be of fp32 accuracy (scores of
    up to +-100: a value of X or W as one fp16 value would be seen), in the loss and in both
    gradients."""
    announce(f"balance scores T={T} Nh={Nh} dh={dh} Ne={Ne} {dtype}")
    g, X, W, idx, _ = _problem(T, Nh, dh, Ne, min(Ne, 3), dtype, None, T + Ne + 1)
    col = (T + Ne) % dh
    X, keep = torch.zeros_like(X), X[:, :, col]
    X[:, :, col] = 100 * keep
    counts = mh.mhlmoe_expert_counts(idx, Ne)
    dloss = 1 + 0.2 * torch.rand((Nh,), generator=g, device="cuda")
    loss, stats = mh.mhlmoe_balance_loss(X, W, counts)
    dX, dW = mh.mhlmoe_balance_loss_backward(X, W, counts, stats, dloss)
    # the reference of that column alone, whose sums have one term
    X64, W64 = ref.host(X), ref.host(W)
    b = ref.Balance(X64[:, :, col:col + 1], W64[:, :, col:col + 1], counts.cpu().numpy().astype(np.int64),
                    None)
    s = ref.host(stats)[:T]
    assert np.all(np.abs(s[..., 0] - b.lse) <= b.e_lse)
    assert np.all(np.abs(s[..., 1] - b.u) <= b.e_u + 2 * ref.U * np.abs(b.u))
    assert np.all(np.abs(ref.host(loss) - b.loss) <= b.e_loss)
    b.W = W64
    wX, wW, x_off, w_off = b.backward(ref.host(dloss), None, None, False)
    err = np.abs(ref.host(dX) - wX)
    assert np.all(err <= x_off + ref.HALF[dtype] * (np.abs(wX) + x_off)), err.max()
    dW = ref.host(dW)
    assert np.all(np.abs(dW[:, :, col:col + 1] - wW) <= w_off)
    assert not np.delete(dW, col, axis=2).any()


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("T,Nh,dh,Ne", [(70, 2, 64, 129), (130, 1, 128, 300), (8200, 1, 128, 100),
                                        (2900, 3, 64, 257), (4150, 2, 128, 300)])
@pytest.mark.parametrize("order", [1, -1])
def test_balance_blocks_of_different_size(T, Nh, dh, Ne, dtype, order):
    """Blocks of 32 experts whose weights differ by up to 2^30, growing or shrinking with the
    experts, and rows that differ by 2^24: each block and row has a power of two of its own,
    dX's sums have the head's (or the largest one's so far)."""
    announce(f"balance sizes T={T} Nh={Nh} dh={dh} Ne={Ne} {dtype} order={order}")
    g, X, W, idx, m = _problem(T, Nh, dh, Ne, 3, dtype, "some", T + Ne)
    nb = -(-Ne // 32)
    power = torch.linspace(-20, 10, nb, device="cuda").round()
    power = power if order == 1 else power.flip(0)
    W = W * torch.exp2(power).repeat_interleave(32)[:Ne, None]
    rows = torch.exp2(torch.randint(-28, -3, (T, Nh, 1), generator=g, device="cuda").float())
    X = (X.float() * rows).to(dtype)
    counts = mh.mhlmoe_expert_counts(idx, Ne, mask=m)
    dloss = 1 + 0.2 * torch.rand((Nh,), generator=g, device="cuda")
    _, stats = mh.mhlmoe_balance_loss(X, W, counts, mask=m)
    dX, dW = mh.mhlmoe_balance_loss_backward(X, W, counts, stats, dloss, mask=m)
    W64 = ref.host(W)
    b = ref.Balance(ref.host(X), W64, counts.cpu().numpy().astype(np.int64), m.cpu().numpy())
    s, on = ref.host(stats)[:T], b.keep[:, None]
    assert np.all(np.abs(s[..., 0] - on * b.lse) <= on * b.e_lse)
    assert np.all(np.abs(s[..., 1] - on * b.u) <= on * (b.e_u + 2 * ref.U * np.abs(b.u)))
    wX, wW, x_off, w_off = b.backward(ref.host(dloss), None, None, False)
    # ds up is below 2^14 and at least 2^13 for the head's largest |f - u| <= R, w up below 2^15
    # and at least 2^14 for its largest weight; ds up is off by 2^-25, half its type's last
    # step, so a term by 2^-25 2^15 2^-13 R 2^-14 max |w|, whatever its own size
    R = (b.f.max(axis=1) - b.f.min(axis=1)) * np.abs(W64).max(axis=(1, 2))
    x_off = x_off + (Ne * 2.0 ** -37 * R * np.abs(ref.host(dloss)) / b.n)[:, None]
    err = np.abs(ref.host(dX) - wX)
    assert np.all(err <= x_off + ref.HALF[dtype] * (np.abs(wX) + x_off)), (err / x_off).max()
    assert np.all(np.abs(ref.host(dW) - wW) <= w_off + 2.0 ** -70 * ref.host(dloss)[:, None, None])


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("T,Nh,dh,Ne", [(70, 2, 64, 33), (33100, 1, 64, 20), (16601, 1, 128, 50),
                                        (66000, 1, 128, 10), (4150, 2, 128, 300)])
def test_balance_powers_of_two(T, Nh, dh, Ne, dtype):
    """X 2^a and W 2^-a have the same scores: the loss keeps its bits, dX is 2^-a times what it
    was and dW 2^a times, for rows of up to 2^63.  dW's has not the same bits: a row's power of
    two, at most 2^75 away from 1, is added in the argument of ds's exponential, which is so
    rounded by up to 2 * 75 U more on either side, a relative error of 2 * 75 U: less than
    the reference's (6 T + 10) U."""
    announce(f"balance powers T={T} Nh={Nh} dh={dh} Ne={Ne} {dtype}")
    g, X, W, idx, m = _problem(T, Nh, dh, Ne, 3, dtype, "some", T + Ne)
    X = torch.nan_to_num(X)
    counts = mh.mhlmoe_expert_counts(idx, Ne, mask=m)
    dloss = 1 + 0.2 * torch.rand((Nh,), generator=g, device="cuda")
    loss, stats = mh.mhlmoe_balance_loss(X, W, counts, mask=m)
    dX, dW = mh.mhlmoe_balance_loss_backward(X, W, counts, stats, dloss, mask=m)
    b = ref.Balance(ref.host(X), ref.host(W), counts.cpu().numpy().astype(np.int64), m.cpu().numpy())
    _, _, _, w_off = b.backward(ref.host(dloss), None, None, False)
    for a in (-40, -20, 20, 60):
        up, down = 2.0 ** a, 2.0 ** -a
        Xa, Wa = X * up, W * down
        la, sa = mh.mhlmoe_balance_loss(Xa, Wa, counts, mask=m)
        assert torch.equal(la, loss) and torch.equal(sa, stats)
        gX, gW = mh.mhlmoe_balance_loss_backward(Xa, Wa, counts, sa, dloss, mask=m)
        assert torch.equal(gX * up, dX), a
        # (the terms of small rows are lifted by 2^60 only)
        assert np.all(np.abs(ref.host(gW * down) - ref.host(dW))
                      <= 2 * w_off + down * 2.0 ** -70 * ref.host(dloss)[:, None, None]), a


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("T,Nh,dh,Ne", [(70, 2, 64, 33), (33100, 1, 64, 20), (4150, 2, 128, 300)])
def test_balance_denormal_rows(T, Nh, dh, Ne, dtype):
    """Rows of denormal numbers are zeros, or next to it."""
    announce(f"balance denormal T={T} Nh={Nh} dh={dh} Ne={Ne} {dtype}")
    g, X, W, idx, m = _problem(T, Nh, dh, Ne, 3, dtype, "some", T + Ne)
    X[::3] = (X[::3].float() * 2.0 ** -120 * 2.0 ** -10).to(dtype)
    assert (X[::3].float().abs() < 2.0 ** -126).any() and X[::3].any()
    counts = mh.mhlmoe_expert_counts(idx, Ne, mask=m)
    _check(X, W, counts, m, 1 + 0.2 * torch.rand((Nh,), generator=g, device="cuda"))
