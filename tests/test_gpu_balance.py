"""Expert counts, the balance loss and its gradient on the GPU, against plain
64-bit references (tests/training_ref.py, which derives the tolerances)."""
import numpy as np
import pytest
import torch

import paper_2602_04870_amd as mh
from tests import training_ref as ref
from tests.gpu_util import announce, needs_gpu
from tests.test_gpu_scaled import _gen, _guarded, _randn

pytestmark = [pytest.mark.gpu, needs_gpu]

BF16, F32 = torch.bfloat16, torch.float32


def _problem(T, Nh, dh, Ne, k, dtype, mask, seed):
    g = _gen(seed)
    X = _randn(g, T, Nh, dh, dtype=dtype)
    W = _randn(g, Nh, Ne, dh) * (1.5 * dh ** -0.5)
    idx = (torch.rand((T, Nh, k), generator=g, device="cuda") ** 2 * Ne).int().clamp(max=Ne - 1)
    m = None
    if mask == "some":
        m = torch.rand((T,), generator=g, device="cuda") < 0.8
    elif mask == "none":
        m = torch.zeros((T,), dtype=torch.bool, device="cuda")
    if m is not None:  # padded tokens hold anything
        X[~m] = float("nan")
    return g, X, W, idx, m


@pytest.mark.parametrize("T,Nh,Ne,k", [(1, 1, 1, 1), (5, 3, 7, 3), (129, 2, 1024, 32), (4097, 5, 64, 8),
                                       (20000, 1, 16, 5), (1000, 1024, 3, 1)])
@pytest.mark.parametrize("mask", [None, "some", "none"])
def test_expert_counts(T, Nh, Ne, k, mask):
    announce(f"expert_counts T={T} Nh={Nh} Ne={Ne} k={k} mask={mask}")
    g, X, W, idx, m = _problem(T, Nh, 64, Ne, k, BF16, mask, T + Ne)
    idx.view(-1)[::7] = -1  # outside: not counted
    idx.view(-1)[3::11] = Ne
    counts, ok = _guarded((Nh, Ne), torch.int32)
    mh.mhlmoe_expert_counts(idx, Ne, mask=m, counts=counts)
    torch.cuda.synchronize()
    ok()
    want = ref.counts64(idx.cpu().numpy(), None if m is None else m.cpu().numpy(), Ne)
    assert np.array_equal(counts.cpu().numpy(), want)


def test_expert_counts_are_the_routers():
    """Without a mask, the counts that routing gives with its indices."""
    g, X, W, _, _ = _problem(777, 3, 128, 50, 6, BF16, None, 1)
    idx, _, counts = mh.mhlmoe_route(X, W, None, 6)
    assert torch.equal(mh.mhlmoe_expert_counts(idx, 50), counts)


CASES = [  # T, Nh, dh, Ne, k
    (1, 1, 64, 1, 1), (1, 2, 128, 4, 2), (31, 1, 64, 31, 3), (33, 3, 128, 33, 4), (130, 2, 64, 65, 8),
    (257, 2, 128, 96, 4), (300, 1, 128, 1024, 32), (515, 3, 64, 200, 4), (1100, 2, 128, 130, 2),
    (2500, 1, 64, 8, 2),
    # enough tokens that the weights are laid out first: one, two, four and more blocks of experts
    (33100, 1, 64, 20, 2), (16601, 1, 128, 50, 2), (8200, 1, 128, 100, 3), (2900, 3, 64, 129, 3),
    (4150, 2, 128, 300, 4), (66000, 1, 128, 10, 2), (8200, 1, 64, 600, 4),
    # dX and dW in one pass over X: chunks of two to four tiles
    (15001, 3, 128, 77, 3), (33100, 2, 128, 128, 4), (4997, 11, 128, 65, 2)]


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("T,Nh,dh,Ne,k", CASES)
@pytest.mark.parametrize("mask", [None, "some", "none"])
def test_balance_loss_and_gradient(T, Nh, dh, Ne, k, dtype, mask):
    announce(f"balance T={T} Nh={Nh} dh={dh} Ne={Ne} {dtype} mask={mask}")
    g, X, W, idx, m = _problem(T, Nh, dh, Ne, k, dtype, mask, T * 3 + Ne)
    counts = mh.mhlmoe_expert_counts(idx, Ne, mask=m)
    loss, loss_ok = _guarded((Nh,), F32)
    stats, stats_ok = _guarded((T + 1, Nh, 2), F32)
    ws, ws_ok = _guarded((mh.mhlmoe_balance_loss_workspace(T, Nh, dh, Ne),), torch.uint8)
    mh.mhlmoe_balance_loss(X, W, counts, mask=m, loss=loss, stats=stats, workspace=ws)
    torch.cuda.synchronize()
    loss_ok(), stats_ok(), ws_ok()
    keep = None if m is None else m.cpu().numpy()
    b = ref.Balance(ref.host(X), ref.host(W), counts.cpu().numpy().astype(np.int64), keep)
    s = ref.host(stats)
    on = b.keep[:, None]
    assert np.all(np.abs(s[:T, :, 0] - on * b.lse) <= on * b.e_lse)
    assert np.all(np.abs(s[:T, :, 1] - on * b.u) <= on * (b.e_u + 2 * ref.U * np.abs(b.u)))
    assert np.all(np.abs(s[T, :, 0] - 1 / b.n) <= ref.U / b.n) and np.all(s[T, :, 1] == 0)
    assert np.all(np.abs(ref.host(loss) - b.loss) <= b.e_loss)
    for add in (False, True):
        dloss = 1 + 0.2 * _randn(g, Nh)
        size = 1.0 / T
        aX = size * _randn(g, T, Nh, dh) if add else None
        aX = aX.to(dtype) if add else None
        aW = size * _randn(g, Nh, Ne, dh) if add else None
        dX, dX_ok = _guarded((T, Nh, dh), dtype)
        dW, dW_ok = _guarded((Nh, Ne, dh), F32)
        ws, ws_ok = _guarded((mh.mhlmoe_balance_loss_backward_workspace(T, Nh, dh, Ne),), torch.uint8)
        mh.mhlmoe_balance_loss_backward(X, W, counts, stats, dloss, mask=m, dX_add=aX, dW_add=aW, dX=dX,
                                        dW_router=dW, workspace=ws)
        torch.cuda.synchronize()
        dX_ok(), dW_ok(), ws_ok()
        wX, wW, x_off, w_off = b.backward(ref.host(dloss), ref.host(aX) if add else None,
                                          ref.host(aW) if add else None, dtype == BF16)
        ex, ew = np.abs(ref.host(dX) - wX), np.abs(ref.host(dW) - wW)
        assert np.all(ex <= x_off + ref.HALF[dtype] * (np.abs(wX) + x_off)), ex.max()
        assert np.all(ew <= w_off), (ew / np.maximum(w_off, 1e-300)).max()
        if add:  # in place, and the same bits again
            gX, gW = mh.mhlmoe_balance_loss_backward(X, W, counts, stats, dloss, mask=m, dX_add=aX,
                                                     dW_add=aW, dX=aX, dW_router=aW)
            assert torch.equal(gX, dX) and torch.equal(gW, dW)


def test_balance_past_4_gib():
    """More than 2^31 elements of X: the last tokens are those of a call of their own on
    the same counts."""
    T, Nh, dh, Ne, n = 140000, 128, 128, 6, 300
    announce(f"balance T={T} Nh={Nh}")
    g = _gen(92)
    X = torch.zeros(T, Nh, dh, dtype=BF16, device="cuda")
    X[-n:] = _randn(g, n, Nh, dh, dtype=BF16)
    W = _randn(g, Nh, Ne, dh) * 0.1
    counts = torch.randint(1, 1000, (Nh, Ne), generator=g, device="cuda", dtype=torch.int32)
    loss, stats = mh.mhlmoe_balance_loss(X, W, counts)
    _, tail = mh.mhlmoe_balance_loss(X[-n:], W, counts)
    # every form is within e_lse and e_u of the exact value: twice that apart
    b = ref.Balance(ref.host(X[-n:, :2]), ref.host(W[:2]), counts[:2].cpu().numpy().astype(np.int64), None)
    s, t = ref.host(stats[T - n:T, :2]), ref.host(tail[:n, :2])
    assert np.all(np.abs(s[..., 0] - t[..., 0]) <= 2 * b.e_lse)
    assert np.all(np.abs(s[..., 1] - t[..., 1]) <= 2 * b.e_u + 4 * ref.U * np.abs(b.u))
    dloss = torch.ones(Nh, device="cuda")
    dX, dW = mh.mhlmoe_balance_loss_backward(X, W, counts, stats, dloss)
    part = torch.cat([stats[T - n:T], stats[T:]]).contiguous()
    tX, _ = mh.mhlmoe_balance_loss_backward(X[-n:].contiguous(), W, counts, part, dloss)
    wX, _, off, _ = b.backward(np.full(2, n / T), None, None, True)  # (its n is that of the tail)
    for got in (dX[-n:, :2], tX[:, :2]):
        assert np.all(np.abs(ref.host(got) - wX) <= off + ref.HALF[BF16] * (np.abs(wX) + off) + 2.0 ** -133)
    assert torch.isfinite(dW).all() and torch.isfinite(loss).all()


def test_balance_on_another_stream_than_the_current():
    """Given by argument: the call's own workspace and outputs belong to that stream."""
    g, X, W, idx, m = _problem(5000, 4, 64, 100, 4, BF16, "some", 21)
    counts = mh.mhlmoe_expert_counts(idx, 100, mask=m)
    want = mh.mhlmoe_balance_loss(X, W, counts, mask=m)
    wantb = mh.mhlmoe_balance_loss_backward(X, W, counts, want[1], torch.ones(4, device="cuda"), mask=m)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    one = torch.ones(4, device="cuda")
    side.wait_stream(torch.cuda.current_stream())
    c = mh.mhlmoe_expert_counts(idx, 100, mask=m, stream=side)
    got = mh.mhlmoe_balance_loss(X, W, c, mask=m, stream=side)
    gotb = mh.mhlmoe_balance_loss_backward(X, W, c, got[1], one, mask=m, stream=side)
    side.synchronize()
    for a, b in zip((counts, *want, *wantb), (c, *got, *gotb)):
        assert torch.equal(a, b)


def test_balance_gradient_against_differences():
    """dX and dW against central differences of the 64-bit loss."""
    T, Nh, dh, Ne = 40, 2, 64, 24
    g, X, W, idx, m = _problem(T, Nh, dh, Ne, 3, F32, "some", 5)
    X = torch.nan_to_num(X)
    counts = mh.mhlmoe_expert_counts(idx, Ne, mask=m)
    _, stats = mh.mhlmoe_balance_loss(X, W, counts, mask=m)
    dloss = 1 + 0.2 * _randn(g, Nh)
    dX, dW = (ref.host(t) for t in mh.mhlmoe_balance_loss_backward(X, W, counts, stats, dloss, mask=m))
    X, W, dl, c, keep = ref.host(X), ref.host(W), ref.host(dloss), counts.cpu().numpy(), m.cpu().numpy()
    f = lambda X, W: (dl * ref.Balance(X, W, c, keep).loss).sum()  # noqa: E731
    rng, s = np.random.default_rng(4), 1e-5
    v, w = rng.standard_normal(X.shape), rng.standard_normal(W.shape)
    for grad, d, diff in ((dX, v, f(X + s * v, W) - f(X - s * v, W)),
                          (dW, w, f(X, W + s * w) - f(X, W - s * w))):
        assert abs((grad * d).sum() - diff / (2 * s)) <= 1e-5 * np.abs(grad * d).sum()


def test_balance_even_and_collapsed_loads():
    """An even load has loss 1 and no gradient; all tokens on one expert that every
    token is sure of: loss Ne; no counts: 0."""
    T, Nh, dh, Ne = 200, 2, 64, 16
    g, X, W, _, _ = _problem(T, Nh, dh, Ne, 1, BF16, None, 6)
    even = torch.full((Nh, Ne), 25, dtype=torch.int32, device="cuda")
    loss, stats = mh.mhlmoe_balance_loss(X, W, even)
    assert torch.all(loss == 1)
    dX, dW = mh.mhlmoe_balance_loss_backward(X, W, even, stats, torch.ones(Nh, device="cuda"))
    assert torch.all(dX == 0) and torch.all(dW == 0)
    one = torch.zeros_like(even)
    one[:, 3] = T
    X = torch.ones_like(X)
    W = torch.zeros_like(W)
    W[:, 3] = 2.0  # a score of 128 against zeros
    loss, stats = mh.mhlmoe_balance_loss(X, W, one)
    assert torch.all(loss == Ne)
    dX, dW = mh.mhlmoe_balance_loss_backward(X, W, one, stats, torch.ones(Nh, device="cuda"))
    assert torch.all(dX == 0) and torch.all(dW == 0)
    loss, _ = mh.mhlmoe_balance_loss(X, W, torch.zeros_like(one))
    assert torch.all(loss == 0)


def test_balance_large_scores_and_nan_rows():
    """Scores of +-1000 (whose exponentials overflow without the maximum); a token
    with a NaN makes its own row and its head's loss NaN and leaves the others."""
    T, Nh, dh, Ne = 70, 2, 128, 40
    g, X, W, idx, _ = _problem(T, Nh, dh, Ne, 2, F32, None, 7)
    W = W * 300
    counts = mh.mhlmoe_expert_counts(idx, Ne)
    loss, stats = mh.mhlmoe_balance_loss(X, W, counts)
    b = ref.Balance(ref.host(X), ref.host(W), counts.cpu().numpy().astype(np.int64), None)
    s = ref.host(stats)[:T]
    assert np.all(np.abs(s[..., 0] - b.lse) <= b.e_lse) and np.all(np.abs(s[..., 1] - b.u) <= b.e_u)
    Xn = X.clone()
    Xn[11, 1, 5] = float("nan")
    ln, sn = mh.mhlmoe_balance_loss(Xn, W, counts)
    assert torch.isnan(ln[1]) and ln[0] == loss[0]
    same = torch.ones((T, Nh), dtype=torch.bool, device="cuda")
    same[11, 1] = False
    assert torch.equal(sn[:T][same], stats[:T][same]) and torch.isnan(sn[11, 1]).all()


def test_balance_empty_batch():
    X = torch.empty(0, 2, 64, dtype=BF16, device="cuda")
    W = torch.ones(2, 5, 64, device="cuda")
    idx = torch.empty(0, 2, 3, dtype=torch.int32, device="cuda")
    counts = mh.mhlmoe_expert_counts(idx, 5, counts=torch.ones(2, 5, dtype=torch.int32, device="cuda"))
    assert torch.all(counts == 0)
    loss, stats = mh.mhlmoe_balance_loss(X, W, counts)
    assert torch.all(loss == 0) and torch.all(stats == torch.tensor([1.0, 0.0], device="cuda"))
    for add in (None, torch.full((2, 5, 64), 3.0, device="cuda")):
        _, dW = mh.mhlmoe_balance_loss_backward(X, W, counts, stats, torch.ones(2, device="cuda"),
                                                dW_add=add, dW_router=torch.ones_like(W))
        assert torch.all(dW == (0 if add is None else 3))
