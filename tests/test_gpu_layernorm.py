"""Layer norm and its gradient on the GPU, against plain 64-bit references
(tests/training_ref.py, which derives the tolerances)."""
import numpy as np
import pytest
import torch

import paper_2602_04870_amd as mh
from tests import training_ref as ref
from tests.gpu_util import announce, needs_gpu
from tests.test_gpu_scaled import WIDTHS, _gen, _guarded, _randn

pytestmark = [pytest.mark.gpu, needs_gpu]

BF16, F32 = torch.bfloat16, torch.float32
EPS = 1e-5


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("d", WIDTHS)
@pytest.mark.parametrize("residual", [False, True])
def test_layernorm(d, dtype, residual):
    for T in (1, 5, 67):
        announce(f"layernorm T={T} d={d} {dtype} residual={residual}")
        g = _gen(d * 5 + T)
        x = (_randn(g, T, d) * torch.exp(2 * _randn(g, T, 1)) + 3 * _randn(g, T, 1)).to(dtype)
        r = _randn(g, T, d, dtype=dtype) if residual else None
        w = 1 + 0.3 * _randn(g, d)
        b = 0.5 * _randn(g, d) if T != 5 else None
        quantized = d % 16 == 0
        y, y_ok = _guarded((T, d), dtype)
        kw = {}
        if residual:
            kw["sum"], s_ok = _guarded((T, d), dtype)
        if quantized:
            kw["q"], q_ok = _guarded((T, d), ref.E4M3)
            kw["scales"], sc_ok = _guarded((T, -(-d // 128)), F32)
        out = mh.mhlmoe_layernorm(x, w, EPS, bias=b, residual=r, y=y, quantized=quantized, **kw)
        torch.cuda.synchronize()
        y_ok()
        h = x
        if residual:
            s_ok()
            h = (x.float() + r.float()).to(dtype)
            assert torch.equal(out["sum"], h)
        want, off = ref.layernorm64(ref.host(h), ref.host(w), 0.0 if b is None else ref.host(b), EPS)
        err = np.abs(ref.host(out["y"]) - want)
        assert np.all(err <= off + ref.HALF[dtype] * (np.abs(want) + off)), err.max()
        if quantized:
            q_ok(), sc_ok()
            ref.check_blocks(ref.host(out["q"]), ref.host(out["scales"]), want, off, f"d={d}")


@pytest.mark.parametrize("d", [24, 1024, 5000, 20000, 40000])
def test_layernorm_in_place(d):
    """sum may be x or residual, y may be x."""
    g = _gen(d)
    x, r, w = _randn(g, 9, d, dtype=BF16), _randn(g, 9, d, dtype=BF16), 1 + 0.1 * _randn(g, d)
    b = _randn(g, d)
    want = mh.mhlmoe_layernorm(x, w, EPS, bias=b, residual=r)
    for alias in ("x", "residual"):
        a = {"x": x.clone(), "residual": r.clone()}
        got = mh.mhlmoe_layernorm(a["x"], w, EPS, bias=b, residual=a["residual"], sum=a[alias])
        assert torch.equal(got["sum"], want["sum"]) and torch.equal(got["y"], want["y"])
    a = x.clone()
    assert torch.equal(mh.mhlmoe_layernorm(a, w, EPS, y=a)["y"], mh.mhlmoe_layernorm(x, w, EPS)["y"])


@pytest.mark.parametrize("d", [40, 100, 512, 2048, 4096, 20000, 40000])
def test_layernorm_far_from_zero_and_special_rows(d):
    """Rows whose mean is 2^12 times their deviation keep it (h - mu is taken before
    anything is squared); a constant row has no variance; a row with a NaN or an
    infinity is NaN in itself and nowhere else."""
    g = _gen(d + 1)
    x = _randn(g, 7, d)
    x[1] += 4096.0
    x[2] = 1234.5
    x[3, d // 2] = float("nan")
    x[4, d - 1] = float("inf")
    x[5] = 0
    w, b = 1 + 0.3 * _randn(g, d), _randn(g, d)
    y = ref.host(mh.mhlmoe_layernorm(x, w, EPS, bias=b)["y"])
    rows = [0, 1, 2, 5, 6]
    want, off = ref.layernorm64(ref.host(x)[rows], ref.host(w), ref.host(b), EPS)
    # row 2: c = h - mu is what the mean was rounded by, the same in all columns and taken off
    # again, but for a step of U c (c <= adds U 1234.5), times rs = 1 / sqrt(eps)
    off[2] += (ref.adds(d) * ref.U) ** 2 * 1234.5 * (1e-5) ** -0.5 * np.abs(ref.host(w))
    err = np.abs(y[rows] - want)
    assert np.all(err <= off + ref.U * (np.abs(want) + off)), err.max(axis=1)
    assert np.isnan(y[3]).all() and np.isnan(y[4]).all()


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("d", WIDTHS)
@pytest.mark.parametrize("residual", [False, True])
def test_layernorm_backward(d, dtype, residual):
    for T in (1, 6, 515 if d < 2000 else 70):
        announce(f"layernorm_backward T={T} d={d} {dtype} residual={residual}")
        g = _gen(d * 13 + T)
        h = (_randn(g, T, d) * torch.exp(_randn(g, T, 1)) + _randn(g, T, 1)).to(dtype)
        dy = _randn(g, T, d, dtype=dtype)
        ds = _randn(g, T, d, dtype=dtype) if residual else None
        w = 1 + 0.3 * _randn(g, d)
        dx, dx_ok = _guarded((T, d), dtype)
        dw, dw_ok = _guarded((d,), F32)
        db, db_ok = _guarded((d,), F32)
        ws, ws_ok = _guarded((max(mh.mhlmoe_layernorm_backward_workspace(T, d), 1),), torch.uint8)
        mh.mhlmoe_layernorm_backward(h, w, EPS, dy, dsum=ds, dx=dx, dweight=dw, dbias=db, workspace=ws)
        torch.cuda.synchronize()
        dx_ok(), dw_ok(), db_ok(), ws_ok()
        want, wdw, wdb, x_off, dw_off, db_off = ref.layernorm_backward64(
            ref.host(h), ref.host(w), EPS, ref.host(dy), None if ds is None else ref.host(ds))
        off = np.abs(ref.host(dx) - want)
        assert np.all(off <= x_off + (ref.HALF[dtype] + ref.U) * (np.abs(want) + x_off)), off.max()
        assert np.all(np.abs(ref.host(dw) - wdw) <= dw_off)
        assert np.all(np.abs(ref.host(db) - wdb) <= db_off)


@pytest.mark.parametrize("d", [64, 1001, 2048, 20000, 32768])
def test_layernorm_backward_in_place_and_repeatable(d):
    """dx may be dy or dsum; the same call gives the same bits; no dbias wanted."""
    g = _gen(d + 2)
    h, dy, ds = (_randn(g, 300, d, dtype=BF16) for _ in range(3))
    w = 1 + 0.1 * _randn(g, d)
    want = mh.mhlmoe_layernorm_backward(h, w, EPS, dy, dsum=ds)
    again = mh.mhlmoe_layernorm_backward(h, w, EPS, dy, dsum=ds)
    assert all(torch.equal(a, b) for a, b in zip(want, again))
    for name in ("dy", "dsum"):
        a = {"dy": dy.clone(), "dsum": ds.clone()}
        got = mh.mhlmoe_layernorm_backward(h, w, EPS, a["dy"], dsum=a["dsum"], dx=a[name])
        assert all(torch.equal(x, y) for x, y in zip(want, got))
    lib = mh.load_library()
    dx, dw = torch.empty_like(h), torch.empty(d, device="cuda")
    ws = torch.empty(mh.mhlmoe_layernorm_backward_workspace(300, d), dtype=torch.uint8, device="cuda")
    assert lib.mhlmoe_layernorm_backward(h.data_ptr(), w.data_ptr(), dy.data_ptr(), ds.data_ptr(), 300,
                                         d, EPS, mh.MHLMOE_BF16, dx.data_ptr(), dw.data_ptr(), None,
                                         ws.data_ptr(), ws.numel(), 0) == 0
    torch.cuda.synchronize()
    assert torch.equal(dx, want[0]) and torch.equal(dw, want[1])


def test_layernorm_gradient_against_differences():
    """dx, dw and db against central differences of the 64-bit forward along random
    directions."""
    g = _gen(77)
    T, d, eps = 12, 96, EPS
    x, dy, w, b = _randn(g, T, d), _randn(g, T, d), 1 + 0.2 * _randn(g, d), _randn(g, d)
    dx, dw, db = (ref.host(t) for t in mh.mhlmoe_layernorm_backward(x, w, eps, dy))
    x, dy, w, b = (ref.host(t) for t in (x, dy, w, b))
    rng = np.random.default_rng(3)
    f = lambda x, w, b: (dy * ref.layernorm64(x, w, b, eps)[0]).sum()  # noqa: E731
    s = 1e-5
    for grad, at in ((dx, 0), (dw, 1), (db, 2)):
        v = rng.standard_normal(grad.shape)
        args = [x, w, b]
        up, down = list(args), list(args)
        up[at], down[at] = args[at] + s * v, args[at] - s * v
        diff = (f(*up) - f(*down)) / (2 * s)
        # s^2 / 6 of the third derivative (of the size of the value) and fp32's error
        assert abs((grad * v).sum() - diff) <= 1e-5 * np.abs(grad * v).sum()


@pytest.mark.parametrize("d", [33001, 65535, 65536])
@pytest.mark.parametrize("dtype", [BF16, F32])
def test_layernorm_widest(d, dtype):
    """Rows that no workgroup holds, forward and gradient."""
    g = _gen(d)
    T = 19
    x, dy = (_randn(g, T, d) + _randn(g, T, 1)).to(dtype), _randn(g, T, d, dtype=dtype)
    r, w, b = _randn(g, T, d, dtype=dtype), 1 + 0.3 * _randn(g, d), _randn(g, d)
    out = mh.mhlmoe_layernorm(x, w, EPS, bias=b, residual=r)
    h = (x.float() + r.float()).to(dtype)
    assert torch.equal(out["sum"], h)
    want, off = ref.layernorm64(ref.host(h), ref.host(w), ref.host(b), EPS)
    assert np.all(np.abs(ref.host(out["y"]) - want) <= off + ref.HALF[dtype] * (np.abs(want) + off))
    dx, dw, db = mh.mhlmoe_layernorm_backward(h, w, EPS, dy, dsum=r)
    want, wdw, wdb, x_off, dw_off, db_off = ref.layernorm_backward64(
        ref.host(h), ref.host(w), EPS, ref.host(dy), ref.host(r))
    off = np.abs(ref.host(dx) - want)
    assert np.all(off <= x_off + (ref.HALF[dtype] + ref.U) * (np.abs(want) + x_off)), off.max()
    assert np.all(np.abs(ref.host(dw) - wdw) <= dw_off) and np.all(np.abs(ref.host(db) - wdb) <= db_off)


def test_layernorm_past_4_gib():
    """More than 2^31 elements: the last rows are those of a call of their own."""
    d, T = 2048, (1 << 20) + 4099
    announce(f"layernorm T={T} d={d}")
    g = _gen(91)
    tail = _randn(g, 5000, d, dtype=BF16)
    x = torch.zeros(T, d, dtype=BF16, device="cuda")
    x[-5000:] = tail
    w, b = 1 + 0.1 * _randn(g, d), _randn(g, d)
    y = mh.mhlmoe_layernorm(x, w, EPS, bias=b)["y"]
    assert torch.equal(y[-5000:], mh.mhlmoe_layernorm(tail, w, EPS, bias=b)["y"])
    assert torch.equal(y[0].float(), b.to(BF16).float())
    dx, dw, db = mh.mhlmoe_layernorm_backward(x, w, EPS, x)
    tx, tw, tb = mh.mhlmoe_layernorm_backward(tail, w, EPS, tail)
    assert torch.equal(dx[-5000:], tx) and not dx[:1000].any()
    # the zero rows add nothing: the same 5000 terms per column in another order
    n, _ = ref.norm_parts(ref.host(tail), EPS)
    mag = np.abs(ref.host(tail) * n).sum(axis=0)
    assert np.all(np.abs(ref.host(dw) - ref.host(tw)) <= 2 * 5002 * ref.U * mag)
    assert np.all(np.abs(ref.host(db) - ref.host(tb)) <= 2 * 5002 * ref.U * np.abs(ref.host(tail)).sum(axis=0))


def test_layernorm_empty():
    x = torch.empty(0, 64, dtype=BF16, device="cuda")
    w = torch.ones(64, device="cuda")
    assert mh.mhlmoe_layernorm(x, w, EPS)["y"].shape == (0, 64)
    dw, db = torch.ones(64, device="cuda"), torch.ones(64, device="cuda")
    mh.mhlmoe_layernorm_backward(x, w, EPS, x, dweight=dw, dbias=db)
    assert torch.all(dw == 0) and torch.all(db == 0)
