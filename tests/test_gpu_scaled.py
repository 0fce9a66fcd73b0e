"""The operators around the heads on the GPU, against plain 64-bit references
(tests/scaled_ref.py, which derives the tolerances)."""
import numpy as np
import pytest
import torch

import paper_2602_04870_amd as mh
from tests import scaled_ref as ref
from tests.gpu_util import announce, needs_gpu

pytestmark = [pytest.mark.gpu, needs_gpu]

BF16, F32 = torch.bfloat16, torch.float32
EPS = 1e-6


def _gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def _randn(gen, *shape, dtype=F32):
    return torch.randn(shape, generator=gen, device="cuda").to(dtype)


def _guarded(shape, dtype, fill=93):
    """A tensor in the middle of a buffer of bytes, and a check that the bytes
    around it are still what they were."""
    n = int(np.prod(shape)) * torch.empty((), dtype=dtype).element_size()
    buf = torch.full((n + 512 + 256,), fill, dtype=torch.uint8, device="cuda")
    t = buf[256:256 + n].view(dtype).view(shape)

    def untouched():
        end = 256 + n
        assert torch.all(buf[:256] == fill) and torch.all(buf[end:] == fill)
    return t, untouched


# widths of every form of the kernels: full, one short of it, one past it, odd,
# and wider than the registers' forms
WIDTHS = [1, 7, 8, 16, 28, 63, 65, 100, 112, 128, 136, 250, 256, 264, 512, 513, 520, 1000, 1001,
          1024, 1032, 2048, 2056, 4095, 4096, 4097, 4112, 8192, 8208, 12304, 16384, 16400, 20001,
          32768, 32784]


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("d", WIDTHS)
@pytest.mark.parametrize("residual", [False, True])
def test_rmsnorm(d, dtype, residual):
    for T in (1, 5, 67):
        announce(f"rmsnorm T={T} d={d} {dtype} residual={residual}")
        g = _gen(d * 7 + T)
        x = (_randn(g, T, d) * torch.exp(2 * _randn(g, T, 1))).to(dtype)
        r = _randn(g, T, d, dtype=dtype) if residual else None
        w = 1 + 0.3 * _randn(g, d)
        quantized = d % 16 == 0
        y, y_ok = _guarded((T, d), dtype)
        kw = {}
        if residual:
            kw["sum"], s_ok = _guarded((T, d), dtype)
        if quantized:
            kw["q"], q_ok = _guarded((T, d), ref.E4M3)
            kw["scales"], sc_ok = _guarded((T, -(-d // 128)), F32)
        out = mh.mhlmoe_rmsnorm(x, w, EPS, residual=r, y=y, quantized=quantized, **kw)
        torch.cuda.synchronize()
        y_ok()
        h = x
        if residual:
            s_ok()
            h = (x.float() + r.float()).to(dtype)
            assert torch.equal(out["sum"], h)
        want = ref.norm64(ref.host(h), ref.host(w), EPS)
        eps = ref.norm_eps(d)
        assert np.all(np.abs(ref.host(out["y"]) - want) <= (eps + ref.HALF[dtype]) * np.abs(want))
        if quantized:
            q_ok(), sc_ok()
            ref.check_blocks(ref.host(out["q"]), ref.host(out["scales"]), want, 1, eps, f"d={d}")


@pytest.mark.parametrize("d", [24, 1024, 5000, 20000, 40000])
def test_rmsnorm_in_place(d):
    """sum may be x or residual, y may be x."""
    g = _gen(d)
    x, r, w = _randn(g, 9, d, dtype=BF16), _randn(g, 9, d, dtype=BF16), 1 + 0.1 * _randn(g, d)
    want = mh.mhlmoe_rmsnorm(x, w, EPS, residual=r)
    for alias in ("x", "residual"):
        a = {"x": x.clone(), "residual": r.clone()}
        got = mh.mhlmoe_rmsnorm(a["x"], w, EPS, residual=a["residual"], sum=a[alias])
        assert torch.equal(got["sum"], want["sum"]) and torch.equal(got["y"], want["y"])
        assert got["sum"].data_ptr() == a[alias].data_ptr()
    a = x.clone()
    assert torch.equal(mh.mhlmoe_rmsnorm(a, w, EPS, y=a)["y"], mh.mhlmoe_rmsnorm(x, w, EPS)["y"])


def test_rmsnorm_special_rows():
    """A zero row stays zero (its blocks' scales at their smallest), a row with
    a NaN or an infinity is NaN or zero in itself and nowhere else."""
    g = _gen(3)
    x = _randn(g, 5, 256)
    w = torch.ones(256, device="cuda")
    x[1] = 0
    x[2, 7] = float("nan")
    x[3, 200] = float("inf")
    out = mh.mhlmoe_rmsnorm(x, w, EPS, quantized=True, y=torch.empty_like(x))
    q, s, y = ref.host(out["q"]), ref.host(out["scales"]), ref.host(out["y"])
    assert np.all(y[1] == 0) and np.all(q[1] == 0) and np.all(s[1] == ref.SCALE_MIN)
    assert np.isnan(y[2]).all() and np.isnan(q[2] * np.repeat(s[2], 128)).all()
    assert np.isnan(y[3, 200])
    clean = mh.mhlmoe_rmsnorm(x[[0, 4]].contiguous(), w, EPS, quantized=True)
    assert torch.equal(out["q"].view(torch.uint8)[[0, 4]], clean["q"].view(torch.uint8))


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("d", WIDTHS)
@pytest.mark.parametrize("residual", [False, True])
def test_rmsnorm_backward(d, dtype, residual):
    for T in (1, 6, 515 if d < 2000 else 70):
        announce(f"rmsnorm_backward T={T} d={d} {dtype} residual={residual}")
        g = _gen(d * 11 + T)
        h = (_randn(g, T, d) * torch.exp(_randn(g, T, 1))).to(dtype)
        dy = _randn(g, T, d, dtype=dtype)
        ds = _randn(g, T, d, dtype=dtype) if residual else None
        w = 1 + 0.3 * _randn(g, d)
        dx, dx_ok = _guarded((T, d), dtype)
        dw, dw_ok = _guarded((d,), F32)
        ws, ws_ok = _guarded((max(mh.mhlmoe_rmsnorm_backward_workspace(T, d), 1),), torch.uint8)
        mh.mhlmoe_rmsnorm_backward(h, w, EPS, dy, dsum=ds, dx=dx, dweight=dw, workspace=ws)
        torch.cuda.synchronize()
        dx_ok(), dw_ok(), ws_ok()
        want, wdw, t_abs, dw_abs = ref.norm_backward64(
            ref.host(h), ref.host(w), EPS, ref.host(dy), None if ds is None else ref.host(ds))
        # g h's sum has a product more per term than h^2's, and all of its error reaches dx
        eps = 3 * ref.norm_eps(d) + 4 * ref.U
        off = np.abs(ref.host(dx) - want)
        assert np.all(off <= eps * t_abs + (ref.HALF[dtype] + ref.U) * np.abs(want)), off.max()
        # T terms in some order, each with the norm's error and two products
        assert np.all(np.abs(ref.host(dw) - wdw) <= (T * ref.U + ref.norm_eps(d) + 2 * ref.U) * dw_abs)


def test_rmsnorm_backward_in_place_and_repeatable():
    g = _gen(8)
    h, dy, ds = (_randn(g, 300, 1024, dtype=BF16) for _ in range(3))
    w = 1 + 0.1 * _randn(g, 1024)
    dx, dw = mh.mhlmoe_rmsnorm_backward(h, w, EPS, dy, dsum=ds)
    for alias in (0, 1):
        a = [dy.clone(), ds.clone()]
        dx2, dw2 = mh.mhlmoe_rmsnorm_backward(h, w, EPS, a[0], dsum=a[1], dx=a[alias])
        assert torch.equal(dx, dx2) and torch.equal(dw, dw2)


@pytest.mark.parametrize("d", [40, 96, 1001])
def test_rmsnorm_gradient_against_differences(d):
    """<dx, u> and <dw, u> against central differences of sum(dy y) + sum(dsum
    h) in 64 bits along random directions.  A difference over 2 t leaves t^2 of
    the third derivative: with t = 1e-4 and rows of norm sqrt(d) about 1e-8
    relative, below the fp32 results' own error."""
    T, t = 12, 1e-4
    g = _gen(d)
    x, r, dy, ds = (_randn(g, T, d) for _ in range(4))
    w = 1 + 0.3 * _randn(g, d)
    h = mh.mhlmoe_rmsnorm(x, w, EPS, residual=r)["sum"]
    dx, dw = mh.mhlmoe_rmsnorm_backward(h, w, EPS, dy, dsum=ds)
    h64, w64, dy64, ds64 = (ref.host(v) for v in (h, w, dy, ds))
    rng = np.random.default_rng(d)

    def f(hh, ww):
        return (dy64 * ref.norm64(hh, ww, EPS)).sum() + (ds64 * hh).sum()

    _, _, t_abs, dw_abs = ref.norm_backward64(h64, w64, EPS, dy64, ds64)
    for _ in range(4):
        u, v = rng.standard_normal((T, d)), rng.standard_normal(d)
        num = (f(h64 + t * u, w64) - f(h64 - t * u, w64)) / (2 * t)
        bound = (3 * ref.norm_eps(d) + 6 * ref.U) * (np.abs(u) * (t_abs + np.abs(ds64))).sum()
        assert abs((ref.host(dx) * u).sum() - num) <= bound + 1e-6 * (np.abs(u) * t_abs).sum()
        num = (f(h64, w64 + t * v) - f(h64, w64 - t * v)) / (2 * t)
        bound = (T * ref.U + ref.norm_eps(d) + 2 * ref.U) * (np.abs(v) * dw_abs).sum()
        assert abs((ref.host(dw) * v).sum() - num) <= bound + 1e-6 * (np.abs(v) * dw_abs).sum()


QUANT_SHAPES = [(1, 16), (3, 48), (16, 128), (17, 144), (127, 128), (128, 112), (129, 272),
                (300, 400), (1, 4096), (1000, 16)]


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("rows,cols", QUANT_SHAPES)
@pytest.mark.parametrize("block,transpose", [(1, False), (128, False), (1, True), (128, True)])
def test_quantize(rows, cols, dtype, block, transpose):
    announce(f"quantize {rows}x{cols} {dtype} block={block} transpose={transpose}")
    g = _gen(rows * 31 + cols)
    x = (_randn(g, rows, cols) * torch.exp(3 * _randn(g, rows, 1))).to(dtype)
    a, k = (cols, -(-rows // 16) * 16) if transpose else (rows, cols)
    q, q_ok = _guarded((a, k), ref.E4M3)
    scales, s_ok = _guarded((-(-a // block), -(-k // 128)), F32)
    mh.mhlmoe_quantize(x, block_rows=block, transpose=transpose, q=q, scales=scales)
    torch.cuda.synchronize()
    q_ok(), s_ok()
    v = np.zeros((a, k))
    v[:, :rows if transpose else cols] = ref.host(x).T if transpose else ref.host(x)
    ref.check_blocks(ref.host(q), ref.host(scales), v, block, 0.0, f"{rows}x{cols}")
    if transpose:
        assert np.all(ref.host(q)[:, rows:] == 0)


@pytest.mark.parametrize("block,transpose", [(1, False), (128, False), (1, True), (128, True)])
def test_quantize_borders_and_special_blocks(block, transpose):
    """Every e4m3 value and every midpoint of two of them, under scales of a
    power of two: the quotients are exact, so the result is the nearest, ties
    to even.  Blocks with a NaN or an infinity become NaN, zero and tiny blocks
    keep the smallest scale."""
    codes = np.arange(128, dtype=np.uint8)[:127]
    vals = torch.from_numpy(codes).view(ref.E4M3).float().numpy()
    pts = np.concatenate([vals, (vals[1:] + vals[:-1]) / 2, -vals[1:], -(vals[1:] + vals[:-1]) / 2])
    x = np.zeros((384, 128), dtype=np.float32)
    at = np.arange(pts.size)
    x[1 + at // 127, 1 + at % 127] = pts * 4.0
    x[:128, 0] = 448 * 4.0  # every row of the first tile has the largest value,
    x[0, :] = 448 * 4.0     # and every column
    x[130, 5], x[140, 6] = np.nan, np.inf
    x[256:, :] = 2.0 ** -140  # below 448 * 2^-126
    xt = torch.from_numpy(x).cuda()
    q, s = mh.mhlmoe_quantize(xt, block_rows=block, transpose=transpose)
    q, s = ref.host(q), ref.host(s)
    deq = q * ref.spread(s, q.shape, block)
    deq = deq.T if transpose else deq
    want = torch.from_numpy(x[:128] / 4).to(ref.E4M3).float().numpy() * 4.0
    assert np.array_equal(deq[:128], want)
    bad = np.isnan(deq[128:256])
    if block == 128:
        assert bad.all()
    elif transpose:
        assert np.array_equal(bad.all(axis=0), np.isin(np.arange(128), [5, 6])) and bad.sum() == 256
    else:
        assert np.array_equal(bad.all(axis=1), np.isin(np.arange(128), [2, 12])) and bad.sum() == 256
    assert np.all(deq[256:] == 0)  # 2^-140 / 2^-126 = 2^-14, below half of e4m3's smallest, 2^-10


GEMM_SHAPES = [(1, 1, 16), (1, 7, 128), (2, 128, 400), (3, 1000, 144), (15, 16, 112), (16, 33, 256),
               (17, 130, 1040), (31, 512, 2048), (33, 96, 16), (48, 257, 640), (63, 64, 128),
               (64, 512, 384), (65, 127, 272), (100, 300, 512), (127, 129, 128), (128, 128, 1024),
               (129, 384, 160), (255, 257, 256), (256, 256, 128), (300, 520, 896), (513, 640, 1152),
               (1100, 1300, 336),
               # B of 8192 rows and more under few rows of A; over 256 tiles of 64 x 64, of 128 x 128;
               # enough for tiles of 256 x 256, whole and not
               (20, 8209, 272), (32, 8192, 1152), (1, 10249, 272), (16, 16384, 144), (19, 16401, 400),
               (1030, 1100, 144), (1152, 1152, 1152),
               (2310, 2050, 272), (2304, 2048, 896), (3600, 3401, 272), (4096, 3328, 640)]


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("M,N,K", GEMM_SHAPES)
@pytest.mark.parametrize("block", [128, 1])
def test_gemm(M, N, K, block, dtype):
    announce(f"gemm {M}x{N}x{K} block={block} {dtype}")
    g = _gen(M * 3 + N * 5 + K)
    A, sa = mh.mhlmoe_quantize(_randn(g, M, K) * torch.exp(_randn(g, M, 1)))
    B, sb = mh.mhlmoe_quantize(_randn(g, N, K) * torch.exp(_randn(g, N, 1)), block_rows=block)
    C, ok = _guarded((M, N), dtype)
    mh.mhlmoe_gemm_scaled(A, sa, B, sb, b_block_rows=block, dtype=dtype, C=C)
    torch.cuda.synchronize()
    ok()
    want, mag = ref.gemm64(ref.host(A), ref.host(sa), ref.host(B), ref.host(sb), block)
    off = np.abs(ref.host(C) - want)
    bad = off > ref.gemm_bound(want, mag, K, dtype)
    assert not bad.any(), f"{bad.sum()} of {bad.size}, first {np.argwhere(bad)[0]}, {off.max()}"


@pytest.mark.parametrize("M,N,K", [(1, 40, 272), (37, 100, 144), (64, 256, 2048), (130, 270, 400),
                                   (300, 260, 640), (1000, 1024, 512), (31, 8200, 400),
                                   (1, 10300, 272), (9, 16400, 4112), (16, 10240, 528),
                                   (25, 16390, 656),
                                   (1100, 1200, 912), (2400, 2100, 528), (3500, 3600, 400)])
@pytest.mark.parametrize("block", [128, 1])
def test_gemm_exact(M, N, K, block):
    """Small whole numbers under powers of two as scales: every sum is exact in
    fp32, so each element must be the exact product (a swapped row, column,
    scale or block would show)."""
    g = _gen(M + N + K)
    KB = -(-K // 128)

    def ints(*s):
        return torch.randint(-4, 5, s, generator=g, device="cuda").float()

    A, B = ints(M, K).to(ref.E4M3), ints(N, K).to(ref.E4M3)
    sa = torch.exp2(torch.randint(-2, 3, (M, KB), generator=g, device="cuda").float())
    sb = torch.exp2(torch.randint(-2, 3, (-(-N // block), KB), generator=g, device="cuda").float())
    C = mh.mhlmoe_gemm_scaled(A, sa, B, sb, b_block_rows=block, dtype=F32)
    want, _ = ref.gemm64(ref.host(A), ref.host(sa), ref.host(B), ref.host(sb), block)
    assert np.array_equal(ref.host(C), want)


def test_gemm_empty():
    f8 = ref.E4M3

    def t(*s, dtype=f8):
        return torch.zeros(s, device="cuda").to(dtype)

    C = torch.full((5, 6), 7.0, device="cuda")
    mh.mhlmoe_gemm_scaled(t(5, 0), t(5, 0, dtype=F32), t(6, 0), t(1, 0, dtype=F32), dtype=F32, C=C)
    assert torch.all(C == 0)
    for M, N in ((0, 6), (5, 0), (0, 0)):
        C = mh.mhlmoe_gemm_scaled(t(M, 32), t(M, 1, dtype=F32), t(N, 32),
                                  t(-(-N // 128), 1, dtype=F32))
        assert C.shape == (M, N)
    assert mh.mhlmoe_rmsnorm(t(0, 64, dtype=BF16), t(64, dtype=F32), EPS)["y"].shape == (0, 64)
    dw = torch.full((64,), 3.0, device="cuda")
    mh.mhlmoe_rmsnorm_backward(t(0, 64, dtype=BF16), t(64, dtype=F32), EPS, t(0, 64, dtype=BF16),
                               dweight=dw)
    assert torch.all(dw == 0)
    for tr in (False, True):
        q, s = mh.mhlmoe_quantize(t(0, 64, dtype=BF16), transpose=tr)
        assert q.numel() == 0 and s.numel() == 0


@pytest.mark.parametrize("M", [5, 70, 300, 1500])
def test_gemm_special_values_stay_in_their_row(M):
    """A NaN in a row of A, or an infinite scale, reaches that row of C alone."""
    g = _gen(M)
    A, sa = mh.mhlmoe_quantize(_randn(g, M, 384))
    B, sb = mh.mhlmoe_quantize(_randn(g, 200 if M < 1000 else 1100, 384), block_rows=128)
    clean = mh.mhlmoe_gemm_scaled(A, sa, B, sb, dtype=F32)
    A.view(torch.uint8)[1, 130] = 0x7F
    sa[3, 2] = float("inf")
    C = mh.mhlmoe_gemm_scaled(A, sa, B, sb, dtype=F32)
    rows = [i for i in range(M) if i not in (1, 3)]
    assert torch.equal(C[rows], clean[rows])
    assert torch.isnan(C[1]).all() and not torch.isfinite(C[3]).any()


def test_gemm_far_offsets():
    """A of more than 2^32 bytes, K at its largest: what lies in the last rows
    and the last blocks arrives, against the product of those blocks alone."""
    M, N, K, used = 520, 130, (1 << 23) - 128, 272
    g = _gen(6)
    A = torch.zeros((M, K), dtype=torch.uint8, device="cuda").view(ref.E4M3)
    B = torch.zeros((N, K), dtype=torch.uint8, device="cuda").view(ref.E4M3)
    a, _ = mh.mhlmoe_quantize(_randn(g, M, used))
    b, _ = mh.mhlmoe_quantize(_randn(g, N, used))
    at = K - used - 112 - used % 128  # a block's start, and a block behind the last one used
    at -= at % 128
    A.view(torch.uint8)[:, at:at + used] = a.view(torch.uint8)
    B.view(torch.uint8)[:, at:at + used] = b.view(torch.uint8)
    KB, kb = K // 128, at // 128
    sa, sb = torch.ones((M, KB), device="cuda"), torch.ones((2, KB), device="cuda")
    sa[:, kb:] = torch.rand((M, KB - kb), generator=g, device="cuda")
    sb[:, kb:] = torch.rand((2, KB - kb), generator=g, device="cuda")
    C = mh.mhlmoe_gemm_scaled(A, sa, B, sb, dtype=F32)
    n = -(-used // 128)
    want, mag = ref.gemm64(ref.host(a), ref.host(sa[:, kb:kb + n]), ref.host(b),
                           ref.host(sb[:, kb:kb + n]), 128)
    assert np.all(np.abs(ref.host(C) - want) <= ref.gemm_bound(want, mag, used, F32))


def test_gemm_many_columns():
    """So many rows of B that a workgroup for every 16 would pass 2^32 threads."""
    N, K = (1 << 26) + 37, 16
    g = _gen(4)
    A, sa = mh.mhlmoe_quantize(_randn(g, 3, K))
    B = torch.randint(0, 120, (N, K), generator=g, device="cuda", dtype=torch.uint8).view(ref.E4M3)
    sb = torch.rand((-(-N // 128), 1), generator=g, device="cuda")
    C = mh.mhlmoe_gemm_scaled(A, sa, B, sb)
    for at in (0, 1 << 25, N - 100 - N % 128):
        rows = slice(at, min(at + 200, N))
        tiles = sb[at // 128:at // 128 + 3]
        want, mag = ref.gemm64(ref.host(A), ref.host(sa), ref.host(B[rows]),
                               np.repeat(ref.host(tiles), 128, 0)[at % 128:][:B[rows].shape[0]], 1)
        assert np.all(np.abs(ref.host(C[:, rows]) - want) <= ref.gemm_bound(want, mag, K, BF16))


def test_gradient_products():
    """The products of a training step in 8 bits: C = A B^T, dA = dC B, dB =
    dC^T A, each against the 64-bit product of the same 8-bit operands, and
    B's transposed tiles against its tiles."""
    M, N, K = 203, 144, 272
    g = _gen(1)
    a, b, dc = _randn(g, M, K, dtype=BF16), _randn(g, N, K), _randn(g, M, N, dtype=BF16)
    B, sb = mh.mhlmoe_quantize(b, block_rows=128)
    Bt, sbt = mh.mhlmoe_quantize(b, block_rows=128, transpose=True)
    assert torch.equal(sbt, sb.t()) and torch.equal(Bt.view(torch.uint8), B.view(torch.uint8).t())
    At, sat = mh.mhlmoe_quantize(a, transpose=True)          # [K][M16]
    dCq, sdc = mh.mhlmoe_quantize(dc)                        # [M][N]
    dCt, sdct = mh.mhlmoe_quantize(dc, transpose=True)       # [N][M16]
    dA = mh.mhlmoe_gemm_scaled(dCq, sdc, Bt, sbt, dtype=BF16)
    dB = mh.mhlmoe_gemm_scaled(dCt, sdct, At, sat, b_block_rows=1, dtype=F32)
    assert dA.shape == (M, K) and dB.shape == (N, K)
    want, mag = ref.gemm64(ref.host(dCq), ref.host(sdc), ref.host(Bt), ref.host(sbt), 128)
    assert np.all(np.abs(ref.host(dA) - want) <= ref.gemm_bound(want, mag, N, BF16))
    want, mag = ref.gemm64(ref.host(dCt), ref.host(sdct), ref.host(At), ref.host(sat), 1)
    assert np.all(np.abs(ref.host(dB) - want) <= ref.gemm_bound(want, mag, M, F32))
    # and of the unquantised operands: 2^-4 of each factor's magnitude, as its 8 bits are rounded
    # (values below 2^-6 of e4m3's grid by 2^-10 of the scale, 2^-18.8 of the block's largest)
    full = ref.host(dc).T @ ref.host(a)
    tol = np.abs(ref.host(dc)).T @ np.abs(ref.host(a)) * (2 * 2.0 ** -4 + 2.0 ** -8)
    tiny = 2.0 ** -18 * (np.abs(ref.host(dc)).max() * np.abs(ref.host(a)).sum(axis=0)[None, :]
                         + np.abs(ref.host(dc)).sum(axis=0)[:, None] * np.abs(ref.host(a)).max())
    assert np.all(np.abs(ref.host(dB) - full) <= tol + tiny)


def _layer_inputs(T, dm, Nh, dh, Ne, dff, dtype, routing, gelu, seed=0):
    g = _gen(seed)
    N = Nh * dh
    p = dict(x=_randn(g, T, dm, dtype=dtype), residual=_randn(g, T, dm, dtype=dtype),
             norm_weight=1 + 0.1 * _randn(g, dm))
    p["W_in"], p["scale_in"] = mh.mhlmoe_quantize(_randn(g, N, dm) * dm ** -0.5, block_rows=128)
    if routing:
        p["W_r"], p["scale_r"] = mh.mhlmoe_quantize(_randn(g, N, dm) * dm ** -0.5, block_rows=128)
    p["W_out"], p["scale_out"] = mh.mhlmoe_quantize(_randn(g, dm, N) * N ** -0.5, block_rows=128)
    p["W_router"] = _randn(g, Nh, Ne, dh) * dh ** -0.5
    p["bias"] = 0.1 * _randn(g, Nh, Ne)
    p["W1"] = (_randn(g, Nh, Ne, dff, dh) * dh ** -0.5).to(dtype)
    p["W3"] = None if gelu else (_randn(g, Nh, Ne, dff, dh) * dh ** -0.5).to(dtype)
    p["W2"] = (_randn(g, Nh, Ne, dh, dff) * dff ** -0.5).to(dtype)
    return p


def _call_layer(p, Nh, k, **kw):
    args = [p[n] for n in ("x", "norm_weight")] + [EPS] + [
        p[n] for n in ("W_in", "scale_in", "W_router", "bias", "W1", "W3", "W2", "W_out", "scale_out")]
    return mh.mhlmoe_latent_layer_scaled(*args, Nh, k, residual=p["residual"], W_r=p.get("W_r"),
                                         scale_r=p.get("scale_r"), **kw)


def _by_parts(p, Nh, dh, k):
    """The same by the calls that the layer is documented as."""
    dtype, T = p["x"].dtype, p["x"].shape[0]
    n = mh.mhlmoe_rmsnorm(p["x"], p["norm_weight"], EPS, residual=p["residual"], quantized=True)
    X = mh.mhlmoe_gemm_scaled(n["q"], n["scales"], p["W_in"], p["scale_in"], dtype=dtype)
    R = X
    if "W_r" in p:
        R = mh.mhlmoe_gemm_scaled(n["q"], n["scales"], p["W_r"], p["scale_r"], dtype=dtype)
    X, R = X.view(T, Nh, dh), R.view(T, Nh, dh)
    Y, idx, gate, counts = mh.mhlmoe_layer_routed(X, R, p["W_router"], p["bias"], p["W1"], p["W3"],
                                                  p["W2"], k)
    yq, ys = mh.mhlmoe_quantize(Y.view(T, Nh * dh))
    out = mh.mhlmoe_gemm_scaled(yq, ys, p["W_out"], p["scale_out"], dtype=dtype)
    res = dict(out=out, sum=n["sum"], X_lat=X, Y_lat=Y, idx=idx, gate=gate, counts=counts)
    if "W_r" in p:
        res["R_lat"] = R
    return res


LAYERS = [  # T, d_model, n_heads, d_head, n_experts, top_k, d_ff, dtype, routing sub-tokens, GELU
    (1, 1024, 8, 128, 64, 8, 256, BF16, False, False),
    (33, 208, 3, 64, 16, 2, 64, BF16, True, False),
    (257, 512, 4, 128, 32, 4, 128, BF16, True, True),
    (100, 144, 5, 64, 9, 3, 96, F32, False, False),
    (4096, 1024, 8, 128, 64, 8, 256, BF16, False, False)]


@pytest.mark.parametrize("case", LAYERS, ids=lambda c: "T%d_dm%d_h%dx%d" % c[:4])
def test_latent_layer_scaled(case):
    T, dm, Nh, dh, Ne, k, dff, dtype, routing, gelu = case
    announce(f"latent layer scaled {case}")
    p = _layer_inputs(T, dm, Nh, dh, Ne, dff, dtype, routing, gelu)
    got = _call_layer(p, Nh, k)
    want = _by_parts(p, Nh, dh, k)
    torch.cuda.synchronize()
    assert set(got) == set(want)
    for name in want:
        assert torch.equal(got[name], want[name]), name
    # the projections against 64 bits of their own operands
    n = mh.mhlmoe_rmsnorm(p["x"], p["norm_weight"], EPS, residual=p["residual"], quantized=True)
    rows = slice(0, 64)
    C, mag = ref.gemm64(ref.host(n["q"][rows]), ref.host(n["scales"][rows]), ref.host(p["W_in"]),
                        ref.host(p["scale_in"]), 128)
    off = np.abs(ref.host(got["X_lat"][rows]).reshape(C.shape) - C)
    assert np.all(off <= ref.gemm_bound(C, mag, dm, dtype))


def test_latent_layer_scaled_empty_batch():
    p = _layer_inputs(0, 208, 3, 64, 16, 64, BF16, True, False)
    counts = torch.full((3, 16), 7, dtype=torch.int32, device="cuda")
    got = _call_layer(p, 3, 2, counts=counts)
    torch.cuda.synchronize()
    assert got["out"].shape == (0, 208) and torch.all(counts == 0)


def test_side_stream_and_graph():
    """The layer and the norm's gradient on a side stream, and captured into
    one graph that is replayed with new inputs and eager work between."""
    T, dm, Nh, dh, Ne, k, dff = 130, 256, 2, 128, 16, 2, 128
    p = _layer_inputs(T, dm, Nh, dh, Ne, dff, BF16, True, False)
    dy = _randn(_gen(5), T, dm, dtype=BF16)
    ws = torch.empty(mh.mhlmoe_latent_layer_scaled_workspace(T, dm, Nh, dh, Ne, k, dff),
                     dtype=torch.uint8, device="cuda")
    wb = torch.empty(mh.mhlmoe_rmsnorm_backward_workspace(T, dm), dtype=torch.uint8, device="cuda")
    eager = _call_layer(p, Nh, k)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        got = _call_layer(p, Nh, k, workspace=ws)
    explicit = _call_layer(p, Nh, k, stream=side)
    side.synchronize()
    assert torch.equal(got["out"], eager["out"]) and torch.equal(explicit["out"], eager["out"])
    dx, dw = torch.empty_like(dy), torch.empty(dm, device="cuda")
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = _call_layer(p, Nh, k, workspace=ws)
        mh.mhlmoe_rmsnorm_backward(got["sum"], p["norm_weight"], EPS, dy, dx=dx, dweight=dw,
                                   workspace=wb)
    for i in range(4):
        g = _gen(100 + i)
        p["x"].copy_(_randn(g, T, dm))
        dy.copy_(_randn(g, T, dm))
        torch.cuda.synchronize()
        graph.replay()
        want = _call_layer(p, Nh, k)
        dx2, dw2 = mh.mhlmoe_rmsnorm_backward(want["sum"], p["norm_weight"], EPS, dy)
        torch.cuda.synchronize()
        for name in want:
            assert torch.equal(got[name], want[name]), (i, name)
        assert torch.equal(dx, dx2) and torch.equal(dw, dw2), i


def test_many_rows():
    """More rows than one workgroup each: 2^20 workgroups are looped over, and
    offsets pass 2^31 bytes."""
    T, d = (1 << 22) + 3, 520
    x = torch.zeros((T, d), dtype=BF16, device="cuda")
    w = torch.ones(d, device="cuda")
    at = torch.tensor([0, 1 << 21, T - 2, T - 1], device="cuda")
    rows = _randn(_gen(2), len(at), d, dtype=BF16)
    x[at] = rows
    out = mh.mhlmoe_rmsnorm(x, w, EPS)["y"]
    assert torch.equal(out[at], mh.mhlmoe_rmsnorm(rows, w, EPS)["y"])
    del out
    q, s = mh.mhlmoe_quantize(x[:, :512].contiguous())
    q2, s2 = mh.mhlmoe_quantize(rows[:, :512].contiguous())
    assert torch.equal(q.view(torch.uint8)[at], q2.view(torch.uint8)) and torch.equal(s[at], s2)


@pytest.mark.parametrize("T,d", [(16383, 512), (16387, 512), (20001, 100), (40003, 64),
                                 (16384, 1024), (2500, 16392), (600, 65536), (300, 65535)])
def test_rmsnorm_backward_long_batch(T, d):
    """Rows that the workgroups loop over, on both sides of the two numbers of
    workgroups, and more of wide rows than there are chunks."""
    g = _gen(T + d)
    h, dy = _randn(g, T, d, dtype=BF16), _randn(g, T, d, dtype=BF16)
    w = 1 + 0.3 * _randn(g, d)
    dx, dw = mh.mhlmoe_rmsnorm_backward(h, w, EPS, dy)
    want, wdw, t_abs, dw_abs = ref.norm_backward64(ref.host(h), ref.host(w), EPS, ref.host(dy), None)
    eps = 3 * ref.norm_eps(d) + 4 * ref.U
    assert np.all(np.abs(ref.host(dx) - want) <= eps * t_abs + (ref.HALF[BF16] + ref.U) * np.abs(want))
    assert np.all(np.abs(ref.host(dw) - wdw) <= (T * ref.U + ref.norm_eps(d) + 2 * ref.U) * dw_abs)


def test_rmsnorm_backward_far_rows():
    """Offsets that pass 2^31 elements.  A row's dx does not depend on the other
    rows; dy is zero but in four, so dw is their sum in some order."""
    T, d = (1 << 22) + 3, 520
    at = torch.tensor([0, 1 << 21, T - 2, T - 1], device="cuda")
    h = torch.zeros((T, d), dtype=BF16, device="cuda")
    dy = torch.zeros((T, d), dtype=BF16, device="cuda")
    g = _gen(4)
    rows, drows = _randn(g, 4, d, dtype=BF16), _randn(g, 4, d, dtype=BF16)
    h[at], dy[at] = rows, drows
    w = 1 + 0.3 * _randn(g, d)
    dx, dw = mh.mhlmoe_rmsnorm_backward(h, w, EPS, dy)
    dx4, dw4 = mh.mhlmoe_rmsnorm_backward(rows, w, EPS, drows)
    assert torch.equal(dx[at], dx4)
    assert not dx[1:1 << 21].any()
    # two sums of the same four numbers, each within 3 roundings of the exact one
    _, _, _, dw_abs = ref.norm_backward64(ref.host(rows), ref.host(w), EPS, ref.host(drows), None)
    assert np.all(np.abs(ref.host(dw) - ref.host(dw4)) <= 6 * ref.U * dw_abs * (1 + 1e-5))


@pytest.mark.parametrize("raw", [False, True])
def test_tensors_of_a_call_belong_to_its_stream(raw):
    """A workspace that the call makes, and an output that is dropped at once,
    are not handed to the current stream while the given one still uses them."""
    g = _gen(6)
    T, d = 4096, 1024
    h, dy = _randn(g, T, d, dtype=BF16), _randn(g, T, d, dtype=BF16)
    w = 1 + 0.3 * _randn(g, d)
    dx, dw = mh.mhlmoe_rmsnorm_backward(h, w, EPS, dy)
    y = mh.mhlmoe_rmsnorm(h, w, EPS, residual=dy)["y"]
    q, scales = mh.mhlmoe_quantize(h)
    dx2, dw2, y2 = torch.empty_like(dx), torch.empty_like(dw), torch.empty_like(y)
    a = _randn(g, 4096, 4096)
    side = torch.cuda.Stream()
    stream = side.cuda_stream if raw else side
    torch.cuda.synchronize()
    torch.cuda.empty_cache()
    with torch.cuda.stream(side):
        for _ in range(10):  # milliseconds in front of the calls
            a @ a
    mh.mhlmoe_rmsnorm_backward(h, w, EPS, dy, dx=dx2, dweight=dw2, stream=stream)
    mh.mhlmoe_rmsnorm(h, w, EPS, residual=dy, y=y2, stream=stream)
    q2, scales2 = mh.mhlmoe_quantize(h, stream=stream)
    fill = [torch.full((n,), float("nan"), device="cuda") for n in (T * d // 2, 512 * d) * 4]
    torch.cuda.synchronize()
    assert torch.equal(dx, dx2) and torch.equal(dw, dw2) and torch.equal(y, y2)
    assert torch.equal(q.view(torch.uint8), q2.view(torch.uint8)) and torch.equal(scales, scales2)
    assert all(torch.isnan(f).all() for f in fill)


def test_default_stream_by_handle_and_capture_by_argument():
    """stream may be the default stream's handle (0), and the capturing stream
    itself: outputs and workspace are then the graph's."""
    g = _gen(9)
    h, dy, w = _randn(g, 70, 520, dtype=BF16), _randn(g, 70, 520, dtype=BF16), _randn(g, 520)
    dx, dw = mh.mhlmoe_rmsnorm_backward(h, w, EPS, dy)
    dx0, dw0 = mh.mhlmoe_rmsnorm_backward(h, w, EPS, dy, stream=0)
    torch.cuda.synchronize()
    assert torch.equal(dx, dx0) and torch.equal(dw, dw0)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        dx1, dw1 = mh.mhlmoe_rmsnorm_backward(h, w, EPS, dy, stream=torch.cuda.current_stream())
    for i in range(3):
        h.copy_(_randn(g, 70, 520))
        torch.cuda.synchronize()
        graph.replay()
        dx, dw = mh.mhlmoe_rmsnorm_backward(h, w, EPS, dy)
        torch.cuda.synchronize()
        assert torch.equal(dx, dx1) and torch.equal(dw, dw1), i
