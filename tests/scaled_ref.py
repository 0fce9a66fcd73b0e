"""Plain 64-bit references of the operators around the heads (norm, gradient,
8-bit blocks, 8-bit product) and what their results may be off by.

U is half a step of fp32 relative to the value, HALF that of each stored type."""
from __future__ import annotations

import numpy as np
import torch

U = 2.0 ** -24
HALF = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8}
E4M3 = torch.float8_e4m3fn
SCALE_MIN = 2.0 ** -126


def host(t: torch.Tensor) -> np.ndarray:
    """Any tensor's values in 64 bits."""
    return t.detach().float().cpu().numpy().astype(np.float64)


def step(v):
    """The distance of e4m3's values around |v| (3 bits behind the leading one; 2^-9 below 2^-6)."""
    e = np.floor(np.log2(np.maximum(np.abs(v), 2.0 ** -6)))
    return np.exp2(e - 3)


def block_max(v, block_rows):
    """Largest magnitude of every block_rows x 128 block."""
    r, c = v.shape
    rb, cb = -(-r // block_rows), -(-c // 128)
    p = np.zeros((rb * block_rows, cb * 128))
    p[:r, :c] = np.abs(v)
    return p.reshape(rb, block_rows, cb, 128).max(axis=(1, 3))


def spread(scales, shape, block_rows):
    """A block's scale at each of its values."""
    return np.repeat(np.repeat(scales, block_rows, 0), 128, 1)[:shape[0], :shape[1]]


def check_blocks(q, scales, v, block_rows, eps, what):
    """q and scales (64-bit values) as the 8 bits of v, which the kernel knew
    to a relative eps: the scale is amax / 448 rounded once more, and each q is
    within half a step of v / scale.  The steps on the way: eps of v, the
    multiply by 1 / scale with its correction (an ulp, 2 U), and the scale's
    own rounding is in the given scale already."""
    want = np.maximum(block_max(v, block_rows) / 448.0, SCALE_MIN)
    assert np.all(np.abs(scales - want) <= (eps + U) * want), what
    r = v / spread(scales, v.shape, block_rows)
    half = 0.5 * np.maximum(step(r), step(q))
    bad = np.abs(q - r) > half + (eps + 4 * U) * np.abs(r)
    assert not bad.any(), f"{what}: {bad.sum()} values, first {np.argwhere(bad)[0]}"


def norm_eps(d):
    """Relative error of the fp32 norm: a lane adds at most d / 64 squares (d /
    256 in the wider forms) and the lanes' sums in at most 9 steps, half of
    which reaches 1 / sqrt; mean, eps, square root and reciprocal and the two
    products add 8 more."""
    return (d / 128 + 5 + 8 + 3) * U


def norm64(h, w, eps):
    rs = 1.0 / np.sqrt((h * h).mean(axis=1, keepdims=True) + eps)
    return h * rs * w


def norm_backward64(h, w, eps, dy, dsum):
    """(dx, dw) and the sums of magnitudes that their errors scale with."""
    d = h.shape[1]
    rs = 1.0 / np.sqrt((h * h).mean(axis=1, keepdims=True) + eps)
    g = dy * w
    k = (g * h).sum(axis=1, keepdims=True) / d * rs ** 2
    t = rs * (g - h * k)
    k_abs = np.abs(g * h).sum(axis=1, keepdims=True) / d * rs ** 2
    t_abs = rs * (np.abs(g) + np.abs(h) * k_abs)
    dx = t if dsum is None else t + dsum
    return dx, (dy * h * rs).sum(axis=0), t_abs, (np.abs(dy * h) * rs).sum(axis=0)


def gemm64(A, sa, B, sb, block_rows):
    """C and the sum of its terms' magnitudes."""
    a = A * spread(sa, A.shape, 1)
    b = B * spread(sb, B.shape, block_rows)
    return a @ b.T, np.abs(a) @ np.abs(b).T


def gemm_bound(C, mag, K, dtype):
    """A block's 128 terms and the blocks are added in fp32 (each addition at
    most U of the magnitudes so far), scales multiplied and applied (3), the
    result rounded to its type.  For bf16 the 8-bit matrix instructions drop,
    of each product, less than 2^-13 of the power of two of the largest of
    eight, which at most the other seven lose: 7 * 2^-13 of that largest
    product, itself no more than the eight magnitudes' sum."""
    dropped = 7 * 2.0 ** -13 if dtype == torch.bfloat16 else 0.0
    return ((128 + -(-K // 128) + 3) * U + dropped) * mag + HALF[dtype] * (np.abs(C) + dropped * mag)
