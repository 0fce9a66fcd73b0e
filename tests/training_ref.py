"""Plain 64-bit references of the training step's operators (layer norm, balance
loss, AdamW) and what their results may be off by.

U is half a step of fp32 relative to the value, HALF that of each stored type."""
from __future__ import annotations

import numpy as np
import torch

from tests.scaled_ref import E4M3, HALF, SCALE_MIN, U, host, spread, step

__all__ = ["E4M3", "HALF", "SCALE_MIN", "U", "host", "step"]


# ---------------------------------------------------------------------------
# Layer norm
# ---------------------------------------------------------------------------
def adds(d):
    """Additions on the way of a row's sum: a lane's d / 64 (at most 8 more in the
    forms of 16 lanes), 6 steps between lanes, 7 between wavefronts."""
    return d / 64 + 8 + 6 + 7


def norm_parts(h, eps):
    mu = h.mean(axis=1, keepdims=True)
    rs = 1.0 / np.sqrt(((h - mu) ** 2).mean(axis=1, keepdims=True) + eps)
    return (h - mu) * rs, rs


def layernorm64(h, w, b, eps):
    """y, and its error in fp32.  c = h - mu is off by U |c|; the mean that is left,
    mean c, by (adds + 2) U mean |c|, of which rs makes at most (adds + 2) U (mean
    |n| <= 1); the squares' sum by (adds + 6) U, half of which reaches rs, and
    divisions and root by 4 U: together (adds + 10) U (|n| + 1); w and b add one
    rounding."""
    n, _ = norm_parts(h, eps)
    y = n * w + b
    return y, (adds(h.shape[1]) + 10) * U * (np.abs(n) + 1) * np.abs(w) + 2 * U * np.abs(y)


def layernorm_backward64(h, w, eps, dy, dsum):
    """(dx, dw, db) and their errors in fp32 before dx is rounded: every sum over a
    row is off by (adds + 2) U of its terms' magnitudes, its n by (adds + 10) U (|n| +
    1); three of them meet in dx.  dw and db add T terms in some order."""
    T, d = h.shape
    n, rs = norm_parts(h, eps)
    g = dy * w
    mean = lambda v: v.mean(axis=1, keepdims=True)  # noqa: E731
    t = rs * (g - mean(g) - n * mean(g * n))
    n1 = np.abs(n) + 1
    t_off = 3 * (adds(d) + 12) * U * rs * (np.abs(g) + mean(np.abs(g)) + n1 * mean(np.abs(g) * n1))
    dx = t if dsum is None else t + dsum
    dw_off = (T + adds(d) + 12) * U * (np.abs(dy) * n1).sum(axis=0)
    return (dx, (dy * n).sum(axis=0), dy.sum(axis=0), t_off, dw_off,
            (T + 2) * U * np.abs(dy).sum(axis=0))


def check_blocks(q, scales, v, off, what):
    """q and scales (64-bit values) as the 8 bits of the rows v, which the kernel
    knew to within off: a scale is its block's largest magnitude over 448, rounded,
    and each q within half a step of v / scale."""
    T, d = v.shape
    pad = lambda a: np.pad(a, ((0, 0), (0, -d % 128))).reshape(T, -1, 128).max(axis=2)  # noqa: E731
    want = np.maximum(pad(np.abs(v)) / 448.0, SCALE_MIN)
    assert np.all(np.abs(scales - want) <= pad(off) / 448.0 + 2 * U * want), what
    s = spread(scales, v.shape, 1)
    r = v / s
    half = 0.5 * np.maximum(step(r), step(q))
    bad = np.abs(q - r) > half + off / s + 4 * U * np.abs(r)
    assert not bad.any(), f"{what}: {bad.sum()} values, first {np.argwhere(bad)[0]}"


# ---------------------------------------------------------------------------
# Balance loss
# ---------------------------------------------------------------------------
def counts64(idx, mask, Ne):
    T, Nh, k = idx.shape
    c = np.zeros((Nh, Ne), np.int64)
    for h in range(Nh):
        at = idx[mask, h].reshape(-1) if mask is not None else idx[:, h].reshape(-1)
        at = at[(at >= 0) & (at < Ne)]
        np.add.at(c[h], at, 1)
    return c


class Balance:
    """The loss and its gradient of one problem, and their errors.

    A score is exact products of pieces added in fp32: 3 products per term at most
    (2 for bf16), each addition off by U of the magnitudes so far.  Two fp16 pieces are
    off by 2^-23 = 2 U of the value, and with an fp32 X the product of the second pieces
    is left out, 2^-22 = 4 U: ez = (6 dh + 10) U sum |x w|.  An exponential's argument (z - max) log2 e is rounded where it is up to
    2.9 |z|, log2 e itself is off by 2^-26, and exp2 by an ulp: ep = (4 |z| + 8) U
    with the row's largest |z|."""

    def __init__(self, X, W, counts, mask):
        self.X, self.W, self.counts = X, W, counts
        T, Nh, dh = X.shape
        Ne = W.shape[1]
        self.keep = np.ones(T, bool) if mask is None else mask
        self.n = max(int(self.keep.sum()), 1)
        Xk = np.where(self.keep[:, None, None], X, 0.0)
        self.Xk = Xk
        z = np.einsum("thd,hed->the", Xk, W)
        mag = np.einsum("thd,hed->the", np.abs(Xk), np.abs(W))
        top = z.max(axis=2, keepdims=True)
        self.lse = top[..., 0] + np.log(np.exp(z - top).sum(axis=2))
        self.p = np.exp(z - self.lse[..., None])
        total = counts.sum(axis=1, keepdims=True)
        self.f = (counts * Ne - total) / np.maximum(total, 1)
        self.u = (self.p * self.f).sum(axis=2)
        self.loss = np.where(total[:, 0] > 0,
                             1 + (self.u * self.keep[:, None]).sum(axis=0) / self.n, 0.0)
        ez = (6 * dh + 10) * U * mag.max(axis=2)
        ep = (4 * np.abs(z).max(axis=2) + 8) * U
        self.e_lse = ez + ep + (Ne + 8) * U + 2 * U * np.abs(self.lse)
        self.e_u = (2 * ez + 2 * ep + (2 * Ne + 8) * U) * (self.p * np.abs(self.f)).sum(axis=2)
        self.e_p = ez + ep + self.e_lse  # of p in the gradient, relative
        self.e_loss = ((self.e_u * self.keep[:, None]).sum(axis=0) / self.n
                       + 2 * U * (1 + np.abs(self.loss)))

    def backward(self, dloss, dX_add, dW_add, bf16):
        """dX and dW, and their errors before dX is rounded.  bf16: ds and W meet as one
        fp16 value each, 2^-11 of it off: 2^-10 and 2^-22 of the term.  (It was two
        bf16 pieces each, 3 * 2^-18, before the kernel's operands were fp16.)  What lies
        2^-39 below the largest of its scale's values is lost: 2^-20 U."""
        T, Nh, dh = self.X.shape
        Ne = self.W.shape[1]
        c = dloss / self.n
        ds = self.p * (self.f - self.u[..., None]) * self.keep[:, None, None]
        e_ds = self.p * ((np.abs(self.f) + np.abs(self.u)[..., None]) * (self.e_p[..., None] + 4 * U)
                         + self.e_u[..., None]) * self.keep[:, None, None]
        dX = np.einsum("the,hed->thd", ds, self.W) * c[:, None]
        left = 2.0 ** -10 + 2.0 ** -22 if bf16 else 0.0
        x_off = (np.einsum("the,hed->thd", e_ds, np.abs(self.W))
                 + ((6 * Ne + 10) * U + left)
                 * np.einsum("the,hed->thd", np.abs(ds), np.abs(self.W))) * np.abs(c)[:, None]
        dW = np.einsum("the,thd->hed", ds, self.Xk) * c[:, None, None]
        w_off = (np.einsum("the,thd->hed", e_ds, np.abs(self.Xk))
                 + (6 * T + 10) * U * np.einsum("the,thd->hed", np.abs(ds), np.abs(self.Xk))
                 ) * np.abs(c)[:, None, None]
        if dX_add is not None:
            dX = dX + dX_add
            x_off = x_off + U * (np.abs(dX) + np.abs(dX_add))
        if dW_add is not None:
            dW = dW + dW_add
            w_off = w_off + U * (np.abs(dW) + np.abs(dW_add))
        return dX, dW, x_off + 2 * U * np.abs(dX), w_off + 2 * U * np.abs(dW)


# ---------------------------------------------------------------------------
# AdamW
# ---------------------------------------------------------------------------
def _mix(x):
    low = np.uint64(0xFFFFFFFF)
    x = ((x ^ (x >> np.uint64(16))) * np.uint64(0x6A09E667)) & low
    x = ((x ^ (x >> np.uint64(15))) * np.uint64(0xBB67AE85)) & low
    return x ^ (x >> np.uint64(16))


def random16(n, seed, step_no, first=0):
    """The random numbers in [0, 1) of m and of v at elements first .. first + n - 1."""
    low = np.uint64(0xFFFFFFFF)
    i = np.arange(first, first + n, dtype=np.uint64)
    key = _mix((_mix(np.uint64(seed)) + np.uint64(step_no)) & low)
    x = _mix((((i & low) * np.uint64(0x9E3779B9)) + ((i >> np.uint64(32)) * np.uint64(0x3C6EF373))
              + key) & low)
    return (x & np.uint64(0xFFFF)) * 2.0 ** -16, (x >> np.uint64(16)) * 2.0 ** -16


def adamw64(p, g, m, v, lr, b1, b2, eps, wd, t):
    """(p, m, v) after a step and their errors in fp32: the betas' and their
    complements' roundings, a product or two and an addition each; sqrt, a
    multiply and an addition below the step, a division and a multiply above."""
    m1, v1 = b1 * m + (1 - b1) * g, b2 * v + (1 - b2) * g * g
    em = 5 * U * (np.abs(b1 * m) + np.abs((1 - b1) * g))
    ev = 7 * U * v1
    den = np.sqrt(v1 / (1 - b2 ** t)) + eps
    rate = lr / (1 - b1 ** t)
    p1 = p - rate * m1 / den - lr * wd * p
    ep = rate * (em + 12 * U * np.abs(m1)) / den + 3 * U * np.abs(p) + 4 * U * lr * wd * np.abs(p)
    return p1, m1, v1, ep, em, ev


def check_random_blocks(q, scales, v, off, u, keep, what):
    """q and scales (64-bit values) as v [n] in blocks of 128, rounded up where the
    part below the step is over 1 - u; v known to the kernel within off.  Near a
    border (within off and the quotient's 4 U) either side counts."""
    n = v.size
    pad = lambda a: np.pad(a, (0, -n % 128)).reshape(-1, 128)  # noqa: E731
    want = np.maximum(pad(np.abs(v)).max(axis=1) / 448.0, SCALE_MIN)
    assert np.all(np.abs(scales - want) <= pad(off).max(axis=1) / 448.0 + 2 * U * want), what
    s = np.repeat(scales, 128)[:n]
    r, tol = np.abs(v) / s, off / s + 4 * U * np.abs(v) / s
    grid = step(r)  # (across a border of exponents the point itself is on both grids)
    lo, hi = np.floor((r - tol) / grid + u), np.floor((r + tol) / grid + u)
    if keep:
        lo, hi = np.where(r > tol, np.maximum(lo, 1), lo), np.where(r + tol > 0, np.maximum(hi, 1), hi)
    k = np.abs(q) / grid
    bad = (k < lo) | (k > hi)
    assert not bad.any(), f"{what}: {bad.sum()} values, first at {np.argwhere(bad)[0]}"
    assert np.all((q == 0) | (np.sign(q) == np.sign(v))), what


def blocks8(v):
    """(q, scales) of a tensor's values in blocks of 128, to the nearest."""
    n = v.numel()
    b = torch.nn.functional.pad(v.reshape(-1).float(), (0, -n % 128)).view(-1, 128)
    s = (b.abs().amax(dim=1) / 448.0).clamp(min=SCALE_MIN)
    q = (b / s[:, None]).clamp(-448.0, 448.0).view(-1)[:n]
    return q.to(E4M3).view(v.shape), s


def values8(q, scales):
    """What they stand for, in 64 bits."""
    n = q.numel()
    return host(q).reshape(-1) * np.repeat(host(scales), 128)[:n]
