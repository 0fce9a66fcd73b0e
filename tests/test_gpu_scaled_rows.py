"""The norm's gradient in place in each of its forms, and the quantisation of
more blocks than one round of workgroups takes."""
import pytest
import torch

import paper_2602_04870_amd as mh
from tests import scaled_ref as ref
from tests.gpu_util import announce, needs_gpu

pytestmark = [pytest.mark.gpu, needs_gpu]

BF16, F32 = torch.bfloat16, torch.float32


# part of a wavefront (8 columns a piece, and one by one), a wavefront, a workgroup of 256 and of
# 512 threads; two kernels of 8 columns and of one, of which the second overwrites what both read
@pytest.mark.parametrize("d", [40, 60, 100, 200, 264, 1001, 1024, 2048, 4096, 5001, 8192, 16384,
                               16400, 40000])
@pytest.mark.parametrize("dtype", [BF16, F32])
def test_rmsnorm_backward_in_place(d, dtype):
    """dx may be dy or dsum: the same bits as with a dx of its own, in a batch
    that some forms loop over and one that they do not."""
    for T in (3, 600):
        announce(f"rmsnorm_backward in place T={T} d={d} {dtype}")
        g = torch.Generator(device="cuda").manual_seed(d + T)
        h, dy, ds = (torch.randn(T, d, generator=g, device="cuda").to(dtype) for _ in range(3))
        w = 1 + 0.1 * torch.randn(d, generator=g, device="cuda")
        for dsum in (None, ds):
            dx, dw = mh.mhlmoe_rmsnorm_backward(h, w, 1e-6, dy, dsum=dsum)
            for alias in range(1 if dsum is None else 2):
                a = [dy.clone(), None if dsum is None else ds.clone()]
                dx2, dw2 = mh.mhlmoe_rmsnorm_backward(h, w, 1e-6, a[0], dsum=a[1], dx=a[alias])
                assert dx2.data_ptr() == a[alias].data_ptr()
                assert torch.equal(dx, dx2) and torch.equal(dw, dw2), (T, alias)


def test_quantize_more_blocks_than_one_round():
    """2^26 + 5 blocks of 1 x 128: one round of 2^20 workgroups takes 2^26."""
    rows, cols = (1 << 26) + 5, 16
    announce(f"quantize {rows}x{cols}")
    at = torch.tensor([0, 1, 1 << 25, (1 << 26) - 1, 1 << 26, rows - 2, rows - 1], device="cuda")
    g = torch.Generator(device="cuda").manual_seed(1)
    some = torch.randn(len(at), cols, generator=g, device="cuda").to(BF16)
    x = torch.zeros((rows, cols), dtype=BF16, device="cuda")
    x[at] = some
    q = torch.full((rows, cols), 0x55, dtype=torch.uint8, device="cuda").view(ref.E4M3)
    scales = torch.full((rows, 1), 7.0, device="cuda")
    mh.mhlmoe_quantize(x, q=q, scales=scales)
    q2, s2 = mh.mhlmoe_quantize(some)
    ref.check_blocks(ref.host(q2), ref.host(s2), ref.host(some), 1, 0.0, "rows by themselves")
    assert torch.equal(q.view(torch.uint8)[at], q2.view(torch.uint8)) and torch.equal(scales[at], s2)
    rest = torch.ones(rows, dtype=torch.bool, device="cuda")
    rest[at] = False
    assert not q.view(torch.uint8)[rest].any() and torch.all(scales[rest] == ref.SCALE_MIN)
