"""Which of e4m3's values a quotient is rounded to: v / scale is taken in fp32
first."""
import numpy as np
import pytest
import torch

import paper_2602_04870_amd as mh
from tests import scaled_ref as ref
from tests.gpu_util import announce, needs_gpu

pytestmark = [pytest.mark.gpu, needs_gpu]

BF16, F32 = torch.bfloat16, torch.float32


def e4m3(v):
    """v (64 bits) to the nearest of e4m3's values, ties to even."""
    return np.rint(v / ref.step(v)) * ref.step(v)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("block,transpose", [(1, False), (128, False), (1, True), (128, True)])
def test_quotient(block, transpose, dtype):
    """The kernel takes v times about 1 / scale (an ulp off, 2^-23) and corrects
    it by what remains: r is off by 1.5 * 2^-23, what remains is known to 2^-24
    of itself and multiplied by a reciprocal 2^-23 off, so the sum before its
    rounding to fp32 is off by less than 1.5 * 2^-23 (2^-23 + 2 * 2^-24) < 2^-44.
    The result is then that of the fp32 neighbours of v / scale at this distance,
    and the scale is max / 448 rounded once."""
    announce(f"quotient block={block} transpose={transpose} {dtype}")
    g = torch.Generator().manual_seed(11)
    x = (torch.randn(640, 1152, generator=g) * torch.exp(torch.randn(640, 1, generator=g))).to(dtype)
    q, s = mh.mhlmoe_quantize(x.cuda(), block_rows=block, transpose=transpose)
    v = ref.host(x).T if transpose else ref.host(x)
    want = (ref.block_max(v, block) / 448.0).astype(np.float32).astype(np.float64)
    assert np.array_equal(ref.host(s), want)
    r = v / ref.spread(want, v.shape, block)
    lo, hi = (e4m3((r * f).astype(np.float32).astype(np.float64)) for f in (1 - 2.0 ** -44, 1 + 2.0 ** -44))
    assert np.all((ref.host(q) == lo) | (ref.host(q) == hi))
    assert np.mean(lo != hi) < 1e-5
    if dtype == BF16 and block == 1:  # values on a border in fp32 alone: what the rounding decides
        assert np.sum(e4m3(r) != lo) > 100
