"""The 8-bit product over contractions that take every form through all states
of its loop along K, compared exactly, in both types of the result."""
import numpy as np
import pytest
import torch

import paper_2602_04870_amd as mh
from tests import scaled_ref as ref
from tests.gpu_util import announce, needs_gpu

pytestmark = [pytest.mark.gpu, needs_gpu]

BF16, F32 = torch.bfloat16, torch.float32

# The tiles fetch the scales of four steps at a time into two chunks in turn: a chunk's memory is
# written again after 4 steps and read again after 8, so more than 8 steps, of one to four blocks
# of 128.  The few-row forms hold 4, 2 or 1 blocks per wavefront and trip: more than one trip of
# the eight wavefronts.
STEPS = [
    # 64 x 64 tiles, four blocks a step: 10, 14 and 32 steps
    (100, 300, 4752), (65, 127, 6800), (256, 256, 16304),
    # 128 x 128 tiles, two blocks a step: 10, 17 and 64 steps
    (1100, 1300, 2320), (1152, 1152, 4112), (1025, 1030, 16304),
    # 128 x 128 tiles, one block a step: 11 and 17
    (2310, 2050, 1296), (2304, 2048, 2064),
    # 256 x 256 tiles (fp32 results: 128 x 128), one block a step: 11, 14 and 4
    (3600, 3401, 1296), (4096, 3328, 1680), (3500, 3600, 400),
    # up to 16 rows of A, 16 rows of B per workgroup: 3 and 2 trips of 4 blocks
    (1, 40, 8208), (16, 130, 8208), (7, 1000, 4240),
    # 32 rows of B: 2 and 3 trips of 2
    (1, 10249, 2192), (9, 16400, 4112),
    # up to 32 rows of A by 16 rows of B: 2 and 3 trips of 4
    (17, 130, 4240), (32, 1000, 8208),
    # by 32: 2 trips of 2; by 64: 2 trips of 1
    (31, 8200, 2192), (25, 16390, 1168)]


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("M,N,K", STEPS)
@pytest.mark.parametrize("block", [128, 1])
def test_whole_numbers(M, N, K, block, dtype):
    """Operands of -2 .. 2 under scales of 2^-2 .. 2^2: a product is at most 4
    and a whole number, far above 2^-13 of any other, and every partial sum is a
    multiple of 2^-4 below K * 4 * 16 < 2^20, so all of them are exact in fp32
    and the result is the exact product, rounded once."""
    assert K < 1 << 14
    announce(f"whole numbers {M}x{N}x{K} block={block} {dtype}")
    g = torch.Generator(device="cuda").manual_seed(M + 3 * N + 5 * K)
    KB = -(-K // 128)

    def ints(lo, hi, *s):
        return torch.randint(lo, hi + 1, s, generator=g, device="cuda").float()

    A, B = ints(-2, 2, M, K), ints(-2, 2, N, K)
    sa, sb = torch.exp2(ints(-2, 2, M, KB)), torch.exp2(ints(-2, 2, -(-N // block), KB))
    C = mh.mhlmoe_gemm_scaled(A.to(ref.E4M3), sa, B.to(ref.E4M3), sb, b_block_rows=block, dtype=dtype)
    a = ref.host(A) * ref.spread(ref.host(sa), A.shape, 1)
    b = ref.host(B) * ref.spread(ref.host(sb), B.shape, block)
    want = torch.from_numpy(a @ b.T).to(F32).to(dtype)
    off = np.argwhere(ref.host(C) != ref.host(want))
    assert off.size == 0, f"{len(off)} values, first {off[0]}"


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("M,N", [(5, 200), (12, 10300), (25, 300), (30, 8200), (28, 16400), (70, 200),
                                 (1100, 1040), (2310, 2050), (3600, 3401)])
@pytest.mark.parametrize("block", [128, 1])
def test_special_values_stay_where_they_are(M, N, block, dtype):
    """A NaN or an infinite scale of A reaches its row of C, one of B its
    column (its tile's columns), and nothing else."""
    announce(f"special values {M}x{N} block={block} {dtype}")
    K = 1296
    g = torch.Generator(device="cuda").manual_seed(M + N)
    A, sa = mh.mhlmoe_quantize(torch.randn(M, K, generator=g, device="cuda"))
    B, sb = mh.mhlmoe_quantize(torch.randn(N, K, generator=g, device="cuda"), block_rows=block)
    clean = mh.mhlmoe_gemm_scaled(A, sa, B, sb, b_block_rows=block, dtype=dtype)
    A.view(torch.uint8)[1, 1290] = 0x7F
    sa[3, 9] = float("inf")
    B.view(torch.uint8)[N - 1, 700] = 0x7F
    sb[0, 10] = float("nan")
    C = mh.mhlmoe_gemm_scaled(A, sa, B, sb, b_block_rows=block, dtype=dtype)
    finite = torch.isfinite(C)
    assert torch.isfinite(clean).all()
    want = torch.ones(M, N, dtype=torch.bool, device="cuda")
    want[[1, 3]] = False
    want[:, N - 1] = False
    want[:, :block] = False
    assert torch.equal(finite, want)
    assert torch.equal(C[want], clean[want])
