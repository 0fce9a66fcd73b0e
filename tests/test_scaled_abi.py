"""The operators around the heads on the CPU: what their entry points refuse
before anything reaches a GPU, workspace sizes, and the ABI's host code under
sanitizers."""
import ctypes
import os
import re
import shutil
import subprocess

import pytest
import torch

import paper_2602_04870_amd as m

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_2602_04870_amd", "csrc")
A, BAD, OK = 0x10000, 0x10004, m.MHLMOE_OK  # an aligned address, a misaligned one; never read
EINVAL, EUNSUP, EWS = m.MHLMOE_EINVAL, m.MHLMOE_EUNSUPPORTED, m.MHLMOE_EWORKSPACE
BF, F32 = m.MHLMOE_BF16, m.MHLMOE_F32
BIG = 1 << 40


@pytest.fixture(scope="module")
def lib():
    return m.load_library()


def _refuses(fn, good, changes):
    """Each change of `good` gives its status and names the argument."""
    for at, value, status, word in changes:
        args = list(good)
        for i, v in zip(at if isinstance(at, tuple) else (at,),
                        value if isinstance(value, tuple) else (value,)):
            args[i] = v
        assert fn(*args) == status, (at, value, m.mhlmoe_last_error())
        assert word in m.mhlmoe_last_error(), (word, m.mhlmoe_last_error())


def test_rmsnorm_refusals(lib):
    # x, residual, weight, T, d, eps, dtype, sum, y, q, scales, stream
    good = [A, A, A, 4, 64, 1e-6, BF, A + 4096, A + 8192, A + 16384, A + 32768, None]
    _refuses(lib.mhlmoe_rmsnorm, good, [
        (0, None, EINVAL, "x"), (0, BAD, EINVAL, "x"), (1, BAD, EINVAL, "residual"),
        (2, None, EINVAL, "weight"), (3, -1, EINVAL, "T"), (3, 1 << 31, EUNSUP, "T"),
        (4, 0, EUNSUP, "d_model"), (4, 65537, EUNSUP, "d_model"), (4, 72, EUNSUP, "72"),
        (5, 0.0, EINVAL, "eps"), (5, float("nan"), EINVAL, "eps"), (5, float("inf"), EINVAL, "eps"),
        (5, -1.0, EINVAL, "eps"), (6, 7, EINVAL, "dtype"), (7, None, EINVAL, "sum"),
        (1, None, EINVAL, "residual"), (8, BAD, EINVAL, "y"), (9, None, EINVAL, "q is NULL"),
        (10, None, EINVAL, "scales"), ((8, 9, 10), (None, None, None), EINVAL, "both"),
        (8, A + 4096, EINVAL, "y must not")])


def test_rmsnorm_backward_refusals(lib):
    # h, weight, dy, dsum, T, d, eps, dtype, dx, dweight, ws, bytes, stream
    good = [A, A, A + 64, A, 4, 64, 1e-6, BF, A + 4096, A + 8192, A, BIG, None]
    _refuses(lib.mhlmoe_rmsnorm_backward, good, [
        (0, None, EINVAL, "h"), (1, None, EINVAL, "weight"), (2, None, EINVAL, "dy"),
        (3, BAD, EINVAL, "dsum"), (4, -1, EINVAL, "T"), (5, 65537, EUNSUP, "d_model"),
        (6, 0.0, EINVAL, "eps"), (7, 2, EINVAL, "dtype"), (8, None, EINVAL, "dx"),
        (8, A, EINVAL, "dx must not"), (9, None, EINVAL, "dweight"), (10, None, EWS, "NULL"),
        (10, A + 16, EINVAL, "256"), (11, 16, EWS, "need")])


def test_rmsnorm_backward_workspace_sizes(lib):
    with pytest.raises(m.MhlmoeError):
        m.mhlmoe_rmsnorm_backward_workspace(-1, 64)
    assert lib.mhlmoe_rmsnorm_backward_workspace(4, 64, None) == EINVAL
    assert m.mhlmoe_rmsnorm_backward_workspace(0, 64) == 0
    for d in (1, 64, 1001, 4096, 65536):
        sizes = [m.mhlmoe_rmsnorm_backward_workspace(T, d) for T in (1, 100, 10000, 1 << 20)]
        assert sizes == sorted(sizes) and sizes[0] >= 4 * d


def test_quantize_refusals(lib):
    # x, rows, cols, dtype, block_rows, transpose, q, scales, stream
    good = [A, 4, 64, BF, 1, 0, A, A, None]
    _refuses(lib.mhlmoe_quantize, good, [
        (0, None, EINVAL, "x"), (0, BAD, EINVAL, "x"), (1, -1, EINVAL, "rows"),
        (2, -16, EINVAL, "cols"), (2, 24, EUNSUP, "24"), (1, 1 << 31, EUNSUP, "large"),
        (2, 1 << 31, EUNSUP, "large"), ((1, 2), (1 << 30, 1 << 30), EUNSUP, "large"),
        ((1, 2, 4), (1 << 20, 1 << 20, 128), EUNSUP, "large"), (3, 9, EINVAL, "dtype"),
        (4, 64, EINVAL, "block_rows"), (5, 2, EINVAL, "transpose"), (6, None, EINVAL, "q"),
        (7, BAD, EINVAL, "scales")])
    assert lib.mhlmoe_quantize(None, 0, 64, BF, 1, 0, None, None, None) == OK


def test_gemm_refusals(lib):
    # A, scale_a, B, scale_b, M, N, K, b_block_rows, dtype, C, stream
    good = [A, A, A, A, 4, 64, 128, 128, BF, A, None]
    _refuses(lib.mhlmoe_gemm_scaled, good, [
        (0, None, EINVAL, "A"), (1, None, EINVAL, "scale_a"), (2, BAD, EINVAL, "B"),
        (3, None, EINVAL, "scale_b"), (4, -1, EINVAL, "M"), (5, -1, EINVAL, "N"),
        (6, 24, EUNSUP, "16"), (6, -16, EINVAL, "K"), (7, 64, EINVAL, "b_block_rows"),
        (8, 5, EINVAL, "dtype"), (9, None, EINVAL, "C"), (4, 1 << 31, EUNSUP, "large"),
        (6, 1 << 24, EUNSUP, "large"), ((4, 5), (1 << 25, 1 << 25), EUNSUP, "large")])
    assert lib.mhlmoe_gemm_scaled(None, None, None, None, 0, 0, 128, 128, BF, None, None) == OK


def test_latent_layer_scaled_refusals(lib):
    # x, residual, norm_weight, eps, W_in, scale_in, W_r, scale_r, W_router, bias, W1, W3, W2,
    # W_out, scale_out, T, dm, Nh, dh, Ne, k, dff, dtype, out, sum, X, R, Y, idx, gate, counts, ws
    good = ([A, A, A, 1e-6] + [A] * 11 + [4, 64, 2, 64, 8, 2, 64, BF] + [A] * 8 + [A, BIG, None])
    _refuses(lib.mhlmoe_latent_layer_scaled, good, [
        (0, None, EINVAL, "x"), (1, None, EINVAL, "residual"), (2, None, EINVAL, "norm_weight"),
        (3, 0.0, EINVAL, "eps"), (4, None, EINVAL, "W_in"), (5, None, EINVAL, "scale_in"),
        (7, None, EINVAL, "scale_r"), (8, None, EINVAL, "W_router"), (10, None, EINVAL, "W1"),
        (12, BAD, EINVAL, "W2"), (13, None, EINVAL, "W_out"), (14, None, EINVAL, "scale_out"),
        (15, -1, EINVAL, "T"), (16, 72, EUNSUP, "d_model"), (18, 96, EUNSUP, "d_head"),
        (20, 9, EINVAL, "top_k"), (21, 48, EUNSUP, "d_ff"), (22, 5, EINVAL, "dtype"),
        (23, None, EINVAL, "out"), (24, None, EINVAL, "sum"), (28, BAD, EINVAL, "idx"),
        (31, None, EWS, "NULL"), (32, 64, EWS, "need")])
    a = m.mhlmoe_latent_layer_scaled_workspace(100, 512, 4, 128, 16, 2, 128)
    assert a > m.mhlmoe_workspace_size(m.MHLMOE_OP_LAYER, 100, 4, 128, 16, 2, 128)
    with pytest.raises(m.MhlmoeError):
        m.mhlmoe_latent_layer_scaled_workspace(100, 520, 4, 128, 16, 2, 128)


def test_binding_refuses():
    x, w = torch.zeros(4, 64, dtype=torch.bfloat16), torch.zeros(64)
    with pytest.raises(ValueError, match="GPU"):
        m.mhlmoe_rmsnorm(x, w, 1e-6)
    with pytest.raises(ValueError, match="dimensions"):
        m.mhlmoe_rmsnorm(x[0], w, 1e-6)
    with pytest.raises(TypeError):
        m.mhlmoe_rmsnorm(x.half(), w, 1e-6)
    with pytest.raises(ValueError, match="quantized"):
        m.mhlmoe_rmsnorm(x, w, 1e-6, q=torch.zeros(4, 64).to(m.E4M3))
    with pytest.raises(ValueError, match="GPU"):
        m.mhlmoe_quantize(x)
    with pytest.raises(TypeError, match="Tensor"):
        m.mhlmoe_gemm_scaled(None, w, x, w)


def test_binding_refuses_another_device_s_stream():
    class Stream:
        device_index, cuda_stream = 1, 0

    with pytest.raises(ValueError, match="stream is on GPU 1, the tensors are on 0"):
        m._launch(0, Stream(), lambda *a: pytest.fail("launched"))


def test_names_of_the_product_are_declared():
    """Every kernel the scaled entry points time is named in the header."""
    header = open(m.HEADER).read()
    api = open(os.path.join(CSRC, "api_scaled.cpp")).read()
    for name in re.findall(r'run_(?:kernel|gemm)\("(\w+)"', api):
        assert f'"{name}"' in header, name


def test_product_kernels_issue_no_tracked_dma():
    """The product's LDS DMA writes m0 without the compiler's knowledge, so its
    kernels issue no DMA that the compiler tracks."""
    text = open(os.path.join(CSRC, "gemm_scaled.hip")).read()
    assert text.count("offen lds") == 2
    assert "load_lds" not in text and "dma_lds16(" not in re.sub(r"//[^\n]*", "", text)
    # and nothing is in flight when the tiles' LDS is used for the results
    assert text.index("barrier_vm<0>();  // the last blocks' DMA") < text.index("turn = smem")


SAN = ["-O1", "-g", "-fsanitize=address,undefined", "-fno-sanitize-recover=all"]


def test_host_code_under_sanitizers(tmp_path):
    """api_scaled.cpp and api.cpp built by g++ with their launchers replaced by
    stubs that abort: the argument walks above, and the largest sizes, with no
    overflow, and the production library's workspace sizes."""
    gxx = shutil.which("g++")
    if gxx is None:
        pytest.skip("no g++")
    stubs = tmp_path / "stubs.cpp"
    body = ['#include <cstdlib>', '#include "scaled_launch.hpp"', "namespace mhl {"]
    for header in ("launch.hpp", "scaled_launch.hpp"):
        text = open(os.path.join(CSRC, header)).read()
        for name, params in re.findall(r"^hipError_t\s+(\w+)\(([^;{]*)\);", text, flags=re.M):
            body.append(f"hipError_t {name}({params}) {{ std::abort(); }}")
    stubs.write_text("\n".join(body + ["}"]) + "\n")
    exe = str(tmp_path / "scaled_abi_check")
    cmd = [gxx, "-std=c++17", *SAN, "-D__HIP_PLATFORM_AMD__", "-I/opt/rocm/include",
           f"-I{ROOT}/include", f"-I{CSRC}", "-Wno-unused-result", "-Wno-unused-value",
           "-Wno-attributes", os.path.join(CSRC, "api.cpp"), os.path.join(CSRC, "api_scaled.cpp"),
           str(stubs), os.path.join(ROOT, "tests", "scaled_abi_check.cpp"), "-L/opt/rocm/lib",
           "-lamdhip64", "-Wl,-rpath,/opt/rocm/lib", "-o", exe]
    res = subprocess.run(cmd, capture_output=True, text=True, timeout=600)
    assert res.returncode == 0, res.stderr[-4000:]
    res = subprocess.run([exe], capture_output=True, text=True, timeout=300,
                         env=dict(os.environ, ASAN_OPTIONS="detect_leaks=0",
                                  UBSAN_OPTIONS="halt_on_error=1:print_stacktrace=1"))
    out = res.stdout + res.stderr
    assert res.returncode == 0 and "done 0 failures" in res.stdout, out[-4000:]
    assert "runtime error" not in out, out[-4000:]
    lib, n = m.load_library(), 0
    for line in res.stdout.splitlines():
        kind, *v = line.split()
        if kind not in ("norm", "latent"):
            continue
        v = [int(i) for i in v]
        b = ctypes.c_size_t(0)
        fn = (lib.mhlmoe_rmsnorm_backward_workspace if kind == "norm"
              else lib.mhlmoe_latent_layer_scaled_workspace)
        assert fn(*v[:-2], ctypes.byref(b)) == v[-2], line
        assert v[-2] != OK or b.value == v[-1], line
        n += 1
    assert n > 50
