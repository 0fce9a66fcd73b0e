"""The training step's operators on the CPU: what their entry points and the
binding refuse before anything reaches a GPU, workspace sizes, struct layouts,
and the ABI's host code under sanitizers."""
import ctypes
import os
import re
import shutil
import subprocess

import pytest
import torch

import paper_2602_04870_amd as m
from tests.test_scaled_abi import (A, BAD, BF, BIG, CSRC, EINVAL, EUNSUP, EWS, F32, OK, ROOT, SAN,
                                   _refuses)


@pytest.fixture(scope="module")
def lib():
    return m.load_library()


def test_layernorm_refusals(lib):
    # x, residual, weight, bias, T, d, eps, dtype, sum, y, q, scales, stream
    good = [A, A, A, A, 4, 64, 1e-6, BF, A + 4096, A + 8192, A + 16384, A + 32768, None]
    _refuses(lib.mhlmoe_layernorm, good, [
        (0, None, EINVAL, "x"), (0, BAD, EINVAL, "x"), (1, BAD, EINVAL, "residual"),
        (2, None, EINVAL, "weight"), (3, BAD, EINVAL, "bias"), (4, -1, EINVAL, "T"),
        (4, 1 << 31, EUNSUP, "T"), (5, 0, EUNSUP, "d_model"), (5, 65537, EUNSUP, "d_model"),
        (5, 72, EUNSUP, "72"), (6, 0.0, EINVAL, "eps"), (6, float("nan"), EINVAL, "eps"),
        (6, float("inf"), EINVAL, "eps"), (6, -1.0, EINVAL, "eps"), (7, 7, EINVAL, "dtype"),
        (8, None, EINVAL, "sum"), (1, None, EINVAL, "residual"), (9, BAD, EINVAL, "y"),
        (10, None, EINVAL, "q is NULL"), (11, None, EINVAL, "scales"),
        ((9, 10, 11), (None, None, None), EINVAL, "both"), (9, A + 4096, EINVAL, "y must not")])


def test_layernorm_backward_refusals(lib):
    # h, weight, dy, dsum, T, d, eps, dtype, dx, dweight, dbias, ws, bytes, stream
    good = [A, A, A + 64, A, 4, 64, 1e-6, BF, A + 4096, A + 8192, A + 16384, A, BIG, None]
    _refuses(lib.mhlmoe_layernorm_backward, good, [
        (0, None, EINVAL, "h"), (1, None, EINVAL, "weight"), (2, None, EINVAL, "dy"),
        (3, BAD, EINVAL, "dsum"), (4, -1, EINVAL, "T"), (5, 65537, EUNSUP, "d_model"),
        (6, 0.0, EINVAL, "eps"), (7, 2, EINVAL, "dtype"), (8, None, EINVAL, "dx"),
        (8, A, EINVAL, "dx must not"), (9, None, EINVAL, "dweight"), (10, BAD, EINVAL, "dbias"),
        (10, A + 8192, EINVAL, "dbias must not"), (11, None, EWS, "NULL"), (11, A + 16, EINVAL, "256"),
        (12, 16, EWS, "need")])
    assert lib.mhlmoe_layernorm_backward_workspace(4, 64, None) == EINVAL
    for d in (1, 64, 1001, 4096, 65536):
        sizes = [m.mhlmoe_layernorm_backward_workspace(T, d) for T in (1, 100, 10000, 1 << 20)]
        assert sizes == sorted(sizes) and sizes[0] >= 8 * d


def test_counts_refusals(lib):
    # idx, mask, T, Nh, Ne, k, counts, stream
    good = [A, A, 4, 2, 8, 2, A, None]
    _refuses(lib.mhlmoe_expert_counts, good, [
        (0, None, EINVAL, "idx"), (1, A + 1, EINVAL, "mask"), (2, -1, EINVAL, "T"),
        (2, 1 << 30, EUNSUP, "top_k"), (3, 0, EINVAL, "n_heads"), (3, 1025, EUNSUP, "n_heads"),
        (4, 0, EINVAL, "n_experts"), (4, 1025, EUNSUP, "1025"), (5, 0, EINVAL, "top_k"),
        (5, 33, EUNSUP, "top_k"), (6, None, EINVAL, "counts"), (6, BAD, EINVAL, "counts")])


def test_balance_refusals(lib):
    # X, W, counts, mask, T, Nh, dh, Ne, dtype, loss, stats, ws, bytes, stream
    good = [A, A, A, A, 4, 2, 64, 8, BF, A, A, A, BIG, None]
    _refuses(lib.mhlmoe_balance_loss, good, [
        (0, None, EINVAL, "X"), (1, None, EINVAL, "W_router"), (2, None, EINVAL, "counts"),
        (3, BAD, EINVAL, "mask"), (4, -1, EINVAL, "T"), (4, 1 << 30, EUNSUP, "T"),
        (5, 0, EINVAL, "n_heads"), (6, 96, EUNSUP, "d_head"), (7, 1025, EUNSUP, "n_experts"),
        (8, 3, EINVAL, "dtype"), (9, None, EINVAL, "loss"), (10, None, EINVAL, "stats"),
        (10, BAD, EINVAL, "stats"), (11, None, EWS, "NULL"), (12, 64, EWS, "need")])
    # X, W, counts, stats, dloss, mask, dX_add, dW_add, T, Nh, dh, Ne, dtype, dX, dW, ws, bytes, stream
    good = [A, A, A, A, A, A, A, A, 4, 2, 64, 8, F32, A + 4096, A + 4096, A, BIG, None]
    _refuses(lib.mhlmoe_balance_loss_backward, good, [
        (0, None, EINVAL, "X"), (1, None, EINVAL, "W_router"), (2, None, EINVAL, "counts"),
        (3, None, EINVAL, "stats"), (4, None, EINVAL, "dloss"), (5, BAD, EINVAL, "mask"),
        (6, BAD, EINVAL, "dX_add"), (7, BAD, EINVAL, "dW_add"), (8, -1, EINVAL, "T"),
        (10, 32, EUNSUP, "d_head"), (12, 9, EINVAL, "dtype"), (13, None, EINVAL, "dX"),
        (13, A, EINVAL, "dX must not"), (14, None, EINVAL, "dW_router"),
        (14, A, EINVAL, "dW_router must not"), (15, A + 16, EINVAL, "256"), (16, 64, EWS, "need")])
    for f in (lib.mhlmoe_balance_loss_workspace, lib.mhlmoe_balance_loss_backward_workspace):
        assert f(4, 2, 64, 8, None) == EINVAL


def _tensor(**kw):
    t = dict(param=A, master=None, grad=A << 4, m=A << 5, v=A << 6, m_scale=None, v_scale=None, n=100,
             weight_decay=0.1, seed=1, param_dtype=F32, grad_dtype=F32)
    t.update(kw)
    c = m._AdamWTensor()
    for k, v in t.items():
        setattr(c, k, v)
    return c


def _step(**kw):
    s = dict(lr=1e-3, beta1=0.9, beta2=0.99, eps=1e-8, step=1, grad_scale=None)
    s.update(kw)
    return m._AdamWStep(*s.values())


def _adamw(lib, tensors, step):
    arr = (m._AdamWTensor * max(len(tensors), 1))(*tensors)
    return lib.mhlmoe_adamw(ctypes.addressof(arr), len(tensors), ctypes.addressof(step), None)


def test_adamw_refusals(lib):
    def refused(status, word, tensors, **step):
        assert _adamw(lib, tensors, _step(**step)) == status, m.mhlmoe_last_error()
        assert word in m.mhlmoe_last_error(), m.mhlmoe_last_error()

    good = _tensor()
    for kw, word in ((dict(lr=-1.0), "lr"), (dict(lr=float("nan")), "lr"), (dict(beta1=1.0), "beta1"),
                     (dict(beta1=-0.1), "beta1"), (dict(beta2=float("nan")), "beta2"),
                     (dict(eps=0.0), "eps"), (dict(eps=1e-60), "eps"), (dict(eps=float("inf")), "eps"),
                     (dict(step=0), "step"), (dict(grad_scale=A + 2), "grad_scale")):
        refused(EINVAL, word, [good], **kw)
    for kw, word in ((dict(param=None), "param"), (dict(param=BAD), "param"), (dict(grad=None), "grad"),
                     (dict(m=None), "m is NULL"), (dict(v=BAD << 1), "v is not"), (dict(n=-1), "n must"),
                     (dict(weight_decay=-1.0), "weight_decay"), (dict(param_dtype=4), "param_dtype"),
                     (dict(grad_dtype=-1), "grad_dtype"), (dict(master=A << 7), "master"),
                     (dict(m_scale=A << 8), "v_scale"), (dict(v_scale=A << 8), "m_scale"),
                     # memory that is written must be its own: a state that is the gradient, a
                     # parameter that reaches into its state, states that are one
                     (dict(m=A << 4), "overlaps"), (dict(v=A + 384), "overlaps"),
                     (dict(v=A << 5), "overlaps")):
        refused(EINVAL, word, [_tensor(**kw)])
    other = _tensor(param=A << 9, m=A << 10, v=A << 11)
    refused(EINVAL, "overlaps", [good, other, good])  # the same tensor twice
    refused(EINVAL, "overlaps", [good, _tensor(param=A << 9, m=A << 10, v=(A << 5) + 256)])
    refused(EINVAL, "overlaps", [good], grad_scale=A + 396)
    assert lib.mhlmoe_adamw(None, 1, ctypes.addressof(_step()), None) == EINVAL
    assert lib.mhlmoe_adamw(None, -1, ctypes.addressof(_step()), None) == EINVAL
    assert lib.mhlmoe_adamw(None, 0, None, None) == EINVAL
    assert _adamw(lib, [], _step()) == OK
    assert _adamw(lib, [_tensor(n=0, param=None, grad=None, m=None, v=None)], _step()) == OK


def test_binding_refuses():
    x, w = torch.zeros(4, 64, dtype=torch.bfloat16), torch.zeros(64)
    with pytest.raises(ValueError, match="GPU"):
        m.mhlmoe_layernorm(x, w, 1e-6)
    with pytest.raises(ValueError, match="dimensions"):
        m.mhlmoe_layernorm(x[0], w, 1e-6)
    with pytest.raises(ValueError, match="quantized"):
        m.mhlmoe_layernorm(x, w, 1e-6, q=torch.zeros(4, 64).to(m.E4M3))
    with pytest.raises(ValueError, match="GPU"):
        m.mhlmoe_layernorm_backward(x, w, 1e-6, x)
    big = torch.empty(0, (1 << 32) + 64, dtype=torch.bfloat16)
    with pytest.raises(ValueError, match="d_model must fit"):
        m.mhlmoe_layernorm(big, w, 1e-6)
    with pytest.raises(ValueError, match="d_model must fit"):
        m.mhlmoe_layernorm_backward_workspace(4, (1 << 32) + 64)
    idx = torch.zeros(4, 2, 3, dtype=torch.int32)
    with pytest.raises(ValueError, match="GPU"):
        m.mhlmoe_expert_counts(idx, 8)
    with pytest.raises(ValueError, match="3 dimensions"):
        m.mhlmoe_expert_counts(idx[0], 8)
    with pytest.raises(ValueError, match="n_experts"):
        m.mhlmoe_expert_counts(idx, -1)
    with pytest.raises(ValueError, match="n_experts must fit"):
        m.mhlmoe_expert_counts(idx, (1 << 32) + 8)
    X, W, c = torch.zeros(4, 2, 64), torch.zeros(2, 8, 64), torch.zeros(2, 8, dtype=torch.int32)
    with pytest.raises(ValueError, match="GPU"):
        m.mhlmoe_balance_loss(X, W, c)
    with pytest.raises(ValueError, match="GPU"):
        m.mhlmoe_balance_loss_backward(X, W, c, torch.zeros(5, 2, 2), torch.zeros(2))
    for f in (m.mhlmoe_balance_loss_workspace, m.mhlmoe_balance_loss_backward_workspace):
        for at, name in ((1, "n_heads"), (2, "d_head"), (3, "n_experts")):
            args = [4, 2, 64, 8]
            args[at] += 1 << 32
            with pytest.raises(ValueError, match=f"{name} must fit"):
                f(*args)


def test_adamw_binding_refuses():
    p = torch.zeros(4, 5)
    good = dict(param=p, grad=p.clone(), m=p.clone(), v=p.clone())
    with pytest.raises(ValueError, match="tensor 0: param must be a GPU"):
        m.AdamWTensors([good])
    with pytest.raises(TypeError, match="tensor 0: grad"):
        m.AdamWTensors([dict(good, grad=None)])
    with pytest.raises(ValueError, match="unknown momentum"):
        m.AdamWTensors([dict(good, momentum=1)])
    with pytest.raises(TypeError, match="float64"):
        m.AdamWTensors([dict(good, param=p.double())])
    assert m.AdamWTensors([]).device is None
    assert m.mhlmoe_adamw([], 1e-3, step=1) is None


def test_kernel_names_are_declared():
    """Every kernel these entry points time is named in the header."""
    header = open(m.HEADER).read()
    names = re.findall(r'run_kernel\("(\w+)"', open(os.path.join(CSRC, "api_training.cpp")).read())
    assert len(set(names)) == 11
    for name in names:
        assert f'"{name}"' in header, name


def test_host_code_under_sanitizers(tmp_path):
    """api_training.cpp and api.cpp built by g++ with their launchers replaced by stubs
    that abort (AdamW's looks its arguments over): no overflow, the production
    library's workspace sizes, and the binding's struct layouts."""
    gxx = shutil.which("g++")
    if gxx is None:
        pytest.skip("no g++")
    stubs = tmp_path / "stubs.cpp"
    body = ["#include <cstdlib>", '#include "training_launch.hpp"', "namespace mhl {"]
    for header in ("launch.hpp", "scaled_launch.hpp", "training_launch.hpp"):
        text = open(os.path.join(CSRC, header)).read()
        for name, params in re.findall(r"^hipError_t\s+(\w+)\(([^;{]*)\);", text, flags=re.M):
            if name != "launch_adamw":
                body.append(f"hipError_t {name}({params}) {{ std::abort(); }}")
    stubs.write_text("\n".join(body + ["}"]) + "\n")
    exe = str(tmp_path / "training_abi_check")
    cmd = [gxx, "-std=c++17", *SAN, "-D__HIP_PLATFORM_AMD__", "-I/opt/rocm/include",
           f"-I{ROOT}/include", f"-I{CSRC}", "-Wno-unused-result", "-Wno-unused-value",
           "-Wno-attributes", os.path.join(CSRC, "api.cpp"), os.path.join(CSRC, "api_training.cpp"),
           str(stubs), os.path.join(ROOT, "tests", "training_abi_check.cpp"), "-L/opt/rocm/lib",
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
    fns = {"norm": lib.mhlmoe_layernorm_backward_workspace, "loss": lib.mhlmoe_balance_loss_workspace,
           "back": lib.mhlmoe_balance_loss_backward_workspace}
    for line in res.stdout.splitlines():
        kind, *v = line.split()
        if kind == "struct":
            s = {"tensor": m._AdamWTensor, "step": m._AdamWStep}[v[0]]
            assert [int(i) for i in v[1:]] == [ctypes.sizeof(s)] + [getattr(s, f[0]).offset
                                                                    for f in s._fields_], line
            n += 1
        elif kind in fns:
            v = [int(i) for i in v]
            b = ctypes.c_size_t(0)
            assert fns[kind](*v[:-2], ctypes.byref(b)) == v[-2], line
            assert v[-2] != OK or b.value == v[-1], line
            n += 1
    assert n > 1000
