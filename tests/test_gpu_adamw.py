"""AdamW on the GPU, against plain 64-bit references (tests/training_ref.py, which
derives the tolerances)."""
import numpy as np
import pytest
import torch

import paper_2602_04870_amd as mh
from tests import training_ref as ref
from tests.gpu_util import announce, needs_gpu
from tests.test_gpu_scaled import _gen, _guarded, _randn

pytestmark = [pytest.mark.gpu, needs_gpu]

BF16, F32 = torch.bfloat16, torch.float32
LR, B1, B2, EPS = 3e-3, 0.9, 0.95, 1e-8


def _filled(values):
    t, ok = _guarded(tuple(values.shape), values.dtype)
    t.copy_(values)
    return t, ok


def _tensor(g, n, kind, grad_dtype, bits, i):
    """One tensor of n elements and the checks of the bytes around what is written."""
    p = _randn(g, n)
    size = 1e-3 * torch.exp(2 * _randn(g, -(-n // 100)).repeat_interleave(100)[:n])
    t, oks = {"weight_decay": 0.1 * (i % 2), "seed": 1000 + i}, []

    def put(name, v):
        t[name], ok = _filled(v)
        oks.append(ok)

    put("param", p if kind == "f32" else p.to(BF16))
    if kind == "master":
        put("master", p)
    t["grad"] = (size * _randn(g, n)).to(grad_dtype)
    m, root = size * _randn(g, n), size * (_randn(g, n).abs() + 0.1)
    if n > 300:
        m[130:256] = 0  # a block that is nearly all zero
        root[130:256] = 0
    if bits == 32:
        put("m", m)
        put("v", root.square())
    else:
        for name, v in (("m", m), ("v", root)):
            q, s = ref.blocks8(v)
            put(name, q)
            put(name + "_scale", s)
    return t, oks


def _states64(t):
    if "m_scale" in t:
        return ref.values8(t["m"], t["m_scale"]), ref.values8(t["v"], t["v_scale"]) ** 2
    return ref.host(t["m"]), ref.host(t["v"])


def _check(before, t, step, scale, what):
    p0, m0, v0, g = before
    p, m, v, ep, em, ev = ref.adamw64(p0, g * scale, m0, v0, LR, B1, B2, EPS, t["weight_decay"], step)
    # an 8-bit value times its scale is rounded, and the root's square twice more
    if "m_scale" in t:
        em = em + ref.U * np.abs(m0)
        ev = ev + 3 * ref.U * v0
    got = ref.host(t["master"] if "master" in t else t["param"])
    half = ref.HALF[t["param"].dtype] if "master" not in t else ref.U
    assert np.all(np.abs(got - p) <= ep + half * (np.abs(p) + ep)), what
    if "master" in t:
        assert torch.equal(t["param"], t["master"].to(BF16)), what
    if "m_scale" in t:
        um, uv = ref.random16(p.size, t["seed"], step)
        root = np.sqrt(v)
        off = np.where(v > 0, ev / np.maximum(2 * root, 1e-300), 0) + ref.U * root
        ref.check_random_blocks(ref.host(t["m"]), ref.host(t["m_scale"]), m, em, um, False, what)
        ref.check_random_blocks(ref.host(t["v"]), ref.host(t["v_scale"]), root, off, uv, True, what)
    else:
        assert np.all(np.abs(ref.host(t["m"]) - m) <= em + 1e-45), what
        assert np.all(np.abs(ref.host(t["v"]) - v) <= ev + 1e-45), what


SIZES = [1, 7, 8, 127, 128, 129, 1000, 2047, 2048, 2049, 4999, 70001]


@pytest.mark.parametrize("kind,grad_dtype", [("f32", F32), ("f32", BF16), ("master", F32), ("master", BF16),
                                             ("bf16", F32), ("bf16", BF16)])
@pytest.mark.parametrize("bits", [32, 8])
def test_adamw(kind, grad_dtype, bits):
    """Two steps over tensors of every tail, one call for all of them."""
    announce(f"adamw {kind} {grad_dtype} {bits}")
    g = _gen(bits + len(kind))
    made = [_tensor(g, n, kind, grad_dtype, bits, i) for i, n in enumerate(SIZES)]
    plan = mh.AdamWTensors([t for t, _ in made])
    scale = torch.full((1,), 0.7, device="cuda")
    for step in (1, 25):
        before = [(ref.host(t["master"] if "master" in t else t["param"]), *_states64(t),
                   ref.host(t["grad"])) for t, _ in made]
        mh.mhlmoe_adamw(plan, LR, beta1=B1, beta2=B2, eps=EPS, step=step, grad_scale=scale)
        torch.cuda.synchronize()
        for (t, oks), b in zip(made, before):
            for ok in oks:
                ok()
            _check(b, t, step, float(scale), f"{kind} {bits} n={t['param'].numel()} step={step}")


@pytest.mark.parametrize("n", [0, 1, 47, 48, 49, 130])
def test_adamw_many_tensors(n):
    """More tensors than one launch takes, empty ones among them, of mixed kinds."""
    g = _gen(n + 9)
    kinds = [("f32", F32, 32), ("master", F32, 8), ("bf16", BF16, 8), ("bf16", BF16, 32)]
    made = []
    for i in range(n):
        kind, gd, bits = kinds[i % 4]
        size = 0 if i % 5 == 4 else 3 + 37 * i
        made.append(_tensor(g, size, kind, gd, bits, i)[0])
    before = [(ref.host(t["master"] if "master" in t else t["param"]), *_states64(t), ref.host(t["grad"]))
              for t in made]
    mh.mhlmoe_adamw(made, LR, beta1=B1, beta2=B2, eps=EPS, step=3)
    torch.cuda.synchronize()
    for i, (t, b) in enumerate(zip(made, before)):
        _check(b, t, 3, 1.0, f"tensor {i}")


def test_adamw_same_bits_again_and_other_seeds():
    g = _gen(4)
    t, _ = _tensor(g, 5000, "bf16", BF16, 8, 0)
    runs = []
    for seed, step in ((7, 3), (7, 3), (8, 3), (7, 4)):
        c = {k: v.clone() if isinstance(v, torch.Tensor) else v for k, v in t.items()}
        c["seed"] = seed
        mh.mhlmoe_adamw([c], 0.0, step=step)
        runs.append(c["m"].view(torch.uint8))
    assert torch.equal(runs[0], runs[1])
    assert not torch.equal(runs[0], runs[2]) and not torch.equal(runs[0], runs[3])


def test_adamw_8_bit_states_move_by_the_update_on_average():
    """With the gradient 1 and m held in 8 bits next to one large value that fixes
    the scale, every step moves m by less than half a step of e4m3; over many
    elements its mean follows the 32-bit one.  A rounding is off by less than a step
    (2^-3 of the value) and by nothing on average: 30 steps over 1.2e5 elements,
    each error decayed after, stay below 6 of their deviations."""
    n, steps = 128 * 1000, 30
    m = torch.full((n,), 0.4, device="cuda")
    m[::128] = 1.0
    q, s = ref.blocks8(m)
    v, vs = ref.blocks8(torch.ones(n, device="cuda"))
    t = dict(param=torch.zeros(n, device="cuda"), grad=torch.ones(n, device="cuda"), m=q, v=v, m_scale=s,
             v_scale=vs)
    plan = mh.AdamWTensors([t])
    want = ref.values8(q, s)
    for i in range(steps):
        mh.mhlmoe_adamw(plan, 0.0, beta1=0.99, beta2=0.99, step=i + 1)
        want = 0.99 * want + 0.01
    rest = np.arange(n) % 128 != 0
    got = ref.values8(t["m"], t["m_scale"])[rest]
    sigma = 0.5 * 2.0 ** -3 * 1.0 * np.sqrt(steps / rest.sum())
    assert abs(got.mean() - want[rest].mean()) <= 6 * sigma
    assert abs(want[rest].mean() - 0.4) > 0.1  # to the nearest it would not have moved
    root = ref.values8(t["v"], t["v_scale"])
    assert np.all(root > 0)


def test_adamw_small_roots_do_not_become_zero():
    """An element whose v is far below its block's keeps the smallest value: its
    step stays below lr, but for m's own rounding (2^-3 at most), where with v = 0 in
    the state the second one would be a hundred times that."""
    n = 256
    root = torch.full((n,), 1e-6, device="cuda")
    root[::128] = 1.0
    v, vs = ref.blocks8(root)
    m, ms = ref.blocks8(torch.zeros(n, device="cuda"))
    t = dict(param=torch.zeros(n, device="cuda"), grad=torch.full((n,), 1e-6, device="cuda"), m=m, v=v,
             m_scale=ms, v_scale=vs)
    for i in range(1, 20):
        mh.mhlmoe_adamw([t], 1e-3, step=i)
    assert np.all(ref.host(t["v"]) > 0)
    assert float(t["param"].abs().max()) <= 19 * 1e-3 * (1 + 2.0 ** -3)


def test_adamw_not_finite_gradient_stays_in_its_block():
    g = _gen(12)
    t, _ = _tensor(g, 1000, "f32", F32, 8, 0)
    c = {k: v.clone() if isinstance(v, torch.Tensor) else v for k, v in t.items()}
    t["grad"][300] = float("nan")
    t["grad"][700] = float("inf")
    mh.mhlmoe_adamw([t], LR, step=2)
    mh.mhlmoe_adamw([c], LR, step=2)
    p, pc = ref.host(t["param"]), ref.host(c["param"])
    assert np.isnan(p[[300, 700]]).all()
    rest = np.ones(1000, bool)
    rest[[300, 700]] = False
    assert np.array_equal(p[rest], pc[rest])
    for key in ("m", "v"):
        a, b = ref.values8(t[key], t[key + "_scale"]), ref.values8(c[key], c[key + "_scale"])
        hit = np.isin(np.arange(1000) // 128, [300 // 128, 700 // 128])
        assert np.isnan(a[hit]).all() and np.array_equal(a[~hit], b[~hit])


def test_adamw_past_32_bits():
    """2^32 + 1000 bf16 elements with 8-bit states: addresses past 4 GiB, and the random
    numbers of elements past 2^32."""
    n = (1 << 32) + 1000
    announce(f"adamw n={n}")
    p = torch.zeros(n, dtype=BF16, device="cuda")
    grad = torch.full((n,), 1e-3, dtype=BF16, device="cuda")
    m = torch.zeros(n, dtype=torch.uint8, device="cuda").view(ref.E4M3)
    v = torch.zeros(n, dtype=torch.uint8, device="cuda").view(ref.E4M3)
    ms, vs = (torch.full((-(-n // 128),), ref.SCALE_MIN, device="cuda") for _ in range(2))
    t = dict(param=p, grad=grad, m=m, v=v, m_scale=ms, v_scale=vs, seed=5)
    mh.mhlmoe_adamw([t], LR, beta1=B1, beta2=B2, eps=EPS, step=1)
    torch.cuda.synchronize()
    for at, k in ((0, 4096), ((1 << 31) - 128, 4096), ((1 << 32) - 1024, 2024)):
        cut = slice(at, at + k)
        part = dict(t, param=p[cut], grad=grad[cut], m=m[cut], v=v[cut], weight_decay=0.0,
                    m_scale=ms[at // 128:-(-(at + k) // 128)], v_scale=vs[at // 128:-(-(at + k) // 128)])
        g64 = ref.host(part["grad"])
        p1, m1, v1, ep, em, ev = ref.adamw64(np.zeros(k), g64, np.zeros(k), np.zeros(k), LR, B1, B2, EPS,
                                             0.0, 1)
        assert np.all(np.abs(ref.host(part["param"]) - p1) <= ep + 2.0 ** -8 * np.abs(p1))
        um, uv = ref.random16(k, 5, 1, first=at)
        ref.check_random_blocks(ref.host(part["m"]), ref.host(part["m_scale"]), m1, em, um, False, f"m {at}")
        root = np.sqrt(v1)
        ref.check_random_blocks(ref.host(part["v"]), ref.host(part["v_scale"]), root, 5 * ref.U * root, uv,
                                True, f"v {at}")


def test_adamw_tensors_keep_the_memory_they_were_given():
    g = _gen(13)
    t, _ = _tensor(g, 1000, "f32", F32, 32, 0)
    c = {k: v.clone() if isinstance(v, torch.Tensor) else v for k, v in t.items()}
    plan = mh.AdamWTensors([t])
    was = t["param"].detach()
    t["param"].data = torch.zeros(1000, device="cuda")
    del t["grad"], t["m"], t["v"]
    torch.full((8192,), 7.0, device="cuda")  # where freed memory of theirs would be taken again
    mh.mhlmoe_adamw(plan, LR, step=3)
    mh.mhlmoe_adamw([c], LR, step=3)
    assert torch.equal(was, c["param"]) and not t["param"].any()
