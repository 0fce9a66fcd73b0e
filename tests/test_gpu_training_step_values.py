"""A whole training step's loss and updates against the plain 64-bit references
(tests/training_ref.py)."""
import numpy as np
import pytest
import torch

import paper_2602_04870_amd as mh
from tests import training_ref as ref
from tests.gpu_util import announce, needs_gpu
from tests.test_gpu_training_step import BF16, DH, EPS, K, NE, NH, Step, T

pytestmark = [pytest.mark.gpu, needs_gpu]

LR, B1, B2, ADAM_EPS = 1e-3, 0.9, 0.999, 1e-8  # of Step.run


def _states(t):
    if "m_scale" in t:
        return ref.values8(t["m"], t["m_scale"]), ref.values8(t["v"], t["v_scale"]) ** 2
    return ref.host(t["m"]).reshape(-1), ref.host(t["v"]).reshape(-1)


@pytest.mark.parametrize("bits", [32, 8])
def test_step_loss_and_updates(bits):
    """Two steps: the loss is the reference's for the tokens that count, and each tensor and its
    states are what AdamW makes of the step's gradient."""
    announce(f"training step's values bits={bits}")
    s = Step(11, bits)
    for step in (1, 2):
        p = s.p
        X = mh.mhlmoe_layernorm(s.x, p["norm_w"], EPS, bias=p["norm_b"])["y"].view(T, NH, DH)
        idx = mh.mhlmoe_layer(X, p["router"], None, p["W1"], p["W3"], p["W2"], K)[1]
        keep = s.mask.cpu().numpy()
        b = ref.Balance(ref.host(X), ref.host(p["router"]), ref.counts64(idx.cpu().numpy(), keep, NE), keep)
        before = [(ref.host(t.get("master", t["param"])).reshape(-1), *_states(t)) for t in s.tensors]
        loss = s.run(step)
        assert np.all(np.abs(ref.host(loss) - b.loss) <= b.e_loss)
        for i, (t, (p0, m0, v0)) in enumerate(zip(s.tensors, before)):
            what = f"tensor {i} step {step}"
            g = ref.host(t["grad"]).reshape(-1)
            assert g.any(), what
            p1, m, v, ep, em, ev = ref.adamw64(p0, g, m0, v0, LR, B1, B2, ADAM_EPS, t["weight_decay"], step)
            got = ref.host(t.get("master", t["param"])).reshape(-1)
            assert np.all(np.abs(got - p1) <= ep + ref.U * (np.abs(p1) + ep)), what
            if "master" in t:
                assert torch.equal(t["param"], t["master"].to(BF16)), what
            if "m_scale" not in t:
                # (a square below 2^-126 is off by a denormal number's last step besides)
                assert np.all(np.abs(ref.host(t["m"]).reshape(-1) - m) <= em + 2.0 ** -149), what
                assert np.all(np.abs(ref.host(t["v"]).reshape(-1) - v) <= ev + 2.0 ** -148), what
            else:
                em, ev = em + ref.U * np.abs(m0), ev + 3 * ref.U * v0
                um, uv = ref.random16(p1.size, i, step)
                root = np.sqrt(v)
                off = np.where(v > 0, ev / np.maximum(2 * root, 1e-300), 0) + ref.U * root
                ref.check_random_blocks(ref.host(t["m"]).reshape(-1), ref.host(t["m_scale"]), m, em, um, False, what)
                ref.check_random_blocks(ref.host(t["v"]).reshape(-1), ref.host(t["v_scale"]), root, off, uv, True, what)
