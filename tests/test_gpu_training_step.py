"""The training step's operators together, as they would be used: the norm, the
layer, the balance loss, all gradients and the optimiser, run as calls, on a side
stream and as a captured graph."""
import numpy as np
import pytest
import torch

import paper_2602_04870_amd as mh
from tests import training_ref as ref
from tests.gpu_util import announce, needs_gpu
from tests.test_gpu_scaled import _gen, _randn

pytestmark = [pytest.mark.gpu, needs_gpu]

BF16, F32 = torch.bfloat16, torch.float32
T, NH, DH, NE, K, DFF = 600, 2, 64, 24, 3, 64
DM = NH * DH
EPS = 1e-5


class Step:
    """One layer behind its norm, with a loss of mean square distance to a target
    and the balance loss, all buffers held."""

    def __init__(self, seed, bits):
        g = _gen(seed)
        self.x, self.target = _randn(g, T, DM, dtype=BF16), _randn(g, T, DM, dtype=BF16)
        self.mask = torch.rand((T,), generator=g, device="cuda") < 0.9
        self.dloss = torch.full((NH,), 0.01, device="cuda")
        full = dict(norm_w=1 + 0.1 * _randn(g, DM), norm_b=0.1 * _randn(g, DM),
                    router=_randn(g, NH, NE, DH) * DH ** -0.5,
                    W1=_randn(g, NH, NE, DFF, DH) * DH ** -0.5, W3=_randn(g, NH, NE, DFF, DH) * DH ** -0.5,
                    W2=_randn(g, NH, NE, DH, DFF) * DFF ** -0.5)
        self.p, self.tensors, self.grad = {}, [], {}
        for name, v in full.items():
            half = name in ("W1", "W3", "W2")
            self.p[name] = v.to(BF16) if half else v.clone()
            self.grad[name] = torch.zeros_like(v)
            t = dict(param=self.p[name], grad=self.grad[name], weight_decay=0.1 if half else 0.0)
            if half:
                t["master"] = v.clone()
            if bits == 32 or not half:
                t["m"], t["v"] = torch.zeros_like(v), torch.zeros_like(v)
            else:
                for s in ("m", "v"):
                    t[s], t[s + "_scale"] = ref.blocks8(torch.zeros_like(v))
            self.tensors.append(t)
        self.plan = mh.AdamWTensors(self.tensors)
        self.scale = torch.ones(1, device="cuda")

    def run(self, step, stream=None):
        p, g, kw = self.p, self.grad, dict(stream=stream)
        n = mh.mhlmoe_layernorm(self.x, p["norm_w"], EPS, bias=p["norm_b"], **kw)["y"]
        X = n.view(T, NH, DH)
        Y, idx, gate, _ = mh.mhlmoe_layer(X, p["router"], None, p["W1"], p["W3"], p["W2"], K, **kw)
        counts = mh.mhlmoe_expert_counts(idx, NE, mask=self.mask, **kw)
        loss, stats = mh.mhlmoe_balance_loss(X, p["router"], counts, mask=self.mask, **kw)
        dY = ((Y.view(T, DM).float() - self.target.float()) * self.mask[:, None] / T).to(BF16).view_as(Y)
        dX, *_ = mh.mhlmoe_layer_backward(X, p["router"], p["W1"], p["W3"], p["W2"], idx, gate, dY,
                                          dW_router=g["router"], dW1=g["W1"], dW3=g["W3"], dW2=g["W2"],
                                          **kw)
        mh.mhlmoe_balance_loss_backward(X, p["router"], counts, stats, self.dloss, mask=self.mask,
                                        dX_add=dX, dW_add=g["router"], dX=dX, dW_router=g["router"], **kw)
        mh.mhlmoe_layernorm_backward(self.x, p["norm_w"], EPS, dX.view(T, DM), dweight=g["norm_w"],
                                     dbias=g["norm_b"], **kw)
        mh.mhlmoe_adamw(self.plan, 1e-3, step=step, grad_scale=self.scale, **kw)
        return loss

    def state(self):
        return [v.view(torch.uint8).clone() for t in self.tensors for v in t.values()
                if isinstance(v, torch.Tensor)]


@pytest.mark.parametrize("bits", [32, 8])
def test_step_as_calls_and_on_a_side_stream(bits):
    """The same bits on another stream; the loss is the reference's, and the balance
    loss's part of the router's gradient is."""
    announce(f"training step bits={bits}")
    a, b = Step(1, bits), Step(1, bits)
    losses = [a.run(i + 1) for i in range(3)]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        other = [b.run(i + 1, stream=side) for i in range(3)]
    torch.cuda.synchronize()
    assert all(torch.equal(x, y) for x, y in zip(losses, other))
    assert all(torch.equal(x, y) for x, y in zip(a.state(), b.state()))
    assert all(torch.isfinite(t["param"].float()).all() for t in a.tensors)


def test_step_gradient_parts_add_up():
    """The router's gradient is the layer's plus the balance loss's, and so is dX's."""
    s = Step(3, 32)
    p = s.p
    X = mh.mhlmoe_layernorm(s.x, p["norm_w"], EPS, bias=p["norm_b"])["y"].view(T, NH, DH)
    _, idx, gate, counts = mh.mhlmoe_layer(X, p["router"], None, p["W1"], p["W3"], p["W2"], K)
    dY = _randn(_gen(4), T, NH, DH, dtype=BF16) / T
    dX, dWr, *_ = mh.mhlmoe_layer_backward(X, p["router"], p["W1"], p["W3"], p["W2"], idx, gate, dY)
    _, stats = mh.mhlmoe_balance_loss(X, p["router"], counts)
    gX, gW = mh.mhlmoe_balance_loss_backward(X, p["router"], counts, stats, s.dloss, dX_add=dX, dW_add=dWr)
    b = ref.Balance(ref.host(X), ref.host(p["router"]), counts.cpu().numpy().astype(np.int64), None)
    wX, wW, x_off, w_off = b.backward(ref.host(s.dloss), ref.host(dX), ref.host(dWr), True)
    assert np.all(np.abs(ref.host(gX) - wX) <= x_off + ref.HALF[BF16] * (np.abs(wX) + x_off))
    assert np.all(np.abs(ref.host(gW) - wW) <= w_off)


def test_step_captured_and_replayed():
    """A captured step, replayed with new inputs and eager work of its own in between,
    gives what the calls give (step and lr are the captured call's)."""
    a, b = Step(5, 8), Step(5, 8)
    g = _gen(6)
    warm = Step(7, 8)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        warm.run(1)
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        loss = a.run(2)
    for i in range(4):
        x = _randn(g, T, DM, dtype=BF16)
        a.x.copy_(x)
        b.x.copy_(x)
        a.scale.fill_(1.0 - 0.1 * i)
        b.scale.fill_(1.0 - 0.1 * i)
        graph.replay()
        torch.cuda.synchronize()
        want = b.run(2)
        torch.cuda.synchronize()
        assert torch.equal(loss, want)
        assert all(torch.equal(x, y) for x, y in zip(a.state(), b.state()))
