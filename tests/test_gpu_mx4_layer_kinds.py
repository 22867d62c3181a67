"""The layer's inference with 4-bit experts in its other forms: every activation, the gate on the low-width token, the balance loss."""
import numpy as np
import pytest
import torch

import mx4_reference as ref
from oracle import margin
from paper_2502_16927_b200 import workloads as wl

from helpers import make_layer, to_device, to_numpy
from test_gpu_mx4_layer import BOUND, _bf16, _q

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def binding():
    from paper_2502_16927_b200 import binding as b

    return b


def _act(z, act):
    if act == wl.ACT_RELU:
        return np.maximum(z, 0)
    if act == wl.ACT_GELU_ERF:
        from scipy.special import ndtr
        return z * ndtr(z)
    if act == wl.ACT_GELU_TANH:
        return 0.5 * z * (1 + np.tanh(np.sqrt(2 / np.pi) * (z + 0.044715 * z ** 3)))
    return z


def _check(binding, w, **kw):
    inp = wl.make_inputs(w)
    margin.enforce_margin(w, inp, 1e-3)
    dev = to_device(w, inp)
    layer = make_layer(w, **kw)
    four = dict(dev, w1=binding.mx4_quantize_weights(dev["w1"]), w2=binding.mx4_quantize_weights(dev["w2"]))
    y, R = layer.forward(dev["x"], four, want_routing=True)
    want = layer.route(dev["x"], dev)
    for name in ("topk_idx", "row_of_slot", "slot_of_row", "offsets", "counts", "counts_chosen"):
        assert torch.equal(R[name], want[name]), name
    # a routing call adds its logits up in another order: each of the two is off by at most a rounding a product (d or r of them) of sum |x w|,
    # which moves a gate value, and with all of them the balance loss, by as much four times over; a few roundings of the softmax on top
    src = inp["x"] if not w.gate_low else _bf16(inp["x"].astype(np.float64) @ inp["w_down"].astype(np.float64).T)
    off = (np.abs(src).astype(np.float64) @ np.abs(inp["w_gate"]).astype(np.float64).T).max() * (src.shape[1] + 2) * 2.0 ** -24
    for name in ("topk_w",) + (("aux_loss",) if kw else ()):
        a, b = to_numpy(R[name]), to_numpy(want[name])
        assert (np.abs(a - b) <= np.abs(b) * (4 * off + (64 if name == "topk_w" else 64 + w.T) * 2.0 ** -24)).all(), name
    idx, p, rows = (to_numpy(R[n]).reshape(w.T, w.k) for n in ("topk_idx", "topk_w", "row_of_slot"))
    xq = _q(_bf16(inp["x"].astype(np.float64) @ inp["w_down"].astype(np.float64).T))
    y_lo = np.zeros((w.T, w.r))
    for e in range(w.E):
        t, j = np.nonzero((idx == e) & (rows >= 0))
        if t.size:
            np.add.at(y_lo, t, p[t, j][:, None] * (_q(_act(xq[t] @ _q(inp["w1"][e]).T, w.act)) @ _q(inp["w2"][e]).T))
    expect = y_lo @ inp["w_up"].astype(np.float64).T
    assert np.linalg.norm(to_numpy(y) - expect) / np.linalg.norm(expect) <= BOUND
    assert layer.status() == 0
    layer.close()


@pytest.mark.parametrize("act", [wl.ACT_RELU, wl.ACT_GELU_TANH, wl.ACT_IDENTITY])
@pytest.mark.parametrize("T", [5, 300])
def test_activations(binding, act, T):
    _check(binding, wl.Workload("four", T=T, d=256, r=64, h=128, E=8, k=2, dtype=wl.DTYPE_BF16, act=act, seed=81))


@pytest.mark.parametrize("T", [7, 400])
def test_gate_on_the_low_width_token(binding, T):
    _check(binding, wl.Workload("four", T=T, d=256, r=64, h=128, E=8, k=2, dtype=wl.DTYPE_BF16, act=wl.ACT_GELU_ERF, seed=82, gate_low=True))


@pytest.mark.parametrize("T", [7, 400])
def test_balance_loss_and_capacity(binding, T):
    _check(binding, wl.Workload("four", T=T, d=256, r=64, h=128, E=8, k=2, dtype=wl.DTYPE_BF16, act=wl.ACT_GELU_ERF, seed=83), aux_loss_coef=0.01, capacity_factor=1.0)
