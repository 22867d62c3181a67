"""The layer's inference forward with its experts in 4 bits: against the formula in 64 bits with the same quantisations, and around its
edges (few tokens, dropped slots, the projection-free layer, graphs)."""
import numpy as np
import pytest
import torch

import mx4_reference as ref
from oracle import margin
from paper_2502_16927_b200 import workloads as wl

from helpers import make_layer, to_device, to_numpy

pytestmark = pytest.mark.gpu


def _bf16(x):
    return torch.from_numpy(np.ascontiguousarray(x)).to(torch.bfloat16).double().numpy()


def _gelu(z):
    from scipy.special import erfc
    return 0.5 * z * erfc(-z / np.sqrt(2))


def _q(x):
    return ref.values(*ref.quantise(x))


def _formula(w, inp, R):
    """y from the routing that the call reports."""
    idx, p, rows = (to_numpy(R[n]).reshape(w.T, w.k) for n in ("topk_idx", "topk_w", "row_of_slot"))
    x = inp["x"].astype(np.float64)
    x_lo = x if w.cdac else _bf16(x @ inp["w_down"].astype(np.float64).T)
    xq = _q(x_lo)
    y_lo = np.zeros((w.T, w.r))
    for e in range(w.E):
        t, j = np.nonzero((idx == e) & (rows >= 0))
        if t.size:
            a = _q(_gelu(xq[t] @ _q(inp["w1"][e]).T))
            np.add.at(y_lo, t, p[t, j][:, None] * (a @ _q(inp["w2"][e]).T))
    return y_lo if w.cdac else y_lo @ inp["w_up"].astype(np.float64).T


def _setup(binding, w, **kw):
    inp = wl.make_inputs(w)
    margin.enforce_margin(w, inp, 1e-3)
    dev = to_device(w, inp)
    layer = make_layer(w, **kw)
    four = dict(dev, w1=binding.mx4_quantize_weights(dev["w1"]), w2=binding.mx4_quantize_weights(dev["w2"]))
    return inp, dev, layer, four


@pytest.fixture(scope="module")
def binding():
    from paper_2502_16927_b200 import binding as b

    return b


# u, y' and y are bf16: 2^-9 of a value's rms a store, and the gate values' and GELU's own errors are far below it; a code that falls on the other
# side of a border for a last-bit difference of its fp32 value moves one of r or h summands by a step, in about one of 10^4 codes: together within
# the 8e-3 that the layer's other bf16 results are held to
BOUND = 8e-3


@pytest.mark.parametrize("shape", [dict(T=1, d=256, r=64, h=128, E=8, k=2), dict(T=9, d=512, r=128, h=64, E=4, k=4), dict(T=100, d=256, r=64, h=192, E=12, k=3),
                                   dict(T=777, d=1024, r=128, h=512, E=32, k=4), dict(T=300, d=128, r=64, h=64, E=70, k=5), dict(T=64, d=2048, r=256, h=1024, E=64, k=8)])
def test_forward(binding, shape):
    w = wl.Workload("four", dtype=wl.DTYPE_BF16, act=wl.ACT_GELU_ERF, seed=61, **shape)
    inp, dev, layer, four = _setup(binding, w)
    y, R = layer.forward(dev["x"], four, want_routing=True)
    again = layer.forward(dev["x"], four)
    want = layer.route(dev["x"], dev)
    for name in ("topk_idx", "row_of_slot", "slot_of_row", "offsets", "counts"):
        assert torch.equal(R[name], want[name]), name
    assert torch.equal(y, again) and layer.status() == 0
    expect = _formula(w, inp, R)
    err = np.linalg.norm(to_numpy(y) - expect) / np.linalg.norm(expect)
    assert err <= BOUND, err
    layer.close()


def test_capacity_limit(binding):
    w = wl.Workload("four", T=400, d=256, r=64, h=128, E=8, k=2, dtype=wl.DTYPE_BF16, act=wl.ACT_GELU_ERF, seed=62)
    inp, dev, layer, four = _setup(binding, w, capacity_factor=0.6)
    y, R = layer.forward(dev["x"], four, want_routing=True)
    assert bool((R["row_of_slot"] < 0).any())
    expect = _formula(w, inp, R)
    assert np.linalg.norm(to_numpy(y) - expect) / np.linalg.norm(expect) <= BOUND
    layer.close()


def test_projection_free_layer(binding):
    w = wl.Workload("four", T=120, d=128, r=128, h=192, E=6, k=2, dtype=wl.DTYPE_BF16, act=wl.ACT_GELU_ERF, seed=63, cdac=True)
    inp, dev, layer, four = _setup(binding, w)
    y, R = layer.forward(dev["x"], four, want_routing=True)
    expect = _formula(w, inp, R)
    assert np.linalg.norm(to_numpy(y) - expect) / np.linalg.norm(expect) <= BOUND
    layer.close()


def test_captured_and_next_to_the_layer_s_own_forward(binding):
    w = wl.Workload("four", T=64, d=512, r=64, h=256, E=16, k=4, dtype=wl.DTYPE_BF16, act=wl.ACT_GELU_ERF, seed=64)
    inp, dev, layer, four = _setup(binding, w)
    before = layer.forward(dev["x"], dev)
    x, y = dev["x"].clone(), torch.empty_like(dev["x"])
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        layer.forward(x, four, y=y)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            layer.forward(x, four, y=y)
    torch.cuda.current_stream().wait_stream(side)
    for sign in (1, -1):
        x.copy_(dev["x"] * sign)
        graph.replay()
        assert torch.equal(y, layer.forward(x, four))
    assert torch.equal(before, layer.forward(dev["x"], dev))
    layer.close()


def test_refusals(binding):
    w = wl.Workload("four", T=16, d=128, r=64, h=128, E=4, k=2, dtype=wl.DTYPE_BF16, act=wl.ACT_RELU, seed=65)
    inp, dev, layer, four = _setup(binding, w)
    with pytest.raises(ValueError):
        layer.forward(dev["x"], four, training=True)
    with pytest.raises(ValueError):
        layer.forward(dev["x"], dict(four, w2=dev["w2"]))
    for bad in (dict(w1=four["w2"]), dict(w2=four["w1"]), dict(w1=binding.Mx4(four["w1"].codes[:2].contiguous(), four["w1"].scales[:2].contiguous()))):
        with pytest.raises(binding.BigmacError) as e:
            layer.forward(dev["x"], dict(four, **bad))
        assert e.value.status == -1
    scratch = torch.empty(256, dtype=torch.uint8, device="cuda")
    with pytest.raises(binding.BigmacError) as e:
        binding.bigmac_forward_mx4(layer.handle, dev["x"], w.T, {n: dev[n] for n in ("w_gate", "w_down", "w_up")}, four["w1"], four["w2"],
                                   torch.empty_like(dev["x"]), None, scratch)
    assert e.value.status == -3
    layer.close()
    for kw in (dict(dtype=wl.DTYPE_F32), dict(expert_bias=True)):
        import dataclasses
        other = make_layer(dataclasses.replace(w, **kw))
        with pytest.raises(binding.BigmacError) as e:
            binding.bigmac_mx4_workspace_bytes(other.handle, 4)
        assert e.value.status == -2
        other.close()
