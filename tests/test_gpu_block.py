"""The layer as a residual block (binding.Block): a run of the joint before, the layer and the joint behind, as a network uses them."""
import numpy as np
import pytest
import torch

from paper_2502_16927_b200 import workloads as wl

from helpers import empty_grads, make_layer, to_device

pytestmark = pytest.mark.gpu


def _block(dtype, T=300, seed=71):
    from paper_2502_16927_b200 import binding

    w = (wl.Workload("b", T=T, d=128, r=32, h=64, E=8, k=2, dtype=dtype, act=wl.ACT_GELU_ERF, seed=seed) if dtype == wl.DTYPE_F32 else
         wl.Workload("b", T=T, d=256, r=64, h=128, E=8, k=2, dtype=dtype, act=wl.ACT_GELU_ERF, seed=seed))
    dev = to_device(w, wl.make_inputs(w))
    g = torch.Generator(device="cuda").manual_seed(seed)
    v = lambda mean: torch.randn(w.d, generator=g, device="cuda") * 0.2 + mean
    layer = make_layer(w)
    block = binding.Block(layer, binding.Norm(binding.BIGMAC_NORM_RMS, v(1.0)), binding.Norm(binding.BIGMAC_NORM_LAYER, v(1.0), v(0.0)), gate=v(0.5), residual_scale=0.8)
    return binding, w, dev, layer, block


def _grads(w, dev):
    G = empty_grads(w, dev)
    G.update({n: torch.empty(w.d, device="cuda") for n in ("dw_pre", "dw_post", "db_post", "dgate")})
    return G


@pytest.mark.parametrize("dtype", [wl.DTYPE_F32, wl.DTYPE_BF16])
def test_block_is_its_parts(dtype):
    """Forward and backward against the chain written out with the same layer and norms in 64 bits around it."""
    binding, w, dev, layer, block = _block(dtype)
    x, dout = dev["x"], dev["dy"]
    out = block.forward(x, dev, training=True)
    G = _grads(w, dev)
    dx = block.backward(dout, dev, G)

    f = lambda t: t.double().requires_grad_()
    x64, wp, wq, bq, gate = f(x), f(block.pre.weight), f(block.post.weight), f(block.post.bias), f(block.gate)
    n64 = x64 / torch.sqrt((x64 * x64).mean(1, keepdim=True) + block.pre.eps) * wp
    n = n64.detach().to(x.dtype)
    y = layer.forward(n, dev, training=True)
    y64 = y.double().requires_grad_()
    c = y64 - y64.mean(1, keepdim=True)
    out64 = 0.8 * x64 + gate * (c / torch.sqrt((c * c).mean(1, keepdim=True) + block.post.eps) * wq + bq)
    # the layer's own input is rounded to its type in both; y may differ where a last bit of n does
    tol = 2e-5 if dtype == wl.DTYPE_F32 else 8e-3
    near = lambda a, b: float((a.double() - b).norm() / b.norm()) <= tol
    assert near(out, out64.detach())
    out64.backward(dout.double())
    L = empty_grads(w, dev)
    dn = layer.backward(n, y64.grad.to(x.dtype), dev, L)
    n64.backward(dn.double())                                           # adds to the residual's part of x64.grad
    assert near(dx, x64.grad)
    for name, want in (("dw_pre", wp.grad), ("dw_post", wq.grad), ("db_post", bq.grad), ("dgate", gate.grad)):
        assert near(G[name], want), name
    for name in ("dw1", "dw2", "dw_up", "dw_down"):
        assert near(G[name], L[name].double()), name
    layer.close()


def test_two_blocks_in_a_row_share_a_joint():
    """out and the next block's n from one call are those of two blocks after each other."""
    binding, w, dev, layer, block = _block(wl.DTYPE_BF16, seed=72)
    x = dev["x"]
    first = block.forward(x, dev)
    n = binding.residual_norm_forward(x, pre=block.pre, want_r=False)[1]
    y = layer.forward(n, dev)
    r, n2, _ = binding.residual_norm_forward(x, y, block.gate, block.post, block.pre, residual_scale=0.8, gate_kind=binding.BIGMAC_GATE_CHANNEL)
    assert torch.equal(first, r)
    alone = binding.residual_norm_forward(first, pre=block.pre, want_r=False)[1]
    # the fused one normalises r before it is rounded: a bf16 step of the largest element apart at most
    assert float((n2.double() - alone.double()).norm() / alone.double().norm()) <= 2.0 ** -8
    layer.close()


def test_accumulates_over_micro_batches():
    binding, w, dev, layer, block = _block(wl.DTYPE_F32, seed=73)
    G = _grads(w, dev)
    block.forward(dev["x"], dev, training=True)
    block.backward(dev["dy"], dev, G)
    once = {n: t.clone() for n, t in G.items()}
    block.forward(dev["x"], dev, training=True)
    block.backward(dev["dy"], dev, G, accumulate=True)
    for name, t in G.items():
        np.testing.assert_allclose(t.cpu().numpy(), 2 * once[name].cpu().numpy(), rtol=1e-6, atol=1e-6 * float(once[name].abs().max()), err_msg=name)
    with pytest.raises(RuntimeError):
        block.forward(dev["x"], dev)
        block.backward(dev["dy"], dev, G)
    layer.close()


def test_block_with_4_bit_experts():
    """Serving: the same block, its experts in 4 bits."""
    binding, w, dev, layer, block = _block(wl.DTYPE_BF16, T=50, seed=74)
    four = dict(dev, w1=binding.mx4_quantize_weights(dev["w1"]), w2=binding.mx4_quantize_weights(dev["w2"]))
    out, R = block.forward(dev["x"], four, want_routing=True)
    n = binding.residual_norm_forward(dev["x"], pre=block.pre, want_r=False)[1]
    y = layer.forward(n, four)
    want = binding.residual_norm_forward(dev["x"], y, block.gate, block.post, None, residual_scale=0.8, gate_kind=binding.BIGMAC_GATE_CHANNEL)[0]
    assert torch.equal(out, want) and torch.equal(R["topk_idx"], layer.route(n, dev)["topk_idx"])
    layer.close()


def test_two_steps_of_one_layer_at_once_are_refused():
    """The layer keeps one step: gradients of the one before would be those of the wrong activations."""
    binding, w, dev, layer, block = _block(wl.DTYPE_F32, seed=75)
    G = _grads(w, dev)
    other = binding.Block(layer, block.pre)
    block.forward(dev["x"], dev, training=True)
    other.forward(dev["x"], dev, training=True)
    with pytest.raises(RuntimeError):
        block.backward(dev["dy"], dev, G)
    other.backward(dev["dy"], dev, G)
    layer.close()
