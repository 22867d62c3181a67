"""Block.backward when it has to refuse: nothing is written or added before it does."""
import pytest
import torch

from paper_2502_16927_b200 import workloads as wl

from test_gpu_block import _block, _grads

pytestmark = pytest.mark.gpu


def _filled(w, dev):
    return {n: t.fill_(0.25) for n, t in _grads(w, dev).items()}


@pytest.mark.parametrize("accumulate", [False, True])
@pytest.mark.parametrize("between", ["inference", "4 bits", "other tokens", "no step"])
def test_a_step_that_is_gone_leaves_the_gradients_alone(between, accumulate):
    binding, w, dev, layer, block = _block(wl.DTYPE_BF16, seed=91)
    block.forward(dev["x"], dev, training=True)
    if between == "inference":
        layer.forward(dev["x"], dev)
    elif between == "4 bits":
        layer.forward(dev["x"], dict(dev, w1=binding.mx4_quantize_weights(dev["w1"]), w2=binding.mx4_quantize_weights(dev["w2"])))
    elif between == "other tokens":
        layer.forward(dev["x"][:40].contiguous(), dev, training=True)
    else:
        block.forward(dev["x"], dev)
    G = _filled(w, dev)
    with pytest.raises(RuntimeError):
        block.backward(dev["dy"], dev, G, accumulate=accumulate)
    torch.cuda.synchronize()
    assert all(bool((t == 0.25).all()) for t in G.values())
    layer.close()


@pytest.mark.parametrize("accumulate", [False, True])
@pytest.mark.parametrize("pair", [("dw_pre", "dw_post"), ("dw_pre", "db_post"), ("dw_pre", "dgate"), ("db_post", "dgate")])
def test_two_gradients_in_one_place_are_refused(pair, accumulate):
    """Norms that share a vector need a gradient each: the second of the block's calls would write over the first one's."""
    binding, w, dev, layer, block = _block(wl.DTYPE_BF16, seed=92)
    block.forward(dev["x"], dev, training=True)
    G = _filled(w, dev)
    G[pair[1]] = G[pair[0]]
    with pytest.raises(ValueError):
        block.backward(dev["dy"], dev, G, accumulate=accumulate)
    torch.cuda.synchronize()
    assert all(bool((t == 0.25).all()) for t in G.values())
    block.backward(dev["dy"], dev, _grads(w, dev))                     # the step is still there
    layer.close()


@pytest.mark.parametrize("dout", ["shape", "type"])
def test_a_gradient_of_the_wrong_form_is_refused(dout):
    binding, w, dev, layer, block = _block(wl.DTYPE_BF16, seed=93)
    block.forward(dev["x"], dev, training=True)
    G = _filled(w, dev)
    with pytest.raises(ValueError):
        block.backward(dev["dy"][:-1] if dout == "shape" else dev["dy"].float(), dev, G)
    assert all(bool((t == 0.25).all()) for t in G.values())
    layer.close()


def test_parameters_of_the_wrong_form_are_refused_before_anything_is_written():
    binding, w, dev, layer, block = _block(wl.DTYPE_BF16, seed=94)
    block.forward(dev["x"], dev, training=True)
    for name, t in (("dw_pre", torch.empty(w.d - 1, device="cuda")), ("dw_pre", torch.empty(w.d, device="cuda", dtype=torch.bfloat16)),
                    ("db_pre", torch.empty(w.d + 1, device="cuda"))):
        G = _filled(w, dev)
        with pytest.raises(ValueError):
            block.backward(dev["dy"], dev, {**G, name: t}, accumulate=True)
        torch.cuda.synchronize()
        assert all(bool((g == 0.25).all()) for g in G.values()), name
    layer.close()
