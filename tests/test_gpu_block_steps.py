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
