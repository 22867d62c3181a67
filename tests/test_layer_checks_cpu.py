"""What the calls around the layer refuse before anything reaches the library: batches that are not of the handle's width and type."""
import pytest
import torch

from paper_2502_16927_b200 import binding


def _layer(d=64, dtype=torch.bfloat16):
    """A layer without a handle: a call that gets past its checks fails in another way than by a ValueError."""
    layer = binding.Layer.__new__(binding.Layer)
    layer.cfg, layer.tdtype, layer.handle, layer._need, layer._scratch = dict(d=d, E=4, k=2), dtype, None, {}, None
    return layer


def _four():
    w = binding.Mx4.__new__(binding.Mx4)
    return dict(w1=w, w2=w)


BAD = [torch.zeros(3, 32, dtype=torch.bfloat16), torch.zeros(3, 128, dtype=torch.bfloat16), torch.zeros(3, 64), torch.zeros(64, dtype=torch.bfloat16),
       torch.zeros(1, 3, 64, dtype=torch.bfloat16)]


@pytest.mark.parametrize("x", BAD)
def test_forward_with_4_bit_experts(x):
    with pytest.raises(ValueError):
        _layer().forward(x, _four())


@pytest.mark.parametrize("y", BAD + [torch.zeros(2, 64, dtype=torch.bfloat16)])
def test_results_of_a_forward_with_4_bit_experts(y):
    with pytest.raises(ValueError):
        _layer().forward(torch.zeros(3, 64, dtype=torch.bfloat16), _four(), y=y)


@pytest.mark.parametrize("x", BAD)
@pytest.mark.parametrize("training", [False, True])
def test_block(monkeypatch, x, training):
    """The norm before the layer takes any width: its result must not reach a layer of another."""
    monkeypatch.setattr(binding, "residual_norm_forward", lambda x, *a, **k: (None, x, None))
    with pytest.raises(ValueError):
        binding.Block(_layer(), binding.Norm(binding.BIGMAC_NORM_RMS)).forward(x, {}, training=training)


@pytest.mark.parametrize("pre", [None, binding.Norm(binding.BIGMAC_NORM_NONE)])
def test_block_without_a_norm_before(pre):
    with pytest.raises(ValueError):
        binding.Block(_layer(), pre)
