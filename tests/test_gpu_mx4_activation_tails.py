"""Both GELUs of 4-bit products down their negative tails, where 1 + erf and 1 + tanh cancel: results of every type are roundings of precise values."""
import numpy as np
import pytest
import torch
from scipy.special import ndtr

import mx4_reference as ref
from test_gpu_mx4_gelu import _arguments, _bf16

pytestmark = pytest.mark.gpu

ERF, TANH = 1, 2
EXPONENTS = [-20, -8, -4, -3, -2, -1, -1, 0, 0, 0, 1, 1, 1, 2, 60, 124] * 2


@pytest.fixture(scope="module")
def binding():
    from paper_2502_16927_b200 import binding as b

    return b


def _act(z, act):
    """The value and how far an fp32 evaluation may be off.  z/2 erfc(-z / sqrt 2): erfc by 4 units of 2^-23 and, its argument rounded twice, by
    1.5 units of 2^-24 times its sensitivity z^2 + 1; two products.  z / (1 + exp(-2 w)): six roundings of 2 w, which is the
    exponent; exp, sum and quotient.  Powers below the smallest normal number may become zero."""
    with np.errstate(over="ignore", invalid="ignore"):
        if act == ERF:
            want, units = z * ndtr(z), 8 + z * z
        else:
            w = np.sqrt(2 / np.pi) * (z + 0.044715 * z ** 3)
            want, units = z / (1 + np.exp(-2 * w)), 6 * np.abs(w) + 4
        return want, np.where(want == 0, 0, np.abs(want) * np.minimum(units * 2.0 ** -23, 1)) + np.where(z < -8, np.abs(z) * 2.0 ** -126, 0)


@pytest.mark.parametrize("act", [ERF, TANH])
@pytest.mark.parametrize("tile", [64, 128, 256])
def test_fp32_results(binding, act, tile):
    a, w, z = _arguments(np.random.default_rng(tile + act), 9000, EXPONENTS)
    binding.bigmac_debug_set("mx4_tile", tile)
    try:
        y = binding.mx4_matmul(binding.Mx4(*a), binding.Mx4(*w), act=act, dtype=torch.float32).double().cpu().numpy()
    finally:
        binding.bigmac_debug_set("defaults", 0)
    want, err = _act(z, act)
    bad = ~(np.abs(y - want) <= err + np.abs(want) * 2.0 ** -24)
    assert not bad.any(), (int(bad.sum()), z[bad][:5], y[bad][:5], want[bad][:5])


def test_bf16_results_with_tanh(binding):
    a, w, z = _arguments(np.random.default_rng(9), 3000, EXPONENTS)
    y = binding.mx4_matmul(binding.Mx4(*a), binding.Mx4(*w), act=TANH).double().cpu().numpy()
    want, err = _act(z, TANH)
    bad = ~((y >= _bf16(want - err)) & (y <= _bf16(want + err)))
    assert not bad.any(), (int(bad.sum()), z[bad][:5], y[bad][:5], want[bad][:5])


def test_4_bit_blocks_with_tanh(binding):
    rng = np.random.default_rng(6)
    a, w, z = _arguments(rng, 4000, [0] * 32, extra=rng.integers(0, 16, 32))
    got = binding.mx4_dequantize(binding.mx4_matmul_mx4(binding.Mx4(*a), binding.Mx4(*w), act=TANH), torch.float32).double().cpu().numpy()
    want, err = _act(z, TANH)
    top, slack = np.abs(want).max(1, keepdims=True), err.max(1, keepdims=True)
    ok = np.zeros(want.shape, dtype=bool)
    for bound in (top - slack, top + slack):
        scale = 2.0 ** np.maximum(np.floor(np.log2(np.maximum(bound, 2.0 ** -130))) - 2, -127)
        v = np.abs(want) / scale
        step = np.where(v < 2, 0.5, np.where(v < 4, 1.0, 2.0))
        ok |= np.abs(got - want) <= np.where(v > 6, v - 6, step / 2) * scale * (1 + 1e-12) + err
    assert ok.all(), (int((~ok).sum()), z[~ok][:5], got[~ok][:5], want[~ok][:5])


@pytest.mark.parametrize("act", [ERF, TANH])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_infinities_and_nan(binding, act, dtype):
    """z Phi(z) of infinity is infinity; of minus infinity, as of a NaN, the product with zero is a NaN."""
    code = np.zeros((3, 32), dtype=np.int64)
    code[0, 0], code[1, 0] = 7, 15
    byte = np.array([[254], [254], [255]])
    a = binding.Mx4(torch.from_numpy(ref.pack_codes(code)).cuda(), torch.from_numpy(ref.pack_scales(byte)).cuda())
    w = binding.Mx4(torch.from_numpy(ref.pack_codes(code[:1])).cuda(), torch.from_numpy(ref.pack_scales(byte[:1])).cuda())
    y = binding.mx4_matmul(a, w, act=act, dtype=dtype)
    assert y[0, 0] == float("inf") and bool(torch.isnan(y[1:, 0]).all())
