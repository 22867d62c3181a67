"""GELU of 4-bit products over its whole range, tail included: a result is the rounding of a value whose relative error is small everywhere."""
import numpy as np
import pytest
import torch
from scipy.special import ndtr

import mx4_reference as ref

pytestmark = pytest.mark.gpu

GELU = 1


@pytest.fixture(scope="module")
def binding():
    from paper_2502_16927_b200 import binding as b

    return b


def _arguments(rng, M, exponents, extra=None):
    """4-bit matrices whose product has the numbers 2^exponent sum c_b 8^-b, five digits c_b in [-6, 6] a row, an exponent a column: 16 bits wide,
    so that the sums of the product are exact.  extra: codes [N] of one more digit, of 2^-6 times the column's power of two."""
    N, blocks = len(exponents), 6
    code_a, code_w = np.zeros((M, 32 * blocks), dtype=np.int64), np.zeros((N, 32 * blocks), dtype=np.int64)
    code_a[:, :160:32] = rng.integers(0, 16, (M, 5))
    code_w[:, :160:32] = 2
    byte_a = np.full((M, blocks), 127)
    byte_w = 127 + np.asarray(exponents)[:, None] - 3 * np.arange(blocks)[None, :]
    code_a[:, 160], byte_w[:, 5] = 2, 121 + np.asarray(exponents)
    if extra is not None:
        code_w[:, 160] = extra
    pack = lambda c, b: (torch.from_numpy(ref.pack_codes(c)).cuda(), torch.from_numpy(ref.pack_scales(b)).cuda())
    return pack(code_a, byte_a), pack(code_w, byte_w), ref.values(code_a, byte_a) @ ref.values(code_w, byte_w).T


def _gelu(z):
    """z Phi(z), and how far a computed one may be off before it is rounded: log2 Phi(-|z|) by a polynomial whose value is off by 1.0e-5 of Phi up
    to 5 and 1.1e-4 behind it (on 1.5 million numbers a range, every step in fp32), the power of two by 2^-22; powers below 2^-126 become zero."""
    want = z * ndtr(z)
    return want, np.abs(want) * np.where(np.abs(z) <= 5, 1.2e-5, 1.3e-4) + np.where(z < -12, np.abs(z) * 2.0 ** -126, 0)


def _bf16(x):
    return torch.from_numpy(x).to(torch.bfloat16).double().numpy()


# rows enough for the 64 and 128 column tiles of one CTA, and for CTA pairs
@pytest.mark.parametrize("tile", [64, 128, 256])
def test_bf16_results_are_roundings_of_precise_values(binding, tile):
    exponents = [-20, -8, -4, -3, -2, -1, -1, 0, 0, 0, 1, 1, 1, 2, 60, 124]
    a, w, z = _arguments(np.random.default_rng(tile), 9000, exponents)
    assert np.array_equal(z, z.astype(np.float32))
    binding.bigmac_debug_set("mx4_tile", tile)
    try:
        y = binding.mx4_matmul(binding.Mx4(*a), binding.Mx4(*w), act=GELU).double().cpu().numpy()
    finally:
        binding.bigmac_debug_set("defaults", 0)
    want, err = _gelu(z)
    bad = ~((y >= _bf16(want - err)) & (y <= _bf16(want + err)))
    assert not bad.any(), (int(bad.sum()), z[bad][:5], y[bad][:5], want[bad][:5])
    assert binding.operator_status() == 0


def test_4_bit_blocks_in_the_tail(binding):
    """Blocks whose 32 values all lie far down the negative tail take their scale and codes from them."""
    rng = np.random.default_rng(5)
    a, w, z = _arguments(rng, 4000, [0] * 32, extra=rng.integers(0, 16, 32))
    q = binding.mx4_matmul_mx4(binding.Mx4(*a), binding.Mx4(*w), act=GELU)
    got = binding.mx4_dequantize(q, torch.float32).double().cpu().numpy()
    want, err = _gelu(z)
    assert (z.max(1) < -4).sum() > 200                                  # blocks of nothing else
    top, slack = np.abs(want).max(1, keepdims=True), err.max(1, keepdims=True)
    ok = np.zeros(want.shape, dtype=bool)
    for bound in (top - slack, top + slack):                            # the largest magnitude as computed lies between these two
        scale = 2.0 ** np.maximum(np.floor(np.log2(np.maximum(bound, 2.0 ** -130))) - 2, -127)
        v = np.abs(want) / scale
        step = np.where(v < 2, 0.5, np.where(v < 4, 1.0, 2.0))
        ok |= np.abs(got - want) <= np.where(v > 6, v - 6, step / 2) * scale * (1 + 1e-12) + err
    assert ok.all(), (int((~ok).sum()), z[~ok][:5], got[~ok][:5], want[~ok][:5])


def test_infinities_and_nan(binding):
    """Sums that overflow: z Phi(z) of infinity is infinity; of minus infinity, as of a NaN, the product with zero is a NaN."""
    code = np.zeros((3, 32), dtype=np.int64)
    code[0, 0], code[1, 0] = 7, 15                                      # 6, -6
    byte = np.array([[254], [254], [255]])
    a = binding.Mx4(torch.from_numpy(ref.pack_codes(code)).cuda(), torch.from_numpy(ref.pack_scales(byte)).cuda())
    y = binding.mx4_matmul(a, binding.Mx4(torch.from_numpy(ref.pack_codes(code[:1])).cuda(), torch.from_numpy(ref.pack_scales(byte[:1])).cuda()), act=GELU)
    assert y[0, 0] == float("inf") and bool(torch.isnan(y[1:, 0]).all())
