"""The operators around the layer where no GPU is needed: refusals of the C ABI and of the binding, layouts."""
import ctypes as C

import numpy as np
import pytest
import torch

import mx4_reference as ref
from paper_2502_16927_b200 import binding, build

P = C.c_void_p
HERE = 1 << 20            # an aligned address that no refused call may touch


@pytest.fixture(scope="module")
def lib():
    build.build()
    return binding.lib()


def _mx4(codes=HERE, scales=HERE, rows=4, K=64, E=0, offsets=None):
    return binding.bigmac_mx4_t(codes, scales, rows, K, E, offsets)


def test_mx4_bytes(lib):
    code, scale = C.c_size_t(), C.c_size_t()

    def sizes(*args):
        assert lib.bigmac_mx4_bytes(*args, C.byref(code), C.byref(scale)) == 0
        return code.value, scale.value

    assert sizes(0, 32, 0, 0) == (0, 0)
    assert sizes(1, 32, 0, 0) == (16, 512)
    assert sizes(129, 160, 0, 0) == (129 * 80, 2 * 2 * 512)
    assert sizes(129, 160, 3, 0) == (3 * 129 * 80, 3 * 2 * 2 * 512)
    # grouped: any split of the rows over the experts fits, each segment from a multiple of 128 on
    for rows, E in ((0, 4), (1, 4), (5, 4), (300, 7), (1000, 1), (4096, 64)):
        codes, scales = sizes(rows, 64, E, 1)
        rng = np.random.default_rng(rows)
        for _ in range(50):
            counts = np.bincount(rng.integers(0, E, rows), minlength=E)
            assert (-(-counts // 128) * 128).sum() * 32 <= codes
        assert codes % (128 * 32) == 0 and scales == codes // (128 * 32) * 512
        assert codes == binding._mx4_stored(rows, E) * 32
    for bad, status in (((-1, 32, 0, 0), -1), ((1, 0, 0, 0), -1), ((1, 32, -1, 0), -1), ((1, 32, 0, 1), -1), ((1, 32, 1025, 1), -1),
                        ((1, 48, 0, 0), -2)):
        assert lib.bigmac_mx4_bytes(*bad, C.byref(code), C.byref(scale)) == status
    assert lib.bigmac_mx4_bytes(1, 32, 0, 0, None, C.byref(scale)) == -1


def test_mx4_quantize_refusals(lib):
    def call(x=HERE, dtype=1, x_rows=4, ld=64, slot=None, k=1, out=None):
        return lib.bigmac_mx4_quantize(x, dtype, x_rows, ld, slot, k, C.byref(out or _mx4()), None)

    assert lib.bigmac_mx4_quantize(HERE, 1, 4, 64, None, 1, None, None) == -1
    for kw in (dict(x=None), dict(x=HERE + 8), dict(dtype=2), dict(dtype=-1), dict(x_rows=3), dict(x_rows=-1), dict(ld=63), dict(ld=68),
               dict(slot=HERE, k=0), dict(slot=HERE + 2), dict(out=_mx4(codes=None)), dict(out=_mx4(scales=None)), dict(out=_mx4(codes=HERE + 4)),
               dict(out=_mx4(rows=-1)), dict(out=_mx4(K=0)), dict(out=_mx4(E=2)), dict(out=_mx4(E=0, offsets=HERE)), dict(out=_mx4(E=1025, offsets=HERE))):
        assert call(**kw) == -1, kw
    assert call(out=_mx4(K=40)) == -2
    assert call(out=_mx4(rows=2 ** 31 - 1, E=1024, offsets=HERE)) == -2


def test_mx4_dequantize_and_matmul_refusals(lib):
    def back(q=None, y=HERE, dtype=1, ld=64):
        return lib.bigmac_mx4_dequantize(C.byref(q or _mx4()), y, dtype, ld, None)

    for kw in (dict(y=None), dict(y=HERE + 8), dict(dtype=5), dict(ld=60), dict(ld=66), dict(q=_mx4(E=3))):
        assert back(**kw) == -1, kw

    def product(a=None, w=None, act=3, dtype=1, c=HERE, ldc=8):
        return lib.bigmac_mx4_matmul(C.byref(a or _mx4()), C.byref(w or _mx4(rows=8)), act, dtype, c, ldc, None)

    assert lib.bigmac_mx4_matmul(None, C.byref(_mx4()), 3, 1, HERE, 8, None) == -1
    assert lib.bigmac_mx4_matmul(C.byref(_mx4()), None, 3, 1, HERE, 8, None) == -1
    for kw in (dict(c=None), dict(c=HERE + 8), dict(act=4), dict(act=-1), dict(dtype=2), dict(ldc=7), dict(a=_mx4(K=32)), dict(a=_mx4(E=2)),
               dict(w=_mx4(rows=8, E=2)), dict(a=_mx4(E=2, offsets=HERE)), dict(a=_mx4(E=2, offsets=HERE), w=_mx4(rows=8, E=3)),
               dict(a=_mx4(E=2, offsets=HERE), w=_mx4(rows=8, E=2, offsets=HERE))):
        assert product(**kw) == -1, kw
    def product4(a=None, w=None, act=3, out=None):
        return lib.bigmac_mx4_matmul_mx4(C.byref(a or _mx4()), C.byref(w or _mx4(rows=32)), act, C.byref(out or _mx4(2 * HERE, 2 * HERE, K=32)), None)

    assert lib.bigmac_mx4_matmul_mx4(None, C.byref(_mx4()), 3, C.byref(_mx4()), None) == -1
    for kw in (dict(act=4), dict(a=_mx4(K=32)), dict(w=_mx4(rows=64)), dict(out=_mx4(2 * HERE, 2 * HERE, rows=5, K=32)), dict(out=_mx4(K=32)),
               dict(out=_mx4(2 * HERE, 2 * HERE, K=32, E=1, offsets=HERE)), dict(out=_mx4(2 * HERE, 2 * HERE, K=64)),
               dict(a=_mx4(E=1, offsets=HERE), w=_mx4(rows=32, E=1), out=_mx4(2 * HERE, 2 * HERE, K=32, E=1, offsets=2 * HERE))):
        assert product4(**kw) == -1, kw
    assert product4(out=_mx4(2 * HERE, 2 * HERE, K=48), w=_mx4(rows=48)) == -2
    assert product4(a=_mx4(rows=0), out=_mx4(2 * HERE, 2 * HERE, rows=0, K=32)) == 0
    # nothing to do is no error and touches nothing
    assert product(a=_mx4(rows=0)) == 0 and product(w=_mx4(rows=0)) == 0


def test_mx4_products_of_no_rows(lib):
    empty, w = binding.bigmac_mx4_t(None, None, 0, 64, 0, None), _mx4(rows=32)
    assert lib.bigmac_mx4_matmul_mx4(C.byref(empty), C.byref(w), 3, C.byref(binding.bigmac_mx4_t(None, None, 0, 32, 0, None)), None) == 0
    assert lib.bigmac_mx4_matmul(C.byref(empty), C.byref(w), 3, 0, None, 32, None) == 0


def test_binding_refuses_what_is_no_4_bit_matrix():
    u8 = torch.uint8
    for codes, scales, kw in ((torch.zeros(4, 32), torch.zeros(1, 1, 512, dtype=u8), {}),
                              (torch.zeros(4, 32, dtype=u8), torch.zeros(1, 2, 512, dtype=u8), {}),
                              (torch.zeros(129, 32, dtype=u8), torch.zeros(1, 1, 512, dtype=u8), {}),
                              (torch.zeros(2, 4, 32, dtype=u8), torch.zeros(1, 1, 512, dtype=u8), {}),
                              (torch.zeros(4, 32, dtype=u8), torch.zeros(1, 1, 512, dtype=u8), {}),                            # not on a GPU
                              (torch.zeros(4, 32, dtype=u8), torch.zeros(1, 1, 512, dtype=u8), dict(offsets=torch.zeros(3, dtype=torch.int32))),
                              (torch.zeros(4, 32, dtype=u8), torch.zeros(1, 1, 512, dtype=u8), dict(offsets=torch.zeros(3, dtype=torch.int32), rows=4))):
        with pytest.raises(ValueError):
            binding.Mx4(codes, scales, **kw)
    with pytest.raises(ValueError):
        binding._dtype(torch.float16)


def test_reference_quantisation():
    """The reference itself, at places worked out by hand."""
    x = np.zeros((1, 64))
    x[0, :10] = [6, -6, 7.9, 5, 3.5, 2.5, 1.75, 0.75, 0.25, 0.26]       # largest 7.9: scale 1
    x[0, 32:36] = [1.0, 0.0625, -0.1875, 0.2]                            # largest 1: scale 1/4, i.e. 4, 0.25, 0.75, 0.8
    code, byte = ref.quantise(x)
    assert byte.tolist() == [[127, 125]]
    v = ref.values(code, byte)[0]
    assert v[:10].tolist() == [6, -6, 6, 4, 4, 2, 2, 1, 0, 0.5]
    assert v[32:36].tolist() == [1.0, 0.0, -0.25, 0.25]


# ---- the joint of two blocks

_NAMES = ("d dtype post_kind pre_kind gate_kind post_eps pre_eps residual_scale w_post b_post w_pre b_pre x x_ld y y_ld gate gate_ld r r_ld n n_ld "
          "stats dr dr_ld dn dn_ld dx dx_ld dy dy_ld dgate dgate_ld dw_post db_post dw_pre db_pre").split()


def _joint(**kw):
    base = dict.fromkeys(_NAMES, 0)
    base.update(d=64, dtype=1, post_kind=1, pre_kind=2, post_eps=1e-6, pre_eps=1e-6, residual_scale=1.0, x=HERE, x_ld=64, y=HERE, y_ld=64, r=HERE, r_ld=64,
                n=HERE, n_ld=64)
    base.update(kw)
    assert set(base) == set(_NAMES)
    return binding._RESIDUAL_NORM.pack(*[base[n] for n in _NAMES])


_BAD = [dict(d=0), dict(d=-1), dict(dtype=2), dict(post_kind=3), dict(pre_kind=-1), dict(gate_kind=4), dict(post_eps=-1e-6), dict(pre_eps=float("nan")),
        dict(post_eps=float("inf")), dict(residual_scale=float("nan")), dict(x=HERE + 1), dict(x_ld=63), dict(y_ld=63), dict(x=0), dict(w_post=HERE + 2),
        dict(gate_kind=1), dict(gate=HERE), dict(gate_kind=3, gate=HERE, gate_ld=63), dict(y=0), dict(y=0, post_kind=0, w_post=HERE),
        dict(y=0, post_kind=0, gate_kind=1, gate=HERE), dict(stats=HERE + 4)]


def test_residual_norm_refusals(lib):
    assert lib.bigmac_residual_norm_forward(None, 1, None) == -1
    for kw in _BAD + [dict(r=HERE + 1), dict(n_ld=63), dict(n=0), dict(pre_kind=0), dict(pre_kind=0, n=0, w_pre=HERE)]:
        assert lib.bigmac_residual_norm_forward(_joint(**kw), 4, None) == -1, kw
    assert lib.bigmac_residual_norm_forward(_joint(), -1, None) == -1
    assert lib.bigmac_residual_norm_forward(_joint(d=8193, x_ld=8193, y_ld=8193), 4, None) == -2
    assert lib.bigmac_residual_norm_forward(_joint(x=0, y=0, post_kind=0, r=0, n=0), 0, None) == 0       # no rows

    back = dict(r=0, n=0, stats=HERE, dr=HERE, dr_ld=64, dn=HERE, dn_ld=64, dx=HERE, dx_ld=64, dy=HERE, dy_ld=64)

    def call(scratch=HERE, size=1 << 30, T=4, **kw):
        return lib.bigmac_residual_norm_backward(_joint(**{**back, **kw}), T, 0, scratch, size, None)

    assert lib.bigmac_residual_norm_backward(None, 1, 0, None, 0, None) == -1
    for kw in _BAD + [dict(stats=0), dict(dr=0, dn=0), dict(dx_ld=63), dict(dy=HERE + 1), dict(dgate=HERE), dict(pre_kind=0),
                      dict(y=0, post_kind=0), dict(dw_post=HERE + 1), dict(dw_post=HERE, scratch=None), dict(dw_post=HERE, scratch=HERE + 8)]:
        assert call(**kw) == -1, kw
    assert call(dw_post=HERE, size=16) == -3

    sums = dict(dw_post=2 * HERE, db_post=3 * HERE, dw_pre=4 * HERE, db_pre=5 * HERE)                     # a vector that both norms share: two sums
    for pair in (("dw_post", "dw_pre"), ("db_post", "db_pre"), ("dw_pre", "db_pre")):
        assert call(**{**sums, pair[1]: sums[pair[0]]}) == -1, pair
    assert call(**sums, gate_kind=2, gate=HERE, dgate=2 * HERE) == -1
    assert call(**sums, size=16) == -3

    need = C.c_size_t()
    assert lib.bigmac_residual_norm_scratch_bytes(_joint(**back), 4, C.byref(need)) == 0 and need.value == 0
    assert lib.bigmac_residual_norm_scratch_bytes(_joint(**back, db_pre=HERE), 4, C.byref(need)) == 0 and need.value >= 4 * 64 * 4
    assert lib.bigmac_residual_norm_scratch_bytes(_joint(**back, db_pre=HERE), 0, C.byref(need)) == 0 and need.value == 0
    assert lib.bigmac_residual_norm_scratch_bytes(None, 4, C.byref(need)) == -1


def test_forward_with_4_bit_experts_refuses_null_handles(lib):
    size = C.c_size_t()
    assert lib.bigmac_forward_mx4(None, None, 0, None, None, None, None, None, None, 0, None) == -1
    assert lib.bigmac_mx4_workspace_bytes(None, 1, C.byref(size)) == -1
