"""The joint's kernels one by one: sizes that each of them takes, all gates, with and without parameters, in place."""
import pytest
import torch

import test_gpu_residual_norm as base

pytestmark = pytest.mark.gpu

NONE, RMS, LAYER = base.NONE, base.RMS, base.LAYER
BF16, FP32 = torch.bfloat16, torch.float32


@pytest.fixture(scope="module")
def binding():
    from paper_2502_16927_b200 import binding as b

    return b


def _threads(d, columns):
    return -(-d // (32 * columns)) * 32


def _sms():
    return torch.cuda.get_device_properties(torch.cuda.current_device()).multi_processor_count


def _many(d):
    """Just more rows than the forward works on at once: what the persistent blocks are taken for."""
    return 2 * _sms() * (512 // _threads(d, 8) if d <= 4096 else 1) + 13


def _weights_only(monkeypatch):
    inputs = base._inputs

    def without_biases(*args):
        p, dr, dn = inputs(*args)
        return {**p, "b_post": None, "b_pre": None}, dr, dn

    monkeypatch.setattr(base, "_inputs", without_biases)


# eight columns a thread up to 1280, 16 above; rows off 16-byte boundaries where d is odd
@pytest.mark.parametrize("d", [1280, 1279, 1024, 264, 257, 100, 1357, 2048])
@pytest.mark.parametrize("gate_kind", [0, 1, 2, 3])
def test_forward_of_many_rows(binding, d, gate_kind):
    base._run(binding, _many(d), d, BF16, (RMS, LAYER)[gate_kind % 2], (LAYER, RMS)[gate_kind // 2], gate_kind, rho=0.5, seed=d + gate_kind)


@pytest.mark.parametrize("d", [1280, 1279, 264, 257, 1357, 2048, 4104])
def test_forward_of_many_rows_without_parameters(binding, d):
    base._run(binding, _many(d), d, BF16, RMS, LAYER, d % 4, params=False, seed=d)


@pytest.mark.parametrize("d", [1279, 257, 100, 1357, 128, 1024, 2048])
def test_forward_of_many_rows_fp32(binding, d):
    base._run(binding, _many(d), d, FP32, LAYER, RMS, d % 4, seed=d)


@pytest.mark.parametrize("d", [1280, 1279, 264, 257, 100, 1357, 2048, 4104])
@pytest.mark.parametrize("params", [False, True])
def test_norm_of_many_rows_alone(binding, d, params):
    base._run(binding, _many(d), d, BF16, NONE, (RMS, LAYER)[d % 2], 0, with_y=False, params=params, seed=d)


# 16 columns a thread, no sums of biases: more rows than the grid has groups of threads for, so that a group works on several
@pytest.mark.parametrize("d", [264, 1024, 4096, 4104, 8192])
@pytest.mark.parametrize("gate_kind", [0, 1, 2, 3])
def test_backward_with_weights_and_no_biases(binding, monkeypatch, d, gate_kind):
    _weights_only(monkeypatch)
    T = (2 * _sms() + 5) * (512 // _threads(d, 16)) + 1
    base._run(binding, T, d, BF16, (LAYER, RMS)[gate_kind % 2], (RMS, LAYER)[gate_kind // 2], gate_kind, rho=0.5, seed=d + gate_kind)


@pytest.mark.parametrize("d", [264, 4096, 4104])
@pytest.mark.parametrize("which", ["dr", "dn"])
def test_backward_with_weights_and_one_gradient(binding, monkeypatch, d, which):
    _weights_only(monkeypatch)
    T = (_sms() + 5) * (512 // _threads(d, 16)) + 1
    base._run(binding, T, d, BF16, RMS, LAYER, 2, use_dr=which == "dr", use_dn=which == "dn", accumulate=True, seed=d)
    base._run(binding, T, d, BF16, NONE, RMS, 0, with_y=False, use_dr=which == "dr", use_dn=which == "dn", seed=d)


def _joint_inputs(T, d, dtype, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    n = lambda *s: torch.randn(*s, generator=g, device="cuda")
    return [n(T, d).to(dtype) for _ in range(5)], n(d), n(d)


SHAPES = [(3, 1024), (300, 1024), (2000, 1024), (2000, 1023), (5000, 264), (5000, 257), (700, 4096), (700, 4095), (400, 8192), (400, 8191)]


@pytest.mark.parametrize("dtype", [BF16, FP32])
@pytest.mark.parametrize("T,d", SHAPES)
def test_forward_in_place(binding, T, d, dtype):
    """r over x and n over y, by every kernel: bit for bit what separate results are."""
    (x, y, gate, _, _), w, b = _joint_inputs(T, d, dtype, d)
    for post, pre in ((binding.Norm(RMS, w), binding.Norm(RMS, w)), (binding.Norm(LAYER, w, b), binding.Norm(LAYER, w, b))):
        r, n, stats = binding.residual_norm_forward(x, y, gate, post, pre, training=True)
        x2, y2 = x.clone(), y.clone()
        _, _, stats2 = binding.residual_norm_forward(x2, y2, gate, post, pre, training=True, r=x2, n=y2)
        assert torch.equal(r, x2) and torch.equal(n, y2) and torch.equal(stats, stats2)


@pytest.mark.parametrize("dtype", [BF16, FP32])
@pytest.mark.parametrize("T,d", SHAPES)
@pytest.mark.parametrize("full", [False, True])
def test_backward_in_place(binding, T, d, dtype, full):
    """dx over dr and dy over dn (the C call takes them; the binding makes its own), by every kernel."""
    (x, y, gate, dr, dn), w, b = _joint_inputs(T, d, dtype, d + 1)
    gate = gate if full else None
    lib, es = binding.lib(), x.element_size()
    here = torch.cuda.current_device()
    for post, pre in ((binding.Norm(RMS, w), binding.Norm(RMS, w)), (binding.Norm(LAYER, w, b), binding.Norm(LAYER, w, b))):
        _, _, stats = binding.residual_norm_forward(x, y, gate, post, pre, training=True)
        names = ["dw_post", "dw_pre"] + (["db_post", "db_pre"] if post.bias is not None else [])
        G = {name: torch.empty(d, device="cuda") for name in names}
        dx, dy, dgate = binding.residual_norm_backward(x, y, gate, post, pre, dr, dn, stats, G)
        G2 = {name: torch.empty(d, device="cuda") for name in names}
        dx2, dy2, dgate2 = dr.clone(), dn.clone(), torch.empty_like(x)
        at = lambda t: (t.data_ptr(), d)
        grads = [G2[name].data_ptr() if name in G2 else 0 for name in ("dw_post", "db_post", "dw_pre", "db_pre")]
        members = binding._joint(x, x.shape, x.dtype, y, gate, None, post, pre, 1.0, here)
        q = binding._RESIDUAL_NORM.pack(*members, 0, 0, 0, 0, stats.data_ptr(), *at(dx2), *at(dy2), *at(dx2), *at(dy2), *(at(dgate2) if full else (0, 0)), *grads)
        size = binding.C.c_size_t()
        assert lib.bigmac_residual_norm_scratch_bytes(q, T, binding.C.byref(size)) == 0
        scratch = torch.empty(size.value, dtype=torch.uint8, device="cuda")
        assert lib.bigmac_residual_norm_backward(q, T, 0, scratch.data_ptr(), size.value, torch.cuda.current_stream().cuda_stream) == 0
        assert torch.equal(dx, dx2) and torch.equal(dy, dy2) and (not full or torch.equal(dgate, dgate2))
        assert all(torch.equal(G[name], G2[name]) for name in names)
