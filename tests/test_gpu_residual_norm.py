"""The joint of two blocks on the GPU, forward and backward, against its formulas in 64 bits."""
import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu

NONE, RMS, LAYER = 0, 1, 2


@pytest.fixture(scope="module")
def binding():
    from paper_2502_16927_b200 import binding as b

    return b


def _norm(v, kind, w, b, eps):
    if kind == LAYER:
        v = v - v.mean(1, keepdim=True)
    if kind != NONE:
        v = v / torch.sqrt((v * v).mean(1, keepdim=True) + eps)
    if w is not None:
        v = v * w
    return v if b is None else v + b


def _formula(p, post, pre, rho, eps, gate_kind):
    """r and n from 64-bit leaves; a post norm is absent with y."""
    r = rho * p["x"]
    if p["y"] is not None:
        a = _norm(p["y"], post, p["w_post"], p["b_post"], eps)
        if p["gate"] is not None:
            a = a * (p["gate"][:, None] if gate_kind == 1 else p["gate"])
        r = r + a
    return r, None if pre == NONE else _norm(r, pre, p["w_pre"], p["b_pre"], eps)


def _inputs(T, d, dtype, post, pre, gate_kind, with_y, params, seed):
    g = torch.Generator().manual_seed(seed)

    def normal(*shape, std=1.0, mean=0.0):
        return torch.randn(*shape, generator=g) * std + mean

    p = {"x": (normal(T, d) * normal(T, 1).exp()).to(dtype), "y": (normal(T, d, mean=0.3) * normal(T, 1).exp()).to(dtype) if with_y else None}
    p["gate"] = {0: lambda: None, 1: lambda: normal(T), 2: lambda: normal(d), 3: lambda: normal(T, d).to(dtype)}[gate_kind if with_y else 0]()
    p["w_post"] = normal(d, mean=1.0) if params and with_y else None
    p["b_post"] = normal(d) if params and with_y else None
    p["w_pre"] = normal(d, mean=1.0) if params and pre != NONE else None
    p["b_pre"] = normal(d) if params and pre != NONE else None
    return p, normal(T, d).to(dtype), normal(T, d).to(dtype) if pre != NONE else None


def _tol(dtype, *parts):
    """fp32 evaluation: sums of d terms in a tree of partial sums of 8 to 32 terms and further levels, each result a handful of roundings on
    values of the size `parts` name; 64 steps of 2^-24 cover it.  The rounding to the output's type adds half a step."""
    return 64 * 2.0 ** -24 * sum(parts)


def _close(name, got, want, size, dtype):
    want = want.detach()
    err = _tol(dtype, size) + want.abs() * torch.finfo(dtype).eps / 2 * 1.01
    diff = (got.double().cpu() - want).abs()
    assert bool((diff <= err).all()), (name, float((diff - err).max()), float(diff.max()))


def _rowmax(t):
    return t.detach().abs().amax(-1, keepdim=True)


def _run(binding, T, d, dtype, post, pre, gate_kind, with_y=True, params=True, rho=1.0, eps=1e-5, seed=0, ld_pad=0, use_dr=True, use_dn=True,
         accumulate=False):
    p, dr, dn = _inputs(T, d, dtype, post, pre, gate_kind, with_y, params, seed)
    dr, dn = dr if use_dr else None, dn if use_dn else None

    def device(t):
        if t is None:
            return None
        if t.dim() == 2 and ld_pad:
            wide = torch.full((t.shape[0], d + ld_pad), 3.0, dtype=t.dtype, device="cuda")
            wide[:, :d] = t.cuda()
            return wide[:, :d]
        return t.cuda()

    q = {k: device(t) for k, t in p.items()}
    post_norm = binding.Norm(post, q["w_post"], q["b_post"], eps) if with_y else None
    pre_norm = binding.Norm(pre, q["w_pre"], q["b_pre"], eps) if pre != NONE else None
    kind = gate_kind if with_y else 0
    r, n, stats = binding.residual_norm_forward(q["x"], q["y"], q["gate"], post_norm, pre_norm, residual_scale=rho, training=True, gate_kind=kind)
    r2, n2, none = binding.residual_norm_forward(q["x"], q["y"], q["gate"], post_norm, pre_norm, residual_scale=rho, gate_kind=kind)
    assert none is None and torch.equal(r, r2) and (n is None or torch.equal(n, n2))

    leaves = {k: None if t is None else t.double().requires_grad_() for k, t in p.items()}
    r64, n64 = _formula(leaves, post, pre, rho, eps, kind)
    # sizes of what is added up: parts of r in a row (the mean that is taken off included), of n behind its norm
    a_size = 0.0
    if with_y:
        with torch.no_grad():
            y64 = p["y"].double()
            rstd = 1.0 if post == NONE else 1.0 / torch.sqrt((((y64 - (y64.mean(1, keepdim=True) if post == LAYER else 0)) ** 2).mean(1, keepdim=True)) + eps)
            wide = lambda t, one: torch.full((d,), one, dtype=torch.float64) if t is None else t.double().abs()
            g_abs = 1.0 if p["gate"] is None else (p["gate"].double().abs()[:, None] if kind == 1 else p["gate"].double().abs())
            hat_size = (y64.abs() + y64.abs().mean(1, keepdim=True)) * rstd
            a_size = hat_size * wide(p["w_post"], 1.0) + wide(p["b_post"], 0.0)
            r_size = abs(rho) * p["x"].double().abs() + g_abs * a_size
    else:
        r_size = abs(rho) * p["x"].double().abs()
    _close("r", r, r64, r_size, dtype)
    rstd_r = None
    if pre != NONE:
        rd = r64.detach()
        rstd_r = 1.0 / torch.sqrt((((rd - (rd.mean(1, keepdim=True) if pre == LAYER else 0)) ** 2).mean(1, keepdim=True)) + eps)
        w = 1.0 if p["w_pre"] is None else p["w_pre"].double().abs()
        b = 0.0 if p["b_pre"] is None else p["b_pre"].double().abs()
        # an error of one part in 2^24 of r moves hat_r by as much of r / rms; the statistics average over the row
        n_size = (r_size + r_size.mean(1, keepdim=True) + r_size.square().mean(1, keepdim=True).sqrt()) * rstd_r * w * (1 + (rd * rstd_r).abs().clamp(max=1)) + b
        _close("n", n, n64, n_size, dtype)

    loss = 0.0
    if dr is not None:
        loss = loss + (r64 * dr.double()).sum()
    if dn is not None and n64 is not None:
        loss = loss + (n64 * dn.double()).sum()
    loss.backward()
    names = [f"d{k}" for k in ("w_post", "b_post", "w_pre", "b_pre") if p[k] is not None] + (["dgate"] if kind == 2 else [])
    before = {k: torch.full((d,), 0.25 if accumulate else float("nan"), device="cuda") for k in names}
    G = {k: t.clone() for k, t in before.items()}
    args = (q["x"], q["y"], q["gate"], post_norm, pre_norm, device(dr), device(dn), stats)
    dx, dy, dgate = binding.residual_norm_backward(*args, G, residual_scale=rho, accumulate=accumulate, gate_kind=kind)

    # gradients: compared in the 2-norm of the tensor and elementwise against the largest of the row (or of the vector): every element is a
    # difference of terms of the row's size
    def grads_close(name, got, want, vector):
        got, want = got.double().cpu(), want.detach()
        step = torch.finfo(torch.float32 if vector else dtype).eps / 2
        scale = want.abs().max() if vector else _rowmax(want) + _rowmax(leaf_scale[name])
        # fp32 evaluation over rows whose sizes differ by e^+-3: 2^-24 a rounding, a few hundred of them, on terms of `scale`
        err = 512 * 2.0 ** -24 * scale + want.abs() * step * 1.01
        diff = (got - want).abs()
        assert bool((diff <= err).all()), (name, float((diff / err.clamp(min=1e-300)).max()))

    zero = torch.zeros(1, 1, dtype=torch.float64)
    D_size = (dr.double().abs().amax(1, keepdim=True) if dr is not None else zero)
    if dn is not None:
        w = 1.0 if p["w_pre"] is None else p["w_pre"].double().abs().max()
        amplify = (_rowmax(r_size) * rstd_r) if pre != NONE else 1.0
        D_size = D_size + rstd_r * _rowmax(dn.double()) * w * (1 + amplify)
    leaf_scale = {"dx": abs(rho) * D_size}
    grads_close("dx", dx, leaves["x"].grad, False)
    if with_y:
        gmax = 1.0 if p["gate"] is None else (g_abs.amax(-1, keepdim=True) if kind != 2 else g_abs.max())
        wmax = 1.0 if p["w_post"] is None else p["w_post"].double().abs().max()
        leaf_scale["dy"] = D_size * gmax * wmax * rstd * (1 + _rowmax(hat_size))
        grads_close("dy", dy, leaves["y"].grad, False)
        if kind == 1:
            # one number a row: d products D a of either sign add up to it
            err = 512 * 2.0 ** -24 * (D_size * a_size.amax(1, keepdim=True)).squeeze(1) * d ** 0.5 + leaves["gate"].grad.abs() * 2.0 ** -23
            assert bool(((dgate.double().cpu() - leaves["gate"].grad).abs() <= err).all())
        elif kind == 3:
            leaf_scale["dgate"] = D_size * a_size.amax(1, keepdim=True)
            grads_close("dgate", dgate, leaves["gate"].grad, False)
    for name in names:
        grad = leaves[name[1:]].grad                                   # None: not in the function (dn is None), so zero
        want = (torch.zeros(d, dtype=torch.float64) if grad is None else grad) + (0.25 if accumulate else 0.0)
        got = G[name].double().cpu()
        # a column's sum over the rows: as many terms of either sign, each with the rows' errors
        size = D_size.square().sum().sqrt() if name not in ("dw_pre", "db_pre") else (dn.double().abs().amax() * T ** 0.5 if dn is not None else 1.0)
        if name == "dw_pre" and dn is not None:
            size = size * (1 + (_rowmax(r_size) * rstd_r).max())
        if name in ("dw_post", "db_post", "dgate"):
            size = (D_size * (_rowmax(a_size) if name == "dgate" else (gmax * (_rowmax(hat_size) if name == "dw_post" else 1.0)))).square().sum().sqrt()
        err = 512 * 2.0 ** -24 * (size + want.abs().max())
        assert bool(((got - want).abs() <= err).all()), (name, float((got - want).abs().max()), float(err))
    return q


SHAPES = [(1, 1), (1, 2048), (3, 8), (2, 127), (5, 128), (33, 257), (40, 1000), (300, 1024), (64, 1357), (20, 4096), (9, 5000), (6, 8192), (700, 264)]


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("i", range(len(SHAPES)))
def test_shapes(binding, i, dtype):
    T, d = SHAPES[i]
    _run(binding, T, d, dtype, (RMS, LAYER)[i % 2], (RMS, LAYER)[(i // 2) % 2], i % 4, seed=i)


@pytest.mark.parametrize("gate_kind", [0, 1, 2, 3])
@pytest.mark.parametrize("post", [NONE, RMS, LAYER])
@pytest.mark.parametrize("pre", [NONE, RMS, LAYER])
def test_kinds(binding, post, pre, gate_kind):
    _run(binding, 37, 200, torch.bfloat16, post, pre, gate_kind, rho=0.5, seed=post * 3 + pre)
    _run(binding, 37, 72, torch.float32, post, pre, gate_kind, params=False, rho=-1.5, seed=post * 3 + pre)


@pytest.mark.parametrize("pre", [RMS, LAYER])
def test_norm_alone_without_a_block_before(binding, pre):
    _run(binding, 19, 512, torch.bfloat16, NONE, pre, 0, with_y=False, seed=4)
    _run(binding, 19, 30, torch.float32, NONE, pre, 0, with_y=False, rho=2.0, seed=5)


@pytest.mark.parametrize("which", ["dr", "dn"])
def test_one_of_the_two_gradients(binding, which):
    _run(binding, 50, 384, torch.float32, LAYER, RMS, 2, use_dr=which == "dr", use_dn=which == "dn", seed=6)


@pytest.mark.parametrize("pad", [1, 8])
def test_strided_rows(binding, pad):
    _run(binding, 21, 136, torch.bfloat16, RMS, LAYER, 3, ld_pad=pad, seed=7)


def test_accumulated_gradients(binding):
    _run(binding, 400, 136, torch.bfloat16, LAYER, LAYER, 2, accumulate=True, seed=8)


def test_square_gate_is_told_apart_by_its_kind(binding):
    _run(binding, 48, 48, torch.float32, RMS, RMS, 1, seed=9)
    _run(binding, 48, 48, torch.float32, RMS, RMS, 2, seed=9)


def test_gradients_against_differences(binding):
    """Central differences of the GPU's own forward in fp32 (LayerNorm and RMS, all gates), along random directions."""
    g = torch.Generator().manual_seed(3)
    T, d = 6, 40
    for post, pre, kind in ((LAYER, RMS, 1), (RMS, LAYER, 2), (LAYER, LAYER, 3), (NONE, RMS, 0)):
        shapes = {"x": (T, d), "y": (T, d), "w_post": (d,), "b_post": (d,), "w_pre": (d,), "b_pre": (d,)}
        if kind:
            shapes["gate"] = {1: (T,), 2: (d,), 3: (T, d)}[kind]
        p = {k: torch.randn(*s, generator=g).cuda() for k, s in shapes.items()}
        dr, dn = torch.randn(T, d, generator=g).cuda(), torch.randn(T, d, generator=g).cuda()

        def forward(p, training=False):
            norms = binding.Norm(post, p["w_post"], p["b_post"], 1e-3), binding.Norm(pre, p["w_pre"], p["b_pre"], 1e-3)
            return norms, binding.residual_norm_forward(p["x"], p["y"], p.get("gate"), *norms, residual_scale=0.7, training=training, gate_kind=kind)

        norms, (r, n, stats) = forward(p, True)
        G = {k: torch.empty(d, device="cuda") for k in ("dw_post", "db_post", "dw_pre", "db_pre") + (("dgate",) if kind == 2 else ())}
        dx, dy, dgate = binding.residual_norm_backward(p["x"], p["y"], p.get("gate"), *norms, dr, dn, stats, G, residual_scale=0.7, gate_kind=kind)
        grads = dict(x=dx, y=dy, w_post=G["dw_post"], b_post=G["db_post"], w_pre=G["dw_pre"], b_pre=G["db_pre"])
        if kind:
            grads["gate"] = dgate
        for name, grad in grads.items():
            v = torch.randn(shapes[name], generator=g).cuda()
            h = 2.0 ** -7
            value = []
            for sign in (1, -1):
                _, (r, n, _) = forward({**p, name: p[name] + sign * h * v})
                value.append(float((r.double() * dr.double()).sum() + (n.double() * dn.double()).sum()))
            slope, want = (value[0] - value[1]) / (2 * h), float((grad.double() * v.double()).sum())
            # truncation h^2 / 6 times the third derivative (rows of norm about 1: the functional's size), rounding 2^-24 / h a term
            size = float((grad.double().abs() * v.double().abs()).sum()) + T * d
            assert abs(slope - want) <= size * (h * h + 2.0 ** -24 / h * 4), (name, post, pre, kind, slope, want)


def test_rows_of_zeros_and_non_finite_rows(binding):
    """A row of zeros has the norm b; infinities and NaN stay in their row, but for the column sums of the gradients."""
    T, d = 6, 264
    x = torch.randn(T, d, device="cuda", dtype=torch.bfloat16)
    y = torch.randn(T, d, device="cuda", dtype=torch.bfloat16)
    x[1], y[1] = 0, 0
    x[2, 5], y[3, 7], y[4] = float("inf"), float("nan"), torch.finfo(torch.bfloat16).min
    w, b = torch.randn(d, device="cuda"), torch.randn(d, device="cuda")
    for kind in (RMS, LAYER):
        post, pre = binding.Norm(kind, w), binding.Norm(kind, w, b)
        r, n, stats = binding.residual_norm_forward(x, y, None, post, pre, training=True)
        assert torch.equal(r[1], torch.zeros_like(r[1])) and torch.equal(n[1], b.to(torch.bfloat16))
        good = [0, 1, 5]
        r1, n1, _ = binding.residual_norm_forward(x[good], y[good], None, post, pre)
        assert torch.equal(r[good], r1) and torch.equal(n[good], n1)
        dr = torch.randn(T, d, device="cuda", dtype=torch.bfloat16)
        dx, dy, _ = binding.residual_norm_backward(x, y, None, post, pre, dr, dr, stats)
        _, _, s1 = binding.residual_norm_forward(x[good], y[good], None, post, pre, training=True)
        dx1, dy1, _ = binding.residual_norm_backward(x[good], y[good], None, post, pre, dr[good].contiguous(), dr[good].contiguous(), s1)
        assert torch.equal(dx[good], dx1) and torch.equal(dy[good], dy1)
        assert not bool(torch.isfinite(n[3].float()).any())


def test_in_place(binding):
    T, d = 333, 1024
    x = torch.randn(T, d, device="cuda", dtype=torch.bfloat16)
    y = torch.randn(T, d, device="cuda", dtype=torch.bfloat16)
    post, pre = binding.Norm(LAYER), binding.Norm(RMS)
    r, n, _ = binding.residual_norm_forward(x, y, None, post, pre)
    binding.residual_norm_forward(x, y, None, post, pre, r=x, n=y)
    assert torch.equal(r, x) and torch.equal(n, y)


def test_no_rows(binding):
    e = torch.empty(0, 64, device="cuda", dtype=torch.bfloat16)
    post, pre = binding.Norm(RMS, torch.ones(64, device="cuda")), binding.Norm(RMS, torch.ones(64, device="cuda"))
    r, n, stats = binding.residual_norm_forward(e, e, None, post, pre, training=True)
    assert r.shape == n.shape == (0, 64)
    for accumulate, want in ((False, 0.0), (True, 7.0)):
        G = {k: torch.full((64,), 7.0, device="cuda") for k in ("dw_post", "dw_pre")}
        binding.residual_norm_backward(e, e, None, post, pre, e, e, stats, G, accumulate=accumulate)
        assert all(bool((t == want).all()) for t in G.values())


def test_repeats_itself_and_replays(binding):
    T, d = 1500, 512
    g = torch.Generator(device="cuda").manual_seed(1)
    x, y, dr, dn = (torch.randn(T, d, device="cuda", generator=g).bfloat16() for _ in range(4))
    gate = torch.randn(d, device="cuda", generator=g)
    post, pre = binding.Norm(RMS, torch.randn(d, device="cuda", generator=g)), binding.Norm(LAYER, torch.randn(d, device="cuda", generator=g), gate)

    def step():
        G = {k: torch.empty(d, device="cuda") for k in ("dw_post", "dw_pre", "db_pre", "dgate")}
        r, n, stats = binding.residual_norm_forward(x, y, gate, post, pre, training=True)
        dx, dy, _ = binding.residual_norm_backward(x, y, gate, post, pre, dr, dn, stats, G)
        return [r, n, dx, dy, *G.values()]

    first = step()
    assert all(torch.equal(a, b) for a, b in zip(first, step()))
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            out = step()
    torch.cuda.current_stream().wait_stream(side)
    graph.replay()
    assert all(torch.equal(a, b) for a, b in zip(first, out))
    x.neg_()
    graph.replay()
    assert all(torch.equal(a, b) for a, b in zip(step(), out))


def test_binding_refuses_mismatched_tensors(binding):
    x, v = torch.zeros(4, 8, device="cuda"), torch.zeros(8, device="cuda")
    for kw in (dict(x=v), dict(y=torch.zeros(4, 9, device="cuda")), dict(y=x.bfloat16()), dict(gate=torch.zeros(5, device="cuda")),
               dict(gate=torch.zeros(4, 7, device="cuda")), dict(gate=x, gate_kind=1), dict(gate=v.bfloat16()), dict(post=binding.Norm(1, v[:4])),
               dict(pre=binding.Norm(1, v.double())), dict(pre=binding.Norm(1, v.cpu())), dict(y=x.cpu()), dict(x=x.t(), y=x.t()), dict(x=x.half(), y=x.half())):
        kw = {"x": x, "y": x, **kw}
        with pytest.raises(ValueError):
            binding.residual_norm_forward(**kw)
    r, n, stats = binding.residual_norm_forward(x, x, None, binding.Norm(1), binding.Norm(1), training=True)
    for bad in (None, stats[:3], stats.double()):
        with pytest.raises(ValueError):
            binding.residual_norm_backward(x, x, None, binding.Norm(1), binding.Norm(1), r, n, bad)


@pytest.mark.parametrize("T,d", [(310, 4095), (310, 4096), (310, 4097), (310, 8192), (310, 8191), (700, 1281), (700, 1280), (700, 1288)])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_many_rows_with_everything(binding, T, d, dtype):
    """Both LayerNorms with weights and biases and a gate for every element, more rows than are worked on at once: the most shared memory that a
    row of each layout takes."""
    _run(binding, T, d, dtype, LAYER, LAYER, 3, seed=d)


@pytest.mark.parametrize("T,d", [(310, 8192), (310, 4104), (310, 5000)])
@pytest.mark.parametrize("gate_kind", [0, 1, 2, 3])
def test_many_wide_rows_without_parameters(binding, T, d, gate_kind):
    """No biases: rows of more than 4096 columns through shared memory in the backward, too."""
    _run(binding, T, d, torch.bfloat16, RMS, RMS, gate_kind, params=False, seed=d)
    _run(binding, T, d, torch.bfloat16, LAYER, NONE, gate_kind, params=False, seed=d + 1)
