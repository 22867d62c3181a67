"""The operators around and inside the MoE layer whose speed is followed, each with its plain form.

norm      the joint between two blocks: r = rho x + gate * N_post(y), n = N_pre(r), forward, and for training its backward
          (`binding.residual_norm_forward` / `residual_norm_backward`).
quantise  rows to microscaled 4-bit floating point (blocks of 32 along the row: e2m1 elements, one power-of-two scale) and back
          (`binding.mx4_quantize` / `mx4_dequantize`).
product   y = Q(x) W^T with a 4-bit W that a serving program holds laid out (`binding.mx4_quantize` / `mx4_matmul`).
experts   a product of the experts over the segments of a routing (the same two calls): the first one, a = sigma(Q(x'[token of
          row]) W1_e^T), whose rows are gathered while they are quantised, or the second, u = Q(a) W2_e^T.

Widths are those of the configurations of `paper_2502_16927_b200/workloads.py`: small (d 1024, 32 experts, top-4, r 128, h 512),
medium (d 2048, 64 experts, top-8, r 256, h 1024), large (d 4096, 128 experts, top-8, r 512, h 2048), tiny (d 128, fp32).
Activations are N(0, 1), the output of a block somewhat smaller, upstream gradients N(0, 1), weights N(0, 1/fan_in), weights of
norms about 1, gates as a sigmoid gives them.
"""
import math

import torch

own = False

SMALL, MEDIUM, LARGE = (dict(d=1024, r=128, h=512, E=32, k=4), dict(d=2048, r=256, h=1024, E=64, k=8),
                        dict(d=4096, r=512, h=2048, E=128, k=8))
EPS = 1e-6


def _norm(T, d, kind, gate, train, dtype="bf16", rho=1.0):
    return dict(path="norm", T=T, d=d, kind=kind, gate=gate, train=train, dtype=dtype, rho=rho)


def _quantise(T, K, dtype="bf16"):
    return dict(path="quantise", T=T, K=K, dtype=dtype)


def _product(T, N, K):
    return dict(path="product", T=T, N=N, K=K)


def _experts(T, widths, skewed, second=False):
    """The experts' first product (r -> h, with GELU), or their second (h -> r, of rows that lie by expert already)."""
    return dict(path="experts", T=T, K=widths["h"] if second else widths["r"], N=widths["r"] if second else widths["h"], E=widths["E"],
                k=widths["k"], skewed=skewed, second=second)


def listed():
    return [
        # Generation: the joint after one block and before the next, for one new token and for a full server's.
        dict(_norm(1, 2048, "rms", "none", False), name="norm decode 1"),
        dict(_norm(512, 2048, "layer", "token", False), name="norm decode 512"),
        # Training steps, forward and backward: the fp32 configuration, a batch of documents packed without padding, the
        # large widths with a gate for every element.
        dict(_norm(256, 128, "layer", "channel", True, dtype="fp32", rho=0.5), name="norm train fp32 256"),
        dict(_norm(2999, 1024, "rms", "channel", True), name="norm train 2999"),
        dict(_norm(16384, 4096, "rms", "full", True), name="norm train 16384"),
        # Activations to 4 bits and back: a small batch, a long prompt.
        dict(_quantise(64, 2048), name="quantise 64"),
        dict(_quantise(16384, 4096), name="quantise 16384"),
        # A dense layer with 4-bit weights: one new token, a batch of short prompts, long ones.
        dict(_product(1, 4096, 4096), name="product 1"),
        dict(_product(300, 2048, 2048), name="product 300"),
        dict(_product(16384, 4096, 4096), name="product 16384"),
        # The experts' products: 64 running sequences (about eight rows an expert), a long batch with uneven loads.
        dict(_experts(64, MEDIUM, False), name="experts 64"),
        dict(_experts(16384, MEDIUM, True), name="experts 16384"),
    ]


def _log_uniform(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    path = rng.choice(["norm", "norm", "norm", "quantise", "product", "product", "experts", "experts"])
    if path == "norm":
        train = rng.random() < 0.6
        d = rng.choice([128, 1024, 2048, 4096, 8 * _log_uniform(rng, 8, 512), _log_uniform(rng, 100, 4000)])
        kind, gate = rng.choice(["rms", "layer"]), rng.choice(["none", "token", "channel", "full"])
        dtype = rng.choice(["bf16", "bf16", "bf16", "fp32"])
        return _norm(_log_uniform(rng, 1, 16000 if dtype == "bf16" else 8000), d, kind, gate, train, dtype, rng.choice([1.0, 1.0, 0.5]))
    if path == "quantise":
        return _quantise(_log_uniform(rng, 1, 16000), 32 * _log_uniform(rng, 1, 128), rng.choice(["bf16", "bf16", "fp32"]))
    if path == "product":
        N = rng.choice([512, 1024, 2048, 4096, _log_uniform(rng, 100, 4000)])
        return _product(_log_uniform(rng, 1, 16000), N, rng.choice([512, 1024, 2048, 4096, 32 * _log_uniform(rng, 4, 128)]))
    return _experts(_log_uniform(rng, 1, 16000), rng.choice([SMALL, MEDIUM]), rng.random() < 0.5, rng.random() < 0.3)


# ---- inputs ---------------------------------------------------------------------------------------------

_DTYPE = {"bf16": torch.bfloat16, "fp32": torch.float32}


def _pack_scales(e8m0):
    """[..., rows, K / 32] scale bytes in the layout the product reads: tiles of 128 rows by 4 blocks, in a tile byte
    (row % 32) * 16 + (row // 32) * 4 + block."""
    *lead, rows, blocks = e8m0.shape
    rt, kt = -(-rows // 128), -(-blocks // 4)
    full = torch.zeros(*lead, rt * 128, kt * 4, dtype=torch.uint8, device=e8m0.device)
    full[..., :rows, :blocks] = e8m0
    n = len(lead)
    full = full.reshape(*lead, rt, 4, 32, kt, 4)                        # row tile, 32-row group, row, block tile, block
    return full.permute(*range(n), n, n + 3, n + 2, n + 1, n + 4).contiguous().reshape(*lead, rt, kt, 512)


def _unpack_scales(packed, rows, blocks):
    *lead, rt, kt, _ = packed.shape
    n = len(lead)
    full = packed.reshape(*lead, rt, kt, 32, 4, 4).permute(*range(n), n, n + 3, n + 2, n + 1, n + 4)
    return full.reshape(*lead, rt * 128, kt * 4)[..., :rows, :blocks]


def _four_bit(x):
    """Plain quantisation of fp32 rows: (codes 0..15, scale bytes).  The scale of a block of 32 is 2^(floor(log2 max |x|) - 2), the
    largest power of two that puts the block's largest magnitude into [4, 8); magnitudes are rounded to the nearest of
    0 0.5 1 1.5 2 3 4 6 (ties to the even code), those above 6 to 6."""
    blocks = x.reshape(*x.shape[:-1], x.shape[-1] // 32, 32)
    biased = (blocks.abs().amax(-1).contiguous().view(torch.int32) >> 23).to(torch.int32) - 2
    byte = biased.clamp(min=0)
    inverse = ((254 - byte) << 23).view(torch.float32)                # 2^(127 - byte), by its bits: exact
    v = blocks.abs() * inverse.unsqueeze(-1)
    code = (v > 0.25).to(torch.uint8)
    for at, even_above in ((0.75, True), (1.25, False), (1.75, True), (2.5, False), (3.5, True), (5.0, False)):
        code += (v >= at) if even_above else (v > at)
    code += (blocks < 0).to(torch.uint8) * 8
    return code.reshape(x.shape), byte.to(torch.uint8)


def _values(code, byte):
    """The numbers that codes and scale bytes stand for, in fp32."""
    m = (code & 7).int()
    v = torch.where(m < 2, 0.5 * m, ((m + 252) << 22).view(torch.float32))     # from code 2 on: exponent and one bit of mantissa
    v = torch.where(code > 7, -v, v)
    scale = byte.int() << 23                                          # 2^(byte - 127), by its bits; byte 0 is a subnormal
    scale = torch.where(byte == 0, 1 << 22, scale).to(torch.int32).view(torch.float32)
    return (v.reshape(*byte.shape, 32) * scale.unsqueeze(-1)).reshape(code.shape)


def _weights_4bit(w):
    code, byte = _four_bit(w.float())
    return (code[..., 0::2] | (code[..., 1::2] << 4)).contiguous(), _pack_scales(byte)


def _read_weights(codes, scales):
    code = torch.stack((codes & 15, codes >> 4), dim=-1).reshape(*codes.shape[:-1], 2 * codes.shape[-1])
    return _values(code, _unpack_scales(scales, codes.shape[-2], codes.shape[-1] // 16))


def prepare(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)

    def normal(*shape, std=1.0, mean=0.0):
        return torch.randn(*shape, generator=gen, device="cuda").mul_(std).add_(mean)

    T, path = case["T"], case["path"]
    s = {"case": case}
    if path == "norm":
        d, dt = case["d"], _DTYPE[case["dtype"]]
        # a residual stream with some large channels, a block's output, the norms' weights (and a LayerNorm's biases)
        s["x"] = (normal(T, d) * normal(d, std=0.5).exp()).to(dt)
        s["y"] = normal(T, d, std=0.4, mean=0.05).to(dt)
        s["w_post"], s["w_pre"] = normal(d, std=0.1, mean=1.0), normal(d, std=0.1, mean=1.0)
        layer = case["kind"] == "layer"
        s["b_post"], s["b_pre"] = (normal(d, std=0.1), normal(d, std=0.1)) if layer else (None, None)
        s["gate"] = {"none": lambda: None, "token": lambda: torch.sigmoid(normal(T)), "channel": lambda: normal(d, std=0.1, mean=0.5),
                     "full": lambda: torch.sigmoid(normal(T, d)).to(dt)}[case["gate"]]()
        if case["train"]:
            s["dr"], s["dn"] = normal(T, d).to(dt), normal(T, d).to(dt)
            # gradient buffers of the parameters, which the training program owns
            s["G"] = {n: torch.empty(d, device="cuda") for n in ("dw_post", "dw_pre") + (("db_post", "db_pre") if layer else ())
                      + (("dgate",) if case["gate"] == "channel" else ())}
    elif path == "quantise":
        s["x"] = (normal(T, case["K"]) * normal(T, 1).exp()).to(_DTYPE[case["dtype"]])
    elif path == "product":
        s["x"] = normal(T, case["K"]).to(torch.bfloat16)
        s["codes"], s["scales"] = _weights_4bit(normal(case["N"], case["K"], std=case["K"] ** -0.5))
    else:
        E, k, K = case["E"], case["k"], case["K"]
        s["codes"], s["scales"] = _weights_4bit(normal(E, case["N"], K, std=K ** -0.5))
        # the tables of a routing: k experts a token by the largest logits, rows sorted by expert, tokens in order
        logits = normal(T, E)
        if case["skewed"]:
            logits = logits - 1.1 * torch.log(torch.arange(1, E + 1, device="cuda"))
        chosen = torch.topk(logits, k, dim=1).indices.reshape(-1)
        s["slot_of_row"] = torch.sort(chosen, stable=True).indices.to(torch.int32)
        counts = torch.bincount(chosen, minlength=E)
        s["offsets"] = torch.cat((torch.zeros(1, dtype=torch.int64, device="cuda"), counts.cumsum(0))).to(torch.int32)
        s["counts"] = counts.tolist()
        s["x"] = normal(T * k if case["second"] else T, K).to(torch.bfloat16)
    return s


# ---- plain forms ------------------------------------------------------------------------------------------

def _stats(v, kind):
    mean = v.mean(-1, keepdim=True) if kind == "layer" else torch.zeros_like(v[:, :1])
    return mean, torch.rsqrt(((v - mean) ** 2).mean(-1, keepdim=True) + EPS)


def _norm_backward(da, hat, rstd, w, kind):
    g = da * w
    inner = g - hat * (g * hat).mean(-1, keepdim=True)
    return rstd * (inner - g.mean(-1, keepdim=True) if kind == "layer" else inner)


def _plain_norm(s):
    case = s["case"]
    kind, dt = case["kind"], _DTYPE[case["dtype"]]
    x, y = s["x"].float(), s["y"].float()
    gate = s["gate"]
    if gate is not None:
        gate = gate.float()
        gate = gate.unsqueeze(1) if case["gate"] == "token" else gate
    mean, rstd = _stats(y, kind)
    hat = (y - mean) * rstd
    a = hat * s["w_post"]
    if s["b_post"] is not None:
        a = a + s["b_post"]
    r = case["rho"] * x + (a if gate is None else gate * a)
    mean_r, rstd_r = _stats(r, kind)
    hat_r = (r - mean_r) * rstd_r
    n = hat_r * s["w_pre"]
    if s["b_pre"] is not None:
        n = n + s["b_pre"]
    out = {"r": r.to(dt), "n": n.to(dt)}
    if not case["train"]:
        return out
    dn = s["dn"].float()
    D = s["dr"].float() + _norm_backward(dn, hat_r, rstd_r, s["w_pre"], kind)
    out["dx"] = (case["rho"] * D).to(dt)
    da = D if gate is None else gate * D
    out["dy"] = _norm_backward(da, hat, rstd, s["w_post"], kind).to(dt)
    out["dw_post"], out["dw_pre"] = (da * hat).sum(0), (dn * hat_r).sum(0)
    if s["b_post"] is not None:
        out["db_post"], out["db_pre"] = da.sum(0), dn.sum(0)
    if case["gate"] == "token":
        out["dgate"] = (D * a).sum(1)
    elif case["gate"] == "channel":
        out["dgate"] = (D * a).sum(0)
    elif case["gate"] == "full":
        out["dgate"] = (D * a).to(dt)
    return out


def _gelu(z):
    return 0.5 * z * (1.0 + torch.erf(z * 0.5 ** 0.5))


def run(state):
    return _run_own(state) if own else _run_plain(state)


def _run_plain(s):
    case = s["case"]
    if case["path"] == "norm":
        return _plain_norm(s)
    q = _values(*_four_bit(s["x"].float()))
    if case["path"] == "quantise":
        return q.to(s["x"].dtype)
    W = _read_weights(s["codes"], s["scales"])
    if case["path"] == "product":
        return (q @ W.t()).to(torch.bfloat16)
    rows = q if case["second"] else q[s["slot_of_row"].long() // case["k"]]
    z = torch.empty(rows.shape[0], case["N"], device="cuda")
    at = 0
    for e, n in enumerate(s["counts"]):
        if n:
            torch.mm(rows[at:at + n], W[e].t(), out=z[at:at + n])
        at += n
    return (z if case["second"] else _gelu(z)).to(torch.bfloat16)


def _run_own(s):
    from paper_2502_16927_b200 import binding
    from paper_2502_16927_b200.workloads import ACT_GELU_ERF, ACT_IDENTITY

    case = s["case"]
    if case["path"] == "norm":
        kind = binding.BIGMAC_NORM_LAYER if case["kind"] == "layer" else binding.BIGMAC_NORM_RMS
        post, pre = binding.Norm(kind, s["w_post"], s["b_post"], EPS), binding.Norm(kind, s["w_pre"], s["b_pre"], EPS)
        r, n, stats = binding.residual_norm_forward(s["x"], s["y"], s["gate"], post, pre, residual_scale=case["rho"], training=case["train"])
        out = {"r": r, "n": n}
        if case["train"]:
            dx, dy, dgate = binding.residual_norm_backward(s["x"], s["y"], s["gate"], post, pre, s["dr"], s["dn"], stats, s["G"],
                                                           residual_scale=case["rho"])
            out.update(s["G"], dx=dx, dy=dy)
            if dgate is not None:
                out["dgate"] = dgate
        return out
    if case["path"] == "quantise":
        return binding.mx4_dequantize(binding.mx4_quantize(s["x"]), s["x"].dtype)
    W = binding.Mx4(s["codes"], s["scales"])
    if case["path"] == "product":
        return binding.mx4_matmul(binding.mx4_quantize(s["x"]), W)
    rows = {} if case["second"] else {"slot_of_row": s["slot_of_row"], "k": case["k"]}
    return binding.mx4_matmul(binding.mx4_quantize(s["x"], offsets=s["offsets"], **rows), W, act=ACT_IDENTITY if case["second"] else ACT_GELU_ERF)


# ---- what a pass cannot do without, and its value in 64 bits -------------------------------------------------

def work(case):
    T = case["T"]
    if case["path"] == "norm":
        d, es = case["d"], 2 if case["dtype"] == "bf16" else 4
        gate = {"none": 0, "token": 4.0 * T, "channel": 4.0 * d, "full": 1.0 * T * d * es}[case["gate"]]
        params = 4.0 * d * (4 if case["kind"] == "layer" else 2)
        # forward: x, y -> r, n; a step also dr, dn -> dx, dy and, once more, x and y
        forward = 4.0 * T * d * es + gate + params
        if not case["train"]:
            return {"bytes": forward, "flops": 16.0 * T * d}
        return {"bytes": forward + 6.0 * T * d * es + 2 * gate + 2 * params, "flops": 56.0 * T * d}
    if case["path"] == "quantise":
        return {"bytes": T * case["K"] * (2 if case["dtype"] == "bf16" else 4) * 2.0, "flops": 4.0 * T * case["K"]}
    K, N = case["K"], case["N"]
    if case["path"] == "product":
        return {"bytes": 2.0 * T * K + 2.0 * T * N + N * K * 17 / 32, "flops": 2.0 * T * N * K}
    rows, E = T * case["k"], case["E"]
    experts = E * (1.0 - (1.0 - case["k"] / E) ** T)                  # chosen by a batch of this size (even loads)
    return {"bytes": 2.0 * K * (rows if case["second"] else T) + 2.0 * rows * N + experts * N * K * 17 / 32 + 4.0 * rows + 4.0 * E,
            "flops": 2.0 * rows * N * K}


def _power_of_two(exponent):
    return ((exponent.long() + 1023) << 52).view(torch.float64)


def _nearest(x):
    """The 4-bit values of rows in 64 bits, by distance: of the eight magnitudes the nearest, of two equally near ones the
    one with the even place in the list."""
    blocks = x.double().reshape(*x.shape[:-1], -1, 32)
    exponent = torch.frexp(blocks.abs().amax(-1, keepdim=True)).exponent.clamp(min=-124) - 3     # frexp: mantissa in [1/2, 1)
    scale = _power_of_two(exponent)
    v = (blocks.abs() / scale).clamp(max=6.0)
    best, gap = torch.zeros_like(v), v.clone()                        # the first magnitude, 0
    for place, m in enumerate((0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0), start=1):
        away = (v - m).abs()
        nearer = (away < gap) | ((away == gap) & (place % 2 == 0))
        best, gap = torch.where(nearer, torch.full_like(v, m), best), torch.where(nearer, away, gap)
    return (best * scale * torch.sign(blocks)).reshape(x.shape)


def exact(case, seed):
    s = prepare(case, seed)
    if case["path"] == "quantise":
        return _nearest(s["x"])
    if case["path"] in ("product", "experts"):
        rows = _nearest(s["x"])
        low, high = s["codes"] % 16, s["codes"] // 16
        grid = torch.tensor([0, 0.5, 1, 1.5, 2, 3, 4, 6], dtype=torch.float64, device="cuda")
        byte = torch.empty(*s["codes"].shape[:-1], s["codes"].shape[-1] // 16, dtype=torch.int64, device="cuda")
        r, b = torch.meshgrid(torch.arange(byte.shape[-2], device="cuda"), torch.arange(byte.shape[-1], device="cuda"), indexing="ij")
        byte[...] = s["scales"][..., r // 128, b // 4, (r % 32) * 16 + (r % 128) // 32 * 4 + b % 4].long()
        W = torch.empty(*s["codes"].shape[:-1], 2 * s["codes"].shape[-1], dtype=torch.float64, device="cuda")
        for first, nibble in ((0, low), (1, high)):
            W[..., first::2] = grid[(nibble % 8).long()] * (1 - 2 * (nibble // 8).double())
        W *= _power_of_two(byte - 127).repeat_interleave(32, dim=-1)
        if case["path"] == "product":
            return rows @ W.t()
        if not case["second"]:
            rows = rows[torch.div(s["slot_of_row"], case["k"], rounding_mode="floor").long()]
        z = torch.cat([part @ W[e].t() for e, part in enumerate(rows.split(s["counts"]))])
        return z if case["second"] else z * torch.special.ndtr(z)

    # the joint from its definition; its gradients by automatic differentiation
    def leaf(t):
        return None if t is None else t.double().requires_grad_(case["train"])

    x, y, gate = leaf(s["x"]), leaf(s["y"]), leaf(s["gate"])
    params = {n: leaf(s[n]) for n in ("w_post", "b_post", "w_pre", "b_pre")}

    def normalised(v, w, b):
        if case["kind"] == "layer":
            v = v - v.mean(1, keepdim=True)
        v = v / torch.sqrt(v.square().mean(1, keepdim=True) + EPS) * w
        return v if b is None else v + b

    a = normalised(y, params["w_post"], params["b_post"])
    if gate is not None:
        a = a * (gate[:, None] if case["gate"] == "token" else gate)
    r = case["rho"] * x + a
    n = normalised(r, params["w_pre"], params["b_pre"])
    out = {"r": r.detach(), "n": n.detach()}
    if case["train"]:
        ((r * s["dr"].double()).sum() + (n * s["dn"].double()).sum()).backward()
        out.update(dx=x.grad, dy=y.grad, **{"d" + p: t.grad for p, t in params.items() if t is not None})
        if gate is not None:
            out["dgate"] = gate.grad
    return out
