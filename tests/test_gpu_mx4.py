"""Microscaled 4-bit matrices on the GPU against their definition in 64 bits: codes, scale bytes, values, products."""
import numpy as np
import pytest
import torch

import mx4_reference as ref

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def binding():
    from paper_2502_16927_b200 import binding as b

    return b


def _gen(seed):
    return np.random.default_rng(seed)


def _rows(rng, rows, K, dtype):
    """Rows of very different size, some blocks all zero, some tiny, some with ties and values between 6 and 8 scales."""
    x = rng.standard_normal((rows, K)) * np.exp(rng.standard_normal((rows, 1)) * 3)
    b = x.reshape(rows, K // 32, 32)
    b[rng.random(b.shape[:2]) < 0.05] = 0.0
    b[rng.random(b.shape[:2]) < 0.05] *= 2.0 ** -130                   # subnormal in fp32 and bf16
    grid = rng.random(b.shape[:2]) < 0.2                               # quarters up to 8: every tie there is
    b[grid] = rng.integers(-32, 33, (int(grid.sum()), 32)) / 4.0
    t = torch.from_numpy(x.reshape(rows, K).astype(np.float32)).to(dtype)
    return t, t.float().numpy().astype(np.float64)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("rows,K", [(1, 32), (1, 2048), (3, 96), (127, 160), (128, 128), (129, 256), (300, 1056), (1000, 4096)])
def test_quantise_and_read_back(binding, rows, K, dtype):
    x, x64 = _rows(_gen(rows * 7 + K), rows, K, dtype)
    code, byte = ref.quantise(x64)
    q = binding.mx4_quantize(x.cuda())
    got = q.codes.cpu().numpy()
    np.testing.assert_array_equal(got, ref.pack_codes(code))
    want = ref.pack_scales(byte)
    have = q.scales.cpu().numpy()
    used = np.zeros(want.size, dtype=bool)
    kt = want.shape[1]
    for m in range(rows):                                              # bytes behind the last block of a row are zero, too
        at = (np.arange(kt * 4) // 4 + (m // 128) * kt) * 512 + (m % 32) * 16 + (m // 32 % 4) * 4 + np.arange(kt * 4) % 4
        used[at] = True
    np.testing.assert_array_equal(have.reshape(-1)[used], want.reshape(-1)[used])
    for out in (torch.bfloat16, torch.float32):
        y = binding.mx4_dequantize(q, out)
        np.testing.assert_array_equal(y.double().cpu().numpy(), ref.values(code, byte))


def test_non_finite_blocks_and_negative_zero(binding):
    x = torch.zeros(4, 96, dtype=torch.float32)
    x[0, 5], x[1, 40], x[2, 95], x[3, 0] = float("nan"), float("inf"), -float("inf"), -0.0
    x[0, 33], x[3, 1] = 3.0, 3.4e38
    q = binding.mx4_quantize(x.cuda())
    code, byte = ref.quantise(x.numpy())
    np.testing.assert_array_equal(q.codes.cpu().numpy(), ref.pack_codes(code))
    y = binding.mx4_dequantize(q, torch.float32).cpu().numpy()
    np.testing.assert_array_equal(y, ref.values(code, byte).astype(np.float32))
    assert np.isnan(y[0, :32]).all() and np.isnan(y[1, 32:64]).all() and np.isnan(y[2, 64:]).all()
    assert np.isfinite(y[0, 32:]).all() and np.isfinite(y[3]).all()


def test_strided_rows(binding):
    x, x64 = _rows(_gen(5), 40, 128, torch.bfloat16)
    wide = torch.full((40, 136), 7.0, dtype=torch.bfloat16, device="cuda")
    wide[:, :128] = x.cuda()
    code, byte = ref.quantise(x64)
    q = binding.mx4_quantize(wide[:, :128])
    np.testing.assert_array_equal(q.codes.cpu().numpy(), ref.pack_codes(code))
    out = torch.full((40, 144), 9.0, dtype=torch.float32, device="cuda")
    binding.mx4_dequantize(q, out=out[:, :128])
    np.testing.assert_array_equal(out[:, :128].double().cpu().numpy(), ref.values(code, byte))
    assert bool((out[:, 128:] == 9.0).all())


def _weights(rng, lead, N, K):
    code = rng.integers(0, 16, (*lead, N, K))
    byte = rng.integers(118, 131, (*lead, N, K // 32))
    flat = byte.reshape(-1, N, K // 32)
    scales = np.stack([ref.pack_scales(b) for b in flat]).reshape(*lead, -(-N // 128), -(-K // 128), 512)
    return code, byte, torch.from_numpy(ref.pack_codes(code)).cuda(), torch.from_numpy(scales).cuda()


def _act(z, act):
    if act == 0:
        return np.maximum(z, 0)
    if act == 1:
        from scipy.special import erfc
        return 0.5 * z * erfc(-z / np.sqrt(2))
    if act == 2:
        return 0.5 * z * (1 + np.tanh(np.sqrt(2 / np.pi) * (z + 0.044715 * z ** 3)))
    return z


def _check_product(got, a, w, act, dtype):
    """got against act(a w^T).  Products of two elements and their scales are exact.  An instruction adds 64 of them to the
    accumulator and keeps 24 bits or more of the sum, cut or rounded: at most 2^-23 of the largest partial sum, itself at most
    S = sum |a w|, for each of the K / 64 instructions and two more for the order inside one.  The activations' slope is below 1.13 and
    fp32 evaluation of them adds below 2^-20 of |z| (sums of 1 + erf or 1 + tanh cancel to an absolute error of a few units of 1); the rounding to the
    output adds half a step."""
    z = a @ w.T
    S = np.abs(a) @ np.abs(w).T
    K = a.shape[1]
    want = _act(z, act)
    err = 1.13 * (K / 64 + 2) * 2.0 ** -23 * S + (np.abs(z) * 2.0 ** -20 if act in (1, 2) else 0)
    # GELU of a bf16 output is a polynomial under saturation, off by less than 3.6e-5: its minimax error and its fp32 evaluation, looked at on
    # four million points of [-40, 40]; outside Phi is 0 or 1 and so is the polynomial's sum
    err += 3.6e-5 if act == 1 and dtype == torch.bfloat16 else 0
    err += np.abs(want) * torch.finfo(dtype).eps / 2 * 1.01
    diff = np.abs(got.double().cpu().numpy() - want)
    assert (diff <= err).all(), (float((diff - err).max()), float((diff / np.maximum(np.abs(want), 1e-30)).max()))


SHAPES = [(1, 64, 32), (1, 4096, 4096), (5, 40, 96), (33, 128, 256), (64, 100, 160), (97, 257, 288), (128, 192, 512), (129, 65, 1024),
          (300, 333, 416), (1000, 1000, 320), (2500, 4096, 224)]


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("M,N,K", SHAPES)
def test_product(binding, M, N, K, dtype):
    rng = _gen(M * 31 + N + K)
    x, x64 = _rows(rng, M, K, torch.bfloat16)
    x64[np.abs(x64) < 2.0 ** -100] = 0                                 # products with subnormal scales underflow: not meant here
    x = torch.from_numpy(x64.astype(np.float32)).to(torch.bfloat16)
    wc, wb, codes, scales = _weights(rng, (), N, K)
    out = torch.full((M + 1, N), 5.0, dtype=dtype, device="cuda")
    y = binding.mx4_matmul(binding.mx4_quantize(x.cuda()), binding.Mx4(codes, scales), out=out[:M])
    a = ref.values(*ref.quantise(x64))
    _check_product(y, a, ref.values(wc, wb), 3, dtype)
    assert bool((out[M] == 5.0).all())
    assert binding.operator_status() == 0


# enough 256 x 256 tiles for CTA pairs: an odd number of row tiles, ragged columns and K tiles, rows that are no multiple of 16 bytes
@pytest.mark.parametrize("M,N,K", [(2400, 2000, 544), (4700, 1111, 1056), (2304, 2304, 512), (19000, 200, 640)])
def test_product_on_cta_pairs(binding, M, N, K):
    rng = _gen(M + N + K)
    x64 = np.round(rng.standard_normal((M, K)) * 16) / 16
    wc, wb, codes, scales = _weights(rng, (), N, K)
    q, W = binding.mx4_quantize(torch.from_numpy(x64).to(torch.bfloat16).cuda()), binding.Mx4(codes, scales)
    a, w = ref.values(*ref.quantise(x64)), ref.values(wc, wb)
    for act, dtype in ((3, torch.float32), (3, torch.bfloat16), (1, torch.bfloat16), (0, torch.bfloat16)):
        out = torch.full((M + 1, N), 5.0, dtype=dtype, device="cuda")
        binding.mx4_matmul(q, W, act=act, out=out[:M])
        _check_product(out[:M], a, w, act, dtype)
        assert bool((out[M] == 5.0).all())
    assert torch.equal(out[:M], binding.mx4_matmul(q, W, act=0))
    assert binding.operator_status() == 0


@pytest.mark.parametrize("act", [0, 1, 2])
def test_product_with_activation(binding, act):
    rng = _gen(act)
    x64 = np.round(rng.standard_normal((70, 256)) * 64) / 64
    wc, wb, codes, scales = _weights(rng, (), 200, 256)
    wb = wb * 0 + 123
    scales = torch.from_numpy(ref.pack_scales(wb)).cuda()
    y = binding.mx4_matmul(binding.mx4_quantize(torch.from_numpy(x64).float().cuda()), binding.Mx4(codes, scales), act=act, dtype=torch.float32)
    _check_product(y, ref.values(*ref.quantise(x64)), ref.values(wc, wb), act, torch.float32)


def test_product_strided_output(binding):
    rng = _gen(11)
    x, x64 = _rows(rng, 50, 64, torch.bfloat16)
    x64[np.abs(x64) < 2.0 ** -100] = 0
    wc, wb, codes, scales = _weights(rng, (), 70, 64)
    out = torch.full((50, 75), 5.0, dtype=torch.float32, device="cuda")
    binding.mx4_matmul(binding.mx4_quantize(torch.from_numpy(x64).float().cuda()), binding.Mx4(codes, scales), out=out[:, :70])
    _check_product(out[:, :70], ref.values(*ref.quantise(x64)), ref.values(wc, wb), 3, torch.float32)
    assert bool((out[:, 70:] == 5.0).all())


def test_nan_scales_stay_in_their_row_and_column(binding):
    rng = _gen(13)
    x64 = np.round(rng.standard_normal((40, 128)) * 8) / 8
    x64[7, 33] = np.inf
    wc, wb, codes, scales = _weights(rng, (), 60, 128)
    wb[9, 2] = 255
    scales = torch.from_numpy(ref.pack_scales(wb)).cuda()
    y = binding.mx4_matmul(binding.mx4_quantize(torch.from_numpy(x64).float().cuda()), binding.Mx4(codes, scales), dtype=torch.float32).cpu().numpy()
    nan = np.zeros((40, 60), dtype=bool)
    nan[7], nan[:, 9] = True, True
    np.testing.assert_array_equal(np.isnan(y), nan)


def _segments(rng, E, rows, pattern):
    if pattern == "one":
        counts = np.zeros(E, dtype=np.int64)
        counts[E // 2] = rows
    elif pattern == "skewed":
        counts = rng.multinomial(rows, (1.0 / np.arange(1, E + 1)) / (1.0 / np.arange(1, E + 1)).sum())
    else:
        counts = rng.multinomial(rows, np.full(E, 1 / E))
        counts[0] += counts[E - 1]
        counts[E - 1] = 0
    return np.concatenate(([0], np.cumsum(counts)))


@pytest.mark.parametrize("E,T,k,N,K,pattern", [(1, 5, 1, 64, 64, "even"), (4, 3, 2, 100, 96, "one"), (8, 40, 2, 128, 128, "skewed"), (64, 64, 8, 256, 256, "even"),
                                               (64, 700, 4, 136, 160, "skewed"), (5, 600, 1, 512, 288, "one"), (33, 1, 1, 70, 1024, "even")])
def test_grouped_product(binding, E, T, k, N, K, pattern):
    rng = _gen(E * 5 + T + N)
    offsets = _segments(rng, E, T * k, pattern)
    slots = rng.permutation(T * k)
    x64 = np.round(rng.standard_normal((T, K)) * 16) / 16
    x = torch.from_numpy(x64).to(torch.bfloat16).cuda()
    wc, wb, codes, scales = _weights(rng, (E,), N, K)
    off, slot = torch.from_numpy(offsets.astype(np.int32)).cuda(), torch.from_numpy(slots.astype(np.int32)).cuda()
    q = binding.mx4_quantize(x, offsets=off, slot_of_row=slot, k=k)
    a = ref.values(*ref.quantise(x64))[slots // k]
    held = int(offsets[-1])                                             # rows in a segment (none, with one expert that has none)
    np.testing.assert_array_equal(binding.mx4_dequantize(q, torch.float32)[:held].double().cpu().numpy(), a[:held])
    for act, dtype in ((3, torch.float32), (1, torch.bfloat16)):
        y = binding.mx4_matmul(q, binding.Mx4(codes, scales), act=act, dtype=dtype)
        for e in range(E):
            seg = slice(offsets[e], offsets[e + 1])
            if seg.stop > seg.start:
                _check_product(y[seg], a[seg], ref.values(wc[e], wb[e]), act, dtype)
    assert binding.operator_status() == 0


def test_grouped_rows_in_no_segment_are_left(binding):
    """A routing under a capacity limit: rows behind offsets[E] have no slot (-1) and belong to no expert."""
    rng = _gen(3)
    E, rows, K, N = 4, 100, 64, 64
    offsets = torch.tensor([0, 10, 10, 40, 63], dtype=torch.int32, device="cuda")
    slot = torch.arange(rows, dtype=torch.int32, device="cuda")
    slot[63:] = -1
    x64 = np.round(rng.standard_normal((rows, K)) * 16) / 16
    wc, wb, codes, scales = _weights(rng, (E,), N, K)
    q = binding.mx4_quantize(torch.from_numpy(x64).float().cuda(), offsets=offsets, slot_of_row=slot)
    out = torch.full((rows, N), 3.0, dtype=torch.float32, device="cuda")
    binding.mx4_matmul(q, binding.Mx4(codes, scales), out=out)
    a = ref.values(*ref.quantise(x64))
    for e, (i, j) in enumerate(((0, 10), (10, 10), (10, 40), (40, 63))):
        if j > i:
            _check_product(out[i:j], a[i:j], ref.values(wc[e], wb[e]), 3, torch.float32)
    assert bool((out[63:] == 3.0).all())
    back = torch.full((rows, K), 2.0, dtype=torch.float32, device="cuda")
    binding.mx4_dequantize(q, out=back)
    np.testing.assert_array_equal(back[:63].double().cpu().numpy(), a[:63])
    assert bool((back[63:] == 2.0).all())


@pytest.mark.parametrize("act", [0, 1, 2, 3])
@pytest.mark.parametrize("E,rows,N,K", [(0, 1, 32, 64), (0, 300, 160, 256), (0, 1000, 1024, 128), (0, 2600, 4096, 64), (0, 2400, 2048, 512), (8, 700, 96, 96), (64, 512, 1024, 256)])
def test_product_in_4_bits(binding, E, rows, N, K, act):
    """The result's values are roundings of act(a w^T): a block's scale is that of its largest magnitude, a code off by half a step of its
    place (or more where the fp32 value lies next to a border: then the neighbour's half step), magnitudes above 6 scales at 6."""
    rng = _gen(rows + N + act)
    x64 = np.round(rng.standard_normal((rows, K)) * 16) / 16
    wc, wb, codes, scales = _weights(rng, (E,) if E else (), N, K)
    offsets = _segments(rng, E, rows, "skewed") if E else np.array([0, rows])
    off = torch.from_numpy(offsets.astype(np.int32)).cuda() if E else None
    q = binding.mx4_matmul_mx4(binding.mx4_quantize(torch.from_numpy(x64).float().cuda(), offsets=off), binding.Mx4(codes, scales), act=act)
    got = binding.mx4_dequantize(q, torch.float32).double().cpu().numpy()
    a, w = ref.values(*ref.quantise(x64)), ref.values(wc, wb).reshape(-1, N, K)
    for e in range(max(E, 1)):
        seg = slice(offsets[e], offsets[e + 1])
        if seg.start == seg.stop:
            continue
        z = a[seg] @ w[e].T
        want = _act(z, act)
        S = np.abs(a[seg]) @ np.abs(w[e]).T
        err = 1.13 * (K / 64 + 2) * 2.0 ** -23 * S + (3.6e-5 if act == 1 else np.abs(z) * 2.0 ** -20)     # as for a product in bf16, without its rounding
        blocks, slack = want.reshape(-1, N // 32, 32), err.reshape(-1, N // 32, 32)
        top = np.abs(blocks).max(-1, keepdims=True)
        ok = np.zeros(blocks.shape, dtype=bool)
        for lean in (-1, 1):                                            # the largest magnitude as computed lies between these two
            bound = np.maximum(top + lean * slack.max(-1, keepdims=True), 2.0 ** -125)
            scale = 2.0 ** (np.floor(np.log2(bound)) - 2)
            v = np.abs(blocks) / scale
            step = np.where(v < 2, 0.5, np.where(v < 4, 1.0, 2.0))      # of the codes around v
            near = np.where(v > 6, v - 6, step / 2) * scale             # above 6: down to 6
            ok |= np.abs(got[seg].reshape(blocks.shape) - blocks) <= near * (1 + 1e-12) + slack
        assert ok.all(), float((~ok).mean())
    if E == 0 or rows > 128:                                            # what comes out is a matrix that the next product takes
        w2c, w2b, c2, s2 = _weights(rng, (E,) if E else (), 64, N)
        y = binding.mx4_matmul(q, binding.Mx4(c2, s2), dtype=torch.float32)
        for e in range(max(E, 1)):
            seg = slice(offsets[e], offsets[e + 1])
            if seg.stop > seg.start:
                _check_product(y[seg], got[seg], ref.values(w2c, w2b).reshape(-1, 64, N)[e], 3, torch.float32)
    assert binding.operator_status() == 0


def test_slots_that_name_no_row_give_zeros(binding):
    x = torch.ones(3, 32, dtype=torch.float32, device="cuda")
    slot = torch.tensor([0, -1, 5, 6, 2 ** 31 - 1], dtype=torch.int32, device="cuda")
    y = binding.mx4_dequantize(binding.mx4_quantize(x, slot_of_row=slot, k=2), torch.float32)
    assert y[:, 0].tolist() == [1.0, 0.0, 1.0, 0.0, 0.0]


def test_empty(binding):
    q = binding.mx4_quantize(torch.empty(0, 64, dtype=torch.bfloat16, device="cuda"))
    _, _, codes, scales = _weights(_gen(1), (), 32, 64)
    assert binding.mx4_matmul(q, binding.Mx4(codes, scales)).shape == (0, 32)
    assert binding.mx4_dequantize(q).shape == (0, 64)


def test_captured_and_on_another_stream(binding):
    rng = _gen(17)
    T, K, N = 200, 256, 384
    wc, wb, codes, scales = _weights(rng, (), N, K)
    x = torch.zeros(T, K, dtype=torch.bfloat16, device="cuda")
    W = binding.Mx4(codes, scales)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        binding.mx4_matmul(binding.mx4_quantize(x), W)                  # first call outside the capture
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            y = binding.mx4_matmul(binding.mx4_quantize(x), W, dtype=torch.float32)
    torch.cuda.current_stream().wait_stream(side)
    for seed in (1, 2):
        x64 = np.round(_gen(seed).standard_normal((T, K)) * 16) / 16
        x.copy_(torch.from_numpy(x64).to(torch.bfloat16))
        graph.replay()
        other = binding.mx4_matmul(binding.mx4_quantize(x), W, dtype=torch.float32)
        _check_product(y, ref.values(*ref.quantise(x64)), ref.values(wc, wb), 3, torch.float32)
        assert torch.equal(y, other)


def test_binding_refuses_what_is_no_4_bit_matrix(binding):
    u8 = dict(dtype=torch.uint8, device="cuda")
    i32 = dict(dtype=torch.int32, device="cuda")
    ok = torch.zeros(4, 32, **u8), torch.zeros(1, 1, 512, **u8)
    binding.Mx4(*ok)
    for codes, scales, kw in ((torch.zeros(4, 32, device="cuda"), ok[1], {}), (ok[0], torch.zeros(1, 2, 512, **u8), {}), (ok[0], ok[1].cpu(), {}),
                              (torch.zeros(129, 32, **u8), ok[1], {}), (torch.zeros(2, 4, 32, **u8), ok[1], {}), (torch.zeros(4, 64, **u8)[:, :32], ok[1], {}),
                              (*ok, dict(offsets=torch.zeros(3, **i32))), (*ok, dict(offsets=torch.zeros(3, **i32), rows=4)),
                              (torch.zeros(384, 32, **u8), torch.zeros(3, 1, 512, **u8), dict(offsets=torch.zeros(3), rows=4))):
        with pytest.raises(ValueError):
            binding.Mx4(codes, scales, **kw)
    x = torch.zeros(4, 64, device="cuda")
    for bad in (dict(x=x[:, :40]), dict(x=x.half()), dict(x=x.cpu()), dict(x=x.t()), dict(offsets=torch.zeros(3, device="cuda")), dict(slot_of_row=torch.zeros(3, device="cuda"))):
        with pytest.raises(ValueError):
            binding.mx4_quantize(**{"x": x, **bad})
    q, w = binding.mx4_quantize(x), binding.Mx4(torch.zeros(8, 32, **u8), torch.zeros(1, 1, 512, **u8))
    with pytest.raises(ValueError):
        binding.mx4_matmul(q, w, out=torch.empty(4, 9, device="cuda"))
    with pytest.raises(ValueError):
        binding.mx4_matmul(q, w, dtype=torch.float16)
    with pytest.raises(ValueError):
        binding.mx4_matmul_mx4(q, w)                                     # eight columns are no block
    with pytest.raises(binding.BigmacError):
        binding.mx4_matmul(q, binding.mx4_quantize(torch.zeros(8, 32, device="cuda")))


@pytest.mark.parametrize("M,N,E,tile", [(97, 3, 0, 0), (300, 100, 0, 64), (300, 130, 0, 128), (700, 300, 0, 256), (200, 100, 4, 0), (2600, 65, 8, 0)])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_columns_behind_the_result_stay(binding, M, N, E, tile, dtype):
    """A result that is a part of a wider matrix, its rows on 16-byte boundaries and its columns not: the others' columns are left alone."""
    rng = _gen(29)
    K = 96
    _, _, codes, scales = _weights(rng, (E,) if E else (), N, K)
    offsets = torch.from_numpy(_segments(rng, E, M, "skewed").astype(np.int32)).cuda() if E else None
    q = binding.mx4_quantize(torch.from_numpy(rng.standard_normal((M, K))).to("cuda", torch.bfloat16), offsets=offsets)
    W = binding.Mx4(codes, scales)
    wide = torch.full((M + 2, (N + 23) // 8 * 8), 5.0, dtype=dtype, device="cuda")
    binding.bigmac_debug_set("mx4_tile", tile)
    try:
        binding.mx4_matmul(q, W, out=wide[:M, :N])
        alone = binding.mx4_matmul(q, W, dtype=dtype)
    finally:
        binding.bigmac_debug_set("defaults", 0)
    assert torch.equal(wide[:M, :N], alone)
    assert bool((wide[:, N:] == 5.0).all()) and bool((wide[M:] == 5.0).all())
