"""The operators around the layer at their edges: more than 2^31 elements, several streams at once, tables of segments that are none."""
import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def binding():
    from paper_2502_16927_b200 import binding as b

    return b


def _fill(t, seed):
    """Random numbers in place, without a second tensor of this size."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    for part in t.split(1 << 16):
        part.copy_(torch.randn(part.shape, generator=g, device="cuda"))
    return t


def test_joint_of_more_than_2_to_the_31_elements(binding):
    T, d = (1 << 31) // 4096 + 1000, 4096
    x, y = (_fill(torch.empty(T, d, dtype=torch.bfloat16, device="cuda"), s) for s in (1, 2))
    norm = binding.Norm(binding.BIGMAC_NORM_RMS, torch.randn(d, device="cuda"))
    r, n, stats = binding.residual_norm_forward(x, y, None, norm, norm, training=True)
    dx, dy, _ = binding.residual_norm_backward(x, y, None, norm, norm, r, n, stats)
    for rows in (slice(0, 700), slice(T - 700, T)):
        r1, n1, s1 = binding.residual_norm_forward(x[rows], y[rows], None, norm, norm, training=True)
        assert torch.equal(r[rows], r1) and torch.equal(n[rows], n1) and torch.equal(stats[rows], s1)
        dx1, dy1, _ = binding.residual_norm_backward(x[rows], y[rows], None, norm, norm, r1, n1, s1)
        assert torch.equal(dx[rows], dx1) and torch.equal(dy[rows], dy1)


def test_4_bit_matrix_of_more_than_2_to_the_31_elements(binding):
    T, K = (1 << 31) // 4096 // 128 * 128 + 1000, 4096
    x = _fill(torch.empty(T, K, dtype=torch.bfloat16, device="cuda"), 3)
    q = binding.mx4_quantize(x)
    last = slice(T // 128 * 128 - 1280, T)
    q1 = binding.mx4_quantize(x[last])
    assert torch.equal(q.codes[last], q1.codes)
    back = binding.mx4_dequantize(q)
    assert torch.equal(back[last], binding.mx4_dequantize(q1))
    del back
    w = binding.mx4_quantize(torch.randn(64, K, device="cuda"))
    y, y1 = binding.mx4_matmul(q, w, dtype=torch.float32)[last], binding.mx4_matmul(q1, w, dtype=torch.float32)
    # the same products in tiles of another shape: each sum is off by at most 2^-23 of sum |a w| for each of its K / 64 instructions
    S = binding.mx4_dequantize(q1, torch.float32).abs() @ binding.mx4_dequantize(w, torch.float32).abs().t()
    assert bool(((y - y1).abs() <= 2 * (K / 64 + 2) * 2.0 ** -23 * S).all())
    assert binding.operator_status() == 0


def test_output_of_more_than_2_to_the_31_elements(binding):
    T, N, K = (1 << 31) // 4096 + 1000, 4096, 32
    x = _fill(torch.empty(T, K, dtype=torch.bfloat16, device="cuda"), 4)
    w = binding.mx4_quantize(torch.randn(N, K, device="cuda"))
    y = binding.mx4_matmul(binding.mx4_quantize(x), w)
    for rows in (slice(0, 300), slice(T - 300, T)):
        a = binding.mx4_dequantize(binding.mx4_quantize(x[rows]), torch.float32)
        want = a.double() @ binding.mx4_dequantize(w, torch.float32).double().t()
        S = a.abs().double() @ binding.mx4_dequantize(w, torch.float32).abs().double().t()
        assert bool(((y[rows].double() - want).abs() <= 3 * 2.0 ** -23 * S + want.abs() * 2.0 ** -8 * 1.01).all())
    assert binding.operator_status() == 0


def test_streams_at_once(binding):
    """Calls on several streams share nothing: the results of each are those of the call alone."""
    g = torch.Generator(device="cuda").manual_seed(5)
    d, streams = 1024, [torch.cuda.Stream() for _ in range(4)]
    norm = binding.Norm(binding.BIGMAC_NORM_LAYER, torch.randn(d, generator=g, device="cuda"), torch.randn(d, generator=g, device="cuda"))
    W = binding.mx4_quantize(torch.randn(768, d, generator=g, device="cuda"))
    data = [[torch.randn(T, d, generator=g, device="cuda").bfloat16() for _ in range(4)] for T in (3, 500, 1700, 5000)]

    def run(x, y, dr, dn):
        G = {n: torch.empty(d, device="cuda") for n in ("dw_post", "db_post", "dw_pre", "db_pre")}
        r, n, stats = binding.residual_norm_forward(x, y, None, norm, norm, training=True)
        dx, dy, _ = binding.residual_norm_backward(x, y, None, norm, norm, dr, dn, stats, G)
        return [r, n, dx, dy, binding.mx4_matmul(binding.mx4_quantize(n), W), *G.values()]

    alone = [run(*tensors) for tensors in data]
    torch.cuda.synchronize()
    for _ in range(5):
        at_once = []
        for stream, tensors in zip(streams, data):
            with torch.cuda.stream(stream):
                at_once.append(run(*tensors))
        torch.cuda.synchronize()
        for a, b in zip(alone, at_once):
            assert all(torch.equal(s, t) for s, t in zip(a, b))


def test_tables_that_are_no_segments_touch_nothing_else(binding):
    """Descending, negative and too large entries: whatever comes out, rows behind the caller's stay as they are."""
    E, rows, K, N = 6, 300, 64, 96
    x = torch.randn(rows, K, device="cuda")
    w = binding.mx4_quantize_weights(torch.randn(E, N, K, device="cuda"))
    rng = np.random.default_rng(0)
    tables = [rng.integers(-500, 1000, E + 1) for _ in range(6)] + [np.array([0, rows] * 3 + [0]), np.full(E + 1, 2 ** 31 - 1), np.full(E + 1, -2 ** 31)]
    for table in tables:
        offsets = torch.from_numpy(table.astype(np.int32)).cuda()
        q = binding.mx4_quantize(x, offsets=offsets)
        out = torch.full((rows + 64, N), 7.0, device="cuda")
        binding.mx4_matmul(q, w, out=out[:rows])
        back = torch.full((rows + 64, K), 7.0, device="cuda")
        binding.mx4_dequantize(q, out=back[:rows])
        torch.cuda.synchronize()
        assert bool((out[rows:] == 7.0).all()) and bool((back[rows:] == 7.0).all())
    assert binding.operator_status() == 0


def test_tables_whose_counts_pass_32_bits(binding):
    """A table of 512 full segments of all rows, more tiles than 32 bits count: nothing but the results is written."""
    E, rows, K, N = 1024, (1 << 29) + 100, 32, 8
    offsets = torch.tensor([0, rows] * (E // 2) + [0], dtype=torch.int32, device="cuda")
    x = torch.ones(1, K, dtype=torch.bfloat16, device="cuda")
    q = binding.mx4_quantize(x, offsets=offsets, slot_of_row=torch.zeros(rows, dtype=torch.int32, device="cuda"))
    w = binding.mx4_quantize_weights(torch.randn(1, N, K, device="cuda"))
    w = binding.Mx4(w.codes.expand(E, -1, -1).contiguous(), w.scales.expand(E, -1, -1, -1).contiguous())
    guard = 1 << 20
    room = torch.zeros(rows + 2 * guard, N, dtype=torch.bfloat16, device="cuda")
    binding.mx4_matmul(q, w, out=room[guard:guard + rows])
    torch.cuda.synchronize()
    assert not bool(room[:guard].any()) and not bool(room[guard + rows:].any())
    assert binding.operator_status() == 0


def test_rows_that_pass_32_bits_are_refused(binding):
    x = torch.empty((1 << 32) + 5, 1, dtype=torch.bfloat16, device="cuda")
    with pytest.raises(ValueError):
        binding.residual_norm_forward(x, pre=binding.Norm(binding.BIGMAC_NORM_RMS))
    with pytest.raises(binding.BigmacError):
        binding.residual_norm_forward(x[:(1 << 30) + 1], pre=binding.Norm(binding.BIGMAC_NORM_RMS))
    with pytest.raises(ValueError):
        binding.Mx4(torch.empty((1 << 31) + 128, 1, dtype=torch.uint8, device="cuda"), torch.empty((1 << 24) + 1, 1, 512, dtype=torch.uint8, device="cuda"))


def test_4_bit_products_of_no_rows(binding):
    q, w = binding.mx4_quantize(torch.empty(0, 64, device="cuda")), binding.mx4_quantize(torch.randn(96, 64, device="cuda"))
    h = binding.mx4_matmul_mx4(q, w)
    assert h.rows == 0 and binding.mx4_dequantize(h).shape == (0, 96)
    offsets = torch.zeros(5, dtype=torch.int32, device="cuda")
    grouped = binding.mx4_quantize(torch.empty(0, 64, device="cuda"), offsets=offsets)
    h = binding.mx4_matmul_mx4(grouped, binding.mx4_quantize_weights(torch.randn(4, 96, 64, device="cuda")))
    assert h.rows == 0 and binding.mx4_dequantize(h).shape == (0, 96)
