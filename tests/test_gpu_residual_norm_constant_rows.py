"""LayerNorms of rows whose elements are all the same: the mean is that element, and the norm its bias, exactly."""
import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def binding():
    from paper_2502_16927_b200 import binding as b

    return b


# numbers of 8 bits, so that no sum of a row is rounded, at widths whose reciprocal is; few rows and many, on 16-byte boundaries and off them
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("T,d", [(20, 1000), (3000, 1000), (700, 2000), (20, 1504), (400, 4104), (3000, 999), (700, 2001), (20, 5000), (400, 5001)])
def test_norm_of_a_constant_row_is_its_bias(binding, T, d, dtype):
    g = torch.Generator(device="cuda").manual_seed(d)
    value = torch.randint(128, 256, (T, 1), generator=g, device="cuda") * torch.exp2(torch.randint(-12, 8, (T, 1), generator=g, device="cuda").float())
    value = value * torch.where(torch.rand(T, 1, generator=g, device="cuda") < 0.5, -1, 1)
    x = value.expand(T, d).to(dtype).contiguous()
    assert torch.equal(x.float(), value.expand(T, d))
    w, b = torch.randn(d, generator=g, device="cuda"), torch.randn(d, generator=g, device="cuda")
    norm = binding.Norm(binding.BIGMAC_NORM_LAYER, w, b)
    _, n, stats = binding.residual_norm_forward(x, pre=norm, training=True)
    want = b.to(dtype).expand(T, d)
    assert torch.equal(stats[:, 2], value[:, 0]) and torch.equal(n, want)
    zero = torch.zeros_like(x)
    r, _, stats = binding.residual_norm_forward(zero, x, None, norm, training=True)
    assert torch.equal(stats[:, 0], value[:, 0]) and torch.equal(r, want)
