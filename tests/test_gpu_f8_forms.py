"""Products with weights held in 8 bits on the GPU, form by form: what fp32 results keep of silu, rows of one
buffer."""
import pytest
import torch

import paper_2312_04916_amd as ee

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("m", [5, 16, 40, 300, 3000])
def test_silu_keeps_fp32(m):
    """One product a sum, of values that 8 bits hold, so that g and u are exact.  In half steps of 2^-24 silu(g) u = g / (1 + exp(-g)) u is off by 2
    and 1 of the exponential (its unit, the product behind it), by 1 each of the addition, the division and the product: 6.
    A product with log2(e) that is rounded would cost |g| more."""
    n = 2048
    g = torch.Generator(device="cuda:0").manual_seed(m)
    w = (8 + torch.randint(0, 8, (n, 1), device="cuda:0", generator=g)) * 2.0 ** torch.randint(-5, 1, (n, 1), device="cuda:0", generator=g)
    x = (8 + torch.randint(0, 8, (m, 1), device="cuda:0", generator=g)) * 2.0 ** torch.randint(-5, 0, (m, 1), device="cuda:0", generator=g)
    x *= torch.where(torch.arange(m, device="cuda:0")[:, None] % 4 == 3, 1.0, -1.0)
    y = ee.F8Weight(w, up=torch.ones_like(w)).matmul(x)
    gate = x.double() * w.double().T
    want = gate * torch.sigmoid(gate) * x.double()
    fits = gate > -86  # (1 + exp(-g) is infinite behind -88)
    assert m < 16 or int((gate[fits] < -40).sum()) > m  # (five rows hold none)
    err = (y.double() - want).abs() / (want.abs() * 2.0 ** -24)
    assert float(err[fits].max()) <= 6.01, float(err[fits].max())


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("m", [1, 2, 16, 40, 300, 2000])
@pytest.mark.parametrize("n,k,apart", [(130, 200, 0), (64, 257, 5), (512, 128, 8)])
def test_columns_of_one_buffer(m, n, k, apart, dtype):
    """x, rows to add and the result side by side: the bits that buffers of their own give, and the other columns stay."""
    g = torch.Generator(device="cuda:0").manual_seed(m + n)
    w = ee.F8Weight(torch.randn(n, k, device="cuda:0", generator=g).to(dtype))
    at = k + apart, k + apart + n + apart
    b = torch.randn(m, at[1] + n + 3, device="cuda:0", generator=g).to(dtype)
    x, add, y = b[:, :k], b[:, at[0]:at[0] + n], b[:, at[1]:at[1] + n]
    before = b.clone()
    want = w.matmul(x.contiguous(), add=add.contiguous())
    assert w.matmul(x, add=add, out=y) is y and torch.equal(y, want)
    before[:, at[1]:at[1] + n] = want
    assert torch.equal(b, before)
    # onto the added rows themselves
    w.matmul(x, add=add, out=add)
    before[:, at[0]:at[0] + n] = want
    assert torch.equal(b, before)
    if m > 1:
        with pytest.raises(RuntimeError):
            w.matmul(x, out=b[:, k - 1:k - 1 + n])
