"""Products with weights held in 8 bits on the GPU, form by form: what fp32 results keep of silu, rows of one
buffer, every tile that goes through LDS, few
rows with rows and weights of every number of tiles."""
import pytest
import torch

import paper_2312_04916_amd as ee
from test_gpu_f8 import DT, check, rand

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


# m, n, k, pair -> rows of x and of the packed weight in a tile.  Odd sizes; 6 to 11 steps of 128 elements, two stages each, so that every one
# of a tile's three or four buffers is filled again; among 256 x 256 and 256 x 192 XCDs that are left with a few tiles, which go in halves.
TILES = [(1110, 2149, 641, False, (128, 128)), (1451, 2803, 700, False, (128, 192)), (3104, 2515, 1003, False, (192, 192)), (3256, 1827, 1290, False, (256, 128)),
         (4445, 2017, 700, False, (256, 192)), (3101, 3649, 1003, False, (256, 256)), (1355, 873, 1003, True, (128, 128)), (671, 2981, 641, True, (128, 192)),
         (1078, 3529, 700, True, (192, 192)), (797, 3685, 1003, True, (256, 128)), (3815, 1163, 641, True, (256, 192)), (1290, 4037, 700, True, (256, 256)),
         (2048, 2048, 1024, False, (128, 128)), (4096, 4096, 768, False, (256, 256)), (2048, 2048, 1024, True, (256, 128))]


@pytest.mark.parametrize("y", ["bf16", "f32"])
@pytest.mark.parametrize("m,n,k,pair,tile", TILES)
def test_every_tile(m, n, k, pair, tile, y):
    """The result alone, and with rows added in place, in columns of a wider buffer; two rows of every sixteen against 64 bits, in all places."""
    assert ee.f8_launch(m, n, k, pair) == (*tile, 4, 2)
    a, w, up = rand((m, k), "bf16", m), rand((n, k), "bf16", n, k ** -0.5), rand((n, k), "bf16", k, 2 * k ** -0.5) if pair else None
    p = ee.F8Weight(w, up=up)
    some = torch.arange(0, m, 16, device="cuda:0")
    some = torch.cat([some + some // 16 % 16, some + (some // 16 * 5 + 8) % 16]).clamp_max(m - 1).unique()
    got = p.matmul(a, dtype=DT[y])
    check(got[some], a[some], w, up=up)
    wide = rand((m, n + 9), y, 9)
    before = wide.clone()
    at = m % 8
    p.matmul(a, add=wide[:, at:at + n], out=wide[:, at:at + n])
    check(wide[some][:, at:at + n], a[some], w, add=before[some][:, at:at + n], up=up)
    assert torch.equal(wide[:, :at], before[:, :at]) and torch.equal(wide[:, at + n:], before[:, at + n:])
    # the rows between them: the same sums, so the same but for the added rows and a rounding
    both = before[:, at:at + n].float() + got.float()
    near = 4 * torch.finfo(DT[y]).eps * (before[:, at:at + n].float().abs() + got.float().abs()) + 1e-30
    assert ((wide[:, at:at + n].float() - both).abs() <= near).all()
    # and rows that are the same everywhere give the same everywhere
    assert torch.equal(p.matmul(a[:1].expand(m, k), dtype=DT[y]), got[:1].expand(m, n))


# m, n, k, pair -> launch: few rows, by numbers of tiles of the weight and lengths that the sizes of test_gpu_f8 leave out
FEW = [(16, 499, 2177, False, (16, 16, 4, 0)), (3, 4099, 12000, False, (16, 32, 4, 0)), (11, 4501, 3001, False, (16, 32, 4, 0)), (16, 300, 2300, True, (16, 32, 4, 0)),
       (9, 16401, 3700, False, (16, 32, 8, 0)), (16, 16387, 2200, False, (16, 32, 8, 0)), (5, 16401, 300, False, (16, 32, 8, 1)), (14, 17000, 2000, False, (16, 32, 8, 1)),
       (32, 4200, 900, False, (32, 32, 4, 0)), (20, 333, 1500, True, (32, 32, 4, 0)), (64, 4101, 700, False, (64, 32, 4, 0)), (50, 9001, 513, False, (64, 64, 4, 0)),
       (61, 4100, 1000, True, (64, 64, 4, 0)), (40, 2500, 1100, False, (64, 16, 4, 0)), (1, 1, 40000, False, (16, 16, 4, 0)), (17, 3, 10001, True, (32, 32, 4, 0))]


@pytest.mark.parametrize("y", ["bf16", "f32"])
@pytest.mark.parametrize("m,n,k,pair,launch", FEW)
def test_few_rows(m, n, k, pair, launch, y):
    assert ee.f8_launch(m, n, k, pair) == launch
    x = "f32" if m % 2 else "bf16"
    a, w, up = rand((m, k), x, m), rand((n, k), x, n, k ** -0.5), rand((n, k), x, k, 2 * k ** -0.5) if pair else None
    add = rand((m, n), y, 9)
    p = ee.F8Weight(w, up=up)
    check(p.matmul(a, dtype=DT[y]), a, w, up=up)
    check(p.matmul(a, add=add, dtype=DT[y]), a, w, add=add, up=up)
