"""Products with weights held in 8 bits on the GPU against plain forms in 64 bits (f8_reference.py): the format, and the products at
the sizes, types and layouts where they can go wrong."""
import ctypes as C

import pytest
import torch

import paper_2312_04916_amd as ee
from paper_2312_04916_amd import binding

import f8_reference as ref

pytestmark = pytest.mark.gpu
DT = {"bf16": torch.bfloat16, "f32": torch.float32}


def rand(shape, dtype="f32", seed=0, scale=1.0):
    g = torch.Generator(device="cuda:0").manual_seed(seed)
    return (torch.randn(shape, device="cuda:0", generator=g) * scale).to(DT[dtype])


# ---------------------------------------------------------------- the format

@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("n,k", [(1, 1), (16, 128), (17, 129), (128, 128), (130, 250), (300, 1000), (1001, 33)])
def test_weights_hold_what_the_format_says(dtype, n, k):
    w = rand((n, k), dtype, 1)
    w[:, ::7] *= 40
    w[::5] *= 0.01
    assert torch.equal(ee.F8Weight(w).values().cpu().double(), ref.held(w, 128))
    assert torch.equal(ee.F8Weight(w).values(torch.bfloat16).cpu().double(), ref.held(w, 128))
    up = rand((n, k), dtype, 2, 3.0)
    g, u = ee.F8Weight(w, up=up).values()
    assert torch.equal(g.cpu().double(), ref.held(w, 128)) and torch.equal(u.cpu().double(), ref.held(up, 128))


def extremes():
    big = float(torch.finfo(torch.float32).max)
    x = torch.zeros(14, 256)
    x[0, :9] = torch.tensor([448.0, 1.0625, 1.1875, 17.0, -17.0, 2.0 ** -10, 3 * 2.0 ** -10, 5 * 2.0 ** -10, -2.0 ** -9])  # unit 1: ties, subnormals
    x[0, 128:131] = torch.tensor([448.00003, 240.0, 2.0 ** -9])  # behind the line: unit 2
    x[1, :3] = torch.tensor([big, -big, 1.0])
    x[2, :3] = torch.tensor([2.0 ** -126, 2.0 ** -119, 1e-40])
    x[3, :2] = torch.tensor([1e-40, -1e-45])
    x[4, 3] = float("inf")
    x[5, 200] = float("nan")
    x[6] = -0.0
    x[7] = torch.linspace(-448, 448, 256)
    x[8] = torch.linspace(-448, 448, 256) * 2.0 ** 60
    x[9] = torch.linspace(-2, 2, 256) * 2.0 ** -100
    x[10, 127], x[10, 128] = 3.0, 1e-3
    x[11] = torch.arange(256) / 256
    x[12, ::2] = 1e-20
    x[13, 5] = -448.0 * 2.0 ** 119
    return x


def test_weights_of_extreme_values():
    # (a row of the table is a block of its own: 128 copies)
    w = extremes().repeat_interleave(128, 0)
    got = ee.F8Weight(w.cuda()).values().cpu()
    # (fp32's largest, 255.99998 * 2^120, is held as 256 * 2^120 = 2^128: infinite in fp32)
    assert torch.equal(got.nan_to_num(nan=-99.0), ref.held(w, 128).float().nan_to_num(nan=-99.0))
    assert torch.isnan(got[4 * 128, :128]).all() and not torch.isnan(got[4 * 128, 128:]).any()


@pytest.mark.parametrize("m", [1, 14, 40, 300])
def test_rows_of_extreme_values(m):
    """The identity as a weight gives back what the rows are held as: sums of one term."""
    x = extremes().repeat(-(-m // 14), 1)[:m]
    w = ee.F8Weight(torch.eye(256, device="cuda:0"))
    got = w.matmul(x.cuda()).cpu().double()
    want = ref.held(x, 1)
    for i in range(m):
        # 0 * NaN, and 0 * 2^128, which is infinite in fp32: NaN in every column
        if torch.isnan(want[i]).any() or torch.isinf(want[i].float()).any():
            assert torch.isnan(got[i]).all(), i
        else:
            assert torch.equal(got[i], want[i]), i
    # held in bf16 exactly, and one product of a power of two: no rounding (2^128 overflows as a sum, its products with 0 are 0)
    got = w.matmul(x.cuda(), dtype=torch.bfloat16).cpu()
    for i in range(m):
        assert torch.isnan(got[i]).all() if torch.isnan(want[i]).any() else torch.equal(got[i], want[i].to(torch.bfloat16)), i


# ---------------------------------------------------------------- products

def check(y, x, w, add=None, up=None):
    """Elementwise.  Half a step of the result's type; before that, in fp32 a half step of 2^-24 of the sum of |x w| for each of the
    k / 128 + 128 + 16 additions that an element can pass through, in bf16 the 7 * 2^-13 of the matrix cores' sums as well.  silu's slope
    is at most 1.1, and its own arithmetic is good to 2^-20."""
    xh, wh, uh = ref.held(x, 1), ref.held(w, 128), None if up is None else ref.held(up, 128)
    want, size, gate = ref.product(xh, wh, add, uh)
    half = torch.finfo(y.dtype).eps / 2
    part = (x.shape[1] / 128 + 144) * 2.0 ** -24 + (7 * 2.0 ** -13 if y.dtype == torch.bfloat16 else 0)
    if up is None:
        off = part * size
        add_off = 0 if add is None else 2.0 ** -24 * (want.abs() + off)
        tol = off + add_off + half * (want.abs() + off)
    else:
        (g, size_g), (u, size_u) = size, gate
        act = (want if add is None else want - add.double().cpu()).abs()
        off = 1.1 * part * size_g * (u.abs() + part * size_u) + (g * torch.sigmoid(g)).abs() * part * size_u + 2.0 ** -20 * act
        tol = off + 2.0 ** -24 * want.abs() + half * (want.abs() + off)
    err = (y.cpu().double() - want).abs()
    bad = err > tol + 1e-37
    assert not bad.any(), (int(bad.sum()), float((err / (tol + 1e-37)).max()), y.shape, x.shape)
    # and what is likely, not only possible: independent errors, so norms.  The matrix cores' sums cost Gaussian rows 1.5e-5, rows
    # with loud channels up to 1e-4; an fp32 sum of a few hundred additions sqrt(their number) half steps
    likely = 2.0 ** -8 if y.dtype == torch.bfloat16 else 2.0 ** -24 * 64
    assert float(err.norm()) <= likely * float(want.norm()) * (1 if up is None else 2) + 1e-30


SIZES = [(1, 16, 128), (1, 1, 1), (2, 3, 5), (3, 50, 130), (5, 64, 257), (8, 100, 1003), (15, 130, 640), (16, 128, 2048), (17, 260, 384), (31, 48, 1100), (33, 500, 512),
         (48, 96, 4100), (64, 512, 768), (65, 33, 200), (100, 1001, 300), (127, 640, 1024), (128, 256, 640), (129, 257, 129), (200, 300, 2000), (255, 1000, 500),
         (257, 513, 1025), (384, 512, 128), (512, 384, 896), (700, 777, 100), (1024, 1024, 512), (1300, 60, 700)]


@pytest.mark.parametrize("y", ["bf16", "f32"])
@pytest.mark.parametrize("x", ["bf16", "f32"])
@pytest.mark.parametrize("m,n,k", SIZES)
def test_products(m, n, k, x, y):
    a, w = rand((m, k), x, m + n), rand((n, k), x, k, k ** -0.5)
    a *= torch.exp(0.7 * rand((k,), "f32", 3)).to(a.dtype)
    check(ee.F8Weight(w).matmul(a, dtype=DT[y]), a, w)


@pytest.mark.parametrize("y", ["bf16", "f32"])
@pytest.mark.parametrize("m,n,k", SIZES)
def test_pairs_and_added_rows(m, n, k, y):
    a, w, up = rand((m, k), "bf16", m), rand((n, k), "bf16", n, k ** -0.5), rand((n, k), "bf16", k, 2 * k ** -0.5)
    add = rand((m, n), y, 9)
    check(ee.F8Weight(w, up=up).matmul(a, dtype=DT[y]), a, w, up=up)
    check(ee.F8Weight(w, up=up).matmul(a, add=add), a, w, add=add, up=up) if y == "bf16" else None
    check(ee.F8Weight(w).matmul(a, add=add, dtype=DT[y]), a, w, add=add)
    # in place
    want = ee.F8Weight(w).matmul(a, add=add, dtype=DT[y])
    got = add.clone()
    assert ee.F8Weight(w).matmul(a, add=got, out=got) is got and torch.equal(got, want)


@pytest.mark.parametrize("x", ["bf16", "f32"])
@pytest.mark.parametrize("m,n,k", [(1, 40, 300), (9, 130, 256), (70, 200, 513), (300, 260, 384)])
def test_strides_and_alignment(m, n, k, x):
    """Rows of every kind of layout give the bits that contiguous ones do."""
    w = rand((n, k), x, 1)
    p = ee.F8Weight(w)
    odd = rand((n * (k + 3) + 1,), x, 2)
    odd[1:].as_strided((n, k), (k + 3, 1), 1).copy_(w)
    q = ee.F8Weight(odd.as_strided((n, k), (k + 3, 1), 1))
    assert torch.equal(p.packed, q.packed)
    a = rand((m, k), x, 3)
    want = p.matmul(a)
    flat = rand((m * (k + 9) + 16,), x, 4)
    for at, row in ((1, k + 1), (8, k + 8 - k % 8), (3, k + 9)):
        v = flat[:m * row + at].as_strided((m, k), (row, 1), at)
        v.copy_(a)
        assert torch.equal(p.matmul(v), want), (at, row)
    if m > 1:  # one row for all
        assert torch.equal(p.matmul(a[:1].expand(m, k)), p.matmul(a[:1].repeat(m, 1)))
    # results into a wider matrix, from an odd column on: the rest stays
    for at, wide in ((0, n + 4 - n % 4), (3, n + 7), (4, n + 8 - n % 4)):
        y = torch.full((m, wide), 7.0, dtype=DT[x], device="cuda:0")
        p.matmul(a, out=y[:, at:at + n])
        assert torch.equal(y[:, at:at + n], want) and (y[:, :at] == 7).all() and (y[:, at + n:] == 7).all()
        add = rand((m, wide), x, 6)[:, at:at + n]
        assert torch.equal(p.matmul(a, add=add), p.matmul(a, add=add.contiguous()))


@pytest.mark.parametrize("y", ["bf16", "f32"])
@pytest.mark.parametrize("m", [1, 16, 33, 200, 600])
def test_rows_do_not_reach_one_another(m, y):
    n, k = 200, 700
    a, w = rand((m, k), "bf16", 1), rand((n, k), "bf16", 2)
    p = ee.F8Weight(w)
    want = p.matmul(a, dtype=DT[y])
    b = a.clone()
    b[m // 2, 650] = float("nan")
    got = p.matmul(b, dtype=DT[y])
    assert torch.isnan(got[m // 2]).all()
    rest = torch.arange(m, device="cuda:0") != m // 2
    assert torch.equal(got[rest], want[rest])
    # the same call gives the same bits
    assert torch.equal(p.matmul(a, dtype=DT[y]), want)
    # a NaN in a weight is in the columns of its block alone
    v = w.clone()
    v[150, 3] = float("inf")
    got = ee.F8Weight(v).matmul(a, dtype=DT[y])
    assert torch.isnan(got[:, 128:]).all() and torch.equal(got[:, :128], want[:, :128])


def test_no_rows():
    p = ee.F8Weight(rand((30, 40), "bf16", 1))
    assert p.matmul(rand((0, 40), "bf16", 2)).shape == (0, 30)
    assert p.matmul(rand((0, 40), "bf16", 2), add=rand((0, 30), "bf16", 2)).shape == (0, 30)


@pytest.mark.parametrize("m", [1, 48, 400])
def test_weights_past_32_bits(m):
    """A packed weight and results whose offsets pass 2^31."""
    n, k = 36000, 65536
    w = torch.empty(n, k, dtype=torch.bfloat16, device="cuda:0")
    base = rand((128, k), "bf16", 1)
    for i in range(0, n, 128):
        w[i:i + 128] = base[:min(128, n - i)]
    w[n - 3] *= -1
    p = ee.F8Weight(w)
    assert p.packed.numel() > 2 ** 31
    last = n - n % 128
    rest = w[last:].clone()
    del w
    a = rand((m, k), "bf16", 2)
    y = p.matmul(a)
    assert torch.equal(y[:, 128:256], y[:, :128]) and torch.equal(y[:, last - 128:last], y[:, :128])
    # (the last block's 32 rows have a largest element of their own, and with it may have another exponent than the same rows among
    # 128: elements below 2^-6 of it are then held in other steps)
    xh = ref.held(a[:1], 1)
    for part, w in ((y[0, :128], base), (y[0, last:], rest)):
        want = ref.product(xh, ref.held(w, 128))[0][0]
        assert float((part.cpu().double() - want).norm()) <= 2.0 ** -8 * float(want.norm())


def test_many_rows_of_results_past_32_bits():
    m, n, k = 45000, 50304, 128
    w, a = rand((n, k), "bf16", 1), rand((1000, k), "bf16", 2).repeat(45, 1)
    p = ee.F8Weight(w)
    y = p.matmul(a)
    assert y.numel() > 2 ** 31
    assert torch.equal(y[-1000:], y[:1000]) and torch.equal(y[23000:24000], y[:1000])
    check(y[-300:], a[-300:], w)


# ---------------------------------------------------------------- streams and graphs

@pytest.mark.parametrize("m", [1, 40, 300])
def test_another_stream_and_captured_calls(m):
    w, a, add = rand((300, 512), "bf16", 1), rand((m, 512), "bf16", 2), rand((m, 300), "bf16", 3)
    p = ee.F8Weight(w)
    want = p.matmul(a, add=add)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    got = p.matmul(a, add=add, stream=s)
    packed = ee.F8Weight(w, stream=s)
    s.synchronize()
    assert torch.equal(got, want) and torch.equal(packed.packed, p.packed)
    # two graphs, replayed in turn with eager calls between
    xs = [a.clone(), a.clone()]
    ys, graphs = [], []
    for x in xs:
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            ys.append(p.matmul(x, add=add))
        graphs.append(g)
    for i in range(4):
        b = rand((m, 512), "bf16", 10 + i)
        xs[i % 2].copy_(b)
        eager = p.matmul(b, add=add)
        graphs[i % 2].replay()
        torch.cuda.synchronize()
        assert torch.equal(ys[i % 2], eager), i


def test_two_streams_at_once():
    p, q = ee.F8Weight(rand((700, 900), "bf16", 1)), ee.F8Weight(rand((650, 900), "bf16", 2))
    a, b = rand((90, 900), "bf16", 3), rand((250, 900), "bf16", 4)
    want = p.matmul(a), q.matmul(b)
    torch.cuda.synchronize()
    s, t = torch.cuda.Stream(), torch.cuda.Stream()
    got = [(p.matmul(a, stream=s), q.matmul(b, stream=t)) for _ in range(20)]
    torch.cuda.synchronize()
    assert all(torch.equal(x, want[0]) and torch.equal(y, want[1]) for x, y in got)


@pytest.mark.parametrize("m", [1, 6, 16, 24, 40, 64, 70, 200])
@pytest.mark.parametrize("n,k,pair", [(48, 1, False), (64, 128, True), (272, 256, False), (1000, 256, True), (640, 513, False)])
def test_buffers_that_end_where_their_memory_does(m, n, k, pair):
    """Few steps along k, fewer than a workgroup has waves, with the packed weight, the workspace, x and y at the end of their allocations:
    a read behind them would leave what is mapped."""
    size, need = C.c_size_t(), C.c_size_t()
    L = binding.lib()
    assert L.ee_f8_bytes(n, k, pair, C.byref(size)) == 0 and L.ee_f8_matmul_bytes(m, n, k, pair, binding.EE_BF16, C.byref(need)) == 0
    a, w, up = rand((m, k), "bf16", m), rand((n, k), "bf16", n), rand((n, k), "bf16", k)
    memory = [torch.zeros(32 << 20, dtype=torch.uint8, device="cuda:0") for _ in range(4)]
    at = [t.data_ptr() + (t.numel() - length) // 256 * 256 for t, length in zip(memory, (size.value, need.value, 2 * m * k, 2 * m * n))]
    memory[2][at[2] - memory[2].data_ptr():][:2 * m * k].copy_(a.view(-1).view(torch.uint8))
    stream = torch.cuda.current_stream().cuda_stream
    assert L.ee_f8_pack(n, k, pair, binding.EE_BF16, w.data_ptr(), k, up.data_ptr() if pair else None, k, at[0], size.value, stream) == 0
    assert L.ee_f8_matmul(m, n, k, pair, at[0], binding.EE_BF16, at[2], k, binding.EE_BF16, at[3], n, None, 0, at[1] if need.value else None, need.value, stream) == 0
    torch.cuda.synchronize()
    y = memory[3][at[3] - memory[3].data_ptr():][:2 * m * n].view(torch.bfloat16).view(m, n)
    check(y, a, w, up=up if pair else None)
