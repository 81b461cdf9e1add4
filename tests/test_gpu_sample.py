"""Choosing tokens on the GPU against a plain form in 64 bits (f8_reference.choose): every cut, ties, masks, odd sizes and layouts."""
import math

import numpy as np
import pytest
import torch

import paper_2312_04916_amd as ee

import f8_reference as ref

pytestmark = pytest.mark.gpu
DT = {"bf16": torch.bfloat16, "f32": torch.float32}
MOST_U = 1 - 2.0 ** -24


def gen(seed):
    return torch.Generator(device="cuda:0").manual_seed(seed)


def logits(rows, vocab, dtype="f32", seed=0, spread=2.5):
    return (torch.randn(rows, vocab, device="cuda:0", generator=gen(seed)) * spread).to(DT[dtype])


def per_row(v, rows, dt):
    return None if v is None else (v if isinstance(v, torch.Tensor) else torch.tensor(v, dtype=dt, device="cuda:0").expand(rows).contiguous())


def check(z, u, t=None, k=None, p=None, m=None):
    rows = z.shape[0]
    u, t, p, m = (per_row(a, rows, torch.float32) for a in (u, t, p, m))
    k = per_row(k, rows, torch.int32)
    token, logprob, conf = ee.sample(z, u, temperature=t, top_k=k, top_p=p, min_p=m, scores=True)
    assert torch.equal(ee.sample(z, u, temperature=t, top_k=k, top_p=p, min_p=m), token)
    zc = z.double().cpu().numpy()
    args = [[off] * rows if a is None else a.tolist() for a, off in ((u, 0), (t, 1.0), (k, 0), (p, 1.0), (m, 0.0))]
    for i in range(rows):
        want = ref.choose(zc[i], *(a[i] for a in args))
        assert int(token[i]) == want[0], (i, int(token[i]), want, [a[i] for a in args])
        if want[0] < 0:
            assert float(logprob[i]) == -math.inf and float(conf[i]) == 0
        else:
            off = ref.score_tolerance(zc[i])
            assert abs(float(logprob[i]) - want[1]) <= off + 2.0 ** -24 * abs(want[1]) + 2.0 ** -140, (i, float(logprob[i]), want[1], off)
            assert abs(float(conf[i]) - want[2]) <= (off + 2.0 ** -24) * want[2], (i, float(conf[i]), want[2])
    return token


def mixed(rows, seed):
    g = gen(seed)
    r, i = torch.rand(5, rows, device="cuda:0", generator=g), torch.arange(rows, device="cuda:0")
    t = torch.where(i % 7 == 3, torch.zeros_like(r[0]), 0.2 + 1.5 * r[1])
    k = torch.where(i % 3 == 1, torch.zeros_like(i), 1 + (300 * r[2] ** 3).long()).int()
    p = torch.where(i % 4 == 2, torch.ones_like(r[3]), r[3])
    m = torch.where(i % 5 < 2, torch.zeros_like(r[4]), 0.3 * r[4] ** 2)
    return r[0], t, k, p, m


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("vocab", [1, 2, 3, 7, 63, 64, 65, 255, 257, 511, 1000, 1025, 4095, 4097, 8193, 20011, 50304, 65536, 65537, 131073, 262144])
def test_settings_of_every_kind(vocab, dtype):
    rows = 24 if vocab < 60000 else 10
    check(logits(rows, vocab, dtype, vocab), *mixed(rows, vocab + 1))


@pytest.mark.parametrize("rows", [1, 2, 3, 5, 17, 64, 130, 300])
def test_numbers_of_rows(rows):
    """A row's token does not depend on the other rows or their number."""
    z = logits(300, 3001, "f32", 5)
    a = mixed(300, 6)
    every = check(z[:rows], *(x[:rows].contiguous() for x in a))
    assert torch.equal(every, ee.sample(z, a[0], temperature=a[1], top_k=a[2], top_p=a[3], min_p=a[4])[:rows])


@pytest.mark.parametrize("vocab", [50304, 200000])
@pytest.mark.parametrize("one", [dict(), dict(t=0.0), dict(t=0.7), dict(k=1), dict(k=50), dict(k=5000), dict(p=0.0), dict(p=0.3), dict(p=0.9), dict(p=0.9999), dict(m=0.05),
                                 dict(m=1.0), dict(m=1e-9), dict(k=40, p=0.95), dict(k=2000, p=0.5, t=1.3), dict(k=100, p=0.9, m=0.02, t=0.8)])
def test_one_setting_for_all(one, vocab):
    z = logits(4, vocab, "f32", 7, 3.0)
    u = torch.tensor([0.0, 0.37, 0.83, MOST_U], device="cuda:0")
    got = check(z, u, one.get("t"), one.get("k"), one.get("p"), one.get("m"))
    same = ee.sample(z, u, temperature=one.get("t"), top_k=one.get("k"), top_p=one.get("p"), min_p=one.get("m"))  # as numbers
    assert torch.equal(got, same)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_equal_logits_go_by_index(dtype):
    n = 5000
    z = torch.zeros(12, n, device="cuda:0")
    z[1] = -3.25
    z[2, ::2] = 1.0
    z[3, 1::3] = 2.0
    z[4, 4000:] = 1.0
    z[5, 100] = 5.0
    z[6] = -torch.inf
    z[6, 17::50] = 0.5
    z[7] = torch.tensor([0.0, -0.0], device="cuda:0").repeat(n // 2)  # equal: -0 is 0
    z[8] = (torch.arange(n, device="cuda:0") % 3).float()
    z[9] = (torch.arange(n, device="cuda:0") // 1000).float()
    z[10, :2] = 1.0
    z[11, n - 1] = 1e-30
    z = z.to(DT[dtype])
    for u in (0.0, 0.25, 0.5, 0.999, MOST_U):
        for k, p in ((0, 1.0), (1, 1.0), (3, 1.0), (700, 1.0), (4999, 1.0), (0, 0.5), (0, 0.25), (0, 0.999), (2500, 0.5), (10, 0.3)):
            check(z, u, 1.0, k, p, 0.0)
    check(z, 0.5, 0.0)
    check(z, 0.7, 1.0, 0, 1.0, 1.0)  # the largest alone, with its equals


def test_rows_of_close_values():
    """More elements than are ranked one by one fall into a bin, again and again."""
    n = 40000
    a = 1.0 + torch.arange(n, device="cuda:0") * 2.0 ** -23       # neighbours in fp32
    b = torch.arange(n, device="cuda:0").flip(0) * 1e-9
    c = torch.cat([torch.full((n // 2,), 3.0, device="cuda:0"), 3.0 - torch.rand(n // 2, device="cuda:0", generator=gen(1)) * 1e-4])
    d = torch.randn(n, device="cuda:0", generator=gen(2)) * 1e-3 - 700
    z = torch.stack([a, b, c, d])
    for u in (0.1, 0.9):
        for k, p, m in ((0, 0.5, 0.0), (13000, 1.0, 0.0), (20001, 1.0, 0.0), (30000, 0.77, 0.0), (0, 0.9, 0.999), (7, 1.0, 0.0)):
            check(z, u, 1.0, k, p, m)


@pytest.mark.parametrize("t", [1e-40, 1e-20, 1e-3, 0.01, 30.0, 1e10, 3e38])
def test_extreme_temperatures(t):
    z = logits(6, 2000, "f32", 8)
    z[2] *= 1e30
    z[3] *= 1e-30
    z[4, 5] = 3e38
    z[5] = torch.where(z[5] > 0, 3e38, -3e38)
    for k, p, m in ((0, 1.0, 0.0), (50, 0.9, 0.0), (0, 0.7, 0.01)):
        check(z, torch.tensor([0.0, 0.2, 0.5, 0.7, 0.9, MOST_U], device="cuda:0"), t, k, p, m)


def t32(x):
    return float(torch.tensor(x, dtype=torch.float32))


@pytest.mark.parametrize("t", [1.0, 2e37, 3e38])
@pytest.mark.parametrize("vocab", [1500, 5003, 70000])
def test_spreads_that_overflow(vocab, t):
    """Many candidates whose distance to the top, or 32 temperatures, has no fp32 value."""
    z = logits(4, vocab, "f32", 8)
    z[1] = torch.where(z[1] > 0, 3e38, -3e38)
    z[2] = z[2].sign() * 3.4e38 * torch.rand(vocab, device="cuda:0", generator=gen(3))
    z[3, ::3] = -3.4e38
    z = z.contiguous()
    zc, u = z.double().cpu().numpy(), torch.tensor([0.0, 0.2, 0.5, MOST_U], device="cuda:0")
    for k, p, m in ((0, 0.7, 0.0), (vocab - 300, 0.9, 0.0), (vocab // 2, 1.0, 0.0), (0, 0.7, 0.01), (0, 1.0, 0.001)):
        token = ee.sample(z, u, temperature=t, top_k=k, top_p=p, min_p=m)
        for i in range(4):
            assert int(token[i]) == ref.choose(zc[i], float(u[i]), t32(t), k, t32(p), t32(m))[0], (i, k, p, m)


def test_masks_and_rows_without_a_distribution():
    z = logits(9, 3000, "f32", 9)
    z[0] = -torch.inf
    z[1, 77] = float("nan")
    z[2, 2999] = torch.inf
    z[3] = -torch.inf
    z[3, 2998] = -3e38
    z[4, :2990] = -torch.inf
    z[5, ::2] = -torch.inf
    z[6] = torch.where(z[6] > 0, z[6], torch.finfo(torch.float32).min)  # a mask of the type's lowest value
    z[7] = torch.finfo(torch.float32).min
    for dtype in ("f32", "bf16"):
        for k, p, m in ((0, 1.0, 0.0), (2995, 1.0, 0.0), (20, 0.9, 0.0), (0, 0.6, 0.05), (2995, 0.99999, 0.0)):
            # (in bf16 fp32's lowest value is -inf)
            check(z.to(DT[dtype]), torch.rand(9, device="cuda:0", generator=gen(4)), 0.9, k, p, m)


def test_settings_out_of_range_mark_their_row():
    nan, inf = float("nan"), float("inf")
    z = logits(16, 500, "f32", 10)
    f = lambda *a: torch.tensor(a, device="cuda:0")  # noqa: E731
    u = f(-0.1, 1.0, nan, .5, .5, .5, .5, .5, .5, .5, .5, .5, .5, .5, .5, .5)
    t = f(1., 1., 1., -1., nan, inf, 1., 1., 1., 1., 1., 1., 1., 1., 1., -0.0)
    k = torch.tensor([0, 0, 0, 0, 0, 0, -1, 0, 0, 0, 0, 0, 0, 2 ** 31 - 1, 5, 0], dtype=torch.int32, device="cuda:0")
    p = f(1., 1., 1., 1., 1., 1., 1., -.1, 1.1, nan, 1., 1., 1., 1., .5, 1.)
    m = f(0., 0., 0., 0., 0., 0., 0., 0., 0., 0., -.1, 1.1, nan, 0., 0., 0.)
    token = check(z, u, t, k, p, m)
    assert (token[:13] == -1).all() and (token[13:] >= 0).all()


def test_shares_of_tokens_are_their_probabilities():
    """One row for all, u at the middles of n equal parts: a token's count is n times its probability, to one."""
    n, vocab = 4096, 300
    z = logits(1, vocab, "f32", 11, 1.5)
    u = (torch.arange(n, device="cuda:0") + 0.5) / n
    token = ee.sample(z.expand(n, vocab), u, temperature=0.8)
    count = torch.bincount(token.long(), minlength=vocab).cpu().double()
    want = torch.softmax(z[0].double().cpu() / 0.8, 0) * n
    assert ((count - want).abs() <= 1 + 1e-6).all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_layouts(dtype):
    rows, vocab = 5, 2001
    z = logits(rows, vocab, dtype, 12)
    a = mixed(rows, 13)
    want = ee.sample(z, a[0], temperature=a[1], top_k=a[2], top_p=a[3], min_p=a[4], scores=True)
    flat = logits(1, rows * (vocab + 40) + 8, dtype, 14)[0]
    for at, row in ((1, vocab), (8, vocab + 7), (3, vocab + 31), (0, vocab + 39)):
        v = flat[:at + row * rows].as_strided((rows, vocab), (row, 1), at)
        v.copy_(z)
        got = ee.sample(v, a[0], temperature=a[1], top_k=a[2], top_p=a[3], min_p=a[4], scores=True)
        assert all(torch.equal(x, y) for x, y in zip(got, want)), (at, row)


def test_no_rows_and_given_results():
    assert ee.sample(logits(0, 100), torch.zeros(0, device="cuda:0")).shape == (0,)
    z, u = logits(3, 100, "f32", 15), torch.tensor([0.1, 0.5, 0.9], device="cuda:0")
    out = torch.zeros(3, dtype=torch.int32, device="cuda:0")
    assert ee.sample(z, u, out=out) is out and torch.equal(out, ee.sample(z, u))


def test_past_32_bits():
    """Rows whose offsets pass 2^31 elements."""
    rows, vocab = 8600, 262144
    z = torch.empty(rows, vocab, dtype=torch.bfloat16, device="cuda:0")
    z[:] = logits(1, vocab, "bf16", 16)
    z[rows - 1] = logits(1, vocab, "bf16", 17)[0]
    u = torch.full((rows,), 0.3, device="cuda:0")
    token = ee.sample(z, u, top_p=0.9)
    assert (token[:-1] == token[0]).all()
    check(z[-2:], u[-2:], None, None, 0.9)
    assert torch.equal(ee.sample(z[-2:], u[-2:], top_p=0.9), token[-2:])


@pytest.mark.parametrize("rows", [1, 40])
def test_another_stream_and_captured_calls(rows):
    z, (u, t, k, p, m) = logits(rows, 5000, "f32", 18), mixed(rows, 19)
    call = lambda zz, uu, **kw: ee.sample(zz, uu, temperature=t, top_k=k, top_p=p, min_p=m, scores=True, **kw)  # noqa: E731
    want = call(z, u)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    got = call(z, u, stream=s)
    s.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    zs, us, outs, graphs = [z.clone(), z.clone()], [u.clone(), u.clone()], [], []
    for i in range(2):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            outs.append(call(zs[i], us[i]))
        graphs.append(g)
    for i in range(5):
        a, b = logits(rows, 5000, "f32", 30 + i), torch.rand(rows, device="cuda:0", generator=gen(40 + i))
        zs[i % 2].copy_(a), us[i % 2].copy_(b)
        eager = call(a, b)
        graphs[i % 2].replay()
        torch.cuda.synchronize()
        assert all(torch.equal(x, y) for x, y in zip(outs[i % 2], eager)), i


def test_two_streams_at_once():
    z, w = logits(3, 60000, "f32", 20), logits(50, 9000, "bf16", 21)
    a, b = mixed(3, 22), mixed(50, 23)
    call = lambda z, a, **kw: ee.sample(z, a[0], temperature=a[1], top_k=a[2], top_p=a[3], min_p=a[4], **kw)  # noqa: E731
    want = call(z, a), call(w, b)
    torch.cuda.synchronize()
    s, t = torch.cuda.Stream(), torch.cuda.Stream()
    got = [(call(z, a, stream=s), call(w, b, stream=t)) for _ in range(20)]
    torch.cuda.synchronize()
    assert all(torch.equal(x, want[0]) and torch.equal(y, want[1]) for x, y in got)


@pytest.mark.parametrize("rows,vocab", [(127, 16384), (200, 20011), (300, 50304), (700, 16399), (1100, 17000), (2500, 16500)])
def test_a_row_does_not_depend_on_the_others(rows, vocab):
    """However many workgroups a row of many candidates gets, which depends on the number of rows, its token stays the same."""
    z = logits(rows, vocab, "bf16" if rows % 2 else "f32", rows, 1.5)
    u, t, k, p, m = mixed(rows, vocab)
    p = torch.where(torch.arange(rows, device="cuda:0") % 3 == 0, 0.97, p)
    got = ee.sample(z, u, temperature=t, top_k=k, top_p=p, min_p=m)
    few = [ee.sample(z[i:i + 9], u[i:i + 9], temperature=t[i:i + 9], top_k=k[i:i + 9], top_p=p[i:i + 9], min_p=m[i:i + 9]) for i in range(0, rows, 9)]
    assert torch.equal(got, torch.cat(few)) and (got >= 0).all()
    for i in range(0, rows, max(1, rows // 12)):
        assert int(got[i]) == ref.choose(z[i].double().cpu().numpy(), float(u[i]), float(t[i]), int(k[i]), float(p[i]), float(m[i]))[0], i


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("vocab", [5003, 50304])
def test_min_p_above_the_other_cuts(vocab, dtype):
    """Many tokens within min-p's reach, which ends above where top-k and top-p cut, below it, exactly on a logit, at 0 and where all logits are
    equal."""
    z = logits(12, vocab, dtype, 21, 1.0)
    z[3] = (z[3] * 4).round() / 4
    z[4] = 0.0
    z[5] = z[5].abs().clamp_min(2.0 ** -20)
    z[5, :9] = 0.0
    z[6] += 1000
    z[7] = torch.where(z[7] > 0, 1.0, -1.0)
    z[8] -= z[8].max() - 2.0
    z[9, ::3] = -torch.inf
    u = torch.rand(12, device="cuda:0", generator=gen(8))
    for t, k, p, m in ((1.0, 0, 1.0, 1e-3), (1.0, 0, 1.0, math.exp(-2.0)), (1.0, 0, 0.999, 0.02), (2.0, vocab // 2, 0.99, 0.05), (0.5, vocab // 2, 1.0, 1e-4), (1.0, 0, 0.6, 1e-9),
                       (1.0, vocab - 1, 1.0, 1.0), (30.0, 0, 0.9999, 0.8), (1.0, vocab // 3, 1.0, math.exp(-1.5))):
        check(z, u, t, k, p, m)
