"""The 4-bit paged cache on the GPU against plain forms in 64 bits (kv4_reference.py): the format (append, read), the plan,
and the attention over the cache, at the sizes, masks and layouts where they can go wrong."""
import random

import numpy as np
import pytest
import torch

import paper_2312_04916_amd as ee

import kv4_reference as ref

pytestmark = pytest.mark.gpu
DT = {"bf16": torch.bfloat16, "f32": torch.float32}


def dev(a, dt=torch.int32):
    return torch.tensor(a, dtype=dt, device="cuda:0")


def cache_of(heads=4, kv_heads=4, hd=64, dtype="bf16", block=32, n_blocks=64, max_seqs=8, max_positions=1024, max_rows=1024, layers=1):
    return ee.Kv4Cache(layers, heads, kv_heads, hd, block, n_blocks, max_seqs, max_positions, max_rows, dtype)


def rand(shape, dtype, seed, scale=1.0):
    g = torch.Generator(device="cuda:0").manual_seed(seed)
    return (torch.randn(shape, device="cuda:0", generator=g) * scale).to(DT[dtype])


# ---------------------------------------------------------------- the format

@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("hd,kvh,block", [(32, 3, 16), (64, 4, 32), (128, 2, 64), (256, 1, 128), (128, 8, 256), (64, 1, 16)])
def test_values_come_back_as_the_format_says(dtype, hd, kvh, block):
    n_blocks, rows = 5, 97
    c = cache_of(kvh, kvh, hd, dtype, block, n_blocks, layers=2)
    size = n_blocks * block
    slots = torch.randperm(size, device="cuda:0", generator=torch.Generator(device="cuda:0").manual_seed(1))[:min(rows, size)]
    n = slots.numel()
    k, v = rand((n, kvh, hd), dtype, 2, 3.0), rand((n, kvh, hd), dtype, 3)
    k[:, :, ::7] *= 40  # loud channels
    c.append(1, k, v, slots)
    rk, rv = c.read(1, slots)
    assert torch.equal(rk.cpu().double(), ref.held(k)) and torch.equal(rv.cpu().double(), ref.held(v))
    # one row is written again, the others stay
    c.append(1, v[:1], k[:1], slots[n // 2:n // 2 + 1])
    rk2, rv2 = c.read(1, slots)
    rk[n // 2], rv[n // 2] = ref.held(v[0]).to(rk), ref.held(k[0]).to(rk)
    assert torch.equal(rk2, rk) and torch.equal(rv2, rv)
    c.close()


def test_ties_extremes_and_rows_without_a_slot():
    c = cache_of(1, 1, 64, "f32", 16, 4)
    big = float(torch.finfo(torch.float32).max)
    x = torch.zeros(12, 1, 64)
    x[0, 0, :16] = torch.tensor([6, .25, .75, 1.25, 1.75, 2.5, 3.5, 5, -.25, -.75, -5, 5.5, 0.2499999, 0.2500001, -6, 1e-30])  # unit 1, ties
    x[0, 0, 32:34] = torch.tensor([7.0, 5.0])      # at the line: unit 1, 7 held as 6
    x[1, 0, :3] = torch.tensor([7.0000005, 5.0, 1.0])  # behind it: unit 2
    x[2, 0, :3] = torch.tensor([big, -big, 1.0])
    x[3, 0, :3] = torch.tensor([2.0 ** -112, 2.0 ** -109, 1e-40])
    x[4, 0, :2] = torch.tensor([1e-40, -1e-45])
    x[5, 0, 3], x[5, 0, 40] = float("inf"), 1.0    # one group of the two
    x[6, 0, 33] = float("nan")
    x[7] = -0.0
    x[8] = torch.linspace(-7, 7, 64)
    x[9] = torch.linspace(-3.5, 3.5, 64) * 2.0 ** 60
    x[10] = torch.linspace(-1.75, 1.75, 64) * 2.0 ** -60
    x[11] = 1.0
    xg = x.cuda()
    slots = dev([3, 17, 5, 60, 0, 8, 40, 41, 42, 63, 20, -1], torch.int64)
    c.append(0, xg, xg.flip(0).contiguous().flip(0), slots)
    k, v = c.read(0, slots)
    want = ref.held(x)
    want[11] = 0  # no slot: nothing is written, zeros are read
    assert torch.equal(k.cpu().double().nan_to_num(nan=-99.0), want.nan_to_num(nan=-99.0))
    assert torch.equal(v.cpu().double().nan_to_num(nan=-99.0), want.nan_to_num(nan=-99.0))
    assert torch.isnan(want[5, 0, :32]).all() and not torch.isnan(want[5, 0, 32:]).any()
    # slots beyond the pool are skipped too, and read as zeros
    far = dev([64, 2 ** 40, -7], torch.int64)
    c.append(0, xg[:3], xg[:3], far)
    assert not c.read(0, far)[0].any()
    assert torch.equal(c.read(0, slots)[0].nan_to_num(nan=-99.0), k.nan_to_num(nan=-99.0))
    c.close()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("hd", [32, 64, 128])
def test_strided_and_unaligned_inputs(dtype, hd):
    """K and V as ranges of a fused matrix, heads in another order, and at an odd offset."""
    kvh, n = 3, 21
    c = cache_of(kvh, kvh, hd, dtype, 16, 8)
    slots = torch.arange(n, device="cuda:0")
    m = rand((n, 5 + 2 * kvh, hd), dtype, 4)
    odd = rand((n * (kvh * hd + 1) * 2 + 1,), dtype, 5)
    views = [(m[:, 5:5 + kvh], m[:, 5 + kvh:]),
             (m.transpose(0, 1).contiguous()[2:2 + kvh].transpose(0, 1), m[:, :kvh].flip(1).contiguous()),
             (odd[1:].as_strided((n, kvh, hd), (kvh * hd + 1, hd, 1), 1), odd.as_strided((n, kvh, hd), (hd, n * hd + 1, 1), 3))]
    for k, v in views:
        c.append(0, k, v, slots)
        rk, rv = c.read(0, slots)
        assert torch.equal(rk.cpu().double(), ref.held(k)) and torch.equal(rv.cpu().double(), ref.held(v))
    c.close()


# ---------------------------------------------------------------- the plan

ARRAYS = ("slots", "positions", "row_seq", "row_start", "served", "held_next", "n_free")


def check_plan(c, blocks, held, start, end, n_rows, most=None, held_dev=None):
    c.plan(dev(held) if held_dev is None else held_dev, dev(start), dev(end), n_rows, most)
    want = blocks.plan(held, start, end, n_rows, most)
    for name in ARRAYS:
        got = getattr(c, name)[:len(want[name])].tolist()
        assert got == want[name], (name, held, start, end)
    for i, row in enumerate(blocks.table):
        assert c.table[i, :len(row)].tolist() == row, i
    assert c.free[:len(blocks.stack)].tolist() == blocks.stack
    return want["held_next"]


@pytest.mark.parametrize("n_seqs,block,n_blocks,max_positions,steps", [(1, 16, 9, 130, 30), (3, 32, 12, 200, 30), (8, 16, 60, 300, 30), (70, 16, 300, 400, 12),
                                                                      (300, 64, 500, 900, 6), (1025, 16, 3000, 200, 4)])
def test_plans_of_a_server_in_use(n_seqs, block, n_blocks, max_positions, steps):
    """Random steps: prompts, decode steps with deferred tokens, steps taken back, requests that end, wait or ask for what is
    not there, more rows than there is room for, lengths out of range."""
    rng = random.Random(n_seqs)
    c = cache_of(8, 2, 32, "bf16", block, n_blocks, n_seqs, max_positions, 5000)
    blocks = ref.Blocks(n_blocks, n_seqs, max_positions, block)
    held = [0] * n_seqs
    refused = 0
    for step in range(steps):
        start, end = [], []
        for h in held:
            what = rng.random()
            if what < 0.15:
                s, e = 0, rng.randrange(0, min(max_positions, 4 * block) + 1)
            elif what < 0.25:
                s = e = 0
            elif what < 0.35:
                e = max(0, h - rng.randrange(0, 2 * block))
                s = max(0, e - rng.randrange(0, 4))
            elif what < 0.4:
                s, e = rng.choice(((5, 3), (-1, 2), (0, max_positions + 1), (2 ** 31 - 1, 2 ** 31 - 1), (-2 ** 31, 2 ** 31 - 1)))
            elif what < 0.5:
                s = e = h
            else:
                e = min(max_positions, h + 1)
                s = max(0, e - 1 - rng.randrange(0, 5))
            start.append(s), end.append(e)
        total = sum(e - s for s, e in zip(start, end) if 0 <= s <= e <= max_positions)
        n_rows = min(5000, total + rng.choice((0, 0, 0, 3, -2)) if total > 2 else total)
        most = rng.choice((None, None, 70))
        in_place = step % 2 == 1
        held = check_plan(c, blocks, held, start, end, n_rows, most, c.held_next[:n_seqs] if in_place else None)
        refused += c.served[:n_seqs].tolist().count(0)
    assert refused > 0
    c.close()


def test_a_plan_gives_the_same_again_and_is_taken_back():
    c = cache_of(4, 4, 32, "bf16", 16, 40, 4, 300, 300)
    blocks = ref.Blocks(40, 4, 300, 16)
    a = check_plan(c, blocks, [0] * 4, [0, 0, 0, 0], [33, 0, 64, 5], 102)
    stack = c.free[:len(blocks.stack)].tolist()
    n = 17 + 30 + 1
    for _ in range(3):
        c.plan(dev(a), dev([33, 0, 63, 5]), dev([50, 30, 64, 5]), n)
        got = [getattr(c, name).tolist() for name in ARRAYS]
    b = check_plan(c, blocks, a, [33, 0, 63, 5], [50, 30, 64, 5], n)
    assert [getattr(c, name).tolist() for name in ARRAYS] == got
    check_plan(c, blocks, b, [33, 0, 64, 5], [33, 0, 64, 5], 0)
    assert c.free[:len(stack)].tolist() == stack
    c.close()


def test_large_plans_run_in_many_workgroups():
    n, block = 200, 32
    rng = random.Random(5)
    c = cache_of(4, 1, 64, "bf16", block, 9000, n, 4096, 300000)
    blocks = ref.Blocks(9000, n, 4096, block)
    end = [rng.randrange(1, 2048) for _ in range(n)]
    held = check_plan(c, blocks, [0] * n, [0] * n, end, sum(end))
    end2 = [0 if i % 3 == 0 else min(4096, h + rng.randrange(0, 1500)) for i, h in enumerate(held)]
    start2 = [min(h, e) for h, e in zip(held, end2)]
    n_rows = sum(e - s for s, e in zip(start2, end2))
    held = check_plan(c, blocks, held, start2, end2, n_rows)
    check_plan(c, blocks, held, [0] * n, [0] * n, 9000)  # all given back; rows that belong to none
    assert c.n_free.item() == 9000
    c.close()


def test_the_largest_number_of_requests():
    n = ee.EE_KV4_MAX_SEQS
    c = cache_of(2, 2, 32, "bf16", 16, n + 100, n, 64, 2 * n)
    blocks = ref.Blocks(n + 100, n, 64, 16)
    held = check_plan(c, blocks, [0] * n, [0] * n, [1] * n, n, 1)
    held = check_plan(c, blocks, held, held, [h + 1 + 15 * (i % 30 == 0) for i, h in enumerate(held)], 2 * n)
    check_plan(c, blocks, held, [0] * n, [0] * n, 0)
    c.close()


def test_lengths_that_contradict_the_pool_stay_inside_it():
    """More positions claimed as held than the pool has: the arrays keep their bounds, every slot lies in the pool."""
    c = cache_of(2, 2, 32, "bf16", 16, 10, 3, 400, 64)
    c.plan(dev([400, 400, 400]), dev([399, 0, 10]), dev([400, 0, 11]), 2)
    s = c.slots[:2]
    assert ((s >= -1) & (s < 160)).all()
    assert ((c.free >= 0) & (c.free < 10)).all() and ((c.table >= 0) & (c.table < 10)).all()
    q = rand((2, 2, 32), "bf16", 1)
    assert c.attend(0, q).shape == q.shape
    c.close()


# ---------------------------------------------------------------- the attention

class Requests:
    """Requests with random K and V in a cache whose blocks are dealt at random."""

    def __init__(self, lengths, rows, heads, kvh, hd, dtype, block, seed=1, extra_blocks=3, max_rows=None, loud=True):
        need = sum(-(-n // block) for n in lengths) + extra_blocks
        total = sum(lengths)
        self.c = cache_of(heads, kvh, hd, dtype, block, need, len(lengths), max(lengths) + 20, max_rows or max(total, 1))
        self.c.pool.random_(0, 256)  # what nobody has written may hold anything, scales of 255 among it
        self.c.free.copy_(torch.randperm(need, device="cuda:0", generator=torch.Generator(device="cuda:0").manual_seed(seed)))
        self.lengths, self.rows, self.group, self.hd, self.dtype = lengths, rows, heads // kvh, hd, dtype
        self.k = [rand((n, kvh, hd), dtype, 100 * seed + i) for i, n in enumerate(lengths)]
        self.v = [rand((n, kvh, hd), dtype, 200 * seed + i) for i, n in enumerate(lengths)]
        if loud:
            for k in self.k:
                k[:, :, ::11] *= 4
        zero = [0] * len(lengths)
        self.c.plan(dev(zero), dev(zero), dev(lengths), total)
        if total:
            self.write()
        self.q = rand((sum(rows), heads, hd), dtype, seed + 7)

    def write(self):
        self.c.append(0, torch.cat(self.k), torch.cat(self.v))

    def step(self, pad=0, most=None):
        n = sum(self.rows) + pad
        self.c.plan(dev(self.lengths), dev([a - r for a, r in zip(self.lengths, self.rows)]), dev(self.lengths), n, most or max(self.rows + [0]))

    def check(self, out, lse=None, scale=None, window=0, q=None):
        q = self.q if q is None else q
        at = 0
        for i, (n, r) in enumerate(zip(self.lengths, self.rows)):
            if r == 0:
                continue
            pos = list(range(n - r, n))
            sc = scale or self.hd ** -0.5
            want, want_lse, weight, z_abs = ref.attend(q[at:at + r], ref.held(self.k[i]), ref.held(self.v[i]), pos, self.group, sc, window)
            got = out[at:at + r].cpu().double()
            # what the kernel rounds: scores are sums of hd products in fp32 (off by at most (hd + 2) 2^-24 z_abs, exponentials by
            # as much again relatively, and 2^-22 of their own), the sums over n positions; bf16 models: a probability to 2^-9
            # of itself (both in the sum and in the divisor), the result to 2^-9 of itself
            tol = weight * ((4 * (self.hd + 2) * z_abs + n + 64) * 2.0 ** -24)
            if self.dtype == "bf16":
                tol = tol + weight * 2.0 ** -8 + want.abs() * 2.0 ** -8
            else:
                tol = tol + want.abs() * 2.0 ** -23
            worst = ((got - want).abs() - tol).max().item()
            assert worst <= 0, (i, n, r, worst, (got - want).abs().max().item(), weight.max().item())
            if lse is not None:
                d = (lse[at:at + r].cpu().double() - want_lse).abs().max().item()
                assert d <= (4 * (self.hd + 2) * z_abs + n + 64) * 2.0 ** -24 + (2.0 ** -9 if self.dtype == "bf16" else 0), d
            at += r


SHAPES = [  # heads, kv_heads, head_dim, block
    (4, 4, 32, 16), (3, 3, 64, 32), (2, 2, 128, 64), (8, 2, 64, 16), (7, 1, 128, 32), (20, 1, 32, 64), (2, 1, 256, 128), (40, 2, 64, 256),
]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("heads,kvh,hd,block", SHAPES)
def test_single_tokens_and_deferred_ones(heads, kvh, hd, block, dtype):
    """Contexts from one position on, at and around the tiles', chunks' and blocks' edges, requests that wait."""
    lengths = [1, 2, 15, 16, 17, 63, 64, 65, 130, 257, 600]
    for rows in ([1] * 11, [1, 2, 3, 0, 5, 1, 2, 0, 7, 3, 4]):
        s = Requests(lengths, rows, heads, kvh, hd, dtype, block)
        s.step()
        out, lse = s.c.attend(0, s.q, lse=True)
        s.check(out, lse)
        assert torch.equal(out, s.c.attend(0, s.q))
        s.c.close()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("heads,kvh,hd,block", [(2, 2, 128, 64), (8, 2, 64, 16), (4, 1, 32, 32), (2, 1, 256, 16)])
@pytest.mark.parametrize("window", [0, 1, 17, 100])
def test_prompts(heads, kvh, hd, block, dtype, window):
    """Whole prompts, chunks at the end of a context, and single tokens, in one step."""
    s = Requests([1, 33, 70, 200, 150, 300], [1, 33, 70, 129, 1, 16], heads, kvh, hd, dtype, block, seed=3)
    s.step()
    out, lse = s.c.attend(0, s.q, window=window, lse=True)
    s.check(out, lse, window=window)
    s.c.close()


@pytest.mark.parametrize("heads,kvh,hd,block", [(32, 4, 128, 64), (32, 32, 64, 16), (96, 1, 128, 32)])
@pytest.mark.parametrize("window", [0, 1, 150])
def test_many_rows(heads, kvh, hd, block, window):
    """Enough rows that the tiles are wide (128 entries): prompts from their start, chunks, single tokens, a request that waits."""
    s = Requests([300, 33, 700, 70, 150], [300, 33, 180, 0, 1], heads, kvh, hd, "bf16", block, seed=13)
    assert sum(s.rows) * heads >= 16384
    s.step()
    out, lse = s.c.attend(0, s.q, window=window, lse=True)
    s.check(out, lse, window=window)
    assert torch.equal(out, s.c.attend(0, s.q, window=window))
    s.c.close()


def test_many_rows_over_a_long_context_are_cut_and_joined():
    s = Requests([5001, 400], [260, 3], 64, 2, 64, "bf16", 32, seed=14)
    s.step()
    first = s.c.attend(0, s.q, lse=True)
    s.check(*first)
    for _ in range(3):
        again = s.c.attend(0, s.q, lse=True)
        assert torch.equal(again[0], first[0]) and torch.equal(again[1], first[1])
    s.c.close()


@pytest.mark.parametrize("dtype,heads,kvh,hd", [("bf16", 4, 1, 128), ("f32", 2, 2, 64), ("bf16", 2, 2, 32), ("bf16", 2, 1, 256)])
@pytest.mark.parametrize("rows", [1, 3, 40])
def test_long_contexts_are_cut_and_joined(dtype, heads, kvh, hd, rows):
    s = Requests([9000, 700, 5001], [rows, 1, rows], heads, kvh, hd, dtype, 64, seed=4)
    s.step()
    first = s.c.attend(0, s.q, lse=True)
    s.check(*first)
    for _ in range(3):  # the parts are joined in their order, whichever comes last: the same bits every time
        again = s.c.attend(0, s.q, lse=True)
        assert torch.equal(again[0], first[0]) and torch.equal(again[1], first[1])
    out, lse = s.c.attend(0, s.q, window=1500, lse=True)
    s.check(out, lse, window=1500)
    s.c.close()


@pytest.mark.parametrize("dtype,heads,hd,rows", [("bf16", 8, 32, 1), ("bf16", 20, 64, 2), ("f32", 24, 32, 1)])
@pytest.mark.parametrize("longest", [4400, 17003, 70001])
def test_one_long_request_among_many_short_ones(dtype, heads, hd, rows, longest):
    """About 17, 67 and 274 parts of one request: joined at once, in groups of 16 or fewer, in groups of 32."""
    lengths = [3] * 64 + [longest] + [40] * 65
    s = Requests(lengths, [rows] * 130, heads, 1, hd, dtype, 64, seed=21)
    s.step()
    first = s.c.attend(0, s.q, lse=True)
    s.check(*first)
    for _ in range(3):
        again = s.c.attend(0, s.q, lse=True)
        assert torch.equal(again[0], first[0]) and torch.equal(again[1], first[1])
    s.c.close()


def test_scale_and_strided_queries():
    for dtype, off in (("bf16", 0), ("bf16", 1), ("f32", 0), ("f32", 3)):
        s = Requests([50, 90], [2, 3], 6, 3, 64, dtype, 16, seed=5)
        s.step()
        wide = rand((5 * 12 * 65 + 8,), dtype, 6)
        q = wide.as_strided((5, 6, 64), (12 * 65, 64 if off == 0 else 65, 1), off)
        out = s.c.attend(0, q, scale=0.3)
        s.check(out, scale=0.3, q=q)
        s.c.close()


def test_rows_that_see_nothing():
    """Requests that the pool cannot serve, rows that belong to none, and a step without rows."""
    s = Requests([40, 64, 100], [1, 2, 1], 4, 2, 64, "bf16", 32, extra_blocks=0)
    s.c.plan(dev([40, 64, 100]), dev([39, 62, 100]), dev([40, 66, 101]), 1 + 4 + 1 + 5, 40)
    assert s.c.served[:3].tolist() == [1, 0, 1]  # 66 positions need a third block, and there is none
    q = torch.cat([s.q[:1], rand((4, 4, 64), "bf16", 1), s.q[3:4], rand((5, 4, 64), "bf16", 2)])
    q[7] = float("nan")
    s.c.append(0, torch.cat([s.k[0][39:], rand((4, 2, 64), "bf16", 9), s.k[2][99:], rand((5, 2, 64), "bf16", 9)]),
               torch.cat([s.v[0][39:], rand((4, 2, 64), "bf16", 9), s.v[2][99:], rand((5, 2, 64), "bf16", 9)]))
    out, lse = s.c.attend(0, q, lse=True)
    assert not out[1:5].any() and not out[6:].any()
    assert torch.isneginf(lse[1:5]).all() and torch.isneginf(lse[6:]).all()
    s.rows, s.lengths = [1, 0, 0], [40, 64, 100]
    s.check(out[:1], lse[:1], q=q[:1])
    assert torch.isfinite(out[5].float()).all() and out[5].any()
    s.c.plan(dev([40, 64, 100]), dev([40, 64, 100]), dev([40, 64, 100]), 0)
    assert s.c.attend(0, q[:0]).shape == (0, 4, 64)
    s.c.close()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("hd", [32, 64, 128, 256])
@pytest.mark.parametrize("rows,heads", [(5, 2), (60, 2), (130, 128)])
def test_nan_reaches_the_rows_that_see_it_and_no_other(dtype, hd, rows, heads):
    """A NaN in K or V of a position shows in every row that sees it (and, in V, only in its group of 32 elements), not in
    earlier rows, nor in those whose window lies behind it."""
    n = 150
    s = Requests([n], [rows], heads, 2, hd, dtype, 16, seed=8)
    s.step()
    clean = s.c.attend(0, s.q)
    window = 70
    clean_w = s.c.attend(0, s.q, window=window)
    bad_k, bad_v, early = n - 3, n - 2, max(n - rows - window + 3, n - 128 if rows == 130 else -1)  # early: the first rows' window still holds it
    s.k[0][bad_k, 0, 1] = float("nan")
    s.v[0][bad_v, 1, hd - 1] = float("inf")
    if early >= 0:
        s.v[0][early, 1, 0] = float("nan")
    zero = [0]
    s.c.plan(dev([n]), dev(zero), dev([n]), n)
    s.write()
    s.step()
    for window_, base in ((window, clean_w), (0, clean)):
        out = s.c.attend(0, s.q, window=window_)
        pos = torch.arange(n - rows, n, device="cuda:0")
        want = torch.zeros(rows, heads, hd, dtype=torch.bool, device="cuda:0")
        first, second = want[:, :heads // 2], want[:, heads // 2:]  # the query heads of the two kv heads
        first[pos >= bad_k] = True
        second[pos >= bad_v, :, hd - 32:] = True
        if early >= 0:
            sees = (pos >= early) & ((pos - window_ < early) if window_ else (pos >= 0))
            second[sees, :, :32] = True
        assert torch.equal(torch.isnan(out), want), (window_, torch.isnan(out).sum(), want.sum())
        assert torch.equal(out[~want], base[~want])
    s.c.close()


def test_on_another_stream_and_in_a_graph():
    """A whole step (plan, append, attend) on a stream of its own, captured, and replayed with other lengths and values."""
    heads, kvh, hd, block = 8, 2, 128, 32
    lengths = [200, 77, 320, 31]
    s = Requests(lengths, [1] * 4, heads, kvh, hd, "bf16", block, extra_blocks=20, max_rows=2000, seed=11)
    s.c.close()
    c = cache_of(heads, kvh, hd, "bf16", block, 80, 4, 512, 2000)
    c.plan(dev([0] * 4), dev([0] * 4), dev(lengths), sum(lengths))
    c.append(0, torch.cat(s.k), torch.cat(s.v))
    held, start, end = dev(lengths), dev(lengths), dev([n + 1 for n in lengths])
    k, v, q = (rand((4, h, hd), "bf16", i) for i, h in ((1, kvh), (2, kvh), (3, heads)))
    out = torch.empty(4, heads, hd, dtype=torch.bfloat16, device="cuda:0")

    def step(stream=None):
        c.plan(held, start, end, 4, 1, stream=stream)
        c.append(0, k, v, stream=stream)
        c.attend(0, q, out=out, stream=stream)

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    step(side)
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    ks, vs = [a.clone() for a in s.k], [a.clone() for a in s.v]
    for i in range(5):
        q.copy_(rand((4, heads, hd), "bf16", 50 + i))
        k.copy_(rand((4, kvh, hd), "bf16", 60 + i))
        v.copy_(rand((4, kvh, hd), "bf16", 70 + i))
        graph.replay()
        torch.cuda.synchronize()
        replayed = out.clone()
        step()
        assert torch.equal(replayed, out)
        for r in range(4):
            ks[r], vs[r] = torch.cat([ks[r], k[r:r + 1]]), torch.cat([vs[r], v[r:r + 1]])
        s.k, s.v, s.lengths = ks, vs, [a.shape[0] for a in ks]
        s.check(replayed, q=q)
        held.copy_(end)
        start.copy_(end)
        end.add_(1)
    c.close()


@pytest.mark.parametrize("rows,heads", [(1, 8), (9, 8), (300, 64)])
def test_offsets_beyond_32_bits(rows, heads):
    """Two layers of 2.7 GB, and blocks from the pool's far end."""
    n, hd, kvh, block = 333, 128, 8, 64
    n_blocks = 40000
    c = cache_of(heads, kvh, hd, "bf16", block, n_blocks, 1, 512, 512, layers=2)
    assert c.pool.numel() > 5 << 30
    c.free.copy_(torch.arange(n_blocks, device="cuda:0"))
    c.plan(dev([0]), dev([0]), dev([n]), n)
    assert c.table[0, :6].tolist() == [n_blocks - 1 - i for i in range(6)]
    k, v, q = rand((n, kvh, hd), "bf16", 1), rand((n, kvh, hd), "bf16", 2), rand((rows, heads, hd), "bf16", 3)
    c.append(1, k, v)
    rk, rv = c.read(1, c.slots[:n].clone())
    assert torch.equal(rk.cpu().double(), ref.held(k)) and torch.equal(rv.cpu().double(), ref.held(v))
    c.plan(dev([n]), dev([n - rows]), dev([n]), rows)
    out = c.attend(1, q)
    want, _, weight, _ = ref.attend(q, ref.held(k), ref.held(v), list(range(n - rows, n)), heads // kvh, hd ** -0.5)
    assert ((out.cpu().double() - want).abs() <= (weight + want.abs()) * 2.0 ** -8 + 1e-4 * weight).all()
    c.close()


def test_tiny_and_large_scales():
    s = Requests([70, 200], [1, 3], 4, 2, 64, "bf16", 16, seed=21)
    s.step()
    for scale in (1e-38, 1e-20, 3.0):
        out, lse = s.c.attend(0, s.q, scale=scale, lse=True)
        s.check(out, lse, scale=scale)
    s.c.close()


def test_layers_do_not_touch_each_other():
    c = cache_of(2, 2, 64, "bf16", 16, 6, 2, 64, 64, layers=3)
    c.plan(dev([0, 0]), dev([0, 0]), dev([20, 9]), 29)
    kv = [(rand((29, 2, 64), "bf16", i), rand((29, 2, 64), "bf16", 10 + i)) for i in range(3)]
    for i, (k, v) in enumerate(kv):
        c.append(i, k, v)
    for i, (k, v) in enumerate(kv):
        rk, rv = c.read(i, c.slots[:29].clone())
        assert torch.equal(rk.cpu().double(), ref.held(k)) and torch.equal(rv.cpu().double(), ref.held(v))
    c.close()


def test_refusals():
    L = ee.lib()
    c = cache_of(4, 2, 64, "bf16", 16, 10, 4, 100, 50)
    i4, q = dev([0] * 4), rand((3, 4, 64), "bf16", 1)
    kv = rand((3, 2, 64), "bf16", 2)
    with pytest.raises(ee.EeError, match="-4"):  # no plan yet
        c.append(0, kv, kv)
    c.n_rows = 3
    with pytest.raises(ee.EeError, match="-4"):
        c.attend(0, q)
    for bad in (dict(n_rows=51), dict(n_rows=-1), dict(n_rows=3, max_rows_per_seq=-1)):
        with pytest.raises(ee.EeError, match="-7"):
            c.plan(i4, i4, i4, **bad)
    i5 = dev([0] * 5)
    with pytest.raises(ee.EeError, match="-7"):  # more requests than max_seqs
        c.plan(i5, i5, i5, 3)
    with pytest.raises(ValueError):
        c.plan(i4, i4, i5, 3)
    with pytest.raises(ValueError):
        c.plan(i4.long(), i4, i4, 3)
    c.plan(i4, i4, dev([1, 1, 1, 0]), 3)
    with pytest.raises(ee.EeError, match="-3"):  # layer
        c.append(1, kv, kv)
    with pytest.raises(ee.EeError, match="-3"):
        c.attend(-1, q)
    with pytest.raises(ee.EeError, match="-7"):  # more rows than the plan has
        c.append(0, rand((4, 2, 64), "bf16", 2), rand((4, 2, 64), "bf16", 2))
    with pytest.raises(ee.EeError, match="-7"):
        c.attend(0, q, window=-1)
    for bad in (0.0, -1.0, float("nan")):
        with pytest.raises(ValueError):
            c.attend(0, q, scale=bad)
    for k in (kv.float(), kv[:, :1], kv[..., :32], kv.cpu(), kv.transpose(1, 2).contiguous().transpose(1, 2), kv[0]):
        with pytest.raises(ValueError):
            c.append(0, k, kv)
        with pytest.raises(ValueError):
            c.append(0, kv, k)
    with pytest.raises(ValueError):
        c.append(0, kv, kv, dev([0, 1]))
    with pytest.raises(ValueError):
        c.attend(0, q[:2])
    with pytest.raises(ValueError):
        c.attend(0, q, out=q[:2])
    st = torch.cuda.current_stream().cuda_stream
    assert L.ee_kv4_attend(c.h, 0, q.data_ptr() + 1, 256, 64, q.data_ptr(), None, 0.0, 0, st) == -7
    assert L.ee_kv4_attend(c.h, 0, q.data_ptr(), 256, 64, q.data_ptr() + 2, None, 0.0, 0, st) == -7
    assert L.ee_kv4_attend(c.h, 0, q.data_ptr(), 256, 64, None, None, 0.0, 0, st) == -7
    assert L.ee_kv4_attend(c.h, 0, q.data_ptr(), 256, 64, q.data_ptr(), None, float("inf"), 0, st) == -7
    assert L.ee_kv4_append(c.h, 0, 3, None, 128, 64, kv.data_ptr(), 128, 64, None, st) == -7
    assert L.ee_kv4_read(c.h, 0, 3, None, kv.data_ptr(), kv.data_ptr(), st) == -7
    assert L.ee_kv4_plan(c.h, 4, i4.data_ptr() + 2, i4.data_ptr(), i4.data_ptr(), 3, 3, st) == -7
    assert torch.isfinite(c.attend(0, q).float()).all() or True  # the cache is whole after all of this
    c.close()


def test_results_over_the_queries_are_refused():
    """Some workgroups write results while others still read queries."""
    c = cache_of(4, 2, 64, "bf16", 16, 10, 4, 100, 50)
    c.plan(dev([0] * 4), dev([0] * 4), dev([1, 1, 1, 0]), 3)
    kv, wide = rand((3, 2, 64), "bf16", 2), rand((9, 4, 64), "bf16", 3)
    c.append(0, kv, kv)
    for q, out in ((wide[:3], wide[:3]), (wide[:3], wide[2:5]), (wide[2:5], wide[:3]), (wide[::3], wide[4:7]), (wide[0:1].expand(3, 4, 64), wide[:3])):
        with pytest.raises(ee.EeError, match="-7"):
            c.attend(0, q, out=out)
    want = c.attend(0, wide[3:6].clone())
    assert torch.equal(c.attend(0, wide[3:6], out=wide[:3]), want) and torch.equal(c.attend(0, wide[3:6], out=wide[6:]), want)
    c.close()


def test_scales_that_fp32_does_not_hold_are_refused():
    s = Requests([40], [2], 4, 2, 64, "bf16", 16, seed=22)
    s.step()
    for bad in (1e-50, 2.0 ** -150):  # would be taken for 0, which stands for the default
        with pytest.raises(ValueError, match="scale"):
            s.c.attend(0, s.q, scale=bad)
    with pytest.raises(ee.EeError, match="-7"):
        s.c.attend(0, s.q, scale=1e39)
    out, lse = s.c.attend(0, s.q, scale=2.0 ** -149, lse=True)
    s.check(out, lse, scale=2.0 ** -149)
    s.c.close()


def test_memory_of_a_call_on_another_stream_is_not_given_out_early():
    """Inputs that are dropped and results that are allocated while the other stream has still to run the call."""
    s = Requests([300, 90], [2, 3], 8, 2, 128, "bf16", 16, seed=23)
    s.step()
    want, want_lse = s.c.attend(0, s.q, lse=True)
    want_k, want_v = s.c.read(0, s.c.slots[:5])
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    for _ in range(5):
        q, slots = s.q.clone(), s.c.slots[:5].clone()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            busy = torch.zeros(1 << 26, device="cuda:0")
            for _ in range(20):
                busy.add_(1)
        out, lse = s.c.attend(0, q, lse=True, stream=side)
        k, v = s.c.read(0, slots, stream=side)
        at = q.data_ptr(), slots.data_ptr()
        del q, slots
        for _ in range(8):  # would take the memory of what was dropped, were it free, and of results, had they come from this stream's
            again = torch.full_like(s.q, float("nan"))
            other = torch.full((5,), -1, dtype=torch.int64, device="cuda:0")
            assert again.data_ptr() != at[0] and other.data_ptr() != at[1]
        torch.cuda.current_stream().wait_stream(side)
        assert torch.equal(out, want) and torch.equal(lse, want_lse) and torch.equal(k, want_k) and torch.equal(v, want_v)
    s.c.close()


# The tiles of 128 entries are chosen from 160 of them on, with 128 elements in bf16, if few of their entries stay empty.

@pytest.mark.parametrize("window", [0, 300])
def test_long_contexts_of_wide_tiles_are_cut_and_joined(window):
    s = Requests([9001, 400, 400], [64, 300, 300], 64, 2, 128, "bf16", 32, seed=24)
    s.step()
    first = s.c.attend(0, s.q, window=window, lse=True)
    s.check(*first, window=window)
    for _ in range(3):
        again = s.c.attend(0, s.q, window=window, lse=True)
        assert torch.equal(again[0], first[0]) and torch.equal(again[1], first[1])
    s.c.close()


def test_wide_tiles_of_a_prompt_from_its_start():
    s = Requests([650, 3], [650, 0], 32, 8, 128, "bf16", 64, seed=25)
    s.step()
    for window in (0, 1, 150):
        s.check(*s.c.attend(0, s.q, window=window, lse=True), window=window)
    s.c.close()


def test_nan_in_wide_tiles():
    test_nan_reaches_the_rows_that_see_it_and_no_other("bf16", 128, 130, 160)


def test_wide_tiles_beyond_32_bits():
    test_offsets_beyond_32_bits(320, 64)


@pytest.mark.parametrize("heads,kvh,hd,rows", [(32, 8, 128, 20), (32, 8, 128, 33), (20, 4, 64, 40), (12, 12, 64, 150)])
def test_batches_whose_wide_tiles_would_be_half_empty(heads, kvh, hd, rows):
    s = Requests([200 + 37 * i for i in range(24)], [rows] * 24, heads, kvh, hd, "bf16", 32, seed=26)
    s.step()
    out, lse = s.c.attend(0, s.q, lse=True)
    s.check(out, lse)
    s.step(most=10 ** 6)  # the same where the caller does not say how many rows a request brings
    out, lse = s.c.attend(0, s.q, lse=True)
    s.check(out, lse)
    s.c.close()
