"""Values at which the 4-bit cache's attention can go wrong: how probabilities are rounded, the log-sum-exp, NaN that every row sees,
infinities in queries."""
import pytest
import torch

import kv4_reference as ref
import paper_2312_04916_amd as ee
from test_gpu_kv4 import Requests, cache_of, dev, rand

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("hd,rows,heads", [(32, 3, 2), (64, 3, 2), (64, 40, 2), (128, 3, 2), (128, 20, 4), (256, 3, 2), (128, 130, 160)])
@pytest.mark.parametrize("rest", [0.0, 1.0])
def test_nan_that_every_row_sees(dtype, hd, rows, heads, rest):
    """A NaN at the first positions of a context, in a group whose other elements are `rest`: in K it is the rows' whole result, in V
    that of its group of 32 elements, whatever the queries are."""
    n = 400
    s = Requests([n], [rows], heads, 2, hd, dtype, 16, seed=31)
    s.step()
    s.q = -s.q.abs()
    clean = s.c.attend(0, s.q)
    s.k[0][3, 0, :32] = rest
    s.k[0][3, 0, 5] = float("nan")
    s.v[0][4, 1, hd - 32:] = rest
    s.v[0][4, 1, hd - 2] = float("nan")
    s.c.plan(dev([n]), dev([0]), dev([n]), n)
    s.write()
    s.step()
    out, lse = s.c.attend(0, s.q, lse=True)
    half = heads // 2
    assert torch.isnan(out[:, :half]).all() and torch.isnan(lse[:, :half]).all()
    assert torch.isnan(out[:, half:, hd - 32:]).all()
    assert torch.equal(out[:, half:, :hd - 32], clean[:, half:, :hd - 32])
    s.c.close()


@pytest.mark.parametrize("lse", [False, True])
@pytest.mark.parametrize("hd,rows,heads", [(128, 3, 2), (32, 20, 2), (64, 20, 2), (128, 20, 2), (32, 50, 2), (64, 64, 2), (128, 130, 160)])
def test_a_dominant_position_keeps_its_weight(hd, rows, heads, lse):
    """One position outweighs all others, by less than what moves the reference of the running soft-max: its weight there is any
    number up to 2^8, and however that is rounded, what V is multiplied with and what the sum is divided by are the same.
    Tiles of 16, 32, 64 and 128 entries."""
    n, dominant = 640, 500
    s = Requests([n], [rows], heads, 2, hd, "bf16", 64, seed=33, loud=False)
    k, v = s.k[0].zero_(), s.v[0].zero_()
    k[:, :, 1] = 1.0
    k[::32] = 0.0  # score 0: the reference
    k[dominant] = 0.0
    k[dominant, :, 0] = 1.0
    g = torch.Generator(device="cuda:0").manual_seed(34)
    levels = torch.tensor([0.5, 1, 1.5, 2, 3, 4, 6, -0.5, -1, -1.5, -2, -3, -4, -6], device="cuda:0", dtype=torch.bfloat16)
    v[dominant] = levels[torch.randint(0, 14, (2, hd), device="cuda:0", generator=g)]
    s.c.plan(dev([n]), dev([0]), dev([n]), n)
    s.write()
    s.step()
    z = 4.5 + torch.arange(rows * heads, device="cuda:0").reshape(rows, heads) % 34 / 32  # below 8 ln 2
    s.q.zero_()
    s.q[:, :, 0], s.q[:, :, 1] = z.to(torch.bfloat16), -60.0
    out = s.c.attend(0, s.q, scale=1.0, lse=lse)
    if lse:
        out, lse = out
    p = torch.exp(z.double())
    others = ((torch.arange(n - rows, n, device="cuda:0") // 32) + 1).double()[:, None]  # that score 0 and that the row sees
    share = p / (p + others)
    want = share[..., None] * v[dominant].double().repeat_interleave(heads // 2, 0)
    # the result's rounding to bf16 is half a unit of its last place.  The weight's own moves the share by 2^-8 (1 - share) of it, and
    # what fp32 does in exponential, sums and division by less than 2^-17
    half = torch.exp2(torch.floor(torch.log2(want.abs())) - 8)
    assert ((out.double() - want).abs() <= half + want.abs() * ((2.0 ** -8 * (1 - share) + 2.0 ** -17)[..., None])).all()
    if torch.is_tensor(lse):
        assert (lse.double() - torch.log(p + others)).abs().max() <= 2.0 ** -18
    s.c.close()


@pytest.mark.parametrize("hd,heads,kvh,lengths,rows", [
    (32, 4, 2, [1, 40, 333], [1, 3, 2]), (64, 2, 2, [90, 400], [20, 25]), (64, 4, 1, [70, 900], [33, 64]), (128, 4, 2, [65, 300], [9, 12]),
    (256, 2, 1, [500, 33], [3, 20]), (128, 160, 2, [300], [130]),
    (128, 4, 1, [9000, 700, 5001], [3, 1, 3]), (128, 2, 2, [9000, 700, 5001], [40, 1, 40]), (64, 64, 2, [5001, 400], [260, 3]), (128, 64, 2, [9001, 700], [64, 600]),
    (128, 64, 2, [40001, 700], [8, 640]),  # about 26 parts of wide tiles: joined in groups, then these
])
def test_the_log_sum_exp_is_that_of_unrounded_probabilities(hd, heads, kvh, lengths, rows):
    """With bf16 models too: only the products of 16-bit numbers and sums in fp32 stand between the scores and it.  Tiles of all
    sizes, whole and cut; joined at once and in groups."""
    s = Requests(lengths, rows, heads, kvh, hd, "bf16", 32, seed=35)
    s.step()
    out, lse = s.c.attend(0, s.q, lse=True)
    s.check(out)
    assert torch.equal(out, s.c.attend(0, s.q))
    at = 0
    for i, (n, r) in enumerate(zip(lengths, rows)):
        _, want, _, z_abs = ref.attend(s.q[at:at + r], ref.held(s.k[i]), ref.held(s.v[i]), list(range(n - r, n)), s.group, hd ** -0.5)
        # as in Requests.check: scores are off by (hd + 2) 2^-24 z_abs, exponentials and logarithm as much again, sums by n 2^-24
        assert (lse[at:at + r].cpu().double() - want).abs().max() <= (4 * (hd + 2) * z_abs + n + 64) * 2.0 ** -24
        at += r
    s.c.close()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("hd,rows,heads", [(64, 2, 2), (128, 20, 4), (256, 3, 2), (128, 130, 160)])
def test_a_query_with_an_infinity(dtype, hd, rows, heads):
    """inf times an element of K is an infinity or NaN, so the row's soft-max is NaN, also where all its scores are -inf; a row that
    sees nothing is the only one that is zero."""
    n = 300
    s = Requests([n], [rows], heads, 2, hd, dtype, 16, seed=32)
    s.k[0].fill_(1.0)
    s.c.plan(dev([n]), dev([0]), dev([n]), n)
    s.write()
    s.step()
    clean = s.c.attend(0, s.q)
    s.q[1, 0, 7] = float("-inf")
    s.q[0, 1, 7] = float("inf")
    out = s.c.attend(0, s.q)
    assert torch.isnan(out[1, 0]).all() and torch.isnan(out[0, 1]).all()
    out[1, 0], out[0, 1] = clean[1, 0], clean[0, 1]
    assert torch.equal(out, clean)
    s.c.close()


def test_scales_at_the_end_of_fp32():
    """The kernels work in units of ln 2: a scale that overflows there is refused (with it a score of 0 was NaN), one that does not
    is taken."""
    s = Requests([40], [2], 4, 2, 64, "bf16", 16, seed=36)
    s.step()
    s.q.zero_()
    for scale in (2.4e38, 3.4e38):
        with pytest.raises(ee.EeError, match="-7"):
            s.c.attend(0, s.q, scale=scale)
    out, lse = s.c.attend(0, s.q, scale=2.3e38, lse=True)
    s.check(out, lse, scale=2.3e38)
    s.c.close()


@pytest.mark.parametrize("heads,kvh,hd,lengths,rows", [
    (4, 4, 32, [1, 17, 600], [1, 3, 16]), (8, 1, 64, [2, 90, 9000], [1, 2, 1]), (32, 8, 128, [130, 5001], [4, 1]), (8, 1, 128, [300] * 20, [2] * 20),
    (2, 1, 256, [33, 700], [1, 8]), (4, 2, 256, [200, 3000], [200, 40]),
])
@pytest.mark.parametrize("window", [0, 50])
def test_tiles_of_16_entries_leave_the_result_s_rounding_only(heads, kvh, hd, lengths, rows, window):
    """bf16 models, at most 16 entries of a request for a kv head, or 256 elements: the probabilities' second terms leave 2^-16."""
    assert hd == 256 or max(rows) * heads // kvh <= 16
    s = Requests(lengths, rows, heads, kvh, hd, "bf16", 32, seed=37)
    s.step()
    out = s.c.attend(0, s.q, window=window).cpu().double()
    at = 0
    for i, (n, r) in enumerate(zip(lengths, rows)):
        want, _, weight, z_abs = ref.attend(s.q[at:at + r], ref.held(s.k[i]), ref.held(s.v[i]), list(range(n - r, n)), s.group, hd ** -0.5, window)
        got = out[at:at + r]
        half = torch.exp2(torch.floor(torch.log2(torch.maximum(want.abs(), got.abs()))) - 8)  # half a unit of the result's last place
        assert ((got - want).abs() <= half + weight * ((4 * (hd + 2) * z_abs + n + 64) * 2.0 ** -24 + 2.0 ** -16)).all(), (i, n, r)
        at += r
    s.c.close()


@pytest.mark.parametrize("heads,kvh,lengths,rows", [(32, 4, [300, 33, 900, 70, 150], [300, 33, 310, 0, 1]), (40, 40, [700, 400], [700, 400]), (96, 1, [260, 700], [100, 180])])
@pytest.mark.parametrize("window", [0, 1, 150])
def test_wide_tiles_of_several_requests(heads, kvh, lengths, rows, window):
    """Tiles of 128 entries: prompts from their start, chunks, single tokens, a request that waits, with heads that share and that do
    not."""
    flat = sum(rows) * heads // kvh
    assert flat * kvh >= 128 * 160 and len(rows) * 64 * 8 <= flat  # the rule: enough of them, and an eighth empty at most
    s = Requests(lengths, rows, heads, kvh, 128, "bf16", 64, seed=38)
    s.step()
    out, lse = s.c.attend(0, s.q, window=window, lse=True)
    s.check(out, lse, window=window)
    assert torch.equal(out, s.c.attend(0, s.q, window=window))
    s.c.close()


def test_refused_calls_leave_the_cache_as_it_was():
    s = Requests([40, 90], [2, 3], 4, 2, 64, "bf16", 16, seed=39)
    s.step()
    want = s.c.attend(0, s.q)
    arrays = [getattr(s.c, a).clone() for a in ("slots", "positions", "row_seq", "row_start", "served", "held_next", "n_free", "table", "free", "pool")]
    i2, kv = dev([40, 90]), s.k[1][:5]
    for call in (lambda: s.c.plan(i2, i2, i2, 10 ** 7), lambda: s.c.plan(i2, i2, i2, 5, -1), lambda: s.c.append(3, kv, kv),
                 lambda: s.c.append(0, s.k[1][:6], s.k[1][:6]), lambda: s.c.attend(7, s.q), lambda: s.c.attend(0, s.q, window=-5),
                 lambda: s.c.attend(0, s.q, scale=float("inf")), lambda: s.c.attend(0, s.q, out=s.q)):
        with pytest.raises(ee.EeError):
            call()
    for call in (lambda: s.c.plan(i2, i2, i2[:1], 5), lambda: s.c.append(0, kv.float(), kv), lambda: s.c.attend(0, s.q[:4]), lambda: s.c.read(0, i2)):
        with pytest.raises(ValueError):
            call()
    for a, before in zip(("slots", "positions", "row_seq", "row_start", "served", "held_next", "n_free", "table", "free", "pool"), arrays):
        assert torch.equal(getattr(s.c, a), before), a
    out = s.c.attend(0, s.q)
    assert torch.equal(out, want)
    s.check(out)
    s.c.close()


def test_rows_beyond_the_threads_of_a_launch():
    """2^22 rows of 128 heads: 2^32 threads and more.  K and V are one row for all; few rows have a slot."""
    kvh, hd, n = 128, 32, 1 << 22
    c = cache_of(kvh, kvh, hd, "bf16", 16, 4)
    row = rand((2, 1, kvh, hd), "bf16", 40)
    with_slot = torch.tensor([0, 17, n // 2 + 5, n - 1], device="cuda:0")
    slots = torch.full((n,), -1, dtype=torch.int64, device="cuda:0")
    slots[with_slot] = dev([5, 0, 63, 20], torch.int64)
    c.append(0, row[0].expand(n, kvh, hd), row[1].expand(n, kvh, hd), slots)
    for got, want in zip(c.read(0, slots[with_slot]), row):
        assert torch.equal(got.cpu().double(), ref.held(want).expand(4, kvh, hd))
    k = torch.full((n, kvh, hd), 7.0, dtype=torch.bfloat16, device="cuda:0")
    stream = torch.cuda.current_stream().cuda_stream
    assert ee.lib().ee_kv4_read(c.h, 0, n, slots.data_ptr(), k.data_ptr(), None, stream) == 0
    assert torch.equal(k[with_slot].cpu().double(), ref.held(row[0]).expand(4, kvh, hd))
    k[with_slot] = 0
    assert not k.view(torch.int64).any()
    c.close()
