"""Which rows a product with an 8-bit weight takes as overlapping (host arithmetic, no GPU): every call here is refused, for its workspace's size where
nothing overlaps, so that none runs."""
import random

import pytest

import paper_2312_04916_amd as ee

F32, BF16 = ee.EE_F32, ee.EE_BF16
ARG, NOMEM = -7, -2
BASE = 1 << 24


def call(m, n, k, x, xr, y, yr, add=None, ar=0, xd=BF16, yd=BF16):
    """m > 16: a workspace is needed, and 0 bytes are none."""
    return ee.lib().ee_f8_matmul(m, n, k, 0, 1 << 20, xd, x, xr, yd, y, yr, add, ar, 1 << 28, 0, None)


def bytes_of(p, m, row, cols, dtype):
    es = 2 if dtype == BF16 else 4
    return {p + i * row * es + b for i in range(m) for b in range(cols * es)}


def test_columns_of_one_buffer():
    m, n, k = 300, 64, 96
    wide = n + k + 40
    es = 2
    assert call(m, n, k, BASE, wide, BASE + k * es, wide) == NOMEM                  # y behind x
    assert call(m, n, k, BASE + n * es, wide, BASE, wide) == NOMEM                  # y before x
    assert call(m, n, k, BASE, wide, BASE + (k - 1) * es, wide) == ARG              # one column in both
    assert call(m, n, k, BASE + (n - 1) * es, wide, BASE, wide) == ARG
    assert call(m, n, k, BASE, n + k - 1, BASE + k * es, n + k - 1) == ARG          # y's last column is the next row's first of x
    assert call(m, n, k, BASE, n + k, BASE + k * es, n + k) == NOMEM
    # y and added rows, x elsewhere
    far = 1 << 26
    for at, want in ((n, NOMEM), (n - 1, ARG), (0, NOMEM), (1, ARG), (wide, ARG), (wide - 1, ARG), (wide - n, NOMEM), (-n, NOMEM)):
        assert call(m, n, k, far, k, BASE, wide, BASE + at * es, wide) == want, at
    assert call(m, n, k, far, k, BASE, wide, BASE, wide + 1) == ARG                 # the same rows in other places
    assert call(m, n, k, far, k, BASE, wide, BASE + n * es, 2 * wide) == ARG        # strides differ: by their ranges
    assert call(m, n, k, far, k, BASE, wide, BASE + (m - 1) * wide * es, -wide) == ARG
    assert call(m, n, k, far, k, BASE, wide, BASE + ((m - 1) * wide + n) * es, -wide) == NOMEM
    assert call(m, n, k, far, k, BASE + (m - 1) * wide * es, -wide, BASE + n * es, wide) == NOMEM
    # bf16 rows next to fp32 ones: the same stride in bytes
    assert call(m, n, k, BASE, 400, BASE + 200, 200, yd=F32) == NOMEM
    assert call(m, n, k, BASE, 400, BASE + 188, 200, yd=F32) == ARG
    # one row for all, between y's rows and in them
    assert call(m, n, k, BASE + n * es, 0, BASE, wide) == NOMEM
    assert call(m, n, k, BASE + (n - 1) * es, 0, BASE, wide) == ARG
    assert call(m, n, k, BASE + ((m - 1) * wide + n) * es, 0, BASE, wide) == NOMEM
    # rows of x that reach into one another: by their ranges
    assert call(m, n, k, BASE, 1, BASE + k * es, wide) == ARG
    assert call(m, n, k, BASE, 1, BASE + (m - 1 + k) * es, wide) == NOMEM


def test_one_row_has_no_stride():
    call1 = lambda yr, ar, **kw: ee.lib().ee_f8_matmul(1, 300, 1 << 18, 0, 1 << 20, BF16, 1 << 30, 0, BF16, 1 << 31, yr, kw.get("add", 1 << 31), ar, 1 << 29, 0, None)  # noqa: E731
    for yr, ar in ((300, 300), (300, 0), (0, 300), (1, -7)):
        assert call1(yr, ar) == NOMEM, (yr, ar)
    assert call1(300, 300, add=(1 << 31) + 2) == ARG and call1(300, 300, add=(1 << 31) + 600) == NOMEM


@pytest.mark.parametrize("seed", range(6))
def test_against_sets_of_bytes(seed):
    """Equal strides: exactly the calls with a byte in both are refused."""
    rng = random.Random(seed)
    seen = [0, 0]
    for _ in range(1500):
        m, n, k = rng.randint(17, 21), rng.randint(1, 6), rng.randint(1, 6)
        xd, yd = rng.choice((BF16, F32)), rng.choice((BF16, F32))
        step = rng.randint(6, 20) * 4 if F32 in (xd, yd) else rng.randint(6, 20) * 2
        ex, ey = (2 if xd == BF16 else 4), (2 if yd == BF16 else 4)
        if n * ey > step or k * ex > step:
            continue
        sx, sy = rng.choice((1, -1)), rng.choice((1, -1))
        x, y = BASE, BASE + rng.randint(-25 * step, 25 * step) // ey * ey
        want = bool(bytes_of(x, m, sx * step // ex, k, xd) & bytes_of(y, m, sy * step // ey, n, yd))
        assert call(m, n, k, x, sx * step // ex, y, sy * step // ey, xd=xd, yd=yd) == (ARG if want else NOMEM), (m, n, k, x, y, step, sx, sy, xd, yd)
        seen[want] += 1
    assert min(seen) > 100
