"""Plain forms in 64 bits of the products with weights held in 8 bits and of choosing tokens (include/ee.h), written from their
definitions; nothing here uses the library."""
import math
from fractions import Fraction

import numpy as np
import torch

E_MIN, E_MAX = -110, 120
LEVELS = np.array([m * 2.0 ** -9 for m in range(8)] + [(8 + m) * 2.0 ** (e - 10) for e in range(1, 16) for m in range(8) if (e, m) != (15, 7)])


def held(x, rows):
    """What the elements of x [n][k] stand for, groups of rows x 128; a group with an infinity or a NaN is NaN."""
    x = x.detach().cpu().double().numpy()
    n, k = x.shape
    out = np.empty_like(x)
    for i in range(0, n, rows):
        for j in range(0, k, 128):
            g = x[i:i + rows, j:j + 128]
            if not np.isfinite(g).all():
                out[i:i + rows, j:j + 128] = np.nan
                continue
            top = np.abs(g).max(initial=0)
            e = E_MIN
            if top > 448 * 2.0 ** E_MIN:
                e = math.frexp(top)[1] - 9
                e += top > 448 * 2.0 ** e
            a = np.abs(g) * 2.0 ** -e
            hi = np.clip(np.searchsorted(LEVELS, a), 1, len(LEVELS) - 1)
            lo = hi - 1
            up = a - LEVELS[lo] > LEVELS[hi] - a
            tie = a - LEVELS[lo] == LEVELS[hi] - a
            code = np.where(up | (tie & (hi % 2 == 0)), hi, lo)
            out[i:i + rows, j:j + 128] = np.copysign(LEVELS[code], g) * 2.0 ** e
    return torch.from_numpy(out)


def product(x, w, add=None, up=None):
    """-> y and the sums of |x w| that its errors are measured by, from held x and w (and up), in 64 bits."""
    g, size = x @ w.T, x.abs() @ w.abs().T
    if up is None:
        return (g if add is None else g + add.double().cpu()), size, None
    u, size_u = x @ up.T, x.abs() @ up.abs().T
    y = g * torch.sigmoid(g) * u
    return (y if add is None else y + add.double().cpu()), (g, size), (u, size_u)


def choose(z, u, t=1.0, top_k=0, top_p=1.0, min_p=0.0):
    """One row -> token, log-probability, confidence, the weights' running error's scale for the two."""
    z = np.asarray(z, dtype=np.float64)
    ok = 0 <= u < 1 and 0 <= t < math.inf and top_k >= 0 and 0 <= top_p <= 1 and 0 <= min_p <= 1
    if not ok or np.isnan(z).any() or (z == np.inf).any() or not (z > -np.inf).any():
        return -1, -math.inf, 0.0
    z = z + 0.0
    order = np.argsort(-z, kind="stable")
    top = z[order[0]]
    raw = np.exp(z - top)
    total = raw.sum()
    if t == 0:
        token = int(order[0])
    else:
        # whole multiples of 2^-44 of the largest, as the definition has it: their sums are exact, so that equal sums are equal
        with np.errstate(under="ignore", over="ignore"):
            w = np.rint(np.exp((z - top) / t) * 2.0 ** 44).astype(np.int64)
        n = min(top_k, len(z)) if top_k else len(z)
        if top_p < 1:
            run = np.cumsum(w[order[:n]])
            n = max(1, int((run - w[order[:n]] < math.ceil(Fraction(top_p) * int(run[-1]))).sum()))
        if min_p > 0:
            n = int((top - z[order[:n]] <= -math.log(min_p) * t).sum())
        at = np.sort(order[:n])
        run = np.cumsum(w[at])
        token = int(at[np.searchsorted(run, math.floor(Fraction(u) * int(run[-1])), side="right")])
    return token, float(z[token] - top - math.log(total)), float(1 / total)


def score_tolerance(z):
    """What sums of fp32 exponentials of z - top may be off by, relative to their sum: each term by the roundings of z - top and of its
    product with log2(e), two half steps times the argument, and two units of the exponential; the sum of 1024 terms as a tree of
    fp32 additions, a half step for each of its ten levels (all terms are positive)."""
    z = np.asarray(z, dtype=np.float64)
    z = z[z > -np.inf]
    d = z.max() - z
    w = np.exp(-d)
    return float((w * (2 * d + 14)).sum() / w.sum()) * 2.0 ** -24
