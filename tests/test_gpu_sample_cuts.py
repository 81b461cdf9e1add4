"""Choosing tokens on the GPU where one cut meets another (f8_reference.choose is the plain form in 64 bits)."""
import math

import numpy as np
import pytest
import torch

import paper_2312_04916_amd as ee
from test_gpu_sample import DT, MOST_U, check, t32

pytestmark = pytest.mark.gpu
U = (0.0, 0.01, 0.02, 0.05, 0.3, 0.5, 0.9, 0.999, MOST_U)


def groups(vocab, dtype, top, many, far, seed):
    """Rows of nine equal arrangements, one for each of U: the largest logit once, 50 a quarter above `top - far`, `many` at it, the rest below."""
    z = torch.full((vocab,), top - far - 1.0)
    z[:1] = top
    z[1:51] = top - far + 0.25
    z[51:51 + many] = top - far
    z = z[torch.randperm(vocab, generator=torch.Generator().manual_seed(seed))]
    return z.expand(len(U), vocab).contiguous().cuda().to(DT[dtype])


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("far", [0.5, 1.0, 1.5, 4.0])
@pytest.mark.parametrize("vocab,many", [(3001, 1500), (4000, 2400), (5003, 2400), (5003, 200), (50304, 2400), (50304, 30000)])
def test_min_p_ends_one_step_above_the_other_cut(vocab, many, far, dtype):
    """min_p = exp(-far) in fp32, for which the group at that distance is out of reach and the next number above it is not, next to a top-k or a
    top-p that cuts in that very group: 1500 or fewer candidates are cut by the row's own workgroup, more by several or by one."""
    m = t32(math.exp(-far))
    reach = -math.log(m)
    top = 6.0
    edge = np.float32(top - far)
    assert top - float(edge) > reach >= top - float(np.nextafter(edge, np.float32(9.0)))
    z, u = groups(vocab, dtype, top, many, far, vocab + many), torch.tensor(U, device="cuda:0")
    k = 51 + many // 2
    below = math.exp(-far - 1.0) * (vocab - 51 - many)
    above, group = 1 + 50 * math.exp(0.25 - far), many * math.exp(-far)
    p = (above + group / 2) / (above + group + below)
    for kk, pp in ((k, 1.0), (0, p), (k, (above + group / 4) / (above + group / 2))):
        token = check(z, u, 1.0, kk, pp, m)
        assert (z[torch.arange(len(U)), token.long()] > top - far).all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("live", [3, 500, 520, 600, 1500, 2040, 2500, 3000])
@pytest.mark.parametrize("vocab", [3100, 9000, 50304])
def test_top_k_that_leaves_all_before_top_p(vocab, live, dtype):
    """A mask leaves no more tokens than top_k, and top-p's share is of all of them: one wave, a workgroup, or the kernel for many candidates."""
    g = torch.Generator().manual_seed(vocab + live)
    rows = 12
    z = torch.full((rows, vocab), -torch.inf)
    for i in range(rows):
        at = torch.randperm(vocab, generator=g)[:live]
        z[i, at] = torch.randn(live, generator=g) * (0.2 + 0.3 * i)
    z = z.cuda().to(DT[dtype])
    u = torch.rand(rows, generator=g).cuda()
    p = (0.05 + 0.94 * torch.rand(rows, generator=g)).cuda()
    for k in (live, live + 1, min(vocab - 1, 2 * live), vocab - 1):
        check(z, u, 0.9, k, p, 0.0)
        check(z, u, 0.9, k, p, 0.02)


@pytest.mark.parametrize("vocab,n", [(4096, 2), (8192, 3000), (50304, 3000), (50304, 700)])
def test_top_p_is_a_share_of_all_that_is_small_too(vocab, n):
    """n tokens of weight 1 in front, and a tail of exp(-31.5) = 0.367 * 2^-44 each, which is nothing as a multiple of 2^-44 of the largest, but
    not in all: half of the sum is a little more than n / 2 tokens, of which one more is kept.  With top_k (which takes one token of the
    tail away) the sum is of what is kept and the tail is nothing."""
    z = torch.full((2, vocab), -31.5, device="cuda:0")
    z[:, :n] = 0.0
    u = torch.full((2,), MOST_U, device="cuda:0")
    total = n + (vocab - n) * math.exp(-31.5)
    kept = math.floor(0.5 * total) + 1
    assert kept == n // 2 + 1 and 0.5 * total - n // 2 > 2.0 ** -44 * 50
    for dtype in DT.values():
        assert ee.sample(z.to(dtype), u, top_p=0.5).tolist() == [kept - 1] * 2
        assert ee.sample(z.to(dtype), u, top_p=0.5, min_p=0.5).tolist() == [kept - 1] * 2
        assert ee.sample(z.to(dtype), u, top_p=0.5, top_k=vocab - 1).tolist() == [n // 2 - 1] * 2
        assert ee.sample(z.to(dtype), u, top_p=0.5, top_k=vocab).tolist() == [kept - 1] * 2  # (top_k cuts nothing)
