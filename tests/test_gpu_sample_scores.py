"""How near the scores of ee_sample come to 64 bits where the exponentials' arguments decide."""
import pytest
import torch

import paper_2312_04916_amd as ee

pytestmark = pytest.mark.gpu
HALF = 2.0 ** -24  # half a step of fp32, relative


def scores(z):
    token, logprob, conf = ee.sample(z, torch.zeros(z.shape[0], device="cuda:0"), scores=True)
    zd = z.double()
    total = torch.exp(zd - zd.amax(1, keepdim=True)).sum(1)
    return (conf.double() * total - 1) / HALF, (logprob.double() - (zd.gather(1, token.long()[:, None])[:, 0] - zd.amax(1) - total.log())) / HALF


@pytest.mark.parametrize("runs", [1, 16, 49])
def test_a_large_argument_costs_no_bits(runs):
    """Runs of one token at 0 and 1023 at -d, 4 <= d < 6, in which the latter are most of the sum and z - z_max is exact.  In half steps an
    element may be off by 2 (the exponential's unit) and 1 (the product behind it), times the 1023's share s <= 0.95; by additions only
    where the token at 0 takes part (equal terms add up exactly), ten of partial sums that are (1 + 2^l p) / (1 + 1023 p) of all of it, l < 10,
    5 together at most; by 2^-140 of 64-bit sums; by 1 of the result's own rounding: 9 at worst.  Independent and uniform, the squares add up:
    (2 s)^2 / 3 + s^2 / 3 + 1.5 / 3 + 1 / 3 <= 2.4, a mean of 1.55.  A product with log2(e) that is rounded adds up to 4 on its own, 1.5 in the mean,
    and log2(e)'s own rounding 0.5 d s / 2, one way."""
    g = torch.Generator(device="cuda:0").manual_seed(runs)
    d = 4 + 2 * torch.rand(4096 if runs == 1 else 512, 1, device="cuda:0", generator=g)
    z = -d.expand(-1, 1024 * runs).contiguous()
    z[:, ::1024] = 0
    conf, logprob = scores(z)
    assert float(conf.abs().max()) <= 9
    assert float(conf.square().mean().sqrt()) <= 1.55
    # (the chosen token is the first, at 0: minus the sum's logarithm, whose own half step is |logprob| at most)
    assert (logprob.abs() <= 9 + (d[:, 0] + 12)).all()


def test_scores_of_far_and_masked_tokens():
    """What lies further than fp32's exponentials reach, or is masked, adds nothing and spoils nothing."""
    z = torch.full((6, 3000), -torch.inf, device="cuda:0")
    z[:, 1500] = 2.0
    z[1, 100] = -85.5   # 2^-126.2 of the largest
    z[2, 100:900] = -1e30
    z[3, 100:900] = torch.finfo(torch.float32).min
    z[4] = torch.finfo(torch.float32).min
    z[5, 1700] = 2.0
    conf, logprob = scores(z)
    assert (conf.abs() <= 9).all() and (logprob.abs() <= 9 + 12).all()
