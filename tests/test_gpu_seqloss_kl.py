"""The policy loss's KL term where it counts nothing, and where the two models nearly agree."""
from decimal import Decimal, localcontext

import numpy as np
import pytest
import torch

import paper_2608_15665_amd as zo
from _ends import U32, host, i32

pytestmark = pytest.mark.gpu

U64 = 2.0 ** -53
# One workgroup for all rows; a wave, 256 and 1024 threads a sequence.
LENGTHS = {"few": [5, 1, 0, 700, 9], "wave": [21] * 300, "group": [600] * 10, "long": [1800, 1900, 9, 2501]}


def f32(a):
    return torch.from_numpy(np.ascontiguousarray(a, np.float32)).cuda()


def _starts(name):
    return np.concatenate([[0], np.cumsum(LENGTHS[name])])


@pytest.mark.parametrize("name", sorted(LENGTHS))
@pytest.mark.parametrize("nblk", [1, 3])
@pytest.mark.parametrize("aggregate", ["token", "sequence", "sum"])
def test_a_reference_that_is_only_reported(name, nblk, aggregate):
    """kl_coef = 0: loss and gradient are those without a reference, whatever k is; its mean is reported."""
    start, rng = _starts(name), np.random.default_rng(5)
    rows, nseq = int(start[-1]), len(start) - 1
    logp = -rng.random((nblk, rows)).astype(np.float32)
    logp[:, 2::97] = -np.inf
    ref = -rng.random(rows).astype(np.float32)
    ref[5::89] = -np.inf
    old, adv = f32(-rng.random(rows)), f32(rng.standard_normal(nseq))
    d, plain = torch.full((2, nblk, rows), 9.0, device="cuda")
    stats = torch.zeros(nblk, 2, dtype=torch.float64, device="cuda")
    want = zo.policy_loss(f32(logp), old, adv, i32(start), aggregate=aggregate, dlogp=plain)
    got = zo.policy_loss(f32(logp), old, adv, i32(start), ref_logp=f32(ref), kl_coef=0.0, aggregate=aggregate, dlogp=d, stats=stats)
    assert torch.isfinite(want).all() and torch.isfinite(plain).all()
    assert (got == want).all() and (d == plain).all()
    # Where both models exclude a token, d = -inf + inf is none.
    lost = (np.isinf(logp) & np.isinf(ref)).any(1)
    np.testing.assert_array_equal(host(stats)[:, 0], np.where(lost, np.nan, np.inf))
    assert torch.isfinite(stats[:, 1]).all()


def _k(d):
    """(exp(d) - d - 1, exp(d) - 1) of float64 values, rounded from 60 digits."""
    with localcontext() as c:
        c.prec = 60
        e = [(Decimal(float(x)).exp(), Decimal(float(x))) for x in d]
        return np.array([float(y - x - 1) for y, x in e]), np.array([float(y - 1) for y, _ in e])


@pytest.mark.parametrize("name", sorted(LENGTHS))
@pytest.mark.parametrize("nblk", [1, 2])
@pytest.mark.parametrize("size", [1e-9, 1e-6, 1e-3, 0.1, "any"])
def test_models_that_nearly_agree(name, nblk, size):
    """The mean of k, the loss (with advantages of 0) and its gradient keep their digits however small d = ref - logp is; "any"
    takes sizes from 1e-9 to 20, of both signs."""
    start, rng = _starts(name), np.random.default_rng(6)
    rows, nseq = int(start[-1]), len(start) - 1
    if size == "any":
        d = np.exp(rng.uniform(np.log(1e-9), np.log(20.0), rows)) * rng.choice([-1, 1], rows)
    else:
        d = size * rng.standard_normal(rows)
    logp = -1e-3 * (1 + rng.random((nblk, rows)))
    logp = logp.astype(np.float32)
    ref = (logp[0] + d).astype(np.float32)
    out = torch.zeros(nblk, rows, device="cuda")
    stats = torch.zeros(nblk, 2, dtype=torch.float64, device="cuda")
    kl, weight = 0.25, 2.0
    loss = zo.policy_loss(f32(logp), f32(logp[0]), f32(np.zeros(nseq)), i32(start), ref_logp=f32(ref), kl_coef=kl, weight=weight,
                          stats=stats, dlogp=out)
    # A difference of two of these fp32 numbers is exact in float64.  exp(d) is one unit (two roundings) off; where k is taken by
    # subtractions it is at least 0.1 e, so that a few dozen roundings of k cover them; then sums of n positive terms.
    tol = (rows + 100) * U64
    for b in range(nblk):
        k, m = _k(ref.astype(np.float64) - logp[b].astype(np.float64))
        mean = k.mean()
        assert abs(stats[b, 0].item() - mean) <= tol * mean, (b, stats[b, 0].item(), mean)
        assert abs(loss[b].item() - weight * kl * mean) <= (tol + 4 * U64) * weight * kl * mean
        want = -weight * kl * m / rows
        off = np.abs(host(out)[b] - want) - (U32 + 100 * U64) * np.abs(want) - 2.0 ** -149
        assert off.max() <= 0, (b, int(off.argmax()))
    assert (stats[:, 1] == 0).all()
