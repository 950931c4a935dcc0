"""The policy loss's KL term where it counts nothing."""
import numpy as np
import pytest
import torch

import paper_2608_15665_amd as zo
from _ends import host, i32

pytestmark = pytest.mark.gpu

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
