"""Every launch of the sequence losses at float64's precision, and with infinities among the rows that count."""
import numpy as np
import pytest
import torch

import paper_2608_15665_amd as zo
from _ends import U32, host, i32, within
from oracle import ends

pytestmark = pytest.mark.gpu

U64 = 2.0 ** -53
INF = float("inf")
# One workgroup for all rows; a wave, 256 and 1024 threads a sequence or pair.
LENGTHS = {"few": [5, 1, 0, 700, 9, 40], "wave": [21] * 300, "group": [600] * 10, "long": [1800, 1900, 9, 2501]}


def f32(a):
    return torch.from_numpy(np.ascontiguousarray(a, np.float32)).cuda()


def _case(name, nblk):
    rng = np.random.default_rng(len(LENGTHS[name]))
    start = np.concatenate([[0], np.cumsum(LENGTHS[name])])
    rows = int(start[-1])
    labels = np.where(rng.random(rows) < 0.3, -100, 3)
    base = -2 * rng.random(rows)
    logp = (base + 0.02 * rng.standard_normal((nblk, rows))).astype(np.float32)
    ref, old = ((base + 0.02 * rng.standard_normal(rows)).astype(np.float32) for _ in range(2))
    return start, labels, logp, ref, old, rng


@pytest.mark.parametrize("name", sorted(LENGTHS))
@pytest.mark.parametrize("kind,smoothing", [("sigmoid", 0.0), ("sigmoid", 0.1), ("hinge", 0.0), ("ipo", 0.0)])
@pytest.mark.parametrize("average", [False, True])
@pytest.mark.parametrize("nblk", [1, 3])
def test_preferences_to_float64(name, kind, smoothing, average, nblk):
    """Each reward is off by its own sum's roundings, each pair's loss by its slope times that, and the mean by the pairs'."""
    start, labels, logp, ref, _, _ = _case(name, nblk)
    pairs, beta, margin, weight = len(LENGTHS[name]) // 2, 0.3, 0.05, 1.5
    loss = host(zo.preference_loss(f32(logp), i32(start), beta, ref_logp=f32(ref), labels=i32(labels), kind=kind, average=average,
                                   margin=margin, label_smoothing=smoothing, weight=weight))
    for b in range(nblk):
        want, rewards, _ = ends.preference_loss(logp[b], ref, labels, start, beta, kind, average, margin, smoothing, weight)
        off, size = 0.0, 0.0
        for p in range(pairs):
            err, R = [], []
            for s in (2 * p, 2 * p + 1):
                at = np.flatnonzero(labels[start[s]:start[s + 1]] >= 0) + start[s]
                mag = np.abs(logp[b, at].astype(np.float64) - ref[at]).sum() / (len(at) if average and len(at) else 1)
                err.append((len(at) + 8) * U64 * mag)
                R.append(rewards[s] / beta)
                if len(at) == 0:
                    break
            else:
                z = R[0] - R[1] - margin
                err = sum(err) + 4 * U64 * (abs(R[0]) + abs(R[1]) + abs(z))
                slope = 2 * (abs(z - 0.5 / beta) + err) if kind == "ipo" else beta  # the loss's own, at most
                l = (z - 0.5 / beta) ** 2 if kind == "ipo" else 1 + beta * abs(z)  # at most
                off += slope * err + 20 * U64 * (l + slope * (abs(z) + 0.5 / beta))
                size += l
        # Both sides: the oracle adds in another order.
        bound = weight / pairs * 2 * (off + (pairs + 4) * U64 * size)
        assert abs(loss[b] - want) <= bound, (loss[b], want, bound)
        assert bound < 1e-10 * (1 + abs(want))  # no bound that would let half the digits go


@pytest.mark.parametrize("name", sorted(LENGTHS))
@pytest.mark.parametrize("aggregate", ["token", "sequence", "sum"])
@pytest.mark.parametrize("nblk", [1, 3])
@pytest.mark.parametrize("which", ["excluded", "sampled by none", "reference", "both"])
def test_policy_with_infinities(name, aggregate, nblk, which):
    """Tokens that the model excludes now (ratio 0), that the sampling model excluded (an infinite ratio, clipped for a positive
    advantage and an infinite loss for a negative one), that the reference excludes (an infinite KL term), and a ratio that is none."""
    start, labels, logp, ref, old, rng = _case(name, nblk)
    rows = int(start[-1])
    adv = rng.standard_normal(rows).astype(np.float32)
    on = np.flatnonzero(labels >= 0)[::131]
    assert len(on) >= 3
    if which in ("excluded", "both"):
        logp[0, on] = -INF
    if which in ("sampled by none", "both"):
        old[on] = -INF
        adv[on] = np.abs(adv[on]) + 0.1
        if which == "sampled by none" and nblk == 3:
            adv[on[1]] = -1.0
    with_ref = which == "reference"
    if with_ref:
        ref[on] = -INF
    with np.errstate(all="ignore"):
        want = [ends.policy_loss(logp[b], old, adv, labels, start, ref if with_ref else None, True, 0.1, 0.15,
                                 0.05 if with_ref else 0.0, aggregate) for b in range(nblk)]
    dlogp = torch.full((nblk, rows), 9.0, device="cuda")
    stats = torch.zeros(nblk, 2, dtype=torch.float64, device="cuda")
    kw = dict(labels=i32(labels), ref_logp=f32(ref) if with_ref else None, per_token=True, clip_low=0.1, clip_high=0.15,
              kl_coef=0.05 if with_ref else 0.0, aggregate=aggregate)
    loss = zo.policy_loss(f32(logp), f32(old), f32(adv), i32(start), stats=stats, dlogp=dlogp, **kw)
    alone = zo.policy_loss(f32(logp), f32(old), f32(adv), i32(start), **kw)
    term = 4 * (np.abs(adv).max() + 1)
    n = rows if aggregate == "sum" else 1
    within(host(loss), [w[0] for w in want], n * term * (rows + 100) * U64, "loss")
    within(host(alone), host(loss), 0.0, "alone")
    within(host(stats), [w[1] for w in want], 4 * (rows + 100) * U64, "stats")
    d = np.array([w[2] for w in want])
    size = np.where(np.isfinite(d), np.abs(d), 0.0)
    within(host(dlogp), d, (U32 + 400 * U64) * size + 400 * U64 * term, "dlogp")


@pytest.mark.parametrize("name", ["few", "wave", "group", "long"])
@pytest.mark.parametrize("side", [0, 1])
def test_preferences_with_excluded_tokens(name, side):
    """A chosen sequence that the model excludes loses without bound; a rejected one costs nothing."""
    start, labels, logp, ref, _, _ = _case(name, 2)
    pairs = len(LENGTHS[name]) // 2
    s = 2 * (pairs - 1) + side  # in the last pair, and in the first block alone
    at = int(start[s] + np.flatnonzero(labels[start[s]:start[s + 1]] >= 0)[-1])
    plain = host(zo.preference_loss(f32(logp), i32(start), 0.1, ref_logp=f32(ref), labels=i32(labels)))
    logp[0, at] = -INF
    d = torch.full((2, int(start[-1])), 9.0, device="cuda")
    rewards = torch.zeros(2, 2 * pairs, device="cuda")
    loss = host(zo.preference_loss(f32(logp), i32(start), 0.1, ref_logp=f32(ref), labels=i32(labels), dlogp=d, rewards=rewards))
    assert rewards[0, s].item() == -INF and torch.isfinite(rewards[1]).all() and torch.isfinite(d).all()
    assert loss[1] == plain[1]
    if side == 0:
        assert loss[0] == INF
        assert d[0, at].item() == np.float32(-0.1 * (1.0 / pairs))
    else:
        assert 0 <= loss[0] < plain[0] and d[0, at].item() == 0.0
    assert (d[:, torch.from_numpy(labels < 0).cuda()] == 0).all()
