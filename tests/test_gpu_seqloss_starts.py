"""Sequence starts that break their rule (not decreasing, within the rows): flagged, and taken as clamped to it, in every
launch alike."""
import numpy as np
import pytest
import torch

import paper_2608_15665_amd as zo
from _ends import U32, bits, host, i32, within
from oracle import ends

pytestmark = pytest.mark.gpu

U64 = 2.0 ** -53
# One workgroup for all rows; a wave, 256 and 1024 threads a sequence or pair.
LENGTHS = {"few": [5, 1, 0, 700, 9, 40], "wave": [21] * 300, "group": [600] * 10, "long": [1800, 1900, 9, 2501]}


def _break(start, rows, how):
    s, n = start.copy(), len(start)
    if how == "later":  # a start behind the next ones: their rows lie in two sequences, were each taken for itself
        s[n // 2 - 1] = s[min(n // 2 + 1, n - 1)] + 3
    elif how == "first":  # the first behind others
        s[0] = s[3] + 2
    elif how == "outside":
        s[0], s[n // 2], s[-1] = -7, 2 ** 31 - 1, rows + 50
    elif how == "down":
        s = s[::-1].copy()
    elif how == "ends":  # within the rows, all but the last not decreasing
        s[-1] = s[1]
    assert (s != start).any()
    return s


def f32(a):
    return torch.from_numpy(np.ascontiguousarray(a, np.float32)).cuda()


def _case(name, how, nblk, lead=3, behind=4):
    rng = np.random.default_rng(len(LENGTHS[name]))
    start = lead + np.concatenate([[0], np.cumsum(LENGTHS[name])])
    rows = int(start[-1]) + behind
    labels = np.where(rng.random(rows) < 0.3, -100, 3)
    logp, ref, old = (-rng.random(s).astype(np.float32) for s in [(nblk, rows), rows, rows])
    return _break(start, rows, how), rows, labels, logp, ref, old, rng


def _check(name, dlogp, want, nblk, size):
    for b in range(nblk):
        inside = ~np.isnan(want[b])
        w = want[b][inside]
        within(host(dlogp)[b][inside], w, (U32 + 400 * U64) * np.abs(w) + 400 * U64 * size, f"{name} {b}")
        assert (host(dlogp)[b][~inside] == 9.0).all()


HOW = ["later", "first", "outside", "down", "ends"]


@pytest.mark.parametrize("name", sorted(LENGTHS))
@pytest.mark.parametrize("how", HOW)
@pytest.mark.parametrize("nblk", [1, 3])
@pytest.mark.parametrize("average", [False, True])
def test_preference(name, how, nblk, average):
    start, rows, labels, logp, ref, _, _ = _case(name, how, nblk)
    pairs = (len(start) - 1) // 2
    want = [ends.preference_loss(logp[b], ref, labels, start, 0.01, average=average) for b in range(nblk)]
    dlogp, rewards = torch.full((nblk, rows), 9.0, device="cuda"), torch.full((nblk, 2 * pairs), 9.0, device="cuda")
    flag = torch.zeros(1, dtype=torch.int32, device="cuda")
    args = (f32(logp), i32(start), 0.01)
    kw = dict(ref_logp=f32(ref), labels=i32(labels), average=average)
    loss = zo.preference_loss(*args, **kw, rewards=rewards, dlogp=dlogp, bad_flag=flag)
    assert flag.item() == 1
    # Sums of at most rows values of size 1, weighted by 0.01 in the loss, whose slope is at most that.
    tol = (rows + 100) * U64 * rows * 0.01
    for b in range(nblk):
        within(loss[b].item(), want[b][0], tol + 100 * U64, "loss")
        within(host(rewards)[b], want[b][1], U32 * np.abs(want[b][1]) + tol, "rewards")
    _check("dlogp", dlogp, np.array([w[2] for w in want]), nblk, 0.01 * (1 + (rows + 100) * rows * 0.01))
    again = zo.preference_loss(*args, **kw)  # no flag, and nothing optional
    np.testing.assert_array_equal(bits(again), bits(loss))


@pytest.mark.parametrize("name", sorted(LENGTHS))
@pytest.mark.parametrize("how", HOW)
@pytest.mark.parametrize("nblk", [1, 3])
@pytest.mark.parametrize("aggregate", ["token", "sequence", "sum"])
@pytest.mark.parametrize("per_token", [False, True])
def test_policy(name, how, nblk, aggregate, per_token):
    start, rows, labels, logp, ref, old, rng = _case(name, how, nblk)
    nseq = len(start) - 1
    adv = rng.standard_normal(rows if per_token else nseq).astype(np.float32)
    want = [ends.policy_loss(logp[b], old, adv, labels, start, ref, per_token, 0.1, 0.15, 0.05, aggregate) for b in range(nblk)]
    dlogp = torch.full((nblk, rows), 9.0, device="cuda")
    stats = torch.full((nblk, 2), 9.0, dtype=torch.float64, device="cuda")
    flag = torch.zeros(1, dtype=torch.int32, device="cuda")
    args = (f32(logp), f32(old), f32(adv), i32(start))
    kw = dict(labels=i32(labels), ref_logp=f32(ref), per_token=per_token, clip_low=0.1, clip_high=0.15, kl_coef=0.05,
              aggregate=aggregate)
    loss = zo.policy_loss(*args, **kw, stats=stats, dlogp=dlogp, bad_flag=flag)
    assert flag.item() == 1
    term = 4 * (np.abs(adv).max() + 1)  # |A| e and k, with the slopes
    n = rows if aggregate == "sum" else 1
    within(host(loss), [w[0] for w in want], n * term * (rows + 100) * U64, "loss")
    within(host(stats), [w[1] for w in want], 4 * (rows + 100) * U64, "stats")
    _check("dlogp", dlogp, np.array([w[2] for w in want]), nblk, term)
    again = zo.policy_loss(*args, **kw)
    np.testing.assert_array_equal(bits(again), bits(loss))


@pytest.mark.parametrize("how", HOW)
def test_what_is_not_finite_beside_good_starts(how):
    """A loss that is NaN by its inputs stays so, and is no sign of broken starts."""
    start, rows, labels, logp, ref, _, _ = _case("group", how, 2)
    good = 3 + np.concatenate([[0], np.cumsum(LENGTHS["group"])])
    logp[1, 700], labels[700] = np.nan, 1
    flag = torch.zeros(1, dtype=torch.int32, device="cuda")
    for s, bad in ((good, 0), (start, 1)):
        flag.zero_()
        loss = zo.preference_loss(f32(logp), i32(s), 0.01, ref_logp=f32(ref), labels=i32(labels), bad_flag=flag)
        want = [ends.preference_loss(logp[b], ref, labels, s, 0.01)[0] for b in range(2)]
        assert flag.item() == bad and np.isnan(want[1]) == bool(loss[1].isnan())
        within(loss[0].item(), want[0], (rows + 100) * U64 * rows * 0.01 + 100 * U64)
