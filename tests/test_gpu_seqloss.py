"""The preference and policy losses against float64: kinds, masks, empty sequences, ragged batches, blocks."""
import numpy as np
import pytest
import torch

import paper_2608_15665_amd as zo
from _ends import U32, bits, host, i32, within
from oracle import ends

pytestmark = pytest.mark.gpu

# Sums of n float64 values and a few elementary functions of them: n + 100 roundings of 2^-53 of the magnitudes that are added.
U64 = 2.0 ** -53


def f32(a):
    return torch.from_numpy(np.ascontiguousarray(a, np.float32)).cuda()


LENGTHS = {
    "one": [1, 1],
    "small": [5, 1, 0, 4, 7, 3, 0, 0],
    "odd": [63, 64, 65, 255, 256, 257],
    "many": [int(n) for n in np.random.default_rng(0).integers(0, 40, 600)],
    "long": [20000, 9, 1025, 4096],
    "thousand": [3] * 1024 + [5] * 200,
    "short": [int(n) for n in np.random.default_rng(3).integers(0, 90, 256)],
    "several": [480, 3, 0, 511, 700, 290],
    "full": [16] * 250,
    "pairs": [int(n) for n in np.random.default_rng(1).integers(100, 600, 40)],
}


def _batch(name, nblk, lead=2, behind=3, hidden=0.3):
    lengths = LENGTHS[name]
    rng = np.random.default_rng(len(lengths))
    start = lead + np.concatenate([[0], np.cumsum(lengths)])
    rows = int(start[-1]) + behind
    labels = np.where(rng.random(rows) < hidden, -100, 3)
    base = -np.abs(rng.standard_normal(rows))
    logp = (base + 0.05 * rng.standard_normal((nblk, rows))).astype(np.float32)
    ref, old = ((base + 0.15 * rng.standard_normal(rows)).astype(np.float32) for _ in range(2))
    return start, labels, logp, ref, old, rng


def _masked(a, labels):
    """The same with NaN and infinities where nothing counts."""
    a = a.copy()
    off = np.flatnonzero(labels < 0)
    a[..., off[0::3]] = np.nan
    a[..., off[1::3]] = np.inf
    a[..., off[2::3]] = -np.inf
    return a


def _rows(name, got, want, out, start, nblk):
    """A gradient: fp32-rounded where rows are in a sequence, untouched (9) elsewhere."""
    for b in range(nblk):
        inside = ~np.isnan(want[b])
        w = want[b][inside]
        within(out[b][inside], w, (U32 + 400 * U64) * np.abs(w) + 1e-45 + got, f"{name} {b}")
        assert (out[b][~inside] == 9.0).all()


@pytest.mark.parametrize("name", sorted(LENGTHS))
@pytest.mark.parametrize("kind,smoothing", [("sigmoid", 0.0), ("sigmoid", 0.1), ("hinge", 0.0), ("ipo", 0.0)])
@pytest.mark.parametrize("average,nblk,masked,with_ref", [(False, 1, True, True), (True, 3, True, True), (True, 1, False, False),
                                                          (False, 5, False, True)])
def test_preference(name, kind, smoothing, average, nblk, masked, with_ref):
    start, labels, logp, ref, _, _ = _batch(name, nblk)
    pairs, rows = len(LENGTHS[name]) // 2, logp.shape[1]
    if not masked:
        labels = None
    beta, margin, weight = 0.3, 0.05, 1.5
    refs = ref if with_ref else None
    want = [ends.preference_loss(logp[b], refs, labels, start, beta, kind, average, margin, smoothing, weight) for b in range(nblk)]
    x, r = (_masked(logp, labels), _masked(ref, labels)) if masked else (logp, ref)
    rewards = torch.full((nblk, 2 * pairs), 9.0, device="cuda")
    dlogp = torch.full((nblk, rows), 9.0, device="cuda")
    flag = torch.zeros(1, dtype=torch.int32, device="cuda")
    args = dict(ref_logp=f32(r) if with_ref else None, labels=i32(labels) if masked else None, kind=kind, average=average,
                margin=margin, label_smoothing=smoothing, weight=weight)
    loss = zo.preference_loss(f32(x), i32(start), beta, rewards=rewards, dlogp=dlogp, bad_flag=flag, **args)
    assert flag.item() == 0
    # R sums at most rows values of magnitude 5 or so; the slope of each loss in R is at most 4 (|z| + 1 / beta) weight.
    size = np.abs(logp).max() + np.abs(ref).max()
    r_tol = (rows + 100) * U64 * size * (1 if average else rows)
    for b in range(nblk):
        within(host(rewards)[b], want[b][1], U32 * np.abs(want[b][1]) + r_tol, "rewards")
    most = 4 * (np.abs(np.concatenate([w[1] for w in want])).max() / beta + 4)
    within(host(loss), [w[0] for w in want], most * weight * (r_tol + 100 * U64 * most), "loss")
    _rows("dlogp", 4 * weight * (r_tol + 100 * U64 * most), np.array([w[2] for w in want]), host(dlogp), start, nblk)
    # Without what is optional, and again: the same bits.
    alone = zo.preference_loss(f32(x), i32(start), beta, **args)
    np.testing.assert_array_equal(bits(alone), bits(loss))


@pytest.mark.parametrize("name", sorted(LENGTHS))
@pytest.mark.parametrize("aggregate", ["token", "sequence", "sum"])
@pytest.mark.parametrize("per_token,nblk,masked,with_ref", [(False, 1, True, True), (True, 3, True, True), (True, 1, False, False),
                                                            (False, 4, True, False)])
def test_policy(name, aggregate, per_token, nblk, masked, with_ref):
    start, labels, logp, ref, old, rng = _batch(name, nblk)
    nseq, rows = len(LENGTHS[name]), logp.shape[1]
    adv = rng.standard_normal(rows if per_token else nseq).astype(np.float32)
    if not masked:
        labels = None
    low, high, kl, weight = 0.1, 0.15, 0.05 if with_ref else 0.0, 2.0
    want = [ends.policy_loss(logp[b], old, adv, labels, start, ref if with_ref else None, per_token, low, high, kl, aggregate,
                             weight) for b in range(nblk)]
    x, r, o = (_masked(a, labels) if masked else a for a in (logp, ref, old))
    a = _masked(adv, labels) if masked and per_token else adv
    stats = torch.full((nblk, 2), 9.0, dtype=torch.float64, device="cuda")
    dlogp = torch.full((nblk, rows), 9.0, device="cuda")
    flag = torch.zeros(1, dtype=torch.int32, device="cuda")
    args = dict(labels=i32(labels) if masked else None, ref_logp=f32(r) if with_ref else None, per_token=per_token,
                clip_low=low, clip_high=high, kl_coef=kl, aggregate=aggregate, weight=weight)
    loss = zo.policy_loss(f32(x), f32(o), f32(a), i32(start), stats=stats, dlogp=dlogp, bad_flag=flag, **args)
    assert flag.item() == 0
    # Terms of magnitude max |A| e^1 + 1 or so, averaged or summed.
    term = 4 * (np.abs(adv).max() + 1)
    n = rows if aggregate == "sum" else 1
    within(host(loss), [w[0] for w in want], weight * n * term * (rows + 100) * U64, "loss")
    within(host(stats), [w[1] for w in want], 4 * (rows + 100) * U64, "stats")
    _rows("dlogp", 0.0 + weight * term * 100 * U64 * (1 if aggregate == "sum" else 1 / max(1, min(rows, nseq))),
          np.array([w[2] for w in want]), host(dlogp), start, nblk)
    alone = zo.policy_loss(f32(x), f32(o), f32(a), i32(start), **args)
    np.testing.assert_array_equal(bits(alone), bits(loss))


def test_gradients_are_the_slopes_of_the_losses():
    """Central differences of the float64 losses in fp32 inputs: h = 2^-9, exact in logp's format; h^2 / 6 of the third
    derivative, and 2^-53 of the loss over h."""
    start, labels, logp, ref, old, rng = _batch("small", 1, 0, 0)
    adv = rng.standard_normal(8).astype(np.float32)
    logp = np.round(logp * 2 ** 12) / 2 ** 12
    h = 2.0 ** -9
    calls = [lambda x, **kw: zo.preference_loss(f32(x), i32(start), 0.7, ref_logp=f32(ref), labels=i32(labels), **kw),
             lambda x, **kw: zo.preference_loss(f32(x), i32(start), 0.7, labels=i32(labels), kind="ipo", average=True, **kw),
             lambda x, **kw: zo.policy_loss(f32(x), f32(old), f32(adv), i32(start), labels=i32(labels), ref_logp=f32(ref),
                                            clip_low=0.9, clip_high=5.0, kl_coef=0.1, aggregate="sequence", **kw)]
    for call in calls:
        d = torch.zeros(1, logp.shape[1], device="cuda")
        call(logp, dlogp=d)
        for t in range(logp.shape[1]):
            up, down = logp.copy(), logp.copy()
            up[0, t] += h
            down[0, t] -= h
            slope = (call(up).item() - call(down).item()) / (2 * h)
            assert abs(slope - d[0, t].item()) <= 10 * h * h / 6 + U32 * abs(slope) + 1e-12, t


def test_masks_that_leave_nothing():
    start, rows = [0, 3, 3, 8], 9
    x, none = f32(np.full((2, rows), np.nan)), i32(np.full(rows, -1))
    d, rw = torch.full((2, rows), 9.0, device="cuda"), torch.full((2, 4), 9.0, device="cuda")
    loss = zo.preference_loss(x, i32([0, 3, 3, 8, 8]), 0.1, ref_logp=x[0].clone(), labels=none, average=True, rewards=rw, dlogp=d)
    assert (loss == 0).all() and (rw == 0).all() and (d[:, :8] == 0).all() and (d[:, 8] == 9).all()
    for agg in ("token", "sequence", "sum"):
        d.fill_(9.0)
        stats = torch.full((2, 2), 9.0, dtype=torch.float64, device="cuda")
        loss = zo.policy_loss(x, x[0].clone(), f32(np.full(3, np.nan)), i32(start), labels=none, ref_logp=x[0].clone(),
                              kl_coef=0.1, aggregate=agg, stats=stats, dlogp=d)
        assert (loss == 0).all() and (stats == 0).all() and (d[:, :8] == 0).all() and (d[:, 8] == 9).all()


@pytest.mark.parametrize("rows,lead", [(12, 0), (5000, 4700)])
def test_as_many_blocks_as_a_grid_holds(rows, lead):
    """65535 blocks for the small batch's launch, a few hundred for the others'; every block against the others' formula."""
    nblk = 65535 if rows == 12 else 400
    start = np.array([0, 3, 5, 9, 12]) + lead
    g = torch.Generator(device="cuda").manual_seed(1)
    x = -torch.rand(nblk, rows, generator=g, device="cuda")
    seqs = [x[:, a:b].double().sum(1) for a, b in zip(start, start[1:])]
    got = zo.preference_loss(x, i32(start), 0.5)
    want = -torch.nn.functional.logsigmoid(0.5 * torch.stack([seqs[0] - seqs[1], seqs[2] - seqs[3]], 1)).mean(1)
    assert ((got - want).abs() <= 1e-13 * want.abs()).all()
    old = -torch.rand(rows, generator=g, device="cuda")
    got = zo.policy_loss(x, old, f32(np.ones(4)), i32(start), clip_low=1.0, clip_high=1e3)
    r = torch.exp((x.double() - old.double()))[:, start[0]:start[4]]
    assert ((got + r.mean(1)).abs() <= 1e-13 * r.mean(1)).all()


def test_no_rows():
    e = torch.empty(2, 0, device="cuda")
    assert (zo.preference_loss(e, i32([0, 0, 0]), 0.1) == 0).all()
    assert (zo.policy_loss(e, e[0], f32([1.0]), i32([0, 0])) == 0).all()


def test_far_margins():
    """|h| in the thousands, where exp(-h) is 0 or infinite: the loss is h or 0 and the slope beta or 0."""
    x = f32([[-1000.0, -0.5, -0.5, -1000.0]])
    for start, loss, grads in (([0, 1, 2], 9995.0, [-10.0, 10.0]), ([2, 3, 4], 0.0, [0.0, 0.0])):
        d = torch.zeros(1, 4, device="cuda")
        got = zo.preference_loss(x, i32(start), 10.0, dlogp=d)
        assert got.item() == loss and d[0, start[0]:start[2]].tolist() == grads


def test_infinite_ratios():
    """A token that the model now excludes (logp = -infinity): ratio 0, and with a KL term an infinite loss."""
    x = f32([[-np.inf, -1.0]])
    d = torch.zeros(1, 2, device="cuda")
    loss = zo.policy_loss(x, f32([-1.0, -1.0]), f32([1.0]), i32([0, 2]), dlogp=d)
    assert loss.item() == -0.5 and d.tolist() == [[0.0, -0.5]]
    loss = zo.policy_loss(x, f32([-1.0, -1.0]), f32([1.0]), i32([0, 2]), ref_logp=f32([-1.0, -1.0]), kl_coef=0.1, dlogp=d)
    assert loss.item() == np.inf and d[0, 0].item() == -np.inf and d[0, 1].item() == -0.5


@pytest.mark.parametrize("start", [[0, 9, 4, 12, 20], [-3, 2, 4, 6, 8], [0, 5, 10, 15, 50], [2 ** 31 - 1, -2 ** 31, 0, 7, 9]])
def test_sequence_starts_that_break_the_rule(start):
    """They are flagged, and nothing outside the rows is touched."""
    rows = 20
    buf = torch.full((3, rows), 9.0, device="cuda")  # the middle one is the call's
    x = -torch.rand(3, rows, device="cuda")
    for call in (lambda f: zo.preference_loss(x[1], i32(start), 0.1, dlogp=buf[1], bad_flag=f),
                 lambda f: zo.policy_loss(x[1], x[0], f32(np.ones(4)), i32(start), dlogp=buf[1], bad_flag=f)):
        flag = torch.zeros(1, dtype=torch.int32, device="cuda")
        loss = call(flag)
        assert flag.item() == 1 and loss.shape == (1,)
        assert (buf[0] == 9).all() and (buf[2] == 9).all()
