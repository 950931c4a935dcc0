"""Log-probabilities of labels and the logits' gradient against float64: types, odd vocabularies, padded heads, masks,
infinities and NaN."""
import numpy as np
import pytest
import torch

import paper_2608_15665_amd as zo
from paper_2608_15665_amd import _lib
from _ends import DT, NEAR, TINY, U, U32, bits, host, i32, put, within
from oracle import ends

pytestmark = pytest.mark.gpu

INF = float("inf")


def _logp_tol(x, logp, lse, scale):
    """What fp32 may do to (logp, lse).  A term exp(t), t = scale (x - max), is off by four roundings of t (the difference,
    scale log2 e twice, the product) and two of the exponential; weighted by the terms, |t| averages at most log n.  Adding
    n terms over at least 64 lanes: n / 64 + 16 roundings.  Then logarithm and differences in fp64 and one rounding."""
    n = x.shape[-1]
    total = (4 * (np.log(n) + 1) + 2 + n / 64 + 16) * U32
    return (total + U32 * np.abs(logp)) * NEAR, (total + U32 * np.abs(lse)) * NEAR


def _grad_tol(x, labels, lse, g, scale, dt):
    """p = exp(a), a = scale x - lse: a is rounded, times log2 e (two roundings), the exponential twice; then 1 - p, the
    factors and the output's rounding."""
    a = scale * x - lse[:, None]
    p = np.exp(a)
    up = (np.abs(scale * g) * (labels >= 0))[:, None]
    want = ends.token_logprob_backward(x, labels, lse, g, scale)
    return want, (up * p * (3 * np.abs(a) + 3) * U32 + (4 * U32 + U[dt]) * np.abs(want)) * NEAR + TINY[dt] + up * 2.0 ** -125


def _case(seed, dt, rows, vocab, ld, off=0, nblk=1, ignored=0.25):
    """(logits as a view of a wider tensor of NaN, its values, labels)"""
    rng = np.random.default_rng(seed)
    n = nblk * rows
    _, v = put(3 * rng.standard_normal((n, vocab)), dt)
    flat = torch.full((off + n * ld + 16,), float("nan"), dtype=DT[dt], device="cuda")
    X = flat[off:off + n * ld].view(n, ld)
    X[:, :vocab] = torch.from_numpy(v).to(DT[dt]).cuda()
    labels = rng.integers(0, vocab, rows)
    labels[rng.random(rows) < ignored] = -100
    labels[0] = vocab - 1
    if rows > 1:
        labels[-1] = 0
    return X, v, labels, rng


SHAPES = [(1, 1, 1, 0), (1, 7, 7, 0), (3, 8, 8, 0), (5, 9, 16, 0), (2, 63, 64, 3), (9, 255, 255, 0), (4, 1000, 1000, 0),
          (3, 1023, 1031, 1), (2, 4097, 4100, 5), (7, 5003, 5003, 0), (2, 32000, 32000, 0), (3, 50257, 50304, 0),
          (2, 50257, 50257, 7), (1, 151851, 152064, 0), (64, 140000, 140000, 0), (65, 140000, 140000, 0), (300, 130, 131, 0), (4200, 515, 515, 0)]


@pytest.mark.parametrize("dt", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("rows,vocab,ld,off", SHAPES)
@pytest.mark.parametrize("scale", [1.0, 0.7])
def test_forward_and_backward(dt, rows, vocab, ld, off, scale):
    X, x, labels, rng = _case(rows + vocab, dt, rows, vocab, ld, off)
    s = float(np.float32(scale))
    logp, lse = zo.token_logprob(X, i32(labels), vocab=vocab, scale=scale)
    want, want_lse = ends.token_logprob(x, labels, s)
    tol, tol_lse = _logp_tol(x, want, want_lse, s)
    within(host(logp), want, tol, "logp")
    within(host(lse), want_lse, tol_lse, "lse")
    g = rng.standard_normal(rows).astype(np.float32)
    gd = torch.from_numpy(g).cuda()
    gd[torch.from_numpy(labels < 0).cuda()] = float("nan")  # not read
    wide = torch.full((off + rows * ld + 16,), 5.0, dtype=DT[dt], device="cuda")
    out = wide[off:off + rows * ld].view(rows, ld)
    zo.token_logprob_backward(X, i32(labels), lse, gd, vocab=vocab, scale=scale, out=out)
    dx, dtol = _grad_tol(x, labels, host(lse), g.astype(np.float64), s, dt)
    within(host(out)[:, :vocab], dx, dtol, "dX")
    assert (out[:, vocab:] == 5.0).all() and (wide[:off] == 5.0).all() and (wide[off + rows * ld:] == 5.0).all()
    # Into the logits themselves: the same bits.
    zo.token_logprob_backward(X, i32(labels), lse, gd, vocab=vocab, scale=scale, out=X)
    np.testing.assert_array_equal(bits(X[:, :vocab]), bits(out[:, :vocab]))
    assert X[:, vocab:].isnan().all()


@pytest.mark.parametrize("dt", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("vocab,ldx,ldo,off", [(515, 520, 515, 0), (515, 517, 520, 3), (64, 64, 72, 1)])
def test_rows_of_other_distances_and_places(dt, vocab, ldx, ldo, off):
    """The gradient's rows begin elsewhere in a 16-byte word than the logits'."""
    X, x, labels, rng = _case(3, dt, 6, vocab, ldx)
    logp, lse = zo.token_logprob(X, i32(labels), vocab=vocab)
    g = rng.standard_normal(6).astype(np.float32)
    wide = torch.full((off + 6 * ldo + 16,), 5.0, dtype=DT[dt], device="cuda")
    out = wide[off:off + 6 * ldo].view(6, ldo)
    lab, gd = i32(labels), torch.from_numpy(g).cuda()
    _lib._check(zo.lib().zo_token_logprob_backward(1, 6, vocab, _lib._DT[DT[dt]], X.data_ptr(), ldx, lab.data_ptr(), 1.0,
                                                   lse.data_ptr(), None, gd.data_ptr(), out.data_ptr(), ldo, None,
                                                   _lib._stream_handle()))
    dx, tol = _grad_tol(x, labels, host(lse), g.astype(np.float64), 1.0, dt)
    within(host(out)[:, :vocab], dx, tol, "dX")
    assert (out[:, vocab:] == 5.0).all() and (wide[:off] == 5.0).all() and (wide[off + 6 * ldo:] == 5.0).all()


@pytest.mark.parametrize("nblk,rows", [(2, 5), (16, 3), (3, 70)])
def test_blocks_share_labels(nblk, rows):
    X, x, labels, rng = _case(11, "bf16", rows, 777, 784, nblk=nblk)
    logp, lse = zo.token_logprob(X, i32(labels), vocab=777)
    every = np.tile(labels, nblk)
    want, want_lse = ends.token_logprob(x, every, 1.0)
    tol, tol_lse = _logp_tol(x, want, want_lse, 1.0)
    within(host(logp), want, tol)
    within(host(lse), want_lse, tol_lse)
    g = rng.standard_normal(nblk * rows).astype(np.float32)
    out = zo.token_logprob_backward(X, i32(labels), lse, torch.from_numpy(g).cuda(), vocab=777)
    dx, dtol = _grad_tol(x, every, host(lse), g.astype(np.float64), 1.0, "bf16")
    within(host(out)[:, :777], dx, dtol)
    assert (out[:, 777:] == 0).all()


@pytest.mark.parametrize("dt", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("vocab", [9, 1000, 40001, 140001])
def test_masked_tokens(dt, vocab):
    """-infinity and the type's lowest value in place of masked logits: all but one, the first half, the label's own; a row
    of the lowest value alone is uniform, one of -infinity alone is NaN."""
    lowest = float(torch.finfo(DT[dt]).min)
    X, x, _, rng = _case(4, dt, 8, vocab, vocab)
    h = vocab // 2
    for r, (lo, hi, v) in enumerate([(0, h, -INF), (0, h, lowest), (0, vocab - 1, -INF), (0, vocab - 1, lowest), (h, h + 1, -INF),
                                     (0, vocab, lowest), (0, vocab, -INF), (1, vocab, lowest)]):
        x[r, lo:hi] = v
    X.copy_(torch.from_numpy(x).to(DT[dt]))
    x = host(X)
    labels = np.array([vocab - 1, vocab - 1, vocab - 1, vocab - 1, h, 1, 2, 0])
    logp, lse = zo.token_logprob(X, i32(labels))
    want, want_lse = ends.token_logprob(x, labels, 1.0)
    assert want[4] == -INF and np.isnan(want[6]) and abs(want[5] + np.log(vocab)) < 1e-9
    tol, tol_lse = _logp_tol(x, np.where(np.isfinite(want), want, 0), np.where(np.isfinite(want_lse), want_lse, 0), 1.0)
    within(host(logp), want, tol, "logp")
    keep = [0, 1, 2, 3, 4, 5, 7]
    within(host(lse)[keep], want_lse[keep], tol_lse[keep], "lse")
    g = rng.standard_normal(8).astype(np.float32)
    out = zo.token_logprob_backward(X, i32(labels), lse, torch.from_numpy(g).cuda())
    rows = [0, 1, 2, 3, 4, 7]  # of finite sums that fp32 can hold beside their logits
    with np.errstate(over="ignore"):
        a = np.minimum(host(lse)[rows][:, None] - x[rows], 200.0)
    dx = ends.token_logprob_backward(x[rows], labels[rows], host(lse)[rows], g[rows].astype(np.float64), 1.0)
    up = np.abs(g[rows])[:, None]
    within(host(out)[rows], dx, (up * np.exp(-a) * (3 * a + 3) * U32 + (4 * U32 + U[dt]) * np.abs(dx)) * NEAR + TINY[dt]
           + up * 2.0 ** -125, "dX")


@pytest.mark.parametrize("dt", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("vocab,at", [(9, 3), (5000, 0), (5000, 4999), (40001, 20000), (140001, 140000)])
def test_what_is_not_finite_stays_in_its_row(dt, vocab, at):
    X, x, labels, _ = _case(6, dt, 5, vocab, vocab, ignored=0.0)
    labels[4] = -1
    X[1, at], X[2, at], X[4, at] = float("nan"), INF, float("nan")
    logp, lse = zo.token_logprob(X, i32(labels))
    assert logp[[1, 2]].isnan().all() and torch.isfinite(logp[[0, 3, 4]]).all() and logp[4] == 0 and lse[4] == 0
    assert lse[1].isnan()
    out = zo.token_logprob_backward(X, i32(labels), lse, torch.ones(5, device="cuda"))
    assert torch.isfinite(out[[0, 3, 4]]).all() and (out[4] == 0).all() and out[1].isnan().all()


@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("left", [0, 3, 8])
def test_columns_of_a_wider_tensor(dt, left):
    """Logits and their gradient as column ranges of wider tensors, which stay as they are beside them."""
    X, x, labels, rng = _case(13, dt, 5, 1003, 1003)
    wide = torch.full((5, 1003 + left + 9), float("nan"), dtype=DT[dt], device="cuda")
    wide[:, left:left + 1003] = X
    view = wide[:, left:left + 1003]
    logp, lse = zo.token_logprob(view, i32(labels))
    want, want_lse = ends.token_logprob(x, labels, 1.0)
    tol, tol_lse = _logp_tol(x, want, want_lse, 1.0)
    within(host(logp), want, tol)
    within(host(lse), want_lse, tol_lse)
    g = torch.from_numpy(rng.standard_normal(5).astype(np.float32)).cuda()
    out = torch.full_like(wide, 7.0)
    zo.token_logprob_backward(view, i32(labels), lse, g, out=out[:, left:left + 1003])
    dx, dtol = _grad_tol(x, labels, host(lse), host(g), 1.0, dt)
    within(host(out)[:, left:left + 1003], dx, dtol)
    assert (out[:, :left] == 7.0).all() and (out[:, left + 1003:] == 7.0).all()


@pytest.mark.parametrize("rows,vocab", [(70001, 17), (4300001, 8)])
def test_many_short_rows(rows, vocab):
    """More rows than a grid's second dimension holds, and more workgroups than a row of the grid."""
    g = torch.Generator(device="cuda").manual_seed(3)
    X = (2 * torch.randn(rows, vocab, generator=g, device="cuda")).bfloat16()
    labels = torch.randint(-3, vocab, (rows,), generator=g, device="cuda").int()
    up = torch.randn(rows, generator=g, device="cuda")
    logp, lse = zo.token_logprob(X, labels)
    dX = zo.token_logprob_backward(X, labels, lse, up)
    x, on = X.double(), labels >= 0
    z = torch.logsumexp(x, 1)
    want = (x.gather(1, labels.long().clamp(min=0)[:, None])[:, 0] - z) * on
    total = (4 * (np.log(vocab) + 1) + 2 + vocab / 64 + 16) * U32
    assert ((logp - want).abs() <= (total + U32 * want.abs()) * NEAR).all()
    assert ((lse - z * on).abs() <= (total + U32 * z.abs()) * NEAR).all()
    a = x - lse.double()[:, None]
    hit = torch.arange(vocab, device="cuda") == labels[:, None]
    grad = up.double()[:, None] * (hit.double() - a.exp()) * on[:, None]
    tol = ((up.abs()[:, None] * a.exp() * (3 * a.abs() + 3) * U32 + (4 * U32 + U["bf16"]) * grad.abs()) * NEAR + TINY["bf16"]
           + up.abs()[:, None] * 2.0 ** -125)
    assert ((dX - grad).abs() <= tol)[on].all() and (dX[~on] == 0).all()


def test_large_logits_keep_their_differences():
    """Logits around 10^5: lse is coarse there, logp is not."""
    x = np.array([[1e5, 1e5 + 1, 1e5 - 2, 0.0], [-1e5, -1e5 + 0.5, -3e5, -1e5]])
    X, v = put(x, "f32")
    labels = np.array([0, 3])
    logp, _ = zo.token_logprob(X, i32(labels))
    want, _ = ends.token_logprob(v, labels, 1.0)
    within(host(logp), want, (4 * 3 + 30) * U32 + 2 * U32 * np.abs(want))


@pytest.mark.parametrize("dt,mask", [(dt, m) for dt in ["f32", "bf16", "f16"] for m in [-1e4, -1e7, -1.3e9, -1e10, -1e30, "lowest", "largest"]
                                     if dt != "f16" or m in (-1e4, "lowest", "largest")])
@pytest.mark.parametrize("vocab", [9, 1000, 40001, 140001])
@pytest.mark.parametrize("scale", [1.0, 0.5, 1.0 / 128, 40.0])
def test_large_finite_masks(dt, vocab, mask, scale):
    """Masks of any finite size, in all places but one, in the second half, everywhere; the value at the other end, as one
    logit or as all."""
    end = float(torch.finfo(DT[dt]).max)
    value = {"lowest": -end, "largest": end}.get(mask, mask)
    rng = np.random.default_rng(vocab)
    a = 3 * rng.standard_normal((4, vocab))
    a[0, :vocab // 2] = value
    a[0, vocab // 2 + 1:] = value
    a[1, vocab // 2:] = value
    a[2] = value
    a[3, 5] = -value
    X, x = put(a, dt)
    labels = np.array([vocab // 2, 1, 3, 5])
    logp, lse = zo.token_logprob(X, i32(labels), scale=scale)
    d = scale * (x - x.max(-1, keepdims=True))
    ls = np.log(np.exp(d).sum(-1))
    want, want_lse = np.take_along_axis(d, labels[:, None], 1)[:, 0] - ls, scale * x.max(-1) + ls
    tol, tol_lse = _logp_tol(x, want, want_lse, scale)
    over = np.abs(want_lse) > torch.finfo(torch.float32).max
    lost = np.abs(want) > torch.finfo(torch.float32).max
    got, got_lse = host(logp), host(lse)
    assert (got_lse[over] == np.sign(want_lse[over]) * INF).all() and (got[lost] == -INF).all()
    within(got_lse[~over], want_lse[~over], tol_lse[~over], "lse")
    within(got[~lost], want[~lost], tol[~lost], "logp")


@pytest.mark.parametrize("dt", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("vocab", [9, 5003])
def test_gradients_of_large_logits(dt, vocab):
    """With logp the gradient does not hang on lse's rounding: rows around +-30000, a row of the type's lowest value alone
    (uniform), one whose label is masked (lse alone serves it), an ordinary one and one that does not count."""
    rng = np.random.default_rng(vocab)
    lowest = float(torch.finfo(DT[dt]).min)
    a = 3 * rng.standard_normal((6, vocab))
    a[0] = 30000 + 256 * np.round(2 * rng.standard_normal(vocab))  # whole steps of every type there
    a[1] = -30000 + 256 * np.round(2 * rng.standard_normal(vocab))
    a[2] = lowest
    a[3, 4] = -INF
    X, x = put(a, dt)
    labels, scale = np.array([1, 2, 3, 4, 5, -1]), 1.0 / 128
    lab = i32(labels)
    logp, lse = zo.token_logprob(X, lab, scale=scale)
    g = rng.standard_normal(6).astype(np.float32)
    out = host(zo.token_logprob_backward(X, lab, lse, torch.from_numpy(g).cuda(), scale=scale, logp=logp))
    lp = host(logp)
    assert lp[3] == -INF and abs(lp[2] + np.log(vocab)) < 1e-5
    for r in range(5):
        if r == 3:
            t, z = scale * x[r], host(lse)[r]
        else:
            t = scale * (x[r] - x[r, labels[r]])
            z = np.log(np.exp(t - t.max()).sum()) + t.max()  # -logp, exact
        p = np.exp(t - z)
        want = -scale * g[r] * p
        want[labels[r]] += scale * g[r]
        # As for other gradients, and logp's (or, masked, an input's) own rounding and error.
        off = (4 * (np.log(vocab) + 1) + 18 + vocab / 64 + 2 * abs(z) + 4 * np.abs(np.maximum(t - z, -200)) + 3) * U32
        within(out[r], want, (np.abs(scale * g[r]) * p * off + (4 * U32 + U[dt]) * np.abs(want)) * NEAR + TINY[dt] + 2.0 ** -125, f"row {r}")
    assert (out[5] == 0).all()


def test_labels_that_the_vocabulary_lacks():
    X, x, _, _ = _case(7, "bf16", 4, 100, 104)
    flag = torch.zeros(1, dtype=torch.int32, device="cuda")
    zo.token_logprob(X, i32([0, 99, -1, 5]), vocab=100, bad_flag=flag)
    assert flag.item() == 0
    labels = i32([0, 100, 2 ** 31 - 1, 99])
    logp, lse = zo.token_logprob(X, labels, vocab=100, bad_flag=flag)
    assert flag.item() == 1 and logp[1].isnan() and logp[2].isnan() and torch.isfinite(logp[[0, 3]]).all()
    flag.zero_()
    out = zo.token_logprob_backward(X, labels, lse, torch.ones(4, device="cuda"), vocab=100, bad_flag=flag)
    assert flag.item() == 1 and out[1, :100].isnan().all() and torch.isfinite(out[[0, 3], :100]).all()


def test_gradient_is_the_slope_of_the_forward():
    """Central differences in the logits; logp of about 3 is off by 2^-21 or so, over 2 h = 2^-4."""
    X, x, labels, rng = _case(9, "f32", 4, 12, 12, ignored=0.0)
    _, lse = zo.token_logprob(X, i32(labels), scale=1.3)
    g = rng.standard_normal(4).astype(np.float32)
    dX = host(zo.token_logprob_backward(X, i32(labels), lse, torch.from_numpy(g).cuda(), scale=1.3))
    h = 2.0 ** -5
    for j in range(12):
        up, down = X.clone(), X.clone()
        up[:, j] += h
        down[:, j] -= h
        slope = (host(zo.token_logprob(up, i32(labels), scale=1.3)[0]) - host(zo.token_logprob(down, i32(labels), scale=1.3)[0]))
        # The third derivative of a log-sum-exp is at most 1.3^3 / 4 or so: h^2 / 6 of it.
        within(dX[:, j], g * slope / (2 * h), np.abs(g) * (1.3 ** 3 * h * h / 6 + 2 * 2.0 ** -19 / (2 * h)), f"column {j}")


@pytest.mark.parametrize("rows,vocab", [(3, 200), (4, 140001), (5000, 300)])
def test_without_the_log_sums(rows, vocab):
    X, _, labels, _ = _case(5, "bf16", rows, vocab, vocab)
    want, _ = zo.token_logprob(X, i32(labels))
    logp, lab = torch.full((rows,), 9.0, device="cuda"), i32(labels)
    ws = torch.empty(1 << 16, dtype=torch.uint8, device="cuda")
    _lib._check(zo.lib().zo_token_logprob(1, rows, vocab, zo.ZO_BF16, X.data_ptr(), vocab, lab.data_ptr(), 1.0, logp.data_ptr(),
                                          None, None, ws.data_ptr(), ws.numel(), _lib._stream_handle()))
    np.testing.assert_array_equal(bits(logp), bits(want))


def test_no_rows():
    none = torch.empty(0, dtype=torch.int32, device="cuda")
    logp, lse = zo.token_logprob(torch.empty(0, 50, device="cuda"), none)
    assert logp.numel() == 0
    assert zo.token_logprob_backward(torch.empty(0, 50, device="cuda"), none, lse, logp).shape == (0, 50)


def test_logits_past_4_gib():
    """Rows whose offset passes 2^32 elements; the others do not count and are not read."""
    rows, vocab = 29000, 152064
    if torch.cuda.mem_get_info()[0] < 24 << 30:
        pytest.skip("needs 24 GB")
    X = torch.empty(rows, vocab, dtype=torch.bfloat16, device="cuda")
    labels = np.full(rows, -1)
    rng = np.random.default_rng(1)
    for r in (0, 14000, rows - 1):
        X[r] = torch.from_numpy(rng.standard_normal(vocab)).bfloat16()
        labels[r] = int(rng.integers(vocab))
    logp, lse = zo.token_logprob(X, i32(labels))
    at = [0, 14000, rows - 1]
    x = host(X[at])
    want, want_lse = ends.token_logprob(x, labels[at], 1.0)
    within(host(logp)[at], want, _logp_tol(x, want, want_lse, 1.0)[0])
    assert (logp != 0).sum().item() == 3
    g = torch.ones(rows, device="cuda")
    zo.token_logprob_backward(X, i32(labels), lse, g, out=X)
    dx, tol = _grad_tol(x, labels[at], host(lse)[at], np.ones(3), 1.0, "bf16")
    within(host(X[at]), dx, tol)
    assert (X[1:100] == 0).all() and (X[rows - 100:rows - 1] == 0).all()
