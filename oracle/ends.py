"""The two ends of a language model in float64: embedding and its gradient, log-probabilities of labels and the logits'
gradient, the preference and policy losses with theirs.  Written row by row from their formulas."""
import math

import numpy as np


def embedding(ids, table, scale):
    """scale table[id]; zeros for id < 0, NaN for an id the table does not have."""
    vocab, d = table.shape
    out = np.zeros((len(ids), d))
    for t, v in enumerate(ids):
        if v >= vocab:
            out[t] = np.nan
        elif v >= 0:
            out[t] = scale * table[v]
    return out


def embedding_backward(ids, grad, vocab, scale):
    """(G, sums of magnitudes, occurrences): G[v] = scale times the sum of the rows of grad whose token is v."""
    G = np.zeros((vocab, grad.shape[1]))
    mag, count = np.zeros_like(G), np.zeros(vocab, np.int64)
    for t, v in enumerate(ids):
        if 0 <= v < vocab:
            G[v] += scale * grad[t]
            mag[v] += abs(scale) * np.abs(grad[t])
            count[v] += 1
    return G, mag, count


def token_logprob(X, labels, scale):
    """(logp, lse) of one block of rows; labels below 0 give zeros, labels behind the vocabulary a NaN."""
    logp, lse = np.zeros(len(labels)), np.zeros(len(labels))
    for t, y in enumerate(labels):
        if y < 0:
            continue
        x = scale * X[t]
        with np.errstate(invalid="ignore", divide="ignore"):
            m = x.max()
            ls = np.log(np.exp(x - m).sum())
            lse[t] = m + ls
            logp[t] = (x[y] - m) - ls if y < len(x) else np.nan
    return logp, lse


def token_logprob_backward(X, labels, lse, g, scale):
    dX = np.zeros(X.shape)
    for t, y in enumerate(labels):
        if y < 0:
            continue
        if y >= X.shape[1]:
            dX[t] = np.nan
            continue
        dX[t] = -np.exp(scale * X[t] - lse[t])
        dX[t, y] += 1.0
        dX[t] *= scale * g[t]
    return dX


def _span(start, s, rows):
    """A sequence's rows: starts clamped into the rows, and up to the largest one before."""
    start = np.clip(np.asarray(start[:s + 2], np.int64), 0, rows)
    return int(start[:s + 1].max()), int(start.max())


def _log_sigma(h):
    return -np.log1p(np.exp(-h)) if h >= 0 else h - np.log1p(np.exp(h))


def preference_loss(logp, ref, labels, start, beta, kind="sigmoid", average=False, margin=0.0, smoothing=0.0, weight=1.0):
    """(loss, rewards, gradient) of one block; rows of the gradient in no sequence are NaN."""
    rows, pairs = len(logp), (len(start) - 1) // 2
    grad, rewards, loss = np.full(rows, np.nan), np.zeros(2 * pairs), 0.0
    for p in range(pairs):
        R, where, share = [], [], []
        for s in (2 * p, 2 * p + 1):
            lo, hi = _span(start, s, rows)
            grad[lo:hi] = 0.0
            at = [t for t in range(lo, hi) if labels is None or labels[t] >= 0]
            w = 1.0 / len(at) if average and at else 1.0
            total = sum(float(logp[t]) - (0.0 if ref is None else float(ref[t])) for t in at)
            R.append(w * total)
            where.append(at)
            share.append(w)
            rewards[s] = beta * w * total
        if not where[0] or not where[1]:
            continue
        z = R[0] - R[1] - margin
        h = beta * z
        if kind == "sigmoid":
            l = -(1 - smoothing) * _log_sigma(h) - smoothing * _log_sigma(-h)
            slope = beta * (smoothing * np.exp(_log_sigma(h)) - (1 - smoothing) * np.exp(_log_sigma(-h)))
        elif kind == "hinge":
            l, slope = max(0.0, 1.0 - h), -beta if h < 1.0 else 0.0
        else:
            l, slope = (z - 1 / (2 * beta)) ** 2, 2 * (z - 1 / (2 * beta))
        loss += l
        grad[where[0]] = weight / pairs * slope * share[0]
        grad[where[1]] = -weight / pairs * slope * share[1]
    return weight / pairs * loss, rewards, grad


def _kl(d):
    """(exp(d) - d - 1, exp(d) - 1), by exp's series where the differences would cancel."""
    if abs(d) < 0.5:
        k = sum(d ** n / math.factorial(n) for n in range(20, 1, -1))
        return k, k + d
    with np.errstate(over="ignore"):
        m = np.expm1(d)
    return (m - d if d < np.inf else m), m


def policy_loss(logp, old, adv, labels, start, ref=None, per_token=False, low=0.2, high=0.2, kl_coef=0.0, aggregate="token",
                weight=1.0):
    """(loss, [mean k, share of clipped rows], gradient) of one block; rows of the gradient in no sequence are NaN."""
    rows, nseq = len(logp), len(start) - 1
    grad, loss, kl, clipped = np.full(rows, np.nan), 0.0, 0.0, 0
    where = []
    for s in range(nseq):
        lo, hi = _span(start, s, rows)
        grad[lo:hi] = 0.0
        where.append([t for t in range(lo, hi) if labels is None or labels[t] >= 0])
    N = sum(len(at) for at in where)
    for s, at in enumerate(where):
        share = weight * (1.0 / N if aggregate == "token" and N else 1.0 / (nseq * len(at)) if aggregate == "sequence" and at
                          else 1.0)
        for t in at:
            A, p = float(adv[t] if per_token else adv[s]), float(logp[t])
            r = np.exp(p - float(old[t]))
            c = min(max(r, 1 - low), 1 + high)
            l, slope = -min(r * A, c * A), (0.0 if r * A > c * A else -r * A)
            clipped += r * A > c * A
            if ref is not None:
                d = float(ref[t]) - p
                k, m = _kl(d)
                if kl_coef != 0:
                    l += kl_coef * k
                    slope -= kl_coef * m
                kl += k
            loss += share * l
            grad[t] = share * slope
    return loss, np.array([kl, clipped]) / max(N, 1), grad
