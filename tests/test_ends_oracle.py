"""The float64 references of the embedding, the label log-probabilities and the sequence losses against torch's autograd and
against central differences."""
import numpy as np
import pytest
import torch

from oracle import ends


def test_embedding_and_its_gradient():
    rng = np.random.default_rng(1)
    table, ids = rng.standard_normal((11, 8)), np.array([3, 3, -1, 0, 10, 3, 9])
    E = torch.tensor(table, requires_grad=True)
    H = 1.5 * E[torch.tensor(ids).clamp(min=0)] * torch.tensor(ids >= 0)[:, None]
    g = rng.standard_normal(H.shape)
    H.backward(torch.tensor(g))
    np.testing.assert_allclose(ends.embedding(ids, table, 1.5), H.detach().numpy(), rtol=1e-15)
    G, _, count = ends.embedding_backward(ids, g, 11, 1.5)
    np.testing.assert_allclose(G, E.grad.numpy(), rtol=1e-13, atol=1e-15)
    assert count.tolist() == [1, 0, 0, 3, 0, 0, 0, 0, 0, 1, 1]
    assert np.isnan(ends.embedding([11], table, 1.0)).all()


def test_log_probabilities_and_their_gradient():
    rng = np.random.default_rng(2)
    x, labels = 3 * rng.standard_normal((6, 9)), np.array([0, 8, -1, 4, 4, -7])
    X = torch.tensor(x, requires_grad=True)
    lp = torch.log_softmax(0.7 * X, -1).gather(1, torch.tensor(labels).clamp(min=0)[:, None])[:, 0]
    lp = lp * torch.tensor(labels >= 0)
    g = rng.standard_normal(6)
    lp.backward(torch.tensor(g))
    logp, lse = ends.token_logprob(x, labels, 0.7)
    np.testing.assert_allclose(logp, lp.detach().numpy(), rtol=1e-13, atol=1e-14)
    np.testing.assert_allclose(ends.token_logprob_backward(x, labels, lse, g, 0.7), X.grad.numpy(), rtol=1e-12, atol=1e-14)


def _batch(seed, lengths, extra=3):
    rng = np.random.default_rng(seed)
    start = np.concatenate([[0], np.cumsum(lengths)])
    rows = int(start[-1]) + extra
    labels = np.where(rng.random(rows) < 0.3, -100, 1)
    logp, ref, old = (-np.abs(rng.standard_normal(rows)) for _ in range(3))
    return start, labels, logp, ref, old, rng


@pytest.mark.parametrize("kind,smoothing", [("sigmoid", 0.0), ("sigmoid", 0.2), ("hinge", 0.0), ("ipo", 0.0)])
@pytest.mark.parametrize("average", [False, True])
def test_preference_gradient_is_the_slope(kind, smoothing, average):
    start, labels, logp, ref, _, _ = _batch(3, [5, 1, 0, 4, 7, 3])
    f = lambda x: ends.preference_loss(x, ref, labels, start, 0.4, kind, average, 0.1, smoothing, 1.5)
    loss, rewards, grad = f(logp)
    for t in range(len(logp)):
        if np.isnan(grad[t]):
            continue
        up, down = logp.copy(), logp.copy()
        up[t] += 1e-5
        down[t] -= 1e-5
        assert abs((f(up)[0] - f(down)[0]) / 2e-5 - grad[t]) < 1e-8, t
    assert np.isnan(grad[-3:]).all() and not np.isnan(grad[:-3]).any()
    # The pair with the empty sequence: sequences 2 and 3.
    assert (grad[start[2]:start[4]] == 0).all()


def test_preference_loss_against_torch():
    start, labels, logp, ref, _, _ = _batch(4, [6, 5, 4, 9], 0)
    on = labels >= 0
    seq = np.repeat(np.arange(4), np.diff(start))
    R = np.array([((logp - ref) * on)[seq == s].sum() for s in range(4)])
    h = 0.3 * torch.tensor(R[0::2] - R[1::2])
    want = -0.9 * torch.nn.functional.logsigmoid(h) - 0.1 * torch.nn.functional.logsigmoid(-h)
    got = ends.preference_loss(logp, ref, labels, start, 0.3, smoothing=0.1)
    np.testing.assert_allclose(got[0], want.mean().item(), rtol=1e-13)
    np.testing.assert_allclose(got[1], 0.3 * R, rtol=1e-13)


@pytest.mark.parametrize("aggregate", ["token", "sequence", "sum"])
@pytest.mark.parametrize("per_token", [False, True])
@pytest.mark.parametrize("with_ref", [False, True])
def test_policy_loss_against_torch(aggregate, per_token, with_ref):
    start, labels, logp, ref, old, rng = _batch(5, [6, 0, 9, 1, 3], 2)
    nseq, n = 5, start[-1]
    adv = rng.standard_normal(len(logp) if per_token else nseq)
    got = ends.policy_loss(logp, old, adv, labels, start, ref if with_ref else None, per_token, 0.2, 0.3,
                           0.05 if with_ref else 0.0, aggregate, 2.0)
    x = torch.tensor(logp[:n], requires_grad=True)
    seq, on = np.repeat(np.arange(nseq), np.diff(start)), torch.tensor(labels[:n] >= 0)
    A = torch.tensor(adv[:n] if per_token else adv[seq])
    r = torch.exp(x - torch.tensor(old[:n]))
    l = -torch.minimum(r * A, r.clamp(0.8, 1.3) * A)
    if with_ref:
        d = torch.tensor(ref[:n]) - x
        l = l + 0.05 * (torch.exp(d) - d - 1)
    l = l * on
    if aggregate == "token":
        total = l.sum() / on.sum()
    elif aggregate == "sum":
        total = l.sum()
    else:
        total = sum((l[seq == s].sum() / max(1, int(on[seq == s].sum())) for s in range(nseq)), torch.tensor(0.0)) / nseq
    (2.0 * total).backward()
    np.testing.assert_allclose(got[0], 2.0 * total.item(), rtol=1e-12)
    np.testing.assert_allclose(got[2][:n], x.grad.numpy(), rtol=1e-12, atol=1e-16)
    assert np.isnan(got[2][n:]).all()
