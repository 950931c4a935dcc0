"""A model's two ends as they are used: a zeroth-order step from tokens to the update, the gradients of the two tables that no
subspace covers, answers scored for a policy step; captured and replayed, on other streams, two calls at once."""
import numpy as np
import pytest
import torch

import oracle
import paper_2608_15665_amd as zo
import zo_draws as zd
from _common import dev_f32, orth
from _ends import NEAR, U, U32, bits, host, i32, within
from oracle import ends

pytestmark = pytest.mark.gpu


class Model:
    """A layer between an embedding and a head: nblk query blocks of four sequences (two preference pairs)."""

    def __init__(self, dt=torch.bfloat16, seq_len=32, d=256, heads=2, ffn=512, vocab=1003, q=2, r=4, seed=3):
        rng = np.random.default_rng(seed)
        dev = lambda a: torch.from_numpy(np.ascontiguousarray(a)).to(dt).cuda()
        self.dt, self.seq_len, self.d, self.vocab, self.q, self.r, self.eps = dt, seq_len, d, vocab, q, r, 1e-3
        self.T, self.nblk, self.rng = 4 * seq_len, 2 * q, rng
        self.head_rows = (vocab + 7) // 8 * 8  # the head's rows are padded to a multiple of 8
        self.table = dev(0.5 * rng.standard_normal((vocab, d)))
        W = 0.05 * rng.standard_normal((self.head_rows, d))
        W[vocab:] = 50.0  # what the padding gives is not to be seen
        self.head = dev(W)
        shapes = dict(q=(d, d), k=(d, d), v=(d, d), o=(d, d), gate=(ffn, d), up=(ffn, d), down=(d, ffn))
        self.mats = {}
        for i, (nm, (m, n)) in enumerate(shapes.items()):
            self.mats[nm] = dict(W=dev(rng.standard_normal((m, n)) / np.sqrt(n)), U=dev_f32(orth(seed, (i, 1), m, r)),
                                 V=dev_f32(orth(seed, (i, 2), n, r)), Z=dev_f32(zd.z_draws(seed, 0, i, q, r)))
        self.head_uvz = [dev_f32(orth(seed, (9, 1), self.head_rows, r)), dev_f32(orth(seed, (9, 2), d, r)),
                         dev_f32(zd.z_draws(seed, 0, 9, q, r))]
        self.gamma = torch.ones(d, device="cuda")
        bq, bs = [b // 2 for b in range(self.nblk)], [1, -1] * q
        self.layer = zo.LlamaLayer(self.mats, dict(rms1_gamma=self.gamma, rms2_gamma=self.gamma), bq, bs, self.eps, self.T, seq_len,
                                   heads, workspace=torch.empty(64 << 20, dtype=torch.uint8, device="cuda"))
        ids = rng.integers(0, vocab, self.T)
        labels = np.roll(ids, -1)
        hidden = np.arange(self.T) % seq_len
        labels[(hidden < 9) | (hidden == seq_len - 1)] = -100
        self.ids, self.labels = i32(ids), i32(labels)
        self.ids_h, self.labels_h = ids, labels
        self.start = i32(np.arange(5) * seq_len)
        self.ref = torch.from_numpy(np.where(labels < 0, 0.0, -5.0 - rng.random(self.T)).astype(np.float32)).cuda()
        self.hidden = torch.empty(self.nblk * self.T, d, dtype=dt, device="cuda")
        self.X = torch.empty_like(self.hidden)
        self.plin = zo.PerturbedLinear(self.X, self.head, *self.head_uvz, bq, bs, self.eps, self.T, x_block_stride=self.T * d,
                                       out_dtype=torch.float32, workspace=torch.empty(64 << 20, dtype=torch.uint8, device="cuda"))

    def losses(self):
        """One float64 preference loss per query block, and what led to it."""
        H = zo.embedding(self.ids, self.table, scale=1.5)
        self.layer(H, out=self.hidden)
        zo.rmsnorm(self.hidden, self.gamma, 1e-6, out=self.X)
        logits = self.plin()
        logp, lse = zo.token_logprob(logits, self.labels, vocab=self.vocab)
        loss = zo.preference_loss(logp.view(self.nblk, -1), self.start, 0.1, ref_logp=self.ref, labels=self.labels)
        return H, logits, logp, lse, loss

    def step(self):
        H, logits, logp, lse, loss = self.losses()
        return [H, logits, logp, lse, loss, zo.combine_central(loss, self.eps)]


def test_a_zeroth_order_step_from_tokens():
    """Tokens to the update of every matrix.  Each end is checked on what the one before gave it; the estimates are those of
    the losses."""
    m = Model()
    H, logits, logp, lse, loss, g = m.step()
    want = ends.embedding(m.ids_h, host(m.table), 1.5)
    within(host(H), want, (U["bf16"] + U32) * np.abs(want) * NEAR, "embedding")
    # The perturbed head on the layers' own output, against the oracle.
    x, W, (u, v, z) = host(m.X), host(m.head), [host(t) for t in m.head_uvz]
    for b in range(m.nblk):
        rows = slice(b * m.T, (b + 1) * m.T)
        ref = oracle.perturbed_linear(x[rows], W, u, v, z[b // 2], 1 if b % 2 == 0 else -1, m.eps)
        assert np.abs(host(logits)[rows] - ref).max() < 1e-4 * np.abs(ref).max()
    n = m.vocab
    every = np.tile(m.labels_h, m.nblk)
    lp, z = ends.token_logprob(host(logits)[:, :n], every, 1.0)
    tol = (4 * (np.log(n) + 1) + 2 + n / 64 + 16) * U32  # as for the log-probabilities alone
    within(host(logp), lp, (tol + U32 * np.abs(lp)) * NEAR, "logp")
    within(host(lse), z, (tol + U32 * np.abs(z)) * NEAR, "lse")
    got = host(logp).reshape(m.nblk, -1)
    each = [ends.preference_loss(got[b], host(m.ref), m.labels_h, np.arange(5) * m.seq_len, 0.1)[0] for b in range(m.nblk)]
    np.testing.assert_allclose(host(loss), each, rtol=1e-12)
    assert len(set(each)) == m.nblk  # every block is another model
    est = [(each[2 * j] - each[2 * j + 1]) / (2 * float(np.float32(m.eps))) for j in range(m.q)]
    np.testing.assert_allclose(host(g), est, rtol=1e-6)
    # The update takes them.
    items = [dict(W=t["W"], U=t["U"], V=t["V"], Z=t["Z"], M1=torch.zeros(m.r, m.r, device="cuda"),
                  M2=torch.zeros(m.r, m.r, device="cuda")) for t in m.mats.values()]
    before = [bits(t["W"]).copy() for t in items]
    zo.subspace_adam_update(items, g, 1, 1e-2, 0.9, 0.95, 1e-8)
    assert all((bits(t["W"]) != old).any() for t, old in zip(items, before))


def test_gradients_of_the_two_tables():
    """A head tied to the embedding: its gradient comes from the logits' and from the embedding's input rows, added up."""
    m = Model(vocab=1000)
    H, logits, logp, lse, _ = m.losses()
    T = m.T
    x, logits, logp, lse = m.X[:T], logits[:T].contiguous(), logp[:T].contiguous(), lse[:T].contiguous()
    dlogp = torch.zeros(T, device="cuda")
    zo.preference_loss(logp, m.start, 0.1, ref_logp=m.ref, labels=m.labels, dlogp=dlogp)
    dlogits = zo.token_logprob_backward(logits, m.labels, lse, dlogp, vocab=m.vocab)
    tied = (dlogits.t().contiguous() @ x.float())  # vocab x d
    head_part = tied.clone()
    dH = torch.from_numpy(m.rng.standard_normal((T, m.d))).float().cuda()
    zo.embedding_backward(m.ids, dH, m.vocab, scale=1.5, out=tied, accumulate=True)
    # In float64 by autograd, from the same logits.
    X = torch.from_numpy(host(logits)).requires_grad_()
    lab = torch.from_numpy(m.labels_h).long()
    on = lab >= 0
    lp = torch.log_softmax(X, -1).gather(1, lab.clamp(min=0)[:, None])[:, 0] * on
    R = ((lp - torch.from_numpy(host(m.ref))) * on).reshape(4, -1).sum(1)
    loss = -torch.nn.functional.logsigmoid(0.1 * (R[0::2] - R[1::2])).mean()
    loss.backward()
    gx = X.grad.numpy()
    # logp and lse are fp32 (2^-24 of about 8, twice), p is 3 |a| + 3 roundings off, |a| <= 20 here; the slope adds 0.1 of the
    # sums' rounding over a sequence.
    bound = np.abs(gx).max(1, keepdims=True) * (64 * U32 + 2 * 8 * U32 + 0.1 * m.seq_len * 8 * U32)
    within(host(dlogits), gx, bound, "dlogits")
    G = ends.embedding_backward(m.ids_h, host(dH), m.vocab, 1.5)
    n = np.maximum(G[2] - 1, 0)[:, None]
    sum_tol = (n * U32 * G[1] + 2 * U32 * (np.abs(host(head_part)) + np.abs(G[0]))) * NEAR + 1e-30
    within(host(tied), host(head_part) + G[0], sum_tol, "tied")


def test_a_policy_step_of_sampled_answers():
    """Two answers to each of two prompts, advantages by group: the policy gradient reaches the logits."""
    m = Model()
    _, logits, logp, lse, _ = m.losses()
    T = m.T
    old = (logp[:T] + 0.1 * torch.from_numpy(m.rng.standard_normal(T)).float().cuda()).clamp(max=0.0)
    adv = torch.tensor([0.7, -0.7, 0.3, -0.3], device="cuda")
    stats, dlogp = torch.zeros(m.nblk, 2, dtype=torch.float64, device="cuda"), torch.zeros(m.nblk, T, device="cuda")
    loss = zo.policy_loss(logp.view(m.nblk, -1), old, adv, m.start, labels=m.labels, ref_logp=m.ref, kl_coef=0.05,
                          aggregate="sequence", stats=stats, dlogp=dlogp)
    for b in range(m.nblk):
        want = ends.policy_loss(host(logp)[b * T:(b + 1) * T], host(old), host(adv), m.labels_h, np.arange(5) * m.seq_len,
                                host(m.ref), kl_coef=0.05, aggregate="sequence")
        np.testing.assert_allclose(loss[b].item(), want[0], rtol=1e-11)
        np.testing.assert_allclose(host(stats)[b], want[1], rtol=1e-11, atol=1e-14)
        within(host(dlogp)[b], want[2], U32 * np.abs(want[2]) * NEAR + 1e-14)
    zo.token_logprob_backward(logits, m.labels, lse, dlogp.view(-1), vocab=m.vocab, out=logits)
    assert (host(logits)[np.tile(m.labels_h, m.nblk) < 0, :m.vocab] == 0).all() and torch.isfinite(logits).all()


# --------------------------------------------------------------------------- how calls may be made
class Calls:
    """Every entry point once, on sizes that take each of its launches; inputs that can be drawn again in place."""

    def __init__(self, n, vocab, d, few=False, dt=torch.bfloat16, seed=0):
        self.g = torch.Generator(device="cuda")
        self.n, self.vocab, self.dt = n, vocab, dt
        self.ids = torch.empty(n, dtype=torch.int32, device="cuda")
        self.table = torch.empty(vocab, d, dtype=dt, device="cuda")
        self.grad = torch.empty(n, d, dtype=dt, device="cuda")
        self.rows = 3 if few else 150
        self.V = 140001 if few else 5003
        self.x = torch.empty(2 * self.rows, self.V, dtype=dt, device="cuda")
        self.labels = torch.empty(self.rows, dtype=torch.int32, device="cuda")
        self.dl = torch.empty(2 * self.rows, device="cuda")
        self.seqs = 8 if few else 64
        self.T = self.seqs * (20 if few else 150)
        self.start = torch.arange(0, self.T + 1, self.T // self.seqs, dtype=torch.int32, device="cuda")
        self.logp, self.old, self.ref = (torch.empty(k, self.T, device="cuda") for k in (3, 1, 1))
        self.adv = torch.empty(self.seqs, device="cuda")
        self.count = torch.empty(self.T, dtype=torch.int32, device="cuda")
        self.sum = torch.zeros(vocab, d, device="cuda")
        self.draw(seed)

    def draw(self, seed):
        self.g.manual_seed(seed)
        for t in (self.table, self.grad, self.x, self.dl, self.logp, self.old, self.ref, self.adv, self.sum):
            t.copy_(torch.randn(t.shape, generator=self.g, device="cuda"))
        self.ids.copy_((torch.rand(self.n, generator=self.g, device="cuda").square() * self.vocab).int() - 1)
        self.labels.copy_(torch.randint(-20, self.V, (self.rows,), generator=self.g, device="cuda").int())
        self.count.copy_(torch.randint(-1, 2, (self.T,), generator=self.g, device="cuda").int())

    def run(self):
        out = [zo.embedding(self.ids, self.table, scale=1.25)]
        out.append(zo.embedding_backward(self.ids, self.grad, self.vocab, out=torch.empty_like(self.table)))
        out.append(zo.embedding_backward(self.ids, self.grad, self.vocab, out=self.sum.clone(), accumulate=True))
        logp, lse = zo.token_logprob(self.x, self.labels, vocab=self.V - 3)
        out += [logp, lse, zo.token_logprob_backward(self.x, self.labels, lse, self.dl, vocab=self.V - 3)]
        for kw in (dict(kind="sigmoid", label_smoothing=0.1), dict(kind="ipo", average=True)):
            d = torch.zeros_like(self.logp)
            out += [zo.preference_loss(self.logp, self.start, 0.2, ref_logp=self.ref[0], labels=self.count, dlogp=d, **kw), d]
        for agg in ("token", "sequence"):
            d, st = torch.zeros_like(self.logp), torch.zeros(3, 2, dtype=torch.float64, device="cuda")
            out += [zo.policy_loss(self.logp, self.old[0], self.adv, self.start, labels=self.count, ref_logp=self.ref[0],
                                   kl_coef=0.1, aggregate=agg, stats=st, dlogp=d), st, d]
        return out


def _same(a, b):
    for k, (x, y) in enumerate(zip(a, b)):
        np.testing.assert_array_equal(bits(x), bits(y), err_msg=f"output {k}")


SIZES = [(200, 3000, 264, True), (5000, 3000, 264, False), (20000, 9000, 136, False)]


@pytest.mark.parametrize("n,vocab,d,few", SIZES)
def test_captured_calls(n, vocab, d, few):
    """Two graphs of the same calls on inputs of their own, replayed in turn with eager calls between them."""
    made = [Calls(n, vocab, d, few, seed=s) for s in (1, 2)]
    for c in made:
        c.run()
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    graphs, outs = [], []
    for c in made:
        side.wait_stream(torch.cuda.current_stream())
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=side):
            outs.append(c.run())
        graphs.append(g)
    for rep in range(4):
        for c, g, out in zip(made, graphs, outs):
            c.draw(100 * rep + 7)
            g.replay()
            want = c.run()
            torch.cuda.synchronize()
            _same(out, want)
    # The two at once, on two streams.
    others = [torch.cuda.Stream() for _ in made]
    want = [c.run() for c in made]
    torch.cuda.synchronize()
    for rep in range(3):
        for st, g in zip(others, graphs):
            with torch.cuda.stream(st):
                g.replay()
    torch.cuda.synchronize()
    for out, w in zip(outs, want):
        _same(out, w)


@pytest.mark.parametrize("n,vocab,d,few", SIZES)
def test_two_streams_at_once(n, vocab, d, few):
    """The same calls from two streams, neither the one that made the tensors."""
    made = [Calls(n, vocab, d, few, seed=s) for s in (3, 4)]
    want = [c.run() for c in made]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in made]
    got = [[] for _ in made]
    for rep in range(3):
        for k, (c, st) in enumerate(zip(made, streams)):
            with torch.cuda.stream(st):
                got[k].append(c.run())
    torch.cuda.synchronize()
    for outs, w in zip(got, want):
        for out in outs:
            _same(out, w)


def test_a_workspace_of_the_callers():
    """One buffer for calls in a row, larger than they need and full of anything."""
    c = Calls(5000, 3000, 264, False, seed=5)
    want = c.run()
    ws = torch.full((64 << 20,), 255, dtype=torch.uint8, device="cuda")
    dE = zo.embedding_backward(c.ids, c.grad, c.vocab, out=torch.empty_like(c.table), workspace=ws)
    np.testing.assert_array_equal(bits(dE), bits(want[1]))
    few = Calls(200, 3000, 264, True, seed=6)
    logp, lse = zo.token_logprob(few.x, few.labels, vocab=few.V - 3, workspace=ws)
    ref = zo.token_logprob(few.x, few.labels, vocab=few.V - 3)
    _same([logp, lse], ref)
    loss = zo.policy_loss(c.logp, c.old[0], c.adv, c.start, labels=c.count, ref_logp=c.ref[0], kl_coef=0.1, workspace=ws)
    np.testing.assert_array_equal(bits(loss), bits(want[10]))
    with pytest.raises(zo.ZoError, match="workspace"):
        zo.embedding_backward(c.ids, c.grad, c.vocab, workspace=ws[:256])
