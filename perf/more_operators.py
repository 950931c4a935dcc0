"""The two ends of a language model whose layers are tuned: tokens in, log-probabilities and losses out, and their gradients.

Six operators:

    embed        rows of a table by token, scaled; a negative token is padding (a row of zeros)
    embed_grad   the table's gradient: the scaled sum of the incoming rows of each token, dense or added to what is there
    logprob      log-softmax of scaled logits at each row's label, and the row's log-sum-exp; a negative label is not counted
    logprob_grad the logits' gradient from the gradient of those log-probabilities
    preference   loss of pairs of sequences (2p chosen, 2p + 1 rejected) from token log-probabilities of the model and of a
                 reference, with its gradient
    policy       clipped policy loss with a KL term over sequences of sampled tokens, with its gradient

Logits and log-probabilities come in blocks, one for each query of a zeroth-order step (or one block); tokens, labels,
reference log-probabilities and advantages are shared by the blocks.  Logits may be wider than the vocabulary (a padded
head): columns behind it belong to nobody.  Rows behind the last sequence stay as they are.

    listed()            the cases, with a name each
    draw(rng)           one more case of the same ranges
    prepare(case, seed) inputs on the GPU, and the output buffers that a program keeps from step to step
    run(state)          one pass; returns its outputs.  own: by the package's entry points, else in plain torch
    work(case)          bytes and operations of one pass that no implementation can do without
    exact(case, seed)   the same outputs in float64
"""
import math

import torch

own = False

DTYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}
SIZE = {"bf16": 2, "f16": 2, "f32": 4}
HIDDEN = 0.3  # share of a sequence that is its prompt: not counted
PAD_ID = 0.02  # share of padding tokens


def listed():
    return [
        # The next token of one answer: nothing but latency.
        dict(name="embed_token_bf16", kind="embed", dtype="bf16", rows=1, vocab=32000, d=4096, scale=1.0),
        # The prompts of 16 x 16 sequences of 256 tokens, a scaled table.
        dict(name="embed_prompts_f16", kind="embed", dtype="f16", rows=65536, vocab=50272, d=5120, scale=64.0),
        # Some answers' tokens added to the gradient of a table that the head shares.
        dict(name="embed_grad_few_bf16", kind="embed_grad", dtype="bf16", rows=61, vocab=32000, d=4096, scale=1.0, add=True),
        # 16 sequences of 512 tokens: the dense gradient of a large table, nearly all of it zeros.
        dict(name="embed_grad_batch_bf16", kind="embed_grad", dtype="bf16", rows=8192, vocab=50272, d=5120, scale=1.0,
             add=False),
        # Many tokens in fp32, added: sorting and long runs of frequent tokens count.
        dict(name="embed_grad_many_f32", kind="embed_grad", dtype="f32", rows=131071, vocab=151936, d=1024, scale=32.0,
             add=True),
        # Scoring a handful of tokens against a very large vocabulary.
        dict(name="logprob_few_bf16", kind="logprob", dtype="bf16", nblk=1, rows=5, vocab=151936, ld=151936, scale=1.0),
        # 16 sequences of 512 tokens, the prompts not counted, a vocabulary of odd size in a padded head.
        dict(name="logprob_batch_bf16", kind="logprob", dtype="bf16", nblk=1, rows=8192, vocab=151851, ld=152064, scale=1.0),
        # Eight query blocks of 1000 tokens each, logits in fp32 at a temperature.
        dict(name="logprob_blocks_f32", kind="logprob", dtype="f32", nblk=8, rows=1000, vocab=32000, ld=32000, scale=1.25),
        # The logits' gradient of a training batch.
        dict(name="logprob_grad_f16", kind="logprob_grad", dtype="f16", nblk=1, rows=8192, vocab=50272, ld=50272, scale=1.0),
        # 64 preference pairs with the gradient: an ordinary batch.
        dict(name="preference_batch", kind="preference", nblk=1, nseq=128, new=512, ragged=True, pad=7, loss="sigmoid",
             average=False, ref=True, grad=True),
        # A group of 8 answers to each of 2 prompts: the smallest policy step.
        dict(name="policy_group", kind="policy", nblk=1, nseq=16, new=200, ragged=True, pad=0, aggregate="sequence",
             ref=False, per_token=False, grad=True),
        # 512 answers of up to 1024 tokens under 16 query blocks with the KL term, the loss alone.
        dict(name="policy_blocks", kind="policy", nblk=16, nseq=512, new=1024, ragged=True, pad=100, aggregate="token",
             ref=True, per_token=True, grad=False),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


# What the largest listed cases of each kind move.
MOST_BYTES = dict(embed=8.4e8, embed_grad=8.4e8, logprob=1.74e9, logprob_grad=1.4e9, preference=2.2e7, policy=2.2e7)


def draw(rng):
    kind = rng.choice(sorted(MOST_BYTES))
    c = dict(kind=kind)
    if kind in ("embed", "embed_grad"):
        c.update(dtype=rng.choice(["bf16", "f16", "f32"]), rows=_log_int(rng, 1, 131072), vocab=_log_int(rng, 1000, 160000),
                 d=8 * _log_int(rng, 16, 1024), scale=rng.choice([1.0, 1.0, 32.0, 71.5]))
        if kind == "embed_grad":
            c["add"] = rng.random() < 0.5
    elif kind in ("logprob", "logprob_grad"):
        c.update(dtype=rng.choice(["bf16", "f16", "f32"]), nblk=rng.choice([1, 1, 2, 8, 16]), rows=_log_int(rng, 1, 8192),
                 vocab=_log_int(rng, 1000, 160000), scale=rng.choice([1.0, 1.0, 0.7, 1.25]))
        c["ld"] = c["vocab"] + rng.choice([0, 0, 1, 37, -c["vocab"] % 128])
    else:
        c.update(nblk=rng.choice([1, 1, 2, 8, 16]), nseq=_log_int(rng, 2, 1024), new=_log_int(rng, 1, 8192),
                 ragged=rng.random() < 0.75, pad=rng.choice([0, 0, 1, 50]), ref=rng.random() < 0.7, grad=rng.random() < 0.7)
        if kind == "preference":
            c["nseq"] += c["nseq"] % 2
            c.update(loss=rng.choice(["sigmoid", "sigmoid", "ipo", "hinge"]), average=rng.random() < 0.4)
        else:
            c.update(aggregate=rng.choice(["token", "sequence", "sum"]), per_token=rng.random() < 0.5)
    while work(c)["bytes"] > MOST_BYTES[kind]:
        if kind == "embed_grad" and not c["add"] and c["rows"] < c["vocab"]:
            c["vocab"] = c["vocab"] * 2 // 3
        elif "rows" in c:
            c["rows"] = c["rows"] * 2 // 3
        else:
            c["new"] = c["new"] * 2 // 3
    return c


def _lengths(c):
    """Rows of every sequence: the same for every seed.  Some are a single token."""
    if not c["ragged"]:
        return [c["new"]] * c["nseq"]
    return [max(1, round(c["new"] * ((0.381966 + 0.618034 * s) % 1.0))) for s in range(c["nseq"])]


def _counted(c):
    """Rows whose label counts, for the cases whose rows are one run of sequences of 512 tokens."""
    return [t for t in range(c["rows"]) if c["rows"] < 64 or t % 512 >= HIDDEN * min(512, c["rows"])]


# --------------------------------------------------------------------------- inputs
class _Gen:
    """Tensors drawn on the GPU from one seed."""

    def __init__(self, seed):
        self.g = torch.Generator(device="cuda")
        self.g.manual_seed(int(seed))

    def normal(self, *shape, dtype=torch.float32):
        return torch.randn(*shape, generator=self.g, device="cuda", dtype=dtype)

    def uniform(self, *shape, dtype=torch.float32):
        return torch.rand(*shape, generator=self.g, device="cuda", dtype=dtype)

    def tokens(self, n, vocab):
        """Tokens as text has them: the r-th most frequent one with a share of about 1 / r."""
        rank = torch.exp(self.uniform(n, dtype=torch.float64) * math.log(vocab + 1.0)).long() - 1
        step = next(s for s in range(vocab // 3 + 7, 2 * vocab + 7) if math.gcd(s, vocab) == 1)
        return (rank.clamp(0, vocab - 1) * step % vocab).int()


def prepare(case, seed):
    c = dict(case)
    g = _Gen(seed)
    s = dict(case=c)
    if c["kind"] in ("embed", "embed_grad"):
        dt, rows, vocab, d = DTYPES[c["dtype"]], c["rows"], c["vocab"], c["d"]
        ids = g.tokens(rows, vocab)
        s["ids"] = ids.masked_fill(g.uniform(rows) < PAD_ID, -1) if rows >= 64 else ids
        if c["kind"] == "embed":
            s["table"] = torch.cat([(0.02 * g.normal(min(8192, vocab - v), d)).to(dt) for v in range(0, vocab, 8192)])
            s["out"] = torch.zeros(rows, d, dtype=dt, device="cuda")
        else:
            s["grad"] = torch.cat([(0.1 * g.normal(min(8192, rows - t), d)).to(dt) for t in range(0, rows, 8192)])
            # A gradient that is added to is kept in fp32; one that is whole comes in the type of the rows.
            s["dE"] = g.normal(vocab, d) if c["add"] else torch.zeros(vocab, d, dtype=dt, device="cuda")
    elif c["kind"] in ("logprob", "logprob_grad"):
        dt, rows, n, vocab, ld = DTYPES[c["dtype"]], c["rows"], c["nblk"] * c["rows"], c["vocab"], c["ld"]
        label = torch.full((rows,), -100, dtype=torch.int32)
        at = torch.tensor(_counted(c))
        label[at] = g.tokens(at.numel(), vocab).cpu()
        s["label"] = label.cuda()
        x = torch.empty(n, ld, dtype=dt, device="cuda")
        for r in range(0, n, 1024):
            x[r:r + 1024] = 2.5 * g.normal(min(1024, n - r), ld)
        # The label is likely, now more and now less so.
        rise = (4.0 + 5.0 * g.normal(n)).to(dt)
        col = s["label"].long().clamp(min=0).repeat(c["nblk"])
        x[torch.arange(n, device="cuda"), col] += rise
        s["x"] = x
        if c["kind"] == "logprob":
            s["logp"], s["lse"] = torch.zeros(n, device="cuda"), torch.zeros(n, device="cuda")
        else:
            s["lse"] = torch.cat([torch.logsumexp(x[r:r + 256, :vocab].double() * c["scale"], -1)
                                  for r in range(0, n, 256)]).float()
            s["g"] = g.normal(n).masked_fill(s["label"].repeat(c["nblk"]) < 0, 0.0)
            s["out"] = torch.zeros(n, ld, dtype=dt, device="cuda")
    else:
        length = _lengths(c)
        rows, nblk, nseq = sum(length) + c["pad"], c["nblk"], c["nseq"]
        start, label = [0], []
        for n in length:
            start.append(start[-1] + n)
            hid = int(n * HIDDEN)
            label += [-100] * hid + [5] * (n - hid)
        s["start"] = torch.tensor(start, dtype=torch.int32).cuda()
        s["label"] = torch.tensor(label + [-100] * c["pad"], dtype=torch.int32).cuda()
        off = s["label"] < 0
        base = -2.0 * g.normal(rows).abs() * g.uniform(rows)
        s["logp"] = (base + 0.05 * g.normal(nblk, rows)).clamp(max=0.0).masked_fill(off, 0.0)
        s["ref"] = (base + 0.1 * g.normal(rows)).clamp(max=0.0).masked_fill(off, 0.0) if c["ref"] else None
        s["dlogp"] = torch.zeros(nblk, rows, device="cuda") if c["grad"] else None
        s["loss"] = torch.zeros(nblk, dtype=torch.float64, device="cuda")
        if c["kind"] == "preference":
            s["rewards"] = torch.zeros(nblk, nseq, device="cuda")
        else:
            s["old"] = (base + 0.12 * g.normal(rows)).clamp(max=0.0).masked_fill(off, 0.0)
            s["adv"] = g.normal(rows if c["per_token"] else nseq)
            s["stats"] = torch.zeros(nblk, 2, dtype=torch.float64, device="cuda")
    return s


BETA, SMOOTH = 0.1, 0.05  # of the preference loss
LOW, HIGH, KL = 0.2, 0.28, 0.04  # of the policy loss


def _smooth(c):
    return SMOOTH if c["loss"] == "sigmoid" else 0.0


# --------------------------------------------------------------------------- plain form
def _embed(s):
    ids = s["ids"].long()
    h = s["table"][ids.clamp(min=0)].float() * s["case"]["scale"]
    s["out"].copy_(h.masked_fill_((ids < 0)[:, None], 0.0))
    return s["out"]


def _embed_grad(s):
    c, ids = s["case"], s["ids"].long()
    rows = (s["grad"].float() * c["scale"]).masked_fill_((ids < 0)[:, None], 0.0)
    if c["add"]:
        s["dE"].index_add_(0, ids.clamp(min=0), rows)
    else:
        s["dE"].copy_(torch.zeros(c["vocab"], c["d"], device="cuda").index_add_(0, ids.clamp(min=0), rows))
    return s["dE"]


def _logprob(s):
    c = s["case"]
    label = s["label"].long().repeat(c["nblk"])
    x = s["x"][:, :c["vocab"]].float() * c["scale"]
    at = x.gather(1, label.clamp(min=0)[:, None])[:, 0]
    top = x.amax(-1, keepdim=True)
    total = x.sub_(top).exp_().sum(-1)
    lse = top[:, 0] + total.log()
    s["logp"].copy_(torch.where(label < 0, 0.0, at - lse))
    s["lse"].copy_(torch.where(label < 0, 0.0, lse))
    return [s["logp"], s["lse"]]


def _logprob_grad(s):
    c = s["case"]
    label = s["label"].long().repeat(c["nblk"])
    p = (s["x"][:, :c["vocab"]].float() * c["scale"]).sub_(s["lse"][:, None]).exp_().neg_()
    p[torch.arange(label.numel(), device="cuda"), label.clamp(min=0)] += 1.0
    p.mul_((s["g"] * c["scale"])[:, None]).masked_fill_((label < 0)[:, None], 0.0)
    s["out"][:, :c["vocab"]] = p
    return s["out"]


def _sums(x, start):
    """Sums of x (blocks x rows, float64) over each sequence."""
    run = torch.cat([torch.zeros_like(x[:, :1]), x.cumsum(1)], 1)
    return run[:, start[1:]] - run[:, start[:-1]]


def _preference(s):
    c, start, n = s["case"], s["start"].long(), sum(_lengths(s["case"]))
    on = s["label"] >= 0
    ratio = s["logp"].double() if s["ref"] is None else s["logp"].double() - s["ref"].double()
    count = _sums(on[None].double(), start)
    share = 1.0 / count.clamp(min=1.0) if c["average"] else torch.ones_like(count)
    reward = _sums(ratio.masked_fill(~on, 0.0), start) * share
    z = reward[:, 0::2] - reward[:, 1::2]
    h = BETA * z
    if c["loss"] == "sigmoid":
        up = torch.exp(-h.abs())
        log1 = torch.log1p(up)  # -log sigma(|h|)
        lose = (1 - SMOOTH) * (log1 + (-h).clamp(min=0.0)) + SMOOTH * (log1 + h.clamp(min=0.0))
        right = torch.where(h >= 0, 1.0, up) / (1.0 + up)  # sigma(h)
        slope = BETA * (SMOOTH * right - (1 - SMOOTH) * (1.0 - right))
    elif c["loss"] == "hinge":
        lose, slope = (1.0 - h).clamp(min=0.0), torch.where(h < 1.0, -BETA, 0.0).double()
    else:
        lose, slope = (z - 0.5 / BETA).square(), 2.0 * (z - 0.5 / BETA)
    s["loss"].copy_(lose.mean(1))
    s["rewards"].copy_(BETA * reward)
    if c["grad"]:
        coef = torch.stack([slope, -slope], -1).reshape(c["nblk"], -1) * share / z.shape[1]
        seq = torch.repeat_interleave(torch.arange(c["nseq"], device="cuda"), start[1:] - start[:-1], output_size=n)
        s["dlogp"][:, :n] = coef[:, seq].masked_fill_(~on[:n], 0.0)
        return [s["loss"], s["rewards"], s["dlogp"]]
    return [s["loss"], s["rewards"]]


def _policy(s):
    c, start, n = s["case"], s["start"].long(), sum(_lengths(s["case"]))
    on = s["label"][:n] >= 0
    seq = torch.repeat_interleave(torch.arange(c["nseq"], device="cuda"), start[1:] - start[:-1], output_size=n)
    adv = (s["adv"][:n] if c["per_token"] else s["adv"][seq]).double()
    p = s["logp"][:, :n].double()
    ratio = torch.exp(p - s["old"][:n].double())
    plain, kept = ratio * adv, ratio.clamp(1.0 - LOW, 1.0 + HIGH) * adv
    cut = plain > kept
    lose, slope = -torch.minimum(plain, kept), torch.where(cut, 0.0, -plain)
    kl = torch.zeros_like(lose)
    if c["ref"]:
        gap = s["ref"][:n].double() - p
        kl = torch.exp(gap) - gap - 1.0
        lose, slope = lose + KL * kl, slope + KL * (1.0 - torch.exp(gap))
    total = on.sum().clamp(min=1).double()
    if c["aggregate"] == "token":
        share = (1.0 / total).expand(n)
    elif c["aggregate"] == "sequence":
        share = (1.0 / _sums(on[None].double(), start)[0].clamp(min=1.0) / c["nseq"])[seq]
    else:
        share = torch.ones(n, dtype=torch.float64, device="cuda")
    share = share.masked_fill(~on, 0.0)
    s["loss"].copy_((lose * share).sum(1))
    s["stats"][:, 0] = kl.masked_fill(~on, 0.0).sum(1) / total
    s["stats"][:, 1] = (cut & on).double().sum(1) / total
    if c["grad"]:
        s["dlogp"][:, :n] = slope * share
        return [s["loss"], s["stats"], s["dlogp"]]
    return [s["loss"], s["stats"]]


PLAIN = dict(embed=_embed, embed_grad=_embed_grad, logprob=_logprob, logprob_grad=_logprob_grad, preference=_preference,
             policy=_policy)


def run(s):
    if own:
        import paper_2608_15665_amd as zo
        c = s["case"]
        if c["kind"] == "embed":
            return zo.embedding(s["ids"], s["table"], scale=c["scale"], out=s["out"])
        if c["kind"] == "embed_grad":
            return zo.embedding_backward(s["ids"], s["grad"], c["vocab"], scale=c["scale"], out=s["dE"], accumulate=c["add"])
        if c["kind"] == "logprob":
            return list(zo.token_logprob(s["x"], s["label"], vocab=c["vocab"], scale=c["scale"], logp=s["logp"],
                                         lse=s["lse"]))
        if c["kind"] == "logprob_grad":
            return zo.token_logprob_backward(s["x"], s["label"], s["lse"], s["g"], vocab=c["vocab"], scale=c["scale"],
                                             out=s["out"])
        if c["kind"] == "preference":
            zo.preference_loss(s["logp"], s["start"], BETA, ref_logp=s["ref"], labels=s["label"], kind=c["loss"],
                               average=c["average"], label_smoothing=_smooth(c), loss=s["loss"], rewards=s["rewards"],
                               dlogp=s["dlogp"])
            return [s["loss"], s["rewards"]] + ([s["dlogp"]] if c["grad"] else [])
        zo.policy_loss(s["logp"], s["old"], s["adv"], s["start"], labels=s["label"], ref_logp=s["ref"],
                       per_token=c["per_token"], clip_low=LOW, clip_high=HIGH, kl_coef=KL if c["ref"] else 0.0,
                       aggregate=c["aggregate"], loss=s["loss"], stats=s["stats"], dlogp=s["dlogp"])
        return [s["loss"], s["stats"]] + ([s["dlogp"]] if c["grad"] else [])
    return PLAIN[s["case"]["kind"]](s)


# --------------------------------------------------------------------------- work
def _distinct(c):
    """About how many different tokens prepare() draws: a token of share p is among n with 1 - (1 - p)^n."""
    n, vocab, most = c["rows"], c["vocab"], 0.0
    lo = 1
    while lo <= vocab:  # ranks lo .. hi - 1 taken together
        hi = min(vocab + 1, lo + max(1, lo // 8))
        p = math.log((hi) / lo) / math.log(vocab + 1.0) / (hi - lo)
        most += (hi - lo) * -math.expm1(n * math.log1p(-min(p, 0.999999)))
        lo = hi
    return min(most, n)


def work(case):
    c = case
    if c["kind"] in ("embed", "embed_grad"):
        e, rows, d = SIZE[c["dtype"]], c["rows"], c["d"]
        if c["kind"] == "embed":
            return dict(bytes=4.0 * rows + e * d * (rows + _distinct(c)), flops=1.0 * rows * d)
        table = 8.0 * _distinct(c) * d if c["add"] else 1.0 * e * c["vocab"] * d
        return dict(bytes=4.0 * rows + e * rows * d + table, flops=2.0 * rows * d)
    if c["kind"] in ("logprob", "logprob_grad"):
        e, n, on = SIZE[c["dtype"]], c["nblk"] * c["rows"], c["nblk"] * len(_counted(c))
        if c["kind"] == "logprob":
            return dict(bytes=1.0 * on * c["vocab"] * e + 8.0 * n + 4.0 * c["rows"], flops=4.0 * on * c["vocab"])
        return dict(bytes=1.0 * (on + n) * c["vocab"] * e + 8.0 * n + 4.0 * c["rows"], flops=4.0 * on * c["vocab"])
    rows = sum(_lengths(c))
    shared = 1 + c["ref"] + (1 + c["per_token"] if c["kind"] == "policy" else 0)
    flops = (60.0 if c["kind"] == "policy" else 3.0) * c["nblk"] * rows
    return dict(bytes=4.0 * rows * (shared + c["nblk"] * (1 + c["grad"])) + 8.0 * c["nseq"], flops=flops)


# --------------------------------------------------------------------------- float64
def exact(case, seed):
    c = dict(case)
    s = prepare(c, seed)
    if c["kind"] == "embed":
        out = torch.zeros(c["rows"], c["d"], dtype=torch.float64, device="cuda")
        for t in range(0, c["rows"], 4096):
            ids = s["ids"][t:t + 4096].long()
            keep = ids >= 0
            out[t:t + 4096][keep] = s["table"][ids[keep]].double() * c["scale"]
        return out
    if c["kind"] == "embed_grad":
        dE = s["dE"].double() if c["add"] else torch.zeros(c["vocab"], c["d"], dtype=torch.float64, device="cuda")
        order = torch.argsort(s["ids"].long(), stable=True)
        order = order[int((s["ids"] < 0).sum()):]
        tokens, counts = torch.unique_consecutive(s["ids"][order].long(), return_counts=True)
        ends = torch.cumsum(counts, 0) - 1
        for col in range(0, c["d"], 256):  # running sums over the sorted rows, and their differences
            run = torch.cumsum(s["grad"][order, col:col + 256].double(), 0)[ends]
            dE[tokens, col:col + 256] += c["scale"] * torch.diff(run, dim=0, prepend=torch.zeros_like(run[:1]))
        return dE
    if c["kind"] in ("logprob", "logprob_grad"):
        n, vocab = c["nblk"] * c["rows"], c["vocab"]
        label = s["label"].long().repeat(c["nblk"])
        first, second = torch.zeros(2, n, dtype=torch.float64, device="cuda")
        out = s["out"].double() if c["kind"] == "logprob_grad" else None
        for r in range(0, n, 256):
            lab = label[r:r + 256]
            on = lab >= 0
            x = c["scale"] * s["x"][r:r + 256, :vocab].double()
            if out is None:
                z = torch.logsumexp(x, 1)
                hit = x.take_along_dim(lab.clamp(min=0)[:, None], 1)[:, 0]
                first[r:r + 256], second[r:r + 256] = (hit - z) * on, z * on
            else:
                is_label = torch.arange(vocab, device="cuda") == lab[:, None]
                up = (s["g"][r:r + 256].double() * c["scale"] * on)[:, None]
                out[r:r + 256, :vocab] = up * (is_label.double() - torch.exp(x - s["lse"][r:r + 256, None].double()))
        return [first, second] if out is None else out
    start, nblk, nseq = s["start"].tolist(), c["nblk"], c["nseq"]
    counted = [torch.nonzero(s["label"][a:b] >= 0)[:, 0] + a for a, b in zip(start, start[1:])]
    loss = torch.zeros(nblk, dtype=torch.float64, device="cuda")
    dlogp = torch.zeros_like(s["logp"], dtype=torch.float64)
    p = s["logp"].double()
    if c["kind"] == "preference":
        q = torch.zeros_like(p[0]) if s["ref"] is None else s["ref"].double()
        rewards = torch.zeros(nblk, nseq, dtype=torch.float64, device="cuda")
        for i in range(nseq // 2):
            leaf, sides = [], []
            for at in counted[2 * i:2 * i + 2]:
                x = p[:, at].clone().requires_grad_()
                r = (x - q[at]).sum(1)
                leaf.append(x)
                sides.append(r / at.numel() if c["average"] else r)
            z = sides[0] - sides[1]
            if c["loss"] == "sigmoid":
                one = -(1 - SMOOTH) * torch.nn.functional.logsigmoid(BETA * z) - SMOOTH * torch.nn.functional.logsigmoid(
                    -BETA * z)
            elif c["loss"] == "hinge":
                one = torch.relu(1 - BETA * z)
            else:
                one = (z - 1 / (2 * BETA)) ** 2
            one = one / (nseq // 2)
            one.sum().backward()
            loss += one.detach()
            for k in (0, 1):
                dlogp[:, counted[2 * i + k]] = leaf[k].grad
                rewards[:, 2 * i + k] = BETA * sides[k].detach()
        return [loss, rewards] + ([dlogp] if c["grad"] else [])
    stats = torch.zeros(nblk, 2, dtype=torch.float64, device="cuda")
    total = sum(at.numel() for at in counted)
    for i, at in enumerate(counted):
        x = p[:, at].clone().requires_grad_()
        a = s["adv"][at].double() if c["per_token"] else s["adv"][i].double()
        r = torch.exp(x - s["old"][at].double())
        gains = torch.where(a >= 0, a * r.clamp(max=1 + HIGH), a * r.clamp(min=1 - LOW))
        kl = torch.zeros_like(x)
        if c["ref"]:
            gap = s["ref"][at].double() - x
            kl = torch.expm1(gap) - gap
        each = (KL * kl - gains).sum(1)
        each = each / (total if c["aggregate"] == "token" else at.numel() * nseq if c["aggregate"] == "sequence" else 1)
        each.sum().backward()
        loss += each.detach()
        dlogp[:, at] = x.grad
        stats[:, 0] += kl.detach().sum(1) / total
        stats[:, 1] += ((a > 0) & (r > 1 + HIGH) | (a < 0) & (r < 1 - LOW)).double().sum(1) / total
    return [loss, stats] + ([dlogp] if c["grad"] else [])
