"""Answering with a tuned model: the paged key/value cache of one layer and the attention that reads it.

Four operators, each with 16-bit inputs (bf16 or fp16):

    append   the new rows' keys and values into a paged cache, keys and queries rotated to their positions
    append8  the same into a cache of 8-bit floats (e4m3) with a power-of-two scale per page, head and tensor
    attend   causal attention of the new rows' queries over a paged 16-bit cache
    attend8  the same over the 8-bit cache

Sequence s of a batch has the rows q_start[s] .. q_start[s + 1] - 1 of Q, K and V (one row each where there is no
q_start) and, those included, kv_len[s] keys: its rows are its last positions.  Position t lies in slot t % page of
page page_table[s][t // page]; a cache is pages x kv_heads x page x dh.  Rows behind the last sequence (a batch padded
to a fixed size) belong to nobody and stay as they are.

    listed()            the cases, with a name each
    draw(rng)           one more case of the same ranges
    prepare(case, seed) inputs on the GPU, and the buffers and tables a program keeps from step to step
    run(state)          one pass; returns its outputs.  own: by the package's entry points, else in plain torch
    work(case)          bytes and operations of one pass that no implementation can do without
    exact(case, seed)   the same outputs in float64, one sequence after another
"""
import math

import torch

own = False

DTYPES = {"bf16": torch.bfloat16, "f16": torch.float16}
E4M3 = torch.float8_e4m3fn
E4M3_MAX = 448.0
SPARE = 3  # pages of the pool that no sequence holds


def listed():
    qwen = dict(heads=40, kv_heads=8, dh=128, rope=1e6)
    llama = dict(heads=32, kv_heads=32, dh=128, rope=1e4)
    opt13b = dict(heads=40, kv_heads=40, dh=128, rope=0.0)
    opt1b = dict(heads=32, kv_heads=32, dh=64, rope=0.0)
    return [
        # One answer of a LLaMA-7B-shaped model, one layer's next token: nothing but latency.
        dict(name="append_one_bf16", kind="append", dtype="bf16", nseq=1, new=1, ctx=300, ragged=False, page=16,
             pad=0, **llama),
        # 61 answers at once from a Qwen-32B-shaped model, in a batch padded to 64 rows.
        dict(name="append_batch_f16", kind="append", dtype="f16", nseq=61, new=1, ctx=2048, ragged=True, page=64,
             pad=3, **qwen),
        # The prompts of the method's batch (16 sequences of up to 512 tokens), from nothing.
        dict(name="append_prompts_bf16", kind="append", dtype="bf16", nseq=16, new=512, ctx=0, ragged=True, page=64,
             pad=0, **qwen),
        # The 61 answers with the cache in 8 bits: new tokens fall into pages that earlier ones share.
        dict(name="append8_batch_bf16", kind="append8", dtype="bf16", nseq=61, new=1, ctx=2048, ragged=True, page=64,
             pad=3, **qwen),
        # The prompts of an OPT-1.3B-shaped model (heads of 64, no rotation), in 8 bits.
        dict(name="append8_prompts_f16", kind="append8", dtype="f16", nseq=16, new=512, ctx=0, ragged=True, page=32,
             pad=0, **opt1b),
        # One answer, a short context: the latency of a token.
        dict(name="attend_one_bf16", kind="attend", dtype="bf16", nseq=1, new=1, ctx=300, ragged=False, page=16,
             pad=0, **llama),
        # 61 answers with contexts of up to 8192 tokens, grouped heads: the ordinary step of answering.
        dict(name="attend_batch_bf16", kind="attend", dtype="bf16", nseq=61, new=1, ctx=8192, ragged=True, page=64,
             pad=3, **qwen),
        # One answer over a very long document.
        dict(name="attend_long_f16", kind="attend", dtype="f16", nseq=1, new=1, ctx=131071, ragged=False, page=128,
             pad=0, **qwen),
        # Pieces of four long prompts over what is cached of them: the products bound it.
        dict(name="attend_pieces_bf16", kind="attend", dtype="bf16", nseq=4, new=1000, ctx=7000, ragged=True, page=64,
             pad=0, **qwen),
        # The 61 answers with the cache in 8 bits.
        dict(name="attend8_batch_bf16", kind="attend8", dtype="bf16", nseq=61, new=1, ctx=8192, ragged=True, page=64,
             pad=3, **qwen),
        # Four drafted tokens of each of 24 answers looked at together, an OPT-13B-shaped model (one
        # key/value head per query head), small pages.
        dict(name="attend8_drafts_f16", kind="attend8", dtype="f16", nseq=24, new=4, ctx=2048, ragged=True, page=16,
             pad=0, **opt13b),
        # Pieces of prompts over an 8-bit cache, a LLaMA-7B-shaped model.
        dict(name="attend8_pieces_bf16", kind="attend8", dtype="bf16", nseq=8, new=256, ctx=4096, ragged=True, page=64,
             pad=0, **llama),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


# What the largest listed cases take: gathered keys, bytes and operations.
MOST_KEYS, MOST_BYTES, MOST_FLOPS = 61 * 8192 * 8 * 128, 1.08e9, 2.17e11


def draw(rng):
    kind = rng.choice(["append", "append8", "attend", "attend", "attend8", "attend8"])
    group = rng.choice([1, 1, 2, 4, 5, 7, 8])
    kv_heads = rng.randint(1, 40 if group == 1 else 8)
    c = dict(kind=kind, dtype=rng.choice(["bf16", "f16"]), nseq=_log_int(rng, 1, 96), ragged=rng.random() < 0.75,
             page=rng.choice([16, 32, 64, 128, 256]), pad=rng.choice([0, 0, 1, 5]), heads=group * kv_heads,
             kv_heads=kv_heads, dh=rng.choice([64, 128, 128]), rope=rng.choice([0.0, 1e4, 1e6]))
    form = rng.choice(["token", "token", "drafts", "piece"])
    c["new"] = 1 if form == "token" else rng.randint(2, 8) if form == "drafts" else _log_int(rng, 16, 1024)
    top = 4096 if kind in ("append", "append8") else 65536
    c["ctx"] = 0 if form == "piece" and rng.random() < 0.3 else _log_int(rng, 1, top)
    while (c["nseq"] * (c["ctx"] + c["new"]) * kv_heads * c["dh"] > MOST_KEYS or work(c)["bytes"] > MOST_BYTES
           or work(c)["flops"] > MOST_FLOPS):
        if c["nseq"] > 1:
            c["nseq"] = c["nseq"] * 2 // 3
        else:
            c["ctx"], c["new"] = c["ctx"] * 2 // 3, max(1, c["new"] * 2 // 3)
    return c


def _lengths(c):
    """(new rows, keys with them) of every sequence: the same for every seed."""
    new, total = [], []
    for s in range(c["nseq"]):
        u, v = (0.381966 + 0.618034 * s) % 1.0, (0.754878 + 0.569840 * s) % 1.0
        n = c["new"] if not c["ragged"] else max(1, round(c["new"] * (0.3 + 0.7 * u)))
        cached = c["ctx"] if not c["ragged"] else round(c["ctx"] * (0.05 + 0.95 * v))
        new.append(n)
        total.append(cached + n)
    return new, total


# --------------------------------------------------------------------------- inputs
class _Gen:
    """Tensors drawn on the GPU from one seed."""

    def __init__(self, seed):
        self.g = torch.Generator(device="cuda")
        self.g.manual_seed(int(seed))

    def normal(self, *shape, dtype=torch.float32):
        return torch.randn(*shape, generator=self.g, device="cuda", dtype=dtype)

    def perm(self, n):
        return torch.randperm(n, generator=self.g, device="cuda")


def _cache8(x):
    """e4m3 codes and scales of a pool of pages (pages x kv_heads x page x dh), as a filled cache holds them."""
    m, e = torch.frexp(x.abs().amax((2, 3)).float())
    scale = torch.ldexp(torch.ones_like(m), e - 9 + (m > 0.875))
    return (x.float() / scale[..., None, None]).to(E4M3), scale


def prepare(case, seed):
    c = dict(case)
    g, dt = _Gen(seed), DTYPES[c["dtype"]]
    H, KV, dh, ps, nseq = c["heads"], c["kv_heads"], c["dh"], c["page"], c["nseq"]
    new, total = _lengths(c)
    rows = sum(new) + c["pad"]
    held = [-(-t // ps) for t in total]
    pages = sum(held) + SPARE
    s = dict(case=c, max_new=max(new))
    # Entries behind a sequence's last page are not in use and hold no page.
    order, width = g.perm(pages).int(), max(held) + 2
    table = torch.full((nseq, width), -1, dtype=torch.int32)
    where = torch.cat([torch.arange(n) + i * width for i, n in enumerate(held)])
    table = table.cuda()
    table.view(-1)[where.cuda()] = order[:sum(held)]
    starts = [0]
    for n in new:
        starts.append(starts[-1] + n)
    s["page_table"] = table
    s["kv_len"] = torch.tensor(total, dtype=torch.int32).cuda()
    s["q_start"] = None if c["new"] == 1 else torch.tensor(starts, dtype=torch.int32).cuda()
    # Keys have channels that are larger than others, each head its own; values do not.  Pages differ too.
    chan = torch.exp(0.5 * g.normal(KV, 1, dh))
    size = torch.exp(0.4 * g.normal(pages, 1, 1, 1))
    pool = lambda f: torch.cat([(g.normal(min(256, pages - p), KV, ps, dh) * f * size[p:p + 256]).to(dt)
                                for p in range(0, pages, 256)])
    kc, vc = pool(chan), pool(0.5)
    s["k_scale"] = s["v_scale"] = None
    if c["kind"] in ("append8", "attend8"):
        (kc, s["k_scale"]), (vc, s["v_scale"]) = _cache8(kc), _cache8(vc)
    s["k_cache"], s["v_cache"] = kc, vc
    if c["kind"] in ("append", "append8"):
        # One product gives queries, keys and values: they are column ranges of its output.
        qkv = g.normal(rows, (H + 2 * KV) * dh)
        qkv[:, H * dh:(H + KV) * dh] *= chan.reshape(-1)
        qkv = qkv.to(dt)
        s["Q"], s["K"], s["V"] = qkv[:, :H * dh], qkv[:, H * dh:(H + KV) * dh], qkv[:, (H + KV) * dh:]
        s["q_out"] = torch.zeros(rows, H * dh, dtype=dt, device="cuda") if c["rope"] else None
    else:
        s["Q"] = (1.5 * g.normal(rows, H * dh)).to(dt)
        s["out"] = torch.zeros(rows, H * dh, dtype=dt, device="cuda")
    return s


# --------------------------------------------------------------------------- plain form
def _rows(s):
    """Sequence and position of every row that belongs to one."""
    kv_len, nseq = s["kv_len"].long(), s["case"]["nseq"]
    if s["q_start"] is None:
        return torch.arange(nseq, device="cuda"), kv_len - 1
    start = s["q_start"].long()
    n = start[1:] - start[:-1]
    seq = torch.repeat_interleave(torch.arange(nseq, device="cuda"), n, output_size=sum(_lengths(s["case"])[0]))
    r = torch.arange(seq.numel(), device="cuda")
    return seq, kv_len[seq] - start[1:][seq] + r


def _rotate(x, pos, base):
    """x: rows x heads x dh in fp32; angles in 64 bits, their sine and cosine and the rotation in 32."""
    h = x.shape[-1] // 2
    theta = torch.exp2(torch.arange(h, device="cuda", dtype=torch.float64) * (-math.log2(base) / h))
    ang = (pos.double()[:, None] * theta)[:, None, :]
    cs, sn = torch.cos(ang).float(), torch.sin(ang).float()
    a, b = x[..., :h], x[..., h:]
    return torch.cat([a * cs - b * sn, b * cs + a * sn], -1)


def _append(s):
    c = s["case"]
    dt, dh, ps = DTYPES[c["dtype"]], c["dh"], c["page"]
    seq, pos = _rows(s)
    n = seq.numel()
    k = s["K"][:n].reshape(n, -1, dh).float()
    v = s["V"][:n].reshape(n, -1, dh).float()
    if c["rope"]:
        k = _rotate(k, pos, c["rope"])
        s["q_out"][:n] = _rotate(s["Q"][:n].reshape(n, -1, dh).float(), pos, c["rope"]).reshape(n, -1).to(dt)
    page = s["page_table"][seq, pos // ps].long()
    slot = pos % ps
    outs = [] if s["q_out"] is None else [s["q_out"]]
    if c["kind"] == "append":
        s["k_cache"][page, :, slot] = k.to(dt)
        s["v_cache"][page, :, slot] = v.to(dt)
        return outs + [s["k_cache"], s["v_cache"]]
    # The page that a sequence's first new row falls into may hold earlier tokens: slots below `old`.
    first = s["kv_len"].long() - (1 if s["q_start"] is None else (s["q_start"][1:] - s["q_start"][:-1]).long())
    fpage = s["page_table"][torch.arange(c["nseq"], device="cuda"), first // ps].long()
    old = first % ps
    return outs + _store8(s["k_cache"], s["k_scale"], k, page, slot, fpage, old) + _store8(
        s["v_cache"], s["v_scale"], v, page, slot, fpage, old)


def _store8(cache, scale, x, page, slot, fpage, old):
    pages, heads = scale.shape
    codes = cache.view(torch.uint8)
    # The smallest power of two s with amax <= 448 s.
    amax = torch.zeros(pages, heads, device="cuda").index_reduce_(0, page, x.abs().amax(-1), "amax")
    m, e = torch.frexp(amax)
    need = torch.ldexp(torch.ones_like(m), (e - 9 + (m > 0.875)).clamp(-126, 120))
    keeps = torch.zeros(pages, dtype=torch.bool, device="cuda")
    keeps[fpage] = old > 0
    touched = torch.zeros(pages, dtype=torch.bool, device="cuda")
    touched[page] = True
    after = torch.where(keeps[:, None], torch.maximum(scale, need), need)
    after = torch.where(touched[:, None], after, scale)
    held = codes[fpage].view(E4M3).float() * (scale / after)[fpage][..., None, None]
    stays = (torch.arange(cache.shape[2], device="cuda") < old[:, None])[:, None, :, None]
    codes[fpage] = torch.where(stays, held.to(E4M3).view(torch.uint8), codes[fpage])
    codes[page, :, slot] = (x / after[page][..., None]).to(E4M3).view(torch.uint8)
    scale.copy_(after)
    return [cache, scale]


def _gather(s, cache, scale, keys_last):
    """Every sequence's keys or values in 32 bits: nseq x kv_heads x length x dh, or x dh x length."""
    c = s["case"]
    table = s["page_table"].long().clamp(min=0)
    x = cache.view(torch.uint8)[table].view(E4M3) if scale is not None else cache[table]
    x = x.float() if scale is None else x.float() * scale[table][..., None, None]
    if keys_last:
        return x.permute(0, 2, 4, 1, 3).reshape(c["nseq"], c["kv_heads"], c["dh"], -1)
    return x.permute(0, 2, 1, 3, 4).reshape(c["nseq"], c["kv_heads"], -1, c["dh"])


def _attend(s):
    c = s["case"]
    dt, H, KV, dh, nseq, most = DTYPES[c["dtype"]], c["heads"], c["kv_heads"], c["dh"], c["nseq"], s["max_new"]
    seq, pos = _rows(s)
    n = seq.numel()
    start = torch.arange(nseq + 1, device="cuda") if s["q_start"] is None else s["q_start"].long()
    i = torch.arange(n, device="cuda") - start[seq]  # the row's place among its sequence's new rows
    q = torch.zeros(nseq, most, H, dh, device="cuda")
    q[seq, i] = s["Q"][:n].reshape(n, H, dh).float()
    p = torch.full((nseq, most), -1, device="cuda", dtype=torch.long)
    p[seq, i] = pos
    q = q.reshape(nseq, most, KV, H // KV, dh).permute(0, 2, 3, 1, 4).reshape(nseq, KV, -1, dh)
    x = torch.matmul(q, _gather(s, s["k_cache"], s["k_scale"], True)) / math.sqrt(dh)
    sees = torch.arange(x.shape[-1], device="cuda") <= p[..., None]
    x = x.reshape(nseq, KV, H // KV, most, -1).masked_fill_(~sees[:, None, None], -math.inf)
    x = x.sub_(x.amax(-1, keepdim=True).clamp(min=-3e38)).exp_()
    total = x.sum(-1, keepdim=True)
    v = _gather(s, s["v_cache"], s["v_scale"], False).masked_fill_(
        (torch.arange(x.shape[-1], device="cuda") >= s["kv_len"][:, None])[:, None, :, None], 0.0)
    o = torch.matmul(x.reshape(nseq, KV, -1, x.shape[-1]), v).reshape(nseq, KV, H // KV, most, dh)
    o = o / total.masked_fill(total == 0, 1.0)
    s["out"][:n] = o.permute(0, 3, 1, 2, 4).reshape(nseq, most, H * dh)[seq, i].to(dt)
    return s["out"]


def run(s):
    if own:
        from paper_2608_15665_amd import kv_append, paged_attention
        if s["case"]["kind"] in ("attend", "attend8"):
            return paged_attention(s["Q"], s["k_cache"], s["v_cache"], s["page_table"], s["kv_len"],
                                   q_start=s["q_start"], max_q=s["max_new"], k_scale=s["k_scale"],
                                   v_scale=s["v_scale"], out=s["out"])
        rope = s["case"]["rope"]
        kv_append(s["K"], s["V"], s["k_cache"], s["v_cache"], s["page_table"], s["kv_len"], q_start=s["q_start"],
                  max_q=s["max_new"], Q=s["Q"] if rope else None, q_out=s["q_out"], rope_base=rope or None,
                  k_scale=s["k_scale"], v_scale=s["v_scale"])
        outs = [] if s["q_out"] is None else [s["q_out"]]
        if s["k_scale"] is None:
            return outs + [s["k_cache"], s["v_cache"]]
        return outs + [s["k_cache"], s["k_scale"], s["v_cache"], s["v_scale"]]
    return _attend(s) if s["case"]["kind"] in ("attend", "attend8") else _append(s)


# --------------------------------------------------------------------------- work
def work(case):
    c = case
    H, KV, dh = c["heads"], c["kv_heads"], c["dh"]
    new, total = _lengths(c)
    rows = sum(new)
    tables = 4.0 * (c["nseq"] * (1 if c["new"] == 1 else 2) + sum(-(-t // c["page"]) for t in total))
    cell = 1 if c["kind"] in ("append8", "attend8") else 2
    if c["kind"] in ("attend", "attend8"):
        pairs = sum(n * t - n * (n - 1) // 2 for n, t in zip(new, total))
        scales = 8.0 * KV * sum(-(-t // c["page"]) for t in total) if cell == 1 else 0.0
        return dict(bytes=4.0 * rows * H * dh + 2.0 * cell * sum(total) * KV * dh + scales + tables,
                    flops=4.0 * dh * H * pairs)
    pages = sum(-(-t // c["page"]) - (t - n) // c["page"] for n, t in zip(new, total))
    turned = (H + KV) if c["rope"] else 0
    return dict(bytes=(4.0 * rows * H * dh if c["rope"] else 0.0) + 2.0 * rows * KV * dh * (2 + cell)
                + (16.0 * KV * pages if cell == 1 else 0.0) + tables,
                flops=3.0 * rows * turned * dh + (2.0 * rows * KV * dh * 2 if cell == 1 else 0.0))


# --------------------------------------------------------------------------- float64
def _nearest_e4m3(x):
    """Float64 values rounded to the nearest e4m3 value (4 significant bits, steps of 2^-9 at the least), ties to even."""
    step = torch.exp2(torch.floor(torch.log2(x.abs().clamp(min=2.0 ** -6))) - 3)
    return torch.round(x / step) * step


def _turn64(x, positions, base):
    """x: rows x heads x dh as complex numbers x[i] + j x[i + dh/2], turned by their angles."""
    dh = x.shape[-1]
    freq = torch.tensor([base ** (-2.0 * i / dh) for i in range(dh // 2)], dtype=torch.float64, device="cuda")
    ang = torch.tensor(positions, dtype=torch.float64, device="cuda")[:, None, None] * freq
    z = torch.complex(x[..., :dh // 2], x[..., dh // 2:]) * torch.polar(torch.ones_like(ang), ang)
    return torch.cat([z.real, z.imag], -1)


def _need64(amax):
    """Elementwise the smallest power of two s with amax <= 448 s."""
    s = torch.exp2(torch.ceil(torch.log2(amax.clamp(min=1e-300) / E4M3_MAX)))
    s = torch.where(amax > E4M3_MAX * s, 2 * s, s)
    s = torch.where(amax <= E4M3_MAX * s / 2, s / 2, s)
    return s.clamp(2.0 ** -126, 2.0 ** 120)


def exact(case, seed):
    c = dict(case)
    s = prepare(c, seed)
    H, KV, dh, ps = c["heads"], c["kv_heads"], c["dh"], c["page"]
    new, total = _lengths(c)
    table = s["page_table"].tolist()
    if c["kind"] in ("attend", "attend8"):
        out, r = s["out"].double(), 0
        for i, (n, t) in enumerate(zip(new, total)):
            pages = torch.tensor(table[i][:-(-t // ps)], device="cuda")
            held = []
            for cache, scale in ((s["k_cache"], s["k_scale"]), (s["v_cache"], s["v_scale"])):
                x = cache[pages].double() if scale is None else (
                    cache.view(torch.uint8)[pages].view(E4M3).double() * scale[pages].double()[:, :, None, None])
                held.append(x.transpose(0, 1).reshape(KV, -1, dh)[:, :t])
            future = torch.ones(n, t, dtype=torch.bool, device="cuda").triu(t - n + 1)
            for h in range(H):
                key, value = held[0][h // (H // KV)], held[1][h // (H // KV)]
                q = s["Q"][r:r + n, h * dh:(h + 1) * dh].double()
                w = torch.softmax((q @ key.t().contiguous() / math.sqrt(dh)).masked_fill(future, -math.inf), -1)
                out[r:r + n, h * dh:(h + 1) * dh] = w @ value
            r += n
        return out
    kc, vc = s["k_cache"].double(), s["v_cache"].double()
    scales = [None if x is None else x.double() for x in (s["k_scale"], s["v_scale"])]
    q_out = None if s["q_out"] is None else s["q_out"].double()
    r = 0
    for i, (n, t) in enumerate(zip(new, total)):
        k, v = (s[x][r:r + n].double().reshape(n, KV, dh) for x in ("K", "V"))
        places = list(range(t - n, t))
        if c["rope"]:
            k = _turn64(k, places, c["rope"])
            q_out[r:r + n] = _turn64(s["Q"][r:r + n].double().reshape(n, H, dh), places, c["rope"]).reshape(n, -1)
        for x, cache, scale in ((k, kc, scales[0]), (v, vc, scales[1])):
            for p in range(places[0] // ps, places[-1] // ps + 1):
                page, lo, hi = table[i][p], max(places[0], p * ps), min(t, (p + 1) * ps)
                mine = x[lo - places[0]:hi - places[0]].transpose(0, 1)
                if scale is None:
                    cache[page, :, lo - p * ps:hi - p * ps] = mine
                    continue
                to = _need64(mine.abs().amax((1, 2)))
                if lo > p * ps:
                    to = torch.maximum(to, scale[page])
                    kept = cache[page, :, :lo - p * ps]
                    cache[page, :, :lo - p * ps] = _nearest_e4m3(kept * (scale[page] / to)[:, None, None])
                cache[page, :, lo - p * ps:hi - p * ps] = _nearest_e4m3(mine / to[:, None, None])
                scale[page] = to
        r += n
    outs = [] if q_out is None else [q_out]
    if scales[0] is None:
        return outs + [kc, vc]
    return outs + [kc, scales[0], vc, scales[1]]
