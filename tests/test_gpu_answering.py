"""The paged cache in use: prompts in pieces and then token by token, appended and attended to in turn, against the
whole-sequence rotation and attention in float64; captured into graphs and replayed with other lengths and pages;
on a stream of its own; two sequences that share the pages of a prompt."""
import numpy as np
import pytest
import torch

import oracle
import paper_2608_15665_amd as zo
from _paged import DT, E4M3, bits, check_attention, dev, host64, rows16
from oracle import paged as op

pytestmark = pytest.mark.gpu
BASE = 1e4


class Layer:
    """A layer's cache and the sequences that use it, as a program keeps them."""

    def __init__(self, dt, cache, heads, kvh, dh, ps, nseq, width, seed=0):
        self.dt, self.heads, self.kvh, self.dh, self.ps = dt, heads, kvh, dh, ps
        self.rng = np.random.default_rng(seed)
        pages = nseq * width + 3
        self.table = self.rng.permutation(pages)[:nseq * width].reshape(nseq, width).astype(np.int32)
        shape = (pages, kvh, ps, dh)
        e8 = cache == "e4m3"
        nan = lambda: dev(np.full(shape, np.nan), torch.float32).to(E4M3 if e8 else DT[dt])  # noqa: E731
        self.k, self.v = nan(), nan()
        self.ks, self.vs = (torch.full((pages, kvh), float("nan"), device="cuda") for _ in range(2)) if e8 else (None, None)
        self.len = np.zeros(nseq, np.int32)
        self.flag = torch.zeros(1, dtype=torch.int32, device="cuda")
        self.hist = [[] for _ in range(nseq)]  # (q, k, v) of every position, as given

    def draw(self, news, rows=None):
        rows = sum(news) if rows is None else rows
        H, K, D = self.heads, self.kvh, self.dh
        qkv, val = rows16(self.rng.standard_normal((rows, (H + 2 * K) * D)), self.dt)
        r = 0
        for s, n in enumerate(news):
            for _ in range(n):
                x = val[r].reshape(-1, D)
                self.hist[s].append((x[:H], x[H:H + K], x[H + K:]))
                r += 1
        self.len = (self.len + np.array(news)).astype(np.int32)
        return qkv[:, :H * D], qkv[:, H * D:(H + K) * D], qkv[:, (H + K) * D:]

    def step(self, q, k, v, table, kv_len, q_start, max_q, q_rot, out):
        zo.kv_append(k, v, self.k, self.v, table, kv_len, q_start=q_start, max_q=max_q, Q=q, q_out=q_rot, rope_base=BASE,
                     k_scale=self.ks, v_scale=self.vs, bad_flag=self.flag)
        return zo.paged_attention(q_rot, self.k, self.v, table, kv_len, q_start=q_start, max_q=max_q, k_scale=self.ks,
                                  v_scale=self.vs, out=out, bad_flag=self.flag)

    def run(self, news):
        q, k, v = self.draw(news)
        q_start = dev(np.concatenate([[0], np.cumsum(news)]).astype(np.int32))
        out = torch.full((sum(news), self.heads * self.dh), float("nan"), dtype=DT[self.dt], device="cuda")
        self.step(q, k, v, dev(self.table), dev(self.len), q_start, max(news), torch.empty_like(out), out)
        return host64(out).reshape(-1, self.heads, self.dh)

    def want(self, news, table=None):
        """The last `news` rows of every sequence by whole-sequence attention on the rotated, rounded and stored keys and
        values."""
        table = self.table if table is None else table
        scl = None if self.ks is None else [host64(self.ks), host64(self.vs)]
        q = []
        for s, n in enumerate(news):
            for p in range(len(self.hist[s]) - n, len(self.hist[s])):
                x = op.rotate(self.hist[s][p][0], p, BASE)
                q.append(oracle.round_f16(x) if self.dt == "f16" else oracle.round_bf16(x))
        q_start = np.concatenate([[0], np.cumsum(news)])
        caches = [np.nan_to_num(host64(c)) for c in (self.k, self.v)]
        if scl:
            scl = [np.nan_to_num(x) for x in scl]
        return op.paged_attention(np.stack(q), caches, table, q_start, self.len, scl)


def loose(got, ref, mag, dt, what, cache="same"):
    """Half an ulp of the output; 2^-8 (bf16) or 2^-11 of softmax(S) |V| for P's single rounding where rows are many
    (fp16 rows of 8-bit caches: a pair, closer still); and the other side of Q's rounding, which the reference may take for a value next to a border: such
    a step of a q moves a logit by 2^-7 or 2^-10 of |q_i k_i| / sqrt(dh), together under 4 half steps of a weight."""
    assert np.all(np.isfinite(got)), what
    step = 2.0 ** -8 if dt == "bf16" else 2.0 ** -11
    assert bool(np.all(np.abs(got - ref) <= step * np.abs(ref) + 5 * step * mag)), what


@pytest.mark.parametrize("dt", ["bf16", "f16"])
@pytest.mark.parametrize("cache", ["same", "e4m3"])
@pytest.mark.parametrize("heads,kvh,dh,ps", [(10, 2, 128, 16), (3, 3, 64, 32)])
def test_prompts_in_pieces_and_then_token_by_token(dt, cache, heads, kvh, dh, ps):
    L = Layer(dt, cache, heads, kvh, dh, ps, 3, 16, seed=dh)
    for news in ([40, 1, 17], [30, 25, 0], [1, 1, 1], [1, 1, 1], [4, 2, 1], [1, 70, 33], [1, 1, 1]):
        got = L.run(news)
        ref, mag = L.want(news)
        loose(got, ref, mag, dt, news, cache)
    assert int(L.flag) == 0
    if cache == "same":
        # the cache holds the rotated keys and the values of every position, and the NaN of the start elsewhere
        used = np.zeros(L.k.shape[0::2], bool)
        for s in range(3):
            for p, (_, k, v) in enumerate(L.hist[s]):
                page, t = L.table[s, p // ps], p % ps
                used[page, t] = True
                np.testing.assert_array_equal(host64(L.v[page, :, t]), v)
                d = np.abs(host64(L.k[page, :, t]) - op.rotate(k, p, BASE))
                assert np.all(d <= 2.0 ** -8 * np.abs(op.rotate(k, p, BASE)) + 2.0 ** -18)
        for c in (L.k, L.v):
            h = host64(c).transpose(0, 2, 1, 3)
            assert np.all(np.isnan(h[~used])) and not np.any(np.isnan(h[used]))


@pytest.mark.parametrize("dt", ["bf16", "f16"])
def test_whole_sequences_agree_with_the_layer_kernels(dt):
    """From nothing in one piece: what zo.rope and zo.causal_attention of the whole sequences give, to rounding."""
    heads, kvh, dh, n, nseq = 8, 2, 128, 150, 2
    L = Layer(dt, "same", heads, kvh, dh, 64, nseq, 4, seed=7)
    q, k, v = L.draw([n] * nseq)
    out = torch.empty((nseq * n, heads * dh), dtype=DT[dt], device="cuda")
    q_rot = torch.empty_like(out)
    L.step(q, k, v, dev(L.table), dev(L.len), dev(np.array([0, n, 2 * n], np.int32)), n, q_rot, out)
    qr = zo.rope(q.contiguous(), n, heads, BASE)
    kr = zo.rope(k.contiguous(), n, kvh, BASE)
    whole = zo.causal_attention(qr, kr, v.contiguous(), 1, nseq * n, n, heads, kv_heads=kvh)
    assert np.mean(bits(q_rot) != bits(qr)) < 1e-3
    a, b = host64(out), host64(whole)
    assert np.linalg.norm(a - b) <= 2.0 ** -8 * np.linalg.norm(b)


@pytest.mark.parametrize("cache", ["same", "e4m3"])
def test_captured_steps(cache):
    """Two graphs of a padded batch's step (short and long tables, so that both split the keys), replayed in turn with
    new lengths, tables and rows, and with eager calls between them: each replay as the eager call gives it."""
    dt, heads, kvh, dh, ps, nseq = "bf16", 8, 2, 128, 16, 3
    width = 100
    mine = Layer(dt, cache, heads, kvh, dh, ps, nseq, width, seed=3)
    ref = Layer(dt, cache, heads, kvh, dh, ps, nseq, width, seed=3)
    mine.run([500, 90, 700]), ref.run([500, 90, 700])
    rows = nseq + 2
    D = (heads + 2 * kvh) * dh
    table, kv_len = dev(mine.table), dev(mine.len)

    def make():
        qkv = torch.zeros((rows, D), dtype=DT[dt], device="cuda")
        out, q_rot = (torch.zeros((rows, heads * dh), dtype=DT[dt], device="cuda") for _ in range(2))
        cut = lambda: (qkv[:, :heads * dh], qkv[:, heads * dh:(heads + kvh) * dh], qkv[:, (heads + kvh) * dh:])  # noqa: E731
        g = torch.cuda.CUDAGraph()
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.graph(g, stream=side):
            mine.step(*cut(), table, kv_len, None, 1, q_rot, out)
        return qkv, out, g

    graphs = [make(), make()]
    junk = Layer(dt, "same", 4, 4, 64, 16, 1, 300, seed=9)  # its calls grow the stream's own workspace
    for i in range(8):
        qkv, out, g = graphs[i % 2]
        q, k, v = ref.draw([1] * nseq, rows)
        qkv.copy_(torch.cat([q, k, v], 1))
        kv_len.copy_(dev(ref.len))
        out.fill_(7.0)
        g.replay()
        o = torch.full_like(out, 7.0)
        ref.step(q, k, v, dev(ref.table), dev(ref.len), None, 1, torch.empty_like(o), o)
        if i == 4:
            junk.run([4000])
        torch.cuda.synchronize()
        np.testing.assert_array_equal(bits(out), bits(o))
        assert np.all(host64(out)[nseq:] == 7.0)
    for a, b in ((mine.k, ref.k), (mine.v, ref.v)):
        np.testing.assert_array_equal(bits(a), bits(b))


def test_on_another_stream():
    """A step on a stream that is not the tensors' own, beside one on the default stream."""
    A, B = (Layer("f16", "same", 6, 2, 64, 32, 2, 60, seed=s) for s in (1, 2))
    A.run([900, 5]), B.run([1500, 300])
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    for _ in range(3):
        with torch.cuda.stream(side):
            a = A.run([1, 2])
        b = B.run([3, 1])
        side.synchronize()
        loose(a, *A.want([1, 2]), "f16", "side")
        loose(b, *B.want([3, 1]), "f16", "own")


def test_shared_prompt_pages():
    """Several continuations of one prompt: their tables name the prompt's whole pages, which are read only, and pages
    of their own behind them."""
    dt, heads, kvh, dh, ps = "bf16", 4, 2, 128, 16
    L = Layer(dt, "e4m3", heads, kvh, dh, ps, 4, 6, seed=11)
    L.run([48, 0, 0, 0])
    prompt = L.hist[0]
    L.table[1:, :3] = L.table[0, :3]
    for s in (1, 2, 3):
        L.hist[s] = list(prompt)
    L.len[:] = 48
    before = bits(L.k[L.table[0, :3].astype(np.int64)]).copy()
    for news in ([3, 1, 2, 5], [1, 1, 1, 1]):
        got = L.run(news)
        loose(got, *L.want(news), dt, news, "e4m3")
    np.testing.assert_array_equal(bits(L.k[L.table[0, :3].astype(np.int64)]), before)


def test_drafts_taken_back():
    """Drafted tokens that are not kept: the next step writes over their slots."""
    L = Layer("bf16", "same", 4, 4, 64, 16, 2, 8, seed=12)
    L.run([20, 33])
    L.run([4, 4])
    for s, keep in enumerate((1, 3)):
        L.hist[s] = L.hist[s][:len(L.hist[s]) - 4 + keep]
        L.len[s] = len(L.hist[s])
    got = L.run([1, 1])
    loose(got, *L.want([1, 1]), "bf16", "after")


def test_positions_beyond_2_31_bytes():
    """A cache of more than 4 GiB: pages at its far end."""
    dh, ps, kvh = 128, 64, 8
    pages = (5 << 30) // (kvh * ps * dh * 2)
    k, v = (torch.empty((pages, kvh, ps, dh), dtype=torch.float16, device="cuda") for _ in range(2))
    rng = np.random.default_rng(2)
    table = np.array([[pages - 1, 0, pages - 2, pages // 2, 1]], np.int32)
    n = 300
    (K, Kv), (V, Vv), (Q, Qv) = (rows16(rng.standard_normal((n, h * dh)), "f16") for h in (kvh, kvh, 8))
    zo.kv_append(K, V, k, v, dev(table), dev(np.array([n], np.int32)), q_start=dev(np.array([0, n], np.int32)), max_q=n)
    for rows in (1, n):  # the last row alone, and all
        out = zo.paged_attention(Q[n - rows:], k, v, dev(table), dev(np.array([n], np.int32)),
                                 q_start=dev(np.array([0, rows], np.int32)), max_q=rows)
        small = [x.reshape(n, kvh, dh).transpose(1, 0, 2)[None] for x in (Kv, Vv)]
        pad = [np.concatenate([x, np.zeros((1, kvh, 320 - n, dh))], 2).reshape(1, kvh, 5, ps, dh)[0].transpose(1, 0, 2, 3) for x in small]
        ref, mag = op.paged_attention(Qv.reshape(n, 8, dh)[n - rows:], pad, np.arange(5)[None], np.array([0, rows]), np.array([n]))
        check_attention(host64(out).reshape(rows, 8, dh), ref, mag, "f16", rows, many=rows > 16)


def test_python_refusals():
    k = torch.zeros((4, 2, 16, 64), dtype=torch.bfloat16, device="cuda")
    tab, n = dev(np.zeros((1, 4), np.int32)), dev(np.ones(1, np.int32))
    row = torch.zeros((1, 128), dtype=torch.bfloat16, device="cuda")
    ok = dict(k_cache=k, v_cache=k.clone(), page_table=tab, kv_len=n)
    scale = torch.ones((4, 2), device="cuda")
    for exc, kw in [(ValueError, dict(k_cache=k[0])), (ValueError, dict(v_cache=k[:2])), (TypeError, dict(k_cache=k.half(), v_cache=k.half())),
                    (ValueError, dict(k_scale=scale)), (ValueError, dict(page_table=tab[0])), (ValueError, dict(page_table=tab.cpu())),
                    (TypeError, dict(page_table=tab.long())), (ValueError, dict(kv_len=dev(np.ones(2, np.int32)))),
                    (ValueError, dict(q_start=n)), (ValueError, dict(k_cache=k.transpose(0, 1), v_cache=k.transpose(0, 1))),
                    (ValueError, dict(bad_flag=dev(np.zeros(2, np.int32)))),
                    (ValueError, dict(k_cache=k.to(E4M3), v_cache=k.to(E4M3), k_scale=scale)),
                    (ValueError, dict(k_cache=k.to(E4M3), v_cache=k.to(E4M3), k_scale=scale, v_scale=scale[:2])),
                    (TypeError, dict(k_cache=k.to(E4M3), v_cache=k.to(E4M3), k_scale=scale.half(), v_scale=scale))]:
        for call in (lambda **a: zo.kv_append(row, row, **a), lambda **a: zo.paged_attention(row, **a)):
            with pytest.raises(exc):
                call(**{**ok, **kw})
    for exc, a, kw in [(ValueError, (row[:, :64], row), {}), (ValueError, (row, row.t()), {}), (TypeError, (row, row.float()), {}),
                       (TypeError, (row.float(), row.float()), {}), (ValueError, (row, row), dict(q_out=row)),
                       (ValueError, (row, row), dict(Q=row[:, :72])), (zo.ZoError, (row, row), dict(Q=row.clone())),
                       (zo.ZoError, (row, row), dict(rope_base=0.5)), (ValueError, (row.cpu(), row), {})]:
        with pytest.raises(exc):
            zo.kv_append(*a, **{**ok, **kw})
    for exc, q, kw in [(ValueError, row[:, :72], {}), (zo.ZoError, row[:, :64].contiguous(), {}), (ValueError, row, dict(out=row[:, :64])),
                       (TypeError, row, dict(workspace=row))]:
        with pytest.raises(exc):
            zo.paged_attention(q, **{**ok, **kw})
    with pytest.raises(zo.ZoError, match="workspace"):
        zo.paged_attention(row, **{**ok, "page_table": dev(np.zeros((1, 900), np.int32))},
                           workspace=torch.empty(16, dtype=torch.uint8, device="cuda"))
