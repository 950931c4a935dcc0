"""Calls of 2^24 workgroups and more, which is what many sequences ask for without max_q (all rows): a grid's x dimension
holds fewer than 2^32 threads.  Almost all of these workgroups find nothing to do; what the others do is what a call
with a near max_q does, bit by bit."""
import numpy as np
import pytest
import torch

import paper_2608_15665_amd as zo
from _paged import DT, E4M3, batch, bits, dev, rows16

pytestmark = pytest.mark.gpu
NSEQ = 4100


def _batch(rng, ps):
    news = [int(x) for x in rng.integers(0, 3, NSEQ)]
    news[7], news[4000] = 50, 37
    lens = [n + int(c) for n, c in zip(news, rng.integers(0, 9, NSEQ))]
    table, q_start, kv_len, pages = batch(rng, lens, news, ps)
    assert NSEQ * int(q_start[-1]) >= 1 << 24
    return dev(table), dev(q_start), dev(kv_len), pages, int(q_start[-1]), max(news)


@pytest.mark.parametrize("cache", ["same", "e4m3"])
def test_append(cache):
    rng, dh, ps, kvh, heads = np.random.default_rng(1), 64, 32, 2, 3
    table, q_start, kv_len, pages, rows, most = _batch(rng, ps)
    K, V, Q = (rows16(rng.standard_normal((rows, n * dh)), "bf16")[0] for n in (kvh, kvh, heads))
    outs = []
    for max_q in (most, None):
        kc = torch.zeros((pages, kvh, ps, dh), device="cuda").to(E4M3 if cache == "e4m3" else DT["bf16"])
        vc = kc.clone()
        ks, vs = (torch.ones((pages, kvh), device="cuda") for _ in range(2)) if cache == "e4m3" else (None, None)
        flag = torch.zeros(1, dtype=torch.int32, device="cuda")
        q = zo.kv_append(K, V, kc, vc, table, kv_len, q_start=q_start, max_q=max_q, Q=Q, rope_base=1e4, k_scale=ks,
                         v_scale=vs, bad_flag=flag)
        torch.cuda.synchronize()
        assert int(flag) == 0
        outs.append([bits(t) for t in (q, kc, vc, ks, vs) if t is not None])
    for a, b in zip(*outs):
        np.testing.assert_array_equal(a, b)
    assert np.count_nonzero(outs[0][1]) > 0


@pytest.mark.parametrize("kvh", [4, 8])
@pytest.mark.parametrize("cache", ["same", "e4m3"])
def test_attention(cache, kvh):
    rng, dh, ps, group = np.random.default_rng(2), 64, 32, 32
    table, q_start, kv_len, pages, rows, most = _batch(rng, ps)
    assert NSEQ * kvh * (rows * group // 128) >= 1 << 24
    Q, _ = rows16(rng.standard_normal((rows, kvh * group * dh)), "bf16")
    e8 = cache == "e4m3"
    kc, vc = (dev(rng.standard_normal((pages, kvh, ps, dh)), torch.float32).to(E4M3 if e8 else DT["bf16"]) for _ in range(2))
    ks, vs = (torch.ones((pages, kvh), device="cuda") for _ in range(2)) if e8 else (None, None)
    outs = []
    for max_q in (most, None):
        out = torch.full_like(Q, 7.0)
        flag = torch.zeros(1, dtype=torch.int32, device="cuda")
        zo.paged_attention(Q, kc, vc, table, kv_len, q_start=q_start, max_q=max_q, k_scale=ks, v_scale=vs, out=out,
                           bad_flag=flag)
        torch.cuda.synchronize()
        assert int(flag) == 0 and bool(torch.isfinite(out).all())
        outs.append(out)
    assert torch.equal(*outs)


def test_attention_of_single_tokens():
    """2^24 + 32 (sequence, key head) pairs: each sequence has the one key of its page."""
    nseq, heads, dh, ps, pages = (1 << 19) + 1, 32, 64, 16, 97
    g = torch.Generator(device="cuda")
    g.manual_seed(3)
    Q = torch.randn(nseq, heads * dh, generator=g, device="cuda", dtype=DT["bf16"])
    kc, vc = (torch.randn(pages, heads, ps, dh, generator=g, device="cuda", dtype=DT["bf16"]) for _ in range(2))
    page = torch.randint(0, pages, (nseq, 1), generator=g, device="cuda", dtype=torch.int32)
    out = zo.paged_attention(Q, kc, vc, page, torch.ones(nseq, dtype=torch.int32, device="cuda"))
    torch.cuda.synchronize()
    want = vc[:, :, 0].reshape(pages, heads * dh)[page[:, 0].long()]
    assert torch.equal(out, want)
