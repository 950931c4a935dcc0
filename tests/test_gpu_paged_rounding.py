"""zo_paged_attention holds its weights as a hi + lo pair wherever a row goes: many rows of a sequence, or a maximum
of rows (max_q) that the batch does not reach, leave an output as near the exact one as a token alone is.

The bound is check_attention's for few rows: half an ulp of the output + 2^-14 softmax(S) |V|, 64 (bf16) or 8 (fp16)
times below a weight's single rounding, and below the weight of one key of some thousands."""
import numpy as np
import pytest
import torch

import paper_2608_15665_amd as zo
from _paged import DT, attend, batch, bits, check_attention, dev, host64, rows16
from oracle import paged as op

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("cache", ["same", "e4m3"])
@pytest.mark.parametrize("dt", ["bf16", "f16"])
@pytest.mark.parametrize("heads,kvh,dh", [(4, 4, 128), (10, 2, 128), (7, 1, 64), (24, 1, 128), (8, 8, 64)])
@pytest.mark.parametrize("news,lens,ps", [
    ([40, 1, 0, 33], [40, 700, 0, 333], 16),     # a token beside pieces
    ([100, 3], [1150, 290], 64),
    ([129, 64], [129, 2000], 256),
    ([70, 8, 9], [64, 0, 20], 32),               # rows before position 0
])
def test_many_rows_are_as_exact_as_few(news, lens, ps, heads, kvh, dh, dt, cache):
    rng = np.random.default_rng(sum(lens) + heads)
    got, ref, mag = attend(rng, dt, lens, news, ps, heads, kvh, dh, cache, rows_behind=1)
    check_attention(got, ref, mag, dt, (news, heads, kvh))


@pytest.mark.parametrize("cache", ["same", "e4m3"])
@pytest.mark.parametrize("dt", ["bf16", "f16"])
@pytest.mark.parametrize("max_q", [1, 3, 40, 1000])
def test_a_token_is_as_exact_with_any_max_q(max_q, dt, cache):
    lens = [1, 17, 64, 65, 300, 900]
    rng = np.random.default_rng(max_q)
    got, ref, mag = attend(rng, dt, lens, [1] * 6, 32, 10, 2, 128, cache, max_q=max_q)
    check_attention(got, ref, mag, dt, max_q)


@pytest.mark.parametrize("cache", ["same", "e4m3"])
@pytest.mark.parametrize("news,lens,width", [([300, 40], [1700, 900], 0), ([1, 1], [3000, 70], 0), ([9, 2], [2500, 70], 300)])
def test_equal_calls_give_equal_bits(news, lens, width, cache):
    heads, kvh, dh, ps = 10, 2, 128, 32
    rng = np.random.default_rng(news[0])
    table, q_start, kv_len, pages = batch(rng, lens, news, ps, width=width)
    Q, _ = rows16(rng.standard_normal((sum(news), heads * dh)), "bf16")
    kc, vc = (dev(rng.standard_normal((pages, kvh, ps, dh)), torch.float32) for _ in range(2))
    ks = vs = None
    if cache == "e4m3":
        kc, vc = kc.to(torch.float8_e4m3fn), vc.to(torch.float8_e4m3fn)
        ks, vs = (dev(rng.uniform(0.1, 2.0, (pages, kvh)), torch.float32) for _ in range(2))
    else:
        kc, vc = kc.to(DT["bf16"]), vc.to(DT["bf16"])
    call = lambda: bits(zo.paged_attention(Q, kc, vc, dev(table), dev(kv_len), q_start=dev(q_start), max_q=max(news),  # noqa: E731
                                           k_scale=ks, v_scale=vs))
    first = call()
    for _ in range(5):
        np.testing.assert_array_equal(call(), first)


@pytest.mark.parametrize("dt", ["bf16", "f16"])
@pytest.mark.parametrize("news,heads,n", [([70], 1, 500), ([40], 3, 1000), ([200], 2, 3000), ([3], 2, 500)])
def test_an_infinity_among_earlier_values(news, heads, n, dt):
    """In a tile that every row sees, and with a weight that has no low part (equal logits: all weights are powers of
    two where 2^i keys tie, and 1 of the running maximum): the pair's product is the infinity, of its sign, not a NaN."""
    rng = np.random.default_rng(n)
    dh = 64
    for q, where in ((rng.standard_normal((news[0], heads * dh)), 100), (np.zeros((news[0], heads * dh)), 3)):
        v = rng.standard_normal((1, n, dh))
        table, q_start, kv_len, pages = batch(rng, [n], news, 16)
        Q, Qv = rows16(q, dt)
        pool = [np.zeros((pages, 1, 16, dh)) for _ in range(2)]
        k = rng.standard_normal((1, n, dh))
        k[0, where] *= 2.0
        v[0, where, 5], v[0, where + 1, 9], v[0, where + 64, 20], v[0, where + 65, 21] = np.inf, -np.inf, np.nan, np.inf
        for t in range(n):
            pool[0][table[0, t // 16], :, t % 16] = k[:, t]
            pool[1][table[0, t // 16], :, t % 16] = v[:, t]
        kd, vd = (dev(x, DT[dt]) for x in pool)
        got = host64(zo.paged_attention(Q, kd, vd, dev(table), dev(kv_len), q_start=dev(q_start), max_q=news[0]))
        got = got.reshape(news[0], heads, dh)
        held = [np.where(np.isfinite(host64(x)), host64(x), 0.0) for x in (kd, vd)]
        ref, mag = op.paged_attention(Qv.reshape(news[0], heads, dh), held, table, q_start, kv_len)
        assert np.all(got[..., [5, 21]] == np.inf) and np.all(got[..., 9] == -np.inf) and np.all(np.isnan(got[..., 20]))
        rest = [d for d in range(dh) if d not in (5, 9, 20, 21)]
        check_attention(got[..., rest], ref[..., rest], mag[..., rest], dt, (n, where))
