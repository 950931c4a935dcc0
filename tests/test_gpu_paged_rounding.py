"""zo_paged_attention holds its weights as a hi + lo pair wherever a row goes: many rows of a sequence, or a maximum
of rows (max_q) that the batch does not reach, leave an output as near the exact one as a token alone is.

The bound is check_attention's for few rows: half an ulp of the output + 2^-14 softmax(S) |V|, 64 (bf16) or 8 (fp16)
times below a weight's single rounding, and below the weight of one key of some thousands."""
import numpy as np
import pytest
import torch

import paper_2608_15665_amd as zo
from _paged import DT, attend, batch, bits, check_attention, dev, rows16

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
