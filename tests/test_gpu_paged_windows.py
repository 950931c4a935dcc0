"""zo_paged_attention where one workgroup walks thousands of keys: page numbers (and an 8-bit cache's scales) come in
windows of 1024 keys, and every window after the first has to be the right one.

A call splits a sequence's keys over workgroups unless it has 512 (sequence, key head) pairs; here most of its
sequences are short, and two walk three and four windows.  Every output is within half an ulp + 2^-14
softmax(S) |V|: a key lost or taken twice of n moves it by |v| / n, four times as much at 3500 keys."""
import numpy as np
import pytest
import torch

import paper_2608_15665_amd as zo
from _paged import DT, E4M3, attend, batch, check_attention, dev, host64, rows16

pytestmark = pytest.mark.gpu


def crowd(rng, long, news, kvh):
    """Lengths and rows: the long sequences at odd places among enough short ones for 512 pairs."""
    n = -(-512 // kvh) + 3
    lens, new = [int(x) for x in rng.integers(1, 40, n)], [1] * n
    for i, (t, m) in enumerate(zip(long, news)):
        lens[(5 + 37 * i) % n], new[(5 + 37 * i) % n] = t, m
    return lens, new


@pytest.mark.parametrize("cache", ["same", "e4m3"])
@pytest.mark.parametrize("dt", ["bf16", "f16"])
@pytest.mark.parametrize("heads,kvh,dh,ps", [(2, 1, 64, 16), (5, 1, 128, 16), (8, 4, 128, 64), (8, 4, 64, 256)])
@pytest.mark.parametrize("long,news", [
    ([3500, 2049], [1, 1]),
    ([1024, 1025, 2047], [1, 1, 1]),
    ([3000, 2100], [4, 2]),
    ([3333, 2048], [40, 17]),
    ([1100, 2300], [100, 150]),
])
def test_windows(long, news, heads, kvh, dh, ps, dt, cache):
    rng = np.random.default_rng(sum(long) + dh + kvh)
    lens, new = crowd(rng, long, news, kvh)
    got, ref, mag = attend(rng, dt, lens, new, ps, heads, kvh, dh, cache, spread=0.3)
    check_attention(got, ref, mag, dt, (long, news))


@pytest.mark.parametrize("cache", ["same", "e4m3"])
@pytest.mark.parametrize("dh", [64, 128])
@pytest.mark.parametrize("rows", [8, 40])
@pytest.mark.parametrize("where", [900, 1024, 2080, 2600])
def test_a_bad_page_in_any_window(where, rows, dh, cache):
    """Rows from the bad page's first position on are NaN, those before it as ever, and the flag is raised."""
    rng = np.random.default_rng(where)
    ps, heads = 16, 2
    first = where // ps * ps                 # the bad page's first position
    length = first + rows // 2
    lens, new = crowd(rng, [length], [rows], 1)
    s = 5
    table, q_start, kv_len, pages = batch(rng, lens, new, ps)
    table[s, first // ps] = pages + 3
    e8 = cache == "e4m3"
    pool = [rng.standard_normal((pages, 1, ps, dh)) for _ in range(2)]
    kc, vc = (dev(p, torch.float32).to(E4M3 if e8 else DT["bf16"]) for p in pool)
    scl = [2.0 ** rng.integers(-3, 3, (pages, 1)) for _ in range(2)] if e8 else None
    sd = [dev(x, torch.float32) for x in scl] if e8 else [None, None]
    Q, Qv = rows16(rng.standard_normal((sum(new), heads * dh)) * 0.3, "bf16")
    flag = torch.zeros(1, dtype=torch.int32, device="cuda")
    got = host64(zo.paged_attention(Q, kc, vc, dev(table), dev(kv_len), q_start=dev(q_start), max_q=rows, k_scale=sd[0],
                                    v_scale=sd[1], bad_flag=flag)).reshape(-1, heads, dh)
    assert int(flag) == 1
    r0 = int(q_start[s])
    sees = np.arange(length - rows, length) >= first
    assert np.all(np.isnan(got[r0:r0 + rows][sees]))
    from oracle import paged as op
    table[s, first // ps] = 0
    ref, mag = op.paged_attention(Qv.reshape(-1, heads, dh), [host64(kc), host64(vc)], table, q_start, kv_len, scl)
    keep = np.ones(len(got), bool)
    keep[r0:r0 + rows] = ~sees
    check_attention(got[keep], ref[keep], mag[keep], "bf16", (where, rows))
