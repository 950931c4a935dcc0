"""zo_kv_append into 8-bit pages whose scale was set by somebody else and is no power of two: code = e4m3(x / scale), the
quotient rounded to fp32 before the code's own rounding (bitwise), so each value is within half a step of the exact one."""
import numpy as np
import pytest
import torch

import paper_2608_15665_amd as zo
from _paged import E4M3, batch, bits, dev, host64, rows16
from oracle import paged as op

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dt", ["bf16", "f16"])
@pytest.mark.parametrize("dh,ps,kvh", [(64, 16, 3), (128, 64, 2), (128, 256, 4)])
def test_scales_of_any_value(dh, ps, kvh, dt):
    """Pages that are partly filled keep their scale where it is large enough, and get a power of two where it is not;
    what lies in them is then rounded again to that one."""
    rng = np.random.default_rng(dh + ps)
    nseq = 24
    news = [int(x) for x in rng.integers(1, ps // 2, nseq)]
    lens = [n + ps // 2 for n in news]                       # every new row shares a page with earlier ones
    table, q_start, kv_len, pages = batch(rng, lens, news, ps)
    rows = int(q_start[-1])
    (K, Kv), (V, Vv) = (rows16(rng.standard_normal((rows, kvh * dh)), dt) for _ in range(2))
    K3, V3 = Kv.reshape(rows, kvh, dh), Vv.reshape(rows, kvh, dh)
    codes = [op.nearest_e4m3(rng.uniform(-440, 440, (pages, kvh, ps, dh))) for _ in range(2)]
    scales = [rng.uniform(0.001, 0.08, (pages, kvh)).astype(np.float32).astype(np.float64) for _ in range(2)]
    kc, vc = (dev(c, torch.float32).to(E4M3) for c in codes)
    ks, vs = (dev(s, torch.float32) for s in scales)
    zo.kv_append(K, V, kc, vc, dev(table), dev(kv_len), q_start=dev(q_start), max_q=max(news), k_scale=ks, v_scale=vs)
    ref, refs = op.kv_append(K3, V3, codes, table, q_start, kv_len, None, scales)
    kept = grown = 0
    for got, gs, r, rs, x, was in ((kc, ks, ref[0], refs[0], K3, scales[0]), (vc, vs, ref[1], refs[1], V3, scales[1])):
        np.testing.assert_array_equal(host64(gs), rs)
        g, want = host64(got), r.copy()
        for s in range(nseq):
            for row, p in op.rows_of(s, q_start, kv_len):
                page, slot = table[s, p // ps], p % ps
                to = rs[page].astype(np.float32)
                q = x[row].astype(np.float32) / to[:, None]
                want[page, :, slot] = op.nearest_e4m3(q.astype(np.float64))
                err = np.abs(g[page, :, slot] * rs[page][:, None] - x[row])
                half = np.maximum(2.0 ** -4 * np.abs(x[row]), 2.0 ** -10 * rs[page][:, None])
                assert np.all(err <= half * (1 + 2.0 ** -20))
            kept += int(np.sum(rs[table[s, 0]] == was[table[s, 0]]))
            grown += int(np.sum(rs[table[s, 0]] > was[table[s, 0]]))
        np.testing.assert_array_equal(g, want)
    assert kept > 5 and grown > 5


def test_a_border_between_two_codes():
    """Values halfway between two codes: their quotient by the scale is exact, and a tie goes to the even code.  Times the
    scale's rounded reciprocal 104 of these would be beside the border."""
    dh, ps = 64, 16
    scale = np.arange(33, 64, 2, dtype=np.float32) / 64
    n = len(scale)
    half = np.array([b * 2.0 ** sh * sign for b in range(17, 32, 2) for sh in range(-1, 3) for sign in (1, -1)])
    K, Kv = rows16(half * scale[:, None].astype(np.float64), "f16")
    np.testing.assert_array_equal(Kv, half * scale[:, None])  # in fp16 without a rounding
    kc = torch.zeros((n, 1, ps, dh), dtype=torch.float32, device="cuda").to(E4M3)
    vc = kc.clone()
    ks, vs = (dev(scale[:, None]) for _ in range(2))
    zo.kv_append(K, K, kc, vc, dev(np.arange(n, dtype=np.int32)[:, None]), dev(np.full(n, 2, np.int32)), k_scale=ks, v_scale=vs)
    want = np.broadcast_to(op.nearest_e4m3(half), (n, dh))
    for c, sc in ((kc, ks), (vc, vs)):
        np.testing.assert_array_equal(bits(sc), bits(dev(scale[:, None])))
        np.testing.assert_array_equal(host64(c)[:, 0, 1], want)
