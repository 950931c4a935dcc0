"""zo_kv_append into an 8-bit cache, its rotated queries: in the pages' launch (up to 1024 rows, counted as sequences times
max_q) and in one of their own."""
import numpy as np
import pytest
import torch

import paper_2608_15665_amd as zo
from _paged import DT, E4M3, batch, bits, dev, host64, rows16
from oracle import paged as op
from test_gpu_kv_append import check_rotated

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("inplace", [False, True])
@pytest.mark.parametrize("dt", ["bf16", "f16"])
@pytest.mark.parametrize("heads,kvh,dh", [(3, 1, 64), (10, 2, 128), (70, 1, 128)])
@pytest.mark.parametrize("lens,news,apart", [
    ([40, 16, 0, 65, 128, 7], [40, 1, 0, 50, 33, 7], False),
    ([3, 0, 20], [8, 4, 8], False),                          # rows before position 0
    ([700, 30, 0, 341, 90], [300, 30, 0, 341, 1], True),
    ([150, 9, 520], [400, 20, 17], True),                    # 250 rows of the first before position 0
])
def test_queries(lens, news, apart, heads, kvh, dh, dt, inplace):
    assert (len(news) * max(news) > 1024) == apart
    rng = np.random.default_rng(sum(lens) + dh)
    ps, base = 64, 1e4
    table, q_start, kv_len, pages = batch(rng, lens, news, ps)
    rows, n = int(q_start[-1]) + 3, int(q_start[-1])
    (Q, Qv), (K, _), (V, Vv) = (rows16(rng.standard_normal((rows, m * dh)), dt, 8) for m in (heads, kvh, kvh))
    was = bits(Q.contiguous())
    kc, vc = (torch.zeros((pages, kvh, ps, dh), device="cuda").to(E4M3) for _ in range(2))
    ks, vs = (torch.ones((pages, kvh), device="cuda") for _ in range(2))
    flag = torch.zeros(1, dtype=torch.int32, device="cuda")
    out = Q if inplace else torch.full((rows, heads * dh), 77.0, dtype=DT[dt], device="cuda")
    got = zo.kv_append(K, V, kc, vc, dev(table), dev(kv_len), q_start=dev(q_start), max_q=max(news), Q=Q, q_out=out,
                       rope_base=base, k_scale=ks, v_scale=vs, bad_flag=flag)
    assert int(flag) == 0
    go, gb = host64(got.contiguous()), bits(got.contiguous())
    if inplace:
        np.testing.assert_array_equal(gb[n:], was[n:])
    else:
        np.testing.assert_array_equal(go[n:], 77.0)
        np.testing.assert_array_equal(bits(Q.contiguous()), was)
    Q3 = Qv.reshape(rows, heads, dh)
    for s in range(len(lens)):
        for r, p in op.rows_of(s, q_start, kv_len):
            if p < 0:
                np.testing.assert_array_equal(gb[r], was[r])
            else:
                check_rotated(go[r].reshape(heads, dh), op.rotate(Q3[r], p, base), Q3[r], dh, dt)
    # the pages beside them: V's codes and scales, bitwise
    zero = [np.zeros((pages, kvh, ps, dh)) for _ in range(2)]
    ref, refs = op.kv_append(Vv.reshape(rows, kvh, dh), Vv.reshape(rows, kvh, dh), zero, table, q_start, kv_len, None,
                             [np.ones((pages, kvh)) for _ in range(2)])
    np.testing.assert_array_equal(host64(vc), ref[1])
    np.testing.assert_array_equal(host64(vs), refs[1])
