"""zo_kv_append into 8-bit pages at the number of rows from which two waves share a page, and around it (16 rows of heads of
128, 32 of 64), with one key head and several: every row of every head once, as a single wave stores it."""
import numpy as np
import pytest
import torch

import paper_2608_15665_amd as zo
from _paged import E4M3, batch, dev, host64, rows16
from oracle import paged as op

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("ps", [32, 64, 256])
@pytest.mark.parametrize("kvh", [1, 3, 4])
@pytest.mark.parametrize("dh,rows", [(128, 16), (128, 17), (128, 70), (64, 32), (64, 33), (64, 130)])
def test_rows_of_a_page(rows, dh, kvh, ps):
    rng = np.random.default_rng(rows + kvh)
    news = [rows, 1, 0, rows - 1, 5]
    lens = [rows + 7, 40, 0, rows - 1, 3 + ps]
    table, q_start, kv_len, pages = batch(rng, lens, news, ps)
    n = int(q_start[-1])
    (K, Kv), (V, Vv) = (rows16(rng.standard_normal((n + 1, kvh * dh)) * g, "bf16", 8) for g in (1.0, 7.0))
    codes = [op.nearest_e4m3(rng.uniform(-400, 400, (pages, kvh, ps, dh))) for _ in range(2)]
    scales = [2.0 ** rng.integers(-12, -4, (pages, kvh)) for _ in range(2)]
    kc, vc = (dev(c, torch.float32).to(E4M3) for c in codes)
    ks, vs = (dev(s, torch.float32) for s in scales)
    flag = torch.zeros(1, dtype=torch.int32, device="cuda")
    zo.kv_append(K, V, kc, vc, dev(table), dev(kv_len), q_start=dev(q_start), max_q=rows, k_scale=ks, v_scale=vs,
                 bad_flag=flag)
    assert int(flag) == 0
    ref, refs = op.kv_append(Kv.reshape(-1, kvh, dh), Vv.reshape(-1, kvh, dh), codes, table, q_start, kv_len, None, scales)
    for got, want in ((kc, ref[0]), (vc, ref[1]), (ks, refs[0]), (vs, refs[1])):
        np.testing.assert_array_equal(host64(got), want)
