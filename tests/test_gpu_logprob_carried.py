"""Log-probabilities of rows whose largest logits come late: what was summed before them is scaled to their power, in threads
that take many steps.  Logits are large, where that power's rounding is coarse and must not reach the sum."""
import numpy as np
import pytest
import torch

import paper_2608_15665_amd as zo
from _ends import NEAR, U32, host, i32, put, within
from oracle import ends

pytestmark = pytest.mark.gpu


# (rows, vocabulary, columns after which the pattern comes again): a wave a row, 256 threads, 1024, and rows in parts of 4000.
@pytest.mark.parametrize("rows,vocab,period", [(4200, 3000, 3000), (70, 20001, 20001), (70, 40001, 40001), (3, 140001, 4000)])
# (type, size of the logits, a step of the type there, scale): a step is at most a half after scaling.
@pytest.mark.parametrize("dt,base,step,scale", [("f32", 1e5, 2.0 ** -7, 1.0), ("f32", -1e5, 2.0 ** -7, 1.0), ("f32", 1e6, 2.0 ** -4, 1.0),
                                                ("f32", -1e6, 2.0 ** -4, 1.0), ("f32", 3e6, 2.0 ** -2, 0.7),
                                                ("f16", 30000.0, 16.0, 1.0 / 128), ("bf16", -30080.0, 128.0, 1.0 / 1024)])
def test_sums_carried_to_larger_logits(rows, vocab, period, dt, base, step, scale):
    """Two thirds of the columns hold one value, the later third 1 to 8 steps more."""
    x = np.full((rows, vocab), base)
    late = np.arange(vocab) % period >= 2 * period // 3
    x[:, late] += step * (1 + np.arange(rows) % 8)[:, None]
    X, v = put(x, dt)
    np.testing.assert_array_equal(v, x)
    labels = np.where(np.arange(rows) % 3 == 0, 0, vocab - 1)
    logp, lse = zo.token_logprob(X, i32(labels), scale=scale)
    s = float(np.float32(scale))
    want, want_lse = ends.token_logprob(v, labels, s)
    # As for other rows: terms exp(t) are six roundings off, weighted |t| averages at most log n; n / 64 + 16 additions; then
    # float64 and one rounding.
    total = (4 * (np.log(vocab) + 1) + 2 + vocab / 64 + 16) * U32
    within(host(logp), want, (total + U32 * np.abs(want)) * NEAR, "logp")
    within(host(lse), want_lse, (total + U32 * np.abs(want_lse)) * NEAR, "lse")
