"""Labels that the vocabulary lacks, in every launch of the label log-probabilities and in the logits' gradient."""
import numpy as np
import pytest
import torch

import paper_2608_15665_amd as zo
from _ends import DT, bits, i32

pytestmark = pytest.mark.gpu


# A wave, 256 and 1024 threads a row, and split rows with their join.
@pytest.mark.parametrize("rows,vocab,ld", [(4200, 1001, 1008), (70, 20001, 20008), (70, 60001, 60001), (5, 140001, 140008)])
@pytest.mark.parametrize("dt", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("nblk", [1, 3])
def test_labels_that_the_vocabulary_lacks(rows, vocab, ld, dt, nblk):
    """Their rows are NaN and flagged, their log-sums and all other rows as with labels that it has; the padded columns, NaN, are
    not read."""
    g = torch.Generator(device="cuda").manual_seed(rows)
    X = torch.full((nblk * rows, ld), float("nan"), device="cuda").to(DT[dt])
    X[:, :vocab] = torch.randn(nblk * rows, vocab, generator=g, device="cuda").to(DT[dt])
    labels = np.random.default_rng(rows).integers(-2, vocab, rows)
    labels[0] = 5
    bad = np.zeros(rows, bool)
    bad[1::2] = True
    broken = labels.copy()
    broken[bad] = np.resize([vocab, ld, 2 ** 31 - 1], bad.sum())
    labels[bad] = 0  # in their place: the same log-sums
    flag = torch.zeros(1, dtype=torch.int32, device="cuda")
    want, want_lse = zo.token_logprob(X, i32(labels), vocab=vocab, bad_flag=flag)
    assert flag.item() == 0
    logp, lse = zo.token_logprob(X, i32(broken), vocab=vocab, bad_flag=flag)
    assert flag.item() == 1
    lost = np.tile(bad, nblk)
    assert np.isnan(logp.cpu().numpy()[lost]).all()
    np.testing.assert_array_equal(bits(logp)[~lost], bits(want)[~lost])
    np.testing.assert_array_equal(bits(lse), bits(want_lse))
    up = torch.randn(nblk * rows, generator=g, device="cuda")
    flag.zero_()
    for kept in (None, want):
        good = zo.token_logprob_backward(X, i32(labels), lse, up, vocab=vocab, logp=kept, bad_flag=flag)
        assert flag.item() == 0
        dX = zo.token_logprob_backward(X, i32(broken), lse, up, vocab=vocab, logp=kept, bad_flag=flag)
        assert flag.item() == 1 and dX[torch.from_numpy(lost).cuda(), :vocab].isnan().all()
        flag.zero_()
        np.testing.assert_array_equal(bits(dX)[~lost], bits(good)[~lost])
        assert (dX[:, vocab:] == 0).all()
    # Without a flag: the same.
    np.testing.assert_array_equal(bits(zo.token_logprob(X, i32(broken), vocab=vocab)[0]), bits(logp))
