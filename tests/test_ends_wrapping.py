"""Sizes of the model's two ends that a C int would wrap to a legal one."""
import pytest
import torch

import paper_2608_15665_amd as zo
from paper_2608_15665_amd import _lib


@pytest.mark.parametrize("vocab", [5 - 2 ** 32, 5 - 2 ** 33, -1])
def test_a_vocabulary_below_zero(monkeypatch, vocab):
    monkeypatch.setattr(torch._C, "_cuda_getDevice", lambda: -1, raising=False)
    monkeypatch.setattr(_lib, "lib", lambda: pytest.fail("the call was made"))
    X, y = torch.zeros(8, 16), torch.zeros(8, dtype=torch.int32)
    with pytest.raises(ValueError, match="out of range"):
        zo.token_logprob(X, y, vocab=vocab)
    with pytest.raises(ValueError, match="out of range"):
        zo.token_logprob_backward(X, y, torch.zeros(8), torch.zeros(8), vocab=vocab)
