"""What the binding of the paged cache takes and refuses before a call, on host tensors (their device number stands for the
current device)."""
import pytest
import torch

from paper_2608_15665_amd import _lib


class _Library:
    def __init__(self, need=4096):
        self.need, self.calls = need, []

    def zo_paged_attention_workspace(self, *a):
        return self.need

    def zo_paged_attention(self, *a):
        self.calls.append(a)
        return 0

    def zo_kv_append(self, *a):
        self.calls.append(a)
        return 0


class _Elsewhere(torch.Tensor):
    """A tensor of another GPU."""

    @property
    def device(self):
        return torch.device("cuda", 1)

    def get_device(self):
        return 1


@pytest.fixture
def fake(monkeypatch):
    lib = _Library()
    monkeypatch.setattr(torch._C, "_cuda_getDevice", lambda: -1, raising=False)
    monkeypatch.setattr(torch.cuda, "is_current_stream_capturing", lambda: False)
    monkeypatch.setattr(_lib, "_stream_handle", lambda: 0)
    monkeypatch.setattr(_lib, "lib", lambda: lib)
    return lib


def _cache():
    cache = torch.zeros(4, 2, 16, 64, dtype=torch.bfloat16)
    return dict(k_cache=cache, v_cache=cache.clone(), page_table=torch.zeros(1, 4, dtype=torch.int32),
                kv_len=torch.ones(1, dtype=torch.int32))


def test_a_workspace_of_another_device_is_refused(fake):
    ws = torch.empty(8192, dtype=torch.uint8).as_subclass(_Elsewhere)
    assert ws.is_contiguous() and ws.device.type == "cuda"
    with pytest.raises(ValueError, match="workspace must live on the current device"):
        _lib.paged_attention(torch.zeros(1, 128, dtype=torch.bfloat16), **_cache(), workspace=ws)
    assert not fake.calls


@pytest.mark.parametrize("wide", [128, 130, 133, 136])
def test_one_row_has_no_distance(fake, wide):
    """A single row may come from a tensor of any width (its start on 16 bytes): the library's multiple of 8 between
    rows has nothing to be between."""
    row = torch.zeros(1, wide, dtype=torch.bfloat16)[:, :128]
    _lib.kv_append(row, row.clone(), **_cache(), Q=row, q_out=row, rope_base=1e4)
    ldq, ldqo, ldk, ldv = (fake.calls[-1][i] for i in (5, 7, 9, 11))
    assert ldq == ldqo and all(x % 8 == 0 and x >= 128 for x in (ldq, ldk, ldv))
    fake.need = 0
    _lib.paged_attention(row, **_cache(), out=row)
    assert fake.calls[-1][5] == fake.calls[-1][7] and fake.calls[-1][5] % 8 == 0
    two = torch.zeros(2, wide, dtype=torch.bfloat16)[:, :128]
    _lib.kv_append(two, two, **_cache(), max_q=1)
    assert fake.calls[-1][9] == wide  # refused by the library where it is no multiple of 8
