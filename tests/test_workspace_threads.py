"""Scratch memory of the binding where two threads call on one stream (torch's default stream is every thread's): a call
may be several launches, and those of two calls may be enqueued in turn, so no two threads share a buffer."""
import gc
import threading
import weakref

import pytest
import torch

from paper_2608_15665_amd import _lib


class _Library:
    """Stands for the library: each attention call waits until both threads are in theirs."""

    def __init__(self):
        self.both, self.seen = threading.Barrier(2, timeout=30), []

    def zo_paged_attention_workspace(self, *a):
        return 4096

    def zo_paged_attention(self, *a):
        ws, n = a[8], a[9]
        self.seen.append((ws, n))
        self.both.wait()
        return 0


@pytest.fixture
def host(monkeypatch):
    """The binding's own code on host tensors: a device number that they have, one stream."""
    monkeypatch.setattr(torch._C, "_cuda_getDevice", lambda: -1, raising=False)
    monkeypatch.setattr(torch.cuda, "is_current_stream_capturing", lambda: False)
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 0)
    monkeypatch.setattr(_lib, "_stream_handle", lambda: 7)


def _args():
    cache = torch.zeros(4, 2, 16, 64, dtype=torch.bfloat16)
    return dict(Q=torch.zeros(1, 128, dtype=torch.bfloat16), k_cache=cache, v_cache=cache.clone(),
                page_table=torch.zeros(1, 4, dtype=torch.int32), kv_len=torch.ones(1, dtype=torch.int32))


def test_two_attention_calls_at_once_have_a_workspace_each(host, monkeypatch):
    fake = _Library()
    one = torch.empty(1 << 16, dtype=torch.uint8)
    monkeypatch.setattr(_lib, "lib", lambda: fake)
    monkeypatch.setattr(_lib.Workspace, "get", classmethod(lambda cls, n: one))  # the stream's
    threads = [threading.Thread(target=lambda: _lib.paged_attention(**_args())) for _ in range(2)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    (a, na), (b, nb) = fake.seen
    assert na >= 4096 and nb >= 4096
    assert a + na <= b or b + nb <= a


def test_a_thread_has_its_own_buffers(host, monkeypatch):
    """The buffers that every other call takes: one for a thread and stream, grown when it is too small, given up when
    the thread ends or on clear()."""
    empty = torch.empty
    monkeypatch.setattr(torch, "empty", lambda n, dtype, device: empty(n, dtype=dtype))
    get = _lib.Workspace.get
    _lib.Workspace.clear()
    mine = get(1000)
    assert get(900) is mine and get(1000) is mine and mine.numel() >= 1000
    monkeypatch.setattr(_lib, "_stream_handle", lambda: 8)
    assert get(1000) is not mine
    monkeypatch.setattr(_lib, "_stream_handle", lambda: 7)
    others, kept = [], []
    up, down = threading.Barrier(3, timeout=30), threading.Barrier(3, timeout=30)

    def work():
        buf = get(500)
        assert get(400) is buf
        others.append(buf.data_ptr())
        kept.append(weakref.ref(buf))
        up.wait()
        down.wait()

    threads = [threading.Thread(target=work) for _ in range(2)]
    for t in threads:
        t.start()
    up.wait()
    assert len({mine.data_ptr(), *others}) == 3
    down.wait()
    for t in threads:
        t.join()
    gc.collect()
    assert [r() for r in kept] == [None, None]
    assert get(1000) is mine
    grown = get(5000)
    assert grown.numel() >= 5000 and get(1000) is grown
    _lib.Workspace.clear()
    assert get(5000) is not grown
    _lib.Workspace.clear()
