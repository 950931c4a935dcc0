"""What the embedding, the label log-probabilities and the sequence losses refuse, on the host."""
import pytest
import torch

import paper_2608_15665_amd as zo
from paper_2608_15665_amd import _lib

FAKE = 1 << 20  # never dereferenced: the calls refuse first, or have nothing to do
NAN, INF = float("nan"), float("inf")


def _detail():
    return zo.lib().zo_last_error_detail().decode()


def _embedding(rows=4, vocab=10, d=16, dtype=1, ids=FAKE, E=FAKE, scale=1.0, H=FAKE, flag=None):
    return zo.lib().zo_embedding(rows, vocab, d, dtype, ids, E, scale, H, flag, None)


def _backward(rows=4, vocab=10, d=16, dtype=1, ids=FAKE, E=FAKE, scale=1.0, odt=1, H=FAKE, acc=0, flag=None, ws=FAKE, n=1 << 40):
    return zo.lib().zo_embedding_backward(rows, vocab, d, dtype, ids, E, scale, odt, H, acc, flag, ws, n, None)


def _logprob(nblk=1, T=4, vocab=10, dtype=1, X=FAKE, ld=16, labels=FAKE, scale=1.0, logp=FAKE, lse=FAKE, flag=None,
             ws=FAKE, n=1 << 40):
    return zo.lib().zo_token_logprob(nblk, T, vocab, dtype, X, ld, labels, scale, logp, lse, flag, ws, n, None)


def _logprob_grad(nblk=1, T=4, vocab=10, dtype=1, X=FAKE, ld=16, labels=FAKE, scale=1.0, lse=FAKE, g=FAKE, dX=2 * FAKE, ldo=16,
                  flag=None, logp=None):
    return zo.lib().zo_token_logprob_backward(nblk, T, vocab, dtype, X, ld, labels, scale, lse, logp, g, dX, ldo, flag, None)


def _preference(nblk=1, rows=8, pairs=2, kind=0, average=0, beta=0.1, margin=0.0, smoothing=0.0, weight=1.0, logp=FAKE,
                ref=None, labels=None, start=FAKE, loss=FAKE, rewards=None, dlogp=None, flag=None, ws=FAKE, n=1 << 40):
    return zo.lib().zo_preference_loss(nblk, rows, pairs, kind, average, beta, margin, smoothing, weight, logp, ref, labels,
                                       start, loss, rewards, dlogp, flag, ws, n, None)


def _policy(nblk=1, rows=8, nseq=2, agg=0, per_token=0, low=0.2, high=0.2, kl=0.0, weight=1.0, logp=FAKE, old=FAKE, ref=None,
            adv=FAKE, labels=None, start=FAKE, loss=FAKE, stats=None, dlogp=None, flag=None, ws=FAKE, n=1 << 40):
    return zo.lib().zo_policy_loss(nblk, rows, nseq, agg, per_token, low, high, kl, weight, logp, old, ref, adv, labels, start,
                                   loss, stats, dlogp, flag, ws, n, None)


TABLE = [(dict(rows=-1), "rows"), (dict(vocab=0), "vocab"), (dict(vocab=1 << 30), "vocab"), (dict(d=0), "d = 0"),
         (dict(d=12), "d = 12"), (dict(d=(1 << 20) + 8), "d ="), (dict(dtype=3), "dtype 3"), (dict(ids=None), "ids is NULL"),
         (dict(ids=FAKE + 2), "4-byte"), (dict(flag=FAKE + 1), "4-byte"), (dict(scale=NAN), "scale"), (dict(scale=INF), "scale"),
         (dict(E=None), "NULL"), (dict(E=FAKE + 8), "16-byte"), (dict(H=None), "NULL"), (dict(H=FAKE + 2), "16-byte")]


@pytest.mark.parametrize("call", [_embedding, _backward])
@pytest.mark.parametrize("kw,needle", TABLE)
def test_tables(call, kw, needle):
    assert call(**kw) == 1 and needle in _detail(), _detail()


@pytest.mark.parametrize("call,kw,status,needle", [
    (_embedding, dict(rows=(1 << 30) + 1), 1, "rows"), (_backward, dict(rows=(1 << 24) + 1), 1, "rows"),
    (_embedding, dict(rows=1 << 30, d=1 << 20), 1, "too large"),
    (_backward, dict(odt=2), 1, "out_dtype"), (_backward, dict(dtype=0, odt=1), 1, "out_dtype"),
    (_backward, dict(odt=3), 1, "out_dtype"), (_backward, dict(rows=4000, n=100), 6, "workspace 100"),
    (_backward, dict(rows=4000, ws=None), 6, "workspace 0"), (_backward, dict(rows=4000, ws=FAKE + 128), 1, "256-byte"),
])
def test_tables_more(call, kw, status, needle):
    assert call(**kw) == status and needle in _detail(), _detail()


@pytest.mark.parametrize("call", [_logprob, _logprob_grad])
@pytest.mark.parametrize("kw,needle", [
    (dict(nblk=0), "nblk"), (dict(T=-1), "T = -1"), (dict(nblk=1 << 16, T=1 << 15), "nblk T"), (dict(vocab=0), "vocab"),
    (dict(vocab=17), "16 elements apart"), (dict(vocab=(1 << 30) + 1, ld=(1 << 30) + 1), "vocab"), (dict(ld=1 << 31), "apart"), (dict(dtype=3), "dtype 3"), (dict(scale=0.0), "scale"),
    (dict(scale=-1.0), "scale"), (dict(scale=NAN), "scale"), (dict(X=None), "NULL"), (dict(labels=None), "NULL"),
    (dict(X=FAKE + 1), "aligned"), (dict(dtype=0, X=FAKE + 2), "aligned"), (dict(labels=FAKE + 2), "aligned"),
    (dict(lse=FAKE + 2), "4-byte"), (dict(flag=FAKE + 3), "aligned")])
def test_logits(call, kw, needle):
    assert call(**kw) == 1 and needle in _detail(), _detail()


@pytest.mark.parametrize("kw,needle", [(dict(lse=None), "NULL"), (dict(g=None), "NULL"), (dict(dX=None), "dX is NULL"),
                                       (dict(dX=FAKE + 1), "dX"), (dict(ldo=9), "rows of dX"), (dict(dX=FAKE, ldo=24), "dX is X"),
                                       (dict(dX=FAKE, logp=FAKE), "logp is given"), (dict(logp=FAKE + 2), "4-byte"),
                                       (dict(g=FAKE + 1), "4-byte")])
def test_logits_gradient(kw, needle):
    assert _logprob_grad(**kw) == 1 and needle in _detail(), _detail()
    assert _logprob(logp=None) == 1 and "logp is NULL" in _detail()


def test_logits_workspace():
    assert zo.lib().zo_token_logprob_workspace(1, 4, 10, 1) == 0 and zo.lib().zo_token_logprob_workspace(1, 0, 10, 1) == 0
    assert zo.lib().zo_token_logprob_workspace(1, 2, 200000, 1) >= 2 * 2 * 8  # few long rows are split
    long = dict(T=2, vocab=200000, ld=200000)
    assert _logprob(**long, n=8) == 6 and "workspace 8" in _detail()
    assert _logprob(**long, ws=None) == 6 and _logprob(**long, ws=FAKE + 16) == 1 and "256-byte" in _detail()


BOTH = [(dict(nblk=0), "nblk"), (dict(nblk=65536), "nblk"), (dict(rows=-1), "rows"), (dict(nblk=1 << 15, rows=1 << 16), "rows"),
        (dict(rows=(1 << 29) + 1), "rows"),
        (dict(logp=None), "NULL"), (dict(start=None), "NULL"), (dict(loss=None), "NULL"), (dict(loss=FAKE + 4), "aligned"),
        (dict(logp=FAKE + 2), "aligned"), (dict(ref=FAKE + 1), "aligned"), (dict(labels=FAKE + 2), "aligned"),
        (dict(start=FAKE + 1), "aligned"), (dict(dlogp=FAKE + 2), "aligned"), (dict(flag=FAKE + 2), "aligned"),
        (dict(weight=NAN), "weight")]


@pytest.mark.parametrize("call", [_preference, _policy])
@pytest.mark.parametrize("kw,needle", BOTH)
def test_sequences(call, kw, needle):
    assert call(**kw) == 1 and needle in _detail(), _detail()


@pytest.mark.parametrize("call,kw,status,needle", [
    (_preference, dict(pairs=0), 1, "pairs"), (_preference, dict(pairs=(1 << 22) + 1), 1, "pairs"),
    (_preference, dict(kind=3), 1, "kind 3"), (_preference, dict(kind=-1), 1, "kind"), (_preference, dict(beta=0.0), 1, "beta"),
    (_preference, dict(beta=INF), 1, "beta"), (_preference, dict(margin=NAN), 1, "margin"),
    (_preference, dict(smoothing=0.6), 1, "smoothing"), (_preference, dict(smoothing=-0.1), 1, "smoothing"),
    (_preference, dict(smoothing=0.1, kind=1), 1, "smoothing"), (_preference, dict(smoothing=NAN), 1, "smoothing"),
    (_preference, dict(rewards=FAKE + 2), 1, "rewards"), (_preference, dict(rows=3000, n=8), 6, "workspace 8"),
    (_preference, dict(rows=3000, ws=None), 6, "workspace 0"), (_preference, dict(rows=3000, ws=FAKE + 8), 1, "256-byte"),
    (_policy, dict(nseq=0), 1, "nseq"), (_policy, dict(nseq=(1 << 23) + 1), 1, "nseq"),
    (_policy, dict(nblk=1000, nseq=1 << 22), 1, "nseq"), (_policy, dict(agg=3), 1, "aggregate"),
    (_policy, dict(low=-0.1), 1, "clip_low"), (_policy, dict(low=1.5), 1, "clip_low"), (_policy, dict(low=NAN), 1, "clip_low"),
    (_policy, dict(high=-1.0), 1, "clip_high"), (_policy, dict(high=INF), 1, "clip_high"), (_policy, dict(kl=-1.0), 1, "kl_coef"),
    (_policy, dict(kl=0.1), 1, "without ref_logp"), (_policy, dict(old=None), 1, "old_logp"), (_policy, dict(adv=None), 1, "advantage"),
    (_policy, dict(adv=FAKE + 2), 1, "aligned"), (_policy, dict(stats=FAKE + 4), 1, "aligned"), (_policy, dict(rows=9000, n=8), 6, "workspace 8"),
    (_policy, dict(rows=9000, ws=None), 6, "workspace 0"), (_policy, dict(rows=9000, ws=FAKE + 8), 1, "256-byte"),
])
def test_losses(call, kw, status, needle):
    assert call(**kw) == status and needle in _detail(), _detail()


def test_nothing_to_do():
    assert _embedding(rows=0, ids=None, E=None, H=None) == 0
    assert _backward(rows=0, ids=None, E=None, H=None, acc=1, ws=None, n=0) == 0
    assert _logprob(T=0, X=None, labels=None, logp=None, lse=None) == 0
    assert _logprob_grad(T=0, X=None, labels=None, lse=None, g=None, dX=None) == 0
    L = zo.lib()
    assert L.zo_embedding_backward_workspace(0, 10, 16) == 0 and L.zo_embedding_backward_workspace(-1, 10, 16) == 0
    assert L.zo_preference_loss_workspace(0, 8, 2) == 0 and L.zo_policy_loss_workspace(1, 8, 0) == 0


@pytest.fixture
def cpu(monkeypatch):
    """The binding with host tensors in place of the current device's; a call that passes its checks is an error here."""
    monkeypatch.setattr(torch._C, "_cuda_getDevice", lambda: -1, raising=False)
    monkeypatch.setattr(_lib, "_stream_handle", lambda: 0)

    class Library:
        def __getattr__(self, name):
            return lambda *a: 256 if name.endswith("_workspace") else pytest.fail(name)

    monkeypatch.setattr(_lib, "lib", lambda: Library())
    _lib._ws_bytes.cache_clear()
    yield
    _lib._ws_bytes.cache_clear()


I, F = (lambda *s: torch.zeros(*s, dtype=torch.int32)), torch.zeros


@pytest.mark.parametrize("call,error,needle", [
    (lambda: zo.embedding(F(4).long(), F(10, 8)), TypeError, "ids must be torch.int32"),
    (lambda: zo.embedding(I(4), F(10, 8).double()), TypeError, "unsupported dtype"),
    (lambda: zo.embedding(I(4), F(80)), ValueError, "vocab x d"),
    (lambda: zo.embedding(I(4), F(10, 16)[:, :8]), ValueError, "contiguous"),
    (lambda: zo.embedding(I(4), F(10, 8), out=F(3, 8)), ValueError, "32 elements"),
    (lambda: zo.embedding(I(4), F(10, 8), out=F(4, 8).half()), TypeError, "out must be"),
    (lambda: zo.embedding(I(4), F(10, 8), bad_flag=I(2)), ValueError, "bad_flag"),
    (lambda: zo.embedding_backward(I(4), F(3, 8), 10), ValueError, "grad must hold 32"),
    (lambda: zo.embedding_backward(I(4), F(4, 8), 10, accumulate=True), ValueError, "accumulate needs out"),
    (lambda: zo.embedding_backward(I(4), F(4, 8), 10, out=F(9, 8)), ValueError, "out must hold 80"),
    (lambda: zo.embedding_backward(I(4), F(4, 8), 1 << 32, out=F(9, 8)), ValueError, "out of range"),
    (lambda: zo.embedding_backward(I(4), F(4, 8), 10, workspace=F(9)), TypeError, "workspace"),
    (lambda: zo.token_logprob(F(2, 4, 8), I(8)), ValueError, "rows x columns"),
    (lambda: zo.token_logprob(F(8, 8), I(3)), ValueError, "blocks of T = 3"),
    (lambda: zo.token_logprob(F(8, 8), I(0)), ValueError, "blocks of T = 0"),
    (lambda: zo.token_logprob(F(0, 8), I(3)), ValueError, "blocks of T = 3"),
    (lambda: zo.token_logprob(F(8, 8), I(8), vocab=9), ValueError, "8 columns"),
    (lambda: zo.token_logprob(F(8, 16)[:, ::2], I(8)), ValueError, "dense"),
    (lambda: zo.token_logprob(F(8, 8), I(8).long()), TypeError, "labels must be"),
    (lambda: zo.token_logprob(F(8, 8), I(8), lse=F(7)), ValueError, "lse must hold 8"),
    (lambda: zo.token_logprob_backward(F(8, 8), I(8), F(8), F(7)), ValueError, "grad must hold 8"),
    (lambda: zo.token_logprob_backward(F(8, 8), I(8), F(8), F(8), logp=F(7)), ValueError, "logp must hold 8"),
    (lambda: zo.token_logprob_backward(F(8, 8), I(8), F(8), F(8), out=F(8, 9)), ValueError, "out must be 8 x 8"),
    (lambda: zo.token_logprob_backward(F(8, 8), I(8), F(8).double(), F(8)), TypeError, "lse must be"),
    (lambda: zo.preference_loss(F(2, 3, 4), I(5), 0.1), ValueError, "nblk x rows"),
    (lambda: zo.preference_loss(F(2, 8), I(4), 0.1), ValueError, "2 pairs"),
    (lambda: zo.preference_loss(F(2, 8), I(1), 0.1), ValueError, "2 pairs"),
    (lambda: zo.preference_loss(F(2, 8), I(5), 0.1, kind="kto"), ValueError, "kind must be"),
    (lambda: zo.preference_loss(F(2, 8), I(5), 0.1, ref_logp=F(2, 8)), ValueError, "ref_logp must hold 8"),
    (lambda: zo.preference_loss(F(2, 8).half(), I(5), 0.1), TypeError, "logp must be"),
    (lambda: zo.preference_loss(F(2, 8), I(5), 0.1, rewards=F(4)), ValueError, "rewards must hold 8"),
    (lambda: zo.preference_loss(F(2, 8), I(5), 0.1, loss=F(2)), TypeError, "loss must be"),
    (lambda: zo.policy_loss(F(2, 8), F(8), F(8), I(5)), ValueError, "advantage must hold 4"),
    (lambda: zo.policy_loss(F(2, 8), F(8), F(4), I(5), per_token=True), ValueError, "advantage must hold 8"),
    (lambda: zo.policy_loss(F(2, 8), F(2, 8), F(4), I(5)), ValueError, "old_logp must hold 8"),
    (lambda: zo.policy_loss(F(2, 8), F(8), F(1), I(1)), ValueError, "nseq >= 1"),
    (lambda: zo.policy_loss(F(2, 8), F(8), F(4), I(5), aggregate="mean"), ValueError, "aggregate must be"),
    (lambda: zo.policy_loss(F(2, 8), F(8), F(4), I(5), stats=torch.zeros(2, dtype=torch.float64)), ValueError, "stats must hold 4"),
])
def test_binding(cpu, call, error, needle):
    with pytest.raises(error, match=needle):
        call()


def test_binding_refuses_host_tensors(monkeypatch):
    monkeypatch.setattr(torch._C, "_cuda_getDevice", lambda: 0, raising=False)
    for call in (lambda: zo.embedding(I(4), F(10, 8)), lambda: zo.token_logprob(F(8, 8), I(8)),
                 lambda: zo.preference_loss(F(2, 8), I(5), 0.1), lambda: zo.policy_loss(F(2, 8), F(8), F(4), I(5))):
        with pytest.raises(ValueError, match="current device"):
            call()


def test_sizes_that_an_int_would_wrap(cpu):
    """Columns and sequences beyond 2^32, as views of one element."""
    wide = torch.zeros(1, 1).expand(1, 2 ** 32 + 8)
    with pytest.raises(ValueError, match="out of range"):
        zo.embedding(I(1), wide)
    with pytest.raises(ValueError, match="out of range"):
        zo.embedding_backward(I(1), wide, 8)
    starts = torch.zeros(1, dtype=torch.int32).expand(2 ** 33 + 3)
    with pytest.raises(ValueError, match="out of range"):
        zo.preference_loss(F(8), starts, 0.1)
    with pytest.raises(ValueError, match="out of range"):
        zo.policy_loss(F(8), F(8), F(8), starts)
