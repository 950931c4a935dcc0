"""Paged key/value batches for the tests: lengths, pages in shuffled order, caches full of junk that no
call may read or change, and the bars of the two operators."""
import numpy as np
import torch

import paper_2608_15665_amd as zo
from _common import ulp16
from oracle import paged as op

DT = {"bf16": torch.bfloat16, "f16": torch.float16}
E4M3 = torch.float8_e4m3fn


def batch(rng, lens, news, ps, spare=2, width=0):
    """(table, q_start, kv_len, pages): every sequence's pages, shuffled over a pool with `spare` more; entries
    that are not in use hold numbers that are no pages."""
    held = [-(-max(t, 0) // ps) for t in lens]
    pages = sum(held) + spare
    order = rng.permutation(pages)
    table = np.full((len(lens), max([width, 1, *held])), -7, np.int32)
    table[:, ::2] = 1 << 30
    at = 0
    for s, n in enumerate(held):
        table[s, :n] = order[at:at + n]
        at += n
    return table, np.concatenate([[0], np.cumsum(news)]).astype(np.int32), np.asarray(lens, np.int32), pages


def dev(a, dt=None):
    t = torch.from_numpy(np.ascontiguousarray(a))
    return (t if dt is None else t.to(dt)).cuda()


def host64(t):
    if t.dtype == E4M3:
        t = t.view(torch.uint8).cpu().view(E4M3)
    return t.detach().cpu().to(torch.float64).numpy()


def bits(t):
    return t.detach().view(torch.uint8 if t.dtype == E4M3 else torch.int16 if t.element_size() == 2 else torch.int32).cpu().numpy()


def rows16(a, dt, pad=0):
    """A float64 array of rows as a device tensor of 16 bits, and its values.  pad: as a column range of a wider
    tensor whose other columns are NaN."""
    a = np.asarray(a, np.float64).reshape(len(a), -1)
    wide = np.full((a.shape[0], a.shape[1] + 2 * pad), np.nan)
    wide[:, pad:pad + a.shape[1]] = a
    t = dev(wide, DT[dt])[:, pad:pad + a.shape[1]]
    return t, host64(t)


def pool16(rng, shape, dt, junk=np.nan):
    """A 16-bit cache and its values, all junk."""
    t = dev(np.full(shape, junk), DT[dt])
    return t, host64(t)


def attend(rng, dt, lens, news, ps, heads, kvh, dh, cache="same", width=0, spread=1.0, pad=0, seqs=True, q=None, k=None,
           v=None, rows_behind=0, max_q=None):
    """Runs zo.paged_attention on random (or the given) keys and values; slots behind the sequences are NaN.
    Returns (got, ref, mag, table, q_start): got is rows x heads x dh."""
    table, q_start, kv_len, pages = batch(rng, lens, news, ps, width=width)
    rows = int(q_start[-1]) + rows_behind
    Q = rng.standard_normal((rows, heads * dh)) * spread if q is None else q
    Qd, Qv = rows16(Q, dt, pad)
    used = np.zeros((pages, ps), bool)
    for s, n in enumerate(lens):
        for t in range(max(n, 0)):
            used[table[s, t // ps], t % ps] = True
    keep = used[:, None, :, None]
    dense = [rng.standard_normal((pages, kvh, ps, dh)) for _ in range(2)]
    for arr, given in zip(dense, (k, v)):
        if given is not None:  # per sequence: kvh x len x dh
            for s, n in enumerate(lens):
                for t in range(n):
                    arr[table[s, t // ps], :, t % ps] = given[s][:, t]
    scl = None
    if cache == "e4m3":
        scl = [2.0 ** rng.integers(-4, 3, (pages, kvh)) for _ in range(2)]
        scl[1] = scl[1] * 1.37  # any scale is one, not powers of two alone
        scl = [x.astype(np.float32).astype(np.float64) for x in scl]
        vals = [op.nearest_e4m3(np.clip(a / s[:, :, None, None], -448, 448)) for a, s in zip(dense, scl)]
        devs = [dev(np.where(keep, a, np.nan), torch.float32).to(E4M3) for a in vals]
        # pages that nothing holds have scales that are junk too
        hold = used.any(1)[:, None]
        sd = [dev(np.where(hold, s, np.nan), torch.float32) for s in scl]
    else:
        devs = [dev(np.where(keep, a, np.nan), DT[dt]) for a in dense]
        sd = [None, None]
    caches = [np.where(keep, host64(t), 0.0) for t in devs]
    out = torch.full((rows, heads * dh), 77.0, dtype=DT[dt], device="cuda")
    flag = torch.zeros(1, dtype=torch.int32, device="cuda")
    zo.paged_attention(Qd, devs[0], devs[1], dev(table), dev(kv_len), q_start=dev(q_start) if seqs else None,
                       max_q=max(news) if max_q is None else max_q, k_scale=sd[0], v_scale=sd[1], out=out, bad_flag=flag)
    got = host64(out).reshape(rows, heads, dh)
    assert int(flag) == 0
    np.testing.assert_array_equal(got[int(q_start[-1]):], 77.0)
    ref, mag = op.paged_attention(Qv.reshape(rows, heads, dh), caches, table, q_start, kv_len, scl)
    n = int(q_start[-1])
    return got[:n], ref[:n], mag[:n]


def check_attention(got, ref, mag, dt, what, many=False, cache="same"):
    """Few rows: P enters the P V product as a hi + lo pair of 16-bit values (relative error <= 2^-16), and the
    fp32 logits carry an absolute error of a few 2^-24 |q| |k|, which moves P by under 2^-16 relative at logits
    of a few hundred; fp32 sums of up to some thousand terms add 2^-16.  So before its rounding (half an ulp of
    the type) an output is within 2^-14 softmax(S) |V| of the exact one.  Many (see many()): P is rounded once, by 2^-8 (bf16) or 2^-11
    (fp16) of a weight at most, but a pair too for fp16 rows of 8-bit caches."""
    assert np.all(np.isfinite(got)), what
    p = 2.0 ** -14 + (0.0 if not many or (dt == "f16" and cache == "e4m3") else 2.0 ** -11 if dt == "f16" else 2.0 ** -8)
    bound = 0.5 * ulp16(ref, dt) * (1 + 2.0 ** -6) + p * mag
    err = np.abs(got - ref)
    assert np.all(err <= bound), (what, float(np.max(err / np.maximum(bound, 1e-300))))


def many(news, heads, kvh, cache="same"):
    """Whether a sequence may have over 16 rows for a key head (32 with an 8-bit cache)."""
    return max(news) * (heads // kvh) > (32 if cache == "e4m3" else 16)
