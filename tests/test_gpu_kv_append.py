"""zo_kv_append against a float64 reference: lengths and pages at their edges, rows that lie apart, far
positions, 8-bit pages whose scale grows, and batches that break the rules.

Rotated values: sine and cosine carry an absolute error under 2^-23 (fp64 angles, fp32 polynomials), the
products and their sum round three times more at 2^-24: within 2^-21 (|a| + |b|) of the exact value before
the one rounding to the stored type (2^-8 or 2^-11 relative; e4m3: 2^-4, or half of 2^-9 steps of the scale).
fp64 angles are within 2^-51 of their size: 2^-29 at a position of 2^22.  Copied values are bitwise."""
import numpy as np
import pytest
import torch

import paper_2608_15665_amd as zo
from _paged import DT, E4M3, batch, bits, dev, host64, rows16
from oracle import paged as op

pytestmark = pytest.mark.gpu


def reach(x, dh):
    """|a| + |b| of every element's pair."""
    m = np.abs(x[..., :dh // 2]) + np.abs(x[..., dh // 2:])
    return np.concatenate([m, m], -1)


def check_rotated(got, ref, x, dh, dt):
    tol = (2.0 ** -8 if dt == "bf16" else 2.0 ** -11) * np.abs(ref) + 2.0 ** -21 * reach(x, dh) + 2.0 ** -25
    assert np.all(np.abs(got - ref) <= tol), float(np.max(np.abs(got - ref) / tol))


LENS = {
    "one": ([1], [1]),
    "token": ([1, 17, 300, 64, 33], [1] * 5),
    "drafts": ([4, 19, 64, 130], [4, 3, 1, 4]),
    "mixed": ([40, 16, 0, 65, 128, 7], [40, 1, 0, 50, 33, 7]),
    "padded": ([3, 0, 20], [8, 4, 8]),  # rows before position 0
    "prompt": ([257, 100], [257, 99]),
}


@pytest.mark.parametrize("dt", ["bf16", "f16"])
@pytest.mark.parametrize("shape", LENS)
@pytest.mark.parametrize("heads,kvh,dh,ps,base,pad", [(4, 2, 128, 16, 1e4, 0), (3, 3, 64, 64, 1e6, 8), (10, 2, 64, 256, 1e4, 16),
                                                      (2, 1, 128, 32, None, 8)])
def test_append16(dt, shape, heads, kvh, dh, ps, base, pad):
    lens, news = LENS[shape]
    rng = np.random.default_rng(len(shape) + dh)
    table, q_start, kv_len, pages = batch(rng, lens, news, ps)
    rows = int(q_start[-1]) + 3  # three rows behind the last sequence
    (Q, Qv), (K, Kv), (V, Vv) = (rows16(rng.standard_normal((rows, n * dh)), dt, pad) for n in (heads, kvh, kvh))
    junk = rng.standard_normal((2, pages, kvh, ps, dh))
    kc, vc = dev(junk[0], DT[dt]), dev(junk[1], DT[dt])
    before = [host64(kc), host64(vc)]
    flag = torch.zeros(1, dtype=torch.int32, device="cuda")
    qo = torch.full((rows, heads * dh), 77.0, dtype=DT[dt], device="cuda")
    seqs = None if max(news) == 1 and min(news) == 1 else dev(q_start)
    got = zo.kv_append(K, V, kc, vc, dev(table), dev(kv_len), q_start=seqs, max_q=max(news), Q=Q if base else None,
                       q_out=qo if base else None, rope_base=base, bad_flag=flag)
    assert int(flag) == 0 and (got is qo if base else got is None)
    K3, V3 = Kv.reshape(rows, kvh, dh), Vv.reshape(rows, kvh, dh)
    (ref, refv), _ = op.kv_append(K3, V3, before, table, q_start, kv_len, base)
    np.testing.assert_array_equal(host64(vc), refv)
    gk = host64(kc)
    stored = ref != before[0]
    if base is None:
        np.testing.assert_array_equal(gk, ref)
    else:
        np.testing.assert_array_equal(gk[~stored], before[0][~stored])
        src = np.zeros_like(gk)  # what each slot was made from
        for s in range(len(lens)):
            for r, p in op.rows_of(s, q_start, kv_len):
                if p >= 0:
                    src[table[s, p // ps], :, p % ps] = K3[r]
        tol = (2.0 ** -8 if dt == "bf16" else 2.0 ** -11) * np.abs(ref) + 2.0 ** -21 * reach(src, dh) + 2.0 ** -25
        assert np.all((np.abs(gk - ref) <= tol) | ~stored)
        go = host64(qo)
        np.testing.assert_array_equal(go[int(q_start[-1]):], 77.0)
        Q3 = Qv.reshape(rows, heads, dh)
        for s in range(len(lens)):
            for r, p in op.rows_of(s, q_start, kv_len):
                check_rotated(go[r].reshape(heads, dh), op.rotate(Q3[r], max(p, 0), base), Q3[r], dh, dt)


@pytest.mark.parametrize("pos", [1, 4095, 65535, 1 << 20, (1 << 22) - 1])
def test_far_positions(pos):
    """One row at a far position of a wide table; the queries are rotated in place."""
    rng, dh, ps = np.random.default_rng(pos), 128, 256
    width = pos // ps + 1
    table = np.full((1, width), -1, np.int32)
    table[0, -1] = 1
    (Q, Qv), (K, Kv), (V, _) = (rows16(rng.standard_normal((1, n * dh)), "f16") for n in (4, 2, 2))
    kc = torch.zeros((3, 2, ps, dh), dtype=torch.float16, device="cuda")
    vc = torch.zeros_like(kc)
    zo.kv_append(K, V, kc, vc, dev(table), dev(np.array([pos + 1], np.int32)), Q=Q, q_out=Q, rope_base=1e4)
    K3, Q3 = Kv.reshape(2, dh), Qv.reshape(4, dh)
    check_rotated(host64(kc)[1, :, pos % ps], op.rotate(K3, pos, 1e4), K3, dh, "f16")
    check_rotated(host64(Q).reshape(4, dh), op.rotate(Q3, pos, 1e4), Q3, dh, "f16")


def test_matches_rope_of_a_whole_sequence():
    """From an empty cache the rotation is zo.rope's, to one rounding of fp32 before that to 16 bits."""
    rng, dh, n = np.random.default_rng(5), 128, 70
    K, Kv = rows16(rng.standard_normal((n, 2 * dh)), "bf16")
    whole = zo.rope(K.clone(), n, 2)
    kc = torch.zeros((5, 2, 16, dh), dtype=torch.bfloat16, device="cuda")
    zo.kv_append(K, K, kc, torch.zeros_like(kc), dev(np.arange(5, dtype=np.int32)[None]), dev(np.array([n], np.int32)),
                 q_start=dev(np.array([0, n], np.int32)), max_q=n, rope_base=1e4)
    mine = host64(kc).transpose(0, 2, 1, 3).reshape(80, 2 * dh)[:n]
    d = np.abs(mine - host64(whole))
    assert np.mean(d > 0) < 1e-3 and np.all(d <= 2.0 ** -7 * np.abs(mine) + 2.0 ** -20)


@pytest.mark.parametrize("cache", ["same", "e4m3"])
@pytest.mark.parametrize("inplace", [False, True])
def test_padding_is_copied(cache, inplace):
    """Queries before position 0 keep their bits (infinities, NaN and -0 among them), their keys are not stored."""
    rng, dh, ps, kvh = np.random.default_rng(3), 128, 16, 2
    news, lens = [6, 4, 3], [2, -3, 0]
    a = rng.standard_normal((14, 4 * dh))
    a[:, ::7], a[:, 3::11], a[:, 5::13], a[:, 1::17] = np.inf, np.nan, -0.0, -np.inf
    Q, _ = rows16(a, "bf16")
    was = bits(Q).copy()
    K, _ = rows16(np.where(np.isfinite(a), a, 1.0)[:, :kvh * dh], "bf16")
    table, q_start, kv_len, pages = batch(rng, lens, news, ps)
    kc = torch.zeros((pages, kvh, ps, dh), device="cuda").to(E4M3 if cache == "e4m3" else torch.bfloat16)
    vc = kc.clone()
    ks, vs = ((torch.ones((pages, kvh), device="cuda") for _ in range(2)) if cache == "e4m3" else (None, None))
    got = zo.kv_append(K, K, kc, vc, dev(table), dev(kv_len), q_start=dev(q_start), max_q=6, Q=Q,
                       q_out=Q if inplace else torch.zeros_like(Q), rope_base=1e4, k_scale=ks, v_scale=vs)
    pad = [r for r in range(13) if r not in (4, 5)]  # rows 4, 5 are positions 0, 1 of the first sequence
    np.testing.assert_array_equal(bits(got)[pad], was[pad])
    assert not np.array_equal(bits(got)[5], was[5])
    stored = host64(vc).any((1, 3))
    assert stored.sum() == 2 and stored[table[0, 0], :2].all()


@pytest.mark.parametrize("cache", ["same", "e4m3"])
def test_max_q_by_default(cache):
    """Without max_q every row of a batch with q_start is taken, and one of each sequence without."""
    rng, dh, ps, kvh = np.random.default_rng(4), 64, 32, 2
    table, q_start, kv_len, pages = batch(rng, [40, 9, 70], [35, 0, 3], ps)
    K, V, Q = (rows16(rng.standard_normal((38, n * dh)), "f16")[0] for n in (kvh, kvh, 4))
    outs = []
    for kw in (dict(max_q=35), dict()):
        kc = torch.zeros((pages, kvh, ps, dh), device="cuda").to(E4M3 if cache == "e4m3" else torch.float16)
        vc = kc.clone()
        ks, vs = ((torch.ones((pages, kvh), device="cuda") for _ in range(2)) if cache == "e4m3" else (None, None))
        flag = torch.zeros(1, dtype=torch.int32, device="cuda")
        args = dict(q_start=dev(q_start), k_scale=ks, v_scale=vs, bad_flag=flag, **kw)
        q = zo.kv_append(K, V, kc, vc, dev(table), dev(kv_len), Q=Q, rope_base=1e4, **args)
        o = zo.paged_attention(q, kc, vc, dev(table), dev(kv_len), **args)
        assert int(flag) == 0
        outs.append([bits(t) for t in (q, kc, vc, o)])
    for x, y in zip(*outs):
        np.testing.assert_array_equal(x, y)
    for bad in (-1, 1 << 31, (1 << 32) + 1):
        with pytest.raises(ValueError, match="max_q"):
            zo.paged_attention(q, kc, vc, dev(table), dev(kv_len), q_start=dev(q_start), max_q=bad, k_scale=ks, v_scale=vs)


# ---------------------------------------------------------------- 8-bit cache
def check8(kc, ks, ref, refs, src, what, rotated):
    """Scales as the reference's, but where the largest magnitude is within the rotation's error of a border;
    codes within half a step of the exact value (without a rotation: bitwise)."""
    got, gs = host64(kc), host64(ks)
    if not rotated:
        np.testing.assert_array_equal(gs, refs, err_msg=what)
        np.testing.assert_array_equal(got, ref, err_msg=what)
        return
    assert np.array_equal(gs, refs), what  # no largest magnitude of these draws is near a border
    val, exact = got * gs[:, :, None, None], src
    where = ~np.isnan(exact)
    half = np.maximum(2.0 ** -4 * np.abs(exact), 2.0 ** -10 * gs[:, :, None, None])
    err = np.abs(val - exact)
    assert np.all(err[where] <= (half * (1 + 2.0 ** -10) + 2.0 ** -19)[where]), what


@pytest.mark.parametrize("dt", ["bf16", "f16"])
@pytest.mark.parametrize("base", [None, 1e4])
@pytest.mark.parametrize("kvh,dh,ps", [(1, 128, 16), (3, 64, 32), (5, 128, 64), (2, 64, 256), (2, 128, 256), (3, 128, 128)])
def test_append8_in_pieces(dt, base, kvh, dh, ps):
    """A sequence in pieces of several lengths, with values that grow and shrink, beside one that stands still
    and one of single rows: scales grow within a page, start again in the next, and junk slots stay."""
    rng = np.random.default_rng(kvh * ps)
    pieces = [(3, 0, 1), (1, 0, 1), (1, 0, 1), (ps, 0, 1), (2 * ps + 5, 0, 1), (0, 0, 1), (7, 0, 1)]
    gain = [1.0, 5.0, 0.1, 0.02, 1.0, 1.0, 30.0]
    total = [sum(p[i] for p in pieces) for i in range(3)]
    held = [-(-t // ps) for t in total]
    pages = sum(held) + 2
    table = np.full((3, max(held)), 1 << 29, np.int32)
    order = rng.permutation(pages)
    for s in range(3):
        table[s, :held[s]] = order[sum(held[:s]):sum(held[:s + 1])]
    shape = (pages, kvh, ps, dh)
    codes = [op.nearest_e4m3(rng.uniform(-400, 400, shape)) for _ in range(2)]
    kc, vc = (dev(c, torch.float32).to(E4M3) for c in codes)
    ks, vs = (torch.full((pages, kvh), float("nan"), device="cuda") for _ in range(2))
    caches, scales = codes, [host64(ks), host64(vs)]
    exact = [np.full(shape, np.nan), np.full(shape, np.nan)]
    lens = np.zeros(3, np.int32)
    for news, g in zip(pieces, gain):
        lens = (lens + np.array(news)).astype(np.int32)
        q_start = np.concatenate([[0], np.cumsum(news)]).astype(np.int32)
        rows = int(q_start[-1]) + 1
        (K, Kv), (V, Vv) = (rows16(rng.standard_normal((rows, kvh * dh)) * g, dt, 8) for _ in range(2))
        flag = torch.zeros(1, dtype=torch.int32, device="cuda")
        zo.kv_append(K, V, kc, vc, dev(table), dev(lens), q_start=dev(q_start), max_q=max(news), rope_base=base,
                     k_scale=ks, v_scale=vs, bad_flag=flag)
        assert int(flag) == 0
        K3, V3 = Kv.reshape(rows, kvh, dh), Vv.reshape(rows, kvh, dh)
        was, was_s = caches, scales
        caches, scales = op.kv_append(K3, V3, caches, table, q_start, lens, base, scales)
        for s in range(3):
            for r, p in op.rows_of(s, q_start, lens):
                for e, x in zip(exact, (K3, V3)):
                    e[table[s, p // ps], :, p % ps] = op.rotate(x[r], p, base) if base and x is K3 else x[r]
        check8(vc, vs, caches[1], scales[1], exact[1], "V", False)
        if base is None:
            check8(kc, ks, caches[0], scales[0], exact[0], "K", False)
        else:
            np.testing.assert_array_equal(host64(ks), scales[0])
            # this call's slots: half a step of the exact value; everything else as the reference
            got = host64(kc)
            new = np.zeros(shape, bool)
            for s in range(3):
                for r, p in op.rows_of(s, q_start, lens):
                    new[table[s, p // ps], :, p % ps] = True
            sc = scales[0][:, :, None, None] * np.ones(shape)
            half = np.maximum(2.0 ** -4 * np.abs(exact[0]), 2.0 ** -10 * sc)
            with np.errstate(invalid="ignore"):
                assert np.all((np.abs(got * sc - exact[0]) <= half * (1 + 2.0 ** -10) + 2.0 ** -19 * g) | ~new)
                np.testing.assert_array_equal(got[~new], caches[0][~new])
            caches[0] = got  # later rounds of earlier slots start from these codes
    assert np.all(was_s[0][table[0, 0]] > 0)


def test_append8_special_values():
    """Zeros, values whose scale is at its ends, and values that are not finite (stored as NaN, no part of the
    scale)."""
    dh, ps = 64, 16
    rows = [np.zeros(dh), np.full(dh, 2.0 ** -133), np.full(dh, 2.0 ** 127 * 1.9), np.full(dh, 448.0), np.full(dh, 449.0 + 1),
            np.linspace(-1, 1, dh), np.linspace(-1, 1, dh)]
    a = np.stack(rows)
    a[5, 3], a[5, 40] = np.inf, -np.inf
    a[6] = np.nan
    K, Kv = rows16(a, "bf16")
    n = len(rows)
    kc = torch.zeros((n, 1, ps, dh), dtype=torch.float32, device="cuda").to(E4M3)
    vc, ks, vs = kc.clone(), torch.full((n, 1), float("nan"), device="cuda"), torch.full((n, 1), float("nan"), device="cuda")
    table = dev(np.arange(n, dtype=np.int32)[:, None])
    zo.kv_append(K, K, kc, vc, table, dev(np.ones(n, np.int32)), k_scale=ks, v_scale=vs)
    z = [np.zeros((n, 1, ps, dh)) for _ in range(2)]
    ref, refs = op.kv_append(Kv.reshape(n, 1, dh), Kv.reshape(n, 1, dh), z, np.arange(n)[:, None], None, np.ones(n, int),
                             None, [np.full((n, 1), np.nan) for _ in range(2)])
    for got, s, r, rs in ((kc, ks, ref[0], refs[0]), (vc, vs, ref[1], refs[1])):
        np.testing.assert_array_equal(host64(s), rs)
        np.testing.assert_array_equal(host64(got), r)
    assert np.isnan(host64(kc)[5, 0, 0, 3]) and float(ks[0, 0]) == 2.0 ** -126 and float(ks[3, 0]) == 1.0


@pytest.mark.parametrize("cache", ["same", "e4m3"])
def test_append_again_is_the_same(cache):
    """The same call twice (a step that is taken again) leaves what once leaves."""
    rng, dh, ps, kvh = np.random.default_rng(9), 128, 32, 4
    table, q_start, kv_len, pages = batch(rng, [70, 33, 5], [9, 4, 5], ps)
    K, V, Q = (rows16(rng.standard_normal((18, n * dh)) * 9, "bf16")[0] for n in (kvh, kvh, 8))
    start = rng.uniform(-1, 1, (pages, kvh, ps, dh))
    kc, vc = ((dev(start, torch.float32) * 400).to(E4M3) if cache == "e4m3" else dev(start, DT["bf16"]) for _ in range(2))
    ks, vs = ((torch.full((pages, kvh), 2.0 ** -9, device="cuda") for _ in range(2)) if cache == "e4m3" else (None, None))
    call = lambda: zo.kv_append(K, V, kc, vc, dev(table), dev(kv_len), q_start=dev(q_start), max_q=9, Q=Q,  # noqa: E731
                                rope_base=1e4, k_scale=ks, v_scale=vs)
    q1 = bits(call())
    first = [bits(t) for t in (kc, vc, ks, vs) if t is not None]
    np.testing.assert_array_equal(bits(call()), q1)
    for a, t in zip(first, [t for t in (kc, vc, ks, vs) if t is not None]):
        np.testing.assert_array_equal(bits(t), a)


@pytest.mark.parametrize("cache", ["same", "e4m3"])
def test_batches_that_break_the_rules(cache):
    """A page that is none, a length beyond the table, more rows than max_q, row ranges that leave the tensors:
    the flag is raised, what is legal is stored, nothing else is touched."""
    dh, ps, kvh, pages = 64, 16, 2, 6
    K = torch.full((12, kvh * dh), 3.0, dtype=torch.bfloat16, device="cuda")
    e8 = cache == "e4m3"

    def run(table, kv_len, q_start, max_q):
        kc, vc = (torch.zeros((pages, kvh, ps, dh), device="cuda").to(E4M3 if e8 else torch.bfloat16) for _ in range(2))
        ks, vs = ((torch.ones((pages, kvh), device="cuda") for _ in range(2)) if e8 else (None, None))
        flag = torch.zeros(1, dtype=torch.int32, device="cuda")
        zo.kv_append(K, K, kc, vc, dev(np.array(table, np.int32)), dev(np.array(kv_len, np.int32)),
                     q_start=dev(np.array(q_start, np.int32)), max_q=max_q, k_scale=ks, v_scale=vs, bad_flag=flag)
        a, b = (host64(kc) * (host64(ks)[:, :, None, None] if e8 else 1.0)), host64(vc) * (host64(vs)[:, :, None, None] if e8 else 1.0)
        np.testing.assert_array_equal(a, b)
        assert np.all((a == 0) | (a == 3)) and np.all(a.max((1, 3)) == a.min((1, 3)))
        return int(flag), {(p, t) for p in range(pages) for t in range(ps) if a[p, 0, t, 0] == 3}

    slots = lambda p, lo, hi: {(p, t) for t in range(lo, hi)}  # noqa: E731
    assert run([[4, 2]], [20], [0, 6], 6) == (0, slots(4, 14, 16) | slots(2, 0, 4))
    assert run([[4, 2]], [20], [0, 6], 12) == (0, slots(4, 14, 16) | slots(2, 0, 4))
    assert run([[pages, 2]], [20], [0, 6], 6) == (1, slots(2, 0, 4))
    assert run([[4, -1]], [20], [0, 6], 6) == (1, slots(4, 14, 16))
    assert run([[4, 2]], [34], [0, 6], 6) == (1, slots(2, 12, 16))       # positions 28 .. 33 of 32
    assert run([[4, 2]], [50], [0, 6], 6) == (1, set())
    assert run([[4, 2]], [20], [0, 6], 4) == (1, slots(4, 14, 16) | slots(2, 0, 2))
    assert run([[4, 2], [1, 3]], [2, 3], [0, 2, 15], 12)[0] == 1          # clamped to 12 rows: 10 of 3 positions
    assert run([[4, 2], [1, 3]], [2, 3], [-5, 2, 5], 12) == (1, slots(4, 0, 2) | slots(1, 0, 3))
    assert run([[4, 2], [1, 3]], [2, 3], [4, 2, 5], 12)[0] == 1
    assert run([[4, 2]], [-2 ** 31], [0, 12], 12) == (0, set())           # all padding
    assert run([[4, 2]], [0], [0, 0], 12) == (0, set())
