"""zo_paged_attention against a float64 reference: from one key to long contexts split over workgroups,
lengths around tiles and pages, grouped heads, 8-bit caches, padding, logits that move the running maximum,
keys and values that are not finite, and batches that break the rules."""
import numpy as np
import pytest
import torch

import paper_2608_15665_amd as zo
from _paged import DT, E4M3, attend, batch, check_attention, dev, host64, many, rows16

pytestmark = pytest.mark.gpu

HEADS = [(4, 4, 128), (10, 2, 128), (7, 1, 64), (3, 3, 64), (24, 1, 128)]


@pytest.mark.parametrize("cache", ["same", "e4m3"])
@pytest.mark.parametrize("dt", ["bf16", "f16"])
@pytest.mark.parametrize("heads,kvh,dh", HEADS)
@pytest.mark.parametrize("ps", [16, 64, 256])
def test_single_tokens(ps, heads, kvh, dh, dt, cache):
    lens = [1, 2, 15, 16, 17, 31, 32, 33, 63, 64, 65, 127, 128, 129, 257, 600]
    rng = np.random.default_rng(ps + heads)
    for seqs in (True, False):
        got, ref, mag = attend(rng, dt, lens, [1] * len(lens), ps, heads, kvh, dh, cache, seqs=seqs, rows_behind=2)
        check_attention(got, ref, mag, dt, (ps, heads, seqs), many([1], heads, kvh, cache), cache)


@pytest.mark.parametrize("cache", ["same", "e4m3"])
@pytest.mark.parametrize("dt", ["bf16", "f16"])
@pytest.mark.parametrize("heads,kvh,dh", HEADS)
@pytest.mark.parametrize("news,lens,ps", [
    ([2, 3, 4, 8], [2, 40, 64, 100], 16),
    ([1, 7, 0, 2], [300, 7, 0, 34], 32),
    ([16, 17, 5], [16, 50, 69], 64),
    ([33, 1, 64], [33, 130, 200], 128),
    ([100, 3], [150, 290], 16),
    ([8, 4, 8], [3, 0, 20], 16),       # rows before position 0
])
def test_pieces(news, lens, ps, heads, kvh, dh, dt, cache):
    rng = np.random.default_rng(sum(lens) + heads)
    got, ref, mag = attend(rng, dt, lens, news, ps, heads, kvh, dh, cache, pad=8, rows_behind=1)
    check_attention(got, ref, mag, dt, (news, heads), many(news, heads, kvh, cache), cache)


@pytest.mark.parametrize("cache", ["same", "e4m3"])
@pytest.mark.parametrize("heads,kvh,dh,news,lens,ps,width", [
    (5, 1, 128, [1], [5000], 64, 0),          # one sequence: its keys over many workgroups
    (2, 2, 64, [1, 1], [3000, 1], 16, 400),   # beside one with a single key, in a wide table
    (8, 1, 128, [3, 1], [2500, 40], 128, 0),
    (8, 2, 64, [40, 2], [2100, 900], 32, 0),
    (4, 1, 128, [150], [2300], 256, 20),
])
def test_long_contexts(heads, kvh, dh, news, lens, ps, width, cache):
    rng = np.random.default_rng(lens[0])
    for dt in ("bf16", "f16"):
        got, ref, mag = attend(rng, dt, lens, news, ps, heads, kvh, dh, cache, width=width, spread=2.0)
        check_attention(got, ref, mag, dt, (lens, dt), many(news, heads, kvh, cache), cache)


@pytest.mark.parametrize("cache", ["same", "e4m3"])
@pytest.mark.parametrize("heads,kvh,dh", [(8, 8, 64), (16, 16, 128), (16, 8, 64)])
@pytest.mark.parametrize("seqs", [1, 5, 70])
def test_many_heads_and_sequences(seqs, heads, kvh, dh, cache):
    """Every (sequence, head, row tile) is taken once, whatever order the workgroups go in."""
    rng = np.random.default_rng(seqs + heads)
    news = [int(x) for x in rng.integers(0, 40, seqs)]
    news[0] = 150 if seqs < 70 else 35
    lens = [n + int(c) for n, c in zip(news, rng.integers(0, 90, seqs))]
    got, ref, mag = attend(rng, "bf16", lens, news, 32, heads, kvh, dh, cache=cache)
    check_attention(got, ref, mag, "bf16", (seqs, heads, kvh), many=many(news, heads, kvh, cache), cache=cache)


@pytest.mark.parametrize("shape", ["rise", "fall", "large"])
@pytest.mark.parametrize("heads,kvh,dh,news,lens", [(4, 2, 128, [1, 1], [700, 90]), (2, 1, 64, [60, 9], [333, 200])])
def test_moving_maximum(shape, heads, kvh, dh, news, lens):
    """Logits that rise along the keys (every tile rescales), fall, or spread over hundreds."""
    rng = np.random.default_rng(dh)
    rows = sum(news)
    q = rng.standard_normal((rows, heads, dh)) * (4.0 if shape == "large" else 1.0)
    k = [rng.standard_normal((kvh, n, dh)) * (4.0 if shape == "large" else 1.0) for n in lens]
    if shape != "large":
        q[:, :, 0] = 3.0
        for s, n in enumerate(lens):
            k[s][:, :, 0] = (np.arange(n) if shape == "rise" else n - np.arange(n)) * 0.2 * np.sqrt(dh) / 3.0
    for dt in ("bf16", "f16"):
        got, ref, mag = attend(rng, dt, lens, news, 32, heads, kvh, dh, q=q.reshape(rows, -1), k=k)
        check_attention(got, ref, mag, dt, (shape, dt), many(news, heads, kvh))


@pytest.mark.parametrize("dt,c", [("f16", 1000.0), ("f16", 16376.0), ("bf16", 1024.0), ("bf16", 2.0 ** 45)])
@pytest.mark.parametrize("news", [[1], [70]])
def test_huge_logits(news, dt, c):
    """Logits of dh c^2: equal keys average, and one larger key takes all the weight."""
    dh, n = 128, 300
    rng = np.random.default_rng(3)
    q = np.full((news[0], dh), c)
    v = [rng.standard_normal((1, n, dh))]
    got, ref, mag = attend(rng, dt, [n], news, 64, 1, 1, dh, q=q, k=[np.full((1, n, dh), c)], v=v)
    check_attention(got, ref, mag, dt, "equal", many(news, 1, 1))
    k = [np.full((1, n, dh), c / 4)]
    k[0][0, 77] = c
    got, ref, _ = attend(rng, dt, [n], news, 64, 1, 1, dh, q=q, k=k, v=v)
    np.testing.assert_array_equal(got, ref)
    got, ref, _ = attend(rng, dt, [n], news, 64, 1, 1, dh, q=q, k=[-x for x in k], v=v)
    assert np.all(np.isfinite(got))


@pytest.mark.parametrize("cache", ["same", "e4m3"])
@pytest.mark.parametrize("news,heads", [([4], 2), ([40], 2), ([5], 12), ([90], 5)])
def test_values_that_are_not_finite_stay_with_the_rows_that_see_them(news, heads, cache):
    """A NaN or an infinity among the new keys or values reaches the rows from its position on, not those
    before it."""
    rng, dh, n, ps = np.random.default_rng(8), 64, news[0] + 37, 16
    first = n - news[0]  # position of row 0
    for where in (first, first + news[0] // 2, n - 1):
        for tensor, bad in (("v", np.nan), ("v", np.inf), ("k", np.nan)):
            if cache == "e4m3" and bad == np.inf:
                continue  # it has no infinity
            k, v = [rng.standard_normal((1, n, dh))], [rng.standard_normal((1, n, dh))]
            (v if tensor == "v" else k)[0][0, where, 5] = bad
            table, q_start, kv_len, pages = batch(rng, [n], news, ps)
            Q, Qv = rows16(rng.standard_normal((news[0], heads * dh)), "bf16")
            pool = [np.zeros((pages, 1, ps, dh)) for _ in range(2)]
            for x, src in zip(pool, (k, v)):
                for t in range(n):
                    x[table[0, t // ps], :, t % ps] = src[0][:, t]
            to = (lambda a: dev(a, torch.float32).to(E4M3)) if cache == "e4m3" else (lambda a: dev(a, DT["bf16"]))
            kd, vd = (to(x) for x in pool)
            ones = torch.ones((pages, 1), device="cuda") if cache == "e4m3" else None
            got = host64(zo.paged_attention(Q, kd, vd, dev(table), dev(kv_len), q_start=dev(q_start), max_q=news[0],
                                            k_scale=ones, v_scale=ones)).reshape(news[0], heads, dh)
            clean = [np.where(np.isfinite(host64(x)), host64(x), 0.0) for x in (kd, vd)]
            from oracle import paged as op
            ref, mag = op.paged_attention(Qv.reshape(news[0], heads, dh), clean, table, q_start, kv_len)
            sees = np.arange(first, n) >= where
            check_attention(got[~sees], ref[~sees], mag[~sees], "bf16", (tensor, bad, where), many(news, heads, 1, cache), cache)
            if tensor == "k":
                assert np.all(np.isnan(got[sees]))
            else:
                assert np.all(np.isnan(got[sees][..., 5]) if np.isnan(bad) else got[sees][..., 5] == np.inf)
                rest = np.arange(dh) != 5
                check_attention(got[sees][..., rest], ref[sees][..., rest], mag[sees][..., rest], "bf16", (tensor, bad, where),
                                many(news, heads, 1, cache), cache)


def _call(table, kv_len, q_start, max_q, pages=6, ps=16, rows=12, heads=2, dh=64):
    kc = torch.ones((pages, 1, ps, dh), dtype=torch.bfloat16, device="cuda")
    Q = torch.ones((rows, heads * dh), dtype=torch.bfloat16, device="cuda")
    out, flag = torch.full_like(Q, 7.0), torch.zeros(1, dtype=torch.int32, device="cuda")
    zo.paged_attention(Q, kc, kc, dev(np.array(table, np.int32)), dev(np.array(kv_len, np.int32)),
                       q_start=dev(np.array(q_start, np.int32)), max_q=max_q, out=out, bad_flag=flag)
    h = host64(out)
    assert np.all((h == h[:, :1]) | np.isnan(h) & np.isnan(h[:, :1]))
    return int(flag), ["n" if np.isnan(x) else int(x) for x in h[:, 0]]


def test_batches_that_break_the_rules():
    """The flag is raised; rows that attend to a page that is none are NaN, the others as ever (ones average to
    one); rows that no sequence has stay (7); padding is 0."""
    ok = [1] * 6 + [7] * 6
    assert _call([[4, 2]], [20], [0, 6], 6) == (0, ok)
    assert _call([[4, 2, 99]], [20], [0, 6], 12) == (0, ok)
    assert _call([[4, 6]], [20], [0, 6], 6) == (1, [1, 1, "n", "n", "n", "n"] + [7] * 6)
    assert _call([[-1, 2]], [20], [0, 6], 6) == (1, ["n"] * 6 + [7] * 6)
    assert _call([[4, 2]], [34], [0, 6], 6) == (1, [1, 1, 1, 1, "n", "n"] + [7] * 6)
    assert _call([[4, 2]], [20], [0, 6], 4) == (1, [1] * 4 + [7] * 8)
    assert _call([[4, 2], [1, 3]], [2, 3], [-5, 2, 5], 12) == (1, [1] * 5 + [7] * 7)
    assert _call([[4, 2], [1, 3]], [20, 13], [0, 2, 15], 12) == (1, [1] * 12)
    assert _call([[4, 2]], [3], [0, 6], 6) == (0, [0, 0, 0, 1, 1, 1] + [7] * 6)
    assert _call([[4, 2]], [-2 ** 31], [0, 6], 6) == (0, [0] * 6 + [7] * 6)
    # the same over splits: a bad page at the far end of a long table
    wide = [[i % 6 for i in range(200)]]
    wide[0][150] = -3
    assert _call(wide, [2500], [0, 2], 2) == (1, ["n", "n"] + [7] * 10)
    assert _call(wide, [2400], [0, 2], 2) == (0, [1, 1] + [7] * 10)
    assert _call(wide, [2403], [0, 6], 6) == (1, [1, 1, 1, "n", "n", "n"] + [7] * 6)


def test_queries_may_be_overwritten_and_rows_reused():
    """O over Q, and a call with no rows or no sequences does nothing."""
    rng = np.random.default_rng(4)
    table, q_start, kv_len, pages = batch(rng, [40, 700], [3, 2], 16)
    Q, _ = rows16(rng.standard_normal((5, 256)), "bf16")
    kc, vc = (dev(rng.standard_normal((pages, 1, 16, 128)), DT["bf16"]) for _ in range(2))
    args = dict(q_start=dev(q_start), max_q=3)
    want = host64(zo.paged_attention(Q, kc, vc, dev(table), dev(kv_len), **args))
    zo.paged_attention(Q, kc, vc, dev(table), dev(kv_len), out=Q, **args)
    np.testing.assert_array_equal(host64(Q), want)
    none = torch.empty((0, 256), dtype=torch.bfloat16, device="cuda")
    assert zo.paged_attention(none, kc, vc, dev(table), dev(kv_len), q_start=dev(0 * q_start), max_q=3).shape == (0, 256)
    zo.paged_attention(Q, kc, vc, dev(table)[:0], dev(kv_len)[:0], q_start=dev(q_start)[:1], max_q=3, out=Q)
    np.testing.assert_array_equal(host64(Q), want)
