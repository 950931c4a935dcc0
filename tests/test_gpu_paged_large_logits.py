"""zo_paged_attention at logits of some 2^20 in log2 units, where a running maximum is no longer folded into the exponent's
addend but subtracted first: keys on both sides of that border, whose weights all count, in one workgroup's range or
in ranges that are joined; 16-bit and 8-bit caches; few and many rows.  And one key that dwarfs all others."""
import numpy as np
import pytest
import torch

from _paged import DT, attend, check_attention, host64

pytestmark = pytest.mark.gpu
DH, PS = 64, 16


def near(dt, border, n, rng, first, scale):
    """A query and keys whose dot products are whole numbers (exact in fp32) next to `border`: `first` of the keys 24
    below it, the others 24 above, all +- 16.  Key values are e4m3 codes times `scale` = 8."""
    r = lambda x: float(host64(torch.tensor([float(round(x))]).to(DT[dt]))[0])  # noqa: E731
    k = np.zeros((1, n, DH))
    q = np.zeros(DH)
    k[..., 0], k[..., 1], k[..., 2] = 352 * scale, 256 * scale, scale
    q[0] = r(border / k[0, 0, 0])
    q[1] = r((border - q[0] * k[0, 0, 0]) / k[0, 0, 1])
    q[2] = r((border - q[0] * k[0, 0, 0] - q[1] * k[0, 0, 1]) / scale)
    q[3] = q[4] = 1.0
    k[0, :, 3] = scale * rng.integers(-2, 3, n)
    k[0, :, 4] = scale * np.where(np.arange(n) < first, -3, 3)
    s = k[0] @ q
    assert np.all(s == np.round(s)) and np.all(np.abs(s - border) <= 48) and np.all(np.abs(s) < 2 ** 24)
    assert np.max(s[:first], initial=-np.inf) < border < np.min(np.sort(s[first:])[-8:])
    return q, k


@pytest.mark.parametrize("cache", ["same", "e4m3"])
@pytest.mark.parametrize("dt", ["bf16", "f16"])
@pytest.mark.parametrize("news", [[1], [70]])
@pytest.mark.parametrize("n,first", [(400, 200), (2000, 1000), (2000, 1990), (2000, 0)])
def test_both_sides_of_the_border(n, first, news, dt, cache):
    rng = np.random.default_rng(n + first)
    border = 2.0 ** 20 * np.sqrt(DH) / 1.4426950408889634
    q, k = near(dt, border, n, rng, first, 8)
    if cache == "e4m3":
        got, ref, mag = _attend8(rng, dt, n, news, q, k)
    else:
        got, ref, mag = attend(rng, dt, [n], news, PS, 1, 1, DH, q=np.tile(q, (news[0], 1)), k=[k])
    check_attention(got, ref, mag, dt, (n, first))


def _attend8(rng, dt, n, news, q, k):
    """attend() with page scales of 8 for the keys, so that their values are the given ones."""
    import paper_2608_15665_amd as zo
    from _paged import E4M3, batch, dev, rows16
    from oracle import paged as op
    table, q_start, kv_len, pages = batch(rng, [n], news, PS)
    codes = [np.full((pages, 1, PS, DH), np.nan), np.full((pages, 1, PS, DH), np.nan)]
    v = op.nearest_e4m3(np.clip(rng.standard_normal((1, n, DH)) * 100, -448, 448))
    for t in range(n):
        codes[0][table[0, t // PS], :, t % PS] = k[:, t] / 8
        codes[1][table[0, t // PS], :, t % PS] = v[:, t]
    scl = [np.full((pages, 1), 8.0), rng.uniform(0.005, 0.02, (pages, 1)).astype(np.float32).astype(np.float64)]
    kc, vc = (dev(c, torch.float32).to(E4M3) for c in codes)
    Q, Qv = rows16(np.tile(q, (news[0], 1)), dt)
    got = host64(zo.paged_attention(Q, kc, vc, dev(table), dev(kv_len), q_start=dev(q_start), max_q=news[0],
                                    k_scale=dev(scl[0], torch.float32), v_scale=dev(scl[1], torch.float32)))
    held = [np.nan_to_num(host64(c)) for c in (kc, vc)]
    ref, mag = op.paged_attention(Qv.reshape(-1, 1, DH), held, table, q_start, kv_len, scl)
    return got.reshape(-1, 1, DH), ref, mag


@pytest.mark.parametrize("dt,c", [("f16", 1000.0), ("bf16", 1024.0), ("bf16", 2.0 ** 45)])
@pytest.mark.parametrize("news", [[1], [70]])
@pytest.mark.parametrize("at", [0, 777, 1800])
def test_one_key_of_many_ranges(at, news, dt, c):
    """Its range's maximum is subtracted first, the other ranges' is 0: they add nothing to the joined row."""
    n = 2000
    rng = np.random.default_rng(at)
    k = [np.zeros((1, n, DH))]
    k[0][0, at] = c
    got, ref, _ = attend(rng, dt, [n], news, PS, 1, 1, DH, q=np.full((news[0], DH), c), k=k)
    np.testing.assert_array_equal(got, ref)
