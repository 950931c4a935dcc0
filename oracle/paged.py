"""The paged key/value cache and the attention over it, one position at a time, in float64.

A batch is (q_start, kv_len, table): sequence s has the rows q_start[s] .. q_start[s + 1] - 1 of the row
tensors, its last positions of kv_len[s]; position t is slot t % ps of page table[s][t // ps].  Caches are
arrays of pages x kv_heads x ps x dh; with 8 bits they hold code values, and scales of pages x kv_heads."""
import numpy as np

E4M3_MAX = 448.0


def nearest_e4m3(x):
    """The nearest value of 4 exponent bits (bias 7) and 3 mantissa bits, ties to even: steps of 2^(e - 3)
    for 2^e <= |x| < 2^(e + 1), and of 2^-9 below 2^-6."""
    x = np.asarray(x, np.float64)
    _, e = np.frexp(np.where(x == 0, 1.0, x))
    step = np.ldexp(1.0, np.maximum(e - 1, -6) - 3)
    return np.round(x / step) * step


def need_scale(amax):
    """The smallest power of two s with amax <= 448 s, within [2^-126, 2^120]."""
    s = 2.0 ** -126
    while amax > E4M3_MAX * s and s < 2.0 ** 120:
        s *= 2
    return s


def rotate(x, p, base):
    """x: ... x dh at position p: pairs (i, i + dh / 2) turned by p base^(-2 i / dh)."""
    half = x.shape[-1] // 2
    ang = p * base ** (-2.0 * np.arange(half, dtype=np.float64) / x.shape[-1])
    a, b = x[..., :half], x[..., half:]
    return np.concatenate([a * np.cos(ang) - b * np.sin(ang), b * np.cos(ang) + a * np.sin(ang)], -1)


def rows_of(s, q_start, kv_len):
    """(row, position) of sequence s's rows."""
    r0, r1 = (s, s + 1) if q_start is None else (int(q_start[s]), int(q_start[s + 1]))
    return [(r, int(kv_len[s]) - (r1 - r)) for r in range(r0, r1)]


def kv_append(K, V, caches, table, q_start, kv_len, base=None, scales=None):
    """caches (K's, V's) and, with 8 bits, scales as they are after the call.  K, V: rows x kv_heads x dh."""
    out = [c.copy() for c in caches]
    scl = None if scales is None else [s.copy() for s in scales]
    ps = caches[0].shape[2]
    for s in range(len(kv_len)):
        stored = {}
        for r, p in rows_of(s, q_start, kv_len):
            if p >= 0:
                stored.setdefault(p // ps, []).append((r, p))
        for j, rp in stored.items():
            page = int(table[s][j])
            for x, cache, scale in zip((K, V), out, scl or (None, None)):
                vals = np.stack([rotate(x[r], p, base) if base and x is K else x[r] for r, p in rp])
                slots = [p % ps for _, p in rp]
                if scale is None:
                    cache[page][:, slots] = vals.transpose(1, 0, 2)
                    continue
                for h in range(vals.shape[1]):
                    mags = np.abs(vals[:, h])
                    to = need_scale(np.max(mags[np.isfinite(mags)], initial=0.0))
                    if slots[0] > 0:
                        to = max(to, scale[page][h])
                        if to > scale[page][h]:
                            kept = cache[page][h][:slots[0]]
                            cache[page][h][:slots[0]] = nearest_e4m3(kept * (scale[page][h] / to))
                    scale[page][h] = to
                    with np.errstate(invalid="ignore"):
                        q = np.where(np.isfinite(vals[:, h]), nearest_e4m3(np.where(np.isfinite(vals[:, h]), vals[:, h], 0) / to),
                                     np.nan)
                    cache[page][h][slots] = q
    return (out, scl)


def paged_attention(Q, caches, table, q_start, kv_len, scales=None):
    """Rows of heads x dh outputs (rows of no sequence: NaN), and the same averages of |V|."""
    rows, heads, dh = Q.shape
    kvh, ps = caches[0].shape[1:3]
    out = np.full(Q.shape, np.nan)
    mag = np.full(Q.shape, np.nan)
    for s in range(len(kv_len)):
        n = max(int(kv_len[s]), 0)
        pages = [int(table[s][j]) for j in range(-(-n // ps))]
        kv = []
        for i in range(2):
            x = [caches[i][p] * (1.0 if scales is None else scales[i][p][:, None, None]) for p in pages]
            kv.append(np.concatenate(x, 1)[:, :n] if x else np.zeros((kvh, 0, dh)))
        for r, p in rows_of(s, q_start, kv_len):
            if p < 0:
                out[r] = mag[r] = 0.0
                continue
            for h in range(heads):
                k, v = (x[h // (heads // kvh)][:p + 1] for x in kv)
                z = k @ Q[r, h] / np.sqrt(dh)
                w = np.exp(z - np.max(z))
                w /= np.sum(w)
                out[r, h], mag[r, h] = w @ v, w @ np.abs(v)
    return out, mag
