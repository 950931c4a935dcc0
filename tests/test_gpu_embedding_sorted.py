"""The table's gradient where tokens are sorted: by one workgroup, in tiles, in hundreds of tiles; tokens that the table lacks;
dense and added, in every type, with 16, 32 and 64 positions a wave."""
import numpy as np
import pytest
import torch

import paper_2608_15665_amd as zo
from _ends import DT, NEAR, TINY, U, bits, host, i32, put, within

pytestmark = pytest.mark.gpu


def _sums(ids, g, vocab):
    """Sums of the rows of g by token, exact for whole numbers; tokens outside 0 .. vocab - 1 are left out."""
    order = np.argsort(ids, kind="stable")
    first = np.flatnonzero(np.diff(ids[order], prepend=ids[order[0]] - 1))
    tokens = ids[order][first]
    sums = np.add.reduceat(g[order].astype(np.float64), first)
    here = (tokens >= 0) & (tokens < vocab)
    G, count = np.zeros((vocab, g.shape[1])), np.zeros(vocab, np.int64)
    G[tokens[here]] = sums[here]
    count[tokens[here]] = np.diff(np.append(first, len(ids)))[here]
    return G, count


# One workgroup sorts (16 and 32 positions a wave), tiles in two passes and three, 64 positions a wave.
SIZES = [(600, 40, 136), (1000, 5000, 8), (5000, 3000, 520), (9000, 2000, 72), (20000, 262200, 8), (70001, 5000, 520)]


@pytest.mark.parametrize("rows,vocab,d", SIZES)
@pytest.mark.parametrize("dt,out", [("f32", "f32"), ("bf16", "bf16"), ("bf16", "f32"), ("f16", "f16"), ("f16", "f32")])
@pytest.mark.parametrize("add", [False, True])
def test_every_path_with_tokens_that_the_table_lacks(rows, vocab, d, dt, out, add):
    """Whole numbers of at most 8 a row: the fp32 sums are exact, and the output is rounded once."""
    rng = np.random.default_rng(rows)
    ids = np.minimum(np.exp(rng.random(rows) * np.log(vocab + 1.0)).astype(np.int64) - 1, vocab - 1)
    ids[::5] = vocab - 1
    bad = rng.choice(rows, 37, replace=False)
    ids[bad] = np.resize([vocab, vocab + 1, 2 ** 31 - 1, -1, -2 ** 31], 37)
    g = rng.integers(-8, 9, (rows, d))
    x, _ = put(g, dt)
    G, count = _sums(ids, g, vocab)
    base, bv = put(rng.integers(-100, 101, (vocab, d)), out)
    kept = bits(base)
    flag = torch.zeros(1, dtype=torch.int32, device="cuda")
    zo.embedding_backward(i32(ids), x, vocab, out=base, accumulate=add, bad_flag=flag)
    assert flag.item() == 1
    want = G + bv if add else G
    within(host(base), want, U[out] * np.abs(want) * (out != "f32") * NEAR + TINY[out], "sums")
    if add:
        np.testing.assert_array_equal(bits(base)[count == 0], kept[count == 0])
    # Without them the flag stays, and without a flag the sums do.
    good = ids.copy()
    good[bad] = -3
    again = torch.from_numpy(bv).to(DT[out]).cuda()
    flag.zero_()
    zo.embedding_backward(i32(good), x, vocab, out=again, accumulate=add, bad_flag=flag)
    assert flag.item() == 0
    np.testing.assert_array_equal(bits(again), bits(base))
    again = torch.from_numpy(bv).to(DT[out]).cuda()
    zo.embedding_backward(i32(ids), x, vocab, out=again, accumulate=add)
    np.testing.assert_array_equal(bits(again), bits(base))


@pytest.mark.parametrize("add", [False, True])
def test_hundreds_of_tiles(add):
    """More than 2^20 tokens, three sorting passes over 587 tiles; one token fills a third of them."""
    rows, vocab, d = 1200001, 300000, 8
    rng = np.random.default_rng(2)
    ids = rng.integers(-3, vocab + 3, rows)
    ids[1::3] = 77
    g = rng.integers(-2, 3, (rows, d))  # sums of 400000 stay below 2^24
    G, count = _sums(ids, g, vocab)
    base, bv = put(rng.integers(-9, 10, (vocab, d)), "f32")
    zo.embedding_backward(i32(ids), put(g, "bf16")[0], vocab, out=base, accumulate=add)
    np.testing.assert_array_equal(host(base), G + bv if add else G)
