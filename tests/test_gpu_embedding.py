"""The embedding lookup and its table's gradient against float64, at the sizes and tokens where they can go wrong."""
import numpy as np
import pytest
import torch

import paper_2608_15665_amd as zo
from _ends import DT, NEAR, TINY, U, U32, bits, host, i32, put, within
from oracle import ends

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dt", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("rows,vocab,d", [(1, 1, 8), (1, 500, 4096), (3, 7, 24), (64, 333, 72), (257, 1000, 1000),
                                          (1000, 50, 520), (40, 300, 5120), (5, 20, 20008)])
@pytest.mark.parametrize("scale", [1.0, 71.5, -0.3])
def test_lookup(dt, rows, vocab, d, scale):
    rng = np.random.default_rng(rows + d)
    E, e = put(rng.standard_normal((vocab, d)), dt)
    ids = rng.integers(0, vocab, rows)
    ids[rng.random(rows) < 0.1] = -1
    ids[0], ids[-1] = 0, vocab - 1
    behind = torch.full((rows * d + 64,), 3.0, dtype=DT[dt], device="cuda")
    out = zo.embedding(i32(ids), E, scale=scale, out=behind[:rows * d].view(rows, d))
    s = float(np.float32(scale))
    want = ends.embedding(ids, e, s)
    # One fp32 product, then the type's rounding.
    within(host(out), want, (U[dt] * np.abs(want) + U32 * np.abs(want)) * NEAR + TINY[dt], dt)
    if scale == 1.0:
        np.testing.assert_array_equal(host(out), want)
    assert (behind[rows * d:] == 3.0).all()


def test_lookup_of_a_shape_and_of_nothing():
    E = torch.arange(80, dtype=torch.float32, device="cuda").view(10, 8)
    ids = torch.tensor([[1, 2, 3], [9, -5, 0]], dtype=torch.int32, device="cuda")
    out = zo.embedding(ids, E)
    assert out.shape == (2, 3, 8) and (out[1, 1] == 0).all() and (out[1, 0] == E[9]).all()
    assert zo.embedding(ids[:0], E).shape == (0, 3, 8)


def test_tokens_that_the_table_lacks():
    E = torch.ones(10, 16, device="cuda", dtype=torch.bfloat16)
    flag = torch.zeros(1, dtype=torch.int32, device="cuda")
    zo.embedding(i32([0, 9, -1]), E, bad_flag=flag)
    assert flag.item() == 0
    out = zo.embedding(i32([0, 10, 9, 2 ** 31 - 1, -2 ** 31]), E, bad_flag=flag)
    assert flag.item() == 1
    assert out[1].isnan().all() and out[3].isnan().all() and (out[[0, 2]] == 1).all() and (out[4] == 0).all()
    dE = torch.zeros(10, 16, device="cuda")
    flag.zero_()
    zo.embedding_backward(i32([0, 10, 9, 2 ** 31 - 1, -2 ** 31]), torch.ones(5, 16, device="cuda"), 10, out=dE, bad_flag=flag)
    assert flag.item() == 1 and dE.sum().item() == 32 and (dE[[0, 9]] == 1).all()
    flag.zero_()
    zo.embedding_backward(i32([0, -3]), torch.ones(2, 16, device="cuda"), 10, out=dE, bad_flag=flag)
    assert flag.item() == 0 and dE.sum().item() == 16


def _tokens(rng, form, rows, vocab):
    if form == "same":
        return np.full(rows, vocab - 1)
    if form == "none":
        return np.full(rows, -1)
    if form == "each":
        return rng.permutation(rows) % vocab
    ids = np.minimum((np.exp(rng.random(rows) * np.log(vocab + 1)) - 1).astype(np.int64), vocab - 1)  # as text has them
    ids[rng.random(rows) < 0.05] = -1
    return ids


SIZES = [(1, 1, 8), (1, 40000, 512), (31, 3, 24), (32, 40, 72), (33, 40, 520), (63, 2, 8), (64, 1000, 1024), (65, 511, 8),
         (200, 512, 136), (257, 600, 8), (700, 50000, 264), (1024, 7, 64), (2047, 513, 24), (2049, 5000, 512),
         (5000, 262143, 8), (4097, 262144, 16), (8192, 3000, 8), (8193, 3000, 8), (9000, 300, 1032)]


@pytest.mark.parametrize("dt,out", [("f32", "f32"), ("bf16", "bf16"), ("bf16", "f32"), ("f16", "f16"), ("f16", "f32")])
@pytest.mark.parametrize("rows,vocab,d", SIZES)
@pytest.mark.parametrize("form", ["text", "same"])
def test_gradient(dt, out, rows, vocab, d, form):
    rng = np.random.default_rng(rows * 7 + d)
    ids = _tokens(rng, form, rows, vocab)
    g, gv = put(0.1 * rng.standard_normal((rows, d)), dt)
    scale = float(np.float32(1.7))
    G, mag, count = ends.embedding_backward(ids, gv, vocab, scale)
    # n rows added in fp32 in any order: (n - 1) roundings of at most the sum of magnitudes; the product's, the output's.
    tol = (np.maximum(count - 1, 0)[:, None] * U32 * mag + U32 * np.abs(G) + U[out] * np.abs(G)) * NEAR + TINY[out]
    behind = torch.full((vocab * d + 64,), 5.0, dtype=DT[out], device="cuda")
    dE = zo.embedding_backward(i32(ids), g, vocab, scale=scale, out=behind[:vocab * d].view(vocab, d))
    within(host(dE), G, tol, "dense")
    assert (behind[vocab * d:] == 5.0).all()
    again = zo.embedding_backward(i32(ids), g, vocab, scale=scale, out=torch.full_like(dE, 9.0))
    np.testing.assert_array_equal(bits(dE), bits(again))
    # Added: rows of other tokens keep their bits.
    base, bv = put(rng.standard_normal((vocab, d)), out)
    kept = bits(base)
    zo.embedding_backward(i32(ids), g, vocab, scale=scale, out=base, accumulate=True)
    want = bv + G
    within(host(base), want, tol + (U32 + U[out]) * np.abs(want) * NEAR, "added")
    np.testing.assert_array_equal(bits(base)[count == 0], kept[count == 0])


@pytest.mark.parametrize("form", ["none", "each"])
@pytest.mark.parametrize("rows,vocab,d", [(1, 9, 16), (100, 300, 40), (3000, 3000, 16)])
def test_gradient_of_padding_and_of_each_token_once(form, rows, vocab, d):
    rng = np.random.default_rng(5)
    ids = _tokens(rng, form, rows, vocab)
    g, gv = put(rng.standard_normal((rows, d)), "f32")
    got = zo.embedding_backward(i32(ids), g, vocab)
    np.testing.assert_array_equal(host(got), ends.embedding_backward(ids, gv, vocab, 1.0)[0])  # nothing to round


def test_gradient_without_rows():
    dE = torch.full((6, 8), 2.0, device="cuda")
    none, g = torch.empty(0, dtype=torch.int32, device="cuda"), torch.empty(0, 8, device="cuda")
    zo.embedding_backward(none, g, 6, out=dE, accumulate=True)
    assert (dE == 2).all()
    zo.embedding_backward(none, g, 6, out=dE)
    assert (dE == 0).all()


def test_gradient_keeps_what_is_not_finite_to_its_token():
    g = torch.ones(70, 8, device="cuda")
    g[3, 1], g[60, 2] = float("nan"), float("inf")
    ids = torch.arange(70, dtype=torch.int32, device="cuda") % 7
    ids[5] = -1
    g[5] = float("nan")  # padding
    dE = zo.embedding_backward(ids, g, 7)
    bad = ~torch.isfinite(dE)
    assert bad.sum().item() == 2 and dE[3, 1].isnan() and dE[60 % 7, 2] == float("inf")


@pytest.mark.parametrize("n,vocab,d", [(131071, 70000, 8), (70001, 5000, 520), (66000, 3, 520)])
def test_many_rows_of_few_tokens_are_sorted(n, vocab, d):
    """Tens of sorting tiles, runs over thousands of chunks; whole numbers, so that every sum is exact."""
    rng = np.random.default_rng(8)
    ids = _tokens(rng, "text", n, vocab)
    ids[::3] = vocab - 1
    g = rng.integers(-8, 9, (n, d))
    dE = zo.embedding_backward(i32(ids), torch.tensor(g, dtype=torch.float32, device="cuda"), vocab)
    want = np.zeros((vocab + 1, d))
    order = np.argsort(ids, kind="stable")
    first = np.flatnonzero(np.diff(ids[order], prepend=-2))
    want[ids[order][first]] = np.add.reduceat(g[order].astype(np.float64), first)  # padding, -1, is the last row
    np.testing.assert_array_equal(host(dE), want[:vocab])


def test_tables_past_4_gib():
    """Rows whose offset passes 2^32 elements."""
    vocab, d = (1 << 20) + 3, 4104
    if torch.cuda.mem_get_info()[0] < 24 << 30:
        pytest.skip("needs 24 GB")
    E = torch.empty(vocab, d, dtype=torch.bfloat16, device="cuda")
    ids = [0, vocab - 1, (1 << 20) - 5, 77, vocab - 1]
    for k, v in enumerate(ids):
        E[v] = float(k + 1)
    out = zo.embedding(i32(ids), E)
    for k, v in enumerate(ids):
        assert (out[k] == E[v]).all()
    for v in set(ids):
        E[v] = 1.0
    zo.embedding_backward(i32(ids), torch.ones(5, d, dtype=torch.bfloat16, device="cuda"), vocab, out=E, accumulate=True)
    for v in set(ids):
        assert (E[v] == 1 + ids.count(v)).all()


def test_a_result_of_more_workgroups_than_a_row_of_the_grid():
    """2^31 words and some: 2^22 workgroups and more."""
    n, d = (1 << 22) + 77, 4096
    if torch.cuda.mem_get_info()[0] < 48 << 30:
        pytest.skip("needs 48 GB")
    E = torch.randn(1000, d, device="cuda").bfloat16()
    ids = torch.randint(-1, 1000, (n,), device="cuda").int()
    H = zo.embedding(ids, E)
    for a in [*range(0, n, 1 << 20), n - 1000]:
        i = ids[a:a + 5000].long()
        assert (H[a:a + 5000] == torch.where((i < 0)[:, None], 0.0, E[i.clamp(min=0)].float()).bfloat16()).all()
