"""fasth_embed and fasth_embed_backward against the fp64 definition, entry by entry."""
import numpy as np
import pytest

from oracle import tokens as tok
from token_helpers import TYPES, U, assert_within, host, normal, tokens, torch_type

SHAPES = [(1, 1, 1), (7, 3, 5), (64, 64, 64), (65, 65, 65), (100, 130, 77), (1000, 33, 513), (50, 784, 1001), (3, 20, 4000),
          (5000, 64, 65), (70001, 9, 300), (257, 5, 65535), (30, 16384, 3), (200000, 4, 128)]


def _run(table, ids, G, scale):
    import torch
    from paper_2009_13977_amd import binding as B
    vocab, d = table.shape
    m = ids.shape[0]
    X = torch.full((d, m), float("nan"), device="cuda")
    B.fasth_embed(table, ids, X, scale)
    dTable = torch.full_like(table, float("nan"))
    ws = B.new_workspace(B.fasth_embed_workspace_bytes(vocab, d, m)).fill_(0xFF)
    B.fasth_embed_backward(ids, G, dTable, ws, scale)
    torch.cuda.synchronize()
    return X, dTable


def _check(table, t64, ids, i64, G, g64, dtype, scale=1.25):
    X, dTable = _run(table, ids, G, scale)
    vocab = table.shape[0]
    want = tok.embed(t64, i64, scale)
    assert_within(X, want, 0.0, "fp32", "X")
    # a sum of n terms is off by at most n roundings of the sum of the terms' sizes; then the product with the scale
    n = np.bincount(i64[(i64 >= 0) & (i64 < vocab)], minlength=vocab)[:, None]
    # (the terms' sizes are |scale| |g|: a bound is no negative number)
    size = tok.embed_gradient(vocab, i64, np.abs(g64), abs(scale))
    assert_within(dTable, tok.embed_gradient(vocab, i64, g64, scale), (n + 1) * U * size, dtype, "dTable")


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("vocab,d,m", SHAPES)
def test_both_directions(vocab, d, m, dtype):
    table, t64 = normal(1, vocab, d, dtype=dtype)
    ids, i64 = tokens(2, vocab, m, bits=32 if m % 2 else 64)
    G, g64 = normal(3, d, m)
    _check(table, t64, ids, i64, G, g64, dtype)


@pytest.mark.gpu
@pytest.mark.parametrize("which", ["one token", "no token", "all different", "in turn", "far numbers"])
def test_distributions_of_tokens(which):
    import torch
    vocab, d, m = 1500, 70, 1400
    i64 = {"one token": np.full(m, 1499), "no token": np.full(m, -1), "all different": np.random.default_rng(0).permutation(vocab)[:m],
           "in turn": np.arange(m) % 3 * 700,
           # 64-bit numbers whose lower halves are rows of the table are none
           "far numbers": np.where(np.arange(m) % 2, np.arange(m) + 2 ** 32, -(2 ** 62) + 5)}[which].astype(np.int64)
    table, t64 = normal(4, vocab, d)
    G, g64 = normal(5, d, m)
    _check(table, t64, torch.from_numpy(i64).cuda(), i64, G, g64, "fp32", scale=-3.0)


@pytest.mark.gpu
def test_tables_beyond_32_bits():
    """A table of 2^31 + 16384 * 9 entries in 16 bits: its last rows lie beyond 2^32 bytes."""
    import torch
    vocab, d, m = 131081, 16384, 70
    table = torch.zeros(vocab, d, device="cuda", dtype=torch.bfloat16)
    table[-5:], t64 = normal(1, 5, d, dtype="bf16")
    ids = torch.arange(m, device="cuda") % 5 + vocab - 5
    ids[3], ids[4] = 7, -1
    G, g64 = normal(2, d, m)
    X, dTable = _run(table, ids, G, 1.0)
    i64 = ids.cpu().numpy()
    low = np.where(i64 >= vocab - 5, i64 - (vocab - 5), -1)
    np.testing.assert_array_equal(host(X), tok.embed(t64, low, 1.0))
    # 14 terms at most: as many roundings of the sum of their sizes
    assert_within(dTable[-5:], tok.embed_gradient(5, low, g64, 1.0), 15 * U * tok.embed_gradient(5, low, np.abs(g64), 1.0), "bf16", "dTable")
    assert (dTable[7].double().cpu() == G[:, 3].to(torch.bfloat16).double().cpu()).all()
    dTable[-5:] = 0
    dTable[7] = 0
    assert not dTable.any()


@pytest.mark.gpu
def test_repeated_calls_give_the_same_bits():
    table, _ = normal(6, 900, 100)
    ids, _ = tokens(7, 900, 3000)
    G, _ = normal(8, 100, 3000)
    first = _run(table, ids, G, 1.0)
    for _ in range(3):
        again = _run(table, ids, G, 1.0)
        assert all((a == b).all() for a, b in zip(first, again))


@pytest.mark.gpu
def test_infinite_and_nan_rows_stay_in_their_columns():
    import torch
    table, t64 = normal(9, 10, 80)
    table[3], table[4] = float("inf"), float("nan")
    ids = torch.tensor([3, 0, 4, 1, 3, -1], device="cuda")
    G, _ = normal(10, 80, 6)
    G[:, 1] = float("nan")
    X, dTable = _run(table, ids, G, 1.0)
    X, dTable = host(X), host(dTable)
    assert np.isposinf(X[:, [0, 4]]).all() and np.isnan(X[:, 2]).all() and (X[:, 5] == 0).all()
    assert np.isnan(dTable[0]).all() and np.isfinite(dTable[1:]).all()


@pytest.mark.gpu
def test_refuses_what_it_cannot_take():
    import torch
    from paper_2009_13977_amd import binding as B
    table, _ = normal(11, 10, 8)
    ids, X = torch.zeros(4, dtype=torch.int64, device="cuda"), torch.empty(8, 4, device="cuda")
    for bad in (ids.cpu(), ids.to(torch.int16), ids.float(), torch.zeros(8, dtype=torch.int64, device="cuda")[::2], ids[:3]):
        with pytest.raises(ValueError):
            B.fasth_embed(table, bad, X)
    with pytest.raises(TypeError):
        B.fasth_embed(table, [0, 1, 2, 3], X)
    with pytest.raises(ValueError):
        B.fasth_embed(table.double(), ids, X)
    with pytest.raises(ValueError):
        B.fasth_embed(table, ids, torch.empty(4, 8, device="cuda").t())
    with pytest.raises(ValueError):
        B.fasth_embed(table, ids, X.to(torch.bfloat16))
    G, dTable = torch.empty_like(X), torch.empty_like(table)
    small = B.new_workspace(B.fasth_embed_workspace_bytes(10, 8, 4) - 16)
    with pytest.raises(B.FasthError) as e:
        B.fasth_embed_backward(ids, G, dTable, small)
    assert e.value.code == B.FASTH_EWORKSPACE
