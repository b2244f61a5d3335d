"""The embedding's gradient where a few tokens have nearly all columns, and with the largest vocabulary."""
import pytest

from token_helpers import HALF_STEP, SMALLEST, TYPES, U, torch_type


def _gradient(ids, G, vocab, dtype, scale):
    import torch
    from paper_2009_13977_amd import binding as B
    d, m = G.shape
    dTable = torch.full((vocab, d), float("nan"), device="cuda", dtype=torch_type(dtype))
    B.fasth_embed_backward(ids, G, dTable, B.new_workspace(B.fasth_embed_workspace_bytes(vocab, d, m)).fill_(0xFF), scale)
    return dTable


def _within(got, want, size, n, dtype):
    """n terms in some order and the scale: as many roundings of the sum of their sizes, and that to the type."""
    bound = (n + 1) * U * size
    return bool(((got.double() - want).abs() <= bound + HALF_STEP[dtype] * (want.abs() + bound) + SMALLEST[dtype]).all())


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("vocab,d,m", [(64, 64, 16384), (64, 1024, 16384), (2, 1030, 65535), (256, 1024, 16384), (65, 63, 30001)])
def test_few_distinct_tokens(vocab, d, m, dtype):
    import torch
    gen = torch.Generator(device="cuda")
    gen.manual_seed(vocab + d)
    ids = torch.randint(-1, vocab, (m,), device="cuda", generator=gen)
    G = torch.randn(d, m, device="cuda", generator=gen) * 1e-2
    got = _gradient(ids, G, vocab, dtype, 0.75)
    known = (ids >= 0).nonzero()[:, 0]
    rows = 0.75 * G.double()[:, known].t()
    zeros = torch.zeros(vocab, d, device="cuda", dtype=torch.float64)
    want, size = zeros.index_add(0, ids[known], rows), zeros.index_add(0, ids[known], rows.abs())
    n = torch.bincount(ids[known], minlength=vocab)[:, None]
    assert _within(got, want, size, n, dtype)
    again = _gradient(ids, G, vocab, dtype, 0.75)
    assert torch.equal(got, again)


@pytest.mark.gpu
def test_largest_vocabulary_and_mini_batch():
    """2^24 tokens, 65535 columns: frequent ones, the first and the last, and all others zero."""
    import torch
    vocab, d, m = 1 << 24, 5, 65535
    gen = torch.Generator(device="cuda")
    gen.manual_seed(1)
    ids = torch.randint(0, vocab, (m,), device="cuda", generator=gen)
    ids[::3], ids[1], ids[m - 1], ids[5] = vocab - 1, 0, 7, -1
    G = torch.randn(d, m, device="cuda", generator=gen)
    got = _gradient(ids, G, vocab, "fp32", 1.0)
    known = (ids >= 0).nonzero()[:, 0]
    rows = G.double()[:, known].t()
    tokens, at = ids[known].unique(return_inverse=True)
    zeros = torch.zeros(tokens.numel(), d, device="cuda", dtype=torch.float64)
    want, size = zeros.index_add(0, at, rows), zeros.index_add(0, at, rows.abs())
    assert _within(got[tokens], want, size, torch.bincount(at)[:, None], "fp32")
    got[tokens] = 0
    assert not got.any()
