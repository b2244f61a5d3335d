"""fasth_norm and its gradient over columns from 1e-30 to 1e17, and with an eps that leaves a column of zeros a large 1 / rms."""
import numpy as np
import pytest

from oracle import tokens as tok
from token_helpers import TYPES, U, assert_within, host, normal, torch_type

SIZES = (1.0, 1e-30, 1e15, 0.0, 1e-15, 1e12, 1e17, 1e-7, 1e6, 4e12, 1e-19)
# the ways in which the backward call covers a mini-batch: a column per thread, four of them, and split over 16, 64 and 128
SHAPES = [(200, 3), (9001, 2), (100, 1100), (130, 11), (300, 70), (700, 600)]


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("eps", [1e-5, 1e-30, 2e-38])
@pytest.mark.parametrize("d,m", SHAPES)
def test_columns_of_all_sizes(d, m, eps, dtype):
    import torch
    from paper_2009_13977_amd import binding as B
    sizes = torch.tensor(SIZES * (m // len(SIZES) + 2), dtype=torch.float64, device="cuda")
    for first in range(0, len(SIZES), m):  # (few columns: all sizes in turn)
        X, _ = normal(1, d, m)
        X = (X.double() * sizes[first:first + m]).float()
        w, w64 = normal(3, d)
        G, g64 = normal(4, d, m, dtype=dtype)
        Y, rstd = torch.full((d, m), float("nan"), device="cuda", dtype=torch_type(dtype)), torch.full((m,), float("nan"), device="cuda")
        B.fasth_norm(X, w, Y, rstd, eps)
        eps32 = float(np.float32(eps))
        # A sum of at most 16 terms per thread in one pass, or of d / 64 partial sums of 8 in a row; then 6 lanes, 16 waves or
        # 4 waves and 32 splits: d / 64 + 45 roundings one after the other, half of that and some 6 more for 1 / root. Squares
        # below 2^-126 lose up to 2^-150 each: no more than U of an eps of 2^-126
        chain = d / 64 + 45
        rel = (chain / 2 + 7) * U
        x64 = host(X)
        want, want_rstd = tok.norm(x64, w64, eps32)
        assert_within(rstd, want_rstd, rel * want_rstd, "fp32", "rstd")
        # (the product with rstd may be below 2^-126, and so off by 2^-150, before the weight makes it larger)
        assert_within(Y, want, (rel + 2 * U) * np.abs(want) + 2.0 ** -150 * (1 + np.abs(w64))[:, None], dtype, "Y")
        dX, dw = torch.full_like(X, float("nan")), torch.full_like(w, float("nan"))
        ws = B.new_workspace(B.fasth_norm_workspace_bytes(d, m)).fill_(0xFF)
        B.fasth_norm_backward(G, X, w, rstd, dX, dw, ws)
        want, want_dw = tok.norm_gradient(g64, x64, w64, eps32)
        p, u = np.abs(w64[:, None] * g64), np.abs(x64) * want_rstd
        # per entry: rstd's error and three roundings of r p; of r u (sum p u) / d rstd's error three times, the chain of the
        # sum (at most as long as the forward call's), and nine roundings
        term, pull = want_rstd * p, want_rstd * u * np.sum(p * u, axis=0) / d
        assert_within(dX, want, (rel + 3 * U) * term + (3 * rel + (chain + 9) * U) * pull + 2.0 ** -149, "fp32", "dX")
        # m terms in some order, each off by rel and two roundings
        assert_within(dw, want_dw, (rel + (m + 2) * U) * np.sum(np.abs(g64) * u, axis=1), "fp32", "dweight")


@pytest.mark.gpu
def test_a_gradient_of_zeros_has_no_nan():
    """Zeros with any eps: the second term is zero, not infinity times zero."""
    import torch
    from paper_2009_13977_amd import binding as B
    X, w = torch.zeros(64, 40, device="cuda"), torch.ones(64, device="cuda")
    G, g64 = normal(1, 64, 40)
    for eps in (1e-5, 1e-26, 1e-30, 1.2e-38):
        Y, rstd, dX, dw = torch.empty_like(X), torch.empty(40, device="cuda"), torch.empty_like(X), torch.empty_like(w)
        B.fasth_norm(X, w, Y, rstd, eps)
        B.fasth_norm_backward(G, X, w, rstd, dX, dw, B.new_workspace(B.fasth_norm_workspace_bytes(64, 40)))
        assert not Y.any() and not dw.any()
        want = g64 * float(np.float32(eps)) ** -0.5
        assert_within(dX, want, 8 * U * np.abs(want), "fp32", "dX")


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("d,m", [(400, 65504), (385, 65504)])
def test_few_rows_split_over_workgroups(d, m, dtype):
    """The fewest rows whose columns' sums wait in Y between the launches: some columns of each tile, the last ones among them."""
    import torch
    from paper_2009_13977_amd import binding as B
    gen = torch.Generator(device="cuda")
    gen.manual_seed(d)
    X, R = (torch.randn(d, m, device="cuda", generator=gen) for _ in range(2))
    w = torch.randn(d, device="cuda", generator=gen)
    guard = torch.full((d + 2, m), 7.0, device="cuda", dtype=torch_type(dtype))  # what follows Y stays as it is
    Y, S, rstd = guard[:d], torch.full_like(X, float("nan")), torch.full((m,), float("nan"), device="cuda")
    B.fasth_norm(X, w, Y, rstd, 1e-5, R, S)
    assert (guard[d:] == 7).all()
    cols = list(range(0, m, 997)) + [m - 3, m - 2, m - 1]
    s64 = host((X + R)[:, cols])
    np.testing.assert_array_equal(host(S[:, cols]), s64)
    want, want_rstd = tok.norm(s64, host(w), float(np.float32(1e-5)))
    rel = ((d / 64 + 45) / 2 + 7) * U
    assert_within(rstd[cols], want_rstd, rel * want_rstd, "fp32", "rstd")
    assert_within(Y[:, cols], want, (rel + 2 * U) * np.abs(want), dtype, "Y")
