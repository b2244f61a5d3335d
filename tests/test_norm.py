"""fasth_norm and fasth_norm_backward against the fp64 definition, entry by entry."""
import numpy as np
import pytest

from oracle import tokens as tok
from token_helpers import TYPES, U, assert_within, host, normal, torch_type

SHAPES = [(1, 1), (3, 1), (1, 7), (64, 3), (65, 4), (100, 17), (784, 101), (1000, 1), (2048, 5), (4096, 20), (4097, 33), (8191, 9),
          (16384, 2), (16384, 6), (512, 1030), (48, 65535), (256, 4099), (1030, 5000)]
EPS = 1e-5


def _norm(X, R, w, dtype, S=None):
    import torch
    from paper_2009_13977_amd import binding as B
    d, m = X.shape
    Y = torch.full((d, m), float("nan"), device="cuda", dtype=torch_type(dtype))
    rstd = torch.full((m,), float("nan"), device="cuda")
    if R is not None and S is None:
        S = torch.full_like(X, float("nan"))
    B.fasth_norm(X, w, Y, rstd, EPS, R, S)
    return Y, rstd, S


def _norm_backward(G, S, w, rstd, dS, weight_gradient=True, dX=None):
    import torch
    from paper_2009_13977_amd import binding as B
    d, m = S.shape
    dX = torch.full_like(S, float("nan")) if dX is None else dX
    dw = torch.full_like(w, float("nan")) if weight_gradient else None
    ws = B.new_workspace(B.fasth_norm_workspace_bytes(d, m)).fill_(0xFF) if weight_gradient else None
    B.fasth_norm_backward(G, S, w, rstd, dX, dw, ws, dS)
    return dX, dw


def _check(d, m, dtype, residual, seed=0):
    X, x64 = normal(seed + 1, d, m)
    R, r64 = normal(seed + 2, d, m, scale=2.0) if residual else (None, None)
    w, w64 = normal(seed + 3, d)
    G, g64 = normal(seed + 4, d, m, dtype=dtype)
    dS, ds64 = normal(seed + 5, d, m) if residual else (None, None)
    Y, rstd, S = _norm(X, R, w, dtype)
    s64 = x64
    if residual:
        s64 = (x64.astype(np.float32) + r64.astype(np.float32)).astype(np.float64)  # one fp32 addition
        np.testing.assert_array_equal(host(S), s64)
    # the sum of d squares: a thread adds at most 16, then 6 lane steps and 16 waves, so at most 38 roundings and one of the
    # square, all of positive terms; half of that for the root, which with the quotient and the division adds some 6 more
    rel = (39 / 2 + 6) * U
    want, want_rstd = tok.norm(s64, w64, EPS)
    assert_within(rstd, want_rstd, rel * want_rstd, "fp32", "rstd")
    assert_within(Y, want, (rel + 2 * U) * np.abs(want), dtype, "Y")
    dX, dw = _norm_backward(G, S if residual else X, w, rstd, dS)
    want, want_dw = tok.norm_gradient(g64, s64, w64, EPS, ds64)
    term = want_rstd * np.abs(w64[:, None] * g64)
    # the column's sum with its 41 roundings of the terms' sizes, times rstd^3 / d (3 rel and 5 roundings)
    pull = np.abs(s64) * want_rstd ** 3 / d * np.sum(np.abs(w64[:, None] * g64 * s64), axis=0)
    bound = (rel + 3 * U) * term + (46 * U + 3 * rel + 2 * U) * pull + (3 * U * np.abs(ds64) if residual else 0.0)
    assert_within(dX, want, bound, "fp32", "dX")
    # m terms in some order: at most m roundings of the sum of their sizes, each term off by rel and two roundings
    size = np.sum(np.abs(g64 * s64) * want_rstd, axis=1)
    assert_within(dw, want_dw, (rel + (m + 2) * U) * size, "fp32", "dweight")


@pytest.mark.gpu
@pytest.mark.parametrize("residual", [False, True])
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("d,m", SHAPES)
def test_both_directions(d, m, dtype, residual):
    _check(d, m, dtype, residual)


@pytest.mark.gpu
def test_in_place():
    """S over X, S over R, dX over dS: the same bits as with outputs of their own."""
    X, _ = normal(1, 300, 37)
    R, _ = normal(2, 300, 37)
    w, _ = normal(3, 300)
    G, _ = normal(4, 300, 37)
    dS, _ = normal(5, 300, 37)
    Y, rstd, S = _norm(X, R, w, "fp32")
    for over in ("X", "R"):
        x, r = X.clone(), R.clone()
        Y2, rstd2, S2 = _norm(x, r, w, "fp32", S={"X": x, "R": r}[over])
        assert (Y2 == Y).all() and (S2 == S).all() and (rstd2 == rstd).all()
    dX, dw = _norm_backward(G, S, w, rstd, dS)
    again = dS.clone()
    dX2, dw2 = _norm_backward(G, S, w, rstd, again, dX=again)
    assert (dX2 == dX).all() and (dw2 == dw).all()
    dX3, none = _norm_backward(G, S, w, rstd, dS, weight_gradient=False)
    assert none is None and (dX3 == dX).all()


@pytest.mark.gpu
def test_columns_do_not_touch_each_other():
    """Zeros, infinities, NaN and very small and large columns beside ordinary ones."""
    import torch
    X, x64 = normal(1, 130, 9)
    w, w64 = normal(2, 130)
    X[:, 1] = 0.0
    X[5, 2], X[6, 4] = float("inf"), float("nan")
    X[:, 6] *= 1e-30
    X[:, 7] *= 1e15
    Y, rstd, _ = _norm(X, None, w, "fp32")
    x64 = host(X)
    want, _ = tok.norm(x64[:, [0, 3, 5, 6, 7, 8]], w64, EPS)
    assert_within(Y[:, [0, 3, 5, 6, 7, 8]], want, 30 * U * np.abs(want) + 1e-38, "fp32", "Y")
    assert (host(Y)[:, 1] == 0).all() and np.isnan(host(Y)[6, 4]) and np.isnan(host(Y)[5, 2])
    assert host(rstd)[1] == pytest.approx(EPS ** -0.5, rel=1e-6)
    G, g64 = normal(3, 130, 9)
    dX, _ = _norm_backward(G, X, w, rstd, None)
    want, _ = tok.norm_gradient(g64[:, [0, 1, 3, 5, 8]], x64[:, [0, 1, 3, 5, 8]], w64, EPS)
    assert np.abs(host(dX)[:, [0, 1, 3, 5, 8]] - want).max() <= 100 * U * np.abs(want).max()


@pytest.mark.gpu
def test_gradient_by_differences():
    """The loss <G, Y> through the forward kernel, a step of 2^-7 to either side along a direction: the third derivative
    leaves some 2^-14 of the slope, rounding 2^-24 times the loss's terms over 2^-6."""
    X, x64 = normal(1, 96, 24)
    w, _ = normal(2, 96)
    G, g64 = normal(3, 96, 24)
    V, v64 = normal(4, 96, 24)
    h = 2.0 ** -7
    hi, lo = (tuple(host(t) for t in _norm(X + s * h * V, None, w, "fp32")[:1])[0] for s in (1, -1))
    slope = np.sum(g64 * (hi - lo)) / (2 * h)
    _, rstd, _ = _norm(X, None, w, "fp32")
    dX, _ = _norm_backward(G, X, w, rstd, None)
    along = np.sum(host(dX) * v64)
    scale = np.sqrt(np.sum(host(dX) ** 2)) * np.sqrt(np.sum(v64 ** 2))
    assert abs(slope - along) <= 2.0 ** -10 * scale


@pytest.mark.gpu
def test_refuses_what_it_cannot_take():
    import torch
    from paper_2009_13977_amd import binding as B
    X, w = torch.ones(8, 4, device="cuda"), torch.ones(8, device="cuda")
    Y, rstd = torch.empty_like(X), torch.empty(4, device="cuda")
    for kw in (dict(R=X.clone()), dict(S=X.clone())):  # both or neither
        with pytest.raises(B.FasthError):
            B.fasth_norm(X, w, Y, rstd, **kw)
    for eps in (0.0, -1.0, float("nan"), float("inf")):
        with pytest.raises(B.FasthError):
            B.fasth_norm(X, w, Y, rstd, eps)
    with pytest.raises(ValueError):
        B.fasth_norm(X.half(), w, Y, rstd)
    with pytest.raises(ValueError):
        B.fasth_norm(X, w[:7], Y, rstd)
    with pytest.raises(ValueError):
        B.fasth_norm(X.t(), torch.ones(4, device="cuda"), Y.t(), torch.empty(8, device="cuda"))
    with pytest.raises(B.FasthError) as e:
        B.fasth_norm_backward(Y, X, w, rstd, Y.clone(), torch.empty(8, device="cuda"), B.new_workspace(16))
    assert e.value.code == B.FASTH_EWORKSPACE
    with pytest.raises(B.FasthError) as e:  # a base address off a multiple of 16 bytes
        B.fasth_norm(torch.ones(33, device="cuda")[1:].view(8, 4), w, Y, rstd)
    assert e.value.code == B.FASTH_EALIGN
