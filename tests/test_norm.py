"""fasth_norm and fasth_norm_backward against the fp64 definition, entry by entry."""
import numpy as np
import pytest

from oracle import tokens as tok
from token_helpers import TYPES, U, assert_within, host, normal, torch_type

# every way in which a launch covers the mini-batch, and sizes off its tiles
SHAPES = [(1, 1), (2048, 8200), (1100, 4401), (640, 3001), (16384, 70), (9000, 3), (129, 2100), (1000, 8190), (3, 1), (1, 7), (64, 3), (65, 4), (100, 17), (784, 101), (1000, 1), (2048, 5), (4096, 20), (4097, 33), (8191, 9),
          (16384, 2), (16384, 6), (512, 1030), (48, 65535), (256, 4099), (1030, 5000),
          (8192, 2), (4096, 4), (2048, 8), (1024, 16), (3000, 3), (1500, 7), (700, 13)]
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
    ws = B.new_workspace(B.fasth_norm_workspace_bytes(d, m)).fill_(0xFF)
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
    # the sum of d squares, all positive: in one pass a thread adds at most 16, then 6 lane steps and 16 waves; split, a thread
    # adds d / (16 * 4) partial sums of 4 (or half as many of 8), then 2 lane steps, 4 waves and 32 splits. So at most
    # d / 64 + 44 roundings one after the other, and one of the square; half of that for the root, which with the quotient
    # and the division adds some 6 more
    chain = d / 64 + 45
    rel = (chain / 2 + 6) * U
    want, want_rstd = tok.norm(s64, w64, EPS)
    assert_within(rstd, want_rstd, rel * want_rstd, "fp32", "rstd")
    assert_within(Y, want, (rel + 2 * U) * np.abs(want), dtype, "Y")
    dX, dw = _norm_backward(G, S if residual else X, w, rstd, dS)
    want, want_dw = tok.norm_gradient(g64, s64, w64, EPS, ds64)
    term = want_rstd * np.abs(w64[:, None] * g64)
    # the column's sum with its roundings of the terms' sizes (two more each for w g S), times rstd^3 / d (3 rel and 5 roundings)
    pull = np.abs(s64) * want_rstd ** 3 / d * np.sum(np.abs(w64[:, None] * g64 * s64), axis=0)
    bound = (rel + 3 * U) * term + ((chain + 2) * U + 3 * rel + 7 * U) * pull + (3 * U * np.abs(ds64) if residual else 0.0)
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
@pytest.mark.parametrize("d,m,dtype", [(1600, 16000, "bf16"), (4097, 6145, "fp32")])
def test_matrices_larger_than_the_caches(d, m, dtype):
    _check(d, m, dtype, True)


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
@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
def test_largest_mini_batch(dtype):
    """16384 x 65535, 65536 bytes short of 4 GiB in fp32: the last rows and columns against the definition, a few columns at a time."""
    import torch
    d, m = 16384, 65535
    gen = torch.Generator(device="cuda")
    gen.manual_seed(1)
    X, R = (torch.randn(d, m, device="cuda", generator=gen) for _ in range(2))
    w = torch.randn(d, device="cuda", generator=gen)
    cols = [0, 1, 63, 64, 40000, 65531, 65532, 65533, 65534]
    s64 = host(X[:, cols] + R[:, cols])
    Y, rstd, S = _norm(X, R, w, dtype, S=R)  # in place: R becomes S
    chain = d / 64 + 45
    rel = (chain / 2 + 8) * U
    want, _ = tok.norm(s64, host(w), EPS)
    np.testing.assert_array_equal(host(S[:, cols]), s64)
    assert_within(Y[:, cols], want, rel * np.abs(want), dtype, "Y")
    g64 = host(Y[:, cols])
    dX, dw = _norm_backward(Y, S, w, rstd, X, dX=X)  # in place: dS = X becomes dX
    assert torch.isfinite(dX[-1]).all() and torch.isfinite(dw).all()
    gen.manual_seed(1)  # dS once more
    dS = torch.randn(d, m, device="cuda", generator=gen)[:, cols]
    want, _ = tok.norm_gradient(g64, s64, host(w), EPS, host(dS))
    assert np.abs(host(dX[:, cols]) - want).max() <= 2.0 ** -10 * np.abs(want).max()
    sums = torch.zeros(d, device="cuda", dtype=torch.float64)
    for j in range(0, m, 4096):
        sums += (Y[:, j:j + 4096].double() * S[:, j:j + 4096].double() * rstd[j:j + 4096].double()).sum(1)
    assert (dw.double() - sums).abs().max().item() <= 1e-4 * sums.abs().max().item()


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
