"""fasth_log_prob and fasth_log_prob_backward against the fp64 definition, entry by entry."""
import numpy as np
import pytest

from oracle import tokens as tok
from token_helpers import TYPES, U, assert_within, host, normal, tokens, torch_type

SHAPES = [(1, 1, 1), (2, 3, 2), (5, 70, 8), (16, 4, 16), (17, 1, 20), (256, 300, 0), (1000, 15, 5), (1001, 16, 5), (3000, 65, 8), (513, 2, 32),
          (32003, 5, 8), (128000, 1, 8), (200003, 2, 3), (50021, 67, 0), (100, 4097, 0), (33, 1500, 4), (12, 65535, 0), (300000, 1, 32)]


def _log_prob(x, ids, top):
    import torch
    from paper_2009_13977_amd import binding as B
    vocab, m = x.shape
    nan = lambda *shape: torch.full(shape, float("nan"), device="cuda")
    logp, entropy, stats = nan(m), nan(m), nan(2, m)
    top_logp = nan(top, m) if top else None
    top_ids = torch.full((top, m), -7, device="cuda", dtype=torch.int32) if top else None
    ws = B.new_workspace(B.fasth_log_prob_workspace_bytes(vocab, m, top)).fill_(0xFF)
    B.fasth_log_prob(x, ids, logp, entropy, stats, ws, top_logp, top_ids)
    return logp, entropy, stats, top_logp, top_ids


def _sizes(x64):
    """Per column: roundings of the sum, mean distance of the logits from the largest, log of the sum."""
    vocab, m = x64.shape
    # one thread's share of a column (at least a workgroup's 16 rows of threads), its rescalings, and the joins
    count = 1.25 * vocab / 16 + 100
    lp = tok.log_softmax(x64)
    p = np.exp(lp)
    most = np.max(x64, axis=0)
    with np.errstate(invalid="ignore"):
        away = np.where(p > 0, most - x64, 0.0)
    return count, np.sum(p * away, axis=0), lp, p, np.where(p > 0, away, 0.0)


def _check(x, x64, ids, i64, top, dtype, seed=0):
    import torch
    from paper_2009_13977_amd import binding as B
    vocab, m = x64.shape
    logp, entropy, stats, top_logp, top_ids = _log_prob(x, ids, top)
    want = tok.log_prob(x64, i64, top)
    count, mean_away, lp, p, away = _sizes(x64)
    # a term e^-t: t and its product with log2 e are rounded (3 U t), the exponential is off by 2 U; the sum adds `count`
    log_sum = (count + 4 + 3 * mean_away) * U
    total = np.sum(np.exp(-away) * (p > 0), axis=0)
    L = np.abs(np.log(np.where(total > 0, total, 1.0)))
    given = np.zeros(m)
    ok = (i64 >= 0) & (i64 < vocab) if i64 is not None else np.zeros(m, bool)
    with np.errstate(invalid="ignore"):
        given[ok] = away[i64[ok], np.flatnonzero(ok)] if ok.any() else 0.0
    finite = np.isfinite(want[0])
    assert_within(logp, want[0], np.where(finite, log_sum + 3 * U * (L + given + np.abs(np.where(finite, want[0], 0.0))), 0.0), "fp32", "logp")
    spread = np.sum(p * away * (3 * away + count + 6), axis=0) * U  # the second sum's error over the first
    bound_H = log_sum * (1 + mean_away) + spread + 4 * U * (L + mean_away)
    assert_within(entropy, want[1], bound_H, "fp32", "entropy")
    if top:
        np.testing.assert_array_equal(top_ids.cpu().numpy(), want[3])
        has = want[3] >= 0
        t = np.where(has, np.abs(np.where(has, want[2], 0.0)), 0.0)
        assert_within(top_logp, want[2], np.where(has, log_sum + 3 * U * (2 * L + 2 * t), 0.0), "fp32", "top_logp")
    r = np.random.default_rng(seed)
    gl, ge = r.normal(size=m).astype(np.float32), r.normal(size=m).astype(np.float32)
    for g_logp, g_entropy in ((gl, ge), (gl, None), (None, ge)):
        if g_logp is not None and ids is None:
            continue
        dx = torch.full_like(x, float("nan"))
        B.fasth_log_prob_backward(x, ids, stats, entropy, *(None if g is None else torch.from_numpy(g).cuda() for g in (g_logp, g_entropy)), dx)
        exact = tok.log_prob_gradient(x64, i64, g_logp, g_entropy)
        a, b = (np.abs(g) if g is not None else np.zeros(m) for g in (g_logp, g_entropy))
        log_p = np.where(p > 0, np.abs(np.where(p > 0, lp, 0.0)), 0.0)
        # p is off by the error of its logarithm; the bracket of the entropy by that and the entropy's own error
        with np.errstate(invalid="ignore"):
            H = np.where(np.isfinite(want[1]), want[1], 0.0)
        rel_p = log_sum + 3 * U * (away + L + 2 * log_p) + 4 * U
        bound = p * (a + b * (log_p + H)) * (rel_p + 6 * U) + p * b * (rel_p + bound_H) + 3 * U * a
        # the smallest normal fp32 number is 2^-126, and the exponential gives zero below it: a p of 1e-38 may be missing
        # whole, and with it its product with a bracket of log p = -87 (found at p = 1.04e-38 = e^-84 / 31.6, 84 times which is off)
        bound = bound + 2.0 ** -126 * (a + b * (log_p + H))
        assert_within(dx, exact, bound, dtype, "dlogits")
    return logp, entropy, top_ids


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("vocab,m,top", SHAPES)
def test_both_directions(vocab, m, top, dtype):
    x, x64 = normal(1, vocab, m, dtype=dtype, scale=2.0)
    ids, i64 = tokens(2, vocab, m, bits=32 if m % 2 else 64)
    _check(x, x64, ids, i64, top, dtype)


@pytest.mark.gpu
@pytest.mark.parametrize("top", [0, 3])
def test_logits_larger_than_the_caches(top):
    """420 MB: some columns, the last ones among them; their gradients have the bits that they have in a mini-batch of their own."""
    import torch
    from paper_2009_13977_amd import binding as B
    vocab, m = 51203, 4101
    gen = torch.Generator(device="cuda")
    gen.manual_seed(1)
    x = torch.randn(vocab, m, device="cuda", generator=gen).to(torch.bfloat16)
    ids = torch.randint(0, vocab, (m,), device="cuda", generator=gen)
    g = [row.clone() for row in torch.randn(2, m, device="cuda", generator=gen)]  # (a row of 4101 would not be aligned)
    logp, entropy, stats, top_logp, top_ids = _log_prob(x, ids, top)
    dx = torch.full_like(x, float("nan"))
    B.fasth_log_prob_backward(x, ids, stats, entropy, g[0], g[1], dx)
    cols = [0, 1, 127, 128, 255, 256, 2000, 4095, 4096, 4097, 4098, 4099, 4100]
    some, some_ids = x[:, cols].contiguous(), ids[cols].contiguous()
    x64, i64 = host(some), some_ids.cpu().numpy()
    want = tok.log_prob(x64, i64, top)
    # logits of some five units: the bounds of _check with a mean distance of five and a sum below e^11
    count = 1.25 * vocab / 16 + 100
    assert_within(logp[cols], want[0], (count + 4 + 15) * U + 3 * U * (11 + 10 + np.abs(want[0])), "fp32", "logp")
    assert_within(entropy[cols], want[1], (count + 19) * U * 6 + 5 * (15 + count + 6) * U + 4 * U * 16, "fp32", "entropy")
    if top:
        np.testing.assert_array_equal(top_ids[:, cols].cpu().numpy(), want[3])
    exact = tok.log_prob_gradient(x64, i64, host(g[0][cols]), host(g[1][cols]))
    dy = torch.full_like(some, float("nan"))
    B.fasth_log_prob_backward(some, some_ids, stats[:, cols].contiguous(), entropy[cols].contiguous(), g[0][cols].contiguous(),
                              g[1][cols].contiguous(), dy)
    assert (dy == dx[:, cols]).all()  # entries do not meet: the same operations in either launch
    np.testing.assert_allclose(host(dx[:, cols]).sum(0), exact.sum(0), atol=2.0 ** -8 * np.abs(exact).sum(0).max())


@pytest.mark.gpu
@pytest.mark.parametrize("vocab,m", [(700, 5), (700, 33), (20000, 3), (20000, 70)])
def test_masked_logits(vocab, m):
    """Half of the vocabulary masked; one column with one row left, one with nothing left, one whose given token is masked."""
    x, _ = normal(3, vocab, m, scale=3.0)
    x[::2] = float("-inf")
    x[:, 0] = float("-inf")
    x[vocab // 2, 0] = -5.0
    x[:, 1] = float("-inf")
    ids, i64 = tokens(4, vocab, m, padded=False)
    i64[0], i64[1], i64[2] = vocab // 2, 7, 0
    ids.copy_(__import__("torch").from_numpy(i64))
    x[i64[2], 2] = float("-inf")
    logp, entropy, top_ids = _check(x, host(x), ids, i64, 8, "fp32")
    logp, entropy = host(logp), host(entropy)
    assert logp[0] == 0 and entropy[0] == 0 and entropy[1] == 0 and np.isneginf(logp[1:3]).all()
    assert top_ids[0, 0] == vocab // 2 and (top_ids[1:, 0] == -1).all() and (top_ids[:, 1] == -1).all()


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", TYPES)
def test_masks_of_the_lowest_value_and_far_logits(dtype):
    """The type's lowest value as a mask, a column of nothing else (every row the same probability), and logits far from zero."""
    import torch
    x, _ = normal(5, 300, 20, dtype=dtype)
    lowest = torch.finfo(x.dtype).min
    x[100:] = lowest
    x[:, 3] = lowest
    x[:, 4] += 1000.0
    x[:, 5] -= 1000.0
    ids, i64 = tokens(6, 100, 20)
    _, entropy, top_ids = _check(x, host(x), ids, i64, 5, dtype)
    assert host(entropy)[3] == pytest.approx(np.log(300), rel=1e-6)
    assert top_ids[:, 3].tolist() == [0, 1, 2, 3, 4]


@pytest.mark.gpu
@pytest.mark.parametrize("vocab", [9, 64, 1000, 40000])
def test_ties_go_to_the_lower_row(vocab):
    import torch
    x = torch.zeros(vocab, 6, device="cuda", dtype=torch.bfloat16)
    x[:, 1] = torch.arange(vocab, device="cuda") % 3
    x[:, 2] = -(torch.arange(vocab, device="cuda") // 20).float()
    x[vocab - 1, 3], x[vocab // 2, 3] = 1, 1
    _check(x, host(x), None, None, min(32, vocab), "bf16")


@pytest.mark.gpu
@pytest.mark.parametrize("vocab", [40, 9000])
def test_zeros_of_both_signs_are_equal(vocab):
    import torch
    x = torch.zeros(vocab, 3, device="cuda")
    x[::2, 0] = -0.0
    x[1::2, 1] = -0.0
    x[:, 2] = -0.0
    x[vocab // 2, 2] = 0.0
    _, _, _, _, top_ids = _log_prob(x, None, 6)
    np.testing.assert_array_equal(top_ids.cpu().numpy(), np.repeat(np.arange(6)[:, None], 3, axis=1))


@pytest.mark.gpu
@pytest.mark.parametrize("m", [3, 40])
def test_nan_and_infinity_stay_in_their_columns(m):
    import torch
    from paper_2009_13977_amd import binding as B
    x, x64 = normal(7, 5000, m)
    x[4321, 0], x[17, 2] = float("nan"), float("inf")
    ids = torch.zeros(m, dtype=torch.int64, device="cuda")
    logp, entropy, stats, top_logp, top_ids = _log_prob(x, ids, 4)
    assert np.isnan(host(logp)[[0, 2]]).all() and np.isnan(host(entropy)[[0, 2]]).all()
    keep = [j for j in range(m) if j not in (0, 2)]
    want = tok.log_prob(x64[:, keep], np.zeros(len(keep)), 4)
    np.testing.assert_allclose(host(logp)[keep], want[0], rtol=1e-5)
    np.testing.assert_array_equal(host(top_ids)[:, keep], want[3])
    column = np.where(np.arange(5000) == 4321, -np.inf, x64[:, 0])
    np.testing.assert_array_equal(host(top_ids)[:, 0], np.argsort(-column, kind="stable")[:4])  # NaN is no alternative
    assert top_ids[0, 2] == 17
    dx = torch.empty_like(x)
    B.fasth_log_prob_backward(x, ids, stats, entropy, torch.ones(m, device="cuda"), None, dx)
    assert np.isnan(host(dx)[:, [0, 2]]).all() and np.isfinite(host(dx)[:, keep]).all()


@pytest.mark.gpu
def test_gradient_in_place_and_repeated_bits():
    import torch
    from paper_2009_13977_amd import binding as B
    for vocab, m in ((4000, 50), (4000, 3)):
        x, _ = normal(8, vocab, m, dtype="bf16")
        ids, _ = tokens(9, vocab, m)
        first = _log_prob(x, ids, 6)
        for _ in range(3):
            assert all((a == b).all() for a, b in zip(first, _log_prob(x, ids, 6)))
        gl, ge = torch.randn(m, device="cuda"), torch.randn(m, device="cuda")
        dx = torch.empty_like(x)
        B.fasth_log_prob_backward(x, ids, first[2], first[1], gl, ge, dx)
        over = x.clone()
        B.fasth_log_prob_backward(over, ids, first[2], first[1], gl, ge, over)
        assert (over == dx).all()


@pytest.mark.gpu
def test_offsets_beyond_32_bits():
    """2,100,000,000 and more entries: the last rows and columns lie beyond 2^31 elements (2^32 bytes)."""
    import torch
    from paper_2009_13977_amd import binding as B
    vocab, m = 33000, 65535
    x = torch.zeros(vocab, m, device="cuda", dtype=torch.bfloat16)
    x[-1, :] = 5.0
    x[0, -2] = 9.0
    ids = torch.full((m,), vocab - 1, device="cuda")
    logp, entropy, stats, _, _ = _log_prob(x, ids, 0)
    want = -np.log1p((vocab - 1) * np.exp(-5.0))
    got = host(logp)
    np.testing.assert_allclose(np.delete(got, m - 2), want, rtol=1e-4)
    assert got[m - 2] == pytest.approx(-np.log(np.exp(4.0) + 1 + (vocab - 2) * np.exp(-5.0)), rel=1e-4)
    B.fasth_log_prob_backward(x, ids, stats, None, torch.ones(m, device="cuda"), None, x)
    last = host(x[-1])
    np.testing.assert_allclose(np.delete(last, m - 2), 1 - np.exp(want), rtol=1.01 * 2.0 ** -8)
    np.testing.assert_allclose(host(x[vocab // 2, :100]), -np.exp(want - 5.0), rtol=2.0 ** -7)


@pytest.mark.gpu
def test_refuses_what_it_cannot_take():
    import torch
    from paper_2009_13977_amd import binding as B
    x, _ = normal(1, 50, 4)
    f = lambda *s: torch.empty(*s, device="cuda")
    ids, ws = torch.zeros(4, dtype=torch.int32, device="cuda"), B.new_workspace(B.fasth_log_prob_workspace_bytes(50, 4, 3))
    args = (f(4), f(4), f(2, 4), ws)
    with pytest.raises(B.FasthError):  # one of the two alone
        B.fasth_log_prob(x, ids, *args, top_logp=f(3, 4))
    with pytest.raises(ValueError):
        B.fasth_log_prob(x, ids, *args, top_logp=f(3, 4), top_ids=torch.empty(3, 4, dtype=torch.int64, device="cuda"))
    with pytest.raises(B.FasthError) as e:
        B.fasth_log_prob(x, ids, *args, top_logp=f(33, 4), top_ids=torch.empty(33, 4, dtype=torch.int32, device="cuda"))
    assert e.value.code == B.FASTH_EUNSUPPORTED
    with pytest.raises(B.FasthError) as e:
        B.fasth_log_prob(x, ids, f(4), f(4), f(2, 4), B.new_workspace(16))
    assert e.value.code == B.FASTH_EWORKSPACE
    with pytest.raises(ValueError):
        B.fasth_log_prob(x[:, :2], ids[:2], f(2), f(2), f(2, 2), ws)
    for kw in (dict(ids=None, g_logp=f(4), g_entropy=None), dict(ids=ids, g_logp=None, g_entropy=None)):
        with pytest.raises(B.FasthError):
            B.fasth_log_prob_backward(x, kw["ids"], f(2, 4), f(4), kw["g_logp"], kw["g_entropy"], f(50, 4))
    with pytest.raises(ValueError):
        B.fasth_log_prob_backward(x, ids, f(2, 4), f(4), f(4), None, f(50, 4).half())
