"""fasth_log_prob and its gradient where a column is sure of a token: what is left beside it, 1 - p, is the given token's
gradient and most of the entropy, and has to be right relative to itself, at whichever row the token stands."""
import numpy as np
import pytest

from oracle import tokens as tok
from token_helpers import TYPES, U, assert_within, host, torch_type

SURE = (0.5, 0.9, 0.99, 0.9999, 0.999999, 1 - 1e-8)
# (vocab, columns, rows that one thread adds at most): a column per lane, four, 64 and more columns per workgroup,
# columns shared by workgroups, and logits beyond the caches, in rows off the cache lines and of whole ones
SHAPES = [(1000, 2, 16), (3000, 7, 16), (256, 300, 16), (32000, 48, 16), (40000, 700, 64), (51200, 4100, 128), (51200, 4160, 128)]


def _sure_columns(vocab, m, dtype, seed):
    """Normal logits; in column j the row 7 j (mod vocab) gets the probability SURE[j], SURE[j + 1], ... in turn."""
    import torch
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    x = torch.randn(vocab, m, device="cuda", generator=gen)
    cols = torch.arange(m, device="cuda")
    rows = 7 * cols % vocab
    p = torch.tensor(SURE, dtype=torch.float64, device="cuda")[(cols // 16 + cols) % len(SURE)]
    x[rows, cols] = float("-inf")
    x[rows, cols] = (torch.logsumexp(x.double(), 0) + torch.log(p / (1 - p))).float()
    return x.to(torch_type(dtype)), rows


def _run(x, ids, top=0):
    import torch
    from paper_2009_13977_amd import binding as B
    vocab, m = x.shape
    nan = lambda *shape: torch.full(shape, float("nan"), device="cuda")
    logp, entropy, stats, top_logp = nan(m), nan(m), nan(2, m), nan(top, m) if top else None
    top_ids = torch.full((top, m), -7, device="cuda", dtype=torch.int32) if top else None
    ws = B.new_workspace(B.fasth_log_prob_workspace_bytes(vocab, m, top)).fill_(0xFF)
    B.fasth_log_prob(x, ids, logp, entropy, stats, ws, top_logp, top_ids)
    return logp, entropy, stats, top_logp, top_ids


def _left(x64, rows, thread_rows):
    """(-log p, the entropy, a bound of the error of each) per column, for the row that holds the largest logit. With
    r = e^(x - M) of the other rows, R their sum and a = M - x: L = -log p = log(1 + R) and H = L + (sum r a) / (1 + R).

    - The group of eight rows with the largest logit adds its other seven to 1, in three levels. A rounding of 1 + z with
      small z is off by at most U and at most z: at most three U, and at most the seven largest r together.
    - Every r is off by 3 U a (the difference, log2 e and their product), in all its changes of reference together, as these
      add up to a; by 2 U for each exponential and U for each product and sum: three levels of a group, a change and a
      sum per group of its thread, and at most 15 joins of two sums (6 over lanes, 2 over waves, 7 over splits).
    - r a takes one product more at each of these places."""
    m = x64.shape[1]
    at = (rows, np.arange(m))
    a = x64[at] - x64
    a[at] = np.inf
    r = np.exp(-a)
    a[at] = 0.0
    R, Q = r.sum(0), (r * a).sum(0)
    own = np.minimum(3 * U, np.sort(r, axis=0)[-7:].sum(0))
    steps = thread_rows / 8
    dR = own + 3 * U * Q + (4 * steps + 15 * 5 + 5) * U * R
    dQ = 3 * U * (r * a * a).sum(0) + (5 * steps + 15 * 6 + 8) * U * Q + own * Q
    L = np.log1p(R)
    dL = dR / (1 + R) + 4 * U * L
    H = L + Q / (1 + R)
    # the definition adds `vocab` terms to the 1 one after the other, each sum below 2 and so off by 2^-53 at most
    logp, entropy, _, _ = tok.log_prob(x64, rows)
    slack = x64.shape[0] * 2.0 ** -53
    assert np.abs(logp + L).max() <= slack and np.abs(entropy - H).max() <= 2 * slack * (1 + H.max())
    return L, H, dL, dL + dQ + Q * dR + 6 * U * (L + Q)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("vocab,m,thread_rows", SHAPES)
def test_what_is_left_beside_a_sure_token(vocab, m, thread_rows, dtype):
    import torch
    from paper_2009_13977_amd import binding as B
    x, rows = _sure_columns(vocab, m, dtype, seed=vocab)
    logp, entropy, stats, _, _ = _run(x, rows)
    dx = {}
    for name, gl, ge in (("logp", 1.5, None), ("entropy", None, -0.75), ("both", 1.5, -0.75)):
        dx[name] = torch.full_like(x, float("nan"))
        B.fasth_log_prob_backward(x, rows, stats, entropy, *(None if g is None else torch.full((m,), g, device="cuda") for g in (gl, ge)), dx[name])
    given = {name: d[rows, torch.arange(m, device="cuda")] for name, d in dx.items()}
    keep = np.unique(np.r_[0:min(m, 300), max(0, m - 40):m])  # (the definition in 64 bits for some columns of wide ones)
    x64, i64 = host(x[:, keep]), rows[keep].cpu().numpy()
    L, H, dL, dH = _left(x64, i64, thread_rows)
    assert (host(logp) <= 0).all() and (host(entropy) >= 0).all()
    assert_within(logp[keep], -L, dL, "fp32", "logp")
    assert_within(entropy[keep], H, dH, "fp32", "entropy")
    # 1 - p from L: its error, and some 20 roundings of the products and the series; p of the bracket likewise
    left = -np.expm1(-L)
    assert_within(given["logp"][keep], 1.5 * left, 1.5 * (dL + 20 * U * L), dtype, "the given token's gradient")
    assert (host(given["logp"]) >= 0).all()
    bracket = np.exp(-L) * (H - L)  # p (log p + H)
    d_bracket = dL + dH + 12 * U * (L + H)
    assert_within(given["entropy"][keep], 0.75 * bracket, 0.75 * d_bracket, dtype, "its part of the entropy's gradient")
    both, d_both = 1.5 * left + 0.75 * bracket, 1.5 * (dL + 20 * U * L) + 0.75 * d_bracket + 2 * U * (left + np.abs(bracket))
    assert_within(given["both"][keep], both, d_both, dtype, "both")


@pytest.mark.gpu
@pytest.mark.parametrize("vocab,m", [(32000, 48), (5000, 3), (300, 300)])
def test_alternatives_of_sure_columns(vocab, m):
    x, rows = _sure_columns(vocab, m, "fp32", seed=3)
    logp, _, _, top_logp, top_ids = _run(x, rows, top=4)
    assert (top_ids[0] == rows).all() and (top_logp[0] == logp).all() and (top_logp <= 0).all()
    want = tok.log_prob(host(x), None, 4)
    np.testing.assert_array_equal(top_ids.cpu().numpy(), want[3])
    L, _, dL, _ = _left(host(x), rows.cpu().numpy(), 16)
    t = np.abs(want[2])
    assert_within(top_logp, want[2], dL + 3 * U * (t + L), "fp32", "top_logp")


@pytest.mark.gpu
@pytest.mark.parametrize("gap", [12.0, 16.1, 18.3, 20.0, 23.0, 26.0, 27.5, 40.0])
def test_no_probability_above_one_and_no_negative_entropy(gap):
    """Every row of 256 in turn stands out; the error does not grow with the distance."""
    import torch
    gen = torch.Generator(device="cuda")
    gen.manual_seed(5)
    x = torch.randn(256, 256, device="cuda", generator=gen)
    ids = torch.arange(256, device="cuda")
    x[ids, ids] = gap
    logp, entropy, _, _, _ = _run(x, ids)
    assert (logp <= 0).all() and (entropy >= 0).all()
    L, H, dL, dH = _left(host(x), np.arange(256), 16)
    assert_within(logp, -L, dL, "fp32", "logp")
    assert_within(entropy, H, dH, "fp32", "entropy")
