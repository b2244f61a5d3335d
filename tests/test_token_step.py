"""The operators around the layers together, as a token model uses them: one training step through an embedding, norms,
an SVD layer with a residual, a rectangular layer that makes the logits, log probabilities, all gradients and their
clipping; the next token's alternatives; other streams and captured graphs."""
import numpy as np
import pytest

from helpers import assert_close
from oracle import householder as orc
from oracle import tokens as tok
from token_helpers import host

EPS, K = 1e-5, 16


def _parameters(seed, vocab, d):
    r = np.random.default_rng(seed)
    f32 = lambda a: a.astype(np.float32)
    return {"table": f32(r.normal(size=(vocab, d)) * 0.3), "w1": f32(1 + 0.1 * r.normal(size=d)), "w2": f32(1 + 0.1 * r.normal(size=d)),
            "Uv": f32(r.normal(size=(d, d))), "Vv": f32(r.normal(size=(d, d))), "sigma": f32(r.uniform(0.5, 2, d)),
            "Ur": f32(r.normal(size=(vocab, vocab))), "Vr": f32(r.normal(size=(d, d))), "sigma_r": f32(r.uniform(0.5, 2, min(d, vocab)))}


def _reference(p, ids, targets, g_logp, g_entropy):
    """(loss, gradients) in fp64."""
    p = {k: v.astype(np.float64) for k, v in p.items()}
    scale = np.sqrt(p["table"].shape[1])
    X0 = tok.embed(p["table"], ids, scale)
    Y1, _ = tok.norm(X0, p["w1"], EPS)
    Z = orc.svd_layer_apply(p["Uv"], p["sigma"], p["Vv"], Y1)
    S = X0 + Z
    Y2, _ = tok.norm(S, p["w2"], EPS)
    logits = orc.rectangular_apply(p["Ur"], p["sigma_r"], p["Vr"], Y2)
    logp, H, _, _ = tok.log_prob(logits, targets)
    loss = np.sum(g_logp * logp) + np.sum(g_entropy * H)
    g = {}
    dlogits = tok.log_prob_gradient(logits, targets, g_logp, g_entropy)
    _, g["Ur"], g["sigma_r"], g["Vr"], dY2 = orc.rectangular_gradients(p["Ur"], p["sigma_r"], p["Vr"], Y2, dlogits)
    dS, g["w2"] = tok.norm_gradient(dY2, S, p["w2"], EPS)
    _, g["Uv"], g["sigma"], g["Vv"], dY1 = orc.svd_layer_gradients(p["Uv"], p["sigma"], p["Vv"], Y1, dS)
    dX0, g["w1"] = tok.norm_gradient(dY1, X0, p["w1"], EPS, dS)
    g["table"] = tok.embed_gradient(p["table"].shape[0], ids, dX0, scale)
    return loss, g


def _batch(seed, vocab, m):
    r = np.random.default_rng(seed)
    ids, targets = r.integers(0, vocab, m), r.integers(0, vocab, m)
    targets[::7] = -1
    return ids, targets, np.where(targets >= 0, -1.0 / m, 0.0), np.full(m, -0.01 / m)


def test_reference_gradients_by_differences():
    """Along random directions, h = 1e-5 in fp64: h^2 times a third derivative of some tens."""
    vocab, d, m = 32, 16, 6
    p = _parameters(0, vocab, d)
    batch = _batch(1, vocab, m)
    _, g = _reference(p, *batch)
    r = np.random.default_rng(2)
    for name in p:
        v = r.normal(size=p[name].shape)
        at = lambda s: _reference({**p, name: p[name].astype(np.float64) + s * v}, *batch)[0]
        slope = (at(1e-5) - at(-1e-5)) / 2e-5
        assert slope == pytest.approx(np.sum(g[name] * v), rel=1e-5, abs=1e-8), name


class Model:
    """Buffers and calls of one training step, all through the public entry points."""

    def __init__(self, p, m):
        import torch
        from paper_2009_13977_amd import binding as B
        self.B = B
        self.p = {k: torch.from_numpy(v).cuda() for k, v in p.items()}
        self.g = {k: torch.full_like(v, float("nan")) for k, v in self.p.items()}
        vocab, d = p["table"].shape
        f = lambda *s: torch.full(s, float("nan"), device="cuda")
        self.scale = float(np.sqrt(d))
        self.X0, self.Y1, self.Z, self.S, self.Y2, self.dY2, self.dS, self.dY1, self.dX0 = (f(d, m) for _ in range(9))
        self.r1, self.r2, self.logp, self.H = (f(m) for _ in range(4))
        self.logits, self.dlogits, self.stats, self.norm = f(vocab, m), f(vocab, m), f(2, m), f(1)
        self.ids, self.targets = (torch.zeros(m, dtype=torch.int64, device="cuda") for _ in range(2))
        self.gl, self.ge = f(m), f(m)
        ws = B.new_workspace
        self.ws_layer, self.ws_rect = ws(B.svd_layer_workspace_bytes(d, d, m, K)), ws(B.svd_rect_workspace_bytes(vocab, d, vocab, d, m, K))
        self.ws_embed, self.ws_norm = ws(B.fasth_embed_workspace_bytes(vocab, d, m)), ws(B.fasth_norm_workspace_bytes(d, m))
        self.ws_prob = ws(B.fasth_log_prob_workspace_bytes(vocab, m))
        self.grads = B.tensor_list(self.g.values())
        self.ws_grad = ws(B.fasth_grad_workspace_bytes(self.grads))

    def load(self, ids, targets, gl, ge):
        import torch
        for t, a in ((self.ids, ids), (self.targets, targets), (self.gl, gl), (self.ge, ge)):
            t.copy_(torch.from_numpy(np.asarray(a)))

    def forward(self):
        B, p = self.B, self.p
        B.fasth_embed(p["table"], self.ids, self.X0, self.scale)
        B.fasth_norm(self.X0, p["w1"], self.Y1, self.r1, EPS)
        B.svd_layer_apply(p["Uv"], p["sigma"], p["Vv"], self.Y1, self.Z, self.ws_layer, K)
        B.fasth_norm(self.Z, p["w2"], self.Y2, self.r2, EPS, R=self.X0, S=self.S)
        B.svd_rect_apply(p["Ur"], p["sigma_r"], p["Vr"], self.Y2, self.logits, self.ws_rect, K)

    def step(self, max_norm):
        B, p, g = self.B, self.p, self.g
        self.forward()
        B.fasth_log_prob(self.logits, self.targets, self.logp, self.H, self.stats, self.ws_prob)
        B.fasth_log_prob_backward(self.logits, self.targets, self.stats, self.H, self.gl, self.ge, self.dlogits)
        B.svd_rect_apply_backward(p["Ur"], p["sigma_r"], p["Vr"], self.dlogits, g["Ur"], g["sigma_r"], g["Vr"], self.dY2, self.ws_rect, K)
        B.fasth_norm_backward(self.dY2, self.S, p["w2"], self.r2, self.dS, g["w2"], self.ws_norm)
        B.svd_layer_apply_backward(p["Uv"], p["sigma"], p["Vv"], self.dS, g["Uv"], g["sigma"], g["Vv"], self.dY1, self.ws_layer, K)
        B.fasth_norm_backward(self.dY1, self.X0, p["w1"], self.r1, self.dX0, g["w1"], self.ws_norm, dS=self.dS)
        B.fasth_embed_backward(self.ids, self.dX0, g["table"], self.ws_embed, self.scale)
        B.fasth_grad_clip(self.grads, max_norm, self.norm, self.ws_grad)

    def results(self):
        return [t.clone() for t in (self.logp, self.H, self.norm, *self.g.values())]


@pytest.mark.gpu
@pytest.mark.parametrize("m", [1, 40, 150])
def test_training_step_against_fp64(m):
    import torch
    vocab, d = 96, 64
    p = _parameters(3, vocab, d)
    batch = _batch(4, vocab, m)
    if m == 1:
        batch[1][0], batch[2][0] = 5, -1.0
    loss, g = _reference(p, *batch)
    model = Model(p, m)
    model.load(*batch)
    want, factor = tok.grad_clip(list(g.values()), 0.25 * tok.grad_norm(list(g.values())))
    model.step(0.25 * want)
    assert host(model.norm)[0] == pytest.approx(want, rel=1e-4)
    got = float(np.sum(batch[2] * host(model.logp)) + np.sum(batch[3] * host(model.H)))
    assert got == pytest.approx(loss, rel=1e-5)
    for name in g:
        assert_close(host(model.g[name]), g[name] * factor, name)


@pytest.mark.gpu
def test_next_token_alternatives():
    import torch
    from paper_2009_13977_amd import binding as B
    vocab, d = 96, 64
    p = _parameters(5, vocab, d)
    model = Model(p, 1)
    model.load([17], [-1], [0.0], [0.0])
    model.forward()
    top_logp, top_ids = torch.empty(4, 1, device="cuda"), torch.empty(4, 1, dtype=torch.int32, device="cuda")
    ws = B.new_workspace(B.fasth_log_prob_workspace_bytes(vocab, 1, 4))
    B.fasth_log_prob(model.logits, None, model.logp, model.H, model.stats, ws, top_logp, top_ids)
    q = {k: v.astype(np.float64) for k, v in p.items()}
    X0 = tok.embed(q["table"], [17], np.sqrt(d))
    Y1, _ = tok.norm(X0, q["w1"], EPS)
    Y2, _ = tok.norm(X0 + orc.svd_layer_apply(q["Uv"], q["sigma"], q["Vv"], Y1), q["w2"], EPS)
    logits = orc.rectangular_apply(q["Ur"], q["sigma_r"], q["Vr"], Y2)
    assert_close(host(model.logits), logits, "logits")
    _, H, want_logp, want_ids = tok.log_prob(logits, None, 4)
    np.testing.assert_array_equal(top_ids.cpu().numpy(), want_ids)
    np.testing.assert_allclose(host(top_logp), want_logp, rtol=1e-4, atol=1e-4)
    assert host(model.H)[0] == pytest.approx(H[0], rel=1e-4)


@pytest.mark.gpu
def test_step_on_another_stream_and_replayed_from_a_graph():
    """A captured step replayed with new tokens gives the bits of the eager step, with eager work of the same buffers' kind between."""
    import torch
    vocab, d, m = 96, 64, 40
    p = _parameters(6, vocab, d)
    eager, replayed = Model(p, m), Model(p, m)
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(stream):
        replayed.load(*_batch(7, vocab, m))
        replayed.step(0.01)
    stream.synchronize()
    eager.load(*_batch(7, vocab, m))
    eager.step(0.01)
    assert all(torch.equal(a, b) for a, b in zip(eager.results(), replayed.results()))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        replayed.step(0.01)
    for seed in range(10, 14):
        batch = _batch(seed, vocab, m)
        replayed.load(*batch)
        graph.replay()
        eager.load(*batch)
        eager.step(0.01)
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(eager.results(), replayed.results())), seed


@pytest.mark.gpu
def test_wide_operators_replayed_from_a_graph():
    """Sizes at which the operators split their work over workgroups and join it again."""
    import torch
    from paper_2009_13977_amd import binding as B
    vocab, d, m, top = 9000, 200, 700, 3
    f = lambda *s: torch.full(s, float("nan"), device="cuda")
    table, x, G, w = torch.randn(vocab, d, device="cuda"), torch.randn(vocab, m, device="cuda"), torch.randn(d, m, device="cuda"), torch.randn(d, device="cuda")
    ids = torch.randint(-1, vocab, (m,), device="cuda")
    out = {k: f(*s) for k, s in dict(X=(d, m), dTable=(vocab, d), Y=(d, m), rstd=(m,), dX=(d, m), dw=(d,), logp=(m,), H=(m,), stats=(2, m),
                                     top_logp=(top, m), dlogits=(vocab, m), norm=(1,)).items()}
    out["top_ids"] = torch.zeros(top, m, dtype=torch.int32, device="cuda")
    clipped = [torch.empty_like(table), torch.empty_like(w)]
    ws = [B.new_workspace(n) for n in (B.fasth_embed_workspace_bytes(vocab, d, m), B.fasth_norm_workspace_bytes(d, m),
                                       B.fasth_log_prob_workspace_bytes(vocab, m, top), B.fasth_grad_workspace_bytes(clipped))]

    def run(o, clipped):
        B.fasth_embed(table, ids, o["X"], 2.0)
        B.fasth_embed_backward(ids, G, o["dTable"], ws[0], 2.0)
        B.fasth_norm(G, w, o["Y"], o["rstd"])
        B.fasth_norm_backward(o["X"], G, w, o["rstd"], o["dX"], o["dw"], ws[1])
        B.fasth_log_prob(x, ids, o["logp"], o["H"], o["stats"], ws[2], o["top_logp"], o["top_ids"])
        B.fasth_log_prob_backward(x, ids, o["stats"], o["H"], o["logp"], o["H"], o["dlogits"])
        B.fasth_grad_clip([o["dTable"], o["dw"]], 1.0, o["norm"], ws[3], clipped)

    run(out, clipped)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        run(out, clipped)
    want = {k: torch.full_like(v, 0) for k, v in out.items()}
    want_clipped = [torch.empty_like(t) for t in clipped]
    for n in range(3):
        ids.copy_(torch.randint(-1, vocab, (m,), device="cuda"))
        x.normal_()
        G.normal_()
        graph.replay()
        torch.cuda.synchronize()
        got = {k: v.clone() for k, v in out.items()}
        got_clipped = [t.clone() for t in clipped]
        run(want, want_clipped)
        torch.cuda.synchronize()
        for k in got:
            assert torch.equal(got[k], want[k]), (n, k)
        assert all(torch.equal(a, b) for a, b in zip(got_clipped, want_clipped)), n
