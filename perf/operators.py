"""Timed cases of the operators around the layers of a token model: the embedding, the norm with the residual's
addition, the log probabilities of the given tokens, and the clipping of all gradients by their global norm.

Mini-batches are [features][samples], one token per column, as the library's layers take them. A case is a dict:

  op      "embed", "norm", "log_prob" or "grad_clip"
  train   the backward pass runs too, and its gradients are returned
  dtype   of the embedding's table, the norm's output, the logits; "mixed" for a list of gradients of several types
  vocab   rows of the table, rows of the logits
  d, m    features, columns; for "grad_clip" the vector length and the number of layers whose gradients are clipped
  top     alternatives per column ("log_prob")
  extra   "norm": there is a residual. "log_prob": a part of the vocabulary is masked with -infinity.
          "grad_clip": there is an embedding's gradient too
  loose   "grad_clip": the norm stays below its limit, so that the gradients come back as they are
"""
import math

import torch

own = False

_TYPES = {"fp32": torch.float32, "bf16": torch.bfloat16, "fp16": torch.float16}
_SIZE = {"fp32": 4, "bf16": 2, "fp16": 2}
_EPS = 1e-6


def _case(name, op, dtype, vocab, d, m, train=False, top=0, extra=False, loose=False):
    case = {"op": op, "dtype": dtype, "vocab": vocab, "d": d, "m": m, "train": train, "top": top, "extra": extra, "loose": loose}
    if name:
        case["name"] = name
    return case


def listed():
    return [
        # The next token of one sequence: a latency test.
        _case("embed_serve_m1", "embed", "bf16", 32000, 1024, 1),
        # A training step's tokens at the benchmark's vector length.
        _case("embed_train_d1024_m4096", "embed", "fp32", 32000, 1024, 4096, train=True),
        # Nothing a multiple of anything: an odd vocabulary, the length of 28 x 28 inputs, a ragged mini-batch.
        _case("embed_train_d784_m9001", "embed", "bf16", 50021, 784, 9001, train=True),
        # Between two layers while a few sequences are decoded.
        _case("norm_serve_d2048_m5", "norm", "fp32", 0, 2048, 5, extra=True),
        # A mini-batch of the smaller layers, no residual, the output in 16 bits for the product that makes the logits.
        _case("norm_train_d784_m1001", "norm", "bf16", 0, 784, 1001, train=True),
        # A long mini-batch of the largest layers.
        _case("norm_train_d4096_m8192", "norm", "fp32", 0, 4096, 8192, train=True, extra=True),
        # The next token's alternatives, one sequence.
        _case("log_prob_serve_v128000_m1", "log_prob", "bf16", 128000, 0, 1, top=8),
        # The same for a batch of requests, part of the vocabulary masked.
        _case("log_prob_serve_v32003_m48", "log_prob", "fp32", 32003, 0, 48, top=5, extra=True),
        # Characters: few rows, many columns.
        _case("log_prob_train_v256_m16384", "log_prob", "fp32", 256, 0, 16384, train=True),
        # The largest: a large vocabulary, a training step's tokens.
        _case("log_prob_train_v128000_m4096", "log_prob", "bf16", 128000, 0, 4096, train=True),
        # Gradients of twelve layers of the benchmark's size: two matrices and the diagonal each.
        _case("grad_clip_d1024_layers12", "grad_clip", "fp32", 0, 1024, 12),
        # Larger layers in 16 and 32 bits, with an embedding's gradient.
        _case("grad_clip_d2048_layers16", "grad_clip", "mixed", 50021, 2048, 16, extra=True),
    ]


def _log_uniform(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _length(rng, hi):
    """A vector length in [32, hi]: a third are multiples of 64, a third of 4, a third anything."""
    d = _log_uniform(rng, 32, hi)
    kind = rng.randrange(3)
    return max(64, d // 64 * 64) if kind == 0 else max(32, d // 4 * 4) if kind == 1 else d


def draw(rng):
    limit = max(work(c)["bytes"] for c in listed())
    while True:
        op = rng.choice(("embed", "norm", "log_prob", "grad_clip"))
        dtype = rng.choice(("fp32", "bf16", "fp16"))
        train, extra = rng.random() < 0.6, rng.random() < 0.5
        if op == "embed":
            case = _case(None, op, dtype, _log_uniform(rng, 32, 131072), _length(rng, 4096), _log_uniform(rng, 1, 16384), train)
        elif op == "norm":
            case = _case(None, op, dtype, 0, _length(rng, 16384), _log_uniform(rng, 1, 16384), train, extra=extra)
        elif op == "log_prob":
            # alternatives are asked for while tokens are drawn, in training the log probabilities alone
            m = _log_uniform(rng, 1, 16384 if train else 256)
            case = _case(None, op, dtype, _log_uniform(rng, 32, 131072), 0, m, train, 0 if train else rng.randrange(17), extra)
        else:
            dtype = rng.choice(("fp32", "bf16", "mixed"))
            case = _case(None, op, dtype, _log_uniform(rng, 32, 131072) if extra else 0, _length(rng, 4096), _log_uniform(rng, 1, 18),
                         extra=extra, loose=rng.random() < 0.25)
        if work(case)["bytes"] <= limit:
            return case


class _Inputs:
    """Seeded numbers in GPU memory."""

    def __init__(self, seed):
        self.gen = torch.Generator(device="cuda")
        self.gen.manual_seed(seed)

    def normal(self, *shape, dtype=torch.float32, scale=1.0):
        return (torch.randn(*shape, generator=self.gen, device="cuda", dtype=torch.float32) * scale).to(dtype)

    def uniform(self, *shape):
        return torch.rand(*shape, generator=self.gen, device="cuda", dtype=torch.float32)

    def tokens(self, vocab, m, padded):
        """Token numbers whose frequencies fall like one over their rank, the ranks strewn over the vocabulary, and a
        few columns without a token (-1) where the mini-batch is padded."""
        rank = torch.exp(self.uniform(m).double() * math.log(vocab + 1)).long().clamp(1, vocab) - 1
        ids = torch.randperm(vocab, generator=self.gen, device="cuda")[rank]
        return torch.where(self.uniform(m) < 0.03, torch.full_like(ids, -1), ids) if padded else ids


def _gradient_types(case):
    """(shape, type) of every gradient: dUv, dsigma and dVv of each layer, then the table's."""
    d, layers = case["d"], case["m"]
    types = {"fp32": (torch.float32,) * 3, "bf16": (torch.bfloat16,) * 3, "mixed": (torch.float32, torch.float32, torch.bfloat16)}[case["dtype"]]
    got = [(shape, t) for _ in range(layers) for shape, t in zip(((d, d), (d,), (d, d)), types)]
    return got + [((case["vocab"], d), types[2])] * bool(case["extra"])


def prepare(case, seed):
    op, vocab, d, m, train = case["op"], case["vocab"], case["d"], case["m"], case["train"]
    dtype = _TYPES.get(case["dtype"])
    r = _Inputs(seed)
    s = dict(case)
    if op == "embed":
        s["table"] = r.normal(vocab, d, dtype=dtype, scale=0.05)
        s["ids"] = r.tokens(vocab, m, train)
        s["scale"] = math.sqrt(d)
        if train:
            s["G"] = r.normal(d, m, scale=1e-3)
        if own:
            s["X"] = torch.empty(d, m, device="cuda")
            if train:
                s["dTable"] = torch.empty_like(s["table"])
                s["ws"] = _library().new_workspace(_library().fasth_embed_workspace_bytes(vocab, d, m))
    elif op == "norm":
        s["X"] = r.normal(d, m)
        s["R"] = r.normal(d, m, scale=3.0) if case["extra"] else None
        s["w"] = 1.0 + r.normal(d, scale=0.2)
        if train:
            s["G"] = r.normal(d, m, dtype=dtype, scale=1e-2)
            s["dS"] = r.normal(d, m, scale=1e-2) if case["extra"] else None
        if own:
            s["S"] = torch.empty_like(s["X"]) if case["extra"] else None
            s["Y"] = torch.empty(d, m, device="cuda", dtype=dtype)
            s["rstd"] = torch.empty(m, device="cuda")
            if train:
                s["dX"], s["dw"] = torch.empty_like(s["X"]), torch.empty_like(s["w"])
                s["ws"] = _library().new_workspace(_library().fasth_norm_workspace_bytes(d, m))
    elif op == "log_prob":
        s["logits"] = r.normal(vocab, m, dtype=dtype, scale=2.5)
        s["ids"] = r.tokens(vocab, m, train)
        if case["extra"]:
            masked = r.uniform(vocab) < 0.25
            masked[s["ids"].clamp(min=0)] = False
            s["logits"][masked] = -math.inf
        if train:
            count = 1 if case["dtype"] == "fp16" else m  # fp16 gradients of a mean over many columns would underflow
            s["g_logp"] = torch.where(s["ids"] >= 0, -1.0 / count, 0.0)
            s["g_entropy"] = torch.full((m,), -0.01 / count, device="cuda")
        if own:
            s["logp"], s["entropy"], s["stats"] = (torch.empty(*n, device="cuda") for n in ((m,), (m,), (2, m)))
            s["top_logp"] = torch.empty(case["top"], m, device="cuda") if case["top"] else None
            s["top_ids"] = torch.empty(case["top"], m, device="cuda", dtype=torch.int32) if case["top"] else None
            s["ws"] = _library().new_workspace(_library().fasth_log_prob_workspace_bytes(vocab, m, case["top"]))
            if train:
                s["dlogits"] = torch.empty_like(s["logits"])
    else:
        s["grads"] = [r.normal(*shape, dtype=t, scale=1e-3) for shape, t in _gradient_types(case)]
        s["max_norm"] = (2e-3 if case["loose"] else 0.5e-3) * math.sqrt(sum(g.numel() for g in s["grads"]))
        if own:
            s["clipped"] = [torch.empty_like(g) for g in s["grads"]]
            s["norm"] = torch.empty(1, device="cuda")
            # the buffers of a training program do not move: it describes them once
            s["grads_list"], s["clipped_list"] = _library().tensor_list(s["grads"]), _library().tensor_list(s["clipped"])
            s["ws"] = _library().new_workspace(_library().fasth_grad_workspace_bytes(s["grads_list"]))
    return s


def _library():
    from paper_2009_13977_amd import binding
    return binding


def run(s):
    if own:
        return {"embed": _embed_own, "norm": _norm_own, "log_prob": _log_prob_own, "grad_clip": _grad_clip_own}[s["op"]](s)
    return {"embed": _embed_plain, "norm": _norm_plain, "log_prob": _log_prob_plain, "grad_clip": _grad_clip_plain}[s["op"]](s)


def _embed_own(s):
    B = _library()
    B.fasth_embed(s["table"], s["ids"], s["X"], s["scale"])
    if not s["train"]:
        return {"X": s["X"]}
    B.fasth_embed_backward(s["ids"], s["G"], s["dTable"], s["ws"], s["scale"])
    return {"X": s["X"], "dTable": s["dTable"]}


def _norm_own(s):
    B = _library()
    B.fasth_norm(s["X"], s["w"], s["Y"], s["rstd"], _EPS, s["R"], s["S"])
    out = {"Y": s["Y"]}
    if s["extra"]:
        out["S"] = s["S"]
    if s["train"]:
        B.fasth_norm_backward(s["G"], s["S"] if s["extra"] else s["X"], s["w"], s["rstd"], s["dX"], s["dw"], s["ws"], s["dS"])
        out["dX"], out["dw"] = s["dX"], s["dw"]
    return out


def _log_prob_own(s):
    B = _library()
    B.fasth_log_prob(s["logits"], s["ids"], s["logp"], s["entropy"], s["stats"], s["ws"], s["top_logp"], s["top_ids"])
    out = {"logp": s["logp"], "entropy": s["entropy"]}
    if s["top"]:
        out["top_logp"], out["top_ids"] = s["top_logp"], s["top_ids"]
    if s["train"]:
        B.fasth_log_prob_backward(s["logits"], s["ids"], s["stats"], s["entropy"], s["g_logp"], s["g_entropy"], s["dlogits"])
        out["dlogits"] = s["dlogits"]
    return out


def _grad_clip_own(s):
    _library().fasth_grad_clip(s["grads_list"], s["max_norm"], s["norm"], s["ws"], s["clipped_list"])
    return {"norm": s["norm"], "clipped": s["clipped"]}


def _embed_plain(s):
    ids, known = s["ids"].clamp(min=0), s["ids"] >= 0
    out = {"X": (s["table"][ids].float() * s["scale"] * known[:, None]).t().contiguous()}
    if s["train"]:
        rows = s["G"].t() * (known * s["scale"])[:, None]
        out["dTable"] = torch.zeros(s["table"].shape, device="cuda").index_add_(0, ids, rows).to(s["table"].dtype)
    return out


def _norm_plain(s):
    S = s["X"] + s["R"] if s["extra"] else s["X"]
    rstd = torch.rsqrt(S.square().mean(0) + _EPS)
    out = {"Y": (S * rstd * s["w"][:, None]).to(_TYPES[s["dtype"]])}
    if s["extra"]:
        out["S"] = S
    if s["train"]:
        g = s["G"].float()
        wg = g * s["w"][:, None]
        c = (wg * S).sum(0) * rstd.pow(3) / s["d"]
        dX = wg * rstd - S * c
        out["dX"] = dX + s["dS"] if s["extra"] else dX
        out["dw"] = (g * S * rstd).sum(1)
    return out


def _log_prob_plain(s):
    x = s["logits"].float()
    ids, known = s["ids"].clamp(min=0), s["ids"] >= 0
    t = x - x.amax(0)
    e = torch.exp(t)
    total = e.sum(0)
    log_total = total.log()
    p = e / total
    lp = torch.where(p > 0, t - log_total, 0.0)
    entropy = -(p * lp).sum(0)
    given = t.gather(0, ids[None])[0] - log_total
    out = {"logp": torch.where(known, given, 0.0), "entropy": entropy}
    if s["top"]:
        value, row = torch.sort(t, dim=0, descending=True, stable=True)  # ties to the lowest row
        value, row = value[: s["top"]], row[: s["top"]]
        missing = s["top"] - value.shape[0]
        value = torch.cat([value, torch.full((missing, s["m"]), -math.inf, device="cuda")])
        row = torch.cat([row, torch.full((missing, s["m"]), -1, device="cuda")])
        out["top_logp"] = value - log_total
        out["top_ids"] = torch.where(value > -math.inf, row, -1).int()
    if s["train"]:
        dx = -p * (s["g_logp"] + s["g_entropy"] * (lp + entropy))
        out["dlogits"] = dx.scatter_add_(0, ids[None], (s["g_logp"] * known)[None]).to(s["logits"].dtype)
    return out


def _grad_clip_plain(s):
    norm = torch.stack([g.float().square().sum() for g in s["grads"]]).sum().sqrt()
    c = torch.clamp(s["max_norm"] / norm, max=1.0)
    return {"norm": norm.reshape(1), "clipped": [(g.float() * c).to(g.dtype) for g in s["grads"]]}


def exact(case, seed):
    """The definitions in 64 bits."""
    s = prepare(case, seed)
    op, m = case["op"], case["m"]
    if op == "embed":
        known = (s["ids"] >= 0).nonzero()[:, 0]
        rows = s["ids"][known]
        X = torch.zeros(case["d"], m, device="cuda", dtype=torch.float64)
        X[:, known] = s["table"].double()[rows].t() * s["scale"]
        out = {"X": X}
        if case["train"]:
            order = torch.argsort(rows)
            out["dTable"] = torch.zeros(s["table"].shape, device="cuda", dtype=torch.float64)
            out["dTable"].index_add_(0, rows[order], s["G"].double()[:, known[order]].t() * s["scale"])
        return out
    if op == "norm":
        S = s["X"].double() + s["R"].double() if case["extra"] else s["X"].double()
        rms = ((S * S).sum(0) / case["d"] + _EPS).sqrt()
        U, w = S / rms, s["w"].double()[:, None]
        out = {"Y": w * U}
        if case["extra"]:
            out["S"] = S
        if case["train"]:
            G = s["G"].double()
            out["dX"] = (w * G - U * (w * G * U).mean(0)) / rms
            if case["extra"]:
                out["dX"] = out["dX"] + s["dS"].double()
            out["dw"] = (G * U).sum(1)
        return out
    if op == "log_prob":
        out = {"logp": torch.zeros(m, device="cuda", dtype=torch.float64), "entropy": torch.empty(m, device="cuda", dtype=torch.float64)}
        if case["top"]:
            out["top_logp"], out["top_ids"] = torch.full((case["top"], m), -math.inf, device="cuda", dtype=torch.float64), None
        if case["train"]:
            out["dlogits"] = torch.empty(case["vocab"], m, device="cuda", dtype=torch.float64)
        width = max(1, (1 << 26) // case["vocab"])
        for j in range(0, m, width):
            x, ids = s["logits"][:, j:j + width].double(), s["ids"][j:j + width]
            lp = x - torch.logsumexp(x, 0)
            p = lp.exp()
            H = -torch.special.xlogy(p, p).sum(0)
            known = (ids >= 0).nonzero()[:, 0]
            out["entropy"][j:j + width] = H
            out["logp"][j + known] = lp[ids[known], known]
            if case["top"]:
                k = min(case["top"], case["vocab"])
                out["top_logp"][:k, j:j + width] = lp.topk(k, 0).values
            if case["train"]:
                gl, ge = s["g_logp"][j:j + width].double(), s["g_entropy"][j:j + width].double()
                dx = -ge * (torch.special.xlogy(p, p) + p * H) - gl * p
                dx[ids[known], known] += gl[known]
                out["dlogits"][:, j:j + width] = dx
        return out
    squares = [(g.double() ** 2).sum() for g in s["grads"]]
    norm = sum(squares) ** 0.5
    c = 1.0 if norm <= s["max_norm"] else s["max_norm"] / norm
    return {"norm": norm.reshape(1), "clipped": [g.double() * c for g in s["grads"]]}


def work(case):
    """Every input read once and every output written once."""
    op, vocab, d, m, train = case["op"], case["vocab"], case["d"], case["m"], case["train"]
    w = _SIZE.get(case["dtype"], 0)
    if op == "embed":
        moved, flops = 8 * m + d * m * (w + 4), d * m
        if train:
            moved, flops = moved + 4 * d * m + w * vocab * d, flops + 2 * d * m
    elif op == "norm":
        moved, flops = d * m * (4 + w + 8 * case["extra"]) + 4 * d, 5 * d * m
        if train:
            moved, flops = moved + d * m * (4 + w + 4 * case["extra"]) + 4 * d, flops + 10 * d * m
    elif op == "log_prob":
        moved, flops = w * vocab * m + 8 * m * (2 + case["top"]), 5 * vocab * m
        if train:
            moved, flops = moved + w * vocab * m + 8 * m, flops + 8 * vocab * m
    else:
        sizes = [(math.prod(shape), torch.empty(0, dtype=t).element_size()) for shape, t in _gradient_types(case)]
        moved, flops = sum(2 * n * b for n, b in sizes), sum(3 * n for n, _ in sizes)
    return {"bytes": moved, "flops": flops}
