"""fasth_grad_norm and fasth_grad_clip against the fp64 definition."""
import ctypes

import numpy as np
import pytest

from oracle import tokens as tok
from token_helpers import HALF_STEP, U, assert_within, host, normal, torch_type

# sizes around the vector width, the chunk of a workgroup, and many tensors (more than one launch's descriptions)
LISTS = {
    "one entry": [((1,), "fp32")],
    "small": [((3,), "fp32"), ((7, 5), "bf16"), ((1,), "fp16"), ((0,), "fp32"), ((2, 0), "bf16")],
    "around a chunk": [((8191,), "fp32"), ((8192,), "bf16"), ((8193,), "fp16"), ((16384,), "fp32"), ((24577,), "bf16")],
    "layer": [((300, 300), "fp32"), ((300,), "fp32"), ((300, 300), "fp32")],
    "many": [((5 + i % 9,), ("fp32", "bf16", "fp16")[i % 3]) for i in range(250)],
    "large": [((3001, 4003), "fp32"), ((2000, 5000), "bf16"), ((10,), "fp32")],
    "none": [],
}


def _tensors(name):
    return list(zip(*(normal(i + 1, *shape, dtype=dtype) for i, (shape, dtype) in enumerate(LISTS[name])))) or [(), ()]


def _clip(grads, max_norm, out=None):
    import torch
    from paper_2009_13977_amd import binding as B
    norm = torch.full((1,), float("nan"), device="cuda")
    ws = B.new_workspace(B.fasth_grad_workspace_bytes(grads)).fill_(0xFF)
    B.fasth_grad_clip(grads, max_norm, norm, ws, out)
    alone = torch.full((1,), float("nan"), device="cuda")
    return norm, alone


@pytest.mark.gpu
@pytest.mark.parametrize("place", ["in place", "into others"])
@pytest.mark.parametrize("part", [0.0, 0.37, 1.5])
@pytest.mark.parametrize("name", LISTS)
def test_norm_and_clipping(name, part, place):
    import torch
    from paper_2009_13977_amd import binding as B
    grads, g64 = _tensors(name)
    before = [g.clone() for g in grads]
    want, _ = tok.grad_clip(g64, 1.0)
    limit = float(np.float32(part * want))
    _, factor = tok.grad_clip(g64, limit)
    norm = torch.full((1,), float("nan"), device="cuda")
    ws = B.new_workspace(B.fasth_grad_workspace_bytes(grads)).fill_(0xFF)
    B.fasth_grad_norm(grads, norm, ws)
    # squares of fp32 numbers are exact in fp64, and so are the sums but for 2^-53 each: one rounding to fp32 is left
    assert_within(norm, np.array([want]), 2.0 ** -30 * want, "fp32", "norm alone")
    norm.fill_(float("nan"))
    out = None if place == "in place" else [torch.full_like(g, float("nan")) for g in grads]
    B.fasth_grad_clip(grads, limit, norm, ws, out)
    assert_within(norm, np.array([want]), 2.0 ** -30 * want, "fp32", "norm")
    for i, (g, g0, w) in enumerate(zip(grads if out is None else out, before, g64)):
        if factor == 1.0:
            assert (g == g0).all(), i
        else:  # the factor and the product are rounded once each, then the result to its type
            assert_within(g, w * factor, 2.01 * U * np.abs(w * factor), LISTS[name][i][1], f"tensor {i}")
        if out is not None:
            assert (grads[i] == g0).all()


@pytest.mark.gpu
@pytest.mark.parametrize("place", ["in place", "into others"])
def test_more_chunks_than_workgroups_of_a_launch(place):
    """8193 and more chunks: the norm is finished by a launch of its own and every workgroup scales one chunk."""
    import torch
    from paper_2009_13977_amd import binding as B
    gen = torch.Generator(device="cuda")
    gen.manual_seed(1)
    grads = [torch.randn(8192 * 5000 + 3, device="cuda", generator=gen), torch.randn(8192 * 3200 + 1, device="cuda", generator=gen).to(torch.bfloat16)]
    before = [g.clone() for g in grads]
    want = float(sum((g.double() ** 2).sum() for g in grads)) ** 0.5
    limit = float(np.float32(0.3 * want))
    norm = torch.full((1,), float("nan"), device="cuda")
    ws = B.new_workspace(B.fasth_grad_workspace_bytes(grads)).fill_(0xFF)
    out = grads if place == "in place" else [torch.full_like(g, float("nan")) for g in grads]
    B.fasth_grad_clip(grads, limit, norm, ws, None if place == "in place" else out)
    assert abs(float(norm) - want) <= 1.01 * U * want
    for g, o in zip(before, out):
        exact = g.double() * (limit / want)
        bound = (2.01 * U + (2.0 ** -8 if g.dtype == torch.bfloat16 else U)) * exact.abs() * 1.01 + 2.0 ** -130
        assert ((o.double() - exact).abs() <= bound).all()


@pytest.mark.gpu
def test_large_small_and_infinite_gradients():
    import torch
    from paper_2009_13977_amd import binding as B
    a = torch.full((1000,), 1e30, device="cuda")
    b = torch.full((50,), 1e-30, device="cuda")
    norm, _ = _clip([a, b], 1.0)
    assert norm.item() == pytest.approx(1e30 * 1000 ** 0.5, rel=1e-6) and a[0].item() == pytest.approx(1000 ** -0.5, rel=1e-6)
    tiny = torch.full((4,), 1e-30, device="cuda")
    norm, _ = _clip([tiny], 1e-31)
    assert norm.item() == pytest.approx(2e-30, rel=1e-6) and tiny[0].item() == pytest.approx(5e-32, rel=1e-6)
    for bad in (float("inf"), float("nan")):
        g = torch.ones(9000, device="cuda")
        g[8500] = bad
        kept = g.clone()
        norm, _ = _clip([g, torch.ones(5, device="cuda")], 1.0)
        assert not np.isfinite(norm.item()) and torch.equal(g.isnan(), kept.isnan()) and (g[:8500] == 1).all()


@pytest.mark.gpu
def test_repeated_calls_and_lists_kept_by_the_program():
    import torch
    from paper_2009_13977_amd import binding as B
    grads, _ = _tensors("around a chunk")
    kept, out = B.tensor_list(grads), B.tensor_list([torch.empty_like(g) for g in grads])
    ws, norm = B.new_workspace(B.fasth_grad_workspace_bytes(kept)), torch.empty(1, device="cuda")
    B.fasth_grad_clip(kept, 3.0, norm, ws, out)
    first = [norm.clone()] + [t.clone() for t in out.tensors]
    for _ in range(3):
        B.fasth_grad_clip(kept, 3.0, norm, ws, out)
        assert all((a == b).all() for a, b in zip(first, [norm, *out.tensors]))


@pytest.mark.gpu
def test_refuses_what_it_cannot_take():
    import torch
    from paper_2009_13977_amd import binding as B
    g, norm = torch.ones(64, device="cuda"), torch.empty(1, device="cuda")
    ws = B.new_workspace(B.fasth_grad_workspace_bytes([g, g]))
    for max_norm in (-1.0, float("nan")):
        with pytest.raises(B.FasthError):
            B.fasth_grad_clip([g], max_norm, norm, ws)
    for tensors, out in (([g, g], None), ([g[:32], g[16:48]], None), ([g, torch.ones(64, device="cuda")], [torch.empty(64, device="cuda"), g]),
                         ([g[:32]], [g[16:48]])):
        with pytest.raises(B.FasthError) as e:
            B.fasth_grad_clip(tensors, 1.0, norm, ws, out)
        assert e.value.code == B.FASTH_EINVAL
    with pytest.raises(ValueError):
        B.fasth_grad_clip([g], 1.0, norm, ws, [torch.empty(63, device="cuda")])
    with pytest.raises(ValueError):
        B.fasth_grad_norm([g[::2]], norm, ws)
    with pytest.raises(ValueError):
        B.fasth_grad_norm([g.double()], norm, ws)
    with pytest.raises(TypeError):
        B.fasth_grad_norm([None], norm, ws)
    with pytest.raises(B.FasthError) as e:
        B.fasth_grad_norm([g], norm, B.new_workspace(16))
    assert e.value.code == B.FASTH_EWORKSPACE


@pytest.mark.gpu
def test_a_kept_list_refuses_tensors_that_moved():
    import torch
    from paper_2009_13977_amd import binding as B
    grads, _ = _tensors("small")
    kept = B.tensor_list(grads)
    ws, norm = B.new_workspace(B.fasth_grad_workspace_bytes(kept)), torch.empty(1, device="cuda")
    B.fasth_grad_clip(kept, 3.0, norm, ws)
    old = grads[1].data
    grads[1].data = torch.zeros_like(old)
    for call in (lambda: B.fasth_grad_clip(kept, 3.0, norm, ws), lambda: B.fasth_grad_norm(kept, norm, ws),
                 lambda: B.fasth_grad_clip([t.clone() for t in grads], 3.0, norm, ws, kept)):
        with pytest.raises(ValueError, match="not where it was"):
            call()
    grads[1].data = old
    B.fasth_grad_clip(kept, 3.0, norm, ws)
