"""fasth_grad_clip where the norm, or the factor, is at the end of fp32's range."""
import numpy as np
import pytest

from token_helpers import U, assert_within, host, torch_type


def _clip(grads, max_norm, out):
    import torch
    from paper_2009_13977_amd import binding as B
    norm = torch.full((1,), float("nan"), device="cuda")
    B.fasth_grad_clip(grads, max_norm, norm, B.new_workspace(B.fasth_grad_workspace_bytes(grads)), out)
    return norm


@pytest.mark.gpu
@pytest.mark.parametrize("place", ["in place", "into others"])
@pytest.mark.parametrize("more", [0, 120])  # (more tensors than one launch describes: the norm by a launch of its own)
def test_finite_entries_with_a_norm_beyond_fp32(more, place):
    """What *norm reads decides: infinite, and the gradients as they were."""
    import torch
    grads = [torch.full((4,), 3e38, device="cuda"), torch.ones(9000, device="cuda")] + [torch.ones(3, device="cuda") for _ in range(more)]
    kept = [g.clone() for g in grads]
    out = None if place == "in place" else [torch.full_like(g, float("nan")) for g in grads]
    norm = _clip(grads, 1.0, out)
    assert torch.isposinf(norm).all()
    assert all(torch.equal(a, b) for a, b in zip(kept, out or grads))


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("more", [0, 120])
@pytest.mark.parametrize("max_norm", [1.0, 2.5e-3, 1e-10, 3e-30, 0.0])
def test_factors_below_the_smallest_normal_number(max_norm, more, dtype):
    """A norm of some 2.7e38: the factor is 4e-39 and less."""
    import torch
    r = np.random.default_rng(1)
    shapes = [20000, 8192, 5] + [7] * more  # whole chunks and parts
    grads = [torch.from_numpy(r.normal(size=n)).to(torch_type(dtype)).cuda() for n in shapes]
    grads[0] *= 1e36
    grads[1] *= 1e35
    grads[2] *= 7e37
    g64 = [host(g) for g in grads]
    want = np.sqrt(sum((g ** 2).sum() for g in g64))
    assert 1e38 < want < 3.4e38
    norm = _clip(grads, max_norm, None)
    assert_within(norm, np.array([want]), 2.0 ** -30 * want, "fp32", "norm")
    for i, (g, w) in enumerate(zip(grads, g64)):
        exact = w * (float(np.float32(max_norm)) / want)
        # the factor and the product in fp64, one rounding to fp32, then one to the type
        assert_within(g, exact, 2.0 ** -50 * np.abs(exact) + U * np.abs(exact) + 2.0 ** -150, dtype, f"tensor {i}")


@pytest.mark.gpu
def test_a_kept_list_keeps_its_memory():
    """A tensor of a kept list gets other memory, twice: a smaller one never comes to lie where the list's first one was."""
    import torch
    from paper_2009_13977_amd import binding as B
    t = torch.ones(64, device="cuda")
    kept = B.tensor_list([t])
    at, norm, ws = t.data_ptr(), torch.empty(1, device="cuda"), B.new_workspace(B.fasth_grad_workspace_bytes([t]))
    for n in (64, 16, 16, 64, 5):
        t.data = torch.ones(n, device="cuda")
        assert t.data_ptr() != at
        with pytest.raises(ValueError, match="not where it was"):
            B.fasth_grad_clip(kept, 1.0, norm, ws)
