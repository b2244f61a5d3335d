"""Shared by the tests of the operators around the layers: types, inputs on the GPU, elementwise bounds."""
import numpy as np

U = 2.0 ** -24  # a rounding to fp32 is off by at most this part of the value
TYPES = ("fp32", "bf16", "fp16")
HALF_STEP = {"fp32": 2.0 ** -24, "bf16": 2.0 ** -8, "fp16": 2.0 ** -11}
# below the smallest normal number a rounding is off by half the spacing there
SMALLEST = {"fp32": 2.0 ** -150, "bf16": 2.0 ** -134, "fp16": 2.0 ** -25}


def torch_type(name):
    import torch
    return {"fp32": torch.float32, "bf16": torch.bfloat16, "fp16": torch.float16}[name]


def normal(seed, *shape, dtype="fp32", scale=1.0):
    """(GPU tensor, the same numbers in fp64)."""
    import torch
    a = np.random.default_rng(seed).normal(size=shape) * scale
    t = torch.from_numpy(a).to(torch_type(dtype))
    return t.cuda(), t.double().numpy()


def tokens(seed, vocab, m, bits=64, padded=True, dtype_ids=None):
    """Token numbers, some frequent and some rare; a tenth of the columns without one if `padded`."""
    import torch
    r = np.random.default_rng(seed)
    ids = np.minimum((vocab ** r.random(m)).astype(np.int64), vocab) - 1
    ids = r.permutation(vocab)[ids]
    if padded:
        ids = np.where(r.random(m) < 0.1, r.choice([-1, vocab, vocab + 7, -2 ** 31], m), ids)
    return torch.from_numpy(ids.astype(np.int64 if bits == 64 else np.int32)).cuda(), ids


def host(t):
    return t.detach().double().cpu().numpy()


def assert_within(got, want, bound, dtype, what):
    """|got - want| <= bound + the rounding to the output's type, entry by entry."""
    got = host(got)
    assert got.shape == want.shape, (what, got.shape, want.shape)
    limit = bound + HALF_STEP[dtype] * (np.abs(want) + bound) + SMALLEST[dtype]
    with np.errstate(invalid="ignore"):
        off = np.abs(got - want)
    bad = ~(off <= limit) & ~((got == want) | (np.isnan(got) & np.isnan(want)))
    if bad.any():
        at = tuple(np.argwhere(bad)[0])
        raise AssertionError(f"{what}: {bad.sum()} of {bad.size} entries off, first at {at}: {got[at]!r} for {want[at]!r}, "
                             f"bound {np.broadcast_to(limit, want.shape)[at]!r}")
