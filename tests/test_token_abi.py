"""Host-only checks of the entry points around the layers: arguments are refused before any GPU call."""
import ctypes

import pytest

from paper_2009_13977_amd import binding as B

BIG = 1 << 40
P, ODD = 256, 264  # aligned and unaligned addresses, never dereferenced


def _embed(**kw):
    s = {"vocab": 10, "d": 8, "m": 4, "dtype": 0, "id_bits": 64, **kw}
    return B.fasth_embed_shape(s["vocab"], s["d"], s["m"], s["dtype"], s["id_bits"])


def _norm(**kw):
    s = {"d": 8, "m": 4, "dtype": 0, "eps": 1e-6, **kw}
    return B.fasth_norm_shape(s["d"], s["m"], s["dtype"], s["eps"])


def _prob(**kw):
    s = {"vocab": 10, "m": 4, "dtype": 0, "id_bits": 64, "top": 0, **kw}
    return B.fasth_log_prob_shape(s["vocab"], s["m"], s["dtype"], s["id_bits"], s["top"])


BAD_EMBED = [(dict(vocab=0), -1), (dict(d=0), -1), (dict(m=0), -1), (dict(m=-5), -1), (dict(dtype=3), -1), (dict(dtype=-1), -1),
             (dict(id_bits=16), -1), (dict(vocab=(1 << 24) + 1), -5), (dict(d=16385), -5), (dict(m=65536), -5)]


@pytest.mark.parametrize("kw,code", BAD_EMBED)
def test_embed_shapes(kw, code):
    lib, s = B.load_library(), _embed(**kw)
    assert lib.fasth_embed(ctypes.byref(s), P, P, 1.0, P, None) == code
    assert lib.fasth_embed_backward(ctypes.byref(s), P, P, 1.0, P, P, BIG, None) == code
    assert lib.fasth_embed_workspace_bytes(ctypes.byref(s)) == 0


def test_embed_arguments():
    lib, s = B.load_library(), _embed()
    for at in (0, 1, 3):
        for value, code in ((None, B.FASTH_EINVAL), (ODD, B.FASTH_EALIGN)):
            a = [P, P, 1.0, P]
            a[at] = value
            assert lib.fasth_embed(ctypes.byref(s), *a, None) == code
    for at in (0, 1, 3, 4):
        for value, code in ((None, B.FASTH_EINVAL), (ODD, B.FASTH_EALIGN)):
            a = [P, P, 1.0, P, P]
            a[at] = value
            assert lib.fasth_embed_backward(ctypes.byref(s), *a, BIG, None) == code
    need = lib.fasth_embed_workspace_bytes(ctypes.byref(s))
    assert need >= 4 * 8 * 4 + 4 * 11 + 4 * 4
    assert lib.fasth_embed_backward(ctypes.byref(s), P, P, 1.0, P, P, need - 1, None) == B.FASTH_EWORKSPACE
    assert lib.fasth_embed(None, P, P, 1.0, P, None) == B.FASTH_EINVAL
    assert B.fasth_embed_workspace_bytes(1 << 24, 16384, 65535) > 65535 * 16384 * 4


@pytest.mark.parametrize("kw,code", [(dict(d=0), -1), (dict(m=0), -1), (dict(dtype=7), -1), (dict(eps=0.0), -1), (dict(eps=-1.0), -1),
                                     (dict(eps=float("nan")), -1), (dict(eps=float("inf")), -1), (dict(d=16385), -5), (dict(m=65536), -5)])
def test_norm_shapes(kw, code):
    lib, s = B.load_library(), _norm(**kw)
    assert lib.fasth_norm(ctypes.byref(s), P, P, P, P, P, P, None) == code
    assert lib.fasth_norm_backward(ctypes.byref(s), P, P, P, P, P, P, P, P, BIG, None) == code
    assert lib.fasth_norm_workspace_bytes(ctypes.byref(s)) == 0


def test_norm_arguments():
    lib, s = B.load_library(), _norm()
    for at in range(6):
        a = [P] * 6
        a[at] = ODD
        assert lib.fasth_norm(ctypes.byref(s), *a, None) == B.FASTH_EALIGN
        a[at] = None  # (a residual without a place for the sum, and the other way round, too)
        assert lib.fasth_norm(ctypes.byref(s), *a, None) == B.FASTH_EINVAL
    for at in range(8):
        a = [P] * 8
        a[at] = ODD
        assert lib.fasth_norm_backward(ctypes.byref(s), *a, BIG, None) == B.FASTH_EALIGN
        a[at] = None
        if at not in (4, 6):  # dS and dweight may be null
            assert lib.fasth_norm_backward(ctypes.byref(s), *a, BIG, None) == B.FASTH_EINVAL
    need = lib.fasth_norm_workspace_bytes(ctypes.byref(s))
    assert lib.fasth_norm_backward(ctypes.byref(s), *[P] * 8, need - 1, None) == B.FASTH_EWORKSPACE


@pytest.mark.parametrize("kw,code", [(dict(vocab=0), -1), (dict(m=0), -1), (dict(dtype=3), -1), (dict(id_bits=0), -1), (dict(top=-1), -1),
                                     (dict(top=33), -5), (dict(vocab=(1 << 21) + 1), -5), (dict(m=65536), -5)])
def test_log_prob_shapes(kw, code):
    lib, s = B.load_library(), _prob(**kw)
    top = P if s.top > 0 else None
    assert lib.fasth_log_prob(ctypes.byref(s), P, P, P, P, P, top, top, P, BIG, None) == code
    assert lib.fasth_log_prob_backward(ctypes.byref(s), P, P, P, P, P, P, P, None) == code
    assert lib.fasth_log_prob_workspace_bytes(ctypes.byref(s)) == 0


def test_log_prob_arguments():
    lib, s, t = B.load_library(), _prob(), _prob(top=3)
    for at in range(8):
        a = [P] * 8
        a[at] = ODD
        assert lib.fasth_log_prob(ctypes.byref(t), *a, BIG, None) == B.FASTH_EALIGN
        a[at] = None
        if at != 1:  # ids may be null
            assert lib.fasth_log_prob(ctypes.byref(t), *a, BIG, None) == B.FASTH_EINVAL
    assert lib.fasth_log_prob(ctypes.byref(s), *[P] * 8, BIG, None) == B.FASTH_EINVAL  # alternatives with top = 0
    for shape in (s, t):
        top = P if shape.top else None
        need = lib.fasth_log_prob_workspace_bytes(ctypes.byref(shape))
        assert lib.fasth_log_prob(ctypes.byref(shape), P, P, P, P, P, top, top, P, need - 1, None) == B.FASTH_EWORKSPACE
    for at in range(7):
        a = [P] * 7
        a[at] = ODD
        assert lib.fasth_log_prob_backward(ctypes.byref(s), *a, None) == B.FASTH_EALIGN
    for null in ((0,), (2,), (6,), (4, 5), (1,), (3,)):  # without ids no g_logp, without entropy no g_entropy
        a = [None if i in null else P for i in range(7)]
        assert lib.fasth_log_prob_backward(ctypes.byref(s), *a, None) == B.FASTH_EINVAL


def _list(*items):
    return (B.fasth_tensor * len(items))(*(B.fasth_tensor(*i) for i in items)), len(items)


def _out(*addresses):
    return (ctypes.c_void_p * len(addresses))(*addresses)


def test_gradient_lists():
    lib = B.load_library()
    ok, n = _list((4096, 64, 0), (8192, 64, 1), (None, 0, 2))
    assert lib.fasth_grad_workspace_bytes(ok, n) > 0 and lib.fasth_grad_workspace_bytes(None, 0) > 0
    bad = [(_list((4096, 64, 3)), -1), (_list((None, 1, 0)), -1), (_list((4104, 64, 0)), -3), (_list((4096, (1 << 36) + 1, 0)), -5)]
    for (items, n), code in bad:
        assert lib.fasth_grad_workspace_bytes(items, n) == 0
        assert lib.fasth_grad_norm(items, n, P, P, BIG, None) == code
        assert lib.fasth_grad_clip(items, None, n, 1.0, P, P, BIG, None) == code
    ok, n = _list((4096, 64, 0), (8192, 64, 1))
    assert lib.fasth_grad_norm(ok, -1, P, P, BIG, None) == B.FASTH_EINVAL
    assert lib.fasth_grad_norm(None, 2, P, P, BIG, None) == B.FASTH_EINVAL
    assert lib.fasth_grad_norm(ok, n, None, P, BIG, None) == B.FASTH_EINVAL
    assert lib.fasth_grad_norm(ok, n, P, ODD, BIG, None) == B.FASTH_EALIGN
    assert lib.fasth_grad_norm(ok, n, P, P, 64, None) == B.FASTH_EWORKSPACE
    assert lib.fasth_grad_clip(ok, None, n, -1.0, P, P, BIG, None) == B.FASTH_EINVAL
    assert lib.fasth_grad_clip(ok, None, n, float("nan"), P, P, BIG, None) == B.FASTH_EINVAL
    assert lib.fasth_grad_clip(ok, _out(4096, None), n, 1.0, P, P, BIG, None) == B.FASTH_EINVAL
    assert lib.fasth_grad_clip(ok, _out(4096, ODD), n, 1.0, P, P, BIG, None) == B.FASTH_EALIGN


def test_overlapping_gradients_are_refused():
    lib = B.load_library()
    clip = lambda items, out: lib.fasth_grad_clip(items[0], out, items[1], 1.0, P, P, BIG, None)
    twice = _list((4096, 64, 0), (4096, 64, 0))
    assert clip(twice, None) == B.FASTH_EINVAL                       # written twice
    assert clip(_list((4096, 64, 0), (4096 + 240, 64, 0)), None) == B.FASTH_EINVAL
    pair = _list((4096, 64, 0), (8192, 64, 0))
    assert clip(pair, _out(16384, 16384 + 128)) == B.FASTH_EINVAL    # outputs over each other
    assert clip(pair, _out(8192, 16384)) == B.FASTH_EINVAL           # an output over another's input
    assert clip(pair, _out(4096 + 16, 8192)) == B.FASTH_EINVAL       # an output shifted against its input


def test_binding_refuses_cpu_tensors():
    import torch
    t, ids = torch.zeros(4, 4), torch.zeros(4, dtype=torch.int64)
    with pytest.raises(ValueError):
        B.fasth_embed(t, ids, t)
    with pytest.raises(ValueError):
        B.fasth_norm(t, t[0], t, t[0])
    with pytest.raises(ValueError):
        B.fasth_log_prob(t, ids, t[0], t[0], t[:2], t)
    with pytest.raises(ValueError):
        B.tensor_list([t])
    with pytest.raises(TypeError):
        B.fasth_embed([[1.0]], ids, t)
    with pytest.raises(ValueError):
        B.fasth_embed(t[0], ids, t)
