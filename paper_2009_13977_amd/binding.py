"""ctypes binding of libfasth.so: the same entry points as include/fasth.h.

Argument marshalling only. torch supplies device memory and the current HIP
stream; every step of the computation runs in the library's kernels. There is
no fallback: if the shared library is missing or a call fails, an exception is
raised.
"""
from __future__ import annotations

import ctypes
import os
from typing import Optional

PKG_DIR = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(PKG_DIR, "libfasth.so")

FASTH_OK = 0
FASTH_EINVAL = -1
FASTH_EWORKSPACE = -2
FASTH_EALIGN = -3
FASTH_EHIP = -4
FASTH_EUNSUPPORTED = -5
FASTH_ETIMEOUT = -6

EXPORTED_SYMBOLS = (
    "fasth_strerror",
    "fasth_workspace_bytes",
    "fasth_forward",
    "fasth_forward_static",
    "fasth_prepare",
    "fasth_apply",
    "fasth_backward",
    "fasth_tune_block_size",
    "fasth_sequential_workspace_bytes",
    "fasth_sequential_forward",
    "fasth_sequential_backward",
    "svd_layer_workspace_bytes",
    "svd_layer_apply",
    "svd_layer_inverse_apply",
    "svd_layer_apply_backward",
    "svd_layer_inverse_apply_backward",
    "svd_sym_apply",
    "svd_sym_apply_backward",
    "svd_rect_workspace_bytes",
    "svd_rect_apply",
    "svd_rect_apply_backward",
    "svd_layer_log_abs_det",
    "fasth_embed",
    "fasth_embed_workspace_bytes",
    "fasth_embed_backward",
    "fasth_norm",
    "fasth_norm_workspace_bytes",
    "fasth_norm_backward",
    "fasth_log_prob_workspace_bytes",
    "fasth_log_prob",
    "fasth_log_prob_backward",
    "fasth_grad_workspace_bytes",
    "fasth_grad_norm",
    "fasth_grad_clip",
    "fasth_kernel_name",
    "fasth_profile_enable",
    "fasth_profile_collect",
    "fasth_profile_variant",
    "fasth_measure_peaks",
    "fasth_wait_status",
    "fasth_set_wait_limit",
)


class fasth_shape(ctypes.Structure):
    _fields_ = [("d", ctypes.c_int), ("n", ctypes.c_int), ("m", ctypes.c_int), ("k", ctypes.c_int),
                ("transpose", ctypes.c_int)]


class fasth_svd_shape(ctypes.Structure):
    _fields_ = [("d", ctypes.c_int), ("n", ctypes.c_int), ("m", ctypes.c_int), ("k", ctypes.c_int)]


class fasth_rect_shape(ctypes.Structure):
    _fields_ = [("rows", ctypes.c_int), ("cols", ctypes.c_int), ("n_u", ctypes.c_int), ("n_v", ctypes.c_int),
                ("m", ctypes.c_int), ("k", ctypes.c_int)]


class fasth_embed_shape(ctypes.Structure):
    _fields_ = [("vocab", ctypes.c_int), ("d", ctypes.c_int), ("m", ctypes.c_int), ("dtype", ctypes.c_int),
                ("id_bits", ctypes.c_int)]


class fasth_norm_shape(ctypes.Structure):
    _fields_ = [("d", ctypes.c_int), ("m", ctypes.c_int), ("dtype", ctypes.c_int), ("eps", ctypes.c_float)]


class fasth_log_prob_shape(ctypes.Structure):
    _fields_ = [("vocab", ctypes.c_int), ("m", ctypes.c_int), ("dtype", ctypes.c_int), ("id_bits", ctypes.c_int),
                ("top", ctypes.c_int)]


class fasth_tensor(ctypes.Structure):
    _fields_ = [("data", ctypes.c_void_p), ("count", ctypes.c_size_t), ("dtype", ctypes.c_int)]


class FasthError(RuntimeError):
    def __init__(self, code: int, where: str):
        self.code = code
        super().__init__(f"{where}: {strerror(code)} (code {code})")


_lib: Optional[ctypes.CDLL] = None


def load_library() -> ctypes.CDLL:
    """Load libfasth.so (built by `python -m paper_2009_13977_amd.build`)."""
    global _lib
    if _lib is not None:
        return _lib
    path = os.environ.get("FASTH_LIBRARY_PATH", LIB_PATH)  # another build of the same library, e.g. for an A/B timing
    if not os.path.exists(path):
        raise FileNotFoundError(
            f"{path} is missing: build it with `python -m paper_2009_13977_amd.build` "
            "(there is no CPU fallback)")
    lib = ctypes.CDLL(path)
    P, S, I = ctypes.c_void_p, ctypes.c_size_t, ctypes.c_int
    shp, sshp = ctypes.POINTER(fasth_shape), ctypes.POINTER(fasth_svd_shape)
    lib.fasth_strerror.restype = ctypes.c_char_p
    lib.fasth_strerror.argtypes = [I]
    lib.fasth_workspace_bytes.restype = S
    lib.fasth_workspace_bytes.argtypes = [shp]
    lib.fasth_forward.restype = I
    lib.fasth_forward.argtypes = [shp, P, P, P, P, S, P]
    lib.fasth_forward_static.restype = I
    lib.fasth_forward_static.argtypes = [shp, P, P, P, P]
    lib.fasth_backward.restype = I
    lib.fasth_backward.argtypes = [shp, P, P, P, P, P, S, P]
    lib.fasth_tune_block_size.restype = I
    lib.fasth_tune_block_size.argtypes = [shp, ctypes.POINTER(ctypes.c_int), I, I, P, P, P, P, P, P, P, S,
                                          ctypes.POINTER(ctypes.c_int), ctypes.POINTER(ctypes.c_float), P]
    lib.fasth_prepare.restype = I
    lib.fasth_prepare.argtypes = [shp, P, P, S, P]
    lib.fasth_apply.restype = I
    lib.fasth_apply.argtypes = [shp, P, P, P, P, S, I, P]
    lib.fasth_sequential_workspace_bytes.restype = S
    lib.fasth_sequential_workspace_bytes.argtypes = [shp]
    lib.fasth_sequential_forward.restype = I
    lib.fasth_sequential_forward.argtypes = [shp, P, P, P, P]
    lib.fasth_sequential_backward.restype = I
    lib.fasth_sequential_backward.argtypes = [shp, P, P, P, P, P, P, S, P]
    lib.svd_layer_workspace_bytes.restype = S
    lib.svd_layer_workspace_bytes.argtypes = [sshp]
    for name in ("svd_layer_apply", "svd_layer_inverse_apply"):
        fn = getattr(lib, name)
        fn.restype = I
        fn.argtypes = [sshp, P, P, P, P, P, P, S, P]
    for name in ("svd_layer_apply_backward", "svd_layer_inverse_apply_backward"):
        fn = getattr(lib, name)
        fn.restype = I
        fn.argtypes = [sshp, P, P, P, P, P, P, P, P, P, S, P]
    lib.svd_sym_apply.restype = I
    lib.svd_sym_apply.argtypes = [sshp, I, P, P, P, P, P, S, P]
    lib.svd_sym_apply_backward.restype = I
    lib.svd_sym_apply_backward.argtypes = [sshp, I, P, P, P, P, P, P, P, S, P]
    rshp = ctypes.POINTER(fasth_rect_shape)
    lib.svd_rect_workspace_bytes.restype = S
    lib.svd_rect_workspace_bytes.argtypes = [rshp]
    lib.svd_rect_apply.restype = I
    lib.svd_rect_apply.argtypes = [rshp, P, P, P, P, P, P, S, P]
    lib.svd_rect_apply_backward.restype = I
    lib.svd_rect_apply_backward.argtypes = [rshp, P, P, P, P, P, P, P, P, P, S, P]
    lib.svd_layer_log_abs_det.restype = I
    lib.svd_layer_log_abs_det.argtypes = [I, P, P, P, P]
    F = ctypes.c_float
    eshp, nshp, lshp, tens = (ctypes.POINTER(c) for c in (fasth_embed_shape, fasth_norm_shape, fasth_log_prob_shape, fasth_tensor))
    for name, restype, argtypes in (
            ("fasth_embed", I, [eshp, P, P, F, P, P]),
            ("fasth_embed_workspace_bytes", S, [eshp]),
            ("fasth_embed_backward", I, [eshp, P, P, F, P, P, S, P]),
            ("fasth_norm", I, [nshp, P, P, P, P, P, P, P]),
            ("fasth_norm_workspace_bytes", S, [nshp]),
            ("fasth_norm_backward", I, [nshp, P, P, P, P, P, P, P, P, S, P]),
            ("fasth_log_prob_workspace_bytes", S, [lshp]),
            ("fasth_log_prob", I, [lshp, P, P, P, P, P, P, P, P, S, P]),
            ("fasth_log_prob_backward", I, [lshp, P, P, P, P, P, P, P, P]),
            ("fasth_grad_workspace_bytes", S, [tens, I]),
            ("fasth_grad_norm", I, [tens, I, P, P, S, P]),
            ("fasth_grad_clip", I, [tens, ctypes.POINTER(P), I, F, P, P, S, P])):
        fn = getattr(lib, name)
        fn.restype = restype
        fn.argtypes = argtypes
    lib.fasth_kernel_name.restype = ctypes.c_char_p
    lib.fasth_kernel_name.argtypes = [I]
    lib.fasth_profile_enable.restype = I
    lib.fasth_profile_enable.argtypes = [I]
    lib.fasth_profile_collect.restype = I
    lib.fasth_profile_collect.argtypes = [ctypes.POINTER(ctypes.c_float), ctypes.POINTER(ctypes.c_int)]
    lib.fasth_profile_variant.restype = ctypes.c_char_p
    lib.fasth_profile_variant.argtypes = [I]
    lib.fasth_wait_status.restype = I
    lib.fasth_wait_status.argtypes = [P]
    lib.fasth_set_wait_limit.restype = I
    lib.fasth_set_wait_limit.argtypes = [I]
    lib.fasth_measure_peaks.restype = I
    lib.fasth_measure_peaks.argtypes = [P, S, I, ctypes.POINTER(ctypes.c_float), ctypes.POINTER(ctypes.c_float),
                                        ctypes.POINTER(ctypes.c_float), P]
    _lib = lib
    return lib


def strerror(code: int) -> str:
    return load_library().fasth_strerror(int(code)).decode()


def _check(code: int, where: str) -> None:
    if code != FASTH_OK:
        raise FasthError(code, where)


def _ptr(t, name: str) -> int:
    import torch
    if not isinstance(t, torch.Tensor):
        raise TypeError(f"{name}: expected a torch.Tensor")
    if not t.is_cuda:
        raise ValueError(f"{name}: must live in GPU memory")
    if t.dtype != torch.float32 and name != "workspace":
        raise ValueError(f"{name}: must be float32")
    if not t.is_contiguous():
        raise ValueError(f"{name}: must be contiguous")
    return t.data_ptr()


def _stream() -> int:
    import torch
    return torch.cuda.current_stream().cuda_stream


class _Torch:
    """What the checks of the operators around the layers need of torch, looked up once: they are called with few
    microseconds of work on the GPU, beside which an import statement and a stream object per call are long."""

    def __init__(self):
        import torch
        self.tensor = torch.Tensor
        self.kinds = {torch.float32: 0, torch.bfloat16: 1, torch.float16: 2}
        self.f32, self.int32, self.ids, self.bytes = (torch.float32,), (torch.int32,), (torch.int32, torch.int64), (torch.uint8,)
        raw = getattr(torch._C, "_cuda_getCurrentRawStream", None)  # the number behind current_stream(), without the object
        self.stream = raw or (lambda device: torch.cuda.current_stream(device).cuda_stream)
        self.device = torch.cuda.current_device


_torch: Optional[_Torch] = None


def _here():
    """(the above, the current device's number or -2 without one)"""
    global _torch
    if _torch is None:
        _torch = _Torch()
    try:
        return _torch, _torch.device()
    except (RuntimeError, AssertionError):  # no GPU: no tensor can be on the current one
        return _torch, -2


def _shape(d, n, m, k, transpose=False) -> fasth_shape:
    return fasth_shape(int(d), int(n), int(m), int(k), 1 if transpose else 0)


def fasth_workspace_bytes(d: int, n: int, m: int, k: int) -> int:
    return int(load_library().fasth_workspace_bytes(ctypes.byref(_shape(d, n, m, k))))


def fasth_sequential_workspace_bytes(d: int, n: int, m: int) -> int:
    return int(load_library().fasth_sequential_workspace_bytes(ctypes.byref(_shape(d, n, m, 1))))


def svd_layer_workspace_bytes(d: int, n: int, m: int, k: int) -> int:
    return int(load_library().svd_layer_workspace_bytes(ctypes.byref(fasth_svd_shape(int(d), int(n), int(m), int(k)))))


def new_workspace(nbytes: int, device="cuda"):
    import torch
    return torch.empty(max(int(nbytes), 16), dtype=torch.uint8, device=device)


def fasth_forward(V, X, A, workspace, k: int, transpose: bool = False) -> None:
    n, d = V.shape
    m = X.shape[1]
    assert X.shape == (d, m) and A.shape == (d, m)
    shape = _shape(d, n, m, k, transpose)
    rc = load_library().fasth_forward(ctypes.byref(shape), _ptr(V, "V"), _ptr(X, "X"), _ptr(A, "A"),
                                      _ptr(workspace, "workspace"), workspace.numel(), _stream())
    _check(rc, "fasth_forward")


def fasth_forward_static(V, X, A, k: int, transpose: bool = False) -> None:
    n, d = V.shape
    m = X.shape[1]
    assert X.shape == (d, m) and A.shape == (d, m)
    shape = _shape(d, n, m, k, transpose)
    rc = load_library().fasth_forward_static(ctypes.byref(shape), _ptr(V, "V"), _ptr(X, "X"), _ptr(A, "A"), _stream())
    _check(rc, "fasth_forward_static")


def fasth_prepare(V, m: int, workspace, k: int) -> None:
    n, d = V.shape
    shape = _shape(d, n, m, k, False)
    rc = load_library().fasth_prepare(ctypes.byref(shape), _ptr(V, "V"), _ptr(workspace, "workspace"),
                                      workspace.numel(), _stream())
    _check(rc, "fasth_prepare")


def fasth_apply(V, X, A, workspace, k: int, transpose: bool = False, save_for_backward: bool = False) -> None:
    n, d = V.shape
    m = X.shape[1]
    assert X.shape == (d, m) and A.shape == (d, m)
    shape = _shape(d, n, m, k, transpose)
    rc = load_library().fasth_apply(ctypes.byref(shape), _ptr(V, "V"), _ptr(X, "X"), _ptr(A, "A"),
                                    _ptr(workspace, "workspace"), workspace.numel(),
                                    1 if save_for_backward else 0, _stream())
    _check(rc, "fasth_apply")


def fasth_backward(V, G, dV, dX, workspace, k: int, transpose: bool = False) -> None:
    n, d = V.shape
    m = G.shape[1]
    assert G.shape == (d, m) and dX.shape == (d, m) and dV.shape == (n, d)
    shape = _shape(d, n, m, k, transpose)
    rc = load_library().fasth_backward(ctypes.byref(shape), _ptr(V, "V"), _ptr(G, "G"), _ptr(dV, "dV"),
                                       _ptr(dX, "dX"), _ptr(workspace, "workspace"), workspace.numel(), _stream())
    _check(rc, "fasth_backward")


def fasth_tune_block_size(V, X, G, A, dV, dX, workspace, candidates=None, repetitions: int = 5,
                          transpose: bool = False):
    """Returns (best k, milliseconds per forward+backward pass at that k)."""
    n, d = V.shape
    m = X.shape[1]
    shape = _shape(d, n, m, 1, transpose)
    if candidates is None:
        cand, ncand = None, 0
    else:
        cand = (ctypes.c_int * len(candidates))(*[int(c) for c in candidates])
        ncand = len(candidates)
    best_k = ctypes.c_int(0)
    best_ms = ctypes.c_float(0.0)
    rc = load_library().fasth_tune_block_size(ctypes.byref(shape), cand, ncand, int(repetitions), _ptr(V, "V"),
                                              _ptr(X, "X"), _ptr(G, "G"), _ptr(A, "A"), _ptr(dV, "dV"),
                                              _ptr(dX, "dX"), _ptr(workspace, "workspace"), workspace.numel(),
                                              ctypes.byref(best_k), ctypes.byref(best_ms), _stream())
    _check(rc, "fasth_tune_block_size")
    return best_k.value, best_ms.value


def fasth_sequential_forward(V, X, A, transpose: bool = False) -> None:
    n, d = V.shape
    m = X.shape[1]
    shape = _shape(d, n, m, 1, transpose)
    rc = load_library().fasth_sequential_forward(ctypes.byref(shape), _ptr(V, "V"), _ptr(X, "X"), _ptr(A, "A"),
                                                 _stream())
    _check(rc, "fasth_sequential_forward")


def fasth_sequential_backward(V, A, G, dV, dX, workspace, transpose: bool = False) -> None:
    """A is the product fasth_sequential_forward wrote for the same V and X."""
    n, d = V.shape
    m = A.shape[1]
    shape = _shape(d, n, m, 1, transpose)
    rc = load_library().fasth_sequential_backward(ctypes.byref(shape), _ptr(V, "V"), _ptr(A, "A"), _ptr(G, "G"),
                                                  _ptr(dV, "dV"), _ptr(dX, "dX"), _ptr(workspace, "workspace"),
                                                  workspace.numel(), _stream())
    _check(rc, "fasth_sequential_backward")


def _svd_forward(name, Uv, sigma, Vv, X, Y, workspace, k):
    n, d = Uv.shape
    m = X.shape[1]
    assert Vv.shape == (n, d) and sigma.shape == (d,) and X.shape == (d, m) and Y.shape == (d, m)
    shape = fasth_svd_shape(d, n, m, int(k))
    rc = getattr(load_library(), name)(ctypes.byref(shape), _ptr(Uv, "Uv"), _ptr(sigma, "sigma"), _ptr(Vv, "Vv"),
                                       _ptr(X, "X"), _ptr(Y, "Y"), _ptr(workspace, "workspace"), workspace.numel(),
                                       _stream())
    _check(rc, name)


def _svd_backward(name, Uv, sigma, Vv, G, dUv, dsigma, dVv, dX, workspace, k):
    n, d = Uv.shape
    m = G.shape[1]
    shape = fasth_svd_shape(d, n, m, int(k))
    rc = getattr(load_library(), name)(ctypes.byref(shape), _ptr(Uv, "Uv"), _ptr(sigma, "sigma"), _ptr(Vv, "Vv"),
                                       _ptr(G, "G"), _ptr(dUv, "dUv"), _ptr(dsigma, "dsigma"), _ptr(dVv, "dVv"),
                                       _ptr(dX, "dX"), _ptr(workspace, "workspace"), workspace.numel(), _stream())
    _check(rc, name)


def svd_layer_apply(Uv, sigma, Vv, X, Y, workspace, k: int) -> None:
    _svd_forward("svd_layer_apply", Uv, sigma, Vv, X, Y, workspace, k)


def svd_layer_inverse_apply(Uv, sigma, Vv, X, Y, workspace, k: int) -> None:
    _svd_forward("svd_layer_inverse_apply", Uv, sigma, Vv, X, Y, workspace, k)


def svd_layer_apply_backward(Uv, sigma, Vv, G, dUv, dsigma, dVv, dX, workspace, k: int) -> None:
    _svd_backward("svd_layer_apply_backward", Uv, sigma, Vv, G, dUv, dsigma, dVv, dX, workspace, k)


def svd_layer_inverse_apply_backward(Uv, sigma, Vv, G, dUv, dsigma, dVv, dX, workspace, k: int) -> None:
    _svd_backward("svd_layer_inverse_apply_backward", Uv, sigma, Vv, G, dUv, dsigma, dVv, dX, workspace, k)


DIAG_FUNCTIONS = {"identity": 0, "exp": 1, "cayley": 2}


def svd_sym_apply(Uv, sigma, X, Y, workspace, k: int, function: str = "identity") -> None:
    n, d = Uv.shape
    m = X.shape[1]
    assert sigma.shape == (d,) and X.shape == (d, m) and Y.shape == (d, m)
    shape = fasth_svd_shape(d, n, m, int(k))
    rc = load_library().svd_sym_apply(ctypes.byref(shape), DIAG_FUNCTIONS[function], _ptr(Uv, "Uv"),
                                      _ptr(sigma, "sigma"), _ptr(X, "X"), _ptr(Y, "Y"),
                                      _ptr(workspace, "workspace"), workspace.numel(), _stream())
    _check(rc, "svd_sym_apply")


def svd_sym_apply_backward(Uv, sigma, G, dUv, dsigma, dX, workspace, k: int, function: str = "identity") -> None:
    n, d = Uv.shape
    m = G.shape[1]
    shape = fasth_svd_shape(d, n, m, int(k))
    rc = load_library().svd_sym_apply_backward(ctypes.byref(shape), DIAG_FUNCTIONS[function], _ptr(Uv, "Uv"),
                                               _ptr(sigma, "sigma"), _ptr(G, "G"), _ptr(dUv, "dUv"),
                                               _ptr(dsigma, "dsigma"), _ptr(dX, "dX"),
                                               _ptr(workspace, "workspace"), workspace.numel(), _stream())
    _check(rc, "svd_sym_apply_backward")


def _rect_shape(Uv, Vv, m, k) -> fasth_rect_shape:
    return fasth_rect_shape(int(Uv.shape[1]), int(Vv.shape[1]), int(Uv.shape[0]), int(Vv.shape[0]), int(m), int(k))


def svd_rect_workspace_bytes(rows: int, cols: int, n_u: int, n_v: int, m: int, k: int) -> int:
    shape = fasth_rect_shape(int(rows), int(cols), int(n_u), int(n_v), int(m), int(k))
    return int(load_library().svd_rect_workspace_bytes(ctypes.byref(shape)))


def svd_rect_apply(Uv, sigma, Vv, X, Y, workspace, k: int) -> None:
    m = X.shape[1]
    shape = _rect_shape(Uv, Vv, m, k)
    assert sigma.shape == (min(shape.rows, shape.cols),) and X.shape == (shape.cols, m) and Y.shape == (shape.rows, m)
    rc = load_library().svd_rect_apply(ctypes.byref(shape), _ptr(Uv, "Uv"), _ptr(sigma, "sigma"), _ptr(Vv, "Vv"),
                                       _ptr(X, "X"), _ptr(Y, "Y"), _ptr(workspace, "workspace"), workspace.numel(),
                                       _stream())
    _check(rc, "svd_rect_apply")


def svd_rect_apply_backward(Uv, sigma, Vv, G, dUv, dsigma, dVv, dX, workspace, k: int) -> None:
    m = G.shape[1]
    shape = _rect_shape(Uv, Vv, m, k)
    assert G.shape == (shape.rows, m) and dX.shape == (shape.cols, m) and dsigma.shape == sigma.shape
    assert dUv.shape == Uv.shape and dVv.shape == Vv.shape
    rc = load_library().svd_rect_apply_backward(ctypes.byref(shape), _ptr(Uv, "Uv"), _ptr(sigma, "sigma"),
                                                _ptr(Vv, "Vv"), _ptr(G, "G"), _ptr(dUv, "dUv"),
                                                _ptr(dsigma, "dsigma"), _ptr(dVv, "dVv"), _ptr(dX, "dX"),
                                                _ptr(workspace, "workspace"), workspace.numel(), _stream())
    _check(rc, "svd_rect_apply_backward")


def svd_layer_log_abs_det(sigma, out, dsigma=None) -> None:
    rc = load_library().svd_layer_log_abs_det(int(sigma.shape[0]), _ptr(sigma, "sigma"), _ptr(out, "out"),
                                              _ptr(dsigma, "dsigma") if dsigma is not None else None, _stream())
    _check(rc, "svd_layer_log_abs_det")


def _typed(t, name: str, dtypes, device: int, shape=None) -> int:
    """The address of a dense tensor on GPU `device` of one of `dtypes` (and of `shape`); 0 for None."""
    if t is None:
        return 0
    if not isinstance(t, _torch.tensor):
        raise TypeError(f"{name}: expected a torch.Tensor")
    if t.get_device() != device or t.dtype not in dtypes or not t.is_contiguous() or (shape is not None and t.shape != shape):
        if not t.is_cuda:
            raise ValueError(f"{name}: must live in GPU memory")
        if t.get_device() != device:
            raise ValueError(f"{name}: must live on the current device")
        if t.dtype not in dtypes:
            raise ValueError(f"{name}: must be one of {', '.join(str(d) for d in dtypes)}, not {t.dtype}")
        if not t.is_contiguous():
            raise ValueError(f"{name}: must be contiguous")
        raise ValueError(f"{name}: must be of shape {tuple(shape)}, not {tuple(t.shape)}")
    return t.data_ptr()


def _matrix(t, name: str):
    if not isinstance(t, _torch.tensor):
        raise TypeError(f"{name}: expected a torch.Tensor")
    if t.dim() != 2:
        raise ValueError(f"{name}: must have two dimensions")
    rows, cols = shape = t.shape
    if rows > _MOST or cols > _MOST:  # the library would see what is left of it in 32 bits
        raise FasthError(FASTH_EUNSUPPORTED, f"{name} of {rows} x {cols}")
    return shape


_MOST = 2 ** 31 - 1


def _size(n: int) -> int:
    """A size as the library takes it; what 32 bits cannot hold becomes one that it refuses."""
    n = int(n)
    return min(n, _MOST) if n >= 0 else -1


def _space(t, device: int):
    """A workspace's address and bytes."""
    if t is None:
        raise TypeError("workspace: expected a torch.Tensor")
    return _typed(t, "workspace", _torch.bytes, device), t.numel()


def _id_bits(ids) -> int:
    return 32 if ids is None or ids.dtype == _torch.int32[0] else 64


def fasth_embed_workspace_bytes(vocab: int, d: int, m: int) -> int:
    shape = fasth_embed_shape(_size(vocab), _size(d), _size(m), 0, 64)
    return int(load_library().fasth_embed_workspace_bytes(ctypes.byref(shape)))


def fasth_embed(table, ids, X, scale: float = 1.0) -> None:
    """X[:, j] = scale * table[ids[j]]; zero where ids[j] is no row of the table."""
    k, dev = _here()
    (vocab, d), (_, m) = _matrix(table, "table"), _matrix(X, "X")
    where = (_typed(table, "table", k.kinds, dev), _typed(ids, "ids", k.ids, dev, (m,)), float(scale), _typed(X, "X", k.f32, dev, (d, m)))
    shape = fasth_embed_shape(vocab, d, m, k.kinds[table.dtype], _id_bits(ids))
    _check(load_library().fasth_embed(ctypes.byref(shape), *where, k.stream(dev)), "fasth_embed")


def fasth_embed_backward(ids, G, dTable, workspace, scale: float = 1.0) -> None:
    """dTable[t] = scale * sum of G[:, j] over ids[j] = t, for every row t."""
    k, dev = _here()
    (vocab, d), (_, m) = _matrix(dTable, "dTable"), _matrix(G, "G")
    where = (_typed(ids, "ids", k.ids, dev, (m,)), _typed(G, "G", k.f32, dev, (d, m)), float(scale), _typed(dTable, "dTable", k.kinds, dev),
             *_space(workspace, dev))
    shape = fasth_embed_shape(vocab, d, m, k.kinds[dTable.dtype], _id_bits(ids))
    _check(load_library().fasth_embed_backward(ctypes.byref(shape), *where, k.stream(dev)), "fasth_embed_backward")


def fasth_norm_workspace_bytes(d: int, m: int) -> int:
    return int(load_library().fasth_norm_workspace_bytes(ctypes.byref(fasth_norm_shape(_size(d), _size(m), 0, 1.0))))


def fasth_norm(X, weight, Y, rstd, eps: float = 1e-6, R=None, S=None) -> None:
    """S = X + R (without R: S = X, not written), rstd = (mean over rows of S^2 + eps)^(-1/2), Y = weight * S * rstd."""
    k, dev = _here()
    d, m = dm = _matrix(X, "X")
    where = (_typed(X, "X", k.f32, dev), _typed(R, "R", k.f32, dev, dm), _typed(weight, "weight", k.f32, dev, (d,)),
             _typed(S, "S", k.f32, dev, dm), _typed(Y, "Y", k.kinds, dev, dm), _typed(rstd, "rstd", k.f32, dev, (m,)))
    shape = fasth_norm_shape(d, m, k.kinds[Y.dtype] if Y is not None else 0, float(eps))
    _check(load_library().fasth_norm(ctypes.byref(shape), *where, k.stream(dev)), "fasth_norm")


def fasth_norm_backward(G, S, weight, rstd, dX, dweight, workspace, dS=None) -> None:
    """dX = dS + the gradient through the norm, and dweight (None: not wanted)."""
    k, dev = _here()
    d, m = dm = _matrix(G, "G")
    where = (_typed(G, "G", k.kinds, dev), _typed(S, "S", k.f32, dev, dm), _typed(weight, "weight", k.f32, dev, (d,)),
             _typed(rstd, "rstd", k.f32, dev, (m,)), _typed(dS, "dS", k.f32, dev, dm), _typed(dX, "dX", k.f32, dev, dm),
             _typed(dweight, "dweight", k.f32, dev, (d,)), *_space(workspace, dev))
    shape = fasth_norm_shape(d, m, k.kinds[G.dtype], 1.0)  # (the backward call has the forward call's eps in rstd)
    _check(load_library().fasth_norm_backward(ctypes.byref(shape), *where, k.stream(dev)), "fasth_norm_backward")


def fasth_log_prob_workspace_bytes(vocab: int, m: int, top: int = 0) -> int:
    shape = fasth_log_prob_shape(_size(vocab), _size(m), 0, 64, _size(top))
    return int(load_library().fasth_log_prob_workspace_bytes(ctypes.byref(shape)))


def fasth_log_prob(logits, ids, logp, entropy, stats, workspace, top_logp=None, top_ids=None) -> None:
    """Per column of logits [vocab][m]: log probability of ids[j], entropy, and the top_logp.shape[0] best with their rows."""
    k, dev = _here()
    vocab, m = _matrix(logits, "logits")
    top = 0 if top_logp is None else _matrix(top_logp, "top_logp")[0]
    where = (_typed(logits, "logits", k.kinds, dev), _typed(ids, "ids", k.ids, dev, (m,)), _typed(logp, "logp", k.f32, dev, (m,)),
             _typed(entropy, "entropy", k.f32, dev, (m,)), _typed(stats, "stats", k.f32, dev, (2, m)),
             _typed(top_logp, "top_logp", k.f32, dev, (top, m)), _typed(top_ids, "top_ids", k.int32, dev, (top, m)),
             *_space(workspace, dev))
    shape = fasth_log_prob_shape(vocab, m, k.kinds[logits.dtype], _id_bits(ids), top)
    _check(load_library().fasth_log_prob(ctypes.byref(shape), *where, k.stream(dev)), "fasth_log_prob")


def fasth_log_prob_backward(logits, ids, stats, entropy, g_logp, g_entropy, dlogits) -> None:
    """dlogits for the gradients g_logp of logp and g_entropy of entropy (one of them may be None)."""
    k, dev = _here()
    vocab, m = _matrix(logits, "logits")
    where = (_typed(logits, "logits", k.kinds, dev), _typed(ids, "ids", k.ids, dev, (m,)), _typed(stats, "stats", k.f32, dev, (2, m)),
             _typed(entropy, "entropy", k.f32, dev, (m,)), _typed(g_logp, "g_logp", k.f32, dev, (m,)),
             _typed(g_entropy, "g_entropy", k.f32, dev, (m,)), _typed(dlogits, "dlogits", (logits.dtype,), dev, (vocab, m)))
    shape = fasth_log_prob_shape(vocab, m, k.kinds[logits.dtype], _id_bits(ids), 0)
    _check(load_library().fasth_log_prob_backward(ctypes.byref(shape), *where, k.stream(dev)), "fasth_log_prob_backward")


class TensorList:
    """A list of GPU tensors as the library reads it: their memory, sizes and types as they are then. A program whose gradient
    buffers stay where they are describes them once, which takes about a microsecond per tensor. The list keeps that memory,
    so that nothing else can come to lie there, and a call refuses the list once a tensor has other memory."""

    def __init__(self, tensors):
        k, dev = _here()
        self.tensors = tuple(tensors)
        self.items = (fasth_tensor * len(self.tensors))()
        self.data = (ctypes.c_void_p * len(self.tensors))()
        self.device = dev
        for i, t in enumerate(self.tensors):
            if t is None:
                raise TypeError(f"tensors[{i}]: expected a torch.Tensor")
            address = _typed(t, f"tensors[{i}]", k.kinds, dev)
            self.items[i] = fasth_tensor(address, t.numel(), k.kinds[t.dtype])
            self.data[i] = address
        self.memory = [t.untyped_storage() for t in self.tensors]
        self.where = [t.data_ptr for t in self.tensors]
        self.at = [where() for where in self.where]
        self.like = tuple((t.numel(), t.dtype) for t in self.tensors)

    def __len__(self):
        return len(self.tensors)


def tensor_list(tensors) -> TensorList:
    return tensors if isinstance(tensors, TensorList) else TensorList(tensors)


def _listed(tensors, name: str, device: int) -> TensorList:
    tensors = tensor_list(tensors)
    if tensors.device != device:
        raise ValueError(f"{name}: must live on the current device")
    if [where() for where in tensors.where] != tensors.at:
        raise ValueError(f"{name}: a tensor's memory is not where it was when the list was made")
    return tensors


def fasth_grad_workspace_bytes(tensors) -> int:
    tensors = tensor_list(tensors)
    return int(load_library().fasth_grad_workspace_bytes(tensors.items, len(tensors)))


def fasth_grad_norm(tensors, norm, workspace) -> None:
    """norm[0] = the square root of the sum of all squares of all tensors."""
    k, dev = _here()
    tensors = _listed(tensors, "tensors", dev)
    rc = load_library().fasth_grad_norm(tensors.items, len(tensors), _typed(norm, "norm", k.f32, dev, (1,)),
                                        *_space(workspace, dev), k.stream(dev))
    _check(rc, "fasth_grad_norm")


def fasth_grad_clip(tensors, max_norm: float, norm, workspace, out=None) -> None:
    """The tensors times max_norm / norm where their norm is larger, into `out` (tensors like them) or in place."""
    k, dev = _here()
    tensors = _listed(tensors, "tensors", dev)
    if out is not None:
        out = _listed(out, "out", dev)
        if out.like != tensors.like:
            raise ValueError("out: must hold tensors of the same sizes and types")
    rc = load_library().fasth_grad_clip(tensors.items, out.data if out is not None else None, len(tensors), float(max_norm),
                                        _typed(norm, "norm", k.f32, dev, (1,)), *_space(workspace, dev), k.stream(dev))
    _check(rc, "fasth_grad_clip")


FASTH_KERNEL_COUNT = 9


def fasth_profile_enable(on: bool) -> None:
    _check(load_library().fasth_profile_enable(1 if on else 0), "fasth_profile_enable")


def fasth_profile_collect() -> dict:
    """{kernel name: (total milliseconds, launches)} since profiling was enabled or last collected."""
    lib = load_library()
    ms = (ctypes.c_float * FASTH_KERNEL_COUNT)()
    cnt = (ctypes.c_int * FASTH_KERNEL_COUNT)()
    _check(lib.fasth_profile_collect(ms, cnt), "fasth_profile_collect")
    return {lib.fasth_kernel_name(i).decode(): (float(ms[i]), int(cnt[i])) for i in range(FASTH_KERNEL_COUNT)}


def fasth_profile_variants() -> dict:
    """{kernel name: instantiation last launched in that slot since profiling was switched on}."""
    lib = load_library()
    return {lib.fasth_kernel_name(i).decode(): lib.fasth_profile_variant(i).decode() for i in range(FASTH_KERNEL_COUNT)}


def fasth_measure_peaks(buffer, repetitions: int = 3) -> dict:
    """Measured fp32 matrix-instruction rate (TFLOP/s) and streaming read / copy rates (GB/s) of this GPU."""
    mf, rd, cp = ctypes.c_float(0.0), ctypes.c_float(0.0), ctypes.c_float(0.0)
    rc = load_library().fasth_measure_peaks(_ptr(buffer, "workspace"), buffer.numel() * buffer.element_size(),
                                            int(repetitions), ctypes.byref(mf), ctypes.byref(rd), ctypes.byref(cp),
                                            _stream())
    _check(rc, "fasth_measure_peaks")
    return {"fp32_mfma_tflops": mf.value, "hbm_read_gbs": rd.value, "hbm_copy_gbs": cp.value}


def fasth_wait_status() -> int:
    """Waits for the current stream; FASTH_OK, or FASTH_ETIMEOUT if a kernel's wait for another workgroup gave up
    on this GPU since the last check."""
    return int(load_library().fasth_wait_status(_stream()))


def fasth_set_wait_limit(polls: int) -> None:
    _check(load_library().fasth_set_wait_limit(int(polls)), "fasth_set_wait_limit")
