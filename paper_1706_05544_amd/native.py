"""Python binding of libmi355svm.so: argument marshalling only.

Every entry point of ``include/mi355svm.h`` has a function of the same name
here.  Host inputs are NumPy arrays; device inputs are torch tensors on a
ROCm device (PyTorch is used for device memory and streams only).  All
computation happens in the library's HIP kernels; if the library is not
built, loading fails loudly instead of falling back to anything else.
"""
from __future__ import annotations

import ctypes as ct
import os
from typing import Optional

import numpy as np

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libmi355svm.so")

SVM_OK = 0
SVM_W_MAX_ITER = 1
SVM_W_NOT_CONVERGED = 2
SVM_E_INVALID = -1
SVM_E_UNSUPPORTED = -2
SVM_E_NOMEM = -3
SVM_E_DEVICE = -4
SVM_E_INTERNAL = -5

SVM_C_SVC = 0
SVM_EPS_SVR = 1
SVM_KERNEL_LINEAR, SVM_KERNEL_POLY, SVM_KERNEL_RBF, SVM_KERNEL_SIGMOID = range(4)
SVM_DENSE = 0
SVM_CSR = 1
SVM_F32, SVM_BF16, SVM_F16 = range(3)
(SVM_ACT_NONE, SVM_ACT_RELU, SVM_ACT_GELU, SVM_ACT_SILU, SVM_ACT_TANH,
 SVM_ACT_COS) = range(6)
SVM_ADAMW_BLOCK = 256  # values that share a scale (states in 8 bits)

# every symbol the header declares
EXPORTS = [
    "svm_params_default", "svm_train", "svm_train_ovr", "svm_predict",
    "svm_predict_labels", "svm_model_get_info", "svm_model_get",
    "svm_model_free", "svm_last_error", "svm_cross_validate", "svm_tune",
    "svm_test_solver_create",
    "svm_test_solver_free", "svm_test_set_state", "svm_test_get_state",
    "svm_test_select", "svm_test_rows", "svm_test_subproblem",
    "svm_test_apply", "svm_test_iterate", "svm_test_finish",
    "svm_predict_noalloc", "svm_cache_release",
    "svm_linear", "svm_linear_workspace", "svm_linear_backward",
    "svm_linear_backward_workspace", "svm_layer_norm",
    "svm_layer_norm_backward", "svm_layer_norm_backward_workspace",
    "svm_hinge_loss", "svm_hinge_loss_workspace", "svm_adamw_step",
    "svm_adamw_state",
]


class SvmError(RuntimeError):
    def __init__(self, status: int, msg: str):
        super().__init__("status %d: %s" % (status, msg))
        self.status = status


class svm_matrix(ct.Structure):
    _fields_ = [("layout", ct.c_int32), ("on_device", ct.c_int32),
                ("n", ct.c_int64), ("d", ct.c_int64),
                ("values", ct.c_void_p), ("ld", ct.c_int64),
                ("row_ptr", ct.c_void_p), ("col_idx", ct.c_void_p),
                ("nnz", ct.c_int64)]


class svm_params(ct.Structure):
    _fields_ = [("type", ct.c_int32), ("kernel", ct.c_int32),
                ("C", ct.c_double), ("epsilon", ct.c_double),
                ("gamma", ct.c_double), ("tol", ct.c_double),
                ("max_iter", ct.c_int64), ("working_set", ct.c_int32),
                ("device", ct.c_int32), ("cache_bytes", ct.c_int64),
                ("stream", ct.c_void_p), ("check_every", ct.c_int32),
                ("inner_ratio", ct.c_double), ("max_inner", ct.c_int32),
                ("profile", ct.c_int32), ("coef0", ct.c_double),
                ("degree", ct.c_int32), ("scale", ct.c_int32),
                ("alpha0", ct.c_void_p), ("lockstep", ct.c_int32),
                ("fused", ct.c_int32)]


class svm_cv_stats(ct.Structure):
    _fields_ = [("folds", ct.c_int32), ("status", ct.c_int32),
                ("n", ct.c_int64), ("iters", ct.c_int64),
                ("accuracy", ct.c_double), ("mse", ct.c_double),
                ("scc", ct.c_double), ("error", ct.c_double),
                ("kernel_rows", ct.c_int64), ("row_kernel_ms", ct.c_double),
                ("row_kernel_launches", ct.c_int64),
                ("row_kernel_bytes", ct.c_double)]

    def as_dict(self) -> dict:
        return {k: getattr(self, k) for k, _ in self._fields_}


class svm_model_info(ct.Structure):
    _fields_ = [("type", ct.c_int32), ("n_outputs", ct.c_int32),
                ("n_train", ct.c_int64), ("n_features", ct.c_int64),
                ("n_sv", ct.c_int64), ("gamma", ct.c_double),
                ("kernel", ct.c_int32), ("degree", ct.c_int32),
                ("coef0", ct.c_double),
                ("status", ct.c_int32), ("n_sv_output", ct.c_int64),
                ("n_bounded", ct.c_int64), ("iters", ct.c_int64),
                ("gap", ct.c_double), ("b", ct.c_double),
                ("dual_obj", ct.c_double), ("kernel_rows", ct.c_int64),
                ("cache_hits", ct.c_int64), ("cache_fills", ct.c_int64),
                ("train_ms", ct.c_double),
                ("row_kernel_ms", ct.c_double),
                ("row_kernel_launches", ct.c_int64),
                ("row_kernel_rows", ct.c_int64),
                ("row_kernel_bytes", ct.c_double),
                ("cached_kernel_ms", ct.c_double),
                ("cached_kernel_launches", ct.c_int64),
                ("cached_kernel_bytes", ct.c_double),
                ("select_kernel_ms", ct.c_double),
                ("select_kernel_launches", ct.c_int64)]

    def as_dict(self) -> dict:
        return {k: getattr(self, k) for k, _ in self._fields_}


class svm_array(ct.Structure):
    _fields_ = [("data", ct.c_void_p), ("rows", ct.c_int64),
                ("cols", ct.c_int64), ("ld", ct.c_int64),
                ("dtype", ct.c_int32), ("on_device", ct.c_int32)]


class svm_adamw_tensor(ct.Structure):
    _fields_ = [("param", ct.c_void_p), ("grad", ct.c_void_p),
                ("master", ct.c_void_p), ("m", ct.c_void_p),
                ("v", ct.c_void_p), ("m_scale", ct.c_void_p),
                ("v_scale", ct.c_void_p), ("n", ct.c_int64),
                ("dtype", ct.c_int32), ("grad_dtype", ct.c_int32)]


class svm_adamw_params(ct.Structure):
    _fields_ = [("lr", ct.c_double), ("beta1", ct.c_double),
                ("beta2", ct.c_double), ("eps", ct.c_double),
                ("weight_decay", ct.c_double), ("grad_scale", ct.c_double),
                ("step", ct.c_int64), ("bits", ct.c_int32)]


_lib = None


def load(path: Optional[str] = None):
    """Load the built library; raise if it is missing (no fallback path)."""
    global _lib
    if _lib is not None:
        return _lib
    path = path or LIB_PATH
    if not os.path.exists(path):
        raise RuntimeError(
            "libmi355svm.so is not built; run __graft_entry__.build() or "
            "python -m paper_1706_05544_amd.build")
    try:
        # torch bundles its own copy of the HIP runtime under the same soname;
        # loading torch first makes the library bind to that copy, so that
        # one runtime serves both and device pointers are shared.
        import torch  # noqa: F401
    except ImportError:
        pass
    lib = ct.CDLL(path)
    P = ct.POINTER
    vp = ct.c_void_p
    lib.svm_params_default.argtypes = [P(svm_params)]
    lib.svm_params_default.restype = None
    lib.svm_train.argtypes = [P(svm_matrix), vp, P(svm_params), P(vp)]
    lib.svm_train_ovr.argtypes = [P(svm_matrix), vp, ct.c_int32,
                                  P(svm_params), P(vp)]
    lib.svm_predict.argtypes = [vp, P(svm_matrix), vp]
    lib.svm_predict_labels.argtypes = [vp, P(svm_matrix), vp]
    lib.svm_model_get_info.argtypes = [vp, ct.c_int32, P(svm_model_info)]
    lib.svm_model_get.argtypes = [vp, ct.c_int32, vp, vp, vp]
    lib.svm_model_free.argtypes = [vp]
    lib.svm_model_free.restype = None
    lib.svm_cache_release.argtypes = [ct.c_int32, P(ct.c_int64)]
    lib.svm_cross_validate.argtypes = [P(svm_matrix), vp, vp, ct.c_int32,
                                       P(svm_params), ct.c_int32, vp, vp,
                                       P(svm_cv_stats)]
    lib.svm_tune.argtypes = [P(svm_matrix), vp, vp, ct.c_int32,
                             P(svm_params), ct.c_int32, vp, ct.c_int32, vp, vp,
                             vp, vp, P(ct.c_int32)]
    lib.svm_last_error.restype = ct.c_char_p
    lib.svm_last_error.argtypes = []
    lib.svm_test_solver_create.argtypes = [P(svm_matrix), vp, P(svm_params),
                                           P(vp)]
    lib.svm_test_solver_free.argtypes = [vp]
    lib.svm_test_solver_free.restype = None
    lib.svm_test_set_state.argtypes = [vp, vp, vp]
    lib.svm_test_get_state.argtypes = [vp, vp, vp]
    lib.svm_test_select.argtypes = [vp, vp, P(ct.c_int32), P(ct.c_double),
                                    P(ct.c_double)]
    lib.svm_test_rows.argtypes = [vp, vp, ct.c_int32, vp]
    lib.svm_test_subproblem.argtypes = [vp, vp, ct.c_int32, ct.c_double,
                                        ct.c_int32, vp, P(ct.c_int32)]
    lib.svm_test_apply.argtypes = [vp, vp, ct.c_int32, vp]
    lib.svm_test_iterate.argtypes = [vp, ct.c_int64, P(ct.c_int64),
                                     P(ct.c_double)]
    lib.svm_predict_noalloc.argtypes = [vp, P(svm_matrix), vp, vp]
    lib.svm_test_finish.argtypes = [vp, ct.c_int32, P(ct.c_double),
                                    P(ct.c_double), P(ct.c_double),
                                    P(ct.c_int32)]
    pa, i64, i32 = P(svm_array), ct.c_int64, ct.c_int32
    lib.svm_linear.argtypes = [pa, pa, pa, pa, i32, pa, pa, vp, i64, i32, vp]
    lib.svm_linear_workspace.argtypes = [pa, pa, P(i64)]
    lib.svm_linear_backward.argtypes = [pa, pa, pa, pa, i32, pa, pa, pa, vp,
                                        i64, i32, vp]
    lib.svm_linear_backward_workspace.argtypes = [pa, pa, pa, i32, pa, pa, pa,
                                                  P(i64)]
    lib.svm_layer_norm.argtypes = [pa, pa, pa, ct.c_double, pa, vp, vp, i32,
                                   vp]
    lib.svm_layer_norm_backward.argtypes = [pa, pa, vp, vp, pa, pa, pa, pa, pa,
                                            vp, i64, i32, vp]
    lib.svm_layer_norm_backward_workspace.argtypes = [i64, i64, P(i64)]
    lib.svm_hinge_loss.argtypes = [pa, vp, ct.c_double, pa, vp, vp, i64, i32,
                                   vp]
    lib.svm_hinge_loss_workspace.argtypes = [i64, i64, P(i64)]
    lib.svm_adamw_step.argtypes = [vp, i32, P(svm_adamw_params), i32, vp]
    lib.svm_adamw_state.argtypes = [vp, vp, vp, vp, i64, vp, vp, i32, vp]
    for name in EXPORTS:  # fail now, not at first use, if one is missing
        getattr(lib, name)
    _lib = lib
    return lib


def svm_last_error() -> str:
    return load().svm_last_error().decode()


def _check(rc: int) -> int:
    if rc < 0:
        raise SvmError(rc, svm_last_error())
    return rc


def _is_torch(x) -> bool:
    return type(x).__module__.startswith("torch")


def _torch_sparse_csr():
    import torch
    return torch.sparse_csr


def _np_ptr(a: np.ndarray) -> int:
    return a.ctypes.data


class _Mat:
    """svm_matrix for a NumPy array (host), a scipy CSR matrix (host) or a
    contiguous torch tensor on the GPU (device); keeps its buffers alive."""

    def __init__(self, X):
        self.keep = []
        m = svm_matrix()
        if _is_torch(X) and X.layout == _torch_sparse_csr():
            import torch
            assert X.is_cuda and X.dim() == 2
            rp = X.crow_indices().to(torch.int64).contiguous()
            ci = X.col_indices().to(torch.int32).contiguous()
            cv = X.values().to(torch.float32).contiguous()
            self.keep += [rp, ci, cv]
            m.layout, m.on_device = SVM_CSR, 1
            m.n, m.d = X.shape
            m.values, m.row_ptr, m.col_idx = (cv.data_ptr(), rp.data_ptr(),
                                              ci.data_ptr())
            m.nnz = cv.numel()
            self.device = True
        elif _is_torch(X):
            import torch
            assert X.is_cuda and X.dtype == torch.float32 and X.dim() == 2
            X = X.contiguous()
            self.keep.append(X)
            m.layout, m.on_device = SVM_DENSE, 1
            m.n, m.d = X.shape
            m.values, m.ld = X.data_ptr(), X.shape[1]
            self.device = True
        elif hasattr(X, "indptr"):
            data = np.ascontiguousarray(X.data, dtype=np.float32)
            ip = np.ascontiguousarray(X.indptr, dtype=np.int64)
            ix = np.ascontiguousarray(X.indices, dtype=np.int32)
            self.keep += [data, ip, ix]
            m.layout, m.on_device = SVM_CSR, 0
            m.n, m.d = X.shape
            m.values, m.row_ptr, m.col_idx = _np_ptr(data), _np_ptr(ip), _np_ptr(ix)
            m.nnz = len(data)
            self.device = False
        else:
            A = np.ascontiguousarray(X, dtype=np.float32)
            assert A.ndim == 2
            self.keep.append(A)
            m.layout, m.on_device = SVM_DENSE, 0
            m.n, m.d = A.shape
            m.values, m.ld = (_np_ptr(A) if A.size else None), A.shape[1]
            self.device = False
        self.s = m


def _vec(v, dtype, device: bool):
    if device:
        import torch
        tdt = {np.float32: torch.float32, np.int32: torch.int32}[dtype]
        t = v if _is_torch(v) else torch.as_tensor(np.asarray(v))
        t = t.to(device="cuda", dtype=tdt).contiguous()
        return t, t.data_ptr()
    a = np.ascontiguousarray(v, dtype=dtype)
    return a, _np_ptr(a)


def svm_params_default(**overrides) -> svm_params:
    p = svm_params()
    load().svm_params_default(ct.byref(p))
    for k, v in overrides.items():
        if not hasattr(p, k):
            raise TypeError("unknown svm_params field %r" % k)
        setattr(p, k, v)
    return p


class Model:
    """Owns an svm_model*; freed with svm_model_free."""

    def __init__(self, ptr: int, status: int):
        self.ptr = ptr
        self.status = status

    def __del__(self):
        if getattr(self, "ptr", None) and _lib is not None:
            _lib.svm_model_free(self.ptr)
            self.ptr = None

    def info(self, output: int = 0) -> dict:
        return svm_model_get_info(self, output)

    @property
    def n_outputs(self) -> int:
        return self.info(0)["n_outputs"]


def _stream_of(device: bool):
    if not device:
        return None
    import torch
    return torch.cuda.current_stream().cuda_stream


def svm_train(X, y, params: Optional[svm_params] = None, alpha0=None,
              **kw) -> Model:
    p = params or svm_params_default(**kw)
    a0 = None
    if alpha0 is not None:  # warm start (host values, kept alive here)
        a0 = np.ascontiguousarray(alpha0, dtype=np.float64)
        p.alpha0 = _np_ptr(a0)
    M = _Mat(X)
    if M.device and not kw.get("stream") and not (params and params.stream):
        p.stream = _stream_of(True)
    yv, yp = _vec(y, np.float32, M.device)
    out = ct.c_void_p()
    rc = _check(load().svm_train(ct.byref(M.s), yp, ct.byref(p),
                                 ct.byref(out)))
    return Model(out.value, rc)


def svm_train_ovr(X, labels, n_classes: int,
                  params: Optional[svm_params] = None, **kw) -> Model:
    p = params or svm_params_default(**kw)
    M = _Mat(X)
    if M.device and not kw.get("stream") and not (params and params.stream):
        p.stream = _stream_of(True)
    lv, lp = _vec(labels, np.int32, M.device)
    out = ct.c_void_p()
    rc = _check(load().svm_train_ovr(ct.byref(M.s), lp, n_classes,
                                     ct.byref(p), ct.byref(out)))
    return Model(out.value, rc)


def svm_predict(model: Model, X):
    M = _Mat(X)
    n_out = model.n_outputs
    m = M.s.n
    if M.device:
        import torch
        D = torch.empty((m, n_out), dtype=torch.float64, device="cuda")
        ptr = D.data_ptr() if m else None
    else:
        D = np.empty((m, n_out), dtype=np.float64)
        ptr = _np_ptr(D) if m else None
    _check(load().svm_predict(model.ptr, ct.byref(M.s), ptr))
    return D[:, 0] if n_out == 1 else D


def svm_predict_noalloc(model: Model, X, out=None, stream=None):
    """svm_predict_noalloc: X a dense torch tensor on the GPU; the decision
    values go to `out` (a float64 tensor of m x n_outputs, allocated here
    when None) on `stream` (torch's current stream when None), not waited
    for.  Returns out."""
    import torch
    M = _Mat(X)
    if not M.device:
        raise SvmError(SVM_E_UNSUPPORTED, "svm_predict_noalloc takes a "
                       "tensor in device memory")
    n_out = model.n_outputs
    m = M.s.n
    if out is None:
        out = torch.empty((m, n_out), dtype=torch.float64, device=X.device)
    assert out.dtype == torch.float64 and out.is_contiguous()
    assert out.numel() == m * n_out
    st = stream if stream is not None else torch.cuda.current_stream()
    _check(load().svm_predict_noalloc(model.ptr, ct.byref(M.s),
                                      out.data_ptr() if m else None,
                                      st.cuda_stream))
    return out


def svm_predict_labels(model: Model, X):
    M = _Mat(X)
    m = M.s.n
    if M.device:
        import torch
        L = torch.empty((m,), dtype=torch.int32, device="cuda")
        ptr = L.data_ptr() if m else None
    else:
        L = np.empty((m,), dtype=np.int32)
        ptr = _np_ptr(L) if m else None
    _check(load().svm_predict_labels(model.ptr, ct.byref(M.s), ptr))
    return L


def svm_cache_release(device: int = -1) -> int:
    """Frees the row-cache memory the library keeps between trainings on
    `device` (-1: every device); returns the bytes freed."""
    freed = ct.c_int64(0)
    _check(load().svm_cache_release(device, ct.byref(freed)))
    return freed.value


def svm_model_get_info(model: Model, output: int = 0) -> dict:
    info = svm_model_info()
    _check(load().svm_model_get_info(model.ptr, output, ct.byref(info)))
    return info.as_dict()


def _cv_inputs(X, y, labels, fold):
    # X host or device; labels, targets and folds on the host
    M = _Mat(X)
    if hasattr(y, "cpu"):
        y = y.cpu().numpy()
    if hasattr(labels, "cpu"):
        labels = labels.cpu().numpy()
    yv = None if y is None else np.ascontiguousarray(y, dtype=np.float32)
    lv = None if labels is None else np.ascontiguousarray(labels,
                                                          dtype=np.int32)
    fv = None if fold is None else np.ascontiguousarray(fold, dtype=np.int32)
    return (M, yv, lv, fv,
            None if yv is None else _np_ptr(yv),
            None if lv is None else _np_ptr(lv),
            None if fv is None else _np_ptr(fv))


def svm_cross_validate(X, y=None, labels=None, n_classes: int = 0,
                       k: int = 10, fold=None,
                       params: Optional[svm_params] = None, **kw):
    """k-fold cross-validation -> (decision values n x n_outputs, stats)."""
    p = params or svm_params_default(**kw)
    M, yv, lv, fv, yp, lp, fp = _cv_inputs(X, y, labels, fold)
    if M.device and not kw.get("stream") and not (params and params.stream):
        p.stream = _stream_of(True)
    n_out = n_classes if labels is not None else 1
    D = np.empty((M.s.n, n_out), dtype=np.float64)
    st = svm_cv_stats()
    rc = _check(load().svm_cross_validate(ct.byref(M.s), yp, lp, n_classes,
                                          ct.byref(p), k, fp, _np_ptr(D),
                                          ct.byref(st)))
    out = st.as_dict()
    out["rc"] = rc
    return (D[:, 0] if n_out == 1 else D), out


def svm_tune(X, y=None, labels=None, n_classes: int = 0, k: int = 10,
             fold=None, C=None, gamma=None, epsilon=None,
             params: Optional[svm_params] = None, **kw):
    """Grid tuning by k-fold cross-validation -> (errors, best index)."""
    p = params or svm_params_default(**kw)
    M, yv, lv, fv, yp, lp, fp = _cv_inputs(X, y, labels, fold)
    if M.device and not kw.get("stream") and not (params and params.stream):
        p.stream = _stream_of(True)
    arrs = [None if a is None else np.ascontiguousarray(a, dtype=np.float64)
            for a in (C, gamma, epsilon)]
    n_grid = max(len(a) for a in arrs if a is not None)
    err = np.empty(n_grid, dtype=np.float64)
    best = ct.c_int32()
    _check(load().svm_tune(ct.byref(M.s), yp, lp, n_classes, ct.byref(p), k,
                           fp, n_grid,
                           *[None if a is None else _np_ptr(a) for a in arrs],
                           _np_ptr(err), ct.byref(best)))
    return err, best.value


def svm_model_get(model: Model, output: int = 0, with_alpha: bool = False):
    """-> (sv_idx int32, coef fp64, alpha fp64 or None)."""
    info = svm_model_get_info(model, output)
    k = info["n_sv_output"]
    idx = np.empty(max(k, 1), dtype=np.int32)
    coef = np.empty(max(k, 1), dtype=np.float64)
    alpha = None
    if with_alpha:
        N = info["n_train"] * (2 if info["type"] == SVM_EPS_SVR else 1)
        alpha = np.empty(N, dtype=np.float64)
    _check(load().svm_model_get(model.ptr, output, _np_ptr(idx),
                                _np_ptr(coef),
                                _np_ptr(alpha) if alpha is not None else None))
    return idx[:k], coef[:k], alpha


# ---------------------------------------------------------------------------
# Feature maps: layers, their gradients, the loss and the optimiser step.
# These calls take torch tensors on the GPU (float32, bfloat16 or float16, one
# type to a call), queue their work on `stream` (torch's current stream when
# None) and do not wait for it.  A tensor's last dimension is its columns, the
# rest its rows; inputs whose rows are not at one stride, or whose values in a
# row are not side by side, are copied first.
# Outside of autograd: outputs carry no graph, whatever the inputs require;
# gradients come from the _backward calls.  What a call writes in place is
# marked as changed, so that autograd sees a tensor that it saved go stale.
# ---------------------------------------------------------------------------

_ACTS = {"none": SVM_ACT_NONE, "relu": SVM_ACT_RELU, "gelu": SVM_ACT_GELU,
         "silu": SVM_ACT_SILU, "tanh": SVM_ACT_TANH, "cos": SVM_ACT_COS}
_DTYPES: dict = {}


def _act(act) -> int:
    if isinstance(act, str):
        if act not in _ACTS:
            raise SvmError(SVM_E_INVALID, "unknown activation %r" % act)
        return _ACTS[act]
    return act


def _rows_of(t):
    """(rows, cols, ld) of a tensor whose rows are at one stride, else
    None."""
    nd = t.dim()
    if nd == 0:
        return None
    cols = t.shape[-1]
    n = t.numel()
    if n == 0:
        return (0 if cols else 1), cols, cols
    if t.is_contiguous():
        return n // cols, cols, cols
    st = t.stride()
    if cols > 1 and st[-1] != 1:
        return None
    rows, ld = 1, 0
    for k in range(nd - 2, -1, -1):
        size = t.shape[k]
        if size == 1:
            continue
        if rows == 1:
            ld = st[k]
        elif st[k] != ld * rows:
            return None
        rows *= size
    if rows == 1:
        ld = cols
    if ld < cols:
        return None
    return rows, cols, ld


class _Call:
    """The device and stream of a call, and the memory that its queued work
    uses."""

    def __init__(self, t, stream):
        if not _is_torch(t) or not t.is_cuda:
            raise SvmError(SVM_E_UNSUPPORTED,
                           "this call takes tensors in device memory")
        import torch
        if not _DTYPES:
            _DTYPES.update({torch.float32: SVM_F32, torch.bfloat16: SVM_BF16,
                            torch.float16: SVM_F16})
        self.device = t.device
        self.index = t.get_device()
        cur = torch._C._cuda_getCurrentRawStream(self.index)
        self.stream = stream
        self.handle = cur if stream is None else stream.cuda_stream
        self.other = self.handle != cur
        self.keep = []

    def arr(self, t, what: str, out: bool = False):
        """svm_array of a tensor (None: None); a copy with rows side by side
        where it is an input that has none."""
        if t is None:
            return None
        try:
            d, index = _DTYPES[t.dtype], t.get_device()
        except (AttributeError, KeyError, TypeError):
            d, index = None, -1
        if index != self.index:
            if index < 0:
                raise SvmError(SVM_E_UNSUPPORTED, "%s must be a float32, "
                               "bfloat16 or float16 tensor in device memory"
                               % what)
            raise SvmError(SVM_E_INVALID, "%s is on another device" % what)
        if t.is_contiguous() and t.numel() and t.dim():
            cols = ld = t.shape[-1]
            rows = t.numel() // cols
        else:
            r = _rows_of(t)
            if r is None:
                if out:
                    raise SvmError(SVM_E_INVALID, "%s: its rows must be at "
                                   "one stride, the values of a row side by "
                                   "side" % what)
                t = t.contiguous()
                r = _rows_of(t)
                if r is None:
                    raise SvmError(SVM_E_INVALID, "%s must have a dimension"
                                   % what)
            rows, cols, ld = r
        self.keep.append(t)
        return svm_array(t.data_ptr(), rows, cols, ld, d, 1)

    def floats(self, t, rows: int, what: str) -> int:
        """Address of a float32 value for each row."""
        import torch
        if not _is_torch(t) or t.dtype != torch.float32 or \
                t.get_device() < 0:
            raise SvmError(SVM_E_UNSUPPORTED, "%s must be a float32 tensor in "
                           "device memory" % what)
        if t.numel() != rows or t.get_device() != self.index:
            raise SvmError(SVM_E_INVALID, "%s must have a value for each row, "
                           "on the same device" % what)
        t = t.contiguous()
        self.keep.append(t)
        return t.data_ptr()

    def empty(self, shape, dtype):
        import torch
        t = torch.empty(shape, dtype=dtype, device=self.device)
        self.keep.append(t)
        return t

    def work(self, nbytes: int):
        """Address of a workspace (None for no bytes)."""
        if not nbytes:
            return None
        import torch
        return self.empty((nbytes,), torch.uint8).data_ptr()

    def ready(self):
        """Before the launch: on another stream than torch's current one the
        work waits for what that one has queued (copies of inputs, earlier
        users of the memory given out here)."""
        if self.other:
            import torch
            self.stream.wait_stream(torch.cuda.current_stream(self.device))

    def done(self):
        # memory that torch gave out on its own stream is not handed out
        # again before the work on the other one is done
        if self.other:
            for t in self.keep:
                t.record_stream(self.stream)


def _written(tensors):
    """Marks tensors that a call has written in place as changed."""
    import torch
    torch.autograd.graph.increment_version(tensors)


def _ref(a):
    return None if a is None else ct.byref(a)


def _ptr(t):
    return None if t is None else t.data_ptr()


def svm_linear(X, W, bias=None, residual=None, act="none", save: bool = False,
               out=None, stream=None):
    """act(X W^T + bias) + residual -> Y, or (Y, Z) with the pre-activations
    Z when `save`.  `out` receives Y when given (it may be `residual`).
    No autograd graph is made: svm_linear_backward gives the gradients."""
    lib = load()
    c = _Call(X, stream)
    a, w = c.arr(X, "X"), c.arr(W, "W")
    shape = X.shape[:-1] + (w.rows,)
    Y = out if out is not None else X.new_empty(shape)
    Z = X.new_empty(shape) if save else None
    need = ct.c_int64()
    _check(lib.svm_linear_workspace(ct.byref(a), ct.byref(w),
                                    ct.byref(need)))
    ws = c.work(need.value)
    b, r = c.arr(bias, "bias"), c.arr(residual, "residual")
    c.ready()
    _check(lib.svm_linear(ct.byref(a), ct.byref(w), _ref(b), _ref(r),
                          _act(act), ct.byref(c.arr(Y, "out", True)),
                          _ref(c.arr(Z, "Z", True)), ws, need.value,
                          c.index, c.handle))
    c.done()
    if out is not None:
        _written(out)
    return (Y, Z) if save else Y


def svm_linear_backward(dY, X, W, Z=None, act="none", need=(True, True, True),
                        stream=None):
    """Gradients (dX, dW, dbias) of svm_linear; None where `need` is false.
    The residual's gradient is dY itself.  X may be None without dW, W
    without dX."""
    lib = load()
    c = _Call(dY, stream)
    g, a, w = c.arr(dY, "dY"), c.arr(X, "X"), c.arr(W, "W")
    if (a is None and need[1]) or (w is None and need[0]):
        raise SvmError(SVM_E_INVALID, "dW needs X, and dX needs W")
    dX = dW = None
    if need[0]:
        dX = dY.new_empty(dY.shape[:-1] + (w.cols,) if a is None else X.shape)
    if need[1]:
        dW = dY.new_empty(W.shape if w is not None else (g.cols, a.cols))
    db = dY.new_empty(g.cols) if need[2] else None
    rx, rw, rb = (c.arr(dX, "dX", True), c.arr(dW, "dW", True),
                  c.arr(db, "dbias", True))
    size = ct.c_int64()
    act = _act(act)
    _check(lib.svm_linear_backward_workspace(
        ct.byref(g), _ref(a), _ref(w), act, _ref(rx), _ref(rw), _ref(rb),
        ct.byref(size)))
    ws = c.work(size.value)
    z = c.arr(Z, "Z")
    c.ready()
    _check(lib.svm_linear_backward(
        ct.byref(g), _ref(a), _ref(w), _ref(z), act, _ref(rx), _ref(rw),
        _ref(rb), ws, size.value, c.index, c.handle))
    c.done()
    return dX, dW, db


def svm_layer_norm(X, weight=None, bias=None, eps: float = 1e-5,
                   save: bool = False, out=None, stream=None):
    """Layer norm over the last dimension -> Y, or (Y, mean, rstd) when
    `save` (float32, one of each to a row)."""
    import torch
    lib = load()
    c = _Call(X, stream)
    a = c.arr(X, "X")
    Y = out if out is not None else X.new_empty(X.shape)
    mean = c.empty(X.shape[:-1], torch.float32) if save else None
    rstd = c.empty(X.shape[:-1], torch.float32) if save else None
    w, b = c.arr(weight, "weight"), c.arr(bias, "bias")
    c.ready()
    _check(lib.svm_layer_norm(ct.byref(a), _ref(w), _ref(b), eps,
                              ct.byref(c.arr(Y, "out", True)), _ptr(mean),
                              _ptr(rstd), c.index, c.handle))
    c.done()
    if out is not None:
        _written(out)
    return (Y, mean, rstd) if save else Y


def svm_layer_norm_backward(dY, X, mean, rstd, weight=None, residual=None,
                            need=(True, True, True), stream=None):
    """Gradients (dX, dweight, dbias) of svm_layer_norm; None where `need` is
    false.  `residual` is added to dX: the gradient that reaches X past the
    norm."""
    lib = load()
    c = _Call(dY, stream)
    g, a = c.arr(dY, "dY"), c.arr(X, "X")
    mp = c.floats(mean, g.rows, "mean")
    rp = c.floats(rstd, g.rows, "rstd")
    dX = dY.new_empty(X.shape) if need[0] else None
    dw = dY.new_empty(g.cols) if need[1] else None
    db = dY.new_empty(g.cols) if need[2] else None
    size = ct.c_int64()
    if need[1] or need[2]:
        _check(lib.svm_layer_norm_backward_workspace(g.rows, g.cols,
                                                     ct.byref(size)))
    ws = c.work(size.value)
    w, r = c.arr(weight, "weight"), c.arr(residual, "residual")
    c.ready()
    _check(lib.svm_layer_norm_backward(
        ct.byref(g), ct.byref(a), mp, rp, _ref(w), _ref(r),
        _ref(c.arr(dX, "dX", True)), _ref(c.arr(dw, "dweight", True)),
        _ref(c.arr(db, "dbias", True)), ws, size.value, c.index,
        c.handle))
    c.done()
    return dX, dw, db


def svm_hinge_loss(S, labels, scale: Optional[float] = None,
                   need_grad: bool = True, stream=None):
    """Squared hinge loss of the scores S (rows x classes), one class against
    the rest -> (loss, dS): a float32 scalar on the device and the gradient
    (None without `need_grad`).  labels: int32, one to a row; a row whose
    label is no class is left out.  `scale` multiplies both (1 / rows when
    None)."""
    import torch
    lib = load()
    c = _Call(S, stream)
    a = c.arr(S, "S")
    if not _is_torch(labels) or labels.get_device() != c.index or \
            labels.dtype != torch.int32:
        raise SvmError(SVM_E_UNSUPPORTED, "labels must be an int32 tensor in "
                       "device memory")
    if labels.numel() != a.rows:
        raise SvmError(SVM_E_INVALID, "labels must have one for each row")
    labels = labels.contiguous()
    c.keep.append(labels)
    loss = c.empty((), torch.float32)
    dS = S.new_empty(S.shape) if need_grad else None
    size = ct.c_int64()
    _check(lib.svm_hinge_loss_workspace(a.rows, a.cols, ct.byref(size)))
    ws = c.work(size.value)
    c.ready()
    _check(lib.svm_hinge_loss(
        ct.byref(a), labels.data_ptr(),
        1.0 / max(a.rows, 1) if scale is None else scale,
        _ref(c.arr(dS, "dS", True)), loss.data_ptr(), ws, size.value,
        c.index, c.handle))
    c.done()
    return loss, dS


def svm_adamw_parts(params):
    """Where each tensor's states begin in the flat states of
    svm_adamw_step, and their total length: the tensors follow one another,
    each from a multiple of SVM_ADAMW_BLOCK."""
    return _parts_of([p.numel() for p in params])


def _parts_of(sizes):
    at, total = [], 0
    for n in sizes:
        at.append(total)
        total += -(-n // SVM_ADAMW_BLOCK) * SVM_ADAMW_BLOCK
    return np.array(at, dtype=np.int64), total


def svm_adamw_states(params, bits: int = 32, master: bool = False):
    """States to start from -> (m, v, m_scale, v_scale, master) for
    svm_adamw_step: zeros, and with `master` the parameters in 32 bits."""
    import torch
    at, total = svm_adamw_parts(params)
    dev = params[0].device
    z = lambda n, t: torch.zeros(n, dtype=t, device=dev)  # noqa: E731
    ms = vs = flat = None
    if bits == 8:
        m, v = z(total, torch.int8), z(total, torch.uint8)
        ms, vs = (z(total // SVM_ADAMW_BLOCK, torch.float32)
                  for _ in range(2))
    else:
        m, v = z(total, torch.float32), z(total, torch.float32)
    if master:
        flat = z(total, torch.float32)
        for a, p in zip(at, params):
            flat[a:a + p.numel()].copy_(p.detach().reshape(-1))
    return m, v, ms, vs, flat


_ADAMW_ROW = np.dtype([("param", "u8"), ("grad", "u8"), ("master", "u8"),
                       ("m", "u8"), ("v", "u8"), ("m_scale", "u8"),
                       ("v_scale", "u8"), ("n", "i8"), ("dtype", "i4"),
                       ("grad_dtype", "i4")])


def svm_adamw_step(params, grads, m, v, m_scale=None, v_scale=None,
                   master=None, lr: float = 1e-3, beta1: float = 0.9,
                   beta2: float = 0.999, eps: float = 1e-8,
                   weight_decay: float = 0.01, step: int = 1,
                   grad_scale: float = 1.0, stream=None):
    """One AdamW step over the tensors `params` (contiguous, updated in
    place, no two of them overlapping) with the gradients `grads`.  The states are flat tensors as
    svm_adamw_states makes them: m and v in float32, or int8 and uint8 with
    float32 scales, and optionally the master weights."""
    import torch
    if len(params) != len(grads):
        raise SvmError(SVM_E_INVALID, "params and grads differ in number")
    if not len(params):
        return
    lib = load()
    c = _Call(params[0], stream)
    sizes = [p.numel() for p in params]
    at, total = _parts_of(sizes)
    bits = 8 if m.dtype == torch.int8 else 32
    want = [("m", m, torch.int8 if bits == 8 else torch.float32, total),
            ("v", v, torch.uint8 if bits == 8 else torch.float32, total)]
    if bits == 8:
        nb = total // SVM_ADAMW_BLOCK
        want += [("m_scale", m_scale, torch.float32, nb),
                 ("v_scale", v_scale, torch.float32, nb)]
    if master is not None:
        want.append(("master", master, torch.float32, total))
    for what, t, dtype, n in want:
        if not _is_torch(t) or t.dtype != dtype or t.device != c.device or \
                t.numel() != n or not t.is_contiguous():
            raise SvmError(SVM_E_INVALID, "%s must be a contiguous %s tensor "
                           "of %d values on the parameters' device"
                           % (what, dtype, n))
        c.keep.append(t)
    T = torch.Tensor
    if not all(map(T.is_contiguous, params)) or \
            not all(map(T.is_same_size, params, grads)):
        raise SvmError(SVM_E_INVALID, "parameters must be contiguous, "
                       "gradients of their shapes")
    if not all(map(T.is_contiguous, grads)):
        grads = [g.contiguous() for g in grads]
    if set(map(T.get_device, params)) | set(map(T.get_device, grads)) != \
            {c.index}:
        raise SvmError(SVM_E_INVALID, "the tensors are on several devices")
    pd = [_DTYPES.get(p.dtype) for p in params]
    gd = [_DTYPES.get(g.dtype) for g in grads]
    if None in pd or None in gd:
        raise SvmError(SVM_E_UNSUPPORTED, "parameters and gradients must be "
                       "float32, bfloat16 or float16")
    c.keep += params
    written = c.keep[:]  # (the states, and these)
    c.keep += grads
    tab = np.zeros(len(params), dtype=_ADAMW_ROW)
    tab["param"] = list(map(T.data_ptr, params))
    tab["grad"] = list(map(T.data_ptr, grads))
    tab["n"] = sizes
    tab["dtype"], tab["grad_dtype"] = pd, gd
    esize = 1 if bits == 8 else 4
    tab["m"], tab["v"] = m.data_ptr() + at * esize, v.data_ptr() + at * esize
    if bits == 8:
        sc = at // SVM_ADAMW_BLOCK * 4
        tab["m_scale"], tab["v_scale"] = (m_scale.data_ptr() + sc,
                                          v_scale.data_ptr() + sc)
    if master is not None:
        tab["master"] = np.where(tab["dtype"] == SVM_F32, 0,
                                 master.data_ptr() + at * 4)
    h = svm_adamw_params(lr, beta1, beta2, eps, weight_decay, grad_scale,
                         step, bits)
    c.ready()
    _check(lib.svm_adamw_step(_np_ptr(tab), len(params), ct.byref(h), c.index,
                              c.handle))
    c.done()
    _written(written)


def svm_adamw_state(m, v, m_scale, v_scale, stream=None):
    """The values that states in 8 bits stand for -> (m, v) in float32."""
    import torch
    lib = load()
    c = _Call(m, stream)
    n = m.numel()
    nb = -(-n // SVM_ADAMW_BLOCK)
    for what, t, dtype, k in (("m", m, torch.int8, n), ("v", v, torch.uint8, n),
                              ("m_scale", m_scale, torch.float32, nb),
                              ("v_scale", v_scale, torch.float32, nb)):
        if not _is_torch(t) or t.dtype != dtype or t.numel() != k or \
                t.device != c.device or not t.is_contiguous():
            raise SvmError(SVM_E_INVALID, "%s must be a contiguous %s tensor "
                           "of %d values" % (what, dtype, k))
        c.keep.append(t)
    mo, vo = c.empty((n,), torch.float32), c.empty((n,), torch.float32)
    c.ready()
    _check(lib.svm_adamw_state(m.data_ptr(), v.data_ptr(), m_scale.data_ptr(),
                               v_scale.data_ptr(), n, mo.data_ptr(),
                               vo.data_ptr(), c.index, c.handle))
    c.done()
    return mo, vo


class Solver:
    """The svm_test_* hooks: a solver whose state can be set and stepped."""

    def __init__(self, X, y, params: Optional[svm_params] = None, **kw):
        p = params or svm_params_default(**kw)
        M = _Mat(X)
        yv, yp = _vec(y, np.float32, False)
        out = ct.c_void_p()
        _check(load().svm_test_solver_create(ct.byref(M.s), yp, ct.byref(p),
                                             ct.byref(out)))
        self.ptr = out.value
        self.n = M.s.n
        self.N = self.n * (2 if p.type == SVM_EPS_SVR else 1)

    def __del__(self):
        if getattr(self, "ptr", None) and _lib is not None:
            _lib.svm_test_solver_free(self.ptr)
            self.ptr = None

    def set_state(self, alpha, F):
        a = np.ascontiguousarray(alpha, dtype=np.float64)
        f = np.ascontiguousarray(F, dtype=np.float64)
        _check(load().svm_test_set_state(self.ptr, _np_ptr(a), _np_ptr(f)))

    def get_state(self):
        a = np.empty(self.N, dtype=np.float64)
        f = np.empty(self.n, dtype=np.float64)
        _check(load().svm_test_get_state(self.ptr, _np_ptr(a), _np_ptr(f)))
        return a, f

    def select(self):
        B = np.empty(64, dtype=np.int32)
        nB = ct.c_int32()
        m = ct.c_double()
        M = ct.c_double()
        _check(load().svm_test_select(self.ptr, _np_ptr(B), ct.byref(nB),
                                      ct.byref(m), ct.byref(M)))
        return B[: nB.value].copy(), m.value, M.value

    def rows(self, samples):
        s = np.ascontiguousarray(samples, dtype=np.int32)
        out = np.empty((len(s), self.n), dtype=np.float32)
        _check(load().svm_test_rows(self.ptr, _np_ptr(s), len(s),
                                    _np_ptr(out)))
        return out

    def subproblem(self, B, inner_tol: float, max_inner: int):
        b = np.ascontiguousarray(B, dtype=np.int32)
        out = np.empty(len(b), dtype=np.float64)
        steps = ct.c_int32()
        _check(load().svm_test_subproblem(self.ptr, _np_ptr(b), len(b),
                                          inner_tol, max_inner, _np_ptr(out),
                                          ct.byref(steps)))
        return out, steps.value

    def apply(self, B, alpha_B):
        b = np.ascontiguousarray(B, dtype=np.int32)
        a = np.ascontiguousarray(alpha_B, dtype=np.float64)
        _check(load().svm_test_apply(self.ptr, _np_ptr(b), len(b), _np_ptr(a)))

    def iterate(self, k: int):
        it = ct.c_int64()
        gap = ct.c_double()
        _check(load().svm_test_iterate(self.ptr, k, ct.byref(it),
                                       ct.byref(gap)))
        return it.value, gap.value

    def finish(self, max_passes: int = 3):
        """End a training on the current state: (gap, b, obj, status)."""
        gap, b, obj = ct.c_double(), ct.c_double(), ct.c_double()
        st = ct.c_int32()
        _check(load().svm_test_finish(self.ptr, max_passes, ct.byref(gap),
                                      ct.byref(b), ct.byref(obj),
                                      ct.byref(st)))
        return gap.value, b.value, obj.value, st.value
