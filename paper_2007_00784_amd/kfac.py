"""ctypes binding of libkfac_hip.so: the same entry points as ``include/kfac.h``.

Argument marshalling only.  Device buffers are torch tensors (PyTorch is used for device memory and
streams, nothing else) or raw integer device addresses; every step of the path runs in the HIP
library.  Loading fails loudly if the library has not been built (``python -m
paper_2007_00784_amd.build`` or ``__graft_entry__.build()``); there is no fallback.
"""
import ctypes
import os
import warnings

KFAC_OK, KFAC_EINVAL, KFAC_ENOCONV, KFAC_EHIP, KFAC_EWORKSPACE, KFAC_ESCRATCH = 0, -1, -2, -3, -4, -5
KFAC_F32, KFAC_BF16 = 0, 1
KFAC_LAYOUT_RD, KFAC_LAYOUT_NDT = 0, 1

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libkfac_hip.so")

EXPORTS = (
    "kfac_create", "kfac_destroy", "kfac_workspace_bytes", "kfac_eig_workspace_bytes", "kfac_strerror",
    "kfac_unfold", "kfac_unfold_batched", "kfac_unfold_workspace_bytes", "kfac_update_factors", "kfac_eig", "kfac_precondition", "kfac_schedule_due",
    "kfac_profile_begin", "kfac_profile_end", "kfac_precondition_batched", "kfac_precondition_workspace_bytes",
    "kfac_update_factors_batched", "kfac_update_factors_workspace_bytes", "kfac_precondition_batched_scaled",
    "kfac_update_factors_static", "kfac_static_scratch_bytes",
    "kfac_invert_factors", "kfac_invert_workspace_bytes", "kfac_precondition_inverse",
    "kfac_precondition_inverse_batched", "kfac_precondition_inverse_workspace_bytes",
    "kfac_experts_forward", "kfac_experts_input_grad", "kfac_experts_weight_grad", "kfac_update_factors_experts",
    "kfac_experts_workspace_bytes", "kfac_adamw_batched", "kfac_adamw_state_values",
    "kfac_experts_route", "kfac_experts_route_grad", "kfac_experts_dispatch", "kfac_experts_dispatch_workspace_bytes", "kfac_experts_gather",
    "kfac_experts_combine", "kfac_experts_combine_grad", "kfac_grad_norm_batched", "kfac_grad_norm_workspace_bytes", "kfac_clip_grads_batched",
)


class kfac_precond_inv_item(ctypes.Structure):
    _fields_ = [("Ainv", ctypes.c_void_p), ("dA", ctypes.c_int), ("Ginv", ctypes.c_void_p), ("dG", ctypes.c_int),
                ("grad", ctypes.c_void_p), ("grad_dtype", ctypes.c_int)]


class kfac_conv_desc(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int) for n in
                ("N", "C", "H", "W", "kh", "kw", "stride_h", "stride_w", "pad_h", "pad_w", "dtype")]


class kfac_eig_opts(ctypes.Structure):
    _fields_ = [("max_sweeps", ctypes.c_int), ("tol", ctypes.c_float), ("fp32_only", ctypes.c_int),
                ("warm_start", ctypes.c_int)]


class kfac_eig_info(ctypes.Structure):
    _fields_ = [("sweeps", ctypes.c_int), ("off_norm_rel", ctypes.c_float), ("converged", ctypes.c_int)]


class kfac_kernel_stat(ctypes.Structure):
    _fields_ = [("name", ctypes.c_char * 32), ("launches", ctypes.c_int), ("ms", ctypes.c_double),
                ("flops", ctypes.c_double), ("bytes", ctypes.c_double)]


class kfac_precond_item(ctypes.Structure):
    _fields_ = [("QA", ctypes.c_void_p), ("lamA", ctypes.c_void_p), ("dA", ctypes.c_int),
                ("QG", ctypes.c_void_p), ("lamG", ctypes.c_void_p), ("dG", ctypes.c_int),
                ("damping", ctypes.c_float), ("grad", ctypes.c_void_p), ("grad_dtype", ctypes.c_int),
                ("factored_damping", ctypes.c_int), ("split_f16", ctypes.c_int)]


class kfac_factor_item(ctypes.Structure):
    _fields_ = [("X", ctypes.c_void_p), ("dtype", ctypes.c_int), ("layout", ctypes.c_int),
                ("N", ctypes.c_int), ("d", ctypes.c_int), ("T", ctypes.c_int), ("append_ones", ctypes.c_int),
                ("scale", ctypes.c_float), ("decay", ctypes.c_float), ("F", ctypes.c_void_p)]


class kfac_expert_desc(ctypes.Structure):
    _fields_ = [("experts", ctypes.c_int), ("rows", ctypes.c_int), ("d_in", ctypes.c_int), ("d_out", ctypes.c_int),
                ("append_ones", ctypes.c_int), ("dtype", ctypes.c_int), ("offsets", ctypes.c_void_p)]


class kfac_slot_desc(ctypes.Structure):
    _fields_ = [("tokens", ctypes.c_int), ("topk", ctypes.c_int), ("rows", ctypes.c_int), ("d", ctypes.c_int), ("dtype", ctypes.c_int)]


class kfac_grad_item(ctypes.Structure):
    _fields_ = [("grad", ctypes.c_void_p), ("grad_dtype", ctypes.c_int), ("out", ctypes.c_void_p), ("out_dtype", ctypes.c_int), ("n", ctypes.c_int64)]


class kfac_adamw_item(ctypes.Structure):
    _fields_ = [("param", ctypes.c_void_p), ("param_dtype", ctypes.c_int), ("grad", ctypes.c_void_p), ("grad_dtype", ctypes.c_int),
                ("m", ctypes.c_void_p), ("v", ctypes.c_void_p), ("m_scale", ctypes.c_void_p), ("v_scale", ctypes.c_void_p),
                ("copy", ctypes.c_void_p), ("n", ctypes.c_int64)]


class kfac_adamw_opts(ctypes.Structure):
    _fields_ = [("beta1", ctypes.c_double), ("beta2", ctypes.c_double), ("lr", ctypes.c_float), ("eps", ctypes.c_float),
                ("weight_decay", ctypes.c_float), ("step", ctypes.c_int64), ("grad_scale", ctypes.c_void_p),
                ("lr_dev", ctypes.c_void_p), ("step_dev", ctypes.c_void_p), ("seed", ctypes.c_uint64)]


class KfacError(RuntimeError):
    def __init__(self, code, where):
        self.code = code
        super().__init__("%s: %s (%d)" % (where, kfac_strerror(code), code))


_lib = None


def lib():
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(LIB_PATH):
        raise ImportError("libkfac_hip.so is not built: run `python -m paper_2007_00784_amd.build`")
    L = ctypes.CDLL(LIB_PATH)
    vp, i, f, sz, i64 = ctypes.c_void_p, ctypes.c_int, ctypes.c_float, ctypes.c_size_t, ctypes.c_int64
    ip = ctypes.POINTER(ctypes.c_int)
    L.kfac_create.argtypes = [ctypes.POINTER(vp), i, vp, vp, sz]
    L.kfac_destroy.argtypes = [vp]
    L.kfac_workspace_bytes.argtypes = [i, i, i64]
    L.kfac_workspace_bytes.restype = sz
    L.kfac_eig_workspace_bytes.argtypes = [i, ip]
    L.kfac_eig_workspace_bytes.restype = sz
    L.kfac_strerror.argtypes = [i]
    L.kfac_strerror.restype = ctypes.c_char_p
    L.kfac_unfold.argtypes = [vp, ctypes.POINTER(kfac_conv_desc), vp, vp]
    L.kfac_unfold_batched.argtypes = [vp, i, ctypes.POINTER(kfac_conv_desc), ctypes.POINTER(vp), ctypes.POINTER(vp)]
    L.kfac_unfold_workspace_bytes.argtypes = [i]
    L.kfac_unfold_workspace_bytes.restype = sz
    L.kfac_update_factors.argtypes = [vp, vp, i, i, i, i, i, i, f, f, vp]
    L.kfac_update_factors_static.argtypes = [vp, vp, i, i, i, i, i, i, f, f, vp]
    L.kfac_static_scratch_bytes.argtypes = []
    L.kfac_static_scratch_bytes.restype = sz
    L.kfac_eig.argtypes = [vp, i, ctypes.POINTER(vp), ip, ctypes.POINTER(vp), ctypes.POINTER(vp),
                           ctypes.POINTER(kfac_eig_opts), ctypes.POINTER(kfac_eig_info)]
    L.kfac_precondition.argtypes = [vp, vp, vp, i, vp, vp, i, f, vp, i]
    L.kfac_schedule_due.argtypes = [i64, i, i, ip, ip]
    L.kfac_precondition_batched.argtypes = [vp, i, ctypes.POINTER(kfac_precond_item)]
    L.kfac_precondition_batched_scaled.argtypes = [vp, i, ctypes.POINTER(kfac_precond_item), f, f, vp]
    L.kfac_precondition_workspace_bytes.argtypes = [i, ctypes.POINTER(kfac_precond_item)]
    L.kfac_precondition_workspace_bytes.restype = sz
    L.kfac_update_factors_batched.argtypes = [vp, i, ctypes.POINTER(kfac_factor_item)]
    L.kfac_update_factors_workspace_bytes.argtypes = [i, ctypes.POINTER(kfac_factor_item)]
    L.kfac_update_factors_workspace_bytes.restype = sz
    L.kfac_invert_factors.argtypes = [vp, i, ctypes.POINTER(vp), ip, f, ctypes.POINTER(vp)]
    L.kfac_invert_workspace_bytes.argtypes = [i, ip]
    L.kfac_invert_workspace_bytes.restype = sz
    L.kfac_precondition_inverse.argtypes = [vp, vp, i, vp, i, vp, i]
    L.kfac_precondition_inverse_batched.argtypes = [vp, i, ctypes.POINTER(kfac_precond_inv_item)]
    L.kfac_precondition_inverse_workspace_bytes.argtypes = [i, ctypes.POINTER(kfac_precond_inv_item)]
    L.kfac_precondition_inverse_workspace_bytes.restype = sz
    dp = ctypes.POINTER(kfac_expert_desc)
    L.kfac_experts_workspace_bytes.argtypes = [dp]
    L.kfac_experts_workspace_bytes.restype = sz
    L.kfac_experts_forward.argtypes = [vp, dp, vp, i64, vp, vp, i64]
    L.kfac_experts_input_grad.argtypes = [vp, dp, vp, i64, vp, vp, i64]
    L.kfac_experts_weight_grad.argtypes = [vp, dp, vp, i64, vp, i64, i, vp, i]
    L.kfac_update_factors_experts.argtypes = [vp, i, i, vp, vp, i, i64, i, i, i, f, f, vp]
    L.kfac_adamw_batched.argtypes = [vp, i, ctypes.POINTER(kfac_adamw_item), ctypes.POINTER(kfac_adamw_opts)]
    L.kfac_adamw_state_values.argtypes = [vp, vp, vp, i64, vp, i]
    sp, gp = ctypes.POINTER(kfac_slot_desc), ctypes.POINTER(kfac_grad_item)
    L.kfac_experts_route.argtypes = [vp, i, i, i, vp, i, i64, i, vp, vp]
    L.kfac_experts_route_grad.argtypes = [vp, i, i, i, vp, i, i64, vp, vp, i, vp, i64]
    L.kfac_experts_dispatch.argtypes = [vp, sp, i, vp, vp, i64, vp, vp, vp, i64]
    L.kfac_experts_dispatch_workspace_bytes.argtypes = [i, i, i]
    L.kfac_experts_dispatch_workspace_bytes.restype = sz
    L.kfac_experts_gather.argtypes = [vp, sp, vp, vp, i64, vp, i64]
    L.kfac_experts_combine.argtypes = [vp, sp, vp, vp, vp, i64, vp, i64, vp, i64]
    L.kfac_experts_combine_grad.argtypes = [vp, sp, vp, vp, vp, i64, vp, i64, vp, i64, vp]
    L.kfac_grad_norm_batched.argtypes = [vp, i, gp, f, vp, vp, vp]
    L.kfac_grad_norm_workspace_bytes.argtypes = [i, gp]
    L.kfac_grad_norm_workspace_bytes.restype = sz
    L.kfac_clip_grads_batched.argtypes = [vp, i, gp, f, vp, vp, vp]
    L.kfac_profile_begin.argtypes = [vp]
    L.kfac_profile_end.argtypes = [vp, ctypes.POINTER(kfac_kernel_stat), i, ip]
    for name in EXPORTS:
        if name not in ("kfac_workspace_bytes", "kfac_eig_workspace_bytes", "kfac_strerror",
                        "kfac_precondition_workspace_bytes", "kfac_update_factors_workspace_bytes",
                        "kfac_unfold_workspace_bytes", "kfac_static_scratch_bytes", "kfac_invert_workspace_bytes",
                        "kfac_precondition_inverse_workspace_bytes", "kfac_experts_workspace_bytes",
                        "kfac_experts_dispatch_workspace_bytes", "kfac_grad_norm_workspace_bytes"):
            getattr(L, name).restype = i
    _lib = L
    return L


def _ptr(t):
    """Device address of a torch tensor (must be contiguous) or a raw integer address."""
    if t is None:
        return None
    if isinstance(t, int):
        return t
    if not t.is_contiguous():
        raise ValueError("tensor must be contiguous")
    return t.data_ptr()


_codes = {}              # torch dtype -> kfac_dtype; filled at the first use, so that importing this module does not import torch


def _dtype_code(t):
    dtype = t.dtype
    if dtype not in _codes:
        import torch
        _codes.update({torch.float32: KFAC_F32, torch.bfloat16: KFAC_BF16})
        if dtype not in _codes:
            raise ValueError("unsupported dtype %s" % dtype)
    return _codes[dtype]


def _check(rc, where, allow=()):
    if rc != KFAC_OK and rc not in allow:
        raise KfacError(rc, where)
    return rc


def kfac_strerror(code):
    return lib().kfac_strerror(int(code)).decode()


def kfac_workspace_bytes(max_d, max_batch_factors, max_R):
    return int(lib().kfac_workspace_bytes(int(max_d), int(max_batch_factors), int(max_R)))


def kfac_eig_workspace_bytes(dims):
    arr = (ctypes.c_int * len(dims))(*[int(x) for x in dims])
    return int(lib().kfac_eig_workspace_bytes(len(dims), arr))


def kfac_create(device, stream, workspace, workspace_bytes=None):
    """Returns an opaque context handle.  `stream` is a hipStream_t value (torch: stream.cuda_stream),
    `workspace` a uint8 torch tensor (or address) that must stay alive as long as the context."""
    h = ctypes.c_void_p()
    nbytes = workspace_bytes if workspace_bytes is not None else (workspace.numel() * workspace.element_size()
                                                                  if workspace is not None else 0)
    _check(lib().kfac_create(ctypes.byref(h), int(device), stream or None, _ptr(workspace), nbytes), "kfac_create")
    return h


def kfac_destroy(ctx):
    _check(lib().kfac_destroy(ctx), "kfac_destroy")


def kfac_unfold(ctx, x, kh, kw, stride, pad, patches):
    """x [N,C,H,W] -> patches [N, C*kh*kw, Ho*Wo] (same dtype)."""
    N, C, H, W = x.shape
    sh, sw = (stride, stride) if isinstance(stride, int) else stride
    ph, pw = (pad, pad) if isinstance(pad, int) else pad
    d = kfac_conv_desc(N, C, H, W, kh, kw, sh, sw, ph, pw, _dtype_code(x))
    _check(lib().kfac_unfold(ctx, ctypes.byref(d), _ptr(x), _ptr(patches)), "kfac_unfold")


def kfac_unfold_batched(ctx, xs, convs, patches):
    """xs: list of [N,C,H,W] device tensors; convs: list of (kh, kw, stride, pad); patches: list of outputs."""
    n = len(xs)
    descs = (kfac_conv_desc * n)()
    for j, (x, (kh, kw, stride, pad)) in enumerate(zip(xs, convs)):
        N, C, H, W = x.shape
        sh, sw = (stride, stride) if isinstance(stride, int) else stride
        ph, pw = (pad, pad) if isinstance(pad, int) else pad
        descs[j] = kfac_conv_desc(N, C, H, W, kh, kw, sh, sw, ph, pw, _dtype_code(x))
    xp = (ctypes.c_void_p * n)(*[_ptr(x) for x in xs])
    pp = (ctypes.c_void_p * n)(*[_ptr(p) for p in patches])
    _check(lib().kfac_unfold_batched(ctx, n, descs, xp, pp), "kfac_unfold_batched")


def kfac_unfold_workspace_bytes(n):
    return int(lib().kfac_unfold_workspace_bytes(int(n)))


def kfac_update_factors(ctx, X, layout, N, d, T, append_ones, scale, decay, F, dtype=None):
    code = _dtype_code(X) if dtype is None else dtype
    _check(lib().kfac_update_factors(ctx, _ptr(X), code, int(layout), int(N), int(d), int(T), int(append_ones),
                                     float(scale), float(decay), _ptr(F)), "kfac_update_factors")


def kfac_update_factors_static(ctx, X, layout, N, d, T, append_ones, scale, decay, F, dtype=None):
    """kfac_update_factors with its scratch in the library's static device array (allocates nothing)."""
    code = _dtype_code(X) if dtype is None else dtype
    _check(lib().kfac_update_factors_static(ctx, _ptr(X), code, int(layout), int(N), int(d), int(T), int(append_ones),
                                            float(scale), float(decay), _ptr(F)), "kfac_update_factors_static")


def kfac_static_scratch_bytes():
    return int(lib().kfac_static_scratch_bytes())


def _factor_items(items):
    """items: list of dicts with the arguments of kfac_update_factors (X and F may be None for sizing)."""
    arr = (kfac_factor_item * len(items))()
    for j, it in enumerate(items):
        X, F = it.get("X"), it.get("F")
        code = it.get("dtype")
        if code is None:
            code = _dtype_code(X) if X is not None else KFAC_F32
        arr[j] = kfac_factor_item(_ptr(X), int(code), int(it["layout"]), int(it["N"]), int(it["d"]), int(it["T"]),
                                  int(it["append_ones"]), float(it.get("scale", 1.0)), float(it.get("decay", 0.0)), _ptr(F))
    return arr


def factor_items(items):
    """The marshalled item array of a batch of factor updates (see precond_items)."""
    return _factor_items(items)


def kfac_update_factors_batched(ctx, items):
    """items: list of dicts(X, layout, N, d, T, append_ones, scale, decay, F[, dtype]), or the array that
    factor_items() made of such a list; all updated in one call."""
    arr = _factor_items(items) if isinstance(items, list) else items
    _check(lib().kfac_update_factors_batched(ctx, len(arr), arr), "kfac_update_factors_batched")


def kfac_update_factors_workspace_bytes(items):
    return int(lib().kfac_update_factors_workspace_bytes(len(items), _factor_items(items)))


def kfac_eig(ctx, F, Q, lam, max_sweeps=0, tol=0.0, raise_on_noconv=True, fp32_only=False, warm_start=False):
    """F, Q, lam: lists of device tensors.  Returns a list of (sweeps, off_norm_rel, converged)."""
    n = len(F)
    vp = ctypes.c_void_p
    Fa = (vp * n)(*[_ptr(t) for t in F])
    Qa = (vp * n)(*[_ptr(t) for t in Q])
    La = (vp * n)(*[_ptr(t) for t in lam])
    dims = (ctypes.c_int * n)(*[int(t.shape[0]) for t in F])
    opts = kfac_eig_opts(int(max_sweeps), float(tol), int(bool(fp32_only)), int(bool(warm_start)))
    info = (kfac_eig_info * n)()
    rc = lib().kfac_eig(ctx, n, Fa, dims, Qa, La, ctypes.byref(opts), info)
    _check(rc, "kfac_eig", allow=() if raise_on_noconv else (KFAC_ENOCONV,))
    return [(info[i].sweeps, info[i].off_norm_rel, bool(info[i].converged)) for i in range(n)]


def kfac_invert_factors(ctx, F, damping, Finv):
    """F, Finv: lists of device tensors; Finv[b] <- (F[b] + damping I)^-1."""
    n = len(F)
    vp = ctypes.c_void_p
    Fa = (vp * n)(*[_ptr(t) for t in F])
    Ia = (vp * n)(*[_ptr(t) for t in Finv])
    dims = (ctypes.c_int * n)(*[int(t.shape[0]) for t in F])
    _check(lib().kfac_invert_factors(ctx, n, Fa, dims, float(damping), Ia), "kfac_invert_factors")


def kfac_invert_workspace_bytes(dims):
    n = len(dims)
    return int(lib().kfac_invert_workspace_bytes(n, (ctypes.c_int * n)(*[int(v) for v in dims])))


def kfac_precondition_inverse(ctx, Ainv, Ginv, grad):
    dA, dG = int(Ainv.shape[0]), int(Ginv.shape[0])
    if tuple(grad.shape) != (dG, dA):
        raise ValueError("grad must be [dG, dA]")
    _check(lib().kfac_precondition_inverse(ctx, _ptr(Ainv), dA, _ptr(Ginv), dG, _ptr(grad), _dtype_code(grad)),
           "kfac_precondition_inverse")


def precond_inv_items(Ainv, Ginv, grad):
    """Marshalled array of kfac_precond_inv_item for lists of device tensors (reusable across calls)."""
    n = len(grad)
    arr = (kfac_precond_inv_item * n)()
    for j in range(n):
        dA, dG = int(Ainv[j].shape[0]), int(Ginv[j].shape[0])
        if tuple(grad[j].shape) != (dG, dA):
            raise ValueError("grad[%d] must be [dG, dA]" % j)
        arr[j] = kfac_precond_inv_item(_ptr(Ainv[j]), dA, _ptr(Ginv[j]), dG, _ptr(grad[j]), _dtype_code(grad[j]))
    return arr


def kfac_precondition_inverse_batched(ctx, Ainv=None, Ginv=None, grad=None, items=None):
    arr = items if items is not None else precond_inv_items(Ainv, Ginv, grad)
    _check(lib().kfac_precondition_inverse_batched(ctx, len(arr), arr), "kfac_precondition_inverse_batched")


def kfac_precondition(ctx, QA, lamA, QG, lamG, damping, grad):
    dA, dG = int(QA.shape[0]), int(QG.shape[0])
    if tuple(grad.shape) != (dG, dA):
        raise ValueError("grad must be [dG, dA]")
    _check(lib().kfac_precondition(ctx, _ptr(QA), _ptr(lamA), dA, _ptr(QG), _ptr(lamG), dG, float(damping),
                                   _ptr(grad), _dtype_code(grad)), "kfac_precondition")


def _precond_items(QA, lamA, QG, lamG, damping, grad, factored_damping=False, split_f16=False):
    n = len(grad)
    arr = (kfac_precond_item * n)()
    for j in range(n):
        dA, dG = int(QA[j].shape[0]), int(QG[j].shape[0])
        if tuple(grad[j].shape) != (dG, dA):
            raise ValueError("grad[%d] must be [dG, dA]" % j)
        arr[j] = kfac_precond_item(_ptr(QA[j]), _ptr(lamA[j]), dA, _ptr(QG[j]), _ptr(lamG[j]), dG, float(damping),
                                   _ptr(grad[j]), _dtype_code(grad[j]), int(bool(factored_damping)), int(bool(split_f16)))
    return arr


def precond_items(QA, lamA, QG, lamG, damping, grad, factored_damping=False, split_f16=False):
    """The marshalled item array of a batch, for callers that precondition the same buffers every iteration and
    want to marshal them once: pass it as `items=` to the batched calls below."""
    return _precond_items(QA, lamA, QG, lamG, damping, grad, factored_damping, split_f16)


def kfac_precondition_batched(ctx, QA=None, lamA=None, QG=None, lamG=None, damping=None, grad=None, factored_damping=False,
                              split_f16=False, items=None):
    """Lists of per-layer device tensors (or a marshalled `items` array); every grad[j] is preconditioned in
    place.  factored_damping: the explicit-inverse method (G + damping I)^-1 grad (A + damping I)^-1 instead
    of the eigenbasis step.  split_f16: run the GEMM chain on the split-fp16 engine."""
    arr = items if items is not None else _precond_items(QA, lamA, QG, lamG, damping, grad, factored_damping, split_f16)
    _check(lib().kfac_precondition_batched(ctx, len(arr), arr), "kfac_precondition_batched")


def kfac_precondition_batched_scaled(ctx, QA=None, lamA=None, QG=None, lamG=None, damping=None, grad=None, kappa=None, lr=None,
                                     nu=None, split_f16=False, items=None):
    """As kfac_precondition_batched, then every gradient is multiplied by the nu of Sec. V-C; nu: device tensor
    of one float32, written by the call."""
    arr = items if items is not None else _precond_items(QA, lamA, QG, lamG, damping, grad, split_f16=split_f16)
    _check(lib().kfac_precondition_batched_scaled(ctx, len(arr), arr, float(kappa), float(lr), _ptr(nu)),
           "kfac_precondition_batched_scaled")


def kfac_precondition_workspace_bytes(dims):
    """dims: list of (dA, dG)."""
    arr = (kfac_precond_item * len(dims))()
    for j, (dA, dG) in enumerate(dims):
        arr[j].dA, arr[j].dG = int(dA), int(dG)
    return int(lib().kfac_precondition_workspace_bytes(len(dims), arr))


# ---- layers of experts ----
def _on_gpu(*tensors):
    """The last thing that is looked at: a host address would be read by a kernel."""
    for t in tensors:
        if t is not None and not t.is_cuda:
            raise ValueError("tensors must be on the GPU")


def _c_int(n):
    """A count as a C int: one that no C int holds (ctypes would cut it to its lower 32 bits) becomes -1, which the library refuses."""
    return n if -(1 << 31) <= n < 1 << 31 else -1


def _rows(t, name, d):
    """(address, row pitch) of a matrix of samples [R][d]: any pitch, but the elements of a row side by side."""
    shape = t.shape
    if len(shape) != 2 or shape[1] != d:
        raise ValueError("%s must be [R, %d]" % (name, d))
    if shape[0] == 0:
        return None, d
    ld, step = t.stride()
    if d > 1 and step != 1:
        raise ValueError("the rows of %s must be contiguous" % name)
    if shape[0] == 1:
        ld = d
    if ld < d:
        raise ValueError("the rows of %s overlap" % name)
    return t.data_ptr(), ld


def _offsets(t, experts):
    import torch
    if t.dtype != torch.int32 or t.dim() != 1 or t.shape[0] != experts + 1:
        raise ValueError("offsets must be int32 [experts + 1]")
    if not t.is_contiguous():
        raise ValueError("offsets must be contiguous")
    return t


def _expert_desc(weight, offsets, rows, append_ones, dtype):
    """weight: [experts, d_out, d_in + append_ones] (the weights or their gradient), rows: the number of sample rows."""
    experts, d_out, wide = weight.shape
    ones = int(bool(append_ones))
    if wide - ones < 1:
        raise ValueError("weights without inputs")
    _ptr(weight)                                 # contiguous
    _offsets(offsets, experts)
    return kfac_expert_desc(_c_int(experts), _c_int(rows), _c_int(wide - ones), _c_int(d_out), ones, dtype, offsets.data_ptr())


def _same(a, b, names):
    if a.dtype != b.dtype:
        raise ValueError("%s must have one dtype" % names)


def kfac_experts_workspace_bytes(experts, rows, d_in, d_out, append_ones=False, dtype=KFAC_BF16):
    """Bytes of workspace that the products and factors of such a layer make use of (they work with less)."""
    d = kfac_expert_desc(*(_c_int(int(n)) for n in (experts, rows, d_in, d_out)), int(bool(append_ones)), int(dtype), None)
    return int(lib().kfac_experts_workspace_bytes(ctypes.byref(d)))


def kfac_experts_forward(ctx, X, W, offsets, Y, append_ones=False):
    """Y[r] = X[r] W_e^T (+ the last column of W_e).  X [R, d_in], W [experts, d_out, d_in + append_ones], Y [R, d_out] (both with any row
    pitch), offsets int32 [experts + 1] on the GPU."""
    desc = _expert_desc(W, offsets, X.shape[0], append_ones, _dtype_code(X))
    _same(X, W, "X and W")
    _same(X, Y, "X and Y")
    if Y.shape[0] != X.shape[0]:
        raise ValueError("X and Y must have as many rows")
    xp, ldx = _rows(X, "X", desc.d_in)
    yp, ldy = _rows(Y, "Y", desc.d_out)
    _on_gpu(X, W, offsets, Y)
    _check(lib().kfac_experts_forward(ctx, ctypes.byref(desc), xp, ldx, _ptr(W), yp, ldy), "kfac_experts_forward")


def kfac_experts_input_grad(ctx, G, W, offsets, dX, append_ones=False):
    """dX[r] = G[r] W_e, without the bias column.  G [R, d_out], dX [R, d_in]."""
    desc = _expert_desc(W, offsets, G.shape[0], append_ones, _dtype_code(G))
    _same(G, W, "G and W")
    _same(G, dX, "G and dX")
    if dX.shape[0] != G.shape[0]:
        raise ValueError("G and dX must have as many rows")
    gp, ldg = _rows(G, "G", desc.d_out)
    xp, ldx = _rows(dX, "dX", desc.d_in)
    _on_gpu(G, W, offsets, dX)
    _check(lib().kfac_experts_input_grad(ctx, ctypes.byref(desc), gp, ldg, _ptr(W), xp, ldx), "kfac_experts_input_grad")


def kfac_experts_weight_grad(ctx, G, X, offsets, dW, append_ones=False, accumulate=False):
    """dW_e = sum over the rows of e of G[r]^T [X[r] | 1 if append_ones] (added to dW with accumulate).  dW [experts, d_out, d_in + append_ones]
    in fp32 or bf16; dW[e] is the gradient that the preconditioner takes."""
    desc = _expert_desc(dW, offsets, G.shape[0], append_ones, _dtype_code(G))
    _same(G, X, "G and X")
    if X.shape[0] != G.shape[0]:
        raise ValueError("G and X must have as many rows")
    gp, ldg = _rows(G, "G", desc.d_out)
    xp, ldx = _rows(X, "X", desc.d_in)
    code = _dtype_code(dW)
    _on_gpu(G, X, offsets, dW)
    _check(lib().kfac_experts_weight_grad(ctx, ctypes.byref(desc), gp, ldg, xp, ldx, int(bool(accumulate)), _ptr(dW), code),
           "kfac_experts_weight_grad")


def kfac_update_factors_experts(ctx, X, offsets, F, append_ones=False, scale=1.0, decay=0.0, mean=True):
    """F_e <- decay F_e + (1 - decay) s_e Xt^T Xt over the rows of e, Xt = [X | 1 if append_ones]; s_e = scale / rows of e (an expert
    without rows keeps its factor), or scale with mean=False.  X [R, d], F [experts, D, D] fp32."""
    import torch
    ones = int(bool(append_ones))
    if F.dim() != 3 or F.dtype != torch.float32 or F.shape[1] != F.shape[2] or F.shape[1] != X.shape[1] + ones:
        raise ValueError("F must be float32 [experts, D, D], D = d + append_ones")
    experts, d = F.shape[0], X.shape[1]
    xp, ldx = _rows(X, "X", d)
    _offsets(offsets, experts)
    _ptr(F)                                      # contiguous
    _on_gpu(X, offsets, F)
    _check(lib().kfac_update_factors_experts(ctx, _c_int(experts), _c_int(X.shape[0]), offsets.data_ptr(), xp, _dtype_code(X), ldx, _c_int(d), ones,
                                             int(bool(mean)), float(scale), float(decay), _ptr(F)), "kfac_update_factors_experts")


# ---- tokens to experts and back ----
# (Calls of a few microseconds: what a tensor is asked for, it is asked once.)
_slot_types = {}         # torch dtype -> whether it is the one of ids and rows


def _slots(t, name, shape=None, ints=True):
    """(address, shape) of a contiguous matrix [tokens, topk] with an int32 or a float32 for each slot."""
    mine = t.shape
    if len(mine) != 2 or (shape is not None and mine != shape):
        raise ValueError("%s must be [tokens, topk]" % name)
    dtype = t.dtype
    if dtype not in _slot_types:
        import torch
        _slot_types.update({torch.int32: True, torch.float32: False})
    if _slot_types.get(dtype) is not ints:      # (None: neither)
        raise ValueError("%s must be %s" % (name, "int32" if ints else "float32"))
    if not t.is_contiguous():
        raise ValueError("%s must be contiguous" % name)
    return t.data_ptr(), mine


def _matrix(t, name, dtype, rows=None, width=None):
    """(address, row pitch, rows, columns) of a matrix of samples: any pitch, but the elements of a row side by side."""
    shape = t.shape
    n, d = shape if len(shape) == 2 else (-1, -1)
    if d < 0 or (rows is not None and n != rows) or (width is not None and d != width):
        raise ValueError("%s must be [%s, %s]" % (name, "R" if rows is None else rows, "d" if width is None else width))
    if t.dtype != dtype:
        raise ValueError("%s must be %s as the others" % (name, dtype))
    if n == 0:
        return None, d, n, d
    ld, step = t.stride()
    if d > 1 and step != 1:
        raise ValueError("the rows of %s must be contiguous" % name)
    if n == 1:
        ld = d
    if ld < d:
        raise ValueError("the rows of %s overlap" % name)
    return t.data_ptr(), ld, n, d


_MOST = (1 << 31) - 1    # of a C int


def _slot_desc(tokens, topk, rows, width, dtype):
    if tokens > _MOST or topk > _MOST or rows > _MOST or width > _MOST:      # (refused by the library; ctypes would cut it)
        tokens = -1
    return ctypes.byref(kfac_slot_desc(tokens, topk, rows, width, dtype))


def kfac_experts_route(ctx, logits, ids, weights, normalize=False):
    """ids[t] = the experts of the topk largest logits of token t (ties to the lowest index; -1 where only logits of -inf are left), weights[t] their
    softmax over all experts, or with normalize over those chosen.  logits [tokens, experts] (any row pitch), ids int32 and weights float32
    [tokens, topk]: written."""
    code = _dtype_code(logits)
    ip, shape = _slots(ids, "ids")
    wp, _ = _slots(weights, "weights", shape, False)
    lp, ldl, tokens, experts = _matrix(logits, "logits", logits.dtype, shape[0])
    if not (logits.is_cuda and ids.is_cuda and weights.is_cuda):
        _on_gpu(logits, ids, weights)
    _check(lib().kfac_experts_route(ctx, _c_int(tokens), _c_int(experts), _c_int(shape[1]), lp, code, ldl, 1 if normalize else 0, ip, wp), "kfac_experts_route")


def kfac_experts_route_grad(ctx, logits, ids, dweights, dlogits, normalize=False):
    """The gradient of the logits (written to dlogits, of their shape and dtype) from that of the weights; logits, ids and normalize as in
    kfac_experts_route()."""
    code, dtype = _dtype_code(logits), logits.dtype
    ip, shape = _slots(ids, "ids")
    wp, _ = _slots(dweights, "dweights", shape, False)
    lp, ldl, tokens, experts = _matrix(logits, "logits", dtype, shape[0])
    dp, ldd, _, _ = _matrix(dlogits, "dlogits", dtype, tokens, experts)
    if not (logits.is_cuda and ids.is_cuda and dweights.is_cuda and dlogits.is_cuda):
        _on_gpu(logits, ids, dweights, dlogits)
    _check(lib().kfac_experts_route_grad(ctx, _c_int(tokens), _c_int(experts), _c_int(shape[1]), lp, code, ldl, ip, wp, 1 if normalize else 0, dp, ldd),
           "kfac_experts_route_grad")


def kfac_experts_dispatch_workspace_bytes(tokens, topk, experts):
    """Bytes of workspace that sorting so many slots makes use of (it works with less)."""
    return int(lib().kfac_experts_dispatch_workspace_bytes(_c_int(int(tokens)), _c_int(int(topk)), _c_int(int(experts))))


def kfac_experts_dispatch(ctx, ids, X, offsets, rows, Xs):
    """Sorts the slots by expert and copies the tokens there: offsets (int32 [experts + 1]) and Xs [at least tokens * topk, d] are what the products for
    layers of experts take, rows (int32 [tokens, topk]) says where each slot went (-1: it has no expert, its id is outside 0 .. experts - 1).
    X [tokens, d]; ids int32 [tokens, topk].  X = Xs = None: the order alone."""
    ip, shape = _slots(ids, "ids")
    rp, _ = _slots(rows, "rows", shape)
    tokens, topk = shape
    experts = offsets.numel() - 1
    if experts < 1:
        raise ValueError("offsets must be int32 [experts + 1]")
    op = _offsets(offsets, experts).data_ptr()
    if (X is None) != (Xs is None):
        raise ValueError("both X and Xs or none")
    xp = sp = None
    ldx = lds = 0
    if X is None:
        d = _slot_desc(tokens, topk, tokens * topk, 0, KFAC_F32)
    else:
        code, dtype = _dtype_code(X), X.dtype
        xp, ldx, _, width = _matrix(X, "X", dtype, tokens)
        sp, lds, R, _ = _matrix(Xs, "Xs", dtype, None, width)
        if R < tokens * topk:
            raise ValueError("Xs must have a row for each slot")
        d = _slot_desc(tokens, topk, R, width, code)
    if not (ids.is_cuda and offsets.is_cuda and rows.is_cuda and (X is None or (X.is_cuda and Xs.is_cuda))):
        _on_gpu(ids, X, offsets, rows, Xs)
    _check(lib().kfac_experts_dispatch(ctx, d, _c_int(experts), ip, xp, ldx, op, rp, sp, lds), "kfac_experts_dispatch")


def kfac_experts_gather(ctx, rows, X, Xs):
    """Xs[rows[t, j]] = X[t], rows as kfac_experts_dispatch() left them."""
    rp, (tokens, topk) = _slots(rows, "rows")
    code, dtype = _dtype_code(X), X.dtype
    xp, ldx, _, width = _matrix(X, "X", dtype, tokens)
    sp, lds, R, _ = _matrix(Xs, "Xs", dtype, None, width)
    _on_gpu(rows, X, Xs)
    _check(lib().kfac_experts_gather(ctx, _slot_desc(tokens, topk, R, width, code), rp, xp, ldx, sp, lds), "kfac_experts_gather")


def kfac_experts_combine(ctx, Ys, rows, weights, Y, add=None):
    """Y[t] = add[t] + sum over j of weights[t, j] Ys[rows[t, j]].  Ys [R, d], rows int32 [tokens, topk], weights float32 [tokens, topk] or None (ones: the
    gradient of kfac_experts_dispatch()), Y [tokens, d], add [tokens, d] or None, or Y itself."""
    rp, shape = _slots(rows, "rows")
    wp = None if weights is None else _slots(weights, "weights", shape, False)[0]
    tokens, topk = shape
    code, dtype = _dtype_code(Y), Y.dtype
    yp, ldy, _, width = _matrix(Y, "Y", dtype, tokens)
    sp, lds, R, _ = _matrix(Ys, "Ys", dtype, None, width)
    ap, lda, _, _ = (None, 0, 0, 0) if add is None else _matrix(add, "add", dtype, tokens, width)
    if not (Ys.is_cuda and rows.is_cuda and Y.is_cuda and (weights is None or weights.is_cuda) and (add is None or add.is_cuda)):
        _on_gpu(Ys, rows, weights, Y, add)
    _check(lib().kfac_experts_combine(ctx, _slot_desc(tokens, topk, R, width, code), rp, wp, sp, lds, ap, lda, yp, ldy), "kfac_experts_combine")


def kfac_experts_combine_grad(ctx, dY, Ys, rows, weights, dYs, dweights):
    """dYs[rows[t, j]] = weights[t, j] dY[t] and dweights[t, j] = <dY[t], Ys[rows[t, j]]>: the gradients of kfac_experts_combine().  dY [tokens, d], Ys and dYs
    [R, d], weights and dweights float32 [tokens, topk]."""
    rp, shape = _slots(rows, "rows")
    wp, _ = _slots(weights, "weights", shape, False)
    gp, _ = _slots(dweights, "dweights", shape, False)
    tokens, topk = shape
    code, dtype = _dtype_code(dY), dY.dtype
    yp, ldy, _, width = _matrix(dY, "dY", dtype, tokens)
    sp, lds, R, _ = _matrix(Ys, "Ys", dtype, None, width)
    op, ldo, _, _ = _matrix(dYs, "dYs", dtype, R, width)
    if not (dY.is_cuda and Ys.is_cuda and rows.is_cuda and weights.is_cuda and dYs.is_cuda and dweights.is_cuda):
        _on_gpu(dY, Ys, rows, weights, dYs, dweights)
    _check(lib().kfac_experts_combine_grad(ctx, _slot_desc(tokens, topk, R, width, code), rp, wp, yp, ldy, sp, lds, op, ldo, gp), "kfac_experts_combine_grad")


# ---- the global gradient norm ----
def grad_items(grads, out=None):
    """The marshalled item array of kfac_grad_norm_batched() and kfac_clip_grads_batched() for a list of device tensors (float32 or bfloat16, contiguous), reusable
    while they live.  out: for clipping, a list of as many tensors of the same sizes that take the clipped gradients, each the gradient
    itself or a buffer of its own."""
    if out is not None and len(out) != len(grads):
        raise ValueError("as many outputs as gradients")
    arr = (kfac_grad_item * len(grads))()
    written, read = set(), {}
    for j, (d, g) in enumerate(zip(arr, grads)):
        d.grad, d.grad_dtype, d.n = _ptr(g), _dtype_code(g), g.numel()
        o = None if out is None else out[j]
        if o is not None:
            if o.numel() != d.n:
                raise ValueError("buffers of different lengths")
            d.out, d.out_dtype = _ptr(o), _dtype_code(o)
            if d.n > 0:
                if d.out in written:
                    raise ValueError("an output occurs twice")
                written.add(d.out)
                if d.out == d.grad and d.out_dtype != d.grad_dtype:
                    raise ValueError("a gradient can only be clipped in place in its own dtype")
        _on_gpu(g, o)
        if d.n > 0:
            read.setdefault(d.grad, []).append(d.out)
    # a gradient that is written must be read by its own item alone
    for a, outs in read.items():
        if a in written and (len(outs) > 1 or outs[0] != a):
            raise ValueError("an output is another tensor's gradient")
    return arr


def kfac_grad_norm_workspace_bytes(items):
    """items: the array that grad_items() made."""
    return int(lib().kfac_grad_norm_workspace_bytes(len(items), items))


def kfac_grad_norm_batched(ctx, items, norm, max_norm=None, grad_scale=None, coef=None):
    """norm = |s| times the root of the sum of all gradients' squares, coef = s min(1, max_norm / norm) (None: s), s = grad_scale (None: 1).  items: a list of
    gradients, or the array of grad_items(); norm, coef, grad_scale: device tensors of one float32.  coef is what kfac_adamw_batched() takes as
    grad_scale."""
    import torch
    arr = grad_items(items) if isinstance(items, list) else items
    _check(lib().kfac_grad_norm_batched(ctx, len(arr), arr, float("inf") if max_norm is None else float(max_norm), _scalar(grad_scale, torch.float32, "grad_scale"),
                                        _scalar(norm, torch.float32, "norm"), _scalar(coef, torch.float32, "coef")), "kfac_grad_norm_batched")


def kfac_clip_grads_batched(ctx, items, max_norm, norm, coef, grad_scale=None):
    """As kfac_grad_norm_batched(), then every gradient times coef goes to its output (see grad_items()); a list of gradients is clipped in place."""
    import torch
    arr = grad_items(items, items) if isinstance(items, list) else items
    _check(lib().kfac_clip_grads_batched(ctx, len(arr), arr, float(max_norm), _scalar(grad_scale, torch.float32, "grad_scale"), _scalar(norm, torch.float32, "norm"),
                                         _scalar(coef, torch.float32, "coef")), "kfac_clip_grads_batched")


# ---- the optimizer step ----
def adamw_items(items):
    """The marshalled item array of kfac_adamw_batched for a list of dicts(param, grad, m, v[, m_scale, v_scale][, copy]) of device tensors,
    reusable while the buffers live; none that is written may occur twice.  Marshalling takes 4 to 6 us of Python a tensor, for a network's list more
    than the step itself: a training loop keeps the gradients' buffers, marshals once and hands over the array.  State in 32 bits: m, v float32.  State in 8 bits: m, v float8_e4m3fn (or
    uint8), m_scale, v_scale uint8, one for each 128 elements.  copy: bfloat16, takes the updated parameter."""
    import torch
    code = {torch.float32: KFAC_F32, torch.bfloat16: KFAC_BF16}
    codes = (torch.uint8, torch.float8_e4m3fn)
    arr = (kfac_adamw_item * len(items))()
    written = set()
    for d, it in zip(arr, items):
        p, g, m, v = it["param"], it["grad"], it["m"], it["v"]
        ms, vs, copy = it.get("m_scale"), it.get("v_scale"), it.get("copy")
        n = p.numel()
        if g.numel() != n or m.numel() != n or v.numel() != n or (copy is not None and copy.numel() != n):
            raise ValueError("buffers of different lengths")
        if (ms is None) != (vs is None):
            raise ValueError("both scales or none")
        if ms is None:
            if m.dtype != torch.float32 or v.dtype != torch.float32:
                raise ValueError("m and v must be float32 (or come with scales)")
        else:
            blocks = (n + 127) // 128
            if m.dtype not in codes or v.dtype not in codes or any(s.dtype != torch.uint8 or s.numel() != blocks for s in (ms, vs)):
                raise ValueError("m and v must be float8_e4m3fn or uint8, the scales uint8, one for each 128")
            d.m_scale, d.v_scale = _ptr(ms), _ptr(vs)
        if copy is not None:
            if copy.dtype != torch.bfloat16:
                raise ValueError("copy must be bfloat16")
            d.copy = _ptr(copy)
        try:
            d.param_dtype, d.grad_dtype = code[p.dtype], code[g.dtype]
        except KeyError:
            raise ValueError("parameters and gradients must be float32 or bfloat16") from None
        d.param, d.grad, d.m, d.v, d.n = _ptr(p), _ptr(g), _ptr(m), _ptr(v), n
        _on_gpu(p, g, m, v, ms, vs, copy)
        mine = [t for t in (d.param, d.m, d.v, d.m_scale, d.v_scale, d.copy) if t] if n > 0 else []
        if len(set(mine)) < len(mine) or not written.isdisjoint(mine):      # (it would be updated from two sides at once)
            raise ValueError("a buffer occurs twice")
        written.update(mine)
    return arr


def _scalar(t, dtype, name):
    if t is None:
        return None
    if t.dtype != dtype or t.numel() != 1:
        raise ValueError("%s must be one %s" % (name, dtype))
    _on_gpu(t)
    return t.data_ptr()


_told = False


def _tell(arr, step):
    """Says once that a run with 8-bit state has no seed.  (The first steps to nearest do no harm: ExpertRunner.)"""
    global _told
    if len(arr) > 0 and arr[0].m_scale and (step is None or step > 8):
        _told = True
        warnings.warn("8-bit AdamW state is rounded to nearest without a seed and does not follow its moments over a run: give kfac_adamw_batched() a seed",
                      RuntimeWarning, stacklevel=3)


def kfac_adamw_batched(ctx, items, lr, beta1=0.9, beta2=0.999, eps=1e-8, weight_decay=0.01, step=1, grad_scale=None, seed=0):
    """One AdamW step over a list of tensors (see adamw_items()).  lr and step: numbers, or device tensors of one float32 / int64 that the call
    reads on the GPU; grad_scale: None or a device tensor of one float32 that every gradient is multiplied with.
    seed (1 .. 2^64 - 1): training with 8-bit state needs one, together with a step that counts on.  Codes are then rounded up or down
    at random, so that the state follows its moments; with 0 they are rounded half to even, which loses most steps of a run (and is warned of
    once, from the ninth step on)."""
    import torch
    if not 0 <= int(seed) < 1 << 64:
        raise ValueError("seed must be 0 .. 2^64 - 1")
    arr = adamw_items(items) if isinstance(items, list) else items
    lr_dev = _scalar(lr, torch.float32, "lr") if torch.is_tensor(lr) else None
    step_dev = _scalar(step, torch.int64, "step") if torch.is_tensor(step) else None
    if not (seed or _told):
        _tell(arr, None if step_dev else step)
    o = kfac_adamw_opts(float(beta1), float(beta2), 0.0 if lr_dev else float(lr), float(eps), float(weight_decay), 1 if step_dev else int(step),
                        _scalar(grad_scale, torch.float32, "grad_scale"), lr_dev, step_dev, int(seed))
    _check(lib().kfac_adamw_batched(ctx, len(arr), arr, ctypes.byref(o)), "kfac_adamw_batched")


def kfac_adamw_state_values(ctx, codes, scale, out):
    """out[i] = codes[i] * 2^(scale[i // 128] - 127): what an 8-bit state stands for (m, and sqrt(v)), in float32 or
    bfloat16 (exact there for scales from 3 on; smaller ones have codes below bfloat16's smallest number)."""
    import torch
    n = codes.numel()
    if codes.dtype not in (torch.uint8, torch.float8_e4m3fn) or out.numel() != n or scale.dtype != torch.uint8 or scale.numel() != (n + 127) // 128:
        raise ValueError("codes: float8_e4m3fn or uint8, as many as out, scale: uint8, one for each 128")
    code = _dtype_code(out)
    _on_gpu(codes, scale, out)
    _check(lib().kfac_adamw_state_values(ctx, _ptr(codes), _ptr(scale), n, _ptr(out), code), "kfac_adamw_state_values")


def kfac_schedule_due(k, f_fac, f_eig):
    a, b = ctypes.c_int(0), ctypes.c_int(0)
    _check(lib().kfac_schedule_due(int(k), int(f_fac), int(f_eig), ctypes.byref(a), ctypes.byref(b)),
           "kfac_schedule_due")
    return bool(a.value), bool(b.value)


def kfac_profile_begin(ctx):
    _check(lib().kfac_profile_begin(ctx), "kfac_profile_begin")


def kfac_profile_end(ctx):
    """Returns {kernel class: dict(launches, ms, flops, bytes)} for the launches since kfac_profile_begin."""
    out = (kfac_kernel_stat * 64)()     # more than there are kernel classes
    n = ctypes.c_int(0)
    _check(lib().kfac_profile_end(ctx, out, len(out), ctypes.byref(n)), "kfac_profile_end")
    return {out[i].name.decode(): dict(launches=out[i].launches, ms=out[i].ms, flops=out[i].flops, bytes=out[i].bytes)
            for i in range(n.value)}
