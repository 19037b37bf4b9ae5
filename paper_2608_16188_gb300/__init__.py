"""Python binding of libvmoe: one adaptation step of T concurrent V-MoE expert layers on GB300.

Argument marshalling only.  Every step of the path runs in the CUDA kernels of
``libvmoe.so`` (built in-tree by ``_build.build()``); there is no Python, PyTorch
or CPU fallback, and importing a function whose library is missing raises.

The functions carry the C names (``vmoe_route``, ``vmoe_dispatch``,
``vmoe_expert_fwd``, ``vmoe_expert_bwd``, ``vmoe_combine``) and take torch tensors
(device memory, any dtype matching the problem) or raw integer device pointers;
those around the layer (``vmoe_balance``, ``vmoe_block_norm``, ``vmoe_adamw`` and their
backwards) check a tensor's dtype, size, strides and device first;
``stream`` is a ``torch.cuda.Stream``, a raw ``cudaStream_t`` integer, or None for
the current torch stream.  A non-zero status raises ``VmoeError``.
"""
from __future__ import annotations

import ctypes
import os

PKG = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.environ.get("VMOE_LIBRARY", os.path.join(PKG, "libvmoe.so"))

VMOE_OK = 0
VMOE_ERR_INVALID = -1
VMOE_ERR_UNSUPPORTED = -2
VMOE_ERR_CUDA = -3
VMOE_ERR_DEVICE_TIMEOUT = -4

VMOE_F32 = 0
VMOE_BF16 = 1

VMOE_LOGITS_IN = 1 << 0
VMOE_NO_RENORM = 1 << 1
VMOE_GELU_TANH = 1 << 2
VMOE_DLOGITS_ADD = 1 << 3

VMOE_NORM_RMS = 1 << 0
VMOE_NORM_POST = 1 << 1

VMOE_STATE_F32 = 0
VMOE_STATE_E4M3 = 1

# Every symbol include/vmoe.h declares.
EXPORTS = ("vmoe_version", "vmoe_status_string", "vmoe_problem_capacity", "vmoe_route",
           "vmoe_dispatch", "vmoe_expert_fwd", "vmoe_expert_bwd_workspace_size",
           "vmoe_expert_bwd_min_workspace_size",
           "vmoe_expert_bwd", "vmoe_expert_bwd_static_scratch", "vmoe_combine", "vmoe_router_bwd", "vmoe_plan_slices", "vmoe_plan_shares",
           "vmoe_attn_expert_fwd", "vmoe_attn_expert_bwd", "vmoe_attn_expert_bwd_workspace_size",
           "vmoe_balance", "vmoe_balance_workspace_size", "vmoe_balance_bwd", "vmoe_block_norm", "vmoe_block_norm_bwd",
           "vmoe_block_norm_bwd_workspace_size", "vmoe_adamw",
           "vmoe_device_status", "vmoe_selftest_bounded_wait", "vmoe_trace_enable",
           "vmoe_trace_disable", "vmoe_trace_get")


class VmoeError(RuntimeError):
    def __init__(self, status: int, where: str):
        self.status = status
        super().__init__("%s: %s" % (where, status_string(status)))


class VmoeProblem(ctypes.Structure):
    """Mirror of ``vmoe_problem`` in include/vmoe.h."""
    _fields_ = [("T", ctypes.c_int32), ("N", ctypes.c_int32), ("d_model", ctypes.c_int32),
                ("d_ff", ctypes.c_int32), ("E", ctypes.c_int32), ("k", ctypes.c_int32),
                ("capacity_factor", ctypes.c_double), ("capacity", ctypes.c_int32),
                ("dtype", ctypes.c_int32), ("flags", ctypes.c_uint32)]


class VmoeNorm(ctypes.Structure):
    """Mirror of ``vmoe_norm`` in include/vmoe.h."""
    _fields_ = [("eps", ctypes.c_float), ("residual_scale", ctypes.c_float), ("flags", ctypes.c_uint32)]


class VmoeAdamwTensor(ctypes.Structure):
    """Mirror of ``vmoe_adamw_tensor`` in include/vmoe.h."""
    _fields_ = [("param", ctypes.c_void_p), ("grad", ctypes.c_void_p), ("m", ctypes.c_void_p),
                ("v", ctypes.c_void_p), ("m_scale", ctypes.c_void_p), ("v_scale", ctypes.c_void_p),
                ("master", ctypes.c_void_p), ("numel", ctypes.c_int64), ("param_dtype", ctypes.c_int32),
                ("grad_dtype", ctypes.c_int32), ("state", ctypes.c_int32), ("lr_scale", ctypes.c_float),
                ("weight_decay", ctypes.c_float)]


class VmoeAdamwConfig(ctypes.Structure):
    """Mirror of ``vmoe_adamw_config`` in include/vmoe.h."""
    _fields_ = [("lr", ctypes.c_double), ("beta1", ctypes.c_double), ("beta2", ctypes.c_double),
                ("eps", ctypes.c_double), ("step", ctypes.c_int32), ("seed", ctypes.c_uint32),
                ("step_dev", ctypes.c_void_p), ("lr_dev", ctypes.c_void_p), ("grad_scale", ctypes.c_void_p)]


_lib = None
_P = ctypes.c_void_p


def library():
    """The loaded libvmoe (ctypes.CDLL).  Raises if it has not been built."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise RuntimeError(
                "libvmoe.so not found at %s: build it first with "
                "`python -c 'import __graft_entry__ as g; g.build()'`" % LIB_PATH)
        lib = ctypes.CDLL(LIB_PATH)
        PP = ctypes.POINTER(VmoeProblem)
        sig = {
            "vmoe_version": (ctypes.c_int, []),
            "vmoe_status_string": (ctypes.c_char_p, [ctypes.c_int]),
            "vmoe_problem_capacity": (ctypes.c_int, [PP]),
            "vmoe_route": (ctypes.c_int, [PP] + [_P] * 8 + [_P]),
            "vmoe_dispatch": (ctypes.c_int, [PP] + [_P] * 6 + [_P]),
            "vmoe_expert_fwd": (ctypes.c_int, [PP] + [_P] * 7 + [_P]),
            "vmoe_expert_bwd_workspace_size": (ctypes.c_size_t, [PP]),
            "vmoe_expert_bwd_min_workspace_size": (ctypes.c_size_t, [PP]),
            "vmoe_expert_bwd": (ctypes.c_int, [PP] + [_P] * 11 + [ctypes.c_size_t, _P]),
            "vmoe_expert_bwd_static_scratch": (ctypes.c_int, [PP] + [_P] * 10 + [_P]),
            "vmoe_combine": (ctypes.c_int, [PP] + [_P] * 5 + [_P]),
            "vmoe_router_bwd": (ctypes.c_int, [PP] + [_P] * 13 + [_P]),
            "vmoe_attn_expert_fwd": (ctypes.c_int, [PP, ctypes.c_int] + [_P] * 9),
            "vmoe_attn_expert_bwd_workspace_size": (ctypes.c_size_t, [PP, ctypes.c_int]),
            "vmoe_attn_expert_bwd": (ctypes.c_int, [PP, ctypes.c_int] + [_P] * 12 + [ctypes.c_size_t, _P]),
            "vmoe_balance_workspace_size": (ctypes.c_size_t, [PP]),
            "vmoe_balance": (ctypes.c_int, [PP] + [_P] * 8 + [ctypes.c_size_t, _P]),
            "vmoe_balance_bwd": (ctypes.c_int, [PP] + [_P] * 8),
            "vmoe_block_norm": (ctypes.c_int, [PP, ctypes.POINTER(VmoeNorm)] + [_P] * 12),
            "vmoe_block_norm_bwd_workspace_size": (ctypes.c_size_t, [PP]),
            "vmoe_block_norm_bwd": (ctypes.c_int, [PP, ctypes.POINTER(VmoeNorm)] + [_P] * 18 + [ctypes.c_size_t, _P]),
            "vmoe_adamw": (ctypes.c_int, [ctypes.c_int, _P, ctypes.POINTER(VmoeAdamwConfig), _P]),
            "vmoe_plan_slices": (ctypes.c_int, [ctypes.c_int, _P, _P, ctypes.c_int64,
                                                ctypes.c_double, ctypes.c_double, _P, _P]),
            "vmoe_plan_shares": (ctypes.c_int, [ctypes.c_int, _P, _P, _P, ctypes.c_int32, _P]),
            "vmoe_device_status": (ctypes.c_int, [ctypes.c_int]),
            "vmoe_selftest_bounded_wait": (ctypes.c_int, [ctypes.c_longlong, _P]),
            "vmoe_trace_enable": (ctypes.c_int, [ctypes.c_int]),
            "vmoe_trace_disable": (ctypes.c_int, []),
            "vmoe_trace_get": (ctypes.c_int, [ctypes.c_int, ctypes.POINTER(ctypes.c_char_p),
                                              ctypes.POINTER(ctypes.c_float)]),
        }
        for name, (res, args) in sig.items():
            fn = getattr(lib, name)
            fn.restype = res
            fn.argtypes = args
        _lib = lib
    return _lib


def status_string(status: int) -> str:
    try:
        return library().vmoe_status_string(int(status)).decode()
    except Exception:  # library not loadable
        return "status %d" % status


def _ptr(t):
    if t is None:
        return None
    if isinstance(t, int):
        return t
    return t.data_ptr()


_current_raw_stream = None
_get_device = None


def _raw_device_getter():
    """A function that returns the current device's index: torch's own getter where it has one (0.06 us, where
    the public call takes 0.27)."""
    import torch
    torch.cuda.current_device()  # CUDA is up
    return getattr(torch._C, "_cuda_getDevice", None) or torch.cuda.current_device


def _device():
    global _get_device
    if _get_device is None:
        _get_device = _raw_device_getter()
    return _get_device()


def _raw_stream_getter():
    """A function that returns the current torch stream of the current device as an integer.

    torch's own getter of the raw handle where it has one: building the
    ``torch.cuda.Stream`` object that the public call returns takes 3 to 4 us, as
    long as a kernel launch (one forward of four calls: 36 us of host time with it,
    20 us without)."""
    import torch
    raw = getattr(torch._C, "_cuda_getCurrentRawStream", None)
    if raw is None:
        return lambda: torch.cuda.current_stream().cuda_stream
    return lambda: raw(_device())


def _stream(stream):
    if stream is None:
        global _current_raw_stream
        if _current_raw_stream is None:
            _current_raw_stream = _raw_stream_getter()
        return _current_raw_stream()
    if isinstance(stream, int):
        return stream
    return stream.cuda_stream


def _bytes(where, n):
    """A count of bytes; a negative one would reach the library as a huge size_t and pass its checks."""
    if n < 0:
        raise VmoeError(VMOE_ERR_INVALID, "%s: %d bytes of workspace" % (where, n))
    return int(n)


def _check(st: int, where: str):
    if st != VMOE_OK:
        raise VmoeError(st, where)


def problem(T, N, d_model, d_ff, E, k, capacity_factor, dtype="bf16", flags=0, capacity=0):
    """Build a VmoeProblem; ``dtype`` is "bf16", "f32" or a VMOE_* code."""
    if isinstance(dtype, str):
        dtype = {"bf16": VMOE_BF16, "f32": VMOE_F32}[dtype]
    return VmoeProblem(int(T), int(N), int(d_model), int(d_ff), int(E), int(k),
                       float(capacity_factor), int(capacity), int(dtype), int(flags))


def vmoe_version() -> int:
    return library().vmoe_version()


def vmoe_problem_capacity(p: VmoeProblem) -> int:
    c = library().vmoe_problem_capacity(ctypes.byref(p))
    if c < 0:
        raise VmoeError(c, "vmoe_problem_capacity")
    return c


def vmoe_expert_bwd_workspace_size(p: VmoeProblem) -> int:
    return int(library().vmoe_expert_bwd_workspace_size(ctypes.byref(p)))


def vmoe_expert_bwd_min_workspace_size(p: VmoeProblem) -> int:
    return int(library().vmoe_expert_bwd_min_workspace_size(ctypes.byref(p)))


def vmoe_route(p, x, w_router, logit_bias, logits, expert_idx, gate, slot, load, stream=None):
    _check(library().vmoe_route(ctypes.byref(p), _ptr(x), _ptr(w_router), _ptr(logit_bias),
                                _ptr(logits), _ptr(expert_idx), _ptr(gate), _ptr(slot),
                                _ptr(load), _stream(stream)), "vmoe_route")


def vmoe_dispatch(p, src, weight, expert_idx, slot, load, dst, stream=None):
    _check(library().vmoe_dispatch(ctypes.byref(p), _ptr(src), _ptr(weight), _ptr(expert_idx),
                                   _ptr(slot), _ptr(load), _ptr(dst), _stream(stream)),
           "vmoe_dispatch")


def vmoe_expert_fwd(p, xe, w1, w2, load, h, a, ye, stream=None):
    _check(library().vmoe_expert_fwd(ctypes.byref(p), _ptr(xe), _ptr(w1), _ptr(w2), _ptr(load),
                                     _ptr(h), _ptr(a), _ptr(ye), _stream(stream)),
           "vmoe_expert_fwd")


def vmoe_expert_bwd(p, xe, h, a, w1, w2, dye, load, dxe, dw1, dw2, workspace, workspace_bytes=None,
                    stream=None):
    if workspace_bytes is None:
        workspace_bytes = workspace.numel() * workspace.element_size()
    _check(library().vmoe_expert_bwd(ctypes.byref(p), _ptr(xe), _ptr(h), _ptr(a), _ptr(w1),
                                     _ptr(w2), _ptr(dye), _ptr(load), _ptr(dxe), _ptr(dw1),
                                     _ptr(dw2), _ptr(workspace), _bytes("vmoe_expert_bwd", workspace_bytes),
                                     _stream(stream)), "vmoe_expert_bwd")


VMOE_STATIC_SCRATCH_BYTES = 64 << 20


def vmoe_expert_bwd_static_scratch(p, xe, h, a, w1, w2, dye, load, dxe, dw1, dw2, stream=None):
    """vmoe_expert_bwd with its dH scratch in the library's own 64 MiB device
    array, for callers that cannot allocate device memory (see include/vmoe.h)."""
    _check(library().vmoe_expert_bwd_static_scratch(
        ctypes.byref(p), _ptr(xe), _ptr(h), _ptr(a), _ptr(w1), _ptr(w2), _ptr(dye), _ptr(load),
        _ptr(dxe), _ptr(dw1), _ptr(dw2), _stream(stream)), "vmoe_expert_bwd_static_scratch")


def vmoe_combine(p, src, weight, expert_idx, slot, dst, stream=None):
    _check(library().vmoe_combine(ctypes.byref(p), _ptr(src), _ptr(weight), _ptr(expert_idx),
                                  _ptr(slot), _ptr(dst), _stream(stream)), "vmoe_combine")


def vmoe_attn_expert_fwd(p, heads, xe, wqkv, wo, load, qkv, o, lse, ye, stream=None):
    """Attention experts, forward (see include/vmoe.h)."""
    _check(library().vmoe_attn_expert_fwd(ctypes.byref(p), int(heads), _ptr(xe), _ptr(wqkv), _ptr(wo),
                                          _ptr(load), _ptr(qkv), _ptr(o), _ptr(lse), _ptr(ye),
                                          _stream(stream)), "vmoe_attn_expert_fwd")


def vmoe_attn_expert_bwd_workspace_size(p, heads) -> int:
    return int(library().vmoe_attn_expert_bwd_workspace_size(ctypes.byref(p), int(heads)))


def vmoe_attn_expert_bwd(p, heads, xe, qkv, o, lse, wqkv, wo, dye, load, dxe, dwqkv, dwo, workspace,
                         workspace_bytes=None, stream=None):
    """Attention experts, backward (see include/vmoe.h)."""
    if workspace_bytes is None:
        workspace_bytes = workspace.numel() * workspace.element_size()
    _check(library().vmoe_attn_expert_bwd(
        ctypes.byref(p), int(heads), _ptr(xe), _ptr(qkv), _ptr(o), _ptr(lse), _ptr(wqkv), _ptr(wo),
        _ptr(dye), _ptr(load), _ptr(dxe), _ptr(dwqkv), _ptr(dwo), _ptr(workspace),
        _bytes("vmoe_attn_expert_bwd", workspace_bytes),
        _stream(stream)), "vmoe_attn_expert_bwd")


def vmoe_router_bwd(p, x, w_router, logits, expert_idx, gate, slot, dy, ye, dgate, dlogits,
                    dw_router, dbias=None, dx=None, stream=None):
    """Router backward with the routing fixed; dx (if given) is updated in place."""
    _check(library().vmoe_router_bwd(
        ctypes.byref(p), _ptr(x), _ptr(w_router), _ptr(logits), _ptr(expert_idx), _ptr(gate),
        _ptr(slot), _ptr(dy), _ptr(ye), _ptr(dgate), _ptr(dlogits), _ptr(dw_router), _ptr(dbias),
        _ptr(dx), _stream(stream)), "vmoe_router_bwd")


_KINDS = {}


def _kinds():
    """The torch dtypes that the checks below compare with, looked up once."""
    if not _KINDS:
        import torch
        _KINDS.update({"f32": torch.float32, "i32": torch.int32, "u8": torch.uint8, "fp8": torch.float8_e4m3fn,
                       VMOE_F32: torch.float32, VMOE_BF16: torch.bfloat16})
    return _KINDS


def _arrays(where, *args):
    """Device pointers of (tensor, dtype, elements) triples.

    A tensor has to be contiguous, on the current device, of that dtype and of as many
    elements: one that is not would be read as something else, or past its end.  None and
    raw pointers are handed on."""
    kinds, device, out = _KINDS or _kinds(), None, []
    for t, dtype, n in args:
        if t is None or t.__class__ is int:
            out.append(t)
            continue
        at = t.get_device()  # -1 on the host
        if device is None:
            device = _device() if at >= 0 else -2
        if at == device and t.dtype is kinds[dtype] and t.numel() == n and t.is_contiguous():
            out.append(t.data_ptr())
        else:
            raise VmoeError(VMOE_ERR_INVALID, "%s: a tensor of %s, %s on %s, where %d contiguous elements of %s are read on "
                            "the current device" % (where, tuple(t.shape), t.dtype, t.device, n, kinds[dtype]))
    return out


def _workspace(where, t, nbytes):
    if t is None or isinstance(t, int):
        return t, _bytes(where, nbytes or 0)
    have = t.numel() * t.element_size()
    at = t.get_device()
    if at < 0 or at != _device() or not t.is_contiguous() or (nbytes is not None and nbytes > have):
        raise VmoeError(VMOE_ERR_INVALID, "%s: the workspace" % where)
    return t.data_ptr(), have if nbytes is None else _bytes(where, nbytes)


def vmoe_balance_workspace_size(p) -> int:
    return int(library().vmoe_balance_workspace_size(ctypes.byref(p)))


def vmoe_balance(p, logits, expert_idx, token_mask, count, tokens, excess, loss, workspace, workspace_bytes=None,
                 stream=None):
    """Balance losses of the routers and per-expert counts (see include/vmoe.h)."""
    te, tn = p.T * p.E, p.T * p.N
    a = _arrays("vmoe_balance", (logits, "f32", tn * p.E), (expert_idx, "i32", tn * p.k), (token_mask, "u8", tn),
                (count, "i32", te), (tokens, "i32", p.T), (excess, "f32", te), (loss, "f32", 3 * p.T))
    ws, nbytes = _workspace("vmoe_balance", workspace, workspace_bytes)
    _check(library().vmoe_balance(ctypes.byref(p), *a, ws, nbytes, _stream(stream)), "vmoe_balance")


def vmoe_balance_bwd(p, logits, token_mask, count, tokens, excess, dloss, dlogits, stream=None):
    """Gradient of the weighted balance losses by the logits (see include/vmoe.h)."""
    te, tn = p.T * p.E, p.T * p.N
    a = _arrays("vmoe_balance_bwd", (logits, "f32", tn * p.E), (token_mask, "u8", tn), (count, "i32", te),
                (tokens, "i32", p.T), (excess, "f32", te), (dloss, "f32", 3 * p.T), (dlogits, "f32", tn * p.E))
    _check(library().vmoe_balance_bwd(ctypes.byref(p), *a, _stream(stream)), "vmoe_balance_bwd")


def norm_config(rms=False, post=True, eps=1e-6, residual_scale=1.0):
    """Build a VmoeNorm: layer or root-mean-square norms, with or without one on the branch."""
    return VmoeNorm(float(eps), float(residual_scale), (VMOE_NORM_RMS if rms else 0) | (VMOE_NORM_POST if post else 0))


def vmoe_block_norm(p, norm, x, y, post_w, post_b, gate, pre_w, pre_b, z, u, post_stat=None, pre_stat=None, stream=None):
    """z = rho x + gate * norm(y) and u = norm(z) (see include/vmoe.h)."""
    n, td, st = p.T * p.N * p.d_model, p.T * p.d_model, 2 * p.T * p.N
    a = _arrays("vmoe_block_norm", (x, p.dtype, n), (y, p.dtype, n), (post_w, "f32", td), (post_b, "f32", td),
                (gate, "f32", td), (pre_w, "f32", td), (pre_b, "f32", td), (z, p.dtype, n), (u, p.dtype, n),
                (post_stat, "f32", st), (pre_stat, "f32", st))
    _check(library().vmoe_block_norm(ctypes.byref(p), ctypes.byref(norm), *a, _stream(stream)), "vmoe_block_norm")


def vmoe_block_norm_bwd_workspace_size(p) -> int:
    return int(library().vmoe_block_norm_bwd_workspace_size(ctypes.byref(p)))


def vmoe_block_norm_bwd(p, norm, y, z, post_stat, pre_stat, post_w, post_b, gate, pre_w, dz, du, dx, dy, dpost_w, dpost_b,
                        dgate, dpre_w, dpre_b, workspace, workspace_bytes=None, stream=None):
    """Backward of vmoe_block_norm (see include/vmoe.h)."""
    n, td, st = p.T * p.N * p.d_model, p.T * p.d_model, 2 * p.T * p.N
    a = _arrays("vmoe_block_norm_bwd", (y, p.dtype, n), (z, p.dtype, n), (post_stat, "f32", st), (pre_stat, "f32", st),
                (post_w, "f32", td), (post_b, "f32", td), (gate, "f32", td), (pre_w, "f32", td), (dz, p.dtype, n),
                (du, p.dtype, n), (dx, p.dtype, n), (dy, p.dtype, n), (dpost_w, "f32", td), (dpost_b, "f32", td),
                (dgate, "f32", td), (dpre_w, "f32", td), (dpre_b, "f32", td))
    ws, nbytes = _workspace("vmoe_block_norm_bwd", workspace, workspace_bytes)
    _check(library().vmoe_block_norm_bwd(ctypes.byref(p), ctypes.byref(norm), *a, ws, nbytes, _stream(stream)),
           "vmoe_block_norm_bwd")


def adamw_tensors(tensors):
    """The host table of vmoe_adamw, built once for a set of tensors.

    ``tensors``: dicts with param, grad, m, v (torch tensors; fp32 moments, or
    float8_e4m3fn ones with m_scale and v_scale), and optionally master, lr_scale and
    weight_decay.  The table keeps the tensors alive and is for the device that is current
    now.  One array in two places is refused: its update would be a race.  It holds the
    arrays' addresses, so gradients have to stay where they are; building it takes some 20 us
    a tensor on the host, for every array is checked here and not in the calls."""
    tensors = [dict(t) for t in tensors]
    table = (VmoeAdamwTensor * max(1, len(tensors)))()
    kinds = _kinds()
    code = {kinds[VMOE_F32]: VMOE_F32, kinds[VMOE_BF16]: VMOE_BF16}
    written, read = [], []
    for e, t in zip(table, tensors):
        param, n = t["param"], t["param"].numel()
        if param.dtype not in code or t["grad"].dtype not in code:
            raise VmoeError(VMOE_ERR_INVALID, "adamw_tensors")
        e.param_dtype, e.grad_dtype, e.numel = code[param.dtype], code[t["grad"].dtype], n
        eight = t["m"].dtype == kinds["fp8"]
        e.state = VMOE_STATE_E4M3 if eight else VMOE_STATE_F32
        state, blocks = "fp8" if eight else "f32", (n + 255) // 256
        if not eight and (t.get("m_scale") is not None or t.get("v_scale") is not None):
            raise VmoeError(VMOE_ERR_INVALID, "adamw_tensors: scales of fp32 moments")
        if eight and (t.get("m_scale") is None or t.get("v_scale") is None):
            raise VmoeError(VMOE_ERR_INVALID, "adamw_tensors: 8-bit moments without scales")
        names = ("param", "grad", "m", "v", "m_scale", "v_scale", "master")
        sizes = (e.param_dtype, n), (e.grad_dtype, n), (state, n), (state, n), ("f32", blocks), ("f32", blocks), ("f32", n)
        ptrs = _arrays("adamw_tensors", *((t.get(k), *s) for k, s in zip(names, sizes)))
        for name, ptr in zip(names, ptrs):
            setattr(e, name, ptr)
            if ptr and t[name].numel():
                span = (ptr, ptr + t[name].numel() * t[name].element_size())
                (read if name == "grad" else written).append(span)
        e.lr_scale, e.weight_decay = float(t.get("lr_scale", 1.0)), float(t.get("weight_decay", 0.0))
    spans = sorted([(b, e, True) for b, e in written] + [(b, e, False) for b, e in read])
    end, last_write = 0, 0  # of all arrays so far, and of the written ones
    for b, e, w in spans:
        if b < (end if w else last_write):
            raise VmoeError(VMOE_ERR_INVALID, "adamw_tensors: two arrays overlap")
        end, last_write = max(end, e), max(last_write, e) if w else last_write
    table.tensors, table.count = tensors, len(tensors)
    table.device = _device() if tensors else None  # where _arrays has found them all
    return table


def vmoe_adamw(table, step, lr, beta1=0.9, beta2=0.999, eps=1e-8, seed=0, step_dev=None, lr_dev=None, grad_scale=None,
               stream=None):
    """One AdamW update of the tensors of ``table`` (adamw_tensors; see include/vmoe.h)."""
    if table.device is not None and table.device != _device():
        raise VmoeError(VMOE_ERR_INVALID, "vmoe_adamw: tensors on device %d, the current one is %d" % (table.device, _device()))
    a = _arrays("vmoe_adamw", (step_dev, "i32", 1), (lr_dev, "f32", 1), (grad_scale, "f32", 1))
    c = VmoeAdamwConfig(lr, beta1, beta2, eps, step, seed & 0xffffffff, *a)
    _check(library().vmoe_adamw(table.count, table, ctypes.byref(c), _stream(stream)), "vmoe_adamw")


def vmoe_plan_slices(weight, lifespan, capacity: int, eta: float = 0.0, budget: float = 0.0):
    """Host-side slice planner (see include/vmoe.h); returns a list of slices,
    each a list of item indices."""
    import numpy as np
    w = np.ascontiguousarray(weight, dtype=np.int64)
    r = np.ascontiguousarray(lifespan, dtype=np.float64)
    n = int(w.size)
    order = np.zeros(max(n, 1), dtype=np.int32)
    start = np.zeros(n + 2, dtype=np.int32)
    ns = library().vmoe_plan_slices(n, w.ctypes.data, r.ctypes.data, int(capacity), float(eta),
                                    float(budget), order.ctypes.data, start.ctypes.data)
    _check(ns if ns < 0 else 0, "vmoe_plan_slices")
    return [order[start[s]:start[s + 1]].tolist() for s in range(ns)]


def vmoe_plan_shares(work, minimum, saturation, budget: int):
    """Host-side fill-clamp-refill allocation (see include/vmoe.h); returns the
    list of whole-unit shares."""
    import numpy as np
    w = np.ascontiguousarray(work, dtype=np.float64)
    mn = np.ascontiguousarray(minimum, dtype=np.int32)
    sat = np.ascontiguousarray(saturation, dtype=np.int32)
    n = int(w.size)
    out = np.zeros(max(n, 1), dtype=np.int32)
    r = library().vmoe_plan_shares(n, w.ctypes.data, mn.ctypes.data, sat.ctypes.data, int(budget),
                                   out.ctypes.data)
    _check(r if r < 0 else 0, "vmoe_plan_shares")
    return out[:n].tolist()


def vmoe_device_status(reset: bool = False) -> int:
    return library().vmoe_device_status(1 if reset else 0)


def vmoe_selftest_bounded_wait(limit_ns: int, stream=None):
    _check(library().vmoe_selftest_bounded_wait(int(limit_ns), _stream(stream)),
           "vmoe_selftest_bounded_wait")


def vmoe_trace_enable(max_records: int):
    _check(library().vmoe_trace_enable(int(max_records)), "vmoe_trace_enable")


def vmoe_trace_disable() -> int:
    return library().vmoe_trace_disable()


def vmoe_trace_get(i: int):
    name = ctypes.c_char_p()
    ms = ctypes.c_float()
    _check(library().vmoe_trace_get(int(i), ctypes.byref(name), ctypes.byref(ms)),
           "vmoe_trace_get")
    return name.value.decode(), ms.value


from .step import BalanceBuffers, Buffers, HostPipeline, StepRunner  # noqa: E402  (needs the names above)
from .block import BlockStack  # noqa: E402
from .optim import AdamW  # noqa: E402
