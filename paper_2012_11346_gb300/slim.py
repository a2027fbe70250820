"""Python binding of libslim (ctypes): argument marshalling only.

Every computation runs in the CUDA kernels behind the C ABI declared in
include/slim.h, include/slim_lm.h and include/slim_layer.h.  PyTorch supplies device
memory (outputs and workspace, so torch.cuda.max_memory_allocated sees all of it) and the
current stream.  There is no CPU fallback: if libslim.so is missing or no GPU is present,
the calls raise.
"""
import array
import contextlib
import ctypes
import functools
import math
import os

import torch

_LIB_PATH = os.path.join(os.path.dirname(os.path.abspath(__file__)), "libslim.so")
_lib = None

DTYPES = {torch.float32: 0, torch.bfloat16: 1}
FEATURES = {"exp": 0, "relu": 1, "square": 2}
INDEX_DTYPES = {torch.int32: 0, torch.int64: 1}
STATUS = {0: "SLIM_OK", 1: "SLIM_ERR_INVALID_ARG", 2: "SLIM_ERR_UNSUPPORTED",
          3: "SLIM_ERR_WORKSPACE", 4: "SLIM_ERR_CUDA", 5: "SLIM_ERR_TIMEOUT"}

_i, _p, _sz = ctypes.c_int, ctypes.c_void_p, ctypes.c_size_t
_ll, _f = ctypes.c_longlong, ctypes.c_float

# (name, argtypes) for every symbol of include/slim.h, slim_lm.h and slim_layer.h
SIGNATURES = {
    "slim_status_string": ([_i], ctypes.c_char_p),
    "slim_version": ([], _i),
    "slim_fwd_workspace_size": ([_i] * 6 + [_i, _i, ctypes.POINTER(_sz)], _i),
    "slim_bwd_workspace_size": ([_i] * 6 + [_i, _i, ctypes.POINTER(_sz)], _i),
    "slim_fwd": ([_p] * 4 + [_i] * 6 + [_i, _i] + [_p] * 5 + [_p, _sz, _p], _i),
    "slim_bwd": ([_p] * 10 + [_i] * 6 + [_i, _i] + [_p] * 4 + [_p, _sz, _p], _i),
    "slim_fwd_from": ([_p] * 4 + [_i] * 6 + [_i, _i] + [_p] * 4 + [_p] * 5 + [_p, _sz, _p], _i),
    "slim_bwd_from": ([_p] * 12 + [_i] * 6 + [_i, _i] + [_p] * 4 + [_p] * 2 + [_p, _sz, _p], _i),
    "slim_bidir_workspace_size": ([_i] * 6 + [_i, _i, _i, ctypes.POINTER(_sz)], _i),
    "slim_fwd_bidir": ([_p] * 4 + [_i] * 6 + [_i, _i] + [_p] * 3 + [_p, _sz, _p], _i),
    "slim_bwd_bidir": ([_p] * 8 + [_i] * 6 + [_i, _i] + [_p] * 4 + [_p, _sz, _p], _i),
    "slim_stack_workspace_size": ([_i] * 7 + [_i, _i, _i, ctypes.POINTER(_sz)], _i),
    "slim_stack_fwd": ([_p] * 2 + [_i] * 7 + [_i, _i] + [_p] * 5 + [_p, _sz, _p], _i),
    "slim_stack_bwd": ([_p] * 7 + [_i] * 7 + [_i, _i] + [_p] * 2 + [_p, _sz, _p], _i),
    "slim_check_device_error": ([_p, _p], _i),
    "slim_launch_count": ([], ctypes.c_ulonglong),
    "slim_profiler_enable": ([_i], None),
    "slim_profiler_reset": ([], None),
    "slim_profiler_read": ([_p, _i], _i),
    "slim_tc_selftest": ([_i, _i, _i, _i, _p, _p, _p, _p, _p], _i),
    "slim_path_for": ([_i] * 6 + [_i, _i, ctypes.POINTER(_i)], _i),
    "slim_bwd_schedule": ([_i] * 6 + [_i, _i, _p, _i, ctypes.POINTER(_i), ctypes.POINTER(_i)],
                          _i),
    "slim_fwd_noalloc": ([_p] * 4 + [_i] * 6 + [_i, _i] + [_p] * 5 + [_p], _i),
    "slim_diag_wait_timeout": ([_p, _p], _i),
    "slim_embed_fwd": ([_p, _i, _p, _ll, _i, _i, _i, _f, _p, _p], _i),
    "slim_embed_bwd_workspace_size": ([_ll, _i, _i, _i, ctypes.POINTER(_sz)], _i),
    "slim_embed_bwd": ([_p, _i, _p, _ll, _i, _i, _i, _f, _i, _p, _p, _sz, _p], _i),
    "slim_vocab_loss_workspace_size": ([_ll, _i, _i, _i, _i, _i, ctypes.POINTER(_sz)], _i),
    "slim_vocab_loss_fwd": ([_p, _p, _p, _i, _ll, _i, _i, _i, _ll, _p, _p, _p, _p, _sz, _p], _i),
    "slim_vocab_loss_bwd": ([_p, _p, _p, _i, _p, _p, _i, _p, _ll, _i, _i, _i, _i, _ll, _p, _p, _p,
                             _sz, _p], _i),
    "slim_clip_workspace_size": ([_i, ctypes.POINTER(_sz)], _i),
    "slim_clip_grads": ([_p, _p, _p, _p, _i, _f, _p, _p, _sz, _p], _i),
    "slim_qk_norm_fwd": ([_p] * 7 + [_i, _p] + [_i] * 8 + [_f, _f] + [_p] * 5, _i),
    "slim_qk_norm_bwd_workspace_size": ([_i] * 5 + [ctypes.POINTER(_sz)], _i),
    "slim_gated_scan_workspace_size": ([_i] * 4 + [ctypes.POINTER(_sz)], _i),
    "slim_gated_scan_fwd": ([_p, _ll, _p, _ll, _p] + [_i] * 5 + [_p] * 4 + [_sz, _p], _i),
    "slim_gated_scan_bwd": ([_p, _ll, _p, _ll] + [_p] * 3 + [_i] * 5 + [_p, _ll, _p, _ll, _p, _p, _sz, _p],
                            _i),
    "slim_diag_gated_scan_wait": ([_p, _p, _i, _i, _p, _p, _sz, _p], _i),
    "slim_gated_ff_workspace_size": ([_ll, _i, _i, _i, _i, ctypes.POINTER(_sz)], _i),
    "slim_gated_ff_kept_size": ([_ll, _i, _i, _i, ctypes.POINTER(_sz)], _i),
    "slim_gated_ff_fwd": ([_p, _p, _ll] + [_i] * 4 + [_p, _p, _p, _sz, _p], _i),
    "slim_gated_ff_bwd": ([_p, _p, _p, _ll] + [_i] * 4 + [_p] * 4 + [_sz, _p], _i),
    "slim_qk_norm_bwd": ([_p] * 7 + [_i, _p] + [_i] * 8 + [_f, _f] + [_p] * 11 + [_sz, _p], _i),
}


class KernelStats(ctypes.Structure):
    _fields_ = [("name", ctypes.c_char * 48), ("launches", ctypes.c_ulonglong),
                ("total_ms", ctypes.c_double), ("flops", ctypes.c_double),
                ("bytes", ctypes.c_double)]


class SlimError(RuntimeError):
    def __init__(self, status, where):
        self.status = status
        super().__init__(f"{where}: {status_string(status)}")


def library():
    """Loads libslim.so (built by paper_2012_11346_gb300.build); raises if absent."""
    global _lib
    if _lib is None:
        if not os.path.exists(_LIB_PATH):
            raise RuntimeError(f"libslim.so not built ({_LIB_PATH}); run "
                               "python -m paper_2012_11346_gb300.build")
        lib = ctypes.CDLL(_LIB_PATH)
        for name, (args, res) in SIGNATURES.items():
            fn = getattr(lib, name)
            fn.argtypes = args
            fn.restype = res
        _lib = lib
    return _lib


def status_string(status):
    return library().slim_status_string(int(status)).decode()


def _check(status, where):
    if status != 0:
        raise SlimError(status, where)


def _dims(q, omega):
    B, H, L, d = q.shape
    M = omega.shape[0] if omega is not None else d
    return B, H, L, d, M


def workspace_size(B, H, L, d, M, C, dtype, feature, backward):
    n = _sz(0)
    fn = library().slim_bwd_workspace_size if backward else library().slim_fwd_workspace_size
    _check(fn(B, H, L, d, M, C, DTYPES[dtype], FEATURES[feature], ctypes.byref(n)),
           "workspace_size")
    return n.value


def path_for(B, H, L, d, M, C, dtype, feature):
    """1 if the tensor-core kernels serve this problem, 0 for the fp32 path."""
    r = _i(0)
    _check(library().slim_path_for(B, H, L, d, M, C, DTYPES[dtype], FEATURES[feature],
                                   ctypes.byref(r)), "slim_path_for")
    return r.value


def bwd_schedule(B, H, L, d, M, C, dtype, feature):
    """The tensor-core backward's item order and hand-off ring depth R: a list
    of (role, slice, index) per ticket (roles 0 dq side, 1 dk/dv side, 2 and 3
    the final dOmega reduction stages), and R."""
    lib, n, ring = library(), _i(0), _i(0)
    _check(lib.slim_bwd_schedule(B, H, L, d, M, C, DTYPES[dtype], FEATURES[feature], None, 0,
                                 ctypes.byref(n), None), "slim_bwd_schedule")
    buf = (_i * (3 * n.value))()
    _check(lib.slim_bwd_schedule(B, H, L, d, M, C, DTYPES[dtype], FEATURES[feature], buf, n.value,
                                 ctypes.byref(n), ctypes.byref(ring)), "slim_bwd_schedule")
    return [tuple(buf[3 * x:3 * x + 3]) for x in range(n.value)], ring.value


def _stream_handle(stream):
    s = torch.cuda.current_stream() if stream is None else stream
    return ctypes.c_void_p(s.cuda_stream)


def _stream_of(t, stream):
    """The raw stream of a call on tensor t: `stream`, or the current one."""
    if stream is not None:
        return stream.cuda_stream
    return torch._C._cuda_getCurrentRawStream(t.get_device())


def _workspace(nbytes, device):
    return torch.empty(max(nbytes, 256), dtype=torch.uint8, device=device)


def _require_cuda(*ts):
    for t in ts:
        if not t.is_cuda:
            raise RuntimeError("libslim runs on CUDA tensors only (no CPU fallback)")
        if not t.is_contiguous():
            raise RuntimeError("libslim needs contiguous tensors")


def _ptr(t):
    return None if t is None else t.data_ptr()


def _opt_ptr(t):
    if t is None:
        return None
    _require_cuda(t)
    return t.data_ptr()


def forward(q, k, v, omega, C, feature="exp", workspace=None, stream=None, residuals=False,
            S_init=None, z_init=None, S_init_lo=None, z_init_lo=None):
    """slim_fwd (slim_fwd_from when an initial state is given): returns
    (out, S_state, z_state), or with residuals=True (out, S_state, z_state,
    S_state_lo, z_state_lo) -- the low-order parts of the carried state, which
    slim_bwd uses to start its rollback exactly.  S_init / z_init (and their
    residuals): the state B^(0) the sequence starts from, e.g. the state an
    earlier segment returned.  omega may be None for the quadratic map."""
    _require_cuda(q, k, v)
    B, H, L, d = q.shape
    M = omega.shape[0] if omega is not None else d
    out = torch.empty_like(q)
    S_state = torch.empty(B, H, M, d, dtype=torch.float32, device=q.device)
    z_state = torch.empty(B, H, M, dtype=torch.float32, device=q.device)
    S_lo = torch.empty_like(S_state) if residuals else None
    z_lo = torch.empty_like(z_state) if residuals else None
    need = workspace_size(B, H, L, d, M, C, q.dtype, feature, False)
    ws = workspace if workspace is not None else _workspace(need, q.device)
    args = (q.data_ptr(), k.data_ptr(), v.data_ptr(), _opt_ptr(omega), B, H, L, d, M, C,
            DTYPES[q.dtype], FEATURES[feature])
    tail = (out.data_ptr(), S_state.data_ptr(), z_state.data_ptr(), _ptr(S_lo), _ptr(z_lo),
            ws.data_ptr(), ws.numel(), _stream_handle(stream))
    if S_init is None and z_init is None:
        _check(library().slim_fwd(*args, *tail), "slim_fwd")
    else:
        _check(library().slim_fwd_from(*args, _opt_ptr(S_init), _opt_ptr(z_init),
                                       _opt_ptr(S_init_lo), _opt_ptr(z_init_lo), *tail),
               "slim_fwd_from")
    if residuals:
        return out, S_state, z_state, S_lo, z_lo
    return out, S_state, z_state


def backward(q, k, v, omega, out, dout, S_state, z_state, C, feature="exp", workspace=None,
             stream=None, S_lo=None, z_lo=None, G_S_in=None, g_z_in=None, return_state_grad=False):
    """slim_bwd (slim_bwd_from when a state gradient is handed in or asked
    for): returns (dq, dk, dv, domega), and with return_state_grad=True also
    (G_S, g_z) = G^(0), the gradient with respect to the state the sequence
    started from.  S_lo / z_lo: the residuals from forward(..., residuals=True),
    or None.  G_S_in / g_z_in: G^(N) from the backward of a later segment.
    For the quadratic map omega may be None; domega is then None."""
    _require_cuda(q, k, v, out, dout, S_state, z_state)
    B, H, L, d = q.shape
    M = omega.shape[0] if omega is not None else d
    dq, dk, dv = torch.empty_like(q), torch.empty_like(k), torch.empty_like(v)
    domega = (torch.empty(M, d, dtype=torch.float32, device=q.device)
              if omega is not None else None)
    need = workspace_size(B, H, L, d, M, C, q.dtype, feature, True)
    ws = workspace if workspace is not None else _workspace(need, q.device)
    G_S = g_z = None
    head = (q.data_ptr(), k.data_ptr(), v.data_ptr(), _opt_ptr(omega), out.data_ptr(),
            dout.data_ptr(), S_state.data_ptr(), z_state.data_ptr(), _ptr(S_lo), _ptr(z_lo))
    dims = (B, H, L, d, M, C, DTYPES[q.dtype], FEATURES[feature])
    grads = (dq.data_ptr(), dk.data_ptr(), dv.data_ptr(), _ptr(domega))
    tail = (ws.data_ptr(), ws.numel(), _stream_handle(stream))
    if G_S_in is None and g_z_in is None and not return_state_grad:
        _check(library().slim_bwd(*head, *dims, *grads, *tail), "slim_bwd")
    else:
        if return_state_grad:
            G_S = torch.empty(B, H, M, d, dtype=torch.float32, device=q.device)
            g_z = torch.empty(B, H, M, dtype=torch.float32, device=q.device)
        _check(library().slim_bwd_from(*head, _opt_ptr(G_S_in), _opt_ptr(g_z_in), *dims, *grads,
                                       _ptr(G_S), _ptr(g_z), *tail), "slim_bwd_from")
    if return_state_grad:
        return dq, dk, dv, domega, G_S, g_z
    return dq, dk, dv, domega


def bidir_workspace_size(B, H, L, d, M, C, dtype, feature, backward):
    n = _sz(0)
    _check(library().slim_bidir_workspace_size(B, H, L, d, M, C, DTYPES[dtype],
                                               FEATURES[feature], 1 if backward else 0,
                                               ctypes.byref(n)), "slim_bidir_workspace_size")
    return n.value


def forward_bidir(q, k, v, omega, C, feature="exp", workspace=None, stream=None):
    """slim_fwd_bidir (non-causal): returns (out, S_state, z_state), the state
    being the global sum over all rows."""
    _require_cuda(q, k, v)
    B, H, L, d, M = _dims(q, omega)
    out = torch.empty_like(q)
    S_state = torch.empty(B, H, M, d, dtype=torch.float32, device=q.device)
    z_state = torch.empty(B, H, M, dtype=torch.float32, device=q.device)
    ws = workspace if workspace is not None else _workspace(
        bidir_workspace_size(B, H, L, d, M, C, q.dtype, feature, False), q.device)
    _check(library().slim_fwd_bidir(q.data_ptr(), k.data_ptr(), v.data_ptr(), _opt_ptr(omega),
                                    B, H, L, d, M, C, DTYPES[q.dtype], FEATURES[feature],
                                    out.data_ptr(), S_state.data_ptr(), z_state.data_ptr(),
                                    ws.data_ptr(), ws.numel(), _stream_handle(stream)),
           "slim_fwd_bidir")
    return out, S_state, z_state


def backward_bidir(q, k, v, omega, out, dout, S_state, z_state, C, feature="exp", workspace=None,
                   stream=None):
    """slim_bwd_bidir (non-causal): returns (dq, dk, dv, domega)."""
    _require_cuda(q, k, v, out, dout, S_state, z_state)
    B, H, L, d, M = _dims(q, omega)
    dq, dk, dv = torch.empty_like(q), torch.empty_like(k), torch.empty_like(v)
    domega = (torch.empty(M, d, dtype=torch.float32, device=q.device)
              if omega is not None else None)
    ws = workspace if workspace is not None else _workspace(
        bidir_workspace_size(B, H, L, d, M, C, q.dtype, feature, True), q.device)
    _check(library().slim_bwd_bidir(q.data_ptr(), k.data_ptr(), v.data_ptr(), _opt_ptr(omega),
                                    out.data_ptr(), dout.data_ptr(), S_state.data_ptr(),
                                    z_state.data_ptr(), B, H, L, d, M, C, DTYPES[q.dtype],
                                    FEATURES[feature], dq.data_ptr(), dk.data_ptr(),
                                    dv.data_ptr(), _ptr(domega), ws.data_ptr(), ws.numel(),
                                    _stream_handle(stream)), "slim_bwd_bidir")
    return dq, dk, dv, domega


def stack_workspace_size(B, H, L, d, M, C, layers, dtype, feature, backward):
    n = _sz(0)
    _check(library().slim_stack_workspace_size(B, H, L, d, M, C, layers, DTYPES[dtype],
                                               FEATURES[feature], 1 if backward else 0,
                                               ctypes.byref(n)), "slim_stack_workspace_size")
    return n.value


def stack_forward(x, omegas, C, feature="exp", layers=None, workspace=None, stream=None,
                  residuals=True):
    """slim_stack_fwd: x [B,H,L,d]; omegas [layers, M, d] fp32 (None for the
    quadratic map, then give `layers`).  Returns (y, S_state, z_state[, S_lo,
    z_lo]) with per-layer states [layers, B, H, M, d] and [layers, B, H, M]."""
    _require_cuda(x)
    B, H, L, d = x.shape
    layers = omegas.shape[0] if omegas is not None else layers
    M = omegas.shape[1] if omegas is not None else d
    y = torch.empty_like(x)
    S = torch.empty(layers, B, H, M, d, dtype=torch.float32, device=x.device)
    z = torch.empty(layers, B, H, M, dtype=torch.float32, device=x.device)
    S_lo = torch.empty_like(S) if residuals else None
    z_lo = torch.empty_like(z) if residuals else None
    ws = workspace if workspace is not None else _workspace(
        stack_workspace_size(B, H, L, d, M, C, layers, x.dtype, feature, False), x.device)
    _check(library().slim_stack_fwd(x.data_ptr(), _opt_ptr(omegas), B, H, L, d, M, C, layers,
                                    DTYPES[x.dtype], FEATURES[feature], y.data_ptr(),
                                    S.data_ptr(), z.data_ptr(), _ptr(S_lo), _ptr(z_lo),
                                    ws.data_ptr(), ws.numel(), _stream_handle(stream)),
           "slim_stack_fwd")
    return (y, S, z, S_lo, z_lo) if residuals else (y, S, z)


def stack_backward(x, omegas, dy, S_state, z_state, C, feature="exp", S_lo=None, z_lo=None,
                   workspace=None, stream=None):
    """slim_stack_bwd: returns (dx, domegas) (domegas None without omegas)."""
    _require_cuda(x, dy, S_state, z_state)
    B, H, L, d = x.shape
    layers = S_state.shape[0]
    M = S_state.shape[3]
    dx = torch.empty_like(x)
    dom = (torch.empty(layers, M, d, dtype=torch.float32, device=x.device)
           if omegas is not None else None)
    ws = workspace if workspace is not None else _workspace(
        stack_workspace_size(B, H, L, d, M, C, layers, x.dtype, feature, True), x.device)
    _check(library().slim_stack_bwd(x.data_ptr(), _opt_ptr(omegas), dy.data_ptr(),
                                    S_state.data_ptr(), z_state.data_ptr(), _ptr(S_lo),
                                    _ptr(z_lo), B, H, L, d, M, C, layers, DTYPES[x.dtype],
                                    FEATURES[feature], dx.data_ptr(), _ptr(dom), ws.data_ptr(),
                                    ws.numel(), _stream_handle(stream)), "slim_stack_bwd")
    return dx, dom


def forward_into(q, k, v, omega, C, feature, out, S_state, z_state, workspace, stream=None,
                 S_lo=None, z_lo=None, S_init=None, z_init=None, S_init_lo=None, z_init_lo=None):
    """slim_fwd (slim_fwd_from with an initial state) into caller-allocated
    outputs and workspace (no allocation)."""
    B, H, L, d, M = _dims(q, omega)
    args = (q.data_ptr(), k.data_ptr(), v.data_ptr(), _ptr(omega), B, H, L, d, M, C,
            DTYPES[q.dtype], FEATURES[feature])
    tail = (out.data_ptr(), S_state.data_ptr(), z_state.data_ptr(), _ptr(S_lo), _ptr(z_lo),
            workspace.data_ptr(), workspace.numel(), _stream_handle(stream))
    if S_init is None:
        _check(library().slim_fwd(*args, *tail), "slim_fwd")
    else:
        _check(library().slim_fwd_from(*args, _ptr(S_init), _ptr(z_init), _ptr(S_init_lo),
                                       _ptr(z_init_lo), *tail), "slim_fwd_from")


def backward_into(q, k, v, omega, out, dout, S_state, z_state, C, feature, dq, dk, dv, domega,
                  workspace, stream=None, S_lo=None, z_lo=None, G_S_in=None, g_z_in=None,
                  G_S_out=None, g_z_out=None):
    """slim_bwd (slim_bwd_from with state gradients in or out) into
    caller-allocated gradients and workspace (no allocation)."""
    B, H, L, d, M = _dims(q, omega)
    head = (q.data_ptr(), k.data_ptr(), v.data_ptr(), _ptr(omega), out.data_ptr(),
            dout.data_ptr(), S_state.data_ptr(), z_state.data_ptr(), _ptr(S_lo), _ptr(z_lo))
    dims = (B, H, L, d, M, C, DTYPES[q.dtype], FEATURES[feature])
    grads = (dq.data_ptr(), dk.data_ptr(), dv.data_ptr(), _ptr(domega))
    tail = (workspace.data_ptr(), workspace.numel(), _stream_handle(stream))
    if G_S_in is None and G_S_out is None:
        _check(library().slim_bwd(*head, *dims, *grads, *tail), "slim_bwd")
    else:
        _check(library().slim_bwd_from(*head, _ptr(G_S_in), _ptr(g_z_in), *dims, *grads,
                                       _ptr(G_S_out), _ptr(g_z_out), *tail), "slim_bwd_from")


def forward_bidir_into(q, k, v, omega, C, feature, out, S_state, z_state, workspace, stream=None):
    """slim_fwd_bidir into caller-allocated outputs and workspace."""
    B, H, L, d, M = _dims(q, omega)
    _check(library().slim_fwd_bidir(q.data_ptr(), k.data_ptr(), v.data_ptr(), _ptr(omega),
                                    B, H, L, d, M, C, DTYPES[q.dtype], FEATURES[feature],
                                    out.data_ptr(), S_state.data_ptr(), z_state.data_ptr(),
                                    workspace.data_ptr(), workspace.numel(),
                                    _stream_handle(stream)), "slim_fwd_bidir")


def backward_bidir_into(q, k, v, omega, out, dout, S_state, z_state, C, feature, dq, dk, dv,
                        domega, workspace, stream=None):
    """slim_bwd_bidir into caller-allocated gradients and workspace."""
    B, H, L, d, M = _dims(q, omega)
    _check(library().slim_bwd_bidir(q.data_ptr(), k.data_ptr(), v.data_ptr(), _ptr(omega),
                                    out.data_ptr(), dout.data_ptr(), S_state.data_ptr(),
                                    z_state.data_ptr(), B, H, L, d, M, C, DTYPES[q.dtype],
                                    FEATURES[feature], dq.data_ptr(), dk.data_ptr(),
                                    dv.data_ptr(), _ptr(domega), workspace.data_ptr(),
                                    workspace.numel(), _stream_handle(stream)), "slim_bwd_bidir")


def check_device_error(workspace, stream=None):
    """Raises SlimError(SLIM_ERR_TIMEOUT) if a bounded device wait gave up."""
    _check(library().slim_check_device_error(workspace.data_ptr(), _stream_handle(stream)),
           "slim_check_device_error")


def launch_count():
    """Number of libslim kernel launches since the library was loaded."""
    return int(library().slim_launch_count())


def profiler_enable(on=True):
    library().slim_profiler_enable(1 if on else 0)


def profiler_reset():
    library().slim_profiler_reset()


def profiler_read():
    """Per-kernel totals since the last reset: list of dicts with name,
    launches, total_ms (CUDA events), flops and bytes (algorithmic)."""
    arr = (KernelStats * 64)()
    n = library().slim_profiler_read(ctypes.cast(arr, ctypes.c_void_p), 64)
    if n < 0:
        raise SlimError(4, "slim_profiler_read")
    return [{"name": arr[i].name.decode(), "launches": int(arr[i].launches),
             "total_ms": arr[i].total_ms, "flops": arr[i].flops, "bytes": arr[i].bytes}
            for i in range(min(n, 64))]


def tc_selftest(A, B, a_mn, b_mn):
    """D = A @ B through one chain of tcgen05 MMAs (diagnostic of the
    tensor-core operand layouts); A [128, K], B [K, N] bf16 CUDA tensors."""
    _require_cuda(A, B)
    K, N = B.shape
    D = torch.empty(A.shape[0], N, dtype=torch.float32, device=A.device)
    err = torch.zeros(1, dtype=torch.int32, device=A.device)
    _check(library().slim_tc_selftest(a_mn, b_mn, K, N, A.data_ptr(), B.data_ptr(), D.data_ptr(),
                                      err.data_ptr(), _stream_handle(None)), "slim_tc_selftest")
    return D, err


class _FirstDerivative(torch.autograd.Function):
    """A gradient that the kernels computed, tied to what it depends on: its own
    backward refuses."""

    @staticmethod
    def forward(ctx, grad, *depends):
        return grad.clone()

    @staticmethod
    def backward(ctx, *_):
        raise RuntimeError("libslim's calls can be differentiated only once")


def _first_derivatives(grads, *depends):
    """What a Function's backward returns.  The kernels leave no graph: under
    create_graph, differentiating the gradients again would drop their terms
    without a word, and is made an error instead."""
    if not torch.is_grad_enabled() or not any(t.requires_grad for t in depends):
        return grads
    return tuple(_FirstDerivative.apply(g, *depends) for g in grads)


class SlimAttention(torch.autograd.Function):
    """Causal linear attention with the SLiM forward/backward (state carried
    across slices of C rows; backward by rollback, no stored activations).
    Differentiable once."""

    @staticmethod
    def forward(ctx, q, k, v, omega, C, feature):
        out, S, z, S_lo, z_lo = forward(q.contiguous(), k.contiguous(), v.contiguous(),
                                        omega.contiguous(), C, feature, residuals=True)
        ctx.save_for_backward(q, k, v, omega, out, S, z, S_lo, z_lo)
        ctx.C, ctx.feature = C, feature
        return out

    @staticmethod
    def backward(ctx, dout):
        q, k, v, omega, out, S, z, S_lo, z_lo = ctx.saved_tensors
        grads = backward(q.contiguous(), k.contiguous(), v.contiguous(), omega.contiguous(), out,
                         dout.contiguous(), S, z, ctx.C, ctx.feature, S_lo=S_lo, z_lo=z_lo)
        return *_first_derivatives(grads, q, k, v, omega, dout), None, None


def slim_attention(q, k, v, omega, C, feature="exp"):
    return SlimAttention.apply(q, k, v, omega, C, feature)


# ---------------------------------------------------------------- language-model ends
def _require(cond, what):
    if not cond:
        raise ValueError(what)


def _too_large():
    # the library takes these as C ints, of which ctypes would pass the low 32 bits on
    raise ValueError("a size does not fit 32 bits")


def _index_code(ids, what):
    code = INDEX_DTYPES.get(ids.dtype)
    if code is None:
        raise TypeError(f"{what} must be int32 or int64, got {ids.dtype}")
    return code


def _dtype_code(t, what):
    code = DTYPES.get(t.dtype)
    if code is None:
        raise TypeError(f"{what}: float32 or bfloat16 expected, got {t.dtype}")
    return code


_HERE = contextlib.nullcontext()


def _on(stream):
    """The context in which a call on `stream` allocates: memory that the
    caching allocator hands out there is free as far as that stream's order
    goes, and is given out again only behind the call's work."""
    return _HERE if stream is None else torch.cuda.stream(stream)


@functools.lru_cache(maxsize=1024)
def embed_workspace_size(N, D, V, dtype):
    n = _sz(0)
    if (V | D) >> 31:
        _too_large()
    _check(library().slim_embed_bwd_workspace_size(N, D, V, DTYPES[dtype], ctypes.byref(n)),
           "slim_embed_bwd_workspace_size")
    return n.value


def embed_forward(ids, table, scale=1.0, out=None, stream=None):
    """slim_embed_fwd: out [*ids.shape, D] = scale * table[ids], zero rows where
    an id lies outside [0, V).  ids int32 or int64 of any shape; table [V, D]."""
    _require_cuda(ids, table)
    it, dt = _index_code(ids, "ids"), _dtype_code(table, "embed_forward")
    if table.dim() != 2:
        raise ValueError("table must be [V, D]")
    V, D = table.shape
    if (V | D) >> 31:
        _too_large()
    if out is None:
        with _on(stream):
            out = torch.empty(*ids.shape, D, dtype=table.dtype, device=table.device)
    else:
        _require_cuda(out)
        _require(out.dtype == table.dtype and tuple(out.shape) == (*ids.shape, D),
                 "out must be [*ids.shape, D] in the table's dtype")
    _check(library().slim_embed_fwd(ids.data_ptr(), it, table.data_ptr(), ids.numel(), D, V, dt,
                                    scale, out.data_ptr(), _stream_of(table, stream)), "slim_embed_fwd")
    return out


def embed_backward(ids, dout, V, scale=1.0, dtable=None, workspace=None, stream=None):
    """slim_embed_bwd: the gradient of embed_forward with respect to its table,
    [V, D] in dout's dtype.  With dtable given, the gradient is added to it in
    place (and it is returned); rows that no id names are then left alone."""
    _require_cuda(ids, dout)
    it, dt = _index_code(ids, "ids"), _dtype_code(dout, "embed_backward")
    if dout.shape[:-1] != ids.shape:
        raise ValueError("dout must be [*ids.shape, D]")
    D, N = dout.shape[-1], ids.numel()
    if (V | D) >> 31:
        _too_large()
    accumulate = dtable is not None
    if accumulate:
        _require_cuda(dtable)
        _require(dtable.dtype == dout.dtype and tuple(dtable.shape) == (V, D),
                 "dtable must be [V, D] in dout's dtype")
    if workspace is not None:
        _require_cuda(workspace)
    with _on(stream):
        if not accumulate:
            dtable = torch.empty(V, D, dtype=dout.dtype, device=dout.device)
        ws = workspace if workspace is not None else _workspace(
            embed_workspace_size(N, D, V, dout.dtype), dout.device)
    _check(library().slim_embed_bwd(ids.data_ptr(), it, dout.data_ptr(), N, D, V, dt, scale, int(accumulate),
                                    dtable.data_ptr(), ws.data_ptr(), ws.numel(),
                                    _stream_of(dout, stream)), "slim_embed_bwd")
    return dtable


@functools.lru_cache(maxsize=1024)
def clip_workspace_size(n):
    """Workspace bytes of clip_grad_norm for n gradients."""
    b = _sz(0)
    if n >> 31:
        _too_large()
    _check(library().slim_clip_workspace_size(n, ctypes.byref(b)), "slim_clip_workspace_size")
    return b.value


def clip_grad_norm(grads, max_norm, out=None, workspace=None, stream=None):
    """slim_clip_grads: scales the gradients by min(1, max_norm / norm), norm
    being their global 2-norm, and returns norm ([1] fp32, on the device).
    In place, or into the tensors of `out` (same sizes and dtypes).  If the
    norm is not finite nothing is scaled: read it and skip the step."""
    grads = list(grads)
    n = len(grads)
    _require(n > 0, "no gradients")
    _require_cuda(*grads)
    types = [g.dtype for g in grads]
    for t in set(types):
        if t not in DTYPES:
            raise TypeError(f"gradients must be float32 or bfloat16, got {t}")
    bf16 = torch.bfloat16
    dts = array.array("i", [1 if t is bf16 else 0 for t in types])
    sizes = array.array("q", [g.numel() for g in grads])
    src = dst = array.array("Q", [g.data_ptr() for g in grads])
    _require(len(set(src)) == n or len({p for p, k in zip(src, sizes) if k}) ==
             sum(k > 0 for k in sizes), "a gradient is listed twice")
    if out is not None:
        out = list(out)
        _require_cuda(*out)
        _require([o.numel() for o in out] == sizes.tolist() and [o.dtype for o in out] == types,
                 "out must hold one tensor of the same size and dtype per gradient")
        dst = array.array("Q", [o.data_ptr() for o in out])
    if workspace is not None:
        _require_cuda(workspace)
    with _on(stream):
        norm = torch.empty(1, dtype=torch.float32, device=grads[0].device)
        ws = workspace if workspace is not None else _workspace(clip_workspace_size(n),
                                                                norm.device)
    _check(library().slim_clip_grads(src.buffer_info()[0], dst.buffer_info()[0],
                                     sizes.buffer_info()[0], dts.buffer_info()[0], n, max_norm,
                                     norm.data_ptr(), ws.data_ptr(), ws.numel(),
                                     _stream_of(norm, stream)), "slim_clip_grads")
    return norm


class Embedding(torch.autograd.Function):
    @staticmethod
    def forward(ctx, ids, table, scale):
        ids = ids.contiguous()
        ctx.save_for_backward(ids)
        ctx.V, ctx.scale = table.shape[0], scale
        return embed_forward(ids, _ready(table), scale)

    @staticmethod
    def backward(ctx, dout):
        (ids,) = ctx.saved_tensors
        dtable = embed_backward(ids, _ready(dout), ctx.V, ctx.scale)
        return None, *_first_derivatives((dtable,), dout), None


def _ready(t):
    """t as the entry points take it: contiguous, on a 16-byte boundary (a slice
    of rows may begin anywhere)."""
    t = t.contiguous()
    return t if t.data_ptr() % 16 == 0 else t.clone()


def embedding(ids, table, scale=1.0):
    """Differentiable embed_forward (gradient with respect to the table, once)."""
    return Embedding.apply(ids, table, scale)


def vocab_piece(N, V):
    """Words per piece of the vocabulary in vocab_loss_backward, unless the
    caller says otherwise: as many as keep rows x piece within 2^28, and at
    least 8192 (smaller pieces leave the products too few tiles; larger ones
    gain nothing at 32768 rows).  So up to 2^28 logits, or 8192 words, one piece
    is the whole vocabulary, and its gradient (2 bytes an element for bf16, 6 for
    fp32) as large as the logits: a smaller `piece` holds less."""
    return min(V, max(8192, (1 << 28) // max(N, 1)))


@functools.lru_cache(maxsize=1024)
def vocab_loss_workspace_size(N, D, V, dtype, backward, piece=None):
    n = _sz(0)
    piece = vocab_piece(N, V) if piece is None else max(0, min(piece, V))
    if (V | D) >> 31:
        _too_large()
    _check(library().slim_vocab_loss_workspace_size(N, D, V, DTYPES[dtype], piece, int(backward),
                                                    ctypes.byref(n)),
           "slim_vocab_loss_workspace_size")
    return n.value


def _loss_dims(x, w, targets, what):
    _require_cuda(x, w, targets)
    it, dt = _index_code(targets, "targets"), _dtype_code(x, what)
    if w.dtype != x.dtype:
        raise TypeError(f"{what}: one dtype expected, got {x.dtype} and {w.dtype}")
    shape, rows = w.shape, x.shape
    if len(shape) != 2 or rows[-1] != shape[1]:
        raise ValueError("x must be [..., D] and w [V, D]")
    if rows[:-1] != targets.shape:
        raise ValueError("targets must have one entry per row of x")
    V, D = shape
    if (V | D) >> 31:
        _too_large()
    return targets.numel(), D, V, it, dt


def vocab_loss_forward(x, w, targets, ignore_index=-100, workspace=None, stream=None):
    """slim_vocab_loss_fwd: softmax cross entropy of the rows of x [..., D]
    against the words w [V, D], without materialising the logits.  Returns
    (loss, lse, total): per row the loss (0 where the target is ignore_index)
    and the log-sum, both fp32 in targets' shape, and total = [sum of the
    losses, number of rows not ignored]."""
    N, D, V, it, dt = _loss_dims(x, w, targets, "vocab_loss_forward")
    if workspace is not None:
        _require_cuda(workspace)
    with _on(stream):
        dev = x.device
        loss = torch.empty(targets.shape, dtype=torch.float32, device=dev)
        lse = torch.empty_like(loss)
        total = torch.empty(2, dtype=torch.float32, device=dev)
        ws = workspace if workspace is not None else _workspace(
            vocab_loss_workspace_size(N, D, V, x.dtype, False), dev)
    _check(library().slim_vocab_loss_fwd(x.data_ptr(), w.data_ptr(), targets.data_ptr(), it, N, D,
                                         V, dt, ignore_index, loss.data_ptr(), lse.data_ptr(),
                                         total.data_ptr(), ws.data_ptr(), ws.numel(),
                                         _stream_of(x, stream)), "slim_vocab_loss_fwd")
    return loss, lse, total


def vocab_loss_backward(x, w, targets, lse, dloss, count=None, ignore_index=-100,
                        piece=None, workspace=None, stream=None):
    """slim_vocab_loss_bwd: returns (dx, dw), the gradients of sum_i c_i loss_i,
    c_i = dloss_i / count.  lse: from vocab_loss_forward on the same inputs.
    dloss: fp32 on the device, one value per row or a single one for all rows.
    count: None, or one fp32 value on the device (total[1:] of the forward for
    the mean loss).  Memory grows with rows x piece."""
    N, D, V, it, dt = _loss_dims(x, w, targets, "vocab_loss_backward")
    _require_cuda(lse, dloss)
    piece = vocab_piece(N, V) if piece is None else max(0, min(piece, V))
    per_row = dloss.numel()
    if lse.dtype != torch.float32 or lse.numel() != N:
        raise ValueError("lse must be the forward's")
    if dloss.dtype != torch.float32 or (per_row != 1 and per_row != N):
        raise ValueError("dloss must be fp32, one value or one per row")
    if count is not None:
        _require_cuda(count)
        _require(count.dtype == torch.float32 and count.numel() == 1, "count must be one fp32 value")
    if workspace is not None:
        _require_cuda(workspace)
    with _on(stream):
        dx, dw = torch.empty_like(x), torch.empty_like(w)
        ws = workspace if workspace is not None else _workspace(
            vocab_loss_workspace_size(N, D, V, x.dtype, True, piece), x.device)
    _check(library().slim_vocab_loss_bwd(x.data_ptr(), w.data_ptr(), targets.data_ptr(),
                                         it, lse.data_ptr(), dloss.data_ptr(), int(per_row > 1),
                                         _ptr(count), N, D, V, dt, piece, ignore_index,
                                         dx.data_ptr(), dw.data_ptr(), ws.data_ptr(), ws.numel(),
                                         _stream_of(x, stream)), "slim_vocab_loss_bwd")
    return dx, dw


class VocabLoss(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x_in, w_in, targets, reduction, ignore_index, piece):
        x, w, targets = _ready(x_in), _ready(w_in), targets.contiguous()
        loss, lse, total = vocab_loss_forward(x, w, targets, ignore_index)
        ctx.save_for_backward(x_in, w_in, x, w, targets, lse, total)
        ctx.mean, ctx.ignore_index, ctx.piece = reduction == "mean", ignore_index, piece
        if reduction == "none":
            return loss
        return total[0] / total[1] if ctx.mean else total[0].clone()

    @staticmethod
    def backward(ctx, dloss):
        x_in, w_in, x, w, targets, lse, total = ctx.saved_tensors
        grads = vocab_loss_backward(x, w, targets, lse, dloss.float().contiguous(),
                                    count=total[1:] if ctx.mean else None,
                                    ignore_index=ctx.ignore_index, piece=ctx.piece)
        return *_first_derivatives(grads, x_in, w_in, dloss), None, None, None, None


def vocab_loss(x, w, targets, reduction="mean", ignore_index=-100, piece=None):
    """Differentiable (once) softmax cross entropy of x [..., D] against the words w
    [V, D]; reduction "mean" (over the rows not ignored), "sum" or "none"."""
    _require(reduction in ("mean", "sum", "none"), "reduction must be 'mean', 'sum' or 'none'")
    return VocabLoss.apply(_ready(x), _ready(w), targets, reduction, ignore_index, piece)


# ---------------------------------------------------------------- around the attention
# A call's Python is most of a decoding step's time: what depends on sizes, strides and
# types alone is checked once for each of them and kept.
def _at(dev, stream):
    """The context in which a call allocates and launches: tensors' device as the current
    one, and what _on says of `stream`."""
    if stream is None:
        return _HERE if dev == torch._C._cuda_getDevice() else torch.cuda.device(dev)
    # (it makes the stream's device the current one, too)
    _require(stream.device_index == dev, "the stream is on another device than the tensors")
    return torch.cuda.stream(stream)


try:
    # (size, stride, dtype) on the current device, without the dispatcher: half of
    # torch.empty's time
    from torch._C import _len_torch_dispatch_stack as _modes
    from torch._C._dynamo.guards import _empty_strided_cuda as _undispatched
except ImportError:
    def _modes():
        return 1


def _allocate(size, stride, dtype):
    if _modes():  # modes that watch the dispatcher see every tensor
        return torch.empty_strided(size, stride, dtype=dtype, device="cuda")
    return _undispatched(size, stride, dtype)


@functools.lru_cache(maxsize=1024)
def _dense(shape):
    stride, n = [], 1
    for size in reversed(shape):
        stride.append(n)
        n *= max(size, 1)
    return tuple(shape), tuple(reversed(stride))


def _new(shape, dtype):
    """A contiguous tensor on the current device, to be written."""
    return _allocate(*_dense(shape), dtype)


def _raw(dev, stream):
    """The raw stream of a call on device `dev`: `stream`, or the current one."""
    return torch._C._cuda_getCurrentRawStream(dev) if stream is None else stream.cuda_stream


def _device_of(t, *others):
    """The index of the one device that CUDA tensors (None: left out) are on."""
    dev = t.get_device()
    cuda = dev >= 0
    for o in others:
        if o is not None and o.get_device() != dev:
            if cuda and o.is_cuda:
                raise ValueError("tensors on different devices")
            cuda = False
    if not cuda:
        raise RuntimeError("libslim runs on CUDA tensors only (no CPU fallback)")
    return dev


def _fp32_or_none(t, shape, what):
    if t is None:
        return None
    if t.dtype != torch.float32 or t.shape != shape or not t.is_contiguous():
        raise ValueError(f"{what} must be contiguous fp32 of shape {list(shape)}")
    return t.data_ptr()


def rotary_frequencies(rotary, base=10000.0):
    """Radians per position of the rotary / 2 pairs: base^(-2 p / rotary)."""
    _require(rotary >= 0 and rotary % 2 == 0, "rotary must be even")
    return array.array("d", [base ** (-2.0 * p / rotary) for p in range(rotary // 2)])


def _frequencies(inv_freq):
    """inv_freq, numbers or None, as an array of its own."""
    if isinstance(inv_freq, array.array) and inv_freq.typecode == "d":
        return inv_freq[:]
    if isinstance(inv_freq, torch.Tensor) and inv_freq.is_cuda:
        raise TypeError("inv_freq is read on the host: give numbers or a CPU tensor")
    return array.array("d", () if inv_freq is None else map(float, inv_freq))


@functools.lru_cache(maxsize=1024)
def _strides(stride, d):
    """A [B, H, L, d] tensor's slim_strides and their address; the last dimension is
    contiguous."""
    if stride[3] != 1 and d > 1:
        raise RuntimeError("libslim needs rows whose features are contiguous")
    a = array.array("q", stride[:3])
    return a, a.buffer_info()[0]


@functools.lru_cache(maxsize=1024)
def _qk_sizes(q, q_stride, k, k_stride, positions, rotary, dtype, k_dtype, what):
    """(B, Hq, Hk, L, d, dtype code) of checked shapes, and both sides' strides."""
    if len(q) != 4 or (k is not None and len(k) != 4):
        raise ValueError("q and k must be [B, H, L, d]")
    B, Hq, L, d = q
    Hk = 0 if k is None else k[1]
    if k is not None and (k_dtype != dtype or tuple(k) != (B, Hk, L, d)):
        raise ValueError("k must be [B, Hk, L, d] in q's dtype")
    if (B | Hq | Hk | L | d) >> 31:
        _too_large()
    _require(rotary <= d, "more frequencies than pairs of features")
    if positions is not None and tuple(positions) != (B, L):
        raise ValueError("positions must be contiguous [B, L]")
    if dtype not in DTYPES:
        raise TypeError(f"{what}: float32 or bfloat16 expected, got {dtype}")
    return ((B, Hq, Hk, L, d, DTYPES[dtype]), _strides(q_stride, d),
            (None, None) if k is None else _strides(k_stride, d))


def _qk_call(q, k, q_weight, k_weight, positions, inv_freq, what):
    """What both directions of qk_norm marshal alike: (device, sizes, the call's first
    arguments, what they point into)."""
    if not (isinstance(inv_freq, array.array) and inv_freq.typecode == "d"):
        inv_freq = _frequencies(inv_freq)
    rotary = 2 * len(inv_freq)
    at = positions is not None
    if k is None:
        plan = _qk_sizes(q.shape, q.stride(), None, None, positions.shape if at else None, rotary, q.dtype, None, what)
        kp = None
    else:
        plan = _qk_sizes(q.shape, q.stride(), k.shape, k.stride(), positions.shape if at else None, rotary, q.dtype,
                         k.dtype, what)
        kp = k.data_ptr()
    sizes, qs, ks = plan
    pp, ptype = None, 0
    if at:
        ptype = _index_code(positions, "positions")
        if not positions.is_contiguous():
            raise ValueError("positions must be contiguous [B, L]")
        pp = positions.data_ptr()
    weight = (sizes[4],)
    return (_device_of(q, k, q_weight, k_weight, positions), sizes,
            (q.data_ptr(), qs[1], kp, ks[1], _fp32_or_none(q_weight, weight, "q_weight"),
             _fp32_or_none(k_weight, weight, "k_weight"), pp, ptype, inv_freq.buffer_info()[0] if rotary else None,
             rotary), (plan, inv_freq))


def _qk_check(t, given, what):
    """`given` is like t, or None where t is."""
    if t is None or given.dtype != t.dtype or given.shape != t.shape:
        raise ValueError(f"{what} must have the shape and dtype of its input")
    _device_of(t, given)


def _qk_like(t, given, what):
    """(tensor, pointer, strides' address, strides): `given`, checked, or a new contiguous
    one like t (None without t)."""
    if given is not None:
        _qk_check(t, given, what)
        strides, address = _strides(given.stride(), t.shape[3])
        return given, given.data_ptr(), address, strides
    if t is None:
        return None, None, None, None
    out = _new(t.shape, t.dtype)
    return out, out.data_ptr(), None, None


def qk_norm_forward(q, k, q_weight=None, k_weight=None, positions=None, inv_freq=None, interleaved=False,
                    eps=1e-6, scale=1.0, q_out=None, k_out=None, stream=None):
    """slim_qk_norm_fwd: the root-mean-square norm of queries and keys per head,
    times scale and weight ([d] fp32 or None), and the rotation of their first
    2 * len(inv_freq) features by position.  q [B, Hq, L, d] and k [B, Hk, L, d]
    (or None) may be slices and transposes of a projection's rows as long as
    the features are contiguous.  positions: int [B, L], None counts from 0;
    inv_freq: radians per position on the host (see rotary_frequencies), None:
    no rotation.  Returns (q_out, k_out), contiguous unless given; they may be q
    and k themselves."""
    dev, sizes, head, kept = _qk_call(q, k, q_weight, k_weight, positions, inv_freq, "qk_norm_forward")
    with _at(dev, stream):
        q_out, qp, qs, q_strides = _qk_like(q, q_out, "q_out")
        k_out, kp, ks, k_strides = _qk_like(k, k_out, "k_out")
        status = library().slim_qk_norm_fwd(*head, int(interleaved), *sizes, eps, scale, qp, qs, kp, ks,
                                            _raw(dev, stream))
    _check(status, "slim_qk_norm_fwd")
    return q_out, k_out


@functools.lru_cache(maxsize=1024)
def qk_norm_workspace_size(B, Hq, Hk, L, d):
    n = _sz(0)
    if (B | Hq | Hk | L | d) >> 31:
        _too_large()
    _check(library().slim_qk_norm_bwd_workspace_size(B, Hq, Hk, L, d, ctypes.byref(n)),
           "slim_qk_norm_bwd_workspace_size")
    return n.value


def qk_norm_backward(q, k, q_weight, k_weight, dq_out, dk_out, positions=None, inv_freq=None,
                     interleaved=False, eps=1e-6, scale=1.0, dq=None, dk=None, weights=True,
                     workspace=None, stream=None):
    """slim_qk_norm_bwd: returns (dq, dk, dq_weight, dk_weight), the gradients of
    <dq_out, q_out> + <dk_out, k_out> for the same arguments as in the forward.
    dq and dk are contiguous unless given: slices of the projection's gradient,
    or dq_out and dk_out themselves.  A weight's gradient ([d] fp32) is None
    where there is no such weight or with weights=False."""
    dev, sizes, head, kept = _qk_call(q, k, q_weight, k_weight, positions, inv_freq, "qk_norm_backward")
    if dq_out is None or (k is not None and dk_out is None):
        raise ValueError("dq_out and dk_out are needed")
    _, up_qp, up_qs, q_above = _qk_like(q, dq_out, "dq_out")
    up_kp = up_ks = k_above = None
    if dk_out is not None:
        _, up_kp, up_ks, k_above = _qk_like(k, dk_out, "dk_out")
    if workspace is not None:
        _device_of(q, workspace)
        _require_cuda(workspace)
    with _at(dev, stream):
        dq, qp, qs, q_strides = _qk_like(q, dq, "dq")
        dk, kp, ks, k_strides = _qk_like(k, dk, "dk")
        dwq, dwk = (_new(w.shape, w.dtype) if weights and w is not None else None
                    for w in (q_weight, k_weight))
        ws = workspace if workspace is not None else _new((qk_norm_workspace_size(*sizes[:5]),), torch.uint8)
        status = library().slim_qk_norm_bwd(*head, int(interleaved), *sizes, eps, scale, up_qp, up_qs, up_kp, up_ks,
                                            qp, qs, kp, ks, _ptr(dwq), _ptr(dwk), ws.data_ptr(), ws.numel(),
                                            _raw(dev, stream))
    _check(status, "slim_qk_norm_bwd")
    return dq, dk, dwq, dwk


def _dense_rows(t):
    """t with contiguous features: itself, or a copy."""
    return t if t is None or t.stride(-1) == 1 or t.shape[-1] == 1 else t.contiguous()


class QkNorm(torch.autograd.Function):
    @staticmethod
    def forward(ctx, q, k, q_weight, k_weight, positions, inv_freq, interleaved, eps, scale):
        ctx.save_for_backward(q, k, q_weight, k_weight, positions)
        ctx.how = dict(inv_freq=inv_freq, interleaved=interleaved, eps=eps, scale=scale)
        q_out, k_out = qk_norm_forward(_dense_rows(q), _dense_rows(k), q_weight, k_weight,
                                       positions=positions, **ctx.how)
        return q_out, k_out

    @staticmethod
    def backward(ctx, dq_out, dk_out):
        q, k, q_weight, k_weight, positions = ctx.saved_tensors
        grads = qk_norm_backward(_dense_rows(q), _dense_rows(k), q_weight, k_weight,
                                 _dense_rows(dq_out), _dense_rows(dk_out), positions=positions,
                                 weights=any(ctx.needs_input_grad[2:4]), **ctx.how)
        there = [i for i, g in enumerate(grads) if g is not None]
        tied = _first_derivatives(tuple(grads[i] for i in there), *(
            t for t in (q, k, q_weight, k_weight, dq_out, dk_out) if t is not None))
        out = [None] * 4
        for i, g in zip(there, tied):
            out[i] = g
        return *out, None, None, None, None, None


def qk_norm(q, k, q_weight=None, k_weight=None, positions=None, inv_freq=None, interleaved=False,
            eps=1e-6, scale=1.0):
    """Differentiable (once) qk_norm_forward: gradients with respect to q, k and the weights.
    inv_freq is read once, for both directions; positions may be one row expanded."""
    if positions is not None:
        positions = positions.contiguous()
    return QkNorm.apply(q, k, q_weight, k_weight, positions, _frequencies(inv_freq), interleaved, eps, scale)


GATES = {"value": 0, "log": 1, "sigmoid": 2}
SCAN_CHUNK = 64


@functools.lru_cache(maxsize=1024)
def _pitch(shape, stride, what):
    """Elements from a row of [B, L, D] to the next; a slice of wider rows has one, too."""
    B, L, D = shape
    b, l, one = stride
    if D > 1 and one != 1:
        raise RuntimeError(f"{what}: libslim needs rows whose channels are contiguous")
    if L > 1:
        pitch, whole = l, B <= 1 or b == L * l
    else:
        pitch, whole = (b if B > 1 else D), True
    if not whole:
        raise RuntimeError(f"{what}: libslim needs rows at one distance from each other")
    return pitch


@functools.lru_cache(maxsize=1024)
def _scan_sizes(gate, x, gate_stride, x_stride, gate_dtype, dtype, kind, what):
    """(B, L, D, dtype code, kind code) of checked shapes, and both inputs' pitches."""
    if len(gate) != 3 or gate != x:
        raise ValueError("gate and x must be [B, L, D]")
    if gate_dtype != dtype:
        raise TypeError(f"{what}: one dtype expected, got {gate_dtype} and {dtype}")
    if dtype not in DTYPES:
        raise TypeError(f"{what}: float32 or bfloat16 expected, got {dtype}")
    _require(kind in GATES, f"kind must be one of {', '.join(GATES)}")
    B, L, D = gate
    if (B | L | D) >> 31:
        _too_large()
    return (B, L, D, DTYPES[dtype], GATES[kind]), _pitch(gate, gate_stride, "gate"), _pitch(x, x_stride, "x")


@functools.lru_cache(maxsize=1024)
def gated_scan_workspace_size(B, L, D, dtype):
    n = _sz(0)
    _check(library().slim_gated_scan_workspace_size(B, L, D, DTYPES[dtype], ctypes.byref(n)),
           "slim_gated_scan_workspace_size")
    return n.value


def _scan_workspace(given, sizes, t):
    """(tensor or None, pointer, bytes): short sequences need none."""
    if given is None:
        need = gated_scan_workspace_size(*sizes[:3], t.dtype)
        if not need:
            return None, None, 0
        given = _new((need,), torch.uint8)
    else:
        _device_of(t, given)
        _require_cuda(given)
    return given, given.data_ptr(), given.numel()


def gated_scan_forward(gate, x, kind="sigmoid", h0=None, keep=False, last=None, workspace=None, stream=None):
    """slim_gated_scan_fwd: h_t = a_t h_(t-1) + u_t per channel, gate and x [B, L, D]
    (slices of a projection's rows are read where they are).  kind "value": a =
    gate, u = x; "log": a = exp(gate), u = x; "sigmoid": a = sigmoid(gate), u =
    (1 - a) x.  h0: the state to start from, [B, D] fp32 or None (zero).  Returns
    (h, last): all states in x's dtype and the last in fp32 (into `last` if given,
    which may be h0); with keep=True also what gated_scan_backward needs.  Gates beyond 1
    whose product over up to 128 steps passes fp32's range make a state that is not zero
    infinite or NaN, even where it alone would not have left that range."""
    sizes, gp, xp = _scan_sizes(gate.shape, x.shape, gate.stride(), x.stride(), gate.dtype, x.dtype, kind,
                                "gated_scan_forward")
    B, L, D, _, _ = sizes
    dev = _device_of(x, gate, h0, last)
    h0p = _fp32_or_none(h0, (B, D), "h0")
    lastp = _fp32_or_none(last, (B, D), "last")
    kept = None
    with _at(dev, stream):
        h = _new(x.shape, x.dtype)
        if last is None:
            last = _new((B, D), torch.float32)
            lastp = last.data_ptr()
        if keep:
            kept = _new((B, -(-L // SCAN_CHUNK), D), torch.float32)
        ws, wsp, nbytes = _scan_workspace(workspace, sizes, x)
        status = library().slim_gated_scan_fwd(gate.data_ptr(), gp, x.data_ptr(), xp, h0p, *sizes, h.data_ptr(),
                                               lastp, _ptr(kept), wsp, nbytes, _raw(dev, stream))
    _check(status, "slim_gated_scan_fwd")
    return (h, last, kept) if keep else (h, last)


def gated_scan_backward(gate, x, kept, dh, kind="sigmoid", dlast=None, dgate=None, dx=None, dh0=None,
                        workspace=None, stream=None):
    """slim_gated_scan_bwd: returns (dgate, dx, dh0), the gradients of <dh, h> +
    <dlast, last>.  kept: from gated_scan_forward(..., keep=True) on the same inputs;
    dlast: [B, D] fp32 or None (zero).  dgate and dx are contiguous unless given
    (slices of the projection's gradient, or gate and x themselves); dh0 may be given, too,
    also as dlast."""
    sizes, gp, xp = _scan_sizes(gate.shape, x.shape, gate.stride(), x.stride(), gate.dtype, x.dtype, kind,
                                "gated_scan_backward")
    B, L, D, _, _ = sizes
    if kept is None:
        raise ValueError("kept must be the forward's")
    dev = _device_of(x, gate, kept, dh, dlast, dgate, dx, dh0)
    if dh.shape != x.shape or dh.dtype != x.dtype or not dh.is_contiguous():
        raise ValueError("dh must be contiguous [B, L, D] in x's dtype")
    dlp = _fp32_or_none(dlast, (B, D), "dlast")
    _fp32_or_none(dh0, (B, D), "dh0")
    keptp = _fp32_or_none(kept, (B, -(-L // SCAN_CHUNK), D), "kept")
    for t in (dgate, dx):
        if t is not None and (t.shape != x.shape or t.dtype != x.dtype):
            raise ValueError("dgate and dx must be [B, L, D] in x's dtype")
    dgp = D if dgate is None else _pitch(dgate.shape, dgate.stride(), "dgate")
    dxp = D if dx is None else _pitch(dx.shape, dx.stride(), "dx")
    with _at(dev, stream):
        if dgate is None:
            dgate = _new(x.shape, x.dtype)
        if dx is None:
            dx = _new(x.shape, x.dtype)
        if dh0 is None:
            dh0 = _new((B, D), torch.float32)
        ws, wsp, nbytes = _scan_workspace(workspace, sizes, x)
        status = library().slim_gated_scan_bwd(gate.data_ptr(), gp, x.data_ptr(), xp, keptp, dh.data_ptr(), dlp,
                                               *sizes, dgate.data_ptr(), dgp, dx.data_ptr(), dxp, dh0.data_ptr(),
                                               wsp, nbytes, _raw(dev, stream))
    _check(status, "slim_gated_scan_bwd")
    return dgate, dx, dh0


def _even_rows(t):
    """t with contiguous channels and its rows at one distance: itself, or a copy."""
    try:
        return t if _pitch(t.shape, t.stride(), "") >= 0 else t.contiguous()
    except RuntimeError:
        return t.contiguous()


def _wants_gradients(*ts):
    """Whether a differentiable call is recorded (a Function's ctx.needs_input_grad goes by
    its inputs alone, under torch.no_grad, too)."""
    return torch.is_grad_enabled() and any(t is not None and t.requires_grad for t in ts)


class GatedScan(torch.autograd.Function):
    @staticmethod
    def forward(ctx, gate, x, kind, h0, keep=True):
        h, last, *kept = gated_scan_forward(_even_rows(gate), _even_rows(x), kind,
                                            None if h0 is None else h0.contiguous(), keep=keep)
        ctx.save_for_backward(gate, x, h0, *kept)
        ctx.kind = kind
        return h, last

    @staticmethod
    def backward(ctx, dh, dlast):
        gate, x, h0, kept = ctx.saved_tensors
        grads = gated_scan_backward(_even_rows(gate), _even_rows(x), kept, dh.contiguous(), ctx.kind,
                                    dlast=dlast.contiguous())
        if h0 is None:
            grads = grads[:2]
        tied = _first_derivatives(grads, *(t for t in (gate, x, h0, dh, dlast) if t is not None))
        return tied[0], tied[1], None, (tied[2] if h0 is not None else None), None


def gated_scan(gate, x, kind="sigmoid", h0=None):
    """Differentiable (once) gated_scan_forward: returns (h, last), with gradients with
    respect to gate, x and h0."""
    return GatedScan.apply(gate, x, kind, h0, _wants_gradients(gate, x, h0))


ACTIVATIONS = {"silu": 0, "gelu": 1, "gelu_tanh": 2, "relu": 3, "sigmoid": 4}


@functools.lru_cache(maxsize=1024)
def gated_ff_workspace_size(N, D, F, dtype, backward):
    n = _sz(0)
    if (D | F) >> 31:
        _too_large()
    _check(library().slim_gated_ff_workspace_size(N, D, F, DTYPES[dtype], int(backward), ctypes.byref(n)),
           "slim_gated_ff_workspace_size")
    return n.value


@functools.lru_cache(maxsize=1024)
def _ff_sizes(x, w, dtype, w_dtype, act, what):
    """(N, D, F, dtype code, act code) of checked shapes."""
    if w_dtype != dtype:
        raise TypeError(f"{what}: one dtype expected, got {dtype} and {w_dtype}")
    if dtype not in DTYPES:
        raise TypeError(f"{what}: float32 or bfloat16 expected, got {dtype}")
    if len(w) != 2 or w[0] % 2 or len(x) < 1 or x[-1] != w[1]:
        raise ValueError("x must be [..., D] and w [2F, D]")
    _require(act in ACTIVATIONS, f"act must be one of {', '.join(ACTIVATIONS)}")
    F, D = w[0] // 2, w[1]
    if (D | F) >> 31:
        _too_large()
    return math.prod(x[:-1]), D, F, DTYPES[dtype], ACTIVATIONS[act]


@functools.lru_cache(maxsize=1024)
def gated_ff_kept_size(N, D, F, dtype):
    """Bytes of both projections where keeping them makes the backward quicker, else 0."""
    n = _sz(0)
    _check(library().slim_gated_ff_kept_size(N, D, F, DTYPES[dtype], ctypes.byref(n)), "slim_gated_ff_kept_size")
    return n.value


def _ff_workspace(given, sizes, t, backward):
    """(tensor or None, pointer, bytes): a few rows need none."""
    if given is None:
        need = gated_ff_workspace_size(*sizes[:3], t.dtype, backward)
        if not need:
            return None, None, 0
        given = _new((need,), torch.uint8)
    return given, given.data_ptr(), given.numel()


def _apart(a, b):
    """Whether contiguous tensors share no memory."""
    return a.data_ptr() + a.nbytes <= b.data_ptr() or b.data_ptr() + b.nbytes <= a.data_ptr()


def gated_ff_forward(x, w, act="silu", keep=False, out=None, workspace=None, stream=None):
    """slim_gated_ff_fwd: act(x w_gate^T) * (x w_up^T) for x [..., D] and w [2F, D], its
    first F rows the gate's and the others up's; act one of "silu", "gelu",
    "gelu_tanh", "relu", "sigmoid".  With keep=True returns (h, z), z being both
    projections in fp32 for gated_ff_backward, or None where computing them again is
    the quicker (bf16, and a few rows: see gated_ff_kept_size)."""
    dev = _device_of(x, w, out, workspace)
    _require_cuda(x, w)
    sizes = _ff_sizes(x.shape, w.shape, x.dtype, w.dtype, act, "gated_ff_forward")
    shape = (*x.shape[:-1], sizes[2])
    if out is not None:
        _require_cuda(out)
        _require(out.dtype == x.dtype and out.shape == shape, "out must be [..., F] in x's dtype")
        _require(_apart(out, x) and _apart(out, w), "out must not share memory with x or w")
    if workspace is not None:
        _require_cuda(workspace)
    with _at(dev, stream):
        h = out if out is not None else _new(shape, x.dtype)
        z = None
        if keep:
            need = gated_ff_kept_size(*sizes[:3], x.dtype)
            z = _new((need // 4,), torch.float32) if need else None
        ws, wsp, nbytes = _ff_workspace(workspace, sizes, x, False)
        status = library().slim_gated_ff_fwd(x.data_ptr(), w.data_ptr(), *sizes, h.data_ptr(), _ptr(z), wsp,
                                             nbytes, _raw(dev, stream))
    _check(status, "slim_gated_ff_fwd")
    return (h, z) if keep else h


def gated_ff_backward(x, w, dh, act="silu", z=None, workspace=None, stream=None):
    """slim_gated_ff_bwd: returns (dx, dw), the gradients of <dh, h>.  z: from
    gated_ff_forward(..., keep=True) on the same inputs, or None.  The gradients of bf16
    projections are rounded to bf16 before their two products."""
    dev = _device_of(x, w, dh, z, workspace)
    _require_cuda(x, w, dh)
    sizes = _ff_sizes(x.shape, w.shape, x.dtype, w.dtype, act, "gated_ff_backward")
    if dh.shape != (*x.shape[:-1], sizes[2]) or dh.dtype != x.dtype:
        raise ValueError("dh must be [..., F] in x's dtype")
    zp = None if z is None else _fp32_or_none(z, (gated_ff_kept_size(*sizes[:3], x.dtype) // 4,), "z")
    if workspace is not None:
        _require_cuda(workspace)
    with _at(dev, stream):
        dx, dw = _new(x.shape, x.dtype), _new(w.shape, w.dtype)
        ws, wsp, nbytes = _ff_workspace(workspace, sizes, x, True)
        status = library().slim_gated_ff_bwd(x.data_ptr(), w.data_ptr(), dh.data_ptr(), *sizes, zp, dx.data_ptr(),
                                             dw.data_ptr(), wsp, nbytes, _raw(dev, stream))
    _check(status, "slim_gated_ff_bwd")
    return dx, dw


class GatedFeedForward(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x_in, w_in, act, keep=True):
        x, w = _ready(x_in), _ready(w_in)
        h, z = gated_ff_forward(x, w, act, keep=True) if keep else (gated_ff_forward(x, w, act), None)
        ctx.save_for_backward(x_in, w_in, x, w, z)
        ctx.act = act
        return h

    @staticmethod
    def backward(ctx, dh):
        x_in, w_in, x, w, z = ctx.saved_tensors
        grads = gated_ff_backward(x, w, _ready(dh), ctx.act, z=z)
        return *_first_derivatives(grads, x_in, w_in, dh), None, None


def gated_ff(x, w, act="silu"):
    """Differentiable (once) gated_ff_forward: gradients with respect to x and w.  Where one
    is wanted, fp32 keeps both projections (8 F bytes a row) for the backward."""
    return GatedFeedForward.apply(x, w, act, _wants_gradients(x, w))
