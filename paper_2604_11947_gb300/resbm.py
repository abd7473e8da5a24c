"""Python binding of the C ABI in include/resbm.h, include/resbm_train.h and include/resbm_vocab.h (libresbm.so).

Argument marshalling only: every function here has the C function's name, takes torch tensors
(device memory owned by the caller) or None, passes their data pointers and the current CUDA
stream, and raises ResbmError when the C call returns a status other than RESBM_OK. No compute
happens in Python, and there is no fallback: if libresbm.so cannot be loaded, every call raises.
"""
from __future__ import annotations

import ctypes
import os

import torch

from . import build as _build

RESBM_OK, RESBM_ERR_INVALID_ARG, RESBM_ERR_UNSUPPORTED, RESBM_ERR_WORKSPACE, RESBM_ERR_CUDA = range(5)
RESBM_F32, RESBM_BF16 = 0, 1
RESBM_ACT_SILU, RESBM_ACT_GELU_TANH, RESBM_ACT_IDENTITY = 0, 1, 2
(RESBM_OP_ENCODE_FWD, RESBM_OP_DECODE_FWD, RESBM_OP_DECODE_BWD, RESBM_OP_ENCODE_BWD,
 RESBM_OP_BOUNDARY_STEP, RESBM_OP_BOUNDARY_STEP_HOST, RESBM_OP_EFFECTIVE_RANK, RESBM_OP_NEWTON_SCHULZ,
 RESBM_OP_DECODE_FWD_RMSNORM, RESBM_OP_RMSNORM_BWD) = range(10)
(RESBM_HBM_READ_V4, RESBM_HBM_WRITE_V4, RESBM_HBM_COPY_V4, RESBM_HBM_READ_TMA_2D, RESBM_HBM_READ_TMA_2D_PAIR,
 RESBM_HBM_READ_TMA_3D, RESBM_HBM_READ_BULK, RESBM_HBM_WRITE_TMA_2D, RESBM_HBM_WRITE_BULK,
 RESBM_HBM_READ_TMA_2D_TILES, RESBM_HBM_WRITE_TMA_2D_TILES) = range(11)
HBM_FORMS = {"read_v4": RESBM_HBM_READ_V4, "write_v4": RESBM_HBM_WRITE_V4, "copy_v4": RESBM_HBM_COPY_V4,
             "read_tma_2d": RESBM_HBM_READ_TMA_2D, "read_tma_2d_pair": RESBM_HBM_READ_TMA_2D_PAIR,
             "read_tma_3d": RESBM_HBM_READ_TMA_3D, "read_bulk": RESBM_HBM_READ_BULK,
             "write_tma_2d": RESBM_HBM_WRITE_TMA_2D, "write_bulk": RESBM_HBM_WRITE_BULK,
             "read_tma_2d_tiles": RESBM_HBM_READ_TMA_2D_TILES, "write_tma_2d_tiles": RESBM_HBM_WRITE_TMA_2D_TILES}
RESBM_FLAG_GENERIC = 1
RESBM_FLAG_LINEAR = 2
RESBM_FLAG_GEMM = 4
RESBM_STATIC_SCRATCH_BYTES = 32 << 20

ACTS = {"silu": RESBM_ACT_SILU, "gelu_tanh": RESBM_ACT_GELU_TANH, "identity": RESBM_ACT_IDENTITY}
DTYPES = {"f32": RESBM_F32, "bf16": RESBM_BF16}
TORCH_DTYPES = {RESBM_F32: torch.float32, RESBM_BF16: torch.bfloat16}

EXPORTS = ("resbm_version", "resbm_status_string", "resbm_last_cuda_error", "resbm_kernel_launches",
           "resbm_device_error",
           "resbm_workspace_bytes", "resbm_encode_fwd", "resbm_decode_fwd", "resbm_decode_bwd",
           "resbm_encode_bwd", "resbm_boundary_step", "resbm_boundary_step_host",
           "resbm_decode_bwd_noalloc", "resbm_selftest_wait_timeout", "resbm_matrix_workspace_bytes",
           "resbm_newton_schulz", "resbm_effective_rank", "resbm_ffn_down_encode_workspace_bytes",
           "resbm_ffn_down_encode_fwd", "resbm_decode_fwd_rmsnorm", "resbm_rmsnorm_bwd",
           "resbm_measure_hbm_form")
# the functions of include/resbm_train.h
TRAIN_EXPORTS = ("resbm_add_rmsnorm_fwd", "resbm_adamw_plan_bytes", "resbm_adamw_plan", "resbm_adamw_step",
                 "resbm_grad_norm_workspace_bytes", "resbm_grad_norm")
# the functions of include/resbm_vocab.h
VOCAB_EXPORTS = ("resbm_vocab_workspace_bytes", "resbm_linear_ce_fwd", "resbm_linear_ce_bwd", "resbm_distill_fwd",
                 "resbm_distill_bwd", "resbm_embed_fwd", "resbm_embed_bwd")
(RESBM_VOCAB_CE_FWD, RESBM_VOCAB_CE_BWD, RESBM_VOCAB_DISTILL_FWD, RESBM_VOCAB_DISTILL_BWD, RESBM_VOCAB_EMBED_BWD) = range(5)
RESBM_STATE_NONE, RESBM_STATE_E4M3, RESBM_STATE_F32 = 0, 8, 32
RESBM_STATE_BLOCK = 256


class resbm_desc(ctypes.Structure):
    _fields_ = [("T", ctypes.c_int64), ("d", ctypes.c_int64), ("r", ctypes.c_int64),
                ("m", ctypes.c_int64), ("dtype", ctypes.c_int32), ("act", ctypes.c_int32),
                ("merge_identity", ctypes.c_int32), ("flags", ctypes.c_uint32)]


class resbm_step_args(ctypes.Structure):
    _fields_ = [(n, ctypes.c_void_p) for n in
                ("X", "F", "dY", "We1", "We2", "Wd1", "Wd2", "B", "P", "Y", "dB", "dF", "dX",
                 "dWe1", "dWe2", "dWd1", "dWd2", "wait_before_inputs", "inputs_done")]


class resbm_add_norm_desc(ctypes.Structure):
    _fields_ = [("T", ctypes.c_int64), ("d", ctypes.c_int64), ("ldx", ctypes.c_int64), ("lda", ctypes.c_int64),
                ("ldh", ctypes.c_int64), ("ldn", ctypes.c_int64), ("dtype", ctypes.c_int32),
                ("q_group", ctypes.c_int32), ("eps", ctypes.c_float), ("flags", ctypes.c_uint32)]


class resbm_adamw_desc(ctypes.Structure):
    _fields_ = [("w_dtype", ctypes.c_int32), ("g_dtype", ctypes.c_int32), ("state", ctypes.c_int32),
                ("flags", ctypes.c_uint32)]


class resbm_adamw_tensor(ctypes.Structure):
    _fields_ = [(n, ctypes.c_void_p) for n in ("w", "g", "m", "v", "m_scale", "v_scale", "master")] + [("n", ctypes.c_int64)]


class resbm_adamw_hyper(ctypes.Structure):
    _fields_ = [(n, ctypes.c_double) for n in ("lr", "beta1", "beta2", "eps", "weight_decay")] + \
               [("step", ctypes.c_int64)] + [(n, ctypes.c_void_p) for n in ("lr_dev", "step_dev", "grad_scale")]


class resbm_vocab_desc(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int64) for n in ("T", "V", "d", "ldx", "ldw", "K")] + \
               [("dtype", ctypes.c_int32), ("teacher_dtype", ctypes.c_int32), ("temperature", ctypes.c_float),
                ("dloss_each", ctypes.c_int32), ("flags", ctypes.c_uint32)]


class resbm_embed_desc(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int64) for n in ("T", "V", "d", "ldt", "ldo", "padding")] + \
               [("dtype", ctypes.c_int32), ("scale", ctypes.c_float), ("flags", ctypes.c_uint32)]


class ResbmError(RuntimeError):
    def __init__(self, fn, status, cuda_error=0):
        self.status, self.cuda_error = status, cuda_error
        msg = "%s failed: %s" % (fn, status_string(status))
        if status == RESBM_ERR_CUDA:
            msg += " (cudaError %d)" % cuda_error
        super().__init__(msg)


_lib = None


def library_path() -> str:
    return _build.LIB


def load(path: str | None = None) -> ctypes.CDLL:
    """Load libresbm.so (built in-tree by build.build()); raise if it is missing."""
    global _lib
    if _lib is not None and path is None:
        return _lib
    p = path or _build.LIB
    if not os.path.exists(p):
        raise RuntimeError("libresbm.so not found at %s: run paper_2604_11947_gb300.build.build() "
                           "(there is no CPU fallback)" % p)
    lib = ctypes.CDLL(p)
    vp, sz, i32 = ctypes.c_void_p, ctypes.c_size_t, ctypes.c_int
    D = ctypes.POINTER(resbm_desc)
    lib.resbm_version.restype = ctypes.c_char_p
    lib.resbm_status_string.restype = ctypes.c_char_p
    lib.resbm_status_string.argtypes = [i32]
    lib.resbm_last_cuda_error.restype = i32
    lib.resbm_kernel_launches.restype = ctypes.c_uint64
    lib.resbm_device_error.restype = i32
    lib.resbm_device_error.argtypes = [ctypes.POINTER(ctypes.c_uint), i32]
    lib.resbm_workspace_bytes.restype = i32
    lib.resbm_workspace_bytes.argtypes = [D, i32, ctypes.POINTER(sz)]
    lib.resbm_encode_fwd.restype = i32
    lib.resbm_encode_fwd.argtypes = [D] + [vp] * 6 + [vp, sz, vp]
    lib.resbm_decode_fwd.restype = i32
    lib.resbm_decode_fwd.argtypes = [D] + [vp] * 4 + [vp, sz, vp]
    lib.resbm_rmsnorm_bwd.restype = i32
    lib.resbm_rmsnorm_bwd.argtypes = [D, vp, vp, ctypes.c_float] + [vp] * 4 + [vp, sz, vp]
    lib.resbm_decode_fwd_rmsnorm.restype = i32
    lib.resbm_decode_fwd_rmsnorm.argtypes = [D] + [vp] * 4 + [ctypes.c_float] + [vp] * 2 + [vp, sz, vp]
    lib.resbm_decode_bwd.restype = i32
    lib.resbm_decode_bwd.argtypes = [D] + [vp] * 7 + [vp, sz, vp]
    lib.resbm_encode_bwd.restype = i32
    lib.resbm_encode_bwd.argtypes = [D] + [vp] * 9 + [vp, sz, vp]
    lib.resbm_boundary_step.restype = i32
    lib.resbm_selftest_wait_timeout.restype = i32
    lib.resbm_selftest_wait_timeout.argtypes = [vp]
    lib.resbm_decode_bwd_noalloc.restype = i32
    lib.resbm_decode_bwd_noalloc.argtypes = [D] + [vp] * 7 + [vp]
    lib.resbm_boundary_step.argtypes = [D, ctypes.POINTER(resbm_step_args), vp, sz, vp]
    lib.resbm_boundary_step_host.restype = i32
    lib.resbm_boundary_step_host.argtypes = [D, ctypes.POINTER(resbm_step_args), vp, sz, vp]
    i64 = ctypes.c_int64
    lib.resbm_matrix_workspace_bytes.restype = i32
    lib.resbm_matrix_workspace_bytes.argtypes = [i32, i64, i64, ctypes.POINTER(sz)]
    lib.resbm_newton_schulz.restype = i32
    lib.resbm_newton_schulz.argtypes = [i64, i64, vp, ctypes.c_int32, ctypes.c_int32, vp, vp, sz, vp]
    lib.resbm_effective_rank.restype = i32
    lib.resbm_effective_rank.argtypes = [i64, i64, vp, vp, vp, sz, vp]
    lib.resbm_ffn_down_encode_workspace_bytes.restype = i32
    lib.resbm_ffn_down_encode_workspace_bytes.argtypes = [D, i64, ctypes.POINTER(sz)]
    lib.resbm_ffn_down_encode_fwd.restype = i32
    lib.resbm_ffn_down_encode_fwd.argtypes = [D, i64] + [vp] * 8 + [vp, sz, vp]
    lib.resbm_measure_hbm_form.restype = i32
    lib.resbm_measure_hbm_form.argtypes = [i32, vp, vp, i64, vp]
    lib.resbm_add_rmsnorm_fwd.restype = i32
    lib.resbm_add_rmsnorm_fwd.argtypes = [ctypes.POINTER(resbm_add_norm_desc)] + [vp] * 8
    lib.resbm_adamw_plan_bytes.restype = i32
    lib.resbm_adamw_plan_bytes.argtypes = [i64, ctypes.POINTER(sz)]
    lib.resbm_adamw_plan.restype = i32
    lib.resbm_adamw_plan.argtypes = [ctypes.POINTER(resbm_adamw_desc), ctypes.POINTER(resbm_adamw_tensor), i64, vp, sz]
    lib.resbm_adamw_step.restype = i32
    lib.resbm_adamw_step.argtypes = [vp, ctypes.POINTER(resbm_adamw_hyper), vp]
    lib.resbm_grad_norm_workspace_bytes.restype = i32
    lib.resbm_grad_norm_workspace_bytes.argtypes = [ctypes.POINTER(vp), i64, ctypes.POINTER(sz)]
    lib.resbm_grad_norm.restype = i32
    lib.resbm_grad_norm.argtypes = [ctypes.POINTER(vp), i64, ctypes.c_float, vp, vp, sz, vp]
    lib.resbm_vocab_workspace_bytes.restype = i32
    lib.resbm_vocab_workspace_bytes.argtypes = [ctypes.POINTER(resbm_vocab_desc), i32, ctypes.POINTER(sz)]
    for name, tensors in (("linear_ce_fwd", 5), ("linear_ce_bwd", 7), ("distill_fwd", 6), ("distill_bwd", 8)):
        f = getattr(lib, "resbm_" + name)
        f.restype = i32
        f.argtypes = [ctypes.POINTER(resbm_vocab_desc)] + [vp] * tensors + [vp, sz, vp]
    lib.resbm_embed_fwd.restype = i32
    lib.resbm_embed_fwd.argtypes = [ctypes.POINTER(resbm_embed_desc)] + [vp] * 4
    lib.resbm_embed_bwd.restype = i32
    lib.resbm_embed_bwd.argtypes = [ctypes.POINTER(resbm_embed_desc)] + [vp] * 3 + [vp, sz, vp]
    if path is None:
        _lib = lib
    return lib


def status_string(status: int) -> str:
    return load().resbm_status_string(int(status)).decode()


def resbm_version() -> str:
    return load().resbm_version().decode()


def resbm_kernel_launches() -> int:
    return int(load().resbm_kernel_launches())


def resbm_device_error(clear=False) -> int:
    """The tensor-core kernels' error word (synchronizes with the device)."""
    out = ctypes.c_uint(0)
    _check("resbm_device_error", load().resbm_device_error(ctypes.byref(out), int(bool(clear))))
    return int(out.value)


def resbm_selftest_wait_timeout(stream=None):
    """Enqueue the failure-path self-test kernel (a wait that gives up after ~2 s)."""
    _check("resbm_selftest_wait_timeout", load().resbm_selftest_wait_timeout(_stream(stream)))


def resbm_measure_hbm_form(form, a, b, stream=None):
    """One launch of an HBM access-form probe (resbm_hbm_form; a name of HBM_FORMS or its value)
    over a's bytes: a read, b written; both device tensors of the same byte size."""
    f = HBM_FORMS[form] if isinstance(form, str) else int(form)
    n = _nbytes(a)
    if _nbytes(b) != n:
        raise ValueError("a and b must have the same byte size")
    _check("resbm_measure_hbm_form", load().resbm_measure_hbm_form(f, _p(a), _p(b), n, _stream(stream)))


def make_desc(T, d, r, m, dtype="bf16", act="silu", merge_identity=1, flags=0) -> resbm_desc:
    dt = DTYPES[dtype] if isinstance(dtype, str) else int(dtype)
    a = ACTS[act] if isinstance(act, str) else int(act)
    return resbm_desc(int(T), int(d), int(r), int(m), dt, a, int(merge_identity), int(flags))


def desc_from_config(cfg, flags=0) -> resbm_desc:
    return make_desc(cfg.T, cfg.d, cfg.r, cfg.m, cfg.dtype, cfg.act, cfg.merge, flags)


def resbm_workspace_bytes(desc: resbm_desc, op: int) -> int:
    out = ctypes.c_size_t(0)
    st = load().resbm_workspace_bytes(ctypes.byref(desc), int(op), ctypes.byref(out))
    if st != RESBM_OK:
        raise ResbmError("resbm_workspace_bytes", st)
    return int(out.value)


def workspace(desc: resbm_desc, op: int, device="cuda") -> torch.Tensor:
    """A torch-owned scratch buffer of the size the C ABI asks for (allocated by torch)."""
    n = resbm_workspace_bytes(desc, op)
    return torch.empty(max(n, 1), dtype=torch.uint8, device=device)


def _p(t):
    """The address of a tensor's data (an int is an address already, None stays None)."""
    try:
        return t.data_ptr()
    except AttributeError:
        if t is None or isinstance(t, int):
            return t
        raise


def _nbytes(t):
    return 0 if t is None else t.numel() * t.element_size()


# The current stream's handle without building a torch.cuda.Stream around it (3 us a call on the host;
# a small step's launches take ~20), where this torch has the accessor.
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)


def _stream(stream):
    if stream is None:
        if _raw_stream is not None:
            return _raw_stream(torch.cuda.current_device())
        return torch.cuda.current_stream().cuda_stream
    return stream if isinstance(stream, int) else stream.cuda_stream


def _check(fn, st):
    if st != RESBM_OK:
        raise ResbmError(fn, st, load().resbm_last_cuda_error() if st == RESBM_ERR_CUDA else 0)


def resbm_encode_fwd(desc, X, F, We1, We2, B, P_save, ws, stream=None):
    st = load().resbm_encode_fwd(ctypes.byref(desc), _p(X), _p(F), _p(We1), _p(We2), _p(B),
                                 _p(P_save), _p(ws), _nbytes(ws), _stream(stream))
    _check("resbm_encode_fwd", st)


def resbm_decode_fwd(desc, B, Wd1, Wd2, Y, ws, stream=None):
    st = load().resbm_decode_fwd(ctypes.byref(desc), _p(B), _p(Wd1), _p(Wd2), _p(Y), _p(ws),
                                 _nbytes(ws), _stream(stream))
    _check("resbm_decode_fwd", st)


def resbm_decode_fwd_rmsnorm(desc, B, Wd1, Wd2, gamma, eps, Y, N, ws, stream=None):
    st = load().resbm_decode_fwd_rmsnorm(ctypes.byref(desc), _p(B), _p(Wd1), _p(Wd2), _p(gamma), float(eps),
                                         _p(Y), _p(N), _p(ws), _nbytes(ws), _stream(stream))
    _check("resbm_decode_fwd_rmsnorm", st)


def resbm_rmsnorm_bwd(desc, Y, gamma, eps, dN, dY, dY_out, dgamma, ws, stream=None):
    st = load().resbm_rmsnorm_bwd(ctypes.byref(desc), _p(Y), _p(gamma), float(eps), _p(dN), _p(dY), _p(dY_out),
                                  _p(dgamma), _p(ws), _nbytes(ws), _stream(stream))
    _check("resbm_rmsnorm_bwd", st)


def resbm_decode_bwd(desc, dY, B, Wd1, Wd2, dB, dWd1, dWd2, ws, stream=None):
    st = load().resbm_decode_bwd(ctypes.byref(desc), _p(dY), _p(B), _p(Wd1), _p(Wd2), _p(dB),
                                 _p(dWd1), _p(dWd2), _p(ws), _nbytes(ws), _stream(stream))
    _check("resbm_decode_bwd", st)


def resbm_decode_bwd_noalloc(desc, dY, B, Wd1, Wd2, dB, dWd1, dWd2, stream=None):
    """resbm_decode_bwd with the library's fixed device scratch instead of a workspace."""
    st = load().resbm_decode_bwd_noalloc(ctypes.byref(desc), _p(dY), _p(B), _p(Wd1), _p(Wd2),
                                         _p(dB), _p(dWd1), _p(dWd2), _stream(stream))
    _check("resbm_decode_bwd_noalloc", st)


def resbm_encode_bwd(desc, dB, F, P_save, We1, We2, dF, dX, dWe1, dWe2, ws, stream=None):
    st = load().resbm_encode_bwd(ctypes.byref(desc), _p(dB), _p(F), _p(P_save), _p(We1),
                                 _p(We2), _p(dF), _p(dX), _p(dWe1), _p(dWe2), _p(ws),
                                 _nbytes(ws), _stream(stream))
    _check("resbm_encode_bwd", st)


def resbm_boundary_step(desc, ws, stream=None, **tensors):
    """tensors: X, F, dY, We1, We2, Wd1, Wd2 (inputs); B, P, Y, dB, dF, dX, dWe1, dWe2, dWd1,
    dWd2 (outputs; P and dX may be omitted)."""
    args = resbm_step_args(**{k: _p(v) for k, v in tensors.items()})
    st = load().resbm_boundary_step(ctypes.byref(desc), ctypes.byref(args), _p(ws), _nbytes(ws),
                                    _stream(stream))
    _check("resbm_boundary_step", st)


def _event(ev):
    """The cudaEvent_t handle of a torch.cuda.Event (recorded once already, so that it exists)."""
    if ev is None:
        return None
    h = ev.cuda_event if hasattr(ev, "cuda_event") else int(ev)
    if not h:
        raise ValueError("the event has no CUDA handle yet: record it once first")
    return h


def resbm_boundary_step_host(desc, ws, stream=None, wait_before_inputs=None, inputs_done=None, **tensors):
    """resbm_boundary_step with host tensors (CPU torch tensors, pinned for asynchronous
    copies); ws is the device workspace of RESBM_OP_BOUNDARY_STEP_HOST. wait_before_inputs /
    inputs_done: torch.cuda.Event objects chaining consecutive calls' host-to-device copies."""
    args = resbm_step_args(**{k: _p(v) for k, v in tensors.items()},
                           wait_before_inputs=_event(wait_before_inputs), inputs_done=_event(inputs_done))
    st = load().resbm_boundary_step_host(ctypes.byref(desc), ctypes.byref(args), _p(ws), _nbytes(ws),
                                         _stream(stream))
    _check("resbm_boundary_step_host", st)


# ---- convenience: output buffers of one boundary step (allocated by torch) -------------------
def step_outputs(desc: resbm_desc, device="cuda", with_dX=True) -> dict:
    T, d, r, m = desc.T, desc.d, desc.r, desc.m
    io = TORCH_DTYPES[desc.dtype]
    f32 = torch.float32
    out = dict(B=torch.empty(T, r, dtype=io, device=device),
               P=torch.empty(T, m, dtype=f32, device=device),
               Y=torch.empty(T, d, dtype=io, device=device),
               dB=torch.empty(T, r, dtype=io, device=device),
               dF=torch.empty(T, d, dtype=io, device=device),
               dWe1=torch.empty(d, m, dtype=f32, device=device),
               dWe2=torch.empty(m, r, dtype=f32, device=device),
               dWd1=torch.empty(r, m, dtype=f32, device=device),
               dWd2=torch.empty(m, d, dtype=f32, device=device))
    if with_dX:
        out["dX"] = torch.zeros(T, d, dtype=io, device=device)
    return out


# ---- utilities on the bottleneck weights ------------------------------------------------------
def resbm_matrix_workspace_bytes(op: int, rows: int, cols: int) -> int:
    out = ctypes.c_size_t(0)
    _check("resbm_matrix_workspace_bytes", load().resbm_matrix_workspace_bytes(int(op), int(rows), int(cols),
                                                                               ctypes.byref(out)))
    return int(out.value)


def matrix_workspace(op: int, rows: int, cols: int, device="cuda") -> torch.Tensor:
    return torch.empty(max(resbm_matrix_workspace_bytes(op, rows, cols), 1), dtype=torch.uint8, device=device)


def resbm_newton_schulz(G, steps, X, ws, stream=None):
    """X (bf16, G's shape) = Muon's Newton-Schulz orthogonalisation of G (fp32 or bf16)."""
    rows, cols = G.shape
    g_dtype = RESBM_F32 if G.dtype == torch.float32 else RESBM_BF16
    _check("resbm_newton_schulz", load().resbm_newton_schulz(rows, cols, _p(G), g_dtype, int(steps), _p(X), _p(ws),
                                                             _nbytes(ws), _stream(stream)))


def resbm_effective_rank(W, out, ws, stream=None):
    """out (device float64, 4): sigma_max^2, ||W||_F^2, r_eff, the iterations taken (products with the Gram matrix)."""
    rows, cols = W.shape
    _check("resbm_effective_rank", load().resbm_effective_rank(rows, cols, _p(W), _p(out), _p(ws), _nbytes(ws),
                                                               _stream(stream)))


# ---- the encoder fused into the FFN down-projection ------------------------------------------
def resbm_ffn_down_encode_workspace_bytes(desc: resbm_desc, f: int) -> int:
    out = ctypes.c_size_t(0)
    _check("resbm_ffn_down_encode_workspace_bytes",
           load().resbm_ffn_down_encode_workspace_bytes(ctypes.byref(desc), int(f), ctypes.byref(out)))
    return int(out.value)


def ffn_down_encode_workspace(desc: resbm_desc, f: int, device="cuda") -> torch.Tensor:
    return torch.empty(max(resbm_ffn_down_encode_workspace_bytes(desc, f), 1), dtype=torch.uint8, device=device)


def resbm_ffn_down_encode_fwd(desc, H, W2, X, We1, We2, B, P_save, F_out, ws, stream=None):
    """B (and P_save, F_out if given) from the FFN hidden state H (T x f) and the down-projection
    W2 (f x d): the encoder applied to F = H . W2 without storing F unless F_out is given."""
    f = H.shape[1]
    st = load().resbm_ffn_down_encode_fwd(ctypes.byref(desc), int(f), _p(H), _p(W2), _p(X), _p(We1), _p(We2),
                                          _p(B), _p(P_save), _p(F_out), _p(ws), _nbytes(ws), _stream(stream))
    _check("resbm_ffn_down_encode_fwd", st)


# ---- the training step's operators around the boundary (include/resbm_train.h) ----------------
_DT = {torch.float32: RESBM_F32, torch.bfloat16: RESBM_BF16}
_CODES = (torch.float8_e4m3fn, torch.uint8)


def _want(ok, what):
    if not ok:
        raise ValueError(what)


_device = getattr(torch._C, "_cuda_getDevice", None) or torch.cuda.current_device


def _here(t, device, what):
    """t is on the current device (where the library enqueues)"""
    if t.get_device() != device:
        raise ValueError("%s must be on the current CUDA device (%d): got %s" % (what, device, t.device))


def _row_stride(t, shape, dtype, device, what):
    """The row stride of a (T, d) tensor with unit stride along d"""
    stride = t.stride()
    if t.shape != shape or t.dtype != dtype or (stride[1] != 1 and shape[1] > 1):
        raise ValueError("%s must be %s, %s, with unit stride along the columns" % (what, tuple(shape), dtype))
    _here(t, device, what)
    return stride[0]


def resbm_add_rmsnorm_fwd(X, A, gamma, eps, H=None, N=None, Q=None, S=None, q_group=0, stream=None):
    """H = X + A (A None: H = X), N = RMSNorm(H) * gamma, Q and S the same in e4m3 with scales. X, A, H, N: (T, d) of one
    type, unit stride along d, any row stride (A and X: also 0, an expanded row); gamma (d,); Q (T, d) dense, one byte an
    element (float8_e4m3fn or uint8), with S (T, ceil(d / q_group)) fp32, or (T, 1) for q_group = 0."""
    shape, dtype = X.shape, X.dtype
    code = _DT.get(dtype)
    if len(shape) != 2 or code is None:
        raise ValueError("X must be (T, d), fp32 or bf16")
    T, d = shape
    device = _device()
    ldx = _row_stride(X, shape, dtype, device, "X")
    lda = 0 if A is None else _row_stride(A, shape, dtype, device, "A")
    ldh = 0 if H is None else _row_stride(H, shape, dtype, device, "H")
    ldn = 0 if N is None else _row_stride(N, shape, dtype, device, "N")
    if gamma.shape != shape[1:] or gamma.dtype != dtype or not gamma.is_contiguous():
        raise ValueError("gamma must be (%d,), %s" % (d, dtype))
    _here(gamma, device, "gamma")
    if (Q is None) != (S is None):
        raise ValueError("Q and S come together")
    if Q is not None:
        if not 0 <= q_group < 1 << 31:   # (the descriptor's field has 32 bits: more would arrive as another group)
            raise ValueError("q_group must be a power of two >= 32, or 0: got %d" % q_group)
        groups = -(-d // q_group) if q_group else 1
        if Q.shape != shape or Q.dtype not in _CODES or not Q.is_contiguous():
            raise ValueError("Q must be %s, dense, float8_e4m3fn or uint8" % (tuple(shape),))
        if S.shape != (T, groups) or S.dtype != torch.float32 or not S.is_contiguous():
            raise ValueError("S must be (%d, %d), fp32, dense" % (T, groups))
        _here(Q, device, "Q")
        _here(S, device, "S")
    if stream is None and _raw_stream is not None:
        stream = _raw_stream(device)
    st = (_lib or load()).resbm_add_rmsnorm_fwd(
        resbm_add_norm_desc(T, d, ldx, lda, ldh, ldn, code, q_group, eps, 0), X.data_ptr(), None if A is None else A.data_ptr(),
        gamma.data_ptr(), None if H is None else H.data_ptr(), None if N is None else N.data_ptr(),
        None if Q is None else Q.data_ptr(), None if S is None else S.data_ptr(), _stream(stream))
    if st != RESBM_OK:
        _check("resbm_add_rmsnorm_fwd", st)


class AdamWPlan:
    """The tensors of resbm_adamw_step and resbm_grad_norm (resbm_adamw_plan in host memory). Lists of dense CUDA tensors
    of the same lengths, one entry per parameter: weights (fp32 or bf16), gradients (fp32 or bf16), states m and v (fp32,
    or e4m3 codes of m and of sqrt(v): float8_e4m3fn or uint8, with m_scale and v_scale of ceil(n / 256) fp32), optionally
    fp32 master copies of bf16 weights. With gradients alone (params None) the plan serves resbm_grad_norm. The plan
    keeps the tensors alive; gradients that moved are given with set_grads, their memory is let go with release_grads."""

    def __init__(self, params, grads, m=None, v=None, m_scale=None, v_scale=None, master=None):
        self._fields = {"w": params, "g": grads, "m": m, "v": v, "m_scale": m_scale, "v_scale": v_scale, "master": master}
        self._fields = {k: list(x) for k, x in self._fields.items() if x is not None}
        grads = self._fields["g"]
        self.device = _device()
        self.count = len(grads)
        state = RESBM_STATE_NONE
        if params is not None:
            _want(m is not None and v is not None, "weights come with their states m and v")
            coded = self.count > 0 and self._fields["m"][0].element_size() == 1
            state = RESBM_STATE_E4M3 if coded else RESBM_STATE_F32
            _want((m_scale is not None) == coded and (v_scale is not None) == coded, "8-bit states, and only they, have scales")
            _want(master is None or self.count == 0 or self._fields["w"][0].dtype == torch.bfloat16, "master copies are of bf16 weights")
        else:
            _want(set(self._fields) == {"g"}, "states and master copies belong to weights")
        for k, x in self._fields.items():
            _want(len(x) == self.count, "%s: %d tensors, and %d gradients" % (k, len(x), self.count))
        for k in ("w", "g"):
            x = self._fields.get(k)
            _want(not x or (x[0].dtype in _DT and all(t.dtype == x[0].dtype for t in x)), "%s: fp32 or bf16, one type in a plan" % k)
        sizes = [g.numel() for g in grads]
        blocks = [-(-n // RESBM_STATE_BLOCK) for n in sizes]
        codes = _CODES if state == RESBM_STATE_E4M3 else (torch.float32,)
        for k, x in self._fields.items():
            types = (x[0].dtype,) if k in ("w", "g") and x else codes if k in ("m", "v") else (torch.float32,)
            for t, n in zip(x, blocks if k.endswith("_scale") else sizes):
                if t.numel() != n or not t.is_contiguous() or t.dtype not in types:
                    raise ValueError("%s: dense tensors of the gradients' sizes, %s" % (k, " or ".join(map(str, types))))
                _here(t, self.device, k)
        dt = lambda k: _DT[self._fields[k][0].dtype] if self._fields.get(k) else RESBM_F32
        self._desc = resbm_adamw_desc(dt("w"), dt("g"), state, 0)
        self._tensors = (resbm_adamw_tensor * self.count)()
        # (the structure is eight 64-bit words: an array of them is filled column by column)
        words = (ctypes.c_int64 * (8 * self.count)).from_buffer(self._tensors)
        for i, k in enumerate(("w", "g", "m", "v", "m_scale", "v_scale", "master")):
            if k in self._fields:
                words[i::8] = [t.data_ptr() for t in self._fields[k]]
        words[7::8] = self._sizes = sizes
        size = ctypes.c_size_t(0)
        _check("resbm_adamw_plan_bytes", load().resbm_adamw_plan_bytes(self.count, ctypes.byref(size)))
        self._plan = (ctypes.c_uint64 * (-(-size.value // 8)))()
        self._address = ctypes.addressof(self._plan)
        self._build()

    def _check_grads(self, grads):
        _want(len(grads) == self.count, "%d gradients for %d tensors" % (len(grads), self.count))
        for g, n in zip(grads, self._sizes):
            _want(g.is_contiguous() and g.numel() == n and _DT.get(g.dtype) == self._desc.g_dtype, "gradients: dense tensors of the same sizes and type")
            _here(g, self.device, "a gradient")

    def _build(self):
        _check("resbm_adamw_plan", load().resbm_adamw_plan(ctypes.byref(self._desc), self._tensors, self.count, self._address,
                                                           ctypes.sizeof(self._plan)))

    def set_grads(self, grads):
        """The gradients of the next steps: same sizes, types and order. (If they are refused, the plan is as before, or,
        where they overlap what the step writes, refuses steps until it has others.)"""
        grads = list(grads)
        self._check_grads(grads)
        self._fields["g"] = grads
        for e, g in zip(self._tensors, grads):
            e.g = g.data_ptr()
        self._build()

    def release_grads(self):
        """Lets the gradients' memory go: no step before the next set_grads."""
        self._fields["g"] = None

    def release(self):
        """Lets all of the tensors' memory go. The plan still has their addresses: a step after the next set_grads is the caller's
        word that they are where they were."""
        self._fields = {"g": None}

    def _ready(self, device):
        if device != self.device:
            raise ValueError("the plan's tensors are on device %d, not the current one (%d)" % (self.device, device))
        if self._fields["g"] is None:
            raise ValueError("the plan's gradients were released")


def resbm_adamw_step(plan, lr, beta1=0.9, beta2=0.999, eps=1e-8, weight_decay=0.01, step=1, lr_dev=None, step_dev=None,
                     grad_scale=None, stream=None):
    """One AdamW step over the plan's tensors, in place. step counts from 1. lr_dev (fp32), step_dev (int64) and grad_scale
    (fp32): one-element device tensors that the kernel reads instead of lr and step, and as the gradients' factor."""
    for name, t, dt in (("lr_dev", lr_dev, torch.float32), ("step_dev", step_dev, torch.int64), ("grad_scale", grad_scale, torch.float32)):
        if t is not None:
            if t.dtype != dt or t.numel() != 1:
                raise ValueError("%s must be one %s" % (name, dt))
            _here(t, plan.device, name)
    plan._ready(_device())
    hyper = resbm_adamw_hyper(lr, beta1, beta2, eps, weight_decay, step, _p(lr_dev), _p(step_dev), _p(grad_scale))
    st = (_lib or load()).resbm_adamw_step(plan._address, hyper, _stream(stream))
    if st != RESBM_OK:
        _check("resbm_adamw_step", st)


def _plans(plans):
    plans = [plans] if isinstance(plans, AdamWPlan) else list(plans)
    return (ctypes.c_void_p * len(plans))(*[p._address for p in plans]), plans


def resbm_grad_norm_workspace_bytes(plans) -> int:
    out = ctypes.c_size_t(0)
    array, plans = _plans(plans)
    _check("resbm_grad_norm_workspace_bytes", load().resbm_grad_norm_workspace_bytes(array, len(plans), ctypes.byref(out)))
    return int(out.value)


def grad_norm_workspace(plans, device="cuda") -> torch.Tensor:
    return torch.empty(max(resbm_grad_norm_workspace_bytes(plans), 1), dtype=torch.uint8, device=device)


def resbm_grad_norm(plans, max_norm, out, ws, stream=None):
    """out (2 fp32): the norm of the gradients of a plan (or of several together), and the coefficient that clips it to
    max_norm (0: none), which resbm_adamw_step takes as grad_scale = out[1:]."""
    array, plans = _plans(plans)
    device = _device()
    if out.dtype != torch.float32 or out.numel() != 2 or not out.is_contiguous():
        raise ValueError("out must be 2 fp32")
    _here(out, device, "out")
    _here(ws, device, "ws")
    _want(ws.is_contiguous(), "ws must be dense")   # (an expanded one is smaller than its elements)
    for p in plans:
        p._ready(device)
    st = load().resbm_grad_norm(array, len(plans), max_norm, out.data_ptr(), ws.data_ptr(), _nbytes(ws), _stream(stream))
    if st != RESBM_OK:
        _check("resbm_grad_norm", st)


# ---- the vocabulary's operators (include/resbm_vocab.h) ------------------------------------------------
def resbm_vocab_workspace_bytes(op, T, V, d, dtype="bf16", K=0) -> int:
    """Bytes of the workspace of an op (RESBM_VOCAB_*) over T tokens, V words, width d; distillation: K entries a token."""
    dt = DTYPES[dtype] if isinstance(dtype, str) else int(dtype)
    out = ctypes.c_size_t(0)
    desc = resbm_vocab_desc(int(T), int(V), int(d), int(d), int(d), int(K), dt, dt, 1.0, 0, 0)
    _check("resbm_vocab_workspace_bytes", load().resbm_vocab_workspace_bytes(ctypes.byref(desc), int(op), ctypes.byref(out)))
    return int(out.value)


def vocab_workspace(op, T, V, d, dtype="bf16", K=0, device="cuda") -> torch.Tensor:
    return torch.empty(max(resbm_vocab_workspace_bytes(op, T, V, d, dtype, K), 1), dtype=torch.uint8, device=device)


def _dense(t, shape, dtypes, device, what):
    if t.shape != shape or t.dtype not in dtypes or not t.is_contiguous():
        raise ValueError("%s must be %s, dense, %s" % (what, tuple(shape), " or ".join(map(str, dtypes))))
    _here(t, device, what)


_F32, _I64 = (torch.float32,), (torch.int64,)


def _loss_desc(X, W, target, teacher, temperature, device):
    """The descriptor of a loss over the vocabulary, of checked inputs"""
    if X.dim() != 2 or W.dim() != 2 or X.dtype not in _DT or X.shape[1] < 1 or W.shape[0] < 1:
        raise ValueError("X must be (T, d) and W (V, d), fp32 or bf16")
    (T, d), V, dtype = X.shape, W.shape[0], X.dtype
    ldx = _row_stride(X, (T, d), dtype, device, "X")
    ldw = _row_stride(W, (V, d), dtype, device, "W")
    K, tdt = 0, RESBM_F32
    if teacher is None:
        _dense(target, (T,), _I64, device, "labels")
    else:
        if target.dim() != 2 or not 1 <= target.shape[1] <= 1024:
            raise ValueError("index must be (T, K) with K from 1 to 1024")
        K = target.shape[1]
        _dense(target, (T, K), _I64, device, "index")
        _dense(teacher, (T, K), tuple(_DT), device, "teacher")
        tdt = _DT[teacher.dtype]
    return resbm_vocab_desc(T, V, d, ldx if T > 1 else d, ldw if V > 1 else d, K, _DT[dtype], tdt, temperature, 0, 0)


def _loss_fwd(fn, X, W, target, teacher, temperature, loss, lse, ws, stream):
    device = _device()
    desc = _loss_desc(X, W, target, teacher, temperature, device)
    _dense(loss, (desc.T,), _F32, device, "loss")
    _dense(lse, (desc.T,), _F32, device, "lse")
    _workspace_here(ws, device)
    args = [_p(X), _p(W), _p(target)] + ([] if teacher is None else [_p(teacher)])
    _check(fn, getattr(_lib or load(), fn)(desc, *args, _p(loss), _p(lse), _p(ws), _nbytes(ws), _stream(stream)))


def _loss_bwd(fn, X, W, target, teacher, temperature, lse, dloss, dX, dW, ws, stream):
    device = _device()
    desc = _loss_desc(X, W, target, teacher, temperature, device)
    _dense(lse, (desc.T,), _F32, device, "lse")
    if dloss.dtype != torch.float32 or dloss.shape not in ((), (1,), (desc.T,)) or not dloss.is_contiguous():
        raise ValueError("dloss must be (%d,) or one element, fp32, dense" % desc.T)
    _here(dloss, device, "dloss")
    desc.dloss_each = int(dloss.shape == (desc.T,))
    if dX is not None:
        _dense(dX, X.shape, (X.dtype,), device, "dX")
    if dW is not None:
        _dense(dW, W.shape, (W.dtype,), device, "dW")
    _workspace_here(ws, device)
    args = [_p(X), _p(W), _p(target)] + ([] if teacher is None else [_p(teacher)])
    _check(fn, getattr(_lib or load(), fn)(desc, *args, _p(lse), _p(dloss), _p(dX), _p(dW), _p(ws), _nbytes(ws), _stream(stream)))


def _workspace_here(ws, device):
    if ws is not None:
        _here(ws, device, "ws")
        _want(ws.is_contiguous(), "ws must be dense")   # (an expanded one is smaller than its elements)


def resbm_linear_ce_fwd(X, W, labels, loss, lse, ws, stream=None):
    """loss and lse (T fp32): the cross entropy of the logits X . W^T against labels (T int64; negative: no label), without the
    logits. X (T, d) and W (V, d) of one type, unit stride along d, any row stride."""
    _loss_fwd("resbm_linear_ce_fwd", X, W, labels, None, 1.0, loss, lse, ws, stream)


def resbm_linear_ce_bwd(X, W, labels, lse, dloss, dX, dW, ws, stream=None):
    """dX (T, d) and dW (V, d), dense, either may be None: the gradients for dloss (T fp32, or one for all)."""
    _loss_bwd("resbm_linear_ce_bwd", X, W, labels, None, 1.0, lse, dloss, dX, dW, ws, stream)


def resbm_distill_fwd(X, W, index, teacher, temperature, loss, lse, ws, stream=None):
    """loss and lse (T fp32): temperature^2 times the divergence of softmax(X . W^T / temperature) from the softmax of the
    teacher's logits (T, K; fp32 or bf16) at the words index (T, K int64; negative: no entry)."""
    _loss_fwd("resbm_distill_fwd", X, W, index, teacher, temperature, loss, lse, ws, stream)


def resbm_distill_bwd(X, W, index, teacher, temperature, lse, dloss, dX, dW, ws, stream=None):
    _loss_bwd("resbm_distill_bwd", X, W, index, teacher, temperature, lse, dloss, dX, dW, ws, stream)


def _embed_desc(ids, V, rows, scale, padding, device, what):
    if rows.dim() != 2 or rows.dtype not in _DT or ids.dim() != 1 or rows.shape[1] < 1 or V < 1:
        raise ValueError("ids must be (T,), %s (T, d), fp32 or bf16" % what)
    T, d = ids.shape[0], rows.shape[1]
    _dense(ids, (T,), _I64, device, "ids")
    ldo = _row_stride(rows, (T, d), rows.dtype, device, what)
    return resbm_embed_desc(T, V, d, d, ldo if T > 1 else d, padding, _DT[rows.dtype], scale, 0)


def resbm_embed_fwd(ids, table, scale, out, stream=None):
    """out (T, d) = scale * table[ids]; table (V, d); ids (T int64). Unit stride along d, any row stride. An id outside the
    table gives a row of NaN."""
    # (a few tokens' call is the host's time: the checks of _embed_desc without its calls)
    shape, dtype, rows = out.shape, out.dtype, table.shape
    code = _DT.get(dtype)
    if code is None or len(shape) != 2 or ids.shape != shape[:1] or ids.dtype != torch.int64 or not ids.is_contiguous():
        raise ValueError("out must be (T, d), fp32 or bf16, and ids (T,), int64, dense")
    (T, d), device = shape, _device()
    if len(rows) != 2 or rows[1] != d or rows[0] < 1 or d < 1 or table.dtype != dtype:
        raise ValueError("table must be (V, %d), %s" % (d, dtype))
    (ldo, so), (ldt, st) = out.stride(), table.stride()
    if (so != 1 or st != 1) and d > 1:
        raise ValueError("out and table must have unit stride along the columns")
    if ids.get_device() != device or table.get_device() != device or out.get_device() != device:
        raise ValueError("ids, table and out must be on the current CUDA device (%d)" % device)
    if stream is None and _raw_stream is not None:
        stream = _raw_stream(device)
    status = (_lib or load()).resbm_embed_fwd(resbm_embed_desc(T, rows[0], d, ldt if rows[0] > 1 else d, ldo if T > 1 else d, -1, code, scale, 0),
                                              ids.data_ptr(), table.data_ptr(), out.data_ptr(), _stream(stream))
    if status != RESBM_OK:
        _check("resbm_embed_fwd", status)


def resbm_embed_bwd(ids, dout, scale, dtable, ws, padding=-1, stream=None):
    """dtable (V, d), dense = scale * the sum of dout's rows (T, d) over each word's tokens; zero for padding (an id; negative:
    none)."""
    device = _device()
    desc = _embed_desc(ids, dtable.shape[0], dout, scale, padding, device, "dout")
    _dense(dtable, (desc.V, desc.d), (dout.dtype,), device, "dtable")
    _workspace_here(ws, device)
    _check("resbm_embed_bwd", (_lib or load()).resbm_embed_bwd(desc, _p(ids), _p(dout), _p(dtable), _p(ws), _nbytes(ws), _stream(stream)))
