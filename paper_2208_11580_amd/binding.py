"""Thin ctypes binding of libobc.so: argument marshalling only.

Every function has the name of the C entry point it calls (see include/obc.h) and takes torch
tensors that already live on the GPU; torch is used for device memory and the current stream,
nothing else.  All arithmetic of the method runs inside the library's HIP kernels.  There is no
fallback: if the library is missing or a call fails, an exception is raised.
"""
from __future__ import annotations

import ctypes
import os
from ctypes import POINTER, byref, c_char_p, c_float, c_int, c_int64, c_size_t, c_void_p

from typing import NamedTuple

import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libobc.so")

OBC_OK = 0
OBC_ERR_BAD_ARG, OBC_ERR_BAD_SHAPE, OBC_ERR_NOT_SPD = -1, -2, -3
OBC_ERR_WORKSPACE, OBC_ERR_NUMERIC, OBC_ERR_HIP = -4, -5, -6
STRATEGY_AUTO, STRATEGY_RANK1, STRATEGY_BLOCKED = 0, 1, 2
QUANT_OUTLIERS = 1
F32, F16, BF16, I8 = 0, 1, 2, 3
GRID_SYMMETRIC, GRID_ZERO = 1, 2
SELECT_STATIC_MAX_WEIGHTS, SELECT_STATIC_MAX_ROWS = 2359296, 8192   # limits of obc_global_select_static

EXPORTS = [
    "obc_create", "obc_destroy", "obc_last_error", "obc_version", "obc_check",
    "obc_profile_begin", "obc_profile_end", "obc_membench", "obc_mfmabench",
    "obc_hessian_workspace_bytes", "obc_hessian",
    "obc_invert_workspace_bytes", "obc_invert",
    "obc_cross_workspace_bytes", "obc_cross", "obc_refit_workspace_bytes", "obc_refit",
    "obc_rows_workspace_bytes", "obc_prune_rows", "obc_blocks_workspace_bytes", "obc_prune_blocks", "obc_quant_rows", "obc_minmax_grid",
    "obc_global_select_workspace_bytes", "obc_global_select", "obc_global_select_static", "obc_gather_trace",
    "obc_reconstruct_workspace_bytes", "obc_reconstruct_rows",
    "obc_group_grid", "obc_pack4_bytes", "obc_pack4",
    "obc_product4_workspace_bytes", "obc_product4", "obc_product4_grad_workspace_bytes", "obc_product4_grad",
    "obc_rmsnorm", "obc_rmsnorm_grad_workspace_bytes", "obc_rmsnorm_grad", "obc_distill",
    "obc_score_workspace_bytes", "obc_score",
    "obc_layernorm", "obc_layernorm_grad_workspace_bytes", "obc_layernorm_grad",
    "obc_embed", "obc_embed_grad_workspace_bytes", "obc_embed_grad",
    "obc_adamw_plan_bytes", "obc_adamw_plan", "obc_adamw",
]

_TYPES = {torch.float32: F32, torch.float16: F16, torch.bfloat16: BF16, torch.int8: I8}


KERNEL_CLASSES = ("panel", "flush", "rank1")


class KernelStat(ctypes.Structure):
    _fields_ = [("launches", c_int), ("ms", ctypes.c_double), ("bytes", ctypes.c_double),
                ("flops", ctypes.c_double)]


class Packed4(NamedTuple):
    """A layer's weights as obc_pack4 lays them out: opaque bytes, and the sizes they were packed for."""
    data: torch.Tensor
    rows: int
    cols: int
    group: int


class AdamState(NamedTuple):
    """What obc_adamw keeps for a parameter tensor (of its shape, or as many values): moments in fp32, or m and the root of v in
    8-bit floating-point numbers with an fp32 scale for every 256 of them; master: the parameters in fp32, or None."""
    m: torch.Tensor
    v: torch.Tensor
    m_scale: torch.Tensor | None = None
    v_scale: torch.Tensor | None = None
    master: torch.Tensor | None = None


class AdamTensor(ctypes.Structure):
    # as obc_adamw_tensor
    _fields_ = [(name, c_void_p) for name in ("p", "p_out", "g", "m", "m_out", "v", "v_out", "m_scale", "v_scale", "m_scale_out",
                                              "v_scale_out", "master", "master_out")] + [("n", c_int64), ("decay", c_float)]


class ObcError(RuntimeError):
    def __init__(self, code, msg):
        super().__init__("libobc error %d: %s" % (code, msg))
        self.code = code


_lib = None


def load_library():
    """dlopen libobc.so and declare the prototypes.  Raises if it has not been built."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(LIB_PATH):
        raise FileNotFoundError(
            "%s is missing: build it with `python -m paper_2208_11580_amd.build` "
            "(there is no fallback path)" % LIB_PATH)
    lib = ctypes.CDLL(LIB_PATH)
    vp, sp = c_void_p, POINTER(c_size_t)
    lib.obc_create.argtypes = [POINTER(vp), vp]
    lib.obc_destroy.argtypes = [vp]
    lib.obc_last_error.argtypes = [vp]
    lib.obc_last_error.restype = c_char_p
    lib.obc_version.argtypes = []
    lib.obc_version.restype = c_char_p
    lib.obc_check.argtypes = [vp]
    lib.obc_profile_begin.argtypes = [vp]
    lib.obc_profile_end.argtypes = [vp, POINTER(KernelStat)]
    lib.obc_membench.argtypes = [vp, c_int, c_int, vp, vp, c_size_t, c_int, POINTER(ctypes.c_double)]
    lib.obc_mfmabench.argtypes = [vp, c_int, c_int, c_int, POINTER(ctypes.c_double), POINTER(ctypes.c_double)]
    lib.obc_hessian_workspace_bytes.argtypes = [c_int, c_int64, sp]
    lib.obc_hessian.argtypes = [vp, vp, c_int, c_int64, c_int64, c_float, c_int, vp, vp, c_size_t]
    lib.obc_invert_workspace_bytes.argtypes = [c_int, sp]
    lib.obc_invert.argtypes = [vp, vp, c_int, vp, c_size_t]
    lib.obc_rows_workspace_bytes.argtypes = [c_int, c_int, c_int, sp]
    lib.obc_prune_rows.argtypes = [vp, vp, vp, c_int, c_int, c_int, c_int, c_int, vp, vp, vp, vp, vp, vp,
                                   c_int, vp, c_size_t]
    lib.obc_blocks_workspace_bytes.argtypes = [c_int, c_int, c_int, c_int, sp]
    lib.obc_prune_blocks.argtypes = [vp, vp, vp, c_int, c_int, c_int, c_int, vp, vp, vp, vp, vp, c_int, vp, c_size_t]
    lib.obc_quant_rows.argtypes = [vp, vp, vp, c_int, c_int, vp, vp, c_int, vp, c_int, vp, vp, vp, vp, c_int,
                                   vp, c_size_t]
    lib.obc_minmax_grid.argtypes = [vp, vp, vp, c_int, c_int, c_int, c_int, vp, vp]
    lib.obc_cross_workspace_bytes.argtypes = [c_int, c_int, c_int64, sp]
    lib.obc_cross.argtypes = [vp, vp, vp, c_int, c_int, c_int64, c_int64, c_int64, c_int, vp, vp, c_size_t]
    lib.obc_refit_workspace_bytes.argtypes = [c_int, c_int, sp]
    lib.obc_refit.argtypes = [vp, vp, c_int, vp, c_int, vp, c_int, vp, c_size_t]
    lib.obc_global_select_workspace_bytes.argtypes = [c_int, c_int, sp]
    lib.obc_global_select.argtypes = [vp, vp, vp, c_int, c_int, c_int64, vp, vp, vp, c_size_t]
    lib.obc_global_select_static.argtypes = [vp, vp, vp, c_int, c_int, c_int64, vp, vp]
    lib.obc_gather_trace.argtypes = [vp, vp, vp, vp, c_int, c_int, c_int, vp]
    lib.obc_reconstruct_workspace_bytes.argtypes = [c_int, c_int, c_int, sp]
    lib.obc_reconstruct_rows.argtypes = [vp, vp, vp, vp, c_int, c_int, c_int, vp, vp, c_size_t]
    i64 = c_int64
    lib.obc_group_grid.argtypes = [vp, vp, vp, c_int, c_int, c_int, c_int, c_int, vp, vp]
    lib.obc_pack4_bytes.argtypes = [c_int, c_int, c_int, sp]
    lib.obc_pack4.argtypes = [vp, vp, vp, vp, c_int, c_int, c_int, vp]
    lib.obc_product4_workspace_bytes.argtypes = [c_int, c_int, c_int, c_int, c_int, sp]
    lib.obc_product4.argtypes = [vp, vp, c_int, c_int, c_int, vp, c_int, vp, c_int, i64, vp, c_int, i64, vp, c_size_t]
    lib.obc_product4_grad_workspace_bytes.argtypes = [c_int, c_int, c_int, c_int, c_int, sp]
    lib.obc_product4_grad.argtypes = [vp, vp, c_int, c_int, c_int, vp, c_int, c_int, i64, vp, i64, vp, c_size_t]
    lib.obc_rmsnorm.argtypes = [vp, vp, vp, c_int, vp, c_float, c_int, c_int, vp, vp, c_int, vp, vp]
    lib.obc_rmsnorm_grad_workspace_bytes.argtypes = [c_int, c_int, sp]
    lib.obc_rmsnorm_grad.argtypes = [vp, vp, vp, vp, vp, vp, c_int, c_int, c_int, vp, vp, vp, c_size_t]
    lib.obc_distill.argtypes = [vp, vp, c_int, c_int, c_int, i64, vp, vp, c_int, c_float, vp, vp, vp, i64]
    lib.obc_score_workspace_bytes.argtypes = [c_int, c_int, c_int, c_int, sp]
    lib.obc_score.argtypes = [vp, vp, c_int, c_int, c_int, i64, vp, c_float, c_int, vp, vp, vp, vp, vp, vp, c_size_t]
    lib.obc_layernorm.argtypes = [vp, vp, vp, c_int, vp, vp, c_float, c_int, c_int, vp, vp, c_int, vp, vp, vp]
    lib.obc_layernorm_grad_workspace_bytes.argtypes = [c_int, c_int, sp]
    lib.obc_layernorm_grad.argtypes = [vp, vp, vp, vp, vp, vp, vp, c_int, c_int, c_int, vp, vp, vp, vp, c_size_t]
    lib.obc_embed.argtypes = [vp, vp, c_int, c_int, c_int, i64, vp, c_int, c_float, vp, c_int, i64]
    lib.obc_embed_grad_workspace_bytes.argtypes = [c_int, c_int, c_int, sp]
    lib.obc_embed_grad.argtypes = [vp, vp, c_int, vp, c_int, i64, c_float, c_int, c_int, c_int, vp, c_int, i64, vp, c_size_t]
    lib.obc_adamw_plan_bytes.argtypes = [c_int, sp]
    lib.obc_adamw_plan.argtypes = [vp, vp, c_int, c_int, c_int, vp, POINTER(i64)]
    lib.obc_adamw.argtypes = [vp, vp, c_int, i64, c_int, c_int, i64, vp, c_float, vp, ctypes.c_double, ctypes.c_double, c_float, vp,
                              ctypes.c_uint32]
    for name in EXPORTS:
        fn = getattr(lib, name)
        if name not in ("obc_last_error", "obc_version"):
            fn.restype = c_int
    _lib = lib
    return lib


def _ptr(t, dtype=None):
    if t is None:
        return None
    if not t.is_cuda:
        raise ValueError("libobc takes device tensors")
    if not t.is_contiguous():
        raise ValueError("libobc takes contiguous tensors")
    if dtype is not None and t.dtype != dtype:
        raise ValueError("expected %s, got %s" % (dtype, t.dtype))
    return t.data_ptr()


def _type_of(t, what, i8=False):
    code = _TYPES.get(t.dtype)
    if code is None or (code == I8 and not i8):
        raise ValueError("%s: unsupported type %s" % (what, t.dtype))
    return code


def _rows_of(t, what):
    """Address, leading dimension and shape of a device matrix whose rows are contiguous."""
    if not t.is_cuda:
        raise ValueError("libobc takes device tensors")
    shape = t.shape
    if len(shape) != 2:
        raise ValueError("%s must be a matrix" % what)
    rows, cols = shape
    ld, step = t.stride()
    if ld < cols:
        if rows > 1:
            raise ValueError("%s must have rows that do not overlap" % what)
        ld = cols
    if step != 1 and cols > 1:
        raise ValueError("%s must have unit stride along its rows" % what)
    return t.data_ptr(), ld, rows, cols


def _vector(t, n, what):
    if t is None:
        return None
    if not t.is_cuda or t.dtype != torch.float32 or t.numel() != n or not t.is_contiguous():
        raise ValueError("%s must be %d contiguous fp32 values on the device" % (what, n))
    return t.data_ptr()


def _ints(t, n, what):
    if t is None:
        return None
    if not t.is_cuda or t.dtype != torch.int32 or t.numel() != n or not t.is_contiguous():
        raise ValueError("%s must be %d contiguous int32 values on the device" % (what, n))
    return t.data_ptr()


def _no_grad(*tensors):
    """Results are new to autograd, which would take a gradient that ends here for none."""
    if torch.is_grad_enabled():
        for t in tensors:
            if t is not None and t.requires_grad:
                raise ValueError("an argument requires a gradient, which these calls do not record: detach it, or call under "
                                 "torch.no_grad(), and call the operator's own gradient")


class AdamPlan:
    """The tensors of obc_adamw, which it keeps, laid out by obc_adamw_plan for the context's stream.  (Their addresses: a tensor that is
    given other memory needs another plan.  A captured graph needs its plans as long as it is replayed.)  The memory of its
    tensors is not handed out for anything else before the steps that are queued when they go are done."""

    def __init__(self, ctx, params, grads, states, decay=0.01, out=None):
        params, states = list(params), list(states)
        self.ctx, self.params, self.states = ctx, params, states
        self.new = (params, states) if out is None else (list(out[0]), list(out[1]))
        self.count = count = len(params)
        if not len(states) == len(self.new[0]) == len(self.new[1]) == count:
            raise ValueError("there must be as many states and outputs as parameters")
        decays = list(decay) if isinstance(decay, (list, tuple)) else [decay] * count
        if len(decays) != count:
            raise ValueError("there must be as many decays as parameters")
        self.type = _type_of(params[0], "params") if count else F32
        self.bits = 8 if count and states[0].m.dtype == torch.float8_e4m3fn else 32
        kind = torch.float8_e4m3fn if self.bits == 8 else torch.float32
        self.tensors = (AdamTensor * max(count, 1))()
        for i in range(count):
            d, p, st, new = self.tensors[i], params[i], states[i], self.new[1][i]
            ctx._take(p, self.new[0][i], *st, *new)
            self._hold(p, self.new[0][i], *st, *new)
            n = d.n = p.numel()
            d.decay = float(decays[i])
            d.p, d.p_out = self._at(i, p, params[0].dtype, n), self._at(i, self.new[0][i], params[0].dtype, n)
            if (st.master is None) != (new.master is None) or (self.bits == 8) != (st.m_scale is not None):
                raise ValueError("tensor %d: states of 8 bits have scales, and outputs what the states have" % i)
            blocks = -(-n // 256)
            for name, dtype, size in (("m", kind, n), ("v", kind, n), ("m_scale", torch.float32, blocks), ("v_scale", torch.float32, blocks),
                                      ("master", torch.float32, n)):
                setattr(d, name, self._at(i, getattr(st, name), dtype, size))
                setattr(d, name + "_out", self._at(i, getattr(new, name), dtype, size))
        need = c_size_t()
        ctx.lib.obc_adamw_plan_bytes(count, byref(need))
        self.data = ctx._empty((max(need.value, 16),), torch.uint8, ctx.stream.device)
        self.address = self.data.data_ptr()
        self.use(grads)

    def _hold(self, *tensors):
        # steps are queued on the context's stream, which need not be the one that a tensor was allocated on
        for t in tensors:
            if t is not None:
                t.record_stream(self.ctx.stream)

    @staticmethod
    def _at(i, t, dtype, n):
        if t is not None and t.numel() != n:
            raise ValueError("tensor %d: gradients, states and outputs must be as large as the parameters" % i)
        return _ptr(t, dtype)

    def use(self, grads):
        """Other gradients from the next step on (on the context's stream: steps before this call keep theirs)."""
        if self.ctx._capturing():
            # the descriptors would be written by the graph's replays alone, and read by steps before them
            raise ValueError("a plan is laid out before a capture, not in it")
        grads = list(grads)
        if len(grads) != self.count:
            raise ValueError("there must be as many gradients as parameters")
        addresses = [self._at(i, g, self.params[0].dtype, self.params[i].numel()) for i, g in enumerate(grads)]
        self.ctx._take(*grads)
        self._hold(*grads)
        for t, g in zip(self.tensors, addresses):
            t.g = g
        n = c_int64()
        self.ctx._ck(self.ctx.lib.obc_adamw_plan(self.ctx.h, self.tensors, self.count, self.type, self.bits, self.address, byref(n)))
        self.workgroups, self.grads = n.value, grads


class Context:
    """An obc_ctx bound to a torch stream (default: the current one).

    Calls that a CUDA graph captures on that stream have their workspaces in the graph's own memory; a graph must not
    be replayed after the context it was captured from is closed."""

    def __init__(self, stream: torch.cuda.Stream | None = None):
        self.lib = load_library()
        self.stream = stream if stream is not None else torch.cuda.current_stream()
        h = c_void_p()
        rc = self.lib.obc_create(byref(h), c_void_p(self.stream.cuda_stream))
        if rc != OBC_OK:
            raise ObcError(rc, "obc_create failed")
        self.h = h
        # (asked before every call, and these ask in a tenth of the time that torch.cuda's stream objects take)
        self._raw, self._device = self.stream.cuda_stream, self.stream.device.index
        self._ws = None
        self._needs = {}

    def close(self):
        if getattr(self, "h", None):
            self.lib.obc_destroy(self.h)
            self.h = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def _ck(self, rc):
        if rc != OBC_OK:
            raise ObcError(rc, self.lib.obc_last_error(self.h).decode())

    def _is_current(self):
        return torch._C._cuda_getCurrentRawStream(self._device) == self._raw

    def _capturing(self):
        """Whether the context's stream is being captured into a graph."""
        if self._is_current():
            return torch._C._cuda_isCurrentStreamCapturing()
        with torch.cuda.stream(self.stream):
            return torch.cuda.is_current_stream_capturing()

    def workspace(self, nbytes: int) -> torch.Tensor:
        """A cached device byte buffer of at least nbytes (device memory is torch's job).  While the stream is captured: one
        from the graph's memory, for the caller alone -- a graph keeps its addresses, and the cached buffer is replaced
        when a later call needs more, or used by eager calls beside a replay."""
        nbytes = max(int(nbytes), 256)
        if self._capturing():
            with torch.cuda.stream(self.stream):
                return torch.empty(nbytes, dtype=torch.uint8, device=self.stream.device)
        if self._ws is None or self._ws.numel() < nbytes:
            if self._ws is not None:
                # earlier calls queued on the context's stream may still use the old buffer: the
                # allocator must not hand it out again before that stream has passed this point
                self._ws.record_stream(self.stream)
            self._ws = None
            self._ws = torch.empty(nbytes, dtype=torch.uint8, device=torch.device("cuda", torch.cuda.current_device()))
        return self._ws

    def release_workspace(self):
        if self._ws is not None:
            self._ws.record_stream(self.stream)
        self._ws = None

    # ------------------------------------------------------------------ entry points
    def obc_check(self):
        self._ck(self.lib.obc_check(self.h))

    def obc_profile_begin(self):
        self._ck(self.lib.obc_profile_begin(self.h))

    def obc_profile_end(self):
        arr = (KernelStat * len(KERNEL_CLASSES))()
        self._ck(self.lib.obc_profile_end(self.h, arr))
        return {name: dict(launches=arr[i].launches, ms=arr[i].ms, bytes=arr[i].bytes, flops=arr[i].flops)
                for i, name in enumerate(KERNEL_CLASSES)}

    def obc_mfmabench(self, kind, iters=20000, reps=3):
        """TFLOP/s of a loop of independent fp32 (kind 0) / fp64 (kind 1) MFMA instructions."""
        ms, fl = ctypes.c_double(), ctypes.c_double()
        self._ck(self.lib.obc_mfmabench(self.h, int(kind), int(iters), int(reps), byref(ms), byref(fl)))
        return fl.value / (ms.value * 1e-3) / 1e12

    def obc_membench(self, kind, src, dst, nbytes, reps=5, streaming=False):
        """Mean milliseconds per pass of the plain read (0) / write (1) / copy (2) kernel."""
        ms = ctypes.c_double()
        self._ck(self.lib.obc_membench(self.h, int(kind), int(bool(streaming)), _ptr(src), _ptr(dst), int(nbytes),
                                       int(reps), byref(ms)))
        return ms.value

    def obc_hessian(self, X, damp_rel=0.01, H=None, accumulate=False):
        d, N = X.shape
        if H is None:
            H = torch.empty(d, d, dtype=torch.float32, device=X.device)
        need = c_size_t()
        self.lib.obc_hessian_workspace_bytes(d, N, byref(need))
        ws = self.workspace(need.value)
        ldx = X.stride(0)
        if X.stride(1) != 1:
            raise ValueError("X must have unit stride along the sample axis")
        self._ck(self.lib.obc_hessian(self.h, c_void_p(X.data_ptr()), d, N, ldx, float(damp_rel),
                                      int(bool(accumulate)), _ptr(H, torch.float32),
                                      c_void_p(ws.data_ptr()), ws.numel()))
        return H

    def obc_invert(self, H):
        d = H.shape[0]
        need = c_size_t()
        self.lib.obc_invert_workspace_bytes(d, byref(need))
        ws = self.workspace(need.value)
        self._ck(self.lib.obc_invert(self.h, _ptr(H, torch.float32), d, c_void_p(ws.data_ptr()), ws.numel()))
        return H

    def obc_cross(self, X, Y, C=None, accumulate=False):
        d_col, N = X.shape
        d_row, Ny = Y.shape
        if Ny != N:
            raise ValueError("X and Y must hold the same number of samples")
        if X.stride(1) != 1 or Y.stride(1) != 1:
            raise ValueError("X and Y must have unit stride along the sample axis")
        if C is None:
            C = torch.empty(d_row, d_col, dtype=torch.float32, device=X.device)
        need = c_size_t()
        self.lib.obc_cross_workspace_bytes(d_row, d_col, N, byref(need))
        ws = self.workspace(need.value)
        self._ck(self.lib.obc_cross(self.h, c_void_p(X.data_ptr()), c_void_p(Y.data_ptr()), d_col, d_row, N,
                                    X.stride(0), Y.stride(0), int(bool(accumulate)), _ptr(C, torch.float32),
                                    c_void_p(ws.data_ptr()), ws.numel()))
        return C

    def obc_refit(self, H, C, invert_in_place=False, W_out=None):
        d_col = H.shape[0]
        d_row = C.shape[0]
        if C.shape[1] != d_col:
            raise ValueError("C must be d_row x d_col")
        if W_out is None:
            W_out = torch.empty(d_row, d_col, dtype=torch.float32, device=H.device)
        need = c_size_t()
        self.lib.obc_refit_workspace_bytes(d_col, d_row, byref(need))
        ws = self.workspace(need.value)
        self._ck(self.lib.obc_refit(self.h, _ptr(H, torch.float32), d_col, _ptr(C, torch.float32), d_row,
                                    _ptr(W_out, torch.float32), int(bool(invert_in_place)),
                                    c_void_p(ws.data_ptr()), ws.numel()))
        return W_out

    def rows_workspace_bytes(self, R, d, strategy=STRATEGY_AUTO):
        need = c_size_t()
        rc = self.lib.obc_rows_workspace_bytes(R, d, strategy, byref(need))
        if rc != OBC_OK:
            raise ObcError(rc, "obc_rows_workspace_bytes")
        return need.value

    def obc_prune_rows(self, W, Hinv, k_steps=None, nm=(0, 0), stop_counts=None, want_trace=False,
                       strategy=STRATEGY_AUTO, out=None, live=None):
        R, d = W.shape
        if k_steps is None:
            k_steps = d if nm[1] == 0 else (d // nm[1]) * (nm[1] - nm[0])
        dev = W.device
        if out is None:
            out = {}
        order = out.get("order")
        if order is None:
            order = torch.full((R, k_steps), -1, dtype=torch.int32, device=dev)
        loss = out.get("loss")
        if loss is None:
            loss = torch.zeros((R, k_steps), dtype=torch.float32, device=dev)
        W_out = out.get("W")
        if W_out is None:
            W_out = torch.empty((R, d), dtype=torch.float32, device=dev)
        trace = out.get("trace")
        if trace is None and want_trace:
            trace = torch.empty((R, k_steps, d), dtype=torch.float32, device=dev)
        ws = self.workspace(self.rows_workspace_bytes(R, d, strategy))
        self._ck(self.lib.obc_prune_rows(
            self.h, _ptr(W, torch.float32), _ptr(Hinv, torch.float32), R, d, int(k_steps), int(nm[0]),
            int(nm[1]), _ptr(stop_counts, torch.int32), _ptr(live, torch.uint8), _ptr(order), _ptr(loss),
            _ptr(W_out), _ptr(trace),
            int(strategy), c_void_p(ws.data_ptr()), ws.numel()))
        return dict(order=order, loss=loss, W=W_out, trace=trace)

    def obc_prune_blocks(self, W, Hinv, c, k_blocks=None, stop_counts=None, want_trace=False,
                         strategy=STRATEGY_AUTO):
        R, d = W.shape
        if k_blocks is None:
            k_blocks = d // c
        dev = W.device
        order = torch.empty(R, k_blocks, dtype=torch.int32, device=dev)
        loss = torch.empty(R, k_blocks, dtype=torch.float32, device=dev)
        W_out = torch.empty(R, d, dtype=torch.float32, device=dev)
        trace = torch.empty(R, k_blocks, d, dtype=torch.float32, device=dev) if want_trace else None
        need = c_size_t()
        rc = self.lib.obc_blocks_workspace_bytes(R, d, int(c), int(strategy), byref(need))
        if rc != OBC_OK:
            raise ObcError(rc, "obc_blocks_workspace_bytes")
        ws = self.workspace(need.value)
        self._ck(self.lib.obc_prune_blocks(
            self.h, _ptr(W, torch.float32), _ptr(Hinv, torch.float32), R, d, int(c), int(k_blocks),
            _ptr(stop_counts, torch.int32), _ptr(order), _ptr(loss), _ptr(W_out), _ptr(trace),
            int(strategy), c_void_p(ws.data_ptr()), ws.numel()))
        return dict(order=order, loss=loss, W=W_out, trace=trace)

    def obc_minmax_grid(self, W, bits, live=None, symmetric=False):
        R, d = W.shape
        maxq = (1 << bits) - 1
        delta = torch.empty(R, dtype=torch.float32, device=W.device)
        offset = torch.empty(R, dtype=torch.float32, device=W.device)
        self._ck(self.lib.obc_minmax_grid(self.h, _ptr(W, torch.float32), _ptr(live, torch.uint8), R, d,
                                          maxq, int(bool(symmetric)), _ptr(delta), _ptr(offset)))
        return delta, offset, maxq

    def obc_quant_rows(self, W, Hinv, delta, offset, maxq, live=None, strategy=STRATEGY_AUTO, out=None,
                       outliers=False):
        R, d = W.shape
        dev = W.device
        if out is None:
            out = {}
        order = out.get("order")
        if order is None:
            order = torch.full((R, d), -1, dtype=torch.int32, device=dev)
        loss = out.get("loss")
        if loss is None:
            loss = torch.zeros((R, d), dtype=torch.float32, device=dev)
        codes = out.get("codes")
        if codes is None:
            codes = torch.empty((R, d), dtype=torch.int32, device=dev)
        W_out = out.get("W")
        if W_out is None:
            W_out = torch.empty((R, d), dtype=torch.float32, device=dev)
        ws = self.workspace(self.rows_workspace_bytes(R, d, strategy))
        self._ck(self.lib.obc_quant_rows(
            self.h, _ptr(W, torch.float32), _ptr(Hinv, torch.float32), R, d, _ptr(delta, torch.float32),
            _ptr(offset, torch.float32), int(maxq), _ptr(live, torch.uint8), QUANT_OUTLIERS if outliers else 0,
            _ptr(order), _ptr(loss),
            _ptr(codes), _ptr(W_out), int(strategy), c_void_p(ws.data_ptr()), ws.numel()))
        return dict(order=order, loss=loss, codes=codes, W=W_out)

    def obc_global_select(self, loss, order, k):
        R, d = loss.shape
        counts = torch.empty(R, dtype=torch.int32, device=loss.device)
        mask = torch.empty((R, d), dtype=torch.uint8, device=loss.device)
        need = c_size_t()
        self.lib.obc_global_select_workspace_bytes(R, d, byref(need))
        ws = self.workspace(need.value)
        self._ck(self.lib.obc_global_select(self.h, _ptr(loss, torch.float32), _ptr(order, torch.int32), R, d,
                                            int(k), _ptr(counts), _ptr(mask), c_void_p(ws.data_ptr()),
                                            ws.numel()))
        return counts, mask

    def obc_global_select_static(self, loss, order, k, counts, mask):
        """The global step on the library's built-in scratch; every buffer is the caller's."""
        R, d = loss.shape
        self._ck(self.lib.obc_global_select_static(self.h, _ptr(loss, torch.float32), _ptr(order, torch.int32), R, d,
                                                   int(k), _ptr(counts, torch.int32), _ptr(mask, torch.uint8)))
        return counts, mask

    def obc_gather_trace(self, W, trace, counts):
        R, k_steps, d = trace.shape
        W_out = torch.empty((R, d), dtype=torch.float32, device=W.device)
        self._ck(self.lib.obc_gather_trace(self.h, _ptr(W, torch.float32), _ptr(trace, torch.float32),
                                           _ptr(counts, torch.int32), R, d, k_steps, _ptr(W_out)))
        return W_out

    def obc_reconstruct_rows(self, W, Hinv, mask, max_pruned=None, W_out=None):
        """Weights of a mask by the closed form; max_pruned bounds any row's pruned count (default: d)."""
        R, d = W.shape
        if max_pruned is None:
            max_pruned = d
        if W_out is None:
            W_out = torch.empty((R, d), dtype=torch.float32, device=W.device)
        need = c_size_t()
        rc = self.lib.obc_reconstruct_workspace_bytes(R, d, int(max_pruned), byref(need))
        if rc != OBC_OK:
            raise ObcError(rc, "obc_reconstruct_workspace_bytes")
        ws = self.workspace(need.value)
        self._ck(self.lib.obc_reconstruct_rows(self.h, _ptr(W, torch.float32), _ptr(Hinv, torch.float32),
                                               _ptr(mask, torch.uint8), R, d, int(max_pruned), _ptr(W_out),
                                               c_void_p(ws.data_ptr()), ws.numel()))
        return W_out

    # ------------------------------------------------------- running compressed layers
    def _empty(self, shape, dtype, device):
        """An output for kernels on the context's stream: allocated on that stream, which need not be the current
        one, so that the allocator does not hand out memory that the current stream still uses."""
        if self._is_current():
            return torch.empty(shape, dtype=dtype, device=device)
        with torch.cuda.stream(self.stream):
            return torch.empty(shape, dtype=dtype, device=device)

    def _take(self, *tensors):
        """Refuses what the calls below cannot take: tensors that autograd follows, or of another device than the context's, or
        calls while another device is the current one."""
        device = self._device
        if torch._C._cuda_getDevice() != device:
            raise ValueError("the context's device is cuda:%d, the current one is not" % device)
        follows = torch.is_grad_enabled()
        for t in tensors:
            if t is None:
                continue
            if t.get_device() != device:
                raise ValueError("the context's device is cuda:%d, a tensor's is %s" % (device, t.device))
            if follows and t.requires_grad:
                _no_grad(t)

    def _need(self, query, *sizes):
        """Workspace of one of the queries (asked once for each set of sizes): address, bytes, and what keeps it."""
        key = (query,) + sizes
        n = self._needs.get(key)
        if n is None:
            need = c_size_t()
            rc = getattr(self.lib, query)(*sizes, byref(need))
            if rc != OBC_OK:
                raise ObcError(rc, query)
            if len(self._needs) >= 4096:
                self._needs.clear()
            n = self._needs[key] = need.value
        if n == 0:
            return None, 0, None
        ws = self._ws
        if ws is None or ws.numel() < n or self._capturing():
            # like the outputs: memory that the current stream may still use is not for the context's
            with torch.cuda.stream(self.stream):
                ws = self.workspace(n)
        return ws.data_ptr(), ws.numel(), ws

    def obc_group_grid(self, W, bits=4, group=0, live=None, symmetric=False, zero=False):
        """Steps and offsets (R x groups) of a grid of 2^bits values, bits <= 4; group 0: one per row, which
        obc_quant_rows takes as [:, 0]."""
        R, d = W.shape
        maxq = (1 << bits) - 1
        n = 1 if group <= 0 or group >= d else -(-d // group)
        delta = self._empty((R, n), torch.float32, W.device)
        offset = self._empty((R, n), torch.float32, W.device)
        flags = (GRID_SYMMETRIC if symmetric else 0) | (GRID_ZERO if zero else 0)
        if live is not None and live.shape != W.shape:
            raise ValueError("live must have W's shape")
        self._ck(self.lib.obc_group_grid(self.h, _ptr(W, torch.float32), _ptr(live, torch.uint8), R, d, int(group), maxq,
                                         flags, _ptr(delta), _ptr(offset)))
        return delta, offset, maxq

    def obc_pack4(self, codes, delta, offset, group=0):
        """Codes (R x d int32) and their grid (R x groups; R values do for one group) as a Packed4."""
        R, d = codes.shape
        need = c_size_t()
        rc = self.lib.obc_pack4_bytes(R, d, int(group), byref(need))
        if rc != OBC_OK:
            raise ObcError(rc, "obc_pack4_bytes")
        n = 1 if group <= 0 or group >= d else -(-d // group)
        if delta.numel() != R * n or offset.numel() != R * n:
            raise ValueError("delta and offset must hold %d x %d values" % (R, n))
        data = self._empty((max(need.value, 16),), torch.uint8, codes.device)
        self._ck(self.lib.obc_pack4(self.h, _ptr(codes, torch.int32), _ptr(delta, torch.float32),
                                    _ptr(offset, torch.float32), R, d, int(group), _ptr(data)))
        return Packed4(data, R, d, int(group))

    def obc_product4(self, W, x, x_scale=None, out=None, out_dtype=None):
        """y = x W^T (T x rows) of a Packed4.  x: T x cols, fp32, fp16, bf16, or int8 with its scales (T).  y has
        out's type, else out_dtype, else x's (int8: bf16)."""
        data, R, cols, group = W
        _no_grad(x, x_scale, out)
        xt = _type_of(x, "x", i8=True)
        xp, ldx, T, d = _rows_of(x, "x")
        if d != cols:
            raise ValueError("x has %d columns, the weights %d" % (d, cols))
        if out is None:
            if out_dtype is None:
                out_dtype = torch.bfloat16 if xt == I8 else x.dtype
            out = self._empty((T, R), out_dtype, x.device)
        yp, ldy, rows, n = _rows_of(out, "out")
        if rows != T or n != R:
            raise ValueError("out must be %d x %d" % (T, R))
        ws, n, _held = self._need("obc_product4_workspace_bytes", T, R, d, group, xt)
        rc = self.lib.obc_product4(self.h, data.data_ptr(), R, d, group, xp, xt,
                                   None if x_scale is None else _vector(x_scale, T, "x_scale"), T, ldx, yp, _type_of(out, "out"),
                                   ldy, ws, n)
        if rc != OBC_OK:
            self._ck(rc)
        return out

    def obc_product4_grad(self, W, dy, out=None):
        """dx = dy W (T x cols), the gradient of obc_product4's inputs, in dy's type."""
        _no_grad(dy, out)
        t = _type_of(dy, "dy")
        dp, lddy, T, R = _rows_of(dy, "dy")
        if R != W.rows:
            raise ValueError("dy has %d columns, the weights %d rows" % (R, W.rows))
        if out is None:
            out = self._empty((T, W.cols), dy.dtype, dy.device)
        if out.dtype != dy.dtype:
            raise ValueError("out must have dy's type")
        xp, lddx, rows, n = _rows_of(out, "out")
        if rows != T or n != W.cols:
            raise ValueError("out must be %d x %d" % (T, W.cols))
        ws, n, _held = self._need("obc_product4_grad_workspace_bytes", T, R, W.cols, W.group, t)
        self._ck(self.lib.obc_product4_grad(self.h, W.data.data_ptr(), R, W.cols, W.group, dp, t, T, lddy, xp, lddx, ws, n))
        return out

    def obc_rmsnorm(self, x, gain, eps=1e-6, residual=None, quant8=False, want_rstd=False, out=None):
        """h = x + residual and its root-mean-square norm y.  out may hold h, y, scale (quant8) and rstd; without a
        residual, h is x itself."""
        T, d = x.shape
        t = _type_of(x, "x")
        out = {} if out is None else out
        _no_grad(x, gain, residual, *out.values())
        h = out.get("h")
        if h is None and residual is not None:
            h = self._empty((T, d), x.dtype, x.device)
        y = out.get("y")
        if y is None:
            y = self._empty((T, d), torch.int8 if quant8 else x.dtype, x.device)
        scale = out.get("scale")
        if scale is None and quant8:
            scale = self._empty((T,), torch.float32, x.device)
        rstd = out.get("rstd")
        if rstd is None and want_rstd:
            rstd = self._empty((T,), torch.float32, x.device)
        for other in (residual, h, y):
            if other is not None and other.shape != x.shape:
                raise ValueError("residual, h and y must have x's shape")
        self._ck(self.lib.obc_rmsnorm(self.h, _ptr(x), _ptr(residual, x.dtype), t, _vector(gain, d, "gain"), float(eps), T, d,
                                      _ptr(h, x.dtype), _ptr(y, torch.int8 if quant8 else x.dtype), I8 if quant8 else t,
                                      _vector(scale, T, "scale") if quant8 else None, _vector(rstd, T, "rstd")))
        return dict(h=x if h is None else h, y=y, scale=scale, rstd=rstd)

    def obc_rmsnorm_grad(self, h, gain, rstd, dy, dh=None, out=None):
        """Gradients of x (and of the residual) and of the gain, from what the forward pass left; out may hold dx and
        dgain."""
        T, d = h.shape
        t = _type_of(h, "h")
        out = {} if out is None else out
        _no_grad(h, gain, rstd, dy, dh, *out.values())
        dx = out.get("dx")
        if dx is None:
            dx = self._empty((T, d), h.dtype, h.device)
        dgain = out.get("dgain")
        if dgain is None:
            dgain = self._empty((d,), torch.float32, h.device)
        for other in (dy, dh, dx):
            if other is not None and other.shape != h.shape:
                raise ValueError("dy, dh and dx must have h's shape")
        ws, n, _held = self._need("obc_rmsnorm_grad_workspace_bytes", T, d)
        self._ck(self.lib.obc_rmsnorm_grad(self.h, _ptr(h), _vector(gain, d, "gain"), _vector(rstd, T, "rstd"), _ptr(dy, h.dtype),
                                           _ptr(dh, h.dtype), t, T, d, _ptr(dx, h.dtype), _vector(dgain, d, "dgain"), ws, n))
        return dict(dx=dx, dgain=dgain)

    def obc_distill(self, z, top_index, top_logit, temperature=1.0, weight=None, want_grad=False, out=None):
        """Distillation loss (T) of logits z (T x V) against a teacher's top logits (T x k), and the gradient dz with
        want_grad; out may hold loss and dz (z itself, to overwrite the logits)."""
        t = _type_of(z, "z")
        zp, ldz, T, V = _rows_of(z, "z")
        out = {} if out is None else out
        _no_grad(z, top_logit, weight, *out.values())
        loss = out.get("loss")
        if loss is None:
            loss = self._empty((T,), torch.float32, z.device)
        dz = out.get("dz") if want_grad else None
        if dz is None and want_grad:
            dz = self._empty((T, V), z.dtype, z.device)
        gp, ldg = (None, 0)
        if dz is not None:
            if dz.dtype != z.dtype:
                raise ValueError("dz must have z's type")
            gp, ldg, rows, n = _rows_of(dz, "dz")
            if rows != T or n != V:
                raise ValueError("dz must be %d x %d" % (T, V))
        if top_index.shape != top_logit.shape or top_index.dim() != 2 or top_index.shape[0] != T:
            raise ValueError("top_index and top_logit must be T x k")
        k = top_index.shape[1]
        self._ck(self.lib.obc_distill(self.h, zp, t, T, V, ldz, _ptr(top_index, torch.int32), _ptr(top_logit, torch.float32), k,
                                      float(temperature), _vector(weight, T, "weight"), _vector(loss, T, "loss"), gp, ldg))
        return dict(loss=loss, dz=dz)

    # ------------------------------------------------------- judging and tuning them
    def obc_score(self, z, target=None, top=0, temperature=1.0, out=None):
        """Log-sum-exp and entropy (T) of logits z (T x V) at a temperature, the log probabilities of target (T int32; negative:
        none) and the `top` largest logits with their indices, which obc_distill takes.  out may hold logp, entropy, lse, top_index
        and top_logit."""
        t = _type_of(z, "z")
        zp, ldz, T, V = _rows_of(z, "z")
        out = {} if out is None else out
        self._take(z, target, *out.values())
        k = int(top)
        if k < 0:
            raise ValueError("top must not be negative")
        logp, entropy, lse = out.get("logp"), out.get("entropy"), out.get("lse")
        index, logit = (out.get("top_index"), out.get("top_logit")) if k else (None, None)
        if target is None:
            logp = None
        elif logp is None:
            logp = self._empty((T,), torch.float32, z.device)
        if entropy is None:
            entropy = self._empty((T,), torch.float32, z.device)
        if lse is None:
            lse = self._empty((T,), torch.float32, z.device)
        if k:
            if index is None:
                index = self._empty((T, k), torch.int32, z.device)
            if logit is None:
                logit = self._empty((T, k), torch.float32, z.device)
            if index.shape != (T, k) or logit.shape != (T, k):
                raise ValueError("top_index and top_logit must be %d x %d" % (T, k))
        ws, n, _held = self._need("obc_score_workspace_bytes", T, V, t, k)
        rc = self.lib.obc_score(self.h, zp, t, T, V, ldz, _ints(target, T, "target"), float(temperature), k, _vector(logp, T, "logp"),
                                _vector(entropy, T, "entropy"), _vector(lse, T, "lse"), _ints(index, T * k, "top_index"),
                                _vector(logit, T * k, "top_logit"), ws, n)
        if rc != OBC_OK:
            self._ck(rc)
        return dict(logp=logp, entropy=entropy, lse=lse, top_index=index, top_logit=logit)

    def obc_layernorm(self, x, gain, bias=None, eps=1e-5, residual=None, quant8=False, want_stats=False, out=None):
        """h = x + residual and its layer norm y.  out may hold h, y, scale (quant8), mean and rstd; without a residual, h is x
        itself."""
        T, d = shape = x.shape
        t = _type_of(x, "x")
        out = {} if out is None else out
        self._take(x, gain, bias, residual, *out.values())
        h = out.get("h")
        if h is None and residual is not None:
            h = self._empty((T, d), x.dtype, x.device)
        y = out.get("y")
        if y is None:
            y = self._empty((T, d), torch.int8 if quant8 else x.dtype, x.device)
        scale = out.get("scale")
        if scale is None and quant8:
            scale = self._empty((T,), torch.float32, x.device)
        mean, rstd = out.get("mean"), out.get("rstd")
        if want_stats:
            mean = self._empty((T,), torch.float32, x.device) if mean is None else mean
            rstd = self._empty((T,), torch.float32, x.device) if rstd is None else rstd
        for other in (residual, h, y):
            if other is not None and other.shape != shape:
                raise ValueError("residual, h and y must have x's shape")
        self._ck(self.lib.obc_layernorm(self.h, _ptr(x), _ptr(residual, x.dtype), t, _vector(gain, d, "gain"), _vector(bias, d, "bias"),
                                        float(eps), T, d, _ptr(h, x.dtype), _ptr(y, torch.int8 if quant8 else x.dtype),
                                        I8 if quant8 else t, _vector(scale, T, "scale") if quant8 else None, _vector(mean, T, "mean"),
                                        _vector(rstd, T, "rstd")))
        return dict(h=x if h is None else h, y=y, scale=scale, mean=mean, rstd=rstd)

    def obc_layernorm_grad(self, h, gain, mean, rstd, dy, dh=None, out=None):
        """Gradients of x (and of the residual), the gain and the bias, from what the forward pass left; out may hold dx, dgain and
        dbias."""
        T, d = shape = h.shape
        t = _type_of(h, "h")
        out = {} if out is None else out
        self._take(h, gain, mean, rstd, dy, dh, *out.values())
        dx = out.get("dx")
        if dx is None:
            dx = self._empty((T, d), h.dtype, h.device)
        dgain = out.get("dgain")
        if dgain is None:
            dgain = self._empty((d,), torch.float32, h.device)
        dbias = out.get("dbias")
        if dbias is None:
            dbias = self._empty((d,), torch.float32, h.device)
        for other in (dy, dh, dx):
            if other is not None and other.shape != shape:
                raise ValueError("dy, dh and dx must have h's shape")
        ws, n, _held = self._need("obc_layernorm_grad_workspace_bytes", T, d)
        self._ck(self.lib.obc_layernorm_grad(self.h, _ptr(h), _vector(gain, d, "gain"), _vector(mean, T, "mean"), _vector(rstd, T, "rstd"),
                                             _ptr(dy, h.dtype), _ptr(dh, h.dtype), t, T, d, _ptr(dx, h.dtype),
                                             _vector(dgain, d, "dgain"), _vector(dbias, d, "dbias"), ws, n))
        return dict(dx=dx, dgain=dgain, dbias=dbias)

    def obc_embed(self, table, ids, scale=1.0, out=None, out_dtype=None):
        """y[t] = scale table[ids[t]] (T x d); ids: T int32, negative: a row of zeros.  y has out's type, else out_dtype, else the
        table's."""
        self._take(table, ids, out)
        t = _type_of(table, "table")
        tp, ldt, V, d = _rows_of(table, "table")
        T = ids.numel()
        if out is None:
            out = self._empty((T, d), table.dtype if out_dtype is None else out_dtype, table.device)
        yp, ldy, rows, n = _rows_of(out, "out")
        if rows != T or n != d:
            raise ValueError("out must be %d x %d" % (T, d))
        rc = self.lib.obc_embed(self.h, tp, t, V, d, ldt, _ints(ids, T, "ids"), T, float(scale), yp, _type_of(out, "out"), ldy)
        if rc != OBC_OK:
            self._ck(rc)
        return out

    def obc_embed_grad(self, ids, dy, rows, scale=1.0, out=None, out_dtype=None, accumulate=False):
        """The gradient (rows x d) of a table of so many rows that obc_embed read, from dy (T x d).  out's type, else out_dtype, else
        dy's; accumulate: added to out."""
        self._take(ids, dy, out)
        t = _type_of(dy, "dy")
        dp, lddy, T, d = _rows_of(dy, "dy")
        if out is None:
            if accumulate:
                raise ValueError("accumulate adds to out, which is missing")
            out = self._empty((int(rows), d), dy.dtype if out_dtype is None else out_dtype, dy.device)
        gp, ldt, V, n = _rows_of(out, "out")
        if V != rows or n != d:
            raise ValueError("out must be %d x %d" % (rows, d))
        ws, n, _held = self._need("obc_embed_grad_workspace_bytes", T, V, d)
        self._ck(self.lib.obc_embed_grad(self.h, _ints(ids, T, "ids"), T, dp, t, lddy, float(scale), V, d, int(bool(accumulate)), gp,
                                         _type_of(out, "out"), ldt, ws, n))
        return out

    def obc_adamw_state(self, p, bits=32, master=False):
        """Moments of zero for a parameter tensor, in 32 or 8 bits, and an fp32 copy of it with master."""
        n = p.numel()
        if bits not in (8, 32):
            raise ValueError("moments have 8 or 32 bits")
        with torch.no_grad(), torch.cuda.stream(self.stream):
            def zeros(m, dtype):
                return torch.zeros(m, dtype=dtype, device=p.device)

            copy = p.detach().to(torch.float32, copy=True, memory_format=torch.contiguous_format) if master else None
            if bits == 32:
                return AdamState(zeros(p.shape, torch.float32), zeros(p.shape, torch.float32), None, None, copy)
            blocks = -(-n // 256)
            return AdamState(zeros(p.shape, torch.float8_e4m3fn), zeros(p.shape, torch.float8_e4m3fn), zeros(blocks, torch.float32),
                             zeros(blocks, torch.float32), copy)

    def obc_adamw_plan(self, params, grads, states, decay=0.01, out=None):
        """The lists of parameters, gradients of their type, and AdamStates (all of 32 or all of 8 bits) that obc_adamw goes over, as it
        takes them; kept from step to step.  decay: a float or one for each tensor.  Steps are in place, unless out holds other
        parameters and states."""
        return AdamPlan(self, params, grads, states, decay, out)

    def obc_adamw(self, plan, step, lr, beta1=0.9, beta2=0.999, eps=1e-8, grad_scale=None, seed=0):
        """A step of AdamW over an AdamPlan's tensors.  step: an int, 1 for the first, or an int64 tensor on the device; lr: a float or
        an fp32 tensor on the device; grad_scale: an fp32 tensor on the device.  Returns the new parameters and states."""
        if plan.ctx is not self:
            raise ValueError("the plan is another context's, whose stream it was laid out on")
        step_at = lr_at = None
        self._take(grad_scale, *(t for t in (step, lr) if torch.is_tensor(t)))
        if torch.is_tensor(step):
            if step.numel() != 1:
                raise ValueError("step must be one value")
            step_at, step = _ptr(step, torch.int64), 0
        if torch.is_tensor(lr):
            lr_at, lr = _vector(lr, 1, "lr"), 0.0
        rc = self.lib.obc_adamw(self.h, plan.address, plan.count, plan.workgroups, plan.type, plan.bits, int(step), step_at, float(lr),
                                lr_at, float(beta1), float(beta2), float(eps), _vector(grad_scale, 1, "grad_scale"), int(seed) & 0xffffffff)
        if rc != OBC_OK:
            self._ck(rc)
        return plan.new
