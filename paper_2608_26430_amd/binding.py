"""ctypes binding of libframeft.so: argument marshalling only.

Every computation happens in the HIP library; this module turns torch
tensors into device pointers and the current torch stream into the hipStream_t
of the C ABI (include/frameft.h).  There is no fallback: if the library is not
built, or a call fails, a FrameFTError is raised.
"""
from __future__ import annotations

import ctypes
import os
import struct
from typing import Optional, Sequence

import numpy as np

_HERE = os.path.dirname(os.path.abspath(__file__))
_LIB_PATH = os.path.join(_HERE, "libframeft.so")
_lib = None

FF_F32, FF_BF16 = 0, 1
_STATUS = {0: "FF_OK", 1: "FF_EINVAL", 2: "FF_ENOTFF", 3: "FF_EUNSUPPORTED", 4: "FF_ENOMEM",
           5: "FF_EDEVICE"}


class FrameFTError(RuntimeError):
    """A libframeft call returned an error status (or the library is missing)."""

    def __init__(self, status: int, message: str):
        super().__init__(f"{_STATUS.get(status, status)}: {message}")
        self.status = status
        self.name = _STATUS.get(status, str(status))


def library_path() -> str:
    return _LIB_PATH


def _load():
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(_LIB_PATH):
        raise FrameFTError(5, f"{_LIB_PATH} is not built (python -m paper_2608_26430_amd.build)")
    lib = ctypes.CDLL(_LIB_PATH)
    i64, i32, f32, vp = ctypes.c_int64, ctypes.c_int, ctypes.c_float, ctypes.c_void_p
    u64, f64, pi64 = ctypes.c_uint64, ctypes.c_double, ctypes.POINTER(ctypes.c_int64)
    dp = ctypes.POINTER(ctypes.c_double)
    sig = {
        "ff_status_string": (ctypes.c_char_p, [i32]),
        "ff_last_error": (ctypes.c_char_p, []),
        "ff_abi_version": (i32, []),
        "ff_tff_host": (i32, [i64, i64, i64, i64, i64, dp]),
        "ff_framegen": (i32, [i64, i64, i64, ctypes.POINTER(vp)]),
        "ff_frame_export": (i32, [vp, i64, i64, dp]),
        "ff_frame_info": (i32, [vp, ctypes.POINTER(i64), ctypes.POINTER(i64), ctypes.POINTER(i64)]),
        "ff_frame_destroy": (None, [vp]),
        "ff_plan_create": (i32, [vp, vp, i64, vp, vp, i64, i64, ctypes.POINTER(vp)]),
        "ff_plan_destroy": (None, [vp]),
        "ff_plan_query": (i32, [vp, i32, ctypes.POINTER(i64)]),
        "ff_plan_order": (i32, [vp, ctypes.POINTER(i64)]),
        "ff_adapter_fwd": (i32, [vp, i64, i32, vp, i64, vp, f32, f32, vp, i64, vp]),
        "ff_adapter_bwd": (i32, [vp, i64, i32, vp, i64, vp, i64, vp, f32, f32, vp, i64, i32, vp, vp]),
        "ff_adapter_fwd_save": (i32, [vp, i64, i32, vp, i64, vp, f32, f32, vp, i64, vp, vp]),
        "ff_adapter_bwd_saved": (i32, [vp, i64, i32, vp, i64, vp, i64, vp, vp, f32, f32, vp, i64, i32, vp, vp]),
        "ff_merge_delta": (i32, [vp, vp, f32, i32, f32, vp, i64, vp]),
        "ff_adapter_fwd_batched": (i32, [vp, i64, i64, i32, vp, i64, vp, f32, f32, vp, i64, vp]),
        "ff_adapter_bwd_batched": (i32, [vp, i64, i64, i32, vp, i64, vp, i64, vp, f32, f32, vp, i64, i32,
                                         vp, vp]),
        "ff_time_next_kernel": (i32, [vp, vp]),
        "ff_adapter_bwd_noalloc": (i32, [vp, i64, i32, vp, i64, vp, i64, vp, f32, f32, vp, i64, i32, vp, vp]),
        "ff_plan_group_create": (i32, [i64, vp, ctypes.POINTER(vp)]),
        "ff_plan_group_destroy": (None, [vp]),
        "ff_adapter_fwd_group": (i32, [vp, i64, vp, i32, vp, i64, vp, f32, f32, vp, i64, vp]),
        "ff_adapter_bwd_group": (i32, [vp, i64, vp, i32, vp, i64, vp, i64, vp, f32, f32, vp, i64, i32, vp, vp]),
        "ff_adamw_step": (i32, [i64, vp, vp, vp, vp, f32, f32, f32, f32, f32, i64, vp]),
        "ff_adamw_step_batched": (i32, [i64, i64, vp, vp, vp, vp, f32, f32, f32, f32, f32, i64, vp]),
        "ff_lr_linear_warmup": (ctypes.c_double, [i64, i64, i64, ctypes.c_double]),
        "ff_adamw_set_create": (i32, [i64, vp, i32, i32, vp, vp, vp, vp, vp, vp, vp, ctypes.POINTER(vp)]),
        "ff_adamw_set_destroy": (None, [vp]),
        "ff_adamw_set_step": (i32, [vp, vp, vp, vp]),
        "ff_adamw_set_read": (i32, [vp, vp, vp, vp]),
        "ff_coef_to_plan": (i32, [vp, vp, vp, vp]),
        "ff_coef_to_user": (i32, [vp, vp, vp, i32, vp]),
        "ff_layernorm_fwd": (i32, [i64, i64, i32, vp, i64, i32, vp, vp, f32, vp, i64, vp, vp, vp]),
        "ff_layernorm_workspace": (i32, [i64, i64, pi64]),
        "ff_layernorm_bwd": (i32, [i64, i64, i32, vp, i64, vp, i64, i32, vp, vp, vp, f32, vp, i64, i32, vp, vp, vp, i64,
                                   vp]),
        "ff_resnorm_fwd": (i32, [vp, vp, i64, vp, i64, vp, i64, vp, i64, vp, vp]),
        "ff_resnorm_workspace": (i32, [i64, i64, i64, pi64]),
        "ff_resnorm_bwd": (i32, [vp, vp, i64, vp, i64, vp, i64, vp, i64, vp, vp, i64, vp, i64, i32, vp, vp, vp, vp, vp, vp, i64,
                                 vp]),
        "ff_glu_fwd": (i32, [i64, i64, i64, i32, i32, vp, i64, vp, vp, i64, vp, vp, i64, vp, i64, vp, vp, i64, vp]),
        "ff_glu_workspace": (i32, [i64, i64, i64, i32, i32, pi64]),
        "ff_glu_bwd": (i32, [i64, i64, i64, i32, i32, vp, i64, vp, i64, vp, vp, i64, vp, vp, i64, vp, vp, i64, vp, vp, i64, f32,
                             vp, i64, f32, vp, vp, i64, vp, i64, vp]),
        "ff_dropout": (i32, [i64, i64, i32, vp, i64, f64, u64, u64, vp, vp, i64, vp, i64, vp]),
        "ff_xent_workspace": (i32, [i64, i64, i64, i32, i32, pi64]),
        "ff_xent_fwd": (i32, [i64, i64, i64, i32, vp, i64, vp, i64, vp, vp, vp, vp, i64, vp]),
        "ff_xent_bwd": (i32, [i64, i64, i64, i32, vp, i64, vp, i64, vp, vp, vp, vp, f32, f32, vp, i64, f32, vp, i64, vp,
                              i64, vp]),
        "ff_xent_step": (i32, [i64, i64, i64, i32, vp, i64, vp, i64, vp, vp, f32, vp, vp, f32, vp, i64, f32, vp, i64, vp,
                               i64, vp]),
    }
    for name, (res, args) in sig.items():
        fn = getattr(lib, name)
        fn.restype = res
        fn.argtypes = args
    _lib = lib
    return lib


def _check(status: int):
    if status:
        raise FrameFTError(status, _load().ff_last_error().decode())


# ------------------------------------------------------------------ frames

def tff_host(d: int, k: int, rho: int, col0: int = 0, ncols: Optional[int] = None) -> np.ndarray:
    """Columns col0.. of the real (k, rho, d) tight fusion frame from the library's host construction."""
    lib = _load()
    if ncols is None:
        ncols = k * rho - col0
    out = np.zeros((d, max(ncols, 0)), dtype=np.float64)
    _check(lib.ff_tff_host(d, k, rho, col0, ncols, out.ctypes.data_as(ctypes.POINTER(ctypes.c_double))))
    return out


class Frame:
    """A frame on the current device (ff_framegen)."""

    def __init__(self, handle: int, d: int, k: int, rho: int):
        self._h = ctypes.c_void_p(handle)
        self.d, self.k, self.rho = d, k, rho

    @property
    def handle(self):
        return self._h

    def export(self, col0: int = 0, ncols: Optional[int] = None) -> np.ndarray:
        """Columns of P as the kernels see them (fp32 block read back), fp64 d x ncols."""
        if ncols is None:
            ncols = self.k * self.rho - col0
        out = np.zeros((self.d, ncols), dtype=np.float64)
        _check(_load().ff_frame_export(self._h, col0, ncols,
                                       out.ctypes.data_as(ctypes.POINTER(ctypes.c_double))))
        return out

    def close(self):
        if self._h:
            _load().ff_frame_destroy(self._h)
            self._h = ctypes.c_void_p(None)

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


def framegen(d: int, k: int, rho: int) -> Frame:
    """TFF(k, rho, d) on the current device (Algorithm 1, step 2)."""
    lib = _load()
    h = ctypes.c_void_p()
    _check(lib.ff_framegen(d, k, rho, ctypes.byref(h)))
    return Frame(h.value, d, k, rho)


# ------------------------------------------------------------------ plans

class Plan:
    """Support of C on a pair of frames, with device tables and workspace."""

    def __init__(self, f_in: Frame, f_out: Frame, rows, cols, max_tokens: int, max_batch: int = 1):
        lib = _load()
        rows = np.ascontiguousarray(rows, dtype=np.int32)
        cols = np.ascontiguousarray(cols, dtype=np.int32)
        if rows.shape != cols.shape or rows.ndim != 1:
            raise ValueError("rows and cols must be 1-D of equal length")
        h = ctypes.c_void_p()
        _check(lib.ff_plan_create(f_in.handle, f_out.handle, rows.size,
                                  rows.ctypes.data if rows.size else None,
                                  cols.ctypes.data if cols.size else None,
                                  max_tokens, max_batch, ctypes.byref(h)))
        self._h = h
        self.f_in, self.f_out = f_in, f_out
        self.n, self.m = f_in.d, f_out.d
        self.nnz = int(rows.size)
        self.max_tokens, self.max_batch = max_tokens, max_batch
        self._order = None
        # fixed at creation and needed by every call
        self._coef_slots, self._saved_floats = self.query(5), self.query(6)

    @property
    def handle(self):
        return self._h

    def query(self, key: int) -> int:
        v = ctypes.c_int64()
        _check(_load().ff_plan_query(self._h, key, ctypes.byref(v)))
        return v.value

    def tile_tokens(self, dtype: str) -> int:
        return self.query(FF_BF16 if dtype == "bf16" else FF_F32)

    @property
    def workspace_bytes(self) -> int:
        return self.query(2)

    @property
    def fast128(self) -> bool:
        """True when bf16 calls run the fused kernels for 128-wide frame blocks."""
        return bool(self.query(4))

    @property
    def coef_slots(self) -> int:
        """Length L of every c / dC array of this plan (nnz plus padding slots)."""
        return self._coef_slots

    @property
    def saved_floats(self) -> int:
        """Length of the c_saved arrays of adapter_fwd(save=...) / adapter_bwd(saved=...) (0: none needed)."""
        return self._saved_floats

    @property
    def bwd_tile_tokens(self) -> int:
        """Tokens per workgroup tile of the fused 128-wide backward (16 or 8; 0 without it)."""
        return self.query(7)

    @property
    def radix(self):
        """(input, output) frame application: 4 for the factored radix-4 form, 1 for dense blocks."""
        return self.query(8), self.query(9)

    @property
    def gen_chunks(self) -> int:
        """Input-side chunks of a generic-kernel tile (1: the whole input side at once)."""
        return self.query(10)

    def gen_tile_tokens(self, dtype: str) -> int:
        """Most tokens per generic-kernel tile with those chunks."""
        return self.query(12 if dtype == "bf16" else 11)

    @property
    def gen_token_groups(self) -> bool:
        """True when bf16 generic-kernel tiles keep four tokens of a coefficient together."""
        return bool(self.query(13))

    def new_saved(self, device=None):
        """A c_saved array for one adapter of this plan (None when the plan needs none)."""
        torch = _torch()
        n = self.saved_floats
        return torch.empty((n,), dtype=torch.float32, device=device or "cuda") if n else None

    @property
    def order(self) -> np.ndarray:
        """User index of the support entry in each coefficient slot, -1 for padding:
        c_plan[j] = c_user[order[j]] where order[j] >= 0, dC_user[order[j]] = dC_plan[j]."""
        if self._order is None:
            o = np.empty(self.coef_slots, dtype=np.int64)
            _check(_load().ff_plan_order(self._h, o.ctypes.data_as(ctypes.POINTER(ctypes.c_int64))))
            self._order = o
        return self._order

    def to_plan(self, c_user) -> np.ndarray:
        """Host user-order coefficients (nnz) -> plan layout (L, fp32, zero padding)."""
        c_user = np.asarray(c_user)
        o = self.order
        out = np.zeros(o.size, dtype=np.float32)
        keep = o >= 0
        out[keep] = c_user[o[keep]]
        return out

    def to_user(self, c_plan) -> np.ndarray:
        """Host plan-layout array (L) -> user order (nnz)."""
        c_plan = np.asarray(c_plan)
        o = self.order
        out = np.empty(self.nnz, dtype=c_plan.dtype)
        keep = o >= 0
        out[o[keep]] = c_plan[keep]
        return out

    def close(self):
        if self._h:
            _load().ff_plan_destroy(self._h)
            self._h = ctypes.c_void_p(None)

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


def plan_create(f_in: Frame, f_out: Frame, rows, cols, max_tokens: int, max_batch: int = 1) -> Plan:
    return Plan(f_in, f_out, rows, cols, max_tokens, max_batch)


# ------------------------------------------------------------------ hot path

# A call on a small layer takes the GPU about ten microseconds, so the marshalling of the hot calls
# counts: torch is looked up once, plan sizes are kept on the plan, the stream is taken as the raw
# handle (torch.cuda.current_stream() builds a Stream object), and each tensor is checked in one
# expression.
_T = None


def _torch():
    global _T
    if _T is None:
        import torch
        _T = torch
    return _T


def _act_code(t) -> int:
    d = t.dtype
    torch = _T or _torch()
    if d is torch.bfloat16:
        return FF_BF16
    if d is torch.float32:
        return FF_F32
    raise TypeError(f"unsupported activation dtype {d}")


def _mat(t, name):
    st = t.stride()
    if len(st) != 2 or st[1] != 1 or not t.is_cuda:
        raise ValueError(f"{name} must be a 2-D device tensor with unit column stride")
    return t.data_ptr(), st[0]


def _vec(t, name, length=None):
    if t.dtype is not (_T or _torch()).float32 or not t.is_cuda or not t.is_contiguous():
        raise ValueError(f"{name} must be a contiguous fp32 device tensor")
    if length is not None and t.numel() != length:
        raise ValueError(f"{name} must hold the plan's {length} coefficient slots (Plan.coef_slots)")
    return t.data_ptr()


def _stream(stream):
    if stream is not None:
        return stream.cuda_stream
    torch = _T or _torch()
    return torch._C._cuda_getCurrentRawStream(torch._C._cuda_getDevice())


def adapter_fwd(plan: Plan, X, c_vals, scale: float, Y=None, beta: float = 0.0, stream=None, save=None):
    """Y = beta*Y + scale * P_out C P_in^T x for each token row of X; returns Y.  With `save` (a
    c_saved array, Plan.new_saved) the forward also stores the coefficients in the backward's
    order, for adapter_bwd(saved=...) with the same c_vals (ff_adapter_fwd_save)."""
    T = X.shape[0]
    if Y is None:
        if beta != 0.0:
            raise ValueError("beta != 0 needs an existing Y")
        Y = _torch().empty((T, plan.m), dtype=X.dtype, device=X.device)
    xp, ldx = _mat(X, "X")
    yp, ldy = _mat(Y, "Y")
    if Y.dtype != X.dtype or Y.shape[0] != T:
        raise ValueError("Y must match X in dtype and token count")
    cp = _vec(c_vals, "c_vals", plan._coef_slots)
    lib = _lib or _load()
    if save is not None:
        _check(lib.ff_adapter_fwd_save(plan._h, T, _act_code(X), xp, ldx, cp, scale, beta, yp, ldy,
                                       _vec(save, "save", plan._saved_floats), _stream(stream)))
    else:
        _check(lib.ff_adapter_fwd(plan._h, T, _act_code(X), xp, ldx, cp, scale, beta, yp, ldy, _stream(stream)))
    return Y


def adapter_bwd(plan: Plan, X, G, c_vals, scale: float, dX=None, dC=None, beta_dx: float = 0.0,
                accumulate_dc: bool = False, want_dx: bool = True, want_dc: bool = True, stream=None,
                saved=None):
    """Backward of adapter_fwd for upstream gradient G: returns (dX, dC) (None where not wanted).
    `saved`: the c_saved array of adapter_fwd(save=...) with the same c_vals (ff_adapter_bwd_saved)."""
    T = G.shape[0]
    act = _act_code(G)
    if want_dx and dX is None:
        if beta_dx != 0.0:
            raise ValueError("beta_dx != 0 needs an existing dX")
        dX = _torch().empty((T, plan.n), dtype=G.dtype, device=G.device)
    if want_dc and dC is None:
        if accumulate_dc:
            raise ValueError("accumulate_dc needs an existing dC")
        dC = _torch().empty((plan._coef_slots,), dtype=_torch().float32, device=G.device)
    gp, ldg = _mat(G, "G")
    xp, ldx = _mat(X, "X") if X is not None else (None, plan.n)
    dxp, lddx = _mat(dX, "dX") if want_dx else (None, plan.n)
    dcp = _vec(dC, "dC", plan._coef_slots) if want_dc else None
    cp = _vec(c_vals, "c_vals", plan._coef_slots) if c_vals is not None else None
    lib = _lib or _load()
    if saved is not None:
        _check(lib.ff_adapter_bwd_saved(plan._h, T, act, xp, ldx, gp, ldg, cp, _vec(saved, "saved", plan._saved_floats),
                                        scale, beta_dx, dxp, lddx, int(accumulate_dc), dcp, _stream(stream)))
    else:
        _check(lib.ff_adapter_bwd(plan._h, T, act, xp, ldx, gp, ldg, cp, scale, beta_dx, dxp, lddx,
                                  int(accumulate_dc), dcp, _stream(stream)))
    return (dX if want_dx else None), (dC if want_dc else None)


def adapter_bwd_noalloc(plan: Plan, X, G, c_vals, scale: float, dX, dC, beta_dx: float = 0.0,
                        accumulate_dc: bool = False, stream=None):
    """adapter_bwd through ff_adapter_bwd_noalloc: the library allocates nothing and uses its static
    scratch.  The outputs dX and dC (either may be None to skip it) are the caller's."""
    T = G.shape[0]
    gp, ldg = _mat(G, "G")
    xp, ldx = _mat(X, "X") if X is not None else (None, plan.n)
    dxp, lddx = _mat(dX, "dX") if dX is not None else (None, plan.n)
    dcp = _vec(dC, "dC", plan.coef_slots) if dC is not None else None
    cp = _vec(c_vals, "c_vals", plan.coef_slots) if c_vals is not None else None
    _check(_load().ff_adapter_bwd_noalloc(plan.handle, T, _act_code(G), xp, ldx, gp, ldg, cp, scale, beta_dx,
                                          dxp, lddx, int(accumulate_dc), dcp, _stream(stream)))
    return dX, dC


def _fvec(t, name, n=None):
    torch = _torch()
    if t.dtype != torch.float32 or not t.is_contiguous() or not t.is_cuda or (n is not None and t.numel() != n):
        raise ValueError(f"{name} must be a contiguous fp32 device tensor of {n} elements")
    return t.data_ptr()


def adamw_step(c, g, m, v, lr: float, step: int, beta1: float = 0.9, beta2: float = 0.999, eps: float = 1e-8,
               weight_decay: float = 0.0, stream=None):
    """One AdamW step on device fp32 vectors c, m, v (in place) with gradient g (ff_adamw_step)."""
    n = c.numel()
    _check(_load().ff_adamw_step(n, _fvec(c, "c", n), _fvec(g, "g", n), _fvec(m, "m", n), _fvec(v, "v", n),
                                 lr, beta1, beta2, eps, weight_decay, step, _stream(stream)))
    return c


def adamw_step_batched(cs: Sequence, gs: Sequence, ms: Sequence, vs: Sequence, lr: float, step: int,
                       beta1: float = 0.9, beta2: float = 0.999, eps: float = 1e-8, weight_decay: float = 0.0,
                       stream=None):
    """adamw_step over equally long vectors of many adapters in one launch (ff_adamw_step_batched)."""
    n, dev = cs[0].numel(), cs[0].device
    for group, name in ((cs, "c"), (gs, "g"), (ms, "m"), (vs, "v")):
        for t in group:
            _fvec(t, name, n)
            if t.data_ptr() % 16:
                raise ValueError(f"{name} arrays must be 16-byte aligned")
    ptrs = [pointer_array(x, dev) for x in (cs, gs, ms, vs)]
    _check(_load().ff_adamw_step_batched(len(cs), n, *[p.data_ptr() for p in ptrs], lr, beta1, beta2, eps,
                                         weight_decay, step, _stream(stream)))
    return cs


_HYPER = struct.Struct("@5dqQ3P")       # the fields of ff_adamw_hyper


class _Grads:
    """Gradients of an AdamWSet: the set that checked them, the tensors, kept alive, and their addresses."""

    def __init__(self, owner, tensors, ptrs):
        self.owner, self.tensors, self.ptrs = owner, tensors, ptrs


class AdamWSet:
    """AdamW over tensors of any lengths in one launch (ff_adamw_set_*).

    params: contiguous fp32 device tensors, stepped in place.  weight_decay: one number or one for each tensor.  states: "f32"
    or "8bit".  copies: None, or bf16 tensors (None for some) that every step writes the parameters to.  seed: of the random
    rounding of 8-bit states.  The states are made here, zero, on the current stream: flat arrays (m_all, v_all) that hold tensor i from element
    offsets[i], a multiple of 256, on; m, v (and m_exp, v_exp, exponents of the blocks of 8-bit states) are the tensors'
    views of them, 1-D, to be saved and restored as they are.  The set must live as long as graphs that hold its steps are replayed."""

    def __init__(self, params: Sequence, weight_decay=0.0, states: str = "f32", copies: Optional[Sequence] = None,
                 grad_dtype=None, betas=(0.9, 0.999), eps: float = 1e-8, seed: int = 0):
        self._h = ctypes.c_void_p()
        torch = _torch()
        params = list(params)
        if not params:
            raise ValueError("a set needs at least one tensor")
        if states not in ("f32", "8bit"):
            raise ValueError(f"unknown states {states!r}: 'f32' or '8bit'")
        grad_dtype = torch.float32 if grad_dtype is None else grad_dtype
        if grad_dtype not in (torch.float32, torch.bfloat16):
            raise TypeError(f"unsupported gradient dtype {grad_dtype}")
        self.device = params[0].device
        for i, t in enumerate(params):
            if t.dtype is not torch.float32 or t.device != self.device or not t.is_cuda or not t.is_contiguous():
                raise ValueError(f"parameter {i} must be a contiguous fp32 tensor on one device with the others")
        decay = [float(weight_decay)] * len(params) if isinstance(weight_decay, (int, float)) else [float(x) for x in weight_decay]
        copies = None if copies is None else list(copies)
        if len(decay) != len(params) or (copies is not None and len(copies) != len(params)):
            raise ValueError("weight_decay and copies need one entry for each tensor")
        for i, w in enumerate(copies or []):
            if w is not None and (w.dtype is not torch.bfloat16 or w.numel() != params[i].numel() or w.device != self.device
                                  or not w.is_contiguous()):
                raise ValueError(f"copy {i} must be a contiguous bf16 tensor as long as its parameter, on {self.device}")
        self.params, self.copies, self.states, self.grad_dtype = params, copies, states, grad_dtype
        self.betas, self.eps, self.seed = (float(betas[0]), float(betas[1])), float(eps), int(seed)
        self.lengths = [t.numel() for t in params]
        self.offsets = [0]
        for n in self.lengths:
            self.offsets.append(self.offsets[-1] + (n + 255) // 256 * 256)
        total, eight = self.offsets.pop(), states == "8bit"
        dt = torch.uint8 if eight else torch.float32
        self.m_all, self.v_all = (torch.zeros((total,), dtype=dt, device=self.device) for _ in range(2))
        self.m, self.v = self.views(self.m_all), self.views(self.v_all)
        self.m_exp = self.v_exp = None
        if eight:
            self.m_exp_all, self.v_exp_all = (torch.zeros((total // 256,), dtype=dt, device=self.device) for _ in range(2))
            self.m_exp, self.v_exp = ([x[o // 256:o // 256 + (n + 255) // 256] for o, n in zip(self.offsets, self.lengths)]
                                      for x in (self.m_exp_all, self.v_exp_all))
        count = len(params)

        def ptrs(ts):
            return (ctypes.c_void_p * count)(*[None if t is None or t.numel() == 0 else t.data_ptr() for t in ts]) if ts else None

        with torch.cuda.device(self.device):
            _check(_load().ff_adamw_set_create(
                count, (ctypes.c_int64 * count)(*self.lengths), int(eight), FF_BF16 if grad_dtype is torch.bfloat16 else FF_F32,
                ptrs(params), ptrs(copies), ptrs(self.m), ptrs(self.v), ptrs(self.m_exp), ptrs(self.v_exp),
                (ctypes.c_double * count)(*decay), ctypes.byref(self._h)))

    def views(self, flat):
        """The tensors' parts of an array laid out as m_all and v_all are."""
        return [flat[o:o + n] for o, n in zip(self.offsets, self.lengths)]

    def grads(self, tensors: Sequence) -> _Grads:
        """Checked gradients for step(): contiguous tensors of grad_dtype, None for a tensor that is not to be stepped.  For
        programs whose gradients stay in the same memory; step() takes a list as well."""
        if len(tensors) != len(self.params):
            raise ValueError(f"{len(tensors)} gradients for {len(self.params)} tensors")
        out = []
        for i, (g, n) in enumerate(zip(tensors, self.lengths)):
            if g is None or n == 0:
                out.append(None)
                continue
            if g.dtype is not self.grad_dtype or g.numel() != n or g.device != self.device or not g.is_contiguous():
                raise ValueError(f"gradient {i} must be a contiguous {self.grad_dtype} tensor of {n} elements on {self.device}")
            out.append(g.data_ptr())
        return _Grads(self, list(tensors), (ctypes.c_void_p * len(out))(*out))

    def step(self, grads, lr: float, step: int, grad_scale: float = 1.0, lr_dev=None, grad_scale_dev=None, step_dev=None,
             stream=None):
        """Step number `step` (1 for the first) of every tensor that has a gradient (ff_adamw_set_step).  lr_dev, grad_scale_dev
        (fp32) and step_dev (int64): device tensors of one element, read when the call runs: factors of lr and grad_scale, an
        addend of step."""
        torch = _T or _torch()
        dev = self.device.index
        if _elsewhere(dev):
            with torch.cuda.device(dev):
                return self.step(grads, lr, step, grad_scale, lr_dev, grad_scale_dev, step_dev, stream)
        if not isinstance(grads, _Grads):
            grads = self.grads(grads)
        elif grads.owner is not self:
            raise ValueError("these gradients were checked for another set")
        lrp = scale = at = 0
        if lr_dev is not None:
            lrp = _array(lr_dev.view(1), "lr_dev", 1, torch.float32, dev)
        if grad_scale_dev is not None:
            scale = _array(grad_scale_dev.view(1), "grad_scale_dev", 1, torch.float32, dev)
        if step_dev is not None:
            at = _array(step_dev.view(1), "step_dev", 1, torch.int64, dev)
        h = _HYPER.pack(lr, *self.betas, self.eps, grad_scale, step, self.seed & 0xffffffffffffffff, lrp, scale, at)
        _check((_lib or _load()).ff_adamw_set_step(self._h, grads.ptrs, h, _stream(stream)))

    def read(self, stream=None):
        """(m, v), laid out as m_all and v_all: the values of the moments, in bf16 for 8-bit states (ff_adamw_set_read), the states
        themselves for fp32 ones."""
        if self.states == "f32":
            return self.m_all, self.v_all
        torch = _T or _torch()
        if _elsewhere(self.device.index):
            with torch.cuda.device(self.device):
                return self.read(stream)
        m, v = (_new(self.m_all.shape, torch.bfloat16, self.device, stream) for _ in range(2))
        at = 2 * np.asarray(self.offsets, dtype=np.uint64)
        pm, pv = at + np.uint64(m.data_ptr()), at + np.uint64(v.data_ptr())
        _check((_lib or _load()).ff_adamw_set_read(self._h, pm.ctypes.data, pv.ctypes.data, _stream(stream)))
        return m, v

    def close(self):
        if self._h:
            _load().ff_adamw_set_destroy(self._h)
            self._h = ctypes.c_void_p(None)

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


def lr_linear_warmup(step: int, warmup: int, total: int, base_lr: float) -> float:
    """Learning rate of optimizer step `step` (0-based) under the linear schedule with warmup."""
    return float(_load().ff_lr_linear_warmup(step, warmup, total, base_lr))


def coef_to_plan(plan: Plan, c_user, c_plan=None, stream=None):
    """Device user-order coefficients (nnz fp32) -> plan layout (Plan.coef_slots, zero padding),
    on the device (ff_coef_to_plan); returns c_plan."""
    if c_plan is None:
        c_plan = _torch().empty((plan._coef_slots,), dtype=_torch().float32, device=c_user.device)
    _check((_lib or _load()).ff_coef_to_plan(plan._h, _vec(c_user, "c_user", plan.nnz),
                                             _vec(c_plan, "c_plan", plan._coef_slots), _stream(stream)))
    return c_plan


def coef_to_user(plan: Plan, c_plan, c_user=None, accumulate: bool = False, stream=None):
    """Device plan-layout array (Plan.coef_slots) -> user order (nnz), added to c_user when
    accumulate (ff_coef_to_user); returns c_user."""
    if c_user is None:
        if accumulate:
            raise ValueError("accumulate needs an existing c_user")
        c_user = _torch().empty((plan.nnz,), dtype=_torch().float32, device=c_plan.device)
    _check((_lib or _load()).ff_coef_to_user(plan._h, _vec(c_plan, "c_plan", plan._coef_slots),
                                             _vec(c_user, "c_user", plan.nnz), int(accumulate), _stream(stream)))
    return c_user


def merge_delta(plan: Plan, c_vals, scale: float, W, beta: float = 1.0, stream=None):
    """W = beta*W + scale * P_out C P_in^T in place; returns W."""
    torch = _torch()
    wp, ldw = _mat(W, "W")
    if W.dtype not in (torch.float32, torch.bfloat16) or tuple(W.shape) != (plan.m, plan.n):
        raise ValueError("W must be m x n fp32 or bf16")
    code = FF_BF16 if W.dtype == torch.bfloat16 else FF_F32
    _check(_load().ff_merge_delta(plan.handle, _vec(c_vals, "c_vals", plan.coef_slots), scale, code, beta, wp, ldw,
                                  _stream(stream)))
    return W


def pointer_array(tensors: Sequence, device):
    """Device array of data pointers (int64) for the batched calls."""
    torch = _torch()
    return torch.tensor([t.data_ptr() for t in tensors], dtype=torch.int64, device=device)


def adapter_fwd_batched(plan: Plan, Xs: Sequence, cs: Sequence, scale: float, Ys: Sequence,
                        beta: float = 0.0, stream=None, ptrs=None):
    """adapter_fwd for len(Xs) adapters sharing the plan (one launch).  `ptrs` may hold
    precomputed pointer arrays (X, c, Y) from pointer_array()."""
    count, T = len(Xs), Xs[0].shape[0]
    _, ldx = _mat(Xs[0], "X")
    _, ldy = _mat(Ys[0], "Y")
    dev = Xs[0].device
    px, pc, py = ptrs if ptrs is not None else (pointer_array(Xs, dev), pointer_array(cs, dev),
                                                 pointer_array(Ys, dev))
    _check(_load().ff_adapter_fwd_batched(plan.handle, count, T, _act_code(Xs[0]), px.data_ptr(), ldx,
                                          pc.data_ptr(), scale, beta, py.data_ptr(), ldy, _stream(stream)))
    return Ys


def adapter_bwd_batched(plan: Plan, Xs: Sequence, Gs: Sequence, cs: Sequence, scale: float,
                        dXs: Optional[Sequence], dCs: Optional[Sequence], beta_dx: float = 0.0,
                        accumulate_dc: bool = False, stream=None, ptrs=None):
    """adapter_bwd for len(Gs) adapters sharing the plan (one fused launch + one reduction)."""
    count, T = len(Gs), Gs[0].shape[0]
    dev = Gs[0].device
    _, ldg = _mat(Gs[0], "G")
    _, ldx = _mat(Xs[0], "X")
    lddx = _mat(dXs[0], "dX")[1] if dXs is not None else plan.n
    if ptrs is not None:
        px, pg, pc, pdx, pdc = ptrs
    else:
        px, pg = pointer_array(Xs, dev), pointer_array(Gs, dev)
        pc = pointer_array(cs, dev) if cs is not None else None     # not needed without dX
        pdx = pointer_array(dXs, dev) if dXs is not None else None
        pdc = pointer_array(dCs, dev) if dCs is not None else None
    _check(_load().ff_adapter_bwd_batched(plan.handle, count, T, _act_code(Gs[0]), px.data_ptr(), ldx,
                                          pg.data_ptr(), ldg, pc.data_ptr() if pc is not None else None,
                                          scale, beta_dx,
                                          pdx.data_ptr() if pdx is not None else None, lddx,
                                          int(accumulate_dc), pdc.data_ptr() if pdc is not None else None,
                                          _stream(stream)))
    return dXs, dCs


class PlanGroup:
    """Adapters over one frame pair with a support each (ff_plan_group_create): plans[i] serves
    adapter i.  Keeps the plans alive."""

    def __init__(self, plans: Sequence[Plan]):
        h = ctypes.c_void_p()
        arr = (ctypes.c_void_p * len(plans))(*[p.handle.value for p in plans])
        _check(_load().ff_plan_group_create(len(plans), ctypes.cast(arr, ctypes.c_void_p), ctypes.byref(h)))
        self._h = h
        self.plans = list(plans)
        self.count = len(plans)
        self.n, self.m = plans[0].n, plans[0].m

    @property
    def handle(self):
        return self._h

    def close(self):
        if self._h:
            _load().ff_plan_group_destroy(self._h)
            self._h = ctypes.c_void_p(None)

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


def plan_group(plans: Sequence[Plan]) -> PlanGroup:
    return PlanGroup(plans)


def adapter_fwd_group(group: PlanGroup, Xs: Sequence, cs: Sequence, scale: float, Ys: Sequence, beta: float = 0.0,
                      tokens=None, T: Optional[int] = None, stream=None, ptrs=None):
    """Forward of adapter i on plans[i] (one launch).  `tokens`: optional device int32 tensor of
    per-adapter token counts (each clamped to T, the launch size, default Xs[0].shape[0]).  `ptrs`
    may hold precomputed pointer arrays (X, c, Y) from pointer_array()."""
    T = Xs[0].shape[0] if T is None else T
    _, ldx = _mat(Xs[0], "X")
    _, ldy = _mat(Ys[0], "Y")
    dev = Xs[0].device
    px, pc, py = ptrs if ptrs is not None else (pointer_array(Xs, dev), pointer_array(cs, dev),
                                                 pointer_array(Ys, dev))
    tp = _tokens_ptr(tokens, group.count)
    _check(_load().ff_adapter_fwd_group(group.handle, T, tp, _act_code(Xs[0]), px.data_ptr(), ldx, pc.data_ptr(),
                                        scale, beta, py.data_ptr(), ldy, _stream(stream)))
    return Ys


def adapter_bwd_group(group: PlanGroup, Xs: Sequence, Gs: Sequence, cs: Optional[Sequence], scale: float,
                      dXs: Optional[Sequence], dCs: Optional[Sequence], beta_dx: float = 0.0,
                      accumulate_dc: bool = False, tokens=None, T: Optional[int] = None, stream=None, ptrs=None):
    """Backward of adapter i on plans[i] (dX and/or dC; one launch plus the dC reduction).  `ptrs`
    may hold precomputed pointer arrays (X, G, c, dX, dC)."""
    T = Gs[0].shape[0] if T is None else T
    dev = Gs[0].device
    _, ldg = _mat(Gs[0], "G")
    _, ldx = _mat(Xs[0], "X")
    lddx = _mat(dXs[0], "dX")[1] if dXs is not None else group.n
    if ptrs is not None:
        px, pg, pc, pdx, pdc = ptrs
    else:
        px, pg = pointer_array(Xs, dev), pointer_array(Gs, dev)
        pc = pointer_array(cs, dev) if cs is not None else None
        pdx = pointer_array(dXs, dev) if dXs is not None else None
        pdc = pointer_array(dCs, dev) if dCs is not None else None
    tp = _tokens_ptr(tokens, group.count)
    _check(_load().ff_adapter_bwd_group(group.handle, T, tp, _act_code(Gs[0]), px.data_ptr(), ldx, pg.data_ptr(),
                                        ldg, pc.data_ptr() if pc is not None else None, scale, beta_dx,
                                        pdx.data_ptr() if pdx is not None else None, lddx, int(accumulate_dc),
                                        pdc.data_ptr() if pdc is not None else None, _stream(stream)))
    return dXs, dCs


def _tokens_ptr(tokens, count):
    if tokens is None:
        return None
    torch = _torch()
    if tokens.dtype != torch.int32 or not tokens.is_cuda or not tokens.is_contiguous() or tokens.numel() != count:
        raise ValueError("tokens must be a contiguous int32 device tensor with one count per adapter")
    return tokens.data_ptr()


# ------------------------------------------------------------------ layer norm, dropout, loss

def _new(shape, dtype, device, stream):
    """An empty tensor for a call on `stream`: taken on that stream, so that its memory is not still in use there."""
    torch = _T or _torch()
    if stream is None:
        return torch.empty(shape, dtype=dtype, device=device)
    with torch.cuda.stream(stream):
        return torch.empty(shape, dtype=dtype, device=device)


def _out_rows(t, name, like, stream, beta=0.0):
    """(tensor, pointer, leading dimension) of a result shaped as `like`, made when t is None."""
    if t is None:
        if beta != 0.0:
            raise ValueError(f"beta != 0 needs an existing {name}")
        if stream is None and like.is_contiguous():
            t = (_T or _torch()).empty_like(like)
        else:
            t = _new(like.shape, like.dtype, like.device, stream)
        return t, t.data_ptr(), t.shape[1]
    return (t,) + _rows(t, name, like)


def _out_array(t, name, n, device, stream):
    """(tensor, pointer) of n fp32 results, made when t is None."""
    f32 = (_T or _torch()).float32
    if t is None:
        t = _new(n, f32, device, stream)
        return t, t.data_ptr()
    return t, _array(t, name, n, f32, device.index)


def _rows(t, name, like):
    """Pointer and leading dimension of a tensor that must be shaped as `like`, with rows of its own."""
    st = t.stride()
    if (t.dtype is not like.dtype or t.shape != like.shape or t.get_device() != like.get_device()
            or (st[1] != 1 and t.shape[1] != 1)):
        raise ValueError(f"{name} must be a {like.shape[0]} x {like.shape[1]} {like.dtype} tensor with unit column stride "
                         f"on {like.device}")
    # the stride of a single row says nothing
    return t.data_ptr(), t.shape[1] if t.shape[0] < 2 else st[0]


def _matrix(t, name, shape, dtype, dev, T, n):
    """_rows for a matrix whose shape T x n, type and device are known."""
    st = t.stride()
    if t.shape != shape or t.dtype is not dtype or t.get_device() != dev or (st[1] != 1 and n != 1):
        raise ValueError(f"{name} must be a {T} x {n} {dtype} tensor with unit column stride on device {dev}")
    return t.data_ptr(), (st[0] if T > 1 else n)


def _input(t, name):
    """Pointer, leading dimension, sizes and device index of an activation that the call takes type and device from."""
    st = t.stride()
    dev = t.get_device()
    if len(st) != 2 or dev < 0:
        raise ValueError(f"{name} must be a 2-D device tensor with unit column stride")
    T, n = t.shape
    if st[1] != 1 and n != 1:
        raise ValueError(f"{name} must be a 2-D device tensor with unit column stride")
    return t.data_ptr(), (n if T < 2 else st[0]), T, n, dev


def _array(t, name, n, dtype, dev):
    if t.dtype is not dtype or t.get_device() != dev or t.dim() != 1 or t.numel() != n or not t.is_contiguous():
        raise ValueError(f"{name} must be a contiguous {dtype} tensor of {n} elements on device {dev}")
    return t.data_ptr()


def _workspace(ws, nbytes, device, stream):
    if ws is None:
        return _new((nbytes,), (_T or _torch()).uint8, device, stream)
    if ws.device != device or not ws.is_contiguous():
        raise ValueError(f"workspace must be a contiguous tensor on {device}")
    return ws


def _elsewhere(dev):
    """True when the call's device is not the current one (launches and the default stream are the current one's)."""
    return dev != (_T or _torch())._C._cuda_getDevice()


def _norm_vector(t, name, n, dev):
    """Pointer of a layer norm's weight or bias, None for none."""
    if t is None:
        return None
    return _array(t, name, n, t.dtype, dev)


def layernorm_fwd(X, weight=None, bias=None, eps: float = 1e-5, Y=None, mean=None, rstd=None, stream=None):
    """Layer norm of each row of X (bf16 or fp32): returns (Y, mean, rstd), the last two fp32 per row for
    layernorm_bwd (ff_layernorm_fwd).  weight and bias: fp32 or bf16, both of one type; None for ones / zeros.  Y
    may be X."""
    torch = _T or _torch()
    xp, ldx, T, n, dev = _input(X, "X")
    if _elsewhere(dev):
        with torch.cuda.device(dev):
            return layernorm_fwd(X, weight, bias, eps, Y, mean, rstd, stream)
    act = _act_code(X)
    w_dtype = weight.dtype if weight is not None else (bias.dtype if bias is not None else torch.float32)
    if w_dtype not in (torch.float32, torch.bfloat16) or (bias is not None and bias.dtype is not w_dtype):
        raise ValueError("weight and bias must both be fp32 or both bf16")
    Y, yp, ldy = _out_rows(Y, "Y", X, stream)
    mean, mp = _out_array(mean, "mean", T, X.device, stream)
    rstd, rp = _out_array(rstd, "rstd", T, X.device, stream)
    _check((_lib or _load()).ff_layernorm_fwd(
        T, n, act, xp, ldx, FF_BF16 if w_dtype is torch.bfloat16 else FF_F32, _norm_vector(weight, "weight", n, dev),
        _norm_vector(bias, "bias", n, dev), eps, yp, ldy, mp, rp, _stream(stream)))
    return Y, mean, rstd


def _layernorm_bytes(T, n):
    v = ctypes.c_int64()
    _check((_lib or _load()).ff_layernorm_workspace(T, n, ctypes.byref(v)))
    return v.value


def layernorm_workspace(T: int, n: int, device="cuda"):
    """A workspace for layernorm_bwd calls of up to T rows of n, one such call at a time."""
    return _torch().empty((_layernorm_bytes(T, n),), dtype=_torch().uint8, device=device)


def layernorm_bwd(X, G, weight, mean, rstd, dX=None, dweight=None, dbias=None, beta_dx: float = 0.0,
                  accumulate: bool = False, want_dx: bool = True, want_dw: bool = True, workspace=None, stream=None):
    """Backward of layernorm_fwd for upstream gradient G: returns (dX, dweight, dbias) (None where not wanted), dX =
    beta_dx * dX + ..., dweight and dbias fp32, added to the given ones with `accumulate` (ff_layernorm_bwd)."""
    torch = _T or _torch()
    xp, ldx, T, n, dev = _input(X, "X")
    f32 = torch.float32
    if _elsewhere(dev):
        with torch.cuda.device(dev):
            return layernorm_bwd(X, G, weight, mean, rstd, dX, dweight, dbias, beta_dx, accumulate, want_dx, want_dw,
                                 workspace, stream)
    gp, ldg = _rows(G, "G", X)
    w_dtype = weight.dtype if weight is not None else f32
    if w_dtype not in (f32, torch.bfloat16):
        raise ValueError("weight must be fp32 or bf16")
    if want_dw and accumulate and (dweight is None or dbias is None):
        raise ValueError("accumulate needs existing dweight and dbias")
    dxp, lddx, dwp, dbp, wsp, wsn = None, n, None, None, None, 0
    if want_dx:
        dX, dxp, lddx = _out_rows(dX, "dX", X, stream, beta_dx)
    if want_dw:
        dweight, dwp = _out_array(dweight, "dweight", n, X.device, stream)
        dbias, dbp = _out_array(dbias, "dbias", n, X.device, stream)
        workspace = _workspace(workspace, _layernorm_bytes(T, n) if workspace is None else 0, X.device, stream)
        wsp, wsn = workspace.data_ptr(), workspace.nbytes
    _check((_lib or _load()).ff_layernorm_bwd(
        T, n, _act_code(X), xp, ldx, gp, ldg, FF_BF16 if w_dtype is torch.bfloat16 else FF_F32,
        _norm_vector(weight, "weight", n, dev), _array(mean, "mean", T, f32, dev), _array(rstd, "rstd", T, f32, dev),
        beta_dx, dxp, lddx, int(accumulate), dwp, dbp, wsp, wsn, _stream(stream)))
    return (dX if want_dx else None), (dweight if want_dw else None), (dbias if want_dw else None)


_NORMS = {"none": 0, None: 0, "rms": 1, "layer": 2}
_RESNORM = struct.Struct("@2q5i4x5P2q4f")       # the fields of ff_resnorm


def _resnorm(T, n, act, dev, gate, post, post_weight, post_bias, norm, weight, bias, res_scale, block_scale, eps, post_eps):
    """The description of a join, whether it has a norm of its result, and the number of its gate rows."""
    torch = _T or _torch()
    f32, bf16 = torch.float32, torch.bfloat16
    post_code, norm_code = _NORMS.get(post), _NORMS.get(norm)
    if post_code is None or norm_code is None:
        raise ValueError(f"unknown norms {post!r}, {norm!r}: 'none', 'rms' or 'layer'")
    wt, ptrs, at = None, [0, 0, 0, 0], -1
    for v in (post_weight, post_bias, weight, bias):
        at += 1
        if v is None:
            continue
        if wt is None:
            wt = v.dtype
        if (v.dtype is not wt or (wt is not f32 and wt is not bf16) or v.shape != (n,) or v.get_device() != dev
                or not v.is_contiguous() or not (post_code if at < 2 else norm_code)):
            name = ("post_weight", "post_bias", "weight", "bias")[at]
            if not (post_code if at < 2 else norm_code):
                raise ValueError(f"{name} of a norm that is not there")
            raise ValueError(f"{name} must be a contiguous tensor of {n} elements on device {dev}; the norms' vectors must all be "
                             "fp32 or all bf16")
        ptrs[at] = v.data_ptr()
    groups, gp, ldgate, gate_bf16 = 1, 0, n, 0
    if gate is not None:
        gate_bf16 = int(gate.dtype is bf16)
        if not gate_bf16 and gate.dtype is not f32:
            raise ValueError("gate must be fp32 or bf16")
        shape, st = gate.shape, gate.stride()
        dims = len(st)
        if dims == 2:
            groups = shape[0]
        if (dims < 1 or dims > 2 or shape[-1] != n or gate.get_device() != dev or (n != 1 and st[-1] != 1) or groups < 1
                or T % groups):
            raise ValueError(f"gate must have {n} elements, or rows of {n} whose number divides {T}, on device {dev}")
        gp, ldgate = gate.data_ptr(), (st[0] if groups > 1 else n)
    return _RESNORM.pack(T, n, act, int(wt is bf16), gate_bf16, post_code, norm_code, *ptrs, gp, ldgate, groups, res_scale,
                         block_scale, eps if post_eps is None else post_eps, eps), norm_code, groups


def resnorm_fwd(R, B, gate=None, post="none", post_weight=None, post_bias=None, norm="rms", weight=None, bias=None,
                res_scale: float = 1.0, block_scale: float = 1.0, eps: float = 1e-5, post_eps: Optional[float] = None, X=None,
                Y=None, stats=None, want_stats: bool = True, stream=None):
    """The join of two blocks: x = res_scale R + block_scale gate post(B), y = norm(x); returns (X, Y, stats), Y None without a norm,
    stats (T x 4, fp32) for resnorm_bwd (ff_resnorm_fwd).  post, norm: "none", "rms" or "layer", with vectors in fp32 or
    bf16, all of one type.  gate: n elements, or rows of n, each for an equal share of the rows.  X may be R."""
    torch = _T or _torch()
    rp, ldr, T, n, dev = _input(R, "R")
    if _elsewhere(dev):
        with torch.cuda.device(dev):
            return resnorm_fwd(R, B, gate, post, post_weight, post_bias, norm, weight, bias, res_scale, block_scale, eps,
                               post_eps, X, Y, stats, want_stats, stream)
    shape, dtype = R.shape, R.dtype
    bp, ldb = _matrix(B, "B", shape, dtype, dev, T, n)
    d, has_norm, _ = _resnorm(T, n, _act_code(R), dev, gate, post, post_weight, post_bias, norm, weight, bias, res_scale,
                              block_scale, eps, post_eps)
    plain = stream is None and R.is_contiguous()
    ldx = ldy = n
    yp = sp = None
    if X is None:
        X = torch.empty_like(R) if plain else _new(shape, dtype, R.device, stream)
        xp = X.data_ptr()
    else:
        xp, ldx = _matrix(X, "X", shape, dtype, dev, T, n)
    if has_norm:
        if Y is None:
            Y = torch.empty_like(R) if plain else _new(shape, dtype, R.device, stream)
            yp = Y.data_ptr()
        else:
            yp, ldy = _matrix(Y, "Y", shape, dtype, dev, T, n)
    if stats is not None:
        sp = _stats(stats, T, dev)
    elif want_stats:
        stats = _new((T, 4), torch.float32, R.device, stream)
        sp = stats.data_ptr()
    _check((_lib or _load()).ff_resnorm_fwd(d, rp, ldr, bp, ldb, xp, ldx, yp, ldy, sp, _stream(stream)))
    return X, (Y if has_norm else None), stats


def _stats(t, T, dev):
    if t.dtype is not (_T or _torch()).float32 or t.shape != (T, 4) or t.get_device() != dev or not t.is_contiguous():
        raise ValueError(f"stats must be a contiguous {T} x 4 fp32 tensor on device {dev}")
    return t.data_ptr()


def _resnorm_bytes(T, n, groups):
    v = ctypes.c_int64()
    _check((_lib or _load()).ff_resnorm_workspace(T, n, groups, ctypes.byref(v)))
    return v.value


def resnorm_workspace(T: int, n: int, groups: int = 1, device="cuda"):
    """A workspace for resnorm_bwd calls of T rows of n with `groups` gate rows (1 without a gate), one such call at a time."""
    return _torch().empty((_resnorm_bytes(T, n, groups),), dtype=_torch().uint8, device=device)


def resnorm_bwd(R, B, dX, dY, stats, gate=None, post="none", post_weight=None, post_bias=None, norm="rms", weight=None,
                bias=None, res_scale: float = 1.0, block_scale: float = 1.0, eps: float = 1e-5, post_eps: Optional[float] = None,
                dR=None, dB=None, dgate=None, dpost_weight=None, dpost_bias=None, dweight=None, dbias=None,
                accumulate: bool = False, want_dr: bool = True, want_db: bool = True, want_vectors: bool = True, workspace=None,
                stream=None):
    """Backward of resnorm_fwd from the gradients dX (None: zero) and dY (None without a norm): returns (dR, dB, dgate,
    dpost_weight, dpost_bias, dweight, dbias), the last five fp32 and, with want_vectors, those of the gate and of the vectors that
    were given (and of given outputs); None for the others (ff_resnorm_bwd).  accumulate: the five are added to the given ones;
    no two of them may share memory.  dR and dB may each be any of R, B, dX and dY."""
    torch = _T or _torch()
    f32 = torch.float32
    rp, ldr, T, n, dev = _input(R, "R")
    if _elsewhere(dev):
        with torch.cuda.device(dev):
            return resnorm_bwd(R, B, dX, dY, stats, gate, post, post_weight, post_bias, norm, weight, bias, res_scale,
                               block_scale, eps, post_eps, dR, dB, dgate, dpost_weight, dpost_bias, dweight, dbias, accumulate,
                               want_dr, want_db, want_vectors, workspace, stream)
    shape, dtype = R.shape, R.dtype
    bp, ldb = _matrix(B, "B", shape, dtype, dev, T, n)
    d, has_norm, groups = _resnorm(T, n, _act_code(R), dev, gate, post, post_weight, post_bias, norm, weight, bias, res_scale,
                                   block_scale, eps, post_eps)
    dxp, lddx = _matrix(dX, "dX", shape, dtype, dev, T, n) if dX is not None else (None, n)
    if has_norm and dY is None:
        raise ValueError("a norm needs dY")
    dyp, lddy = _matrix(dY, "dY", shape, dtype, dev, T, n) if has_norm else (None, n)
    plain = stream is None and R.is_contiguous()
    drp = dbp = None
    lddr = lddb = n
    if want_dr:
        if dR is None:
            dR = torch.empty_like(R) if plain else _new(shape, dtype, R.device, stream)
            drp = dR.data_ptr()
        else:
            drp, lddr = _matrix(dR, "dR", shape, dtype, dev, T, n)
    if want_db:
        if dB is None:
            dB = torch.empty_like(R) if plain else _new(shape, dtype, R.device, stream)
            dbp = dB.data_ptr()
        else:
            dbp, lddb = _matrix(dB, "dB", shape, dtype, dev, T, n)
    outs, ptrs, made = [dgate, dpost_weight, dpost_bias, dweight, dbias], [None] * 5, []
    for i, (given, name) in enumerate(((gate, "dgate"), (post_weight, "dpost_weight"), (post_bias, "dpost_bias"),
                                       (weight, "dweight"), (bias, "dbias"))):
        if outs[i] is None:
            if not want_vectors or given is None:
                continue
            if accumulate:
                raise ValueError(f"accumulate needs an existing {name}")
            if i == 0 and groups > 1:
                outs[0] = _new(gate.shape, f32, R.device, stream)
                ptrs[0] = outs[0].data_ptr()
            else:
                made.append(i)
        elif i == 0:
            if gate is None or dgate.dtype is not f32 or dgate.shape != gate.shape or dgate.get_device() != dev \
                    or not dgate.is_contiguous():
                raise ValueError("dgate must be a contiguous fp32 tensor of the gate's shape")
            ptrs[0] = dgate.data_ptr()
        else:
            ptrs[i] = _array(outs[i], name, n, f32, dev)
    if len(made) == 1:
        outs[made[0]] = t = _new((1, n) if made[0] == 0 and gate.dim() == 2 else (n,), f32, R.device, stream)
        ptrs[made[0]] = t.data_ptr()
    elif made:          # the results of n elements in one allocation
        block = _new((len(made), n), f32, R.device, stream)
        at = block.data_ptr()
        for i, t in zip(made, block.unbind(0)):
            outs[i] = t if i or gate.dim() == 1 else t.view(1, n)
            ptrs[i] = at
            at += 4 * n
    workspace = _workspace(workspace, _resnorm_bytes(T, n, groups) if workspace is None else 0, R.device, stream)
    _check((_lib or _load()).ff_resnorm_bwd(
        d, rp, ldr, bp, ldb, dxp, lddx, dyp, lddy, _stats(stats, T, dev), drp, lddr, dbp, lddb, int(accumulate), *ptrs,
        workspace.data_ptr(), workspace.nbytes, _stream(stream)))
    return ((dR if want_dr else None), (dB if want_db else None), *outs)


def dropout(X, p: float, seed: int, offset: int = 0, residual=None, Y=None, offset_dev=None, stream=None):
    """Y = [residual +] mask * X / (1 - p) with a mask that is a function of (seed, offset, row, column, width)
    and is never stored (ff_dropout); the backward pass is the same call on the gradient.  offset_dev: a device int64
    tensor of one element added to offset when the call runs (for captured graphs).  Y may be X or residual."""
    torch = _T or _torch()
    xp, ldx, T, n, dev = _input(X, "X")
    if _elsewhere(dev):
        with torch.cuda.device(dev):
            return dropout(X, p, seed, offset, residual, Y, offset_dev, stream)
    act = _act_code(X)
    Y, yp, ldy = _out_rows(Y, "Y", X, stream)
    rp, ldr = _rows(residual, "residual", X) if residual is not None else (None, n)
    op = _array(offset_dev.view(1), "offset_dev", 1, torch.int64, dev) if offset_dev is not None else None
    _check((_lib or _load()).ff_dropout(T, n, act, xp, ldx, p, seed & (1 << 64) - 1, offset & (1 << 64) - 1, op, rp, ldr,
                                        yp, ldy, _stream(stream)))
    return Y


_GLU = {"silu": 0, "gelu": 1, "gelu_tanh": 2}


def _glu_fn(fn):
    if fn not in _GLU:
        raise ValueError(f"unknown function {fn!r}: 'silu', 'gelu' or 'gelu_tanh'")
    return _GLU[fn]


def _glu_weights(X, Wg, Wu):
    """Sizes, activation code, pointers and leading dimensions of X and the two weights."""
    xp, ldx, T, n, dev = _input(X, "X")
    gp, ldw, F, nw, wdev = _input(Wg, "Wg")
    if nw != n or Wg.dtype is not X.dtype or wdev != dev:
        raise ValueError(f"Wg must be an F x {n} {X.dtype} tensor on {X.device}")
    up, ldu = _matrix(Wu, "Wu", Wg.shape, Wg.dtype, dev, F, n)
    return T, n, F, _act_code(X), xp, ldx, gp, up, _pair(ldw, ldu, "Wg and Wu"), dev


def _pair(ld, other, names):
    if ld != other:
        raise ValueError(f"{names} must have one row stride")
    return ld


def _hidden(t, name, X, T, F, dtype=None):
    """Pointer and leading dimension of a T x F tensor of X's device and type, or that given."""
    st = t.stride()
    if t.dtype is not (dtype or X.dtype) or t.shape != (T, F) or t.get_device() != X.get_device() or st[1] != 1:
        raise ValueError(f"{name} must be a {T} x {F} {dtype or X.dtype} tensor with unit column stride on {X.device}")
    return t.data_ptr(), F if T < 2 else st[0]


def _hidden_pair(a, b, names, X, T, F, dtype=None):
    """The pointers of two T x F tensors, either of which may be None, and their leading dimension."""
    pa, la = _hidden(a, names[0], X, T, F, dtype) if a is not None else (None, None)
    pb, lb = _hidden(b, names[1], X, T, F, dtype) if b is not None else (None, None)
    if la is not None and lb is not None:
        _pair(la, lb, f"{names[0]} and {names[1]}")
    return pa, pb, la if la is not None else (lb if lb is not None else F)


def _kept(X):
    """Type of the tensors that keep G and U."""
    torch = _T or _torch()
    return torch.int16 if X.dtype is torch.bfloat16 else X.dtype


def glu_fwd(X, Wg, Wu, fn: str = "silu", Ag=None, Au=None, H=None, G=None, U=None, save: bool = False, stream=None):
    """H = f(X Wg^T [+ Ag]) * (X Wu^T [+ Au]), fn "silu", "gelu" or "gelu_tanh": returns H, with `save` (H, G, U), the last two what f
    and the product were taken of, for glu_bwd (ff_glu_fwd): fp32, or for bf16 activations int16 tensors of words with ten significant
    bits: a sign, 6 bits of exponent with bias 37, 9 of mantissa.  Values beyond 6.7e7 are infinite words, G & 0x7e00 == 0x7e00; a
    backward without G and U has no such limit.  Wg and Wu: F x n with one row stride, e.g. halves of one weight."""
    torch = _T or _torch()
    T, n, F, act, xp, ldx, wg, wu, ldw, dev = _glu_weights(X, Wg, Wu)
    if _elsewhere(dev):
        with torch.cuda.device(dev):
            return glu_fwd(X, Wg, Wu, fn, Ag, Au, H, G, U, save, stream)
    f = _glu_fn(fn)
    ap, bp, lda = _hidden_pair(Ag, Au, ("Ag", "Au"), X, T, F)
    if H is None:
        H = _new((T, F), X.dtype, X.device, stream)
        hp, ldh = H.data_ptr(), F
    else:
        hp, ldh = _hidden(H, "H", X, T, F)
    gp = up = None
    ldg = F
    if save:
        G = _new((T, F), _kept(X), X.device, stream) if G is None else G
        U = _new((T, F), _kept(X), X.device, stream) if U is None else U
        gp, up, ldg = _hidden_pair(G, U, ("G", "U"), X, T, F, _kept(X))
    elif G is not None or U is not None:
        raise ValueError("G and U are written with save")
    _check((_lib or _load()).ff_glu_fwd(T, n, F, act, f, xp, ldx, wg, wu, ldw, ap, bp, lda, hp, ldh, gp, up, ldg, _stream(stream)))
    return (H, G, U) if save else H


def _glu_bytes(T, n, F, act, want):
    v = ctypes.c_int64()
    _check((_lib or _load()).ff_glu_workspace(T, n, F, act, want, ctypes.byref(v)))
    return v.value


def glu_workspace(T: int, n: int, F: int, dtype, want_dx: bool = True, want_dw: bool = False, device="cuda"):
    """A workspace for glu_bwd calls of these sizes and outputs, one such call at a time."""
    torch = _torch()
    if dtype not in (torch.float32, torch.bfloat16):
        raise TypeError(f"unsupported activation dtype {dtype}")
    nbytes = _glu_bytes(T, n, F, FF_BF16 if dtype is torch.bfloat16 else FF_F32, int(want_dx) + 2 * int(want_dw))
    return torch.empty((nbytes,), dtype=torch.uint8, device=device)


def glu_bwd(dH, X, Wg, Wu, fn: str = "silu", G=None, U=None, Ag=None, Au=None, dG=None, dU=None, dX=None, dWg=None, dWu=None,
            beta_dx: float = 0.0, beta_dw: float = 0.0, want_dx: bool = True, want_dw: bool = False, workspace=None, stream=None):
    """Backward of glu_fwd from the gradient dH of H: returns (dG, dU, dX, dWg, dWu), the last three None where not wanted
    (ff_glu_bwd).  G, U: kept by the forward; without them they are made again, and Ag and Au are what the forward added.  dG and dU
    are also the gradients of what adapters added; dG or dU may be dH, and they may take the memory of G and U (G.view(X.dtype))."""
    torch = _T or _torch()
    T, n, F, act, xp, ldx, wg, wu, ldw, dev = _glu_weights(X, Wg, Wu)
    if _elsewhere(dev):
        with torch.cuda.device(dev):
            return glu_bwd(dH, X, Wg, Wu, fn, G, U, Ag, Au, dG, dU, dX, dWg, dWu, beta_dx, beta_dw, want_dx, want_dw, workspace,
                           stream)
    f = _glu_fn(fn)
    if (G is None) != (U is None):
        raise ValueError("G and U are kept together")
    dhp, lddh = _hidden(dH, "dH", X, T, F)
    gp, up, ldg = _hidden_pair(G, U, ("G", "U"), X, T, F, _kept(X))
    ap, bp, lda = _hidden_pair(Ag, Au, ("Ag", "Au"), X, T, F)
    dG = _new((T, F), X.dtype, X.device, stream) if dG is None else dG
    dU = _new((T, F), X.dtype, X.device, stream) if dU is None else dU
    dgp, dup, lddg = _hidden_pair(dG, dU, ("dG", "dU"), X, T, F)
    dxp = dwg = dwu = wsp = None
    lddx = lddw = n
    wsn = 0
    if want_dx:
        dX, dxp, lddx = _out_rows(dX, "dX", X, stream, beta_dx)
    if want_dw:
        dWg, dwg, lddw = _out_rows(dWg, "dWg", Wg, stream, beta_dw)
        dWu, dwu, other = _out_rows(dWu, "dWu", Wg, stream, beta_dw)
        _pair(lddw, other, "dWg and dWu")
    want = int(want_dx) + 2 * int(want_dw)
    if want:
        workspace = _workspace(workspace, _glu_bytes(T, n, F, act, want) if workspace is None else 0, X.device, stream)
        wsp, wsn = workspace.data_ptr(), workspace.nbytes
    _check((_lib or _load()).ff_glu_bwd(T, n, F, act, f, dhp, lddh, xp, ldx, wg, wu, ldw, ap, bp, lda, gp, up, ldg, dgp, dup, lddg,
                                        beta_dx, dxp, lddx, beta_dw, dwg, dwu, lddw, wsp, wsn, _stream(stream)))
    return dG, dU, (dX if want_dx else None), (dWg if want_dw else None), (dWu if want_dw else None)


def _xent_bytes(T, n, V, act, want):
    v = ctypes.c_int64()
    _check((_lib or _load()).ff_xent_workspace(T, n, V, act, want, ctypes.byref(v)))
    return v.value


def xent_workspace(T: int, n: int, V: int, dtype, want_dh: bool = False, want_dw: bool = False, device="cuda"):
    """A workspace for xent_fwd, xent_bwd and xent_step calls of these sizes and outputs, one such call at a time."""
    torch = _torch()
    if dtype not in (torch.float32, torch.bfloat16):
        raise TypeError(f"unsupported activation dtype {dtype}")
    nbytes = _xent_bytes(T, n, V, FF_BF16 if dtype is torch.bfloat16 else FF_F32, int(want_dh) + 2 * int(want_dw))
    return torch.empty((nbytes,), dtype=torch.uint8, device=device)


def _head(H, W, target):
    hp, ldh, T, n, dev = _input(H, "H")
    wp, ldw, V, nw, wdev = _input(W, "W")
    if V < 1 or nw != n or W.dtype is not H.dtype or wdev != dev:
        raise ValueError(f"W must be a V x {n} {H.dtype} tensor on {H.device}")
    return T, n, V, _act_code(H), hp, ldh, wp, ldw, _array(target, "target", T, (_T or _torch()).int64, dev), dev


def xent_fwd(H, W, target, loss=None, lse=None, workspace=None, stream=None):
    """Cross entropy of the logits H W^T of each token, without keeping the logits: returns (loss, lse), fp32 per token.
    Targets outside [0, V) mark tokens without loss (ff_xent_fwd)."""
    T, n, V, act, hp, ldh, wp, ldw, tp, dev = _head(H, W, target)
    if _elsewhere(dev):
        with _torch().cuda.device(dev):
            return xent_fwd(H, W, target, loss, lse, workspace, stream)
    loss, lop = _out_array(loss, "loss", T, H.device, stream)
    lse, lsp = _out_array(lse, "lse", T, H.device, stream)
    ws = _workspace(workspace, _xent_bytes(T, n, V, act, 0) if workspace is None else 0, H.device, stream)
    _check((_lib or _load()).ff_xent_fwd(T, n, V, act, hp, ldh, wp, ldw, tp, lop, lsp, ws.data_ptr(), ws.nbytes,
                                         _stream(stream)))
    return loss, lse


def _head_grads(H, W, dH, dW, beta_dh, beta_dw, want_dh, want_dw, stream):
    """(dH, its pointer and leading dimension, dW, ...), made where they are wanted and not given."""
    dhp = dwp = None
    ldh = ldw = H.shape[1]
    if want_dh:
        dH, dhp, ldh = _out_rows(dH, "dH", H, stream, beta_dh)
    if want_dw:
        dW, dwp, ldw = _out_rows(dW, "dW", W, stream, beta_dw)
    return (dH if want_dh else None), dhp, ldh, (dW if want_dw else None), dwp, ldw


def xent_bwd(H, W, target, lse, dloss=None, scale: float = 1.0, dH=None, dW=None, beta_dh: float = 0.0,
             beta_dw: float = 0.0, want_dh: bool = True, want_dw: bool = False, workspace=None, stream=None, loss=None):
    """Gradients of sum_t scale dloss[t] loss[t] from the lse of xent_fwd: returns (dH, dW) (None where not wanted);
    dloss: fp32 per token, None for ones; loss: that of xent_fwd, for the target's gradient of tokens whose loss is near
    zero (ff_xent_bwd)."""
    f32 = (_T or _torch()).float32
    T, n, V, act, hp, ldh, wp, ldw, tp, dev = _head(H, W, target)
    if _elsewhere(dev):
        with _torch().cuda.device(dev):
            return xent_bwd(H, W, target, lse, dloss, scale, dH, dW, beta_dh, beta_dw, want_dh, want_dw, workspace, stream,
                            loss)
    dH, dhp, lddh, dW, dwp, lddw = _head_grads(H, W, dH, dW, beta_dh, beta_dw, want_dh, want_dw, stream)
    want = int(want_dh) + 2 * int(want_dw)
    ws = _workspace(workspace, _xent_bytes(T, n, V, act, want) if workspace is None else 0, H.device, stream)
    _check((_lib or _load()).ff_xent_bwd(
        T, n, V, act, hp, ldh, wp, ldw, tp, _array(lse, "lse", T, f32, dev),
        _array(loss, "loss", T, f32, dev) if loss is not None else None,
        _array(dloss, "dloss", T, f32, dev) if dloss is not None else None, scale, beta_dh, dhp, lddh, beta_dw, dwp,
        lddw, ws.data_ptr(), ws.nbytes, _stream(stream)))
    return dH, dW


def xent_step(H, W, target, dloss=None, scale: float = 1.0, loss=None, lse=None, dH=None, dW=None, beta_dh: float = 0.0,
              beta_dw: float = 0.0, want_dh: bool = True, want_dw: bool = False, workspace=None, stream=None):
    """xent_fwd and xent_bwd in one call, which computes the logits once: returns (loss, lse, dH, dW), dH and dW the
    gradients of sum_t scale dloss[t] loss[t] (None where not wanted; ff_xent_step).  A weight that all tokens share belongs
    in scale or on the results: in dloss it is rounded to bf16 with the softmax."""
    f32 = (_T or _torch()).float32
    T, n, V, act, hp, ldh, wp, ldw, tp, dev = _head(H, W, target)
    if _elsewhere(dev):
        with _torch().cuda.device(dev):
            return xent_step(H, W, target, dloss, scale, loss, lse, dH, dW, beta_dh, beta_dw, want_dh, want_dw, workspace,
                             stream)
    loss, lop = _out_array(loss, "loss", T, H.device, stream)
    lse, lsp = _out_array(lse, "lse", T, H.device, stream)
    dH, dhp, lddh, dW, dwp, lddw = _head_grads(H, W, dH, dW, beta_dh, beta_dw, want_dh, want_dw, stream)
    want = int(want_dh) + 2 * int(want_dw)
    ws = _workspace(workspace, _xent_bytes(T, n, V, act, want) if workspace is None else 0, H.device, stream)
    _check((_lib or _load()).ff_xent_step(
        T, n, V, act, hp, ldh, wp, ldw, tp, _array(dloss, "dloss", T, f32, dev) if dloss is not None else None, scale,
        lop, lsp, beta_dh, dhp, lddh, beta_dw, dwp, lddw, ws.data_ptr(), ws.nbytes, _stream(stream)))
    return loss, lse, dH, dW


def time_next_kernel(ev_start, ev_stop):
    """Arm the next hot-path call to record torch.cuda.Events around its main kernel."""
    for ev in (ev_start, ev_stop):
        if ev is not None and not ev.cuda_event:
            ev.record()          # torch creates the underlying hipEvent_t on first use
    _check(_load().ff_time_next_kernel(ctypes.c_void_p(ev_start.cuda_event if ev_start else None),
                                       ctypes.c_void_p(ev_stop.cuda_event if ev_stop else None)))
