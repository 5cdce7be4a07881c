"""ctypes binding of liblstmloop.so: argument marshalling only.

Every computation happens in the HIP library; this module turns torch
tensors into device pointers and the current torch stream into a hipStream_t.
The function names follow the C ABI of include/lstmloop.h.
If the library has not been built, every call raises; there is no fallback.
"""
from __future__ import annotations

import atexit
import ctypes
import functools
import os
import weakref
from typing import Optional, Sequence

_PKG = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_PKG, "liblstmloop.so")

LL_OK, LL_EINVAL, LL_ENOMEM, LL_EHIP, LL_ESTATE, LL_EUNSUPPORTED = range(6)
LL_F32, LL_BF16 = 0, 1
LL_DEVERR_SEQ_LEN, LL_DEVERR_BARRIER, LL_DEVERR_SLOT, LL_DEVERR_TARGET = 1, 2, 4, 8
LL_LOOPS_GRID, LL_LOOPS_XCD, LL_LOOPS_CHIP = 0, 1, 2
LL_CELL_LSTM, LL_CELL_RNN, LL_CELL_GRU, LL_CELL_LSTM_SKIP, LL_CELL_LSTM_ACT = 0, 1, 2, 3, 4
LL_ACT_EPS = 0.01
LL_ACT_PONDER_MAX = 8
STATUS_NAMES = {0: "LL_OK", 1: "LL_EINVAL", 2: "LL_ENOMEM", 3: "LL_EHIP",
                4: "LL_ESTATE", 5: "LL_EUNSUPPORTED"}

EXPORTED = ("ll_plan_create", "ll_plan_destroy", "ll_plan_stack_bytes",
            "ll_plan_geometry", "lstm_loop_fwd", "lstm_loop_bwd",
            "ll_status_sync", "ll_last_error", "ll_version",
            "ll_plan_set_timing", "ll_plan_set_timing_stages", "ll_plan_read_timing",
            "ll_measure_mfma_peak", "ll_eval_activations", "lstm_loop_fwd_noalloc",
            "ll_delta_plan_create", "ll_delta_plan_destroy", "ll_delta_plan_bytes", "ll_delta_plan_set_ld",
            "delta_loop_fwd", "delta_loop_bwd", "delta_loop_step", "ll_delta_status_sync",
            "ll_logprob_plan_create", "ll_logprob_plan_destroy", "ll_logprob_fwd",
            "ll_logprob_bwd", "ll_logprob_fwd_bwd", "ll_logprob_status_sync",
            "ll_adamw_plan_create", "ll_adamw_plan_destroy", "ll_adamw_step")
STAGES = ("prep", "input_proj", "fwd_loop", "bwd_loop", "bwd_operands", "dw", "dx", "loop_setup",
          "recompute")


class ll_desc(ctypes.Structure):
    _fields_ = [("T_max", ctypes.c_int32), ("B", ctypes.c_int32),
                ("I", ctypes.c_int32), ("H", ctypes.c_int32),
                ("layers", ctypes.c_int32), ("dtype", ctypes.c_int32),
                ("spill", ctypes.c_int32), ("spill_chunk_steps", ctypes.c_int32),
                ("device_stack_budget_bytes", ctypes.c_int64),
                ("recompute", ctypes.c_int32), ("cell", ctypes.c_int32),
                ("ponder_max", ctypes.c_int32), ("reserved", ctypes.c_int32)]


class ll_delta_desc(ctypes.Structure):
    _fields_ = [("T_max", ctypes.c_int32), ("B", ctypes.c_int32), ("Hk", ctypes.c_int32),
                ("Hv", ctypes.c_int32), ("Dk", ctypes.c_int32), ("Dv", ctypes.c_int32),
                ("dtype", ctypes.c_int32), ("inference", ctypes.c_int32),
                ("q_ld", ctypes.c_int64), ("k_ld", ctypes.c_int64), ("v_ld", ctypes.c_int64),
                ("dq_ld", ctypes.c_int64), ("dk_ld", ctypes.c_int64), ("dv_ld", ctypes.c_int64),
                ("scale", ctypes.c_float), ("reserved", ctypes.c_int32)]


class ll_logprob_desc(ctypes.Structure):
    _fields_ = [("N", ctypes.c_int32), ("V", ctypes.c_int32), ("dtype", ctypes.c_int32),
                ("top_k", ctypes.c_int32), ("ld", ctypes.c_int64),
                ("reserved", ctypes.c_int32 * 2)]


class ll_adamw_tensor(ctypes.Structure):
    _fields_ = [("p", ctypes.c_void_p), ("copy", ctypes.c_void_p), ("m", ctypes.c_void_p),
                ("v", ctypes.c_void_p), ("m_scale", ctypes.c_void_p),
                ("v_scale", ctypes.c_void_p), ("n", ctypes.c_int64),
                ("weight_decay", ctypes.c_float), ("reserved", ctypes.c_int32)]


class ll_adamw_desc(ctypes.Structure):
    _fields_ = [("n_tensors", ctypes.c_int32), ("state_bits", ctypes.c_int32),
                ("grad_dtype", ctypes.c_int32), ("reserved", ctypes.c_int32)]


class ll_adamw_hyper(ctypes.Structure):
    _fields_ = [("lr", ctypes.c_double), ("beta1", ctypes.c_double), ("beta2", ctypes.c_double),
                ("eps", ctypes.c_double), ("step", ctypes.c_int64), ("seed", ctypes.c_uint32),
                ("reserved", ctypes.c_int32)]


class LoopError(RuntimeError):
    def __init__(self, status: int, msg: str):
        super().__init__(f"{STATUS_NAMES.get(status, status)}: {msg}")
        self.status = status


_lib = None
# Plans still open: closed by an exit hook that runs while the HIP runtime is
# alive (its own teardown happens later, in the C library's exit handlers).
_live_plans: "weakref.WeakSet" = weakref.WeakSet()


def _close_live_plans() -> None:
    for plan in list(_live_plans):
        try:
            plan.close()
        except Exception:
            pass


atexit.register(_close_live_plans)


def load_library(path: str = LIB_PATH) -> ctypes.CDLL:
    """Load the HIP library (once).  Raises if it is missing."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(path):
        raise RuntimeError(
            f"{path} is missing: build it with `python -m paper_1805_01772_amd.build_lib` "
            "(or __graft_entry__.build()); there is no CPU fallback")
    # torch ships its own HIP runtime (SONAME libamdhip64.so.7).  Loading torch
    # first makes the library bind to that same runtime instead of a second
    # copy, so torch's streams and device pointers are valid here.
    import torch  # noqa: F401
    lib = ctypes.CDLL(path)
    vp, i32, i64 = ctypes.c_void_p, ctypes.c_int32, ctypes.c_int64
    lib.ll_plan_create.argtypes = [ctypes.POINTER(ll_desc), ctypes.c_int, ctypes.POINTER(vp)]
    lib.ll_plan_destroy.argtypes = [vp]
    lib.ll_plan_stack_bytes.argtypes = [vp, ctypes.POINTER(i64), ctypes.POINTER(i64)]
    lib.ll_plan_geometry.argtypes = [vp, ctypes.POINTER(i32), ctypes.POINTER(i32),
                                     ctypes.POINTER(i32), ctypes.POINTER(i32),
                                     ctypes.POINTER(i32), ctypes.POINTER(i32)]
    lib.lstm_loop_fwd.argtypes = [vp, vp, vp, vp, ctypes.POINTER(vp), ctypes.POINTER(vp),
                                  vp, vp, vp, vp, vp, vp, i32]
    lib.lstm_loop_bwd.argtypes = [vp, vp, vp, vp, ctypes.POINTER(vp), vp, vp, vp, vp,
                                  ctypes.POINTER(vp), ctypes.POINTER(vp), vp, vp]
    lib.ll_status_sync.argtypes = [vp, ctypes.POINTER(i32)]
    lib.ll_plan_set_timing.argtypes = [vp, i32]
    lib.ll_plan_set_timing_stages.argtypes = [vp, ctypes.c_uint32]
    lib.ll_plan_read_timing.argtypes = [vp, i32, ctypes.POINTER(ctypes.c_double),
                                        ctypes.POINTER(i64)]
    lib.ll_measure_mfma_peak.argtypes = [ctypes.c_int, i32, i32, ctypes.POINTER(ctypes.c_double)]
    lib.ll_eval_activations.argtypes = [ctypes.c_int32, vp, vp, i64, i32]
    lib.lstm_loop_fwd_noalloc.argtypes = [ctypes.POINTER(ll_desc), vp, vp, vp, ctypes.POINTER(vp),
                                          ctypes.POINTER(vp), vp, vp, vp, vp, vp, vp, vp]
    pvp = ctypes.POINTER(vp)
    lib.ll_delta_plan_create.argtypes = [ctypes.POINTER(ll_delta_desc), ctypes.c_int, pvp]
    lib.ll_delta_plan_destroy.argtypes = [vp]
    lib.ll_delta_plan_bytes.argtypes = [vp, ctypes.POINTER(i64)]
    lib.ll_delta_plan_set_ld.argtypes = [vp, ctypes.POINTER(i64)]
    lib.delta_loop_fwd.argtypes = [vp] * 11 + [i32]
    lib.delta_loop_bwd.argtypes = [vp] * 16
    lib.delta_loop_step.argtypes = [ctypes.POINTER(ll_delta_desc)] + [vp] * 8 + [i32, vp, vp]
    lib.ll_delta_status_sync.argtypes = [vp, ctypes.POINTER(i32)]
    lib.ll_logprob_plan_create.argtypes = [ctypes.POINTER(ll_logprob_desc), ctypes.c_int, pvp]
    lib.ll_logprob_plan_destroy.argtypes = [vp]
    lib.ll_logprob_fwd.argtypes = [vp, vp, i32] + [vp] * 7
    lib.ll_logprob_bwd.argtypes = [vp, vp, i32] + [vp] * 9
    lib.ll_logprob_fwd_bwd.argtypes = [vp, vp, i32] + [vp] * 8
    lib.ll_logprob_status_sync.argtypes = [vp, ctypes.POINTER(i32)]
    lib.ll_adamw_plan_create.argtypes = [ctypes.POINTER(ll_adamw_desc),
                                         ctypes.POINTER(ll_adamw_tensor), ctypes.c_int, pvp]
    lib.ll_adamw_plan_destroy.argtypes = [vp]
    lib.ll_adamw_step.argtypes = [vp, vp, pvp, ctypes.POINTER(ll_adamw_hyper), vp]
    lib.ll_last_error.restype = ctypes.c_char_p
    lib.ll_version.restype = ctypes.c_char_p
    for name in ("ll_plan_create", "ll_plan_destroy", "ll_plan_stack_bytes", "ll_plan_geometry",
                 "lstm_loop_fwd", "lstm_loop_bwd", "ll_status_sync", "ll_plan_set_timing",
                 "ll_plan_set_timing_stages", "ll_plan_read_timing", "ll_measure_mfma_peak",
                 "ll_eval_activations", "lstm_loop_fwd_noalloc", "ll_delta_plan_create",
                 "ll_delta_plan_destroy", "ll_delta_plan_bytes", "ll_delta_plan_set_ld", "delta_loop_fwd",
                 "delta_loop_bwd", "delta_loop_step", "ll_delta_status_sync",
                 "ll_logprob_plan_create", "ll_logprob_plan_destroy", "ll_logprob_fwd",
                 "ll_logprob_bwd", "ll_logprob_fwd_bwd", "ll_logprob_status_sync",
                 "ll_adamw_plan_create", "ll_adamw_plan_destroy", "ll_adamw_step"):
        getattr(lib, name).restype = ctypes.c_int
    _lib = lib
    return lib


def ll_last_error() -> str:
    return load_library().ll_last_error().decode()


def ll_measure_mfma_peak(dtype: str, shape: int = 32, device: int = 0) -> float:
    """Sustained dense matrix-core rate of the device in TFLOP/s
    (dtype "bf16" or "f32"; shape 16: the loops' 16x16 k-step, 32: 32x32)."""
    v = ctypes.c_double()
    _check(load_library().ll_measure_mfma_peak(device, LL_BF16 if dtype == "bf16" else LL_F32, shape,
                                               ctypes.byref(v)))
    return v.value


def ll_eval_activations(x, fn: str):
    """The loop kernels' sigmoid ("sigmoid") or tanh ("tanh") of the float32
    device tensor x (ll_eval_activations); returns a new tensor."""
    import torch
    out = torch.empty_like(x)
    _check(load_library().ll_eval_activations(x.device.index or 0, _ptr(x), _ptr(out), x.numel(),
                                              {"sigmoid": 0, "tanh": 1}[fn]))
    return out


def ll_version() -> str:
    return load_library().ll_version().decode()


def _check(status: int) -> None:
    if status != LL_OK:
        raise LoopError(status, ll_last_error())


def _ptr(t) -> Optional[int]:
    if t is None:
        return None
    if not t.is_cuda:
        raise ValueError("tensors passed to the library must live on the GPU")
    if not t.is_contiguous():
        raise ValueError("tensors passed to the library must be contiguous")
    return t.data_ptr()


def _ptr_array(ts):
    arr = (ctypes.c_void_p * len(ts))()
    for i, t in enumerate(ts):
        arr[i] = _ptr(t)
    return arr


def _stream(stream) -> Optional[int]:
    if stream is None:
        import torch
        stream = torch.cuda.current_stream()
    return stream.cuda_stream


class Plan:
    """Owner of an ll_plan (ll_plan_create / ll_plan_destroy)."""

    def __init__(self, T_max: int, B: int, I: int, H: int, layers: int = 1,
                 dtype: str = "f32", spill: int = 0, spill_chunk_steps: int = 0,
                 device_stack_budget_bytes: int = 0, device: int = 0, recompute: int = 0,
                 cell: int = 0, ponder_max: int = 0):
        lib = load_library()
        self._lib = lib
        self.desc = make_desc(T_max, B, I, H, layers, dtype, spill, spill_chunk_steps,
                              device_stack_budget_bytes, recompute, cell, ponder_max)
        self.dtype = dtype
        self.device = device
        h = ctypes.c_void_p()
        _check(lib.ll_plan_create(ctypes.byref(self.desc), device, ctypes.byref(h)))
        self._h = h
        _live_plans.add(self)

    def close(self) -> None:
        if getattr(self, "_h", None) is not None and self._h.value:
            self._lib.ll_plan_destroy(self._h)
            self._h = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def __enter__(self):
        return self

    def __exit__(self, *exc):
        self.close()

    @property
    def handle(self) -> int:
        return self._h.value

    def stack_bytes(self):
        d, h = ctypes.c_int64(), ctypes.c_int64()
        _check(self._lib.ll_plan_stack_bytes(self._h, ctypes.byref(d), ctypes.byref(h)))
        return d.value, h.value

    def geometry(self):
        n, hj, rg, xl, wf, dwp = (ctypes.c_int32() for _ in range(6))
        _check(self._lib.ll_plan_geometry(self._h, ctypes.byref(n), ctypes.byref(hj),
                                          ctypes.byref(rg), ctypes.byref(xl), ctypes.byref(wf),
                                          ctypes.byref(dwp)))
        form = {LL_LOOPS_GRID: "grid", LL_LOOPS_XCD: "xcd", LL_LOOPS_CHIP: "chip"}[xl.value]
        return dict(workgroups=n.value, units_per_workgroup=hj.value, row_groups=rg.value,
                    loops=form, xcd_local=form == "xcd", wavefront=bool(wf.value),
                    dw_in_place=[bool(dwp.value >> l & 1) for l in range(self.desc.layers)])

    def fwd(self, x, seq_len, W: Sequence, bias: Sequence, h0, c0, y, hT, cT,
            trip_count=None, save_for_backward: bool = True, stream=None) -> None:
        """lstm_loop_fwd (asynchronous on `stream`, default: torch's current)."""
        _check(self._lib.lstm_loop_fwd(
            self._h, _stream(stream), _ptr(x), _ptr(seq_len), _ptr_array(W), _ptr_array(bias),
            _ptr(h0), _ptr(c0), _ptr(y), _ptr(hT), _ptr(cT), _ptr(trip_count),
            1 if save_for_backward else 0))

    def bwd(self, x, seq_len, W: Sequence, dy, dhT, dcT, dx, dW: Sequence, dbias: Sequence,
            dh0, dc0, stream=None) -> None:
        """lstm_loop_bwd (asynchronous on `stream`); x, seq_len and W are the
        tensors the saved forward was given."""
        _check(self._lib.lstm_loop_bwd(
            self._h, _stream(stream), _ptr(x), _ptr(seq_len), _ptr_array(W), _ptr(dy),
            _ptr(dhT), _ptr(dcT), _ptr(dx), _ptr_array(dW), _ptr_array(dbias), _ptr(dh0),
            _ptr(dc0)))

    def set_timing(self, enable) -> None:
        """ll_plan_set_timing: clear the stage accumulators, start/stop recording
        every stage; a collection of stage names records only those
        (ll_plan_set_timing_stages)."""
        if isinstance(enable, (bool, int)):
            _check(self._lib.ll_plan_set_timing(self._h, 1 if enable else 0))
            return
        mask = 0
        for name in enable:
            mask |= 1 << STAGES.index(name)
        _check(self._lib.ll_plan_set_timing_stages(self._h, mask))

    def read_timing(self) -> dict:
        """ll_plan_read_timing for every stage: {name: (total_ms, instances)}."""
        out = {}
        for i, name in enumerate(STAGES):
            ms, n = ctypes.c_double(), ctypes.c_int64()
            _check(self._lib.ll_plan_read_timing(self._h, i, ctypes.byref(ms), ctypes.byref(n)))
            out[name] = (ms.value, n.value)
        return out

    def status_sync(self) -> int:
        """ll_status_sync: wait, then return (and clear) the device error word."""
        e = ctypes.c_int32()
        _check(self._lib.ll_status_sync(self._h, ctypes.byref(e)))
        return e.value


def lstm_loop_fwd(plan: Plan, *args, **kw):
    return plan.fwd(*args, **kw)


def lstm_loop_bwd(plan: Plan, *args, **kw):
    return plan.bwd(*args, **kw)


NOALLOC_SCRATCH_BYTES = 128 << 20   # LL_NOALLOC_SCRATCH_BYTES


def make_desc(T_max: int, B: int, I: int, H: int, layers: int = 1, dtype: str = "f32",
              spill: int = 0, spill_chunk_steps: int = 0, device_stack_budget_bytes: int = 0,
              recompute: int = 0, cell: int = 0, ponder_max: int = 0) -> ll_desc:
    return ll_desc(T_max, B, I, H, layers,
                   LL_BF16 if dtype == "bf16" else LL_F32 if dtype == "f32" else int(dtype),
                   spill, spill_chunk_steps, device_stack_budget_bytes, recompute, cell, ponder_max, 0)


def lstm_loop_fwd_noalloc(desc: ll_desc, x, seq_len, W: Sequence, bias: Sequence, h0, c0, y, hT,
                          cT, trip_count=None, device_error=None, stream=None) -> None:
    """lstm_loop_fwd_noalloc: the inference forward without a plan, every
    buffer carved from the library's scratch array (asynchronous on `stream`)."""
    _check(load_library().lstm_loop_fwd_noalloc(
        ctypes.byref(desc), _stream(stream), _ptr(x), _ptr(seq_len), _ptr_array(W), _ptr_array(bias),
        _ptr(h0), _ptr(c0), _ptr(y), _ptr(hT), _ptr(cT), _ptr(trip_count), _ptr(device_error)))


def ll_plan_create(*args, **kw) -> Plan:
    return Plan(*args, **kw)


def ll_plan_destroy(plan: Plan) -> None:
    plan.close()


def ll_status_sync(plan: Plan) -> int:
    return plan.status_sync()


def ll_plan_stack_bytes(plan: Plan):
    return plan.stack_bytes()


# --------------------------------------------------------------------------
# the operators beside the loops
# --------------------------------------------------------------------------
@functools.lru_cache(maxsize=None)
def _dtype(name: str):
    """torch's type of a dtype or element type name."""
    import torch
    return getattr(torch, {"f32": "float32", "bf16": "bfloat16"}.get(name, name))


def _refuse(t, name: str, shape, dtype):
    if tuple(t.shape) != tuple(shape) or t.dtype is not dtype:
        raise ValueError(f"{name}: {tuple(shape)} {dtype} is wanted, got {tuple(t.shape)} {t.dtype}")
    if not t.is_cuda:
        raise ValueError("tensors passed to the library must live on the GPU")


def _want(t, name: str, shape: tuple, dtype, optional: bool = False):
    """Address of a contiguous tensor whose shape and type are what the call says."""
    if t is None and optional:
        return None
    if t.shape != shape or t.dtype is not dtype or not t.is_cuda:
        _refuse(t, name, shape, dtype)
    if not t.is_contiguous():
        raise ValueError("tensors passed to the library must be contiguous")
    return t.data_ptr()


def _tokens(t, name: str, shape: tuple, ld: int, dtype):
    """Address of a token array ([T, B, heads, size] or [B, heads, size]) whose
    tokens are ld elements apart."""
    if t.shape != shape or t.dtype is not dtype or not t.is_cuda:
        _refuse(t, name, shape, dtype)
    if ld < shape[-2] * shape[-1]:
        raise ValueError(f"{name}: tokens {ld} elements apart overlap ({shape[-2]} heads of {shape[-1]}); "
                         "an expanded tensor has to be copied")
    want = (ld, shape[-1], 1) if len(shape) == 3 else (shape[1] * ld, ld, shape[-1], 1)
    if t.stride() != want and any(s != w and n > 1 for s, w, n in zip(t.stride(), want, shape)):
        raise ValueError(f"{name}: strides {tuple(t.stride())}, {want} are wanted "
                         f"(tokens {ld} elements apart)")
    return t.data_ptr()


class _OpPlan:
    """Owner of an operator's plan handle."""

    _destroy = ""

    def _create(self, make, desc, *args):
        lib = load_library()
        h = ctypes.c_void_p()
        _check(getattr(lib, make)(ctypes.byref(desc), *args, ctypes.byref(h)))
        self._lib, self._h = lib, h
        _live_plans.add(self)

    def close(self) -> None:
        if getattr(self, "_h", None) is not None and self._h.value:
            getattr(self._lib, self._destroy)(self._h)
            self._h = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def __enter__(self):
        return self

    def __exit__(self, *exc):
        self.close()

    def _status(self, fn) -> int:
        e = ctypes.c_int32()
        _check(getattr(self._lib, fn)(self._h, ctypes.byref(e)))
        return e.value


def make_delta_desc(T_max: int, B: int, Hk: int, Hv: int, Dk: int, Dv: int, dtype: str = "f32",
                    inference: bool = False, q_ld: int = 0, k_ld: int = 0, v_ld: int = 0,
                    dq_ld: int = 0, dk_ld: int = 0, dv_ld: int = 0,
                    scale: float = 0.0) -> ll_delta_desc:
    return ll_delta_desc(T_max, B, Hk, Hv, Dk, Dv,
                         LL_BF16 if dtype == "bf16" else LL_F32 if dtype == "f32" else int(dtype),
                         1 if inference else 0, q_ld, k_ld, v_ld, dq_ld, dk_ld, dv_ld, scale, 0)


class DeltaPlan(_OpPlan):
    """The gated delta rule over [T_max, B] tokens (ll_delta_plan)."""

    _destroy = "ll_delta_plan_destroy"

    def __init__(self, T_max: int, B: int, Hk: int, Hv: int, Dk: int, Dv: int, dtype: str = "f32",
                 inference: bool = False, q_ld: int = 0, k_ld: int = 0, v_ld: int = 0,
                 dq_ld: int = 0, dk_ld: int = 0, dv_ld: int = 0, scale: float = 0.0,
                 device: int = 0):
        self.desc = d = make_delta_desc(T_max, B, Hk, Hv, Dk, Dv, dtype, inference, q_ld, k_ld,
                                        v_ld, dq_ld, dk_ld, dv_ld, scale)
        self.dtype = dtype
        self._t = _dtype(dtype)
        self._create("ll_delta_plan_create", d, device)
        qk, v = Hk * Dk, Hv * Dv
        self._note(dict(q=q_ld or qk, k=k_ld or qk, v=v_ld or v, dq=dq_ld or qk, dk=dk_ld or qk,
                        dv=dv_ld or v))
        self._qk, self._v = (T_max, B, Hk, Dk), (T_max, B, Hv, Dv)
        self._gate, self._state = (T_max, B, Hv), (B, Hv, Dk, Dv)

    def _distances(self, **tokens):
        """The plan's distances as these tensors have them.  The tokens of a single
        row are stride(0) apart; stride(1), of a dimension of one, says nothing (a
        view may hold any number there)."""
        T, B = self._qk[:2]
        if B != 1 or T == 1:
            return self._ld
        new = {n: t.stride(0) for n, t in tokens.items()
               if t.dim() == 4 and t.stride(0) > 0 and t.stride(0) != self._ld[n]}
        return {**self._ld, **new} if new else self._ld

    def _set_distances(self, ld):
        names = ("q", "k", "v", "dq", "dk", "dv")
        _check(self._lib.ll_delta_plan_set_ld(self._h, (ctypes.c_int64 * 6)(*(ld[n] for n in names))))
        self._note(ld)

    def _note(self, ld):
        self._ld = ld
        for n in ld:
            setattr(self.desc, n + "_ld", ld[n])

    def _call(self, ld, fn, *args):
        """One call with the tokens ld apart; a refused one leaves the plan as it was."""
        old = self._ld
        if ld is not old:
            self._set_distances(ld)
        try:
            _check(fn(self._h, *args))
        except LoopError:
            if ld is not old:
                self._set_distances(old)
            raise

    def _inputs(self, q, k, v, g, beta, seq_len, ld):
        t, f = self._t, _dtype("float32")
        return (_tokens(q, "q", self._qk, ld["q"], t), _tokens(k, "k", self._qk, ld["k"], t),
                _tokens(v, "v", self._v, ld["v"], t),
                _want(g, "g", self._gate, f), _want(beta, "beta", self._gate, f),
                _want(seq_len, "seq_len", self._qk[1:2], _dtype("int32"), optional=True))

    def fwd(self, q, k, v, g, beta, seq_len, S0, y, ST, save_for_backward: bool = True,
            stream=None) -> None:
        """delta_loop_fwd (asynchronous on `stream`, default: torch's current)."""
        f = _dtype("float32")
        ld = self._distances(q=q, k=k, v=v)
        self._call(ld, self._lib.delta_loop_fwd,
                   _stream(stream), *self._inputs(q, k, v, g, beta, seq_len, ld),
                   _want(S0, "S0", self._state, f, optional=True), _want(y, "y", self._v, self._t),
                   _want(ST, "ST", self._state, f, optional=True), 1 if save_for_backward else 0)

    def bwd(self, q, k, v, g, beta, seq_len, dy, dST, dq, dk, dv, dg, dbeta, dS0=None,
            stream=None) -> None:
        """delta_loop_bwd (asynchronous on `stream`); q .. seq_len are the tensors the
        saved forward was given.  (q, k or v with tokens at other distances than
        that one's: LL_ESTATE, no forward of such tensors is saved.)"""
        t, f = self._t, _dtype("float32")
        ld = self._distances(q=q, k=k, v=v, dq=dq, dk=dk, dv=dv)
        args = (*self._inputs(q, k, v, g, beta, seq_len, ld),
                _want(dy, "dy", self._v, t), _want(dST, "dST", self._state, f, optional=True),
                _tokens(dq, "dq", self._qk, ld["dq"], t), _tokens(dk, "dk", self._qk, ld["dk"], t),
                _tokens(dv, "dv", self._v, ld["dv"], t),
                _want(dg, "dg", self._gate, f), _want(dbeta, "dbeta", self._gate, f),
                _want(dS0, "dS0", self._state, f, optional=True))
        self._call(ld, self._lib.delta_loop_bwd, _stream(stream), *args)

    def bytes(self) -> int:
        """ll_delta_plan_bytes: device memory that the plan holds."""
        n = ctypes.c_int64()
        _check(self._lib.ll_delta_plan_bytes(self._h, ctypes.byref(n)))
        return n.value

    def status_sync(self) -> int:
        """ll_delta_status_sync: wait, then return (and clear) the device error word."""
        return self._status("ll_delta_status_sync")


def delta_loop_fwd(plan: DeltaPlan, *args, **kw):
    return plan.fwd(*args, **kw)


def delta_loop_bwd(plan: DeltaPlan, *args, **kw):
    return plan.bwd(*args, **kw)


def delta_loop_step(q, k, v, g, beta, S, y, slots=None, scale: float = 0.0, device_error=None,
                    stream=None) -> None:
    """delta_loop_step: one token for the B rows of q [B, Hk, Dk], k, v [B, Hv, Dv]
    (rows may be slices of a projection's), states S [n_slots, Hv, Dk, Dv]
    updated in place (asynchronous on `stream`)."""
    (B, Hk, Dk), (_, Hv, Dv) = q.shape, v.shape
    t, f = q.dtype, _dtype("float32")
    lq, lk, lv = (q.stride(0), k.stride(0), v.stride(0)) if B > 1 else (Hk * Dk, Hk * Dk, Hv * Dv)
    if t is f:
        name = "f32"
    elif t is _dtype("bfloat16"):
        name = "bf16"
    else:
        raise ValueError(f"q: float32 or bfloat16 is wanted, got {t}")
    _check(load_library().delta_loop_step(
        _step_desc(B, Hk, Hv, Dk, Dv, name, lq, lk, lv, scale), _stream(stream),
        _tokens(q, "q", (B, Hk, Dk), lq, t), _tokens(k, "k", (B, Hk, Dk), lk, t),
        _tokens(v, "v", (B, Hv, Dv), lv, t), _want(g, "g", (B, Hv), f),
        _want(beta, "beta", (B, Hv), f), _want(S, "S", (S.shape[0], Hv, Dk, Dv), f),
        _want(slots, "slots", (B,), _dtype("int32"), optional=True), S.shape[0],
        _want(y, "y", (B, Hv, Dv), t),
        _want(device_error, "device_error", (1,), _dtype("int32"), optional=True)))


@functools.lru_cache(maxsize=256)
def _step_desc(B, Hk, Hv, Dk, Dv, dtype, q_ld, k_ld, v_ld, scale):
    return ctypes.byref(make_delta_desc(1, B, Hk, Hv, Dk, Dv, dtype, True, q_ld, k_ld, v_ld,
                                        scale=scale))


class LogprobPlan(_OpPlan):
    """Log probabilities of given tokens, entropy, alternatives (ll_logprob_plan)
    of up to N rows of V logits, rows ld elements apart (0: V)."""

    _destroy = "ll_logprob_plan_destroy"

    def __init__(self, N: int, V: int, dtype: str = "f32", top_k: int = 0, ld: int = 0,
                 device: int = 0):
        d = ll_logprob_desc(N, V, LL_BF16 if dtype == "bf16" else LL_F32, top_k, ld)
        if dtype not in ("f32", "bf16"):
            raise ValueError(f"dtype {dtype!r} is neither 'f32' nor 'bf16'")
        self.desc, self.dtype, self.top_k, self.V = d, dtype, top_k, V
        self._t = _dtype(dtype)
        self.ld = ld or V
        self._create("ll_logprob_plan_create", d, device)

    def _rows(self, x, name: str, n: int):
        sh, st = x.shape, x.stride()
        if (sh != (n, self.V) or x.dtype is not self._t or (self.V > 1 and st[1] != 1)
                or (n > 1 and st[0] != self.ld)):
            raise ValueError(f"{name}: [rows, {self.V}] {self._t} with rows {self.ld} apart is "
                             f"wanted, got {tuple(sh)} {x.dtype} strides {tuple(st)}")
        if not x.is_cuda:
            raise ValueError("tensors passed to the library must live on the GPU")
        return x.data_ptr()

    def fwd(self, logits, targets, logp, entropy=None, lse=None, top_ids=None, top_logp=None,
            stream=None) -> None:
        """ll_logprob_fwd (asynchronous on `stream`)."""
        n, f = logits.shape[0], _dtype("float32")
        _check(self._lib.ll_logprob_fwd(
            self._h, _stream(stream), n, self._rows(logits, "logits", n),
            _want(targets, "targets", (n,), _dtype("int32"), optional=True),
            _want(logp, "logp", (n,), f, optional=True),
            _want(entropy, "entropy", (n,), f, optional=True),
            _want(lse, "lse", (n,), f, optional=True),
            _want(top_ids, "top_ids", (n, self.top_k), _dtype("int32"), optional=True),
            _want(top_logp, "top_logp", (n, self.top_k), f, optional=True)))

    def bwd(self, logits, targets, lse, entropy, top_ids, dlogp, dentropy, dtop, dlogits,
            stream=None) -> None:
        """ll_logprob_bwd (asynchronous on `stream`); dlogits may be logits."""
        n, f = logits.shape[0], _dtype("float32")
        _check(self._lib.ll_logprob_bwd(
            self._h, _stream(stream), n, self._rows(logits, "logits", n),
            _want(targets, "targets", (n,), _dtype("int32"), optional=True),
            _want(lse, "lse", (n,), f),
            _want(entropy, "entropy", (n,), f, optional=True),
            _want(top_ids, "top_ids", (n, self.top_k), _dtype("int32"), optional=True),
            _want(dlogp, "dlogp", (n,), f, optional=True),
            _want(dentropy, "dentropy", (n,), f, optional=True),
            _want(dtop, "dtop", (n, self.top_k), f, optional=True),
            self._rows(dlogits, "dlogits", n)))

    def fwd_bwd(self, logits, targets, dlogp, dentropy, logp, entropy, lse, dlogits,
                stream=None) -> None:
        """ll_logprob_fwd_bwd (asynchronous on `stream`); dlogits may be logits."""
        n, f = logits.shape[0], _dtype("float32")
        _check(self._lib.ll_logprob_fwd_bwd(
            self._h, _stream(stream), n, self._rows(logits, "logits", n),
            _want(targets, "targets", (n,), _dtype("int32"), optional=True),
            _want(dlogp, "dlogp", (n,), f, optional=True),
            _want(dentropy, "dentropy", (n,), f, optional=True),
            _want(logp, "logp", (n,), f, optional=True),
            _want(entropy, "entropy", (n,), f, optional=True),
            _want(lse, "lse", (n,), f, optional=True),
            self._rows(dlogits, "dlogits", n)))

    def status_sync(self) -> int:
        """ll_logprob_status_sync: wait, then return (and clear) the device error word."""
        return self._status("ll_logprob_status_sync")


ADAMW_ROW = 256   # LL_ADAMW_ROW


class AdamWPlan(_OpPlan):
    """AdamW over many tensors (ll_adamw_plan).  params: float32 tensors; m and
    v: float32, or int8 and uint8 with m_scale and v_scale (ceil(n / ADAMW_ROW)
    floats a tensor); copies: bfloat16 tensors or None, a list or None;
    weight_decay: one number or one a tensor.  The plan keeps the tensors."""

    _destroy = "ll_adamw_plan_destroy"

    def __init__(self, params: Sequence, m: Sequence, v: Sequence, m_scale=None, v_scale=None,
                 copies=None, weight_decay=0.0, grad_dtype: str = "f32", device: int = 0):
        n = len(params)
        q8 = m_scale is not None
        if grad_dtype not in ("f32", "bf16"):
            raise ValueError(f"grad_dtype {grad_dtype!r} is neither 'f32' nor 'bf16'")
        if q8 != (v_scale is not None):
            raise ValueError("m_scale and v_scale go together")
        wd = list(weight_decay) if hasattr(weight_decay, "__len__") else [weight_decay] * n
        if n == 0:
            raise ValueError("no tensors")
        lists = [m, v, wd] + [x for x in (m_scale, v_scale, copies) if x is not None]
        if any(len(x) != n for x in lists):
            raise ValueError(f"{n} params, but lists of {[len(x) for x in lists]} for them")
        recs = (ll_adamw_tensor * n)()
        f = _dtype("float32")
        mt, vt = (_dtype("int8"), _dtype("uint8")) if q8 else (f, f)
        for i, p in enumerate(params):
            shape, rows = tuple(p.shape), (-(-p.numel() // ADAMW_ROW),)
            recs[i] = ll_adamw_tensor(
                _want(p, f"params[{i}]", shape, f),
                _want(copies[i] if copies is not None else None, f"copies[{i}]", shape, _dtype("bfloat16"),
                      optional=True),
                _want(m[i], f"m[{i}]", shape, mt), _want(v[i], f"v[{i}]", shape, vt),
                _want(m_scale[i], f"m_scale[{i}]", rows, f) if q8 else None,
                _want(v_scale[i], f"v_scale[{i}]", rows, f) if q8 else None,
                p.numel(), wd[i], 0)
        self._keep = (list(params), list(m), list(v), m_scale, v_scale, copies)
        self._grad_type = _dtype(grad_dtype)
        self._sizes = [p.numel() for p in params]
        self._ptrs = (ctypes.c_void_p * n)()
        desc = ll_adamw_desc(n, 8 if q8 else 32, LL_BF16 if grad_dtype == "bf16" else LL_F32, 0)
        self._create("ll_adamw_plan_create", desc, recs, device)

    def step(self, grads: Sequence, lr: float, beta1: float = 0.9, beta2: float = 0.999,
             eps: float = 1e-8, step: int = 1, seed: int = 0, grad_scale=None, stream=None) -> None:
        """ll_adamw_step (asynchronous on `stream`): grads has a tensor, or None,
        for each parameter; grad_scale a float32 tensor of one value, or None.
        Captured into a graph it repeats this lr, step and seed: call it anew for
        every step instead."""
        if len(grads) != len(self._sizes):
            raise ValueError(f"{len(self._sizes)} tensors, but {len(grads)} gradients")
        ptrs, dtype = self._ptrs, self._grad_type
        for i, (g, n) in enumerate(zip(grads, self._sizes)):
            if g is None:
                ptrs[i] = None
                continue
            if g.numel() != n or g.dtype is not dtype or not g.is_cuda or not g.is_contiguous():
                raise ValueError(f"grads[{i}]: {n} contiguous elements of {dtype} on the GPU are "
                                 f"wanted, got {tuple(g.shape)} {g.dtype}")
            ptrs[i] = g.data_ptr()
        hyper = ll_adamw_hyper(lr, beta1, beta2, eps, step, seed & 0xFFFFFFFF, 0)
        _check(self._lib.ll_adamw_step(
            self._h, _stream(stream), self._ptrs, ctypes.byref(hyper),
            _want(grad_scale, "grad_scale", (1,), _dtype("float32"), optional=True)))
