"""ctypes binding of libswapmoe.so: argument marshalling only.

Every step of the layer runs inside the library's CUDA kernels; this module turns
torch tensors / numpy arrays into the plain pointers and sizes of the C ABI
(include/swapmoe.h) and raises on a non-zero status.  There is no fallback: if
the library cannot be loaded the import of :func:`lib` raises.
"""
from __future__ import annotations

import ctypes
import os
from typing import Optional, Sequence

import numpy as np

from . import build as _build

F32, BF16 = 0, 1
N_STAGES = 6
# stage 1 has had no kernel of its own since the scan moved into the permute kernel: its slot measures an empty interval
STAGE_NAMES = ("router_gate", "(scan: no kernel of its own)", "scan_permute_gather", "gemm1_act", "gemm2", "combine")
ACT_RELU, ACT_SWIGLU = 0, 1

TAPS = {
    "logits": (0, np.float32), "uidx": (1, np.int32), "ugate": (2, np.float32),
    "midx": (3, np.int32), "mgate": (4, np.float32), "slot": (5, np.int32),
    "count": (6, np.int32), "offset": (7, np.int32), "perm": (8, np.int32),
    "inv": (9, np.int32), "xnorm": (10, np.float32),
    "h": (11, None), "y": (12, np.float32),       # h comes in the layer's dtype (bf16 as uint16 bit patterns)
    "token_tiles": (13, np.int32),
}

EXPORTS = [
    "swapmoe_create", "swapmoe_destroy", "swapmoe_set_router", "swapmoe_set_resident",
    "swapmoe_forward", "swapmoe_forward_timed", "swapmoe_debug_rerun_gemm", "swapmoe_forward_from_logits", "swapmoe_forward_host",
    "swapmoe_forward_host_async", "swapmoe_host_wait",
    "swapmoe_read_importance", "swapmoe_read_importance_kind", "swapmoe_topk_importance", "swapmoe_load_slot_async",
    "swapmoe_debug_copy", "swapmoe_device_status", "swapmoe_launch_count",
    "swapmoe_workspace_bytes", "swapmoe_set_gemm_path", "swapmoe_status_string",
    "swapmoe_route_static", "swapmoe_selftest_bounded_wait", "swapmoe_read_touched_slots",
    "swapmoe_read_scores_async", "swapmoe_read_decode_prefetch",
    "swapmoe_rms_norm", "swapmoe_route",
    "swapmoe_adapters_create", "swapmoe_adapters_destroy", "swapmoe_adapters_set_weights", "swapmoe_adapters_forward",
    "swapmoe_adapters_check", "swapmoe_set_gate", "swapmoe_set_norm", "swapmoe_forward_block",
]


class SwapMoEError(RuntimeError):
    def __init__(self, status: int, where: str):
        self.status = int(status)
        super().__init__("%s: %s (%d)" % (where, status_string(status), status))


class Config(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int32) for n in
                ("E", "d_model", "d_ff", "top_k", "K", "dtype", "act", "renorm_topk",
                 "max_tokens", "spare_slots")]


class RmsNormArgs(ctypes.Structure):
    _fields_ = [(n, ctypes.c_void_p) for n in ("x", "residual", "weight", "residual_out", "out", "out8", "scales")] + \
               [(n, ctypes.c_int64) for n in ("x_stride", "residual_stride", "residual_out_stride", "out_stride", "out8_stride",
                                              "scales_stride")] + \
               [(n, ctypes.c_int32) for n in ("n_rows", "d", "dtype", "residual_dtype", "group")] + [("eps", ctypes.c_float)]


class AdaptersConfig(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int32) for n in ("n_adapters", "d_in", "d_out", "rank", "dtype", "max_tokens")]


SCORES = {"softmax": 0, "sigmoid": 1}


class Gate(ctypes.Structure):
    """How logits become experts and weights: softmax or sigmoid scores, groups of experts, renormalised weights.

    The ``topk_groups`` of ``n_groups`` groups with the largest sum of their ``group_top`` (1 or 2) best choices are
    kept, the best choices in them win; weights are scores, with ``renorm`` divided by their sum, times ``scale``.
    """
    _fields_ = [(n, ctypes.c_int32) for n in ("score", "n_groups", "topk_groups", "group_top", "renorm")] + \
               [("scale", ctypes.c_float)]

    def __init__(self, score: str = "softmax", n_groups: int = 1, topk_groups: int = 1, group_top: int = 1, renorm: bool = False,
                 scale: float = 1.0):
        if score not in SCORES:
            raise SwapMoEError(-1, "Gate: score %r, one of %s expected" % (score, sorted(SCORES)))
        super().__init__(SCORES[score], n_groups, topk_groups, group_top, int(bool(renorm)), scale)


_lib = None


def lib() -> ctypes.CDLL:
    """Loads (building if needed) the CUDA library; raises if that fails."""
    global _lib
    if _lib is None:
        path = os.environ.get("SWAPMOE_LIB")      # explicit library file, e.g. an instrumented build
        if not path:
            path = _build.LIB if os.path.exists(_build.LIB) and os.environ.get("SWAPMOE_NO_REBUILD") \
                else _build.build()
        L = ctypes.CDLL(path)
        vp, i32, i64 = ctypes.c_void_p, ctypes.c_int32, ctypes.c_int64
        L.swapmoe_create.argtypes = [ctypes.POINTER(vp), ctypes.POINTER(Config)]
        L.swapmoe_destroy.argtypes = [vp]
        L.swapmoe_set_router.argtypes = [vp, vp, vp, vp]
        L.swapmoe_set_resident.argtypes = [vp, vp, vp, vp, vp, vp]
        L.swapmoe_forward.argtypes = [vp, vp, vp, i32, vp]
        L.swapmoe_forward_timed.argtypes = [vp, vp, vp, i32, vp, ctypes.POINTER(vp)]
        L.swapmoe_debug_rerun_gemm.argtypes = [vp, vp, i32, vp]
        L.swapmoe_forward_from_logits.argtypes = [vp, vp, vp, vp, i32, vp]
        L.swapmoe_forward_host.argtypes = [vp, vp, vp, i32, vp]
        L.swapmoe_forward_host_async.argtypes = [vp, vp, vp, i32, vp]
        L.swapmoe_host_wait.argtypes = [vp]
        L.swapmoe_read_importance.argtypes = [vp, vp, i32, vp]
        L.swapmoe_read_importance_kind.argtypes = [vp, i32, vp, i32, vp]
        L.swapmoe_topk_importance.argtypes = [vp, i32, i32, vp]
        L.swapmoe_load_slot_async.argtypes = [vp, i32, vp, vp, vp, vp, vp]
        L.swapmoe_debug_copy.argtypes = [vp, i32, vp, ctypes.c_size_t, vp]
        L.swapmoe_device_status.argtypes = [vp, vp, vp]
        L.swapmoe_launch_count.argtypes = [vp]
        L.swapmoe_launch_count.restype = i64
        L.swapmoe_workspace_bytes.argtypes = [vp]
        L.swapmoe_workspace_bytes.restype = i64
        L.swapmoe_set_gemm_path.argtypes = [vp, i32]
        L.swapmoe_route_static.argtypes = [vp] * 4 + [i32] * 7 + [vp] * 11
        L.swapmoe_selftest_bounded_wait.argtypes = [vp, i32, vp]
        L.swapmoe_read_touched_slots.argtypes = [vp, vp, i32, vp]
        L.swapmoe_read_scores_async.argtypes = [vp, i32, vp, i32, vp]
        L.swapmoe_read_decode_prefetch.argtypes = [vp, vp, vp, i32, vp]
        L.swapmoe_route.argtypes = [ctypes.POINTER(Gate), vp, i64, vp, vp, i32, i32, i32, vp, vp, vp, vp]
        L.swapmoe_adapters_create.argtypes = [ctypes.POINTER(vp), ctypes.POINTER(AdaptersConfig)]
        L.swapmoe_adapters_destroy.argtypes = [vp]
        L.swapmoe_adapters_set_weights.argtypes = [vp, vp, vp, vp]
        L.swapmoe_adapters_forward.argtypes = [vp, vp, i64, vp, vp, vp, i64, vp, i64, i32, vp]
        L.swapmoe_adapters_check.argtypes = [vp, i32, i32, i32, i32]
        L.swapmoe_set_gate.argtypes = [vp, ctypes.POINTER(Gate), vp]
        L.swapmoe_set_norm.argtypes = [vp, vp, ctypes.c_float]
        L.swapmoe_forward_block.argtypes = [vp, vp, vp, vp, i32, vp, vp, vp]
        L.swapmoe_rms_norm.argtypes = [ctypes.POINTER(RmsNormArgs), vp]
        L.swapmoe_status_string.argtypes = [i32]
        L.swapmoe_status_string.restype = ctypes.c_char_p
        for n in EXPORTS:
            if n not in ("swapmoe_launch_count", "swapmoe_workspace_bytes", "swapmoe_status_string"):
                getattr(L, n).restype = i32
        _lib = L
    return _lib


def status_string(status: int) -> str:
    return lib().swapmoe_status_string(int(status)).decode()


def _check(status: int, where: str) -> None:
    if status != 0:
        raise SwapMoEError(status, where)


def _np_ptr(a: np.ndarray):
    return a.ctypes.data_as(ctypes.c_void_p)


def _stream_ptr(stream) -> Optional[int]:
    if stream is None:
        import torch
        return torch.cuda.current_stream().cuda_stream
    if isinstance(stream, int):
        return stream
    return stream.cuda_stream


def topk_importance(imp: np.ndarray, K: int) -> np.ndarray:
    imp = np.ascontiguousarray(imp, dtype=np.float32)
    out = np.empty(int(K), dtype=np.int32)
    _check(lib().swapmoe_topk_importance(_np_ptr(imp), imp.size, int(K), _np_ptr(out)),
           "swapmoe_topk_importance")
    return out


ROUTE_STATIC_MAX_TOKENS = 8192


def route_static(x, Wr, expert_to_slot, enorm, top_k: int, K: int, dtype: int, renorm_topk: int,
                 logits, uidx, ugate, midx, mgate, slot, xnorm, count, offset, imp, stream=None) -> None:
    """Router stage through the entry point that allocates nothing.

    For callers that may not allocate device memory (all tensors, outputs included,
    are the caller's; the library's scratch is a fixed array inside the library).
    Every argument is a CUDA torch tensor; ``imp`` is accumulated in place.
    """
    T, d = int(x.shape[0]), int(x.shape[1])
    E = int(Wr.shape[0])
    _check(lib().swapmoe_route_static(
        x.data_ptr(), Wr.data_ptr(), expert_to_slot.data_ptr(), enorm.data_ptr(), T, d, E, int(top_k),
        int(K), int(dtype), int(renorm_topk), logits.data_ptr(), uidx.data_ptr(), ugate.data_ptr(),
        midx.data_ptr(), mgate.data_ptr(), slot.data_ptr(), xnorm.data_ptr(), count.data_ptr(),
        offset.data_ptr(), imp.data_ptr(), _stream_ptr(stream)), "swapmoe_route_static")


# ------------------------------------------------------------------ operators around the experts
def _invalid(where: str, what: str) -> SwapMoEError:
    return SwapMoEError(-1, "%s: %s" % (where, what))


def _vector(t, n: int, dtype, device, where: str, name: str) -> int:
    if t.dtype != dtype or t.device != device or t.numel() != n or not t.is_contiguous():
        raise _invalid(where, "%s: %d contiguous values of %s on %s expected, got %s of %s on %s" % (
            name, n, dtype, device, tuple(t.shape), t.dtype, t.device))
    return t.data_ptr()


def _fail(status: int, where: str, text) -> None:
    raise SwapMoEError(status, where) if text is None else SwapMoEError(status, "%s: %s" % (where, text))


def _device_functions():
    """torch's current device, set device and current stream of a device as an address; the bare ones (a tenth of a us
    each, a us through torch.cuda) where torch has them."""
    import torch
    names = ("_cuda_getDevice", "_cuda_setDevice", "_cuda_getCurrentRawStream")
    if all(hasattr(torch._C, n) for n in names):
        return tuple(getattr(torch._C, n) for n in names)
    return torch.cuda.current_device, torch.cuda.set_device, lambda device: torch.cuda.current_stream(device).cuda_stream


_marshal = None


def marshal():
    """The extension that checks and passes the arguments of the calls below (csrc/marshal.c; built if needed)."""
    global _marshal
    if _marshal is None:
        import importlib.util
        import torch
        path = _build.MARSHAL if os.path.exists(_build.MARSHAL) and os.environ.get("SWAPMOE_NO_REBUILD") \
            else _build.build_marshal()
        spec = importlib.util.spec_from_file_location("paper_2308_15030_b200._marshal", path)
        m = importlib.util.module_from_spec(spec)
        spec.loader.exec_module(m)
        L = lib()
        m.init(_fail, tuple(ctypes.cast(f, ctypes.c_void_p).value for f in
                            (L.swapmoe_rms_norm, L.swapmoe_route, L.swapmoe_adapters_forward)),
               (torch.float32, torch.bfloat16, torch.float8_e4m3fn, torch.int32),
               _device_functions())
        _marshal = m
    return _marshal


def rms_norm(x, weight, eps: float, out=None, residual=None, residual_out=None, out8=None, scales=None, group: int = 0,
             stream=None) -> None:
    """Root-mean-square norm of the rows of ``x`` [T, d], float32 or bfloat16, with the residual's addition.

    h = x + residual; residual_out = h; y = h * weight / sqrt(mean(h^2) + eps); out = y; and in 8 bits
    out8 (torch.float8_e4m3fn) = y / scales with scales = max |y| / 448 per row (group = 0, scales [T, 1] or [T]) or per
    ``group`` columns (32, 64, 128 or 256; scales [T, ceil(d / group)]).  ``residual`` may be float32 beside bfloat16
    rows.  Rows may be strided; residual_out may be residual or x, out may be x.
    """
    (_marshal or marshal()).rms_norm(x, weight, eps, out, residual, residual_out, out8, scales, group, stream)


def route(gate: Gate, logits, experts, weights, bias=None, expert_to_slot=None, slots=None, stream=None) -> None:
    """Routes the rows of ``logits`` [T, E] (float32, rows may be strided) by ``gate``.

    ``experts`` [T, top_k] int32 and ``weights`` [T, top_k] float32 receive the choice, best first.  ``bias`` [E] float32 is
    added to the scores for the choice only.  With ``expert_to_slot`` [E] int32 (-1 = not resident) only resident experts are
    chosen and ``slots`` [T, top_k] int32 receives their entries.
    """
    (_marshal or marshal()).route(gate, logits, experts, weights, bias, expert_to_slot, slots, stream)


class AdapterBank:
    """Low-rank adapters of many requests beside a projection that all of them share (thin handle).

    out[t] = y[t] + scale[a] * B[a] (A[a] x[t]) with a = ids[t]; a negative id means no adapter.
    """

    def __init__(self, n_adapters: int, d_in: int, d_out: int, rank: int, dtype: int, max_tokens: int = 1):
        self.cfg = AdaptersConfig(n_adapters, d_in, d_out, rank, dtype, max_tokens)
        self._h = ctypes.c_void_p()
        _check(lib().swapmoe_adapters_create(ctypes.byref(self._h), ctypes.byref(self.cfg)), "swapmoe_adapters_create")
        import torch
        self._dtype = torch.bfloat16 if dtype == BF16 else torch.float32
        self._device = torch.device("cuda", torch.cuda.current_device())
        self._keep = None

    def close(self) -> None:
        if self._h:
            lib().swapmoe_adapters_destroy(self._h)
            self._h = ctypes.c_void_p()

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def set_weights(self, A, B, scale=None) -> None:
        """A [n_adapters, rank, d_in], B [n_adapters, d_out, rank] in the bank's dtype, scale [n_adapters] float32 (none:
        all 1): CUDA tensors, not copied."""
        import torch
        c, where = self.cfg, "swapmoe_adapters_set_weights"
        pa = _vector(A, c.n_adapters * c.rank * c.d_in, self._dtype, self._device, where, "A")
        pb = _vector(B, c.n_adapters * c.d_out * c.rank, self._dtype, self._device, where, "B")
        ps = None if scale is None else _vector(scale, c.n_adapters, torch.float32, self._device, where, "scale")
        _check(lib().swapmoe_adapters_set_weights(self._h, pa, pb, ps), where)
        self._keep = (A, B, scale)

    def forward(self, x, ids, y, out, x_scales=None, stream=None) -> None:
        """x [T, d_in] in the bank's dtype, or torch.float8_e4m3fn with x_scales [T] float32; ids [T] int32; y [T, d_out] or
        None (zeros); out [T, d_out], may be y.  Rows may be strided."""
        c = self.cfg
        (_marshal or marshal()).adapters_forward(self._h.value, self._device.index, self._dtype, c.d_in, c.d_out, x, ids, y, out,
                                                 x_scales, stream)


class Layer:
    """One MoE layer served from K resident Virtual-Expert slots (thin handle)."""

    def __init__(self, E: int, d_model: int, d_ff: int, top_k: int, K: int, dtype: int,
                 act: int = ACT_RELU, renorm_topk: int = 0, max_tokens: int = 1,
                 spare_slots: int = 0):
        self.cfg = Config(E, d_model, d_ff, top_k, K, dtype, act, renorm_topk, max_tokens,
                          spare_slots)
        self._h = ctypes.c_void_p()
        _check(lib().swapmoe_create(ctypes.byref(self._h), ctypes.byref(self.cfg)), "swapmoe_create")
        import torch
        self._device = torch.device("cuda", torch.cuda.current_device())
        self._keep = {}
        self.last_T = 0

    # -- lifetime
    def close(self) -> None:
        if self._h:
            lib().swapmoe_destroy(self._h)
            self._h = ctypes.c_void_p()

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    # -- set-up
    def set_router(self, Wr, enorm: np.ndarray, stream=None) -> None:
        enorm = np.ascontiguousarray(enorm, dtype=np.float32)
        assert enorm.size == self.cfg.E
        self._keep["Wr"] = Wr
        _check(lib().swapmoe_set_router(self._h, Wr.data_ptr(), _np_ptr(enorm), _stream_ptr(stream)),
               "swapmoe_set_router")

    def set_resident(self, slot_to_expert: Sequence[int], arena_in, arena_out,
                     phys_slot: Optional[Sequence[int]] = None, stream=None) -> None:
        s2e = np.ascontiguousarray(slot_to_expert, dtype=np.int32)
        assert s2e.size == self.cfg.K
        ph = None if phys_slot is None else np.ascontiguousarray(phys_slot, dtype=np.int32)
        self._keep["arena_in"], self._keep["arena_out"] = arena_in, arena_out
        _check(lib().swapmoe_set_resident(self._h, _np_ptr(s2e), None if ph is None else _np_ptr(ph),
                                          arena_in.data_ptr(), arena_out.data_ptr(),
                                          _stream_ptr(stream)), "swapmoe_set_resident")

    def set_gemm_path(self, path: int) -> None:
        _check(lib().swapmoe_set_gemm_path(self._h, int(path)), "swapmoe_set_gemm_path")

    def _current(self, where: str) -> None:
        import torch
        now = torch.cuda.current_device()
        if now != self._device.index:
            raise _invalid(where, "the layer is on %s, the current device is cuda:%d" % (self._device, now))

    def set_gate(self, gate: Optional[Gate], bias=None) -> None:
        """Later forwards route by ``gate`` (None: by the layer's configuration); ``bias`` [E] float32 on the layer's device, not
        copied."""
        import torch
        where = "swapmoe_set_gate"
        pb = None if bias is None else _vector(bias, self.cfg.E, torch.float32, self._device, where, "bias")
        _check(lib().swapmoe_set_gate(self._h, None if gate is None else ctypes.byref(gate), pb), where)
        self._keep["gate_bias"] = bias

    def set_norm(self, weight, eps: float) -> None:
        """The norm in front of the layer in forward_block: ``weight`` [d_model] in the layer's dtype on its device, not copied."""
        import torch
        where, dt = "swapmoe_set_norm", torch.bfloat16 if self.cfg.dtype == BF16 else torch.float32
        pw = _vector(weight, self.cfg.d_model, dt, self._device, where, "weight")
        self._current(where)                                       # (the rows behind the norm are allocated there)
        _check(lib().swapmoe_set_norm(self._h, pw, eps), where)
        self._keep["norm"] = weight

    # -- hot path
    def forward_block(self, x, residual, out, adapters: Optional[AdapterBank] = None, ids=None, n_tokens: Optional[int] = None,
                      stream=None) -> None:
        """The pre-norm block around the layer: residual += x (None: no residual); out = layer(norm(residual)), plus each
        token's adapter from ``adapters`` by ``ids`` [T] int32 (negative: none).  Rows [T, d_model] of the layer's dtype,
        contiguous, on the layer's device, which has to be the current one."""
        import torch
        where, dt = "swapmoe_forward_block", torch.bfloat16 if self.cfg.dtype == BF16 else torch.float32
        T = int(x.shape[0]) if n_tokens is None else int(n_tokens)
        need = min(T, self.cfg.max_tokens) * self.cfg.d_model      # (more tokens than that: the library's refusal)
        for name, t in (("x", x), ("residual", residual), ("out", out)):
            if t is not None and (t.dtype != dt or t.device != self._device or not t.is_contiguous() or t.numel() < need):
                raise _invalid(where, "%s: %d contiguous rows of %d values of %s on %s expected, got %s of %s on %s" % (
                    name, T, self.cfg.d_model, dt, self._device, tuple(t.shape), t.dtype, t.device))
        if ids is not None:
            _vector(ids, T, torch.int32, self._device, where, "ids")
        if adapters is not None and adapters._device != self._device:
            raise _invalid(where, "adapters: a bank on %s, the layer on %s" % (adapters._device, self._device))
        self._current(where)
        self.last_T = T
        _check(lib().swapmoe_forward_block(
            self._h, x.data_ptr(), None if residual is None else residual.data_ptr(), out.data_ptr(), T,
            None if adapters is None else adapters._h, None if ids is None else ids.data_ptr(), _stream_ptr(stream)), where)

    def forward(self, x, out, n_tokens: Optional[int] = None, stream=None) -> None:
        T = int(x.shape[0]) if n_tokens is None else int(n_tokens)
        self.last_T = T
        _check(lib().swapmoe_forward(self._h, x.data_ptr(), out.data_ptr(), T, _stream_ptr(stream)),
               "swapmoe_forward")

    def forward_timed(self, x, out, events, n_tokens: Optional[int] = None, stream=None) -> None:
        """Like forward, recording the N_STAGES + 1 torch.cuda.Event objects at stage boundaries."""
        T = int(x.shape[0]) if n_tokens is None else int(n_tokens)
        self.last_T = T
        assert len(events) == N_STAGES + 1
        for e in events:              # torch creates the CUDA event lazily, on its first record
            if not e.cuda_event:
                e.record()
        arr = (ctypes.c_void_p * (N_STAGES + 1))(*[e.cuda_event for e in events])
        _check(lib().swapmoe_forward_timed(self._h, x.data_ptr(), out.data_ptr(), T,
                                           _stream_ptr(stream), arr), "swapmoe_forward_timed")

    def rerun_gemm(self, out, which: int, stream=None) -> None:
        """Launches grouped GEMM-1 (which = 1) or GEMM-2 (2) again on the state the last forward left (timing aid)."""
        _check(lib().swapmoe_debug_rerun_gemm(self._h, out.data_ptr(), int(which), _stream_ptr(stream)),
               "swapmoe_debug_rerun_gemm")

    def forward_from_logits(self, x, logits, out, stream=None) -> None:
        T = int(x.shape[0])
        self.last_T = T
        _check(lib().swapmoe_forward_from_logits(self._h, x.data_ptr(), logits.data_ptr(),
                                                 out.data_ptr(), T, _stream_ptr(stream)),
               "swapmoe_forward_from_logits")

    def forward_host(self, x_host, out_host, n_tokens: Optional[int] = None, stream=None) -> None:
        """x_host/out_host: CPU torch tensors (pinned for speed) or numpy arrays."""
        T = int(x_host.shape[0]) if n_tokens is None else int(n_tokens)
        self.last_T = T
        xp = x_host.data_ptr() if hasattr(x_host, "data_ptr") else x_host.ctypes.data
        op = out_host.data_ptr() if hasattr(out_host, "data_ptr") else out_host.ctypes.data
        _check(lib().swapmoe_forward_host(self._h, xp, op, T, _stream_ptr(stream)),
               "swapmoe_forward_host")

    def forward_host_async(self, x_host, out_host, n_tokens: Optional[int] = None, stream=None) -> None:
        """Pipelined host path (pinned CPU tensors); out_host is valid after host_wait()."""
        T = int(x_host.shape[0]) if n_tokens is None else int(n_tokens)
        self.last_T = T
        _check(lib().swapmoe_forward_host_async(self._h, x_host.data_ptr(), out_host.data_ptr(), T,
                                                _stream_ptr(stream)), "swapmoe_forward_host_async")

    def host_wait(self) -> None:
        _check(lib().swapmoe_host_wait(self._h), "swapmoe_host_wait")

    # -- importance and swapping
    def read_importance(self, reset: bool = False, stream=None) -> np.ndarray:
        imp = np.empty(self.cfg.E, dtype=np.float32)
        _check(lib().swapmoe_read_importance(self._h, _np_ptr(imp), int(bool(reset)),
                                             _stream_ptr(stream)), "swapmoe_read_importance")
        return imp

    def read_scores_async(self, kinds: Sequence[str], out_pinned, reset: bool = False, stream=None) -> None:
        """Enqueues one small kernel that writes the scores named in `kinds` ("eq1", "count", "eq1_masked") into a
        pinned float32 tensor [3, E] (row 0 / 1 / 2 for the three scores); no wait - synchronise with the stream
        before reading it."""
        mask = sum(1 << {"eq1": 0, "count": 1, "eq1_masked": 2}[k] for k in kinds)
        assert out_pinned.is_pinned() and out_pinned.numel() >= 3 * self.cfg.E
        _check(lib().swapmoe_read_scores_async(self._h, mask, out_pinned.data_ptr(), int(bool(reset)),
                                               _stream_ptr(stream)), "swapmoe_read_scores_async")

    def read_decode_prefetch(self, reset: bool = False, stream=None):
        """(hits, touched): slots served by one-launch decode steps whose expert had been prefetched to L2, and all."""
        h, t = ctypes.c_int64(0), ctypes.c_int64(0)
        _check(lib().swapmoe_read_decode_prefetch(self._h, ctypes.byref(h), ctypes.byref(t), int(bool(reset)),
                                                  _stream_ptr(stream)), "swapmoe_read_decode_prefetch")
        return int(h.value), int(t.value)

    def read_touched_slots(self, reset: bool = False, stream=None) -> int:
        """Slots that received at least one pair, summed over the forwards since the last reset."""
        v = ctypes.c_int64(0)
        _check(lib().swapmoe_read_touched_slots(self._h, ctypes.byref(v), int(bool(reset)), _stream_ptr(stream)),
               "swapmoe_read_touched_slots")
        return int(v.value)

    def read_score(self, kind: str, reset: bool = False, stream=None) -> np.ndarray:
        """kind: "eq1" (Eq. 1, unmasked routing), "count" (token counts), "eq1_masked"."""
        k = {"eq1": 0, "count": 1, "eq1_masked": 2}[kind]
        out = np.empty(self.cfg.E, dtype=np.float32)
        _check(lib().swapmoe_read_importance_kind(self._h, k, _np_ptr(out), int(bool(reset)),
                                                  _stream_ptr(stream)), "swapmoe_read_importance_kind")
        return out

    def load_slot_async(self, phys: int, in_host_pinned, out_host_pinned, compute_stream, side_stream,
                        done_event=None) -> None:
        """The copy runs on side_stream behind everything enqueued so far on compute_stream."""
        if done_event is not None and not done_event.cuda_event:
            done_event.record(side_stream)      # torch creates the CUDA event on its first record
        ev = None if done_event is None else done_event.cuda_event
        _check(lib().swapmoe_load_slot_async(self._h, int(phys), in_host_pinned.data_ptr(),
                                             out_host_pinned.data_ptr(), _stream_ptr(compute_stream),
                                             _stream_ptr(side_stream), ev), "swapmoe_load_slot_async")

    # -- inspection
    def tap(self, name: str, stream=None) -> np.ndarray:
        which, dt = TAPS[name]
        c, T = self.cfg, self.last_T
        if dt is None:
            dt = np.uint16 if c.dtype == BF16 else np.float32
        shape = {"logits": (T, c.E), "count": (c.K,), "offset": (c.K + 1,), "perm": (T * c.top_k,),
                 "inv": (T * c.top_k,), "xnorm": (T,), "h": (T * c.top_k, c.d_ff),
                 "y": (T * c.top_k, c.d_model), "token_tiles": (2, 2)}.get(name, (T, c.top_k))
        a = np.empty(shape, dtype=dt)
        _check(lib().swapmoe_debug_copy(self._h, which, _np_ptr(a), a.nbytes, _stream_ptr(stream)),
               "swapmoe_debug_copy")
        return a

    def device_status(self, stream=None):
        detail = ctypes.c_int32(0)
        st = lib().swapmoe_device_status(self._h, ctypes.byref(detail), _stream_ptr(stream))
        return int(st), int(detail.value)

    def selftest_bounded_wait(self, limit_ms: int = 20, stream=None) -> None:
        _check(lib().swapmoe_selftest_bounded_wait(self._h, int(limit_ms), _stream_ptr(stream)),
               "swapmoe_selftest_bounded_wait")

    @property
    def launch_count(self) -> int:
        return int(lib().swapmoe_launch_count(self._h))

    @property
    def workspace_bytes(self) -> int:
        return int(lib().swapmoe_workspace_bytes(self._h))
