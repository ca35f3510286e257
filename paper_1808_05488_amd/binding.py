"""ctypes binding of libcbconv.so: argument marshalling only.

The functions carry the names of the C ABI (include/cbconv.h).  torch is used
for device memory and streams; every step of the path runs in the library's HIP
kernels.  There is no fallback: if the library is not built, loading fails.
"""
from __future__ import annotations

import ctypes as C
import os
import struct
from typing import Optional, Tuple

import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libcbconv.so")

CB_OK, CB_EINVAL, CB_ENOMEM, CB_EHIP, CB_ESTATE = 0, -1, -2, -3, -4
CB_F32, CB_BF16, CB_E4M3 = 0, 1, 8
CB_CLOSED_LOOP, CB_FEED_FORWARD, CB_PROPAGATE = 0, 1, 2
CB_BACKEND_AUTO, CB_BACKEND_EXPLICIT, CB_BACKEND_FUSED = 0, 1, 2
CB_NUM_STEPS = 9
STEP_NAMES = ("detect", "dilate", "compact", "gather", "gemm", "update", "fused", "state", "total")

EXPORTS = (
    "cb_layer_workspace_bytes", "cb_layer_min_scratch_bytes", "cb_layer_create", "cb_process_frame",
    "cb_process_frame_propagated", "cb_process_frame_chained", "cb_layer_changes", "cb_layer_state", "cb_layer_matrices",
    "cb_layer_export_state", "cb_layer_import_state",
    "cb_layer_out_shape", "cb_layer_set_timing", "cb_layer_stats", "cb_set_scan_wait_limit", "cb_layer_reset",
    "cb_layer_destroy",
    "cb_pool_workspace_bytes", "cb_pool_create", "cb_pool_process", "cb_pool_changes", "cb_pool_out_shape",
    "cb_pool_destroy", "cb_strerror", "cb_last_hip_error", "cb_version",
    "cb_network_forward", "cb_sum_squared_diff", "cb_sum_squared_diff_noalloc", "cb_select_workspace_bytes",
    "cb_select_thresholds",
    "cb_rotary_init", "cb_rotate", "cb_norm_rotate", "cb_norm_rotate_back_scratch_bytes", "cb_norm_rotate_back",
    "cb_cache_scratch_bytes", "cb_cache_append", "cb_cache_attend", "cb_cache_bound", "cb_cache_choose", "cb_cache_attend_chosen", "cb_cache_evict",
)
CB_METRIC_WORKSPACE_BYTES = 4096
CB_PAIRS_HALVES, CB_PAIRS_ADJACENT = 0, 1
CB_LADDER_SHARED, CB_LADDER_PER_AXIS = 0, 1
CB_ROTARY_MAX_AXES, CB_ROTARY_MAX_PAIRS = 4, 128


class cb_layer_desc(C.Structure):
    _fields_ = [(n, C.c_int32) for n in ("c_in", "c_out", "kh", "kw", "stride", "pad", "h_in", "w_in",
                                         "dtype", "relu", "mode", "backend", "keep_output_channel_last",
                                         "gather_channel_last")] + [("reserved", C.c_int32 * 2)]


class cb_stage(C.Structure):
    _fields_ = [("layer", C.c_void_p), ("pool", C.c_void_p)]


class cb_select_params(C.Structure):
    _fields_ = [("tau0", C.c_float), ("factor", C.c_float), ("max_steps", C.c_int32), ("reserved", C.c_int32)]


class cb_heads(C.Structure):
    _fields_ = [("data_dev", C.c_void_p), ("token_stride", C.c_int64), ("head_stride", C.c_int64),
                ("heads", C.c_int32), ("reserved", C.c_int32)]


class cb_rotary_desc(C.Structure):
    _fields_ = [("head_dim", C.c_int32), ("n_axes", C.c_int32), ("pairs", C.c_int32 * CB_ROTARY_MAX_AXES),
                ("layout", C.c_int32), ("ladder", C.c_int32), ("base", C.c_float), ("reserved", C.c_int32)]


class cb_rotary(C.Structure):
    _fields_ = [("desc", cb_rotary_desc), ("turns", C.c_double * CB_ROTARY_MAX_PAIRS)]


class cb_cache(C.Structure):
    _fields_ = [(n, C.c_int32) for n in ("n_seq", "n_kv_heads", "head_dim", "page_tokens", "max_pages", "n_pages",
                                         "dtype", "reserved")] + \
               [(n, C.c_void_p) for n in ("k_pages_dev", "v_pages_dev", "table_dev", "lengths_dev", "weight_dev", "time_dev",
                                          "scratch_dev")] + [("scratch_bytes", C.c_size_t), ("values_dtype", C.c_int32), ("reserved2", C.c_int32)] + \
               [(n, C.c_void_p) for n in ("k_scale_dev", "v_scale_dev", "bounds_dev")]


class cb_norm_back(C.Structure):
    _fields_ = [("x", cb_heads), ("out_grad", cb_heads), ("x_grad", cb_heads), ("weight_dev", C.c_void_p), ("weight_grad_dev", C.c_void_p)]


class cb_choose_params(C.Structure):
    _fields_ = [(n, C.c_int32) for n in ("budget", "first", "recent", "reserved")]


class cb_attend_params(C.Structure):
    _fields_ = [("scale", C.c_float), ("softcap", C.c_float), ("decay", C.c_float), ("accumulate", C.c_int32),
                ("reserved", C.c_int32)]


class cb_evict_params(C.Structure):
    _fields_ = [("budget", C.c_int32), ("window", C.c_int32), ("weight_in_dev", C.c_void_p),
                ("time_in_dev", C.c_void_p), ("lengths_in_dev", C.c_void_p)]


class cb_stats(C.Structure):
    _fields_ = [("n_changed_in", C.c_int32), ("n_changed_out", C.c_int32), ("ops", C.c_int64),
                ("us_step", C.c_float * CB_NUM_STEPS), ("scan_recounts", C.c_int32), ("reserved", C.c_int32)]


class CBError(RuntimeError):
    def __init__(self, status: int, where: str):
        self.status = status
        msg = lib().cb_strerror(status).decode()
        if status == CB_EHIP:
            msg += f" (hipError {lib().cb_last_hip_error()})"
        super().__init__(f"{where}: {msg} [{status}]")


_lib = None


def lib():
    """Load libcbconv.so; raises if it has not been built (no fallback path)."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise FileNotFoundError(
                f"{LIB_PATH} is missing: build it with `python -m paper_1808_05488_amd.build` "
                "(or __graft_entry__.build()); there is no non-HIP fallback")
        L = C.CDLL(LIB_PATH)
        # torch's streams and allocations are only valid in the HIP runtime torch loaded
        with open("/proc/self/maps") as f:
            runtimes = {ln.split()[-1] for ln in f if "libamdhip64" in ln}
        if len(runtimes) > 1:
            raise RuntimeError(f"two HIP runtimes are loaded {sorted(runtimes)}; rebuild libcbconv.so "
                               "with paper_1808_05488_amd.build so that it links torch's runtime")
        vp, i32, sz = C.c_void_p, C.c_int32, C.c_size_t
        P = C.POINTER
        L.cb_layer_workspace_bytes.argtypes = [P(cb_layer_desc), P(sz), P(sz)]
        L.cb_layer_min_scratch_bytes.argtypes = [P(cb_layer_desc), P(sz)]
        L.cb_layer_create.argtypes = [P(cb_layer_desc), vp, vp, vp, sz, vp, sz, vp, P(vp)]
        L.cb_process_frame.argtypes = [vp, vp, C.c_float, P(vp)]
        L.cb_process_frame_propagated.argtypes = [vp, vp, vp, vp, P(vp)]
        L.cb_process_frame_chained.argtypes = [vp, vp, vp, vp, C.c_float, P(vp)]
        L.cb_layer_changes.argtypes = [vp, P(vp), P(vp), P(vp), P(vp)]
        L.cb_network_forward.argtypes = [P(cb_stage), C.c_int32, vp, P(C.c_float), P(vp)]
        L.cb_sum_squared_diff.argtypes = [vp, vp, sz, C.c_int32, vp, P(C.c_double), vp]
        L.cb_sum_squared_diff_noalloc.argtypes = [vp, vp, sz, C.c_int32, P(C.c_double), vp]
        L.cb_select_workspace_bytes.argtypes = [P(cb_stage), C.c_int32, C.c_int32, P(sz)]
        L.cb_select_thresholds.argtypes = [P(cb_stage), C.c_int32, P(vp), C.c_int32, C.c_int32, P(cb_select_params),
                                           P(C.c_double), vp, sz, P(C.c_float), P(C.c_double), P(C.c_int32)]
        L.cb_layer_state.argtypes = [vp, P(vp)]
        L.cb_layer_matrices.argtypes = [vp, P(vp), P(vp), P(vp)]
        L.cb_layer_export_state.argtypes = [vp, vp, vp]
        L.cb_layer_import_state.argtypes = [vp, vp, vp]
        L.cb_layer_out_shape.argtypes = [vp, P(i32), P(i32), P(i32)]
        L.cb_layer_set_timing.argtypes = [vp, i32]
        L.cb_layer_stats.argtypes = [vp, P(cb_stats)]
        L.cb_set_scan_wait_limit.argtypes = [i32]
        L.cb_layer_reset.argtypes = [vp]
        L.cb_layer_destroy.argtypes = [vp]
        L.cb_pool_workspace_bytes.argtypes = [vp, i32, P(sz)]
        L.cb_pool_create.argtypes = [vp, i32, vp, sz, vp, P(vp)]
        L.cb_pool_process.argtypes = [vp, P(vp)]
        L.cb_pool_changes.argtypes = [vp, P(vp)]
        L.cb_pool_out_shape.argtypes = [vp, P(i32), P(i32), P(i32)]
        L.cb_pool_destroy.argtypes = [vp]
        # (structures by address: byref(), bytes or the address itself)
        L.cb_rotary_init.argtypes = [vp, vp]
        L.cb_rotate.argtypes = [vp, i32, C.c_int64, vp, vp, vp, vp, vp, i32, vp]
        L.cb_cache_scratch_bytes.argtypes = [vp, i32, P(sz)]
        L.cb_cache_append.argtypes = [vp, vp, i32, vp, vp, vp, vp, vp, vp, vp, vp]
        L.cb_cache_attend.argtypes = [vp, vp, vp, vp, vp, vp]
        L.cb_cache_evict.argtypes = [vp, vp, vp]
        L.cb_norm_rotate.argtypes = [vp, i32, C.c_int64, vp, C.c_float, i32, vp, vp, vp, vp, vp, vp, vp]
        L.cb_norm_rotate_back_scratch_bytes.argtypes = [vp, P(sz)]
        L.cb_norm_rotate_back.argtypes = [vp, i32, C.c_int64, vp, C.c_float, i32, vp, vp, vp, sz, vp]
        L.cb_cache_bound.argtypes = [vp, vp, vp]
        L.cb_cache_choose.argtypes = [vp, vp, vp, vp, vp, vp]
        L.cb_cache_attend_chosen.argtypes = [vp, vp, vp, vp, vp, vp, vp, i32, vp]
        L.cb_strerror.argtypes = [C.c_int]
        L.cb_strerror.restype = C.c_char_p
        L.cb_last_hip_error.restype = C.c_int
        L.cb_version.restype = C.c_int
        for name in EXPORTS:
            if name not in ("cb_strerror",):
                getattr(L, name).restype = getattr(L, name).restype or C.c_int
        _lib = L
    return _lib


def _check(status: int, where: str) -> None:
    if status != CB_OK:
        raise CBError(status, where)


def _ptr(t) -> Optional[int]:
    if t is None:
        return None
    if isinstance(t, int):
        return t
    return t.data_ptr()


def make_desc(c_in, c_out, kh, kw, stride, pad, h_in, w_in, dtype=CB_F32, relu=0, mode=CB_CLOSED_LOOP,
              backend=CB_BACKEND_AUTO, keep_output_channel_last=False, gather_channel_last=False):
    d = cb_layer_desc()
    d.c_in, d.c_out, d.kh, d.kw, d.stride, d.pad, d.h_in, d.w_in = c_in, c_out, kh, kw, stride, pad, h_in, w_in
    d.dtype, d.relu, d.mode, d.backend = dtype, int(relu), mode, backend
    d.keep_output_channel_last, d.gather_channel_last = int(keep_output_channel_last), int(gather_channel_last)
    return d


# ---------------------------------------------------------------- C ABI, one to one
def cb_version() -> int:
    return lib().cb_version()


def cb_layer_workspace_bytes(desc: cb_layer_desc) -> Tuple[int, int]:
    a, b = C.c_size_t(), C.c_size_t()
    _check(lib().cb_layer_workspace_bytes(C.byref(desc), C.byref(a), C.byref(b)), "cb_layer_workspace_bytes")
    return a.value, b.value


def cb_layer_min_scratch_bytes(desc: cb_layer_desc) -> int:
    b = C.c_size_t()
    _check(lib().cb_layer_min_scratch_bytes(C.byref(desc), C.byref(b)), "cb_layer_min_scratch_bytes")
    return b.value


def cb_layer_create(desc, w_dev, bias_dev, state_dev, state_bytes, scratch_dev, scratch_bytes, stream=0) -> int:
    h = C.c_void_p()
    _check(lib().cb_layer_create(C.byref(desc), _ptr(w_dev), _ptr(bias_dev), _ptr(state_dev), state_bytes,
                                 _ptr(scratch_dev), scratch_bytes, stream or None, C.byref(h)), "cb_layer_create")
    return h.value


def cb_process_frame(layer: int, input_dev, tau: float) -> int:
    out = C.c_void_p()
    _check(lib().cb_process_frame(layer, _ptr(input_dev), C.c_float(tau), C.byref(out)), "cb_process_frame")
    return out.value


def cb_process_frame_propagated(layer: int, input_dev, producer_layer=None, producer_pool=None) -> int:
    out = C.c_void_p()
    _check(lib().cb_process_frame_propagated(layer, _ptr(input_dev), producer_layer, producer_pool, C.byref(out)),
           "cb_process_frame_propagated")
    return out.value


def cb_process_frame_chained(layer: int, input_dev, producer_layer=None, producer_pool=None, tau: float = 0.0) -> int:
    out = C.c_void_p()
    _check(lib().cb_process_frame_chained(layer, _ptr(input_dev), producer_layer, producer_pool, C.c_float(tau),
                                          C.byref(out)), "cb_process_frame_chained")
    return out.value


def cb_layer_changes(layer: int) -> Tuple[int, int, int, int]:
    a, b, c, d = C.c_void_p(), C.c_void_p(), C.c_void_p(), C.c_void_p()
    _check(lib().cb_layer_changes(layer, C.byref(a), C.byref(b), C.byref(c), C.byref(d)), "cb_layer_changes")
    return a.value, b.value, c.value, d.value


def cb_layer_state(layer: int) -> int:
    a = C.c_void_p()
    _check(lib().cb_layer_state(layer, C.byref(a)), "cb_layer_state")
    return a.value


def cb_layer_export_state(layer: int, state_out, output_out) -> None:
    _check(lib().cb_layer_export_state(layer, _ptr(state_out), _ptr(output_out)), "cb_layer_export_state")


def cb_layer_import_state(layer: int, state_in, output_in) -> None:
    _check(lib().cb_layer_import_state(layer, _ptr(state_in), _ptr(output_in)), "cb_layer_import_state")


def cb_layer_matrices(layer: int) -> Tuple[int, int, int]:
    a, b, c = C.c_void_p(), C.c_void_p(), C.c_void_p()
    _check(lib().cb_layer_matrices(layer, C.byref(a), C.byref(b), C.byref(c)), "cb_layer_matrices")
    return a.value, b.value, c.value


def cb_layer_out_shape(layer: int) -> Tuple[int, int, int]:
    a, b, c = C.c_int32(), C.c_int32(), C.c_int32()
    _check(lib().cb_layer_out_shape(layer, C.byref(a), C.byref(b), C.byref(c)), "cb_layer_out_shape")
    return a.value, b.value, c.value


def cb_layer_set_timing(layer: int, on: bool) -> None:
    _check(lib().cb_layer_set_timing(layer, int(on)), "cb_layer_set_timing")


def cb_layer_stats(layer: int) -> dict:
    s = cb_stats()
    _check(lib().cb_layer_stats(layer, C.byref(s)), "cb_layer_stats")
    return {"n_changed_in": s.n_changed_in, "n_changed_out": s.n_changed_out, "ops": s.ops,
            "us_step": {n: float(s.us_step[i]) for i, n in enumerate(STEP_NAMES)}, "scan_recounts": s.scan_recounts}


def cb_set_scan_wait_limit(polls: int) -> None:
    _check(lib().cb_set_scan_wait_limit(int(polls)), "cb_set_scan_wait_limit")


def cb_layer_reset(layer: int) -> None:
    _check(lib().cb_layer_reset(layer), "cb_layer_reset")


def cb_layer_destroy(layer: int) -> None:
    _check(lib().cb_layer_destroy(layer), "cb_layer_destroy")


def cb_pool_workspace_bytes(producer: int, window: int = 2) -> int:
    a = C.c_size_t()
    _check(lib().cb_pool_workspace_bytes(producer, window, C.byref(a)), "cb_pool_workspace_bytes")
    return a.value


def cb_pool_create(producer: int, window, state_dev, state_bytes, stream=0) -> int:
    h = C.c_void_p()
    _check(lib().cb_pool_create(producer, window, _ptr(state_dev), state_bytes, stream or None, C.byref(h)),
           "cb_pool_create")
    return h.value


def cb_pool_process(pool: int) -> int:
    out = C.c_void_p()
    _check(lib().cb_pool_process(pool, C.byref(out)), "cb_pool_process")
    return out.value


def cb_pool_changes(pool: int) -> int:
    a = C.c_void_p()
    _check(lib().cb_pool_changes(pool, C.byref(a)), "cb_pool_changes")
    return a.value


def cb_pool_out_shape(pool: int) -> Tuple[int, int, int]:
    a, b, c = C.c_int32(), C.c_int32(), C.c_int32()
    _check(lib().cb_pool_out_shape(pool, C.byref(a), C.byref(b), C.byref(c)), "cb_pool_out_shape")
    return a.value, b.value, c.value


def cb_pool_destroy(pool: int) -> None:
    _check(lib().cb_pool_destroy(pool), "cb_pool_destroy")


# ---------------------------------------------------------------- device-memory helpers
_TORCH_DT = {CB_F32: torch.float32, CB_BF16: torch.bfloat16}


def _alloc(nbytes: int, device) -> torch.Tensor:
    """256-byte aligned byte buffer from torch's allocator."""
    t = torch.empty(nbytes + 256, dtype=torch.uint8, device=device)
    off = (-t.data_ptr()) % 256
    return t[off:off + nbytes]


def _view(owner: torch.Tensor, ptr: int, shape, dtype) -> torch.Tensor:
    """Tensor view of memory at `ptr` inside the byte buffer `owner`."""
    n = 1
    for s in shape:
        n *= s
    nbytes = n * torch.empty((), dtype=dtype).element_size()
    off = ptr - owner.data_ptr()
    assert 0 <= off and off + nbytes <= owner.numel(), "pointer outside its owner buffer"
    return owner[off:off + nbytes].view(dtype).view(*shape)


class _Views:
    """Tensor views of elements of the byte buffer `owner`, one torch operation each (slicing the bytes and viewing them
    as elements and as a shape is three, on every frame)."""

    def __init__(self, owner: torch.Tensor, dtype):
        self.elems = owner.view(dtype)
        self.ptr, self.first, self.size = owner.data_ptr(), self.elems.storage_offset(), self.elems.element_size()

    def __call__(self, ptr: int, shape) -> torch.Tensor:
        c, h, w = shape
        off = (ptr - self.ptr) // self.size
        assert 0 <= off and off + c * h * w <= self.elems.numel(), "pointer outside its owner buffer"
        return self.elems.as_strided(shape, (h * w, w, 1), self.first + off)


class Layer:
    """A cb_layer with its buffers held by torch tensors (memory plumbing only)."""

    def __init__(self, weight: torch.Tensor, bias: Optional[torch.Tensor], stride: int, pad: int, h_in: int,
                 w_in: int, relu: bool, mode: int = CB_CLOSED_LOOP, scratch: Optional[torch.Tensor] = None,
                 scratch_bytes: Optional[int] = None, stream: Optional[torch.cuda.Stream] = None,
                 backend: int = CB_BACKEND_AUTO, keep_output_channel_last: bool = False,
                 gather_channel_last: bool = False):
        assert weight.is_cuda and weight.is_contiguous()
        self.device = weight.device
        self.dtype = CB_BF16 if weight.dtype == torch.bfloat16 else CB_F32
        assert weight.dtype in (torch.float32, torch.bfloat16)
        O, Cc, kh, kw = weight.shape
        self.desc = make_desc(Cc, O, kh, kw, stride, pad, h_in, w_in, self.dtype, relu, mode, backend,
                              keep_output_channel_last, gather_channel_last)
        state_bytes, rec_scratch = cb_layer_workspace_bytes(self.desc)
        self.state_buf = _alloc(state_bytes, self.device)
        if scratch is None:
            scratch = _alloc(scratch_bytes if scratch_bytes is not None else rec_scratch, self.device)
        self.scratch_buf = scratch
        self.stream = stream
        sh = stream.cuda_stream if stream is not None else torch.cuda.current_stream(self.device).cuda_stream
        self.stream_handle = sh
        if bias is not None:
            assert bias.dtype == weight.dtype and bias.is_contiguous()
        self.handle = cb_layer_create(self.desc, weight, bias, self.state_buf, self.state_buf.numel(),
                                      self.scratch_buf, self.scratch_buf.numel(), sh)
        self.C, self.H, self.W = Cc, h_in, w_in
        self.O, self.Ho, self.Wo = cb_layer_out_shape(self.handle)
        self._keep = (weight, bias)
        self._producers = []               # layers whose list this one may have taken over
        self._views = _Views(self.state_buf, _TORCH_DT[self.dtype])

    def _fed_by(self, producer):
        if isinstance(producer, Layer) and producer not in self._producers:
            self._producers.append(producer)

    def close(self):
        if getattr(self, "handle", None):
            cb_layer_destroy(self.handle)
            self.handle = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def process_frame(self, x: torch.Tensor, tau: float) -> torch.Tensor:
        assert x.is_cuda and x.is_contiguous() and x.dtype == _TORCH_DT[self.dtype]
        assert tuple(x.shape[-3:]) == (self.C, self.H, self.W), (tuple(x.shape), (self.C, self.H, self.W))
        p = cb_process_frame(self.handle, x, tau)
        return self._views(p, (self.O, self.Ho, self.Wo))

    def process_frame_chained(self, x: torch.Tensor, producer, tau: float) -> torch.Tensor:
        assert x.is_cuda and x.is_contiguous() and x.dtype == _TORCH_DT[self.dtype]
        assert tuple(x.shape[-3:]) == (self.C, self.H, self.W)
        if isinstance(producer, Pool):
            p = cb_process_frame_chained(self.handle, x, None, producer.handle, tau)
        else:
            p = cb_process_frame_chained(self.handle, x, producer.handle, None, tau)
        return self._views(p, (self.O, self.Ho, self.Wo))

    def process_frame_propagated(self, x: torch.Tensor, producer) -> torch.Tensor:
        assert x.is_cuda and x.is_contiguous() and x.dtype == _TORCH_DT[self.dtype]
        assert tuple(x.shape[-3:]) == (self.C, self.H, self.W)
        if isinstance(producer, Pool):
            p = cb_process_frame_propagated(self.handle, x, None, producer.handle)
        else:
            self._fed_by(producer)
            p = cb_process_frame_propagated(self.handle, x, producer.handle, None)
        return self._views(p, (self.O, self.Ho, self.Wo))

    def changes(self):
        """(m, m~, idx, N) of the last frame as device tensors (idx is sliced to N on the host)."""
        m, mt, idx, cnt = cb_layer_changes(self.handle)
        m_t = _view(self.state_buf, m, (self.H, self.W), torch.uint8)
        mt_t = _view(self.state_buf, mt, (self.Ho, self.Wo), torch.uint8)
        return m_t, mt_t, idx, cnt

    def changes_host(self):
        import numpy as np
        m, mt, idx_p, cnt_p = cb_layer_changes(self.handle)
        m_t = _view(self.state_buf, m, (self.H, self.W), torch.uint8).cpu().numpy()
        mt_t = _view(self.state_buf, mt, (self.Ho, self.Wo), torch.uint8).cpu().numpy()
        n = cb_layer_stats(self.handle)["n_changed_out"]
        idx = _raw_to_host(idx_p, n, self.device)
        return m_t, mt_t, idx.astype(np.int32), n

    def listed(self):
        """(list, count) of the last frame's changed output pixels as views of the memory of the layer that made them (a propagated 1 x 1 layer takes its
        producer's): Ho * Wo int32 linear indices, of which the first count[0] are the last frame's, in ascending order.  Nothing waits; that
        layer's next frame overwrites both."""
        idx, cnt = C.c_void_p(), C.c_void_p()
        _check(lib().cb_layer_changes(self.handle, None, None, C.byref(idx), C.byref(cnt)), "cb_layer_changes")
        made, seen = [self], {id(self)}
        for layer in made:                 # (grows as it goes)
            if layer.state_buf.data_ptr() <= idx.value < layer.state_buf.data_ptr() + layer.state_buf.numel():
                return (_view(layer.state_buf, idx.value, (self.Ho * self.Wo,), torch.int32), _view(layer.state_buf, cnt.value, (1,), torch.int32))
            for p in layer._producers:
                if id(p) not in seen:
                    seen.add(id(p))
                    made.append(p)
        raise RuntimeError("the list is that of a layer that this object has not been given as a producer")

    def state(self) -> torch.Tensor:
        return self._views(cb_layer_state(self.handle), (self.C, self.H, self.W))

    def export_state(self):
        """(input state or None for a CB_PROPAGATE layer, cached output) as new tensors."""
        dt = _TORCH_DT[self.dtype]
        st = None if self.desc.mode == CB_PROPAGATE else torch.empty((self.C, self.H, self.W), dtype=dt, device=self.device)
        out = torch.empty((self.O, self.Ho, self.Wo), dtype=dt, device=self.device)
        cb_layer_export_state(self.handle, st, out)
        return st, out

    def import_state(self, state: Optional[torch.Tensor], out: torch.Tensor):
        dt = _TORCH_DT[self.dtype]
        assert out.is_cuda and out.is_contiguous() and out.dtype == dt and tuple(out.shape) == (self.O, self.Ho, self.Wo)
        if state is not None:
            assert state.is_cuda and state.is_contiguous() and state.dtype == dt
            assert tuple(state.shape) == (self.C, self.H, self.W)
        cb_layer_import_state(self.handle, state, out)

    def stats(self) -> dict:
        return cb_layer_stats(self.handle)

    def set_timing(self, on: bool):
        cb_layer_set_timing(self.handle, on)

    def reset(self):
        cb_layer_reset(self.handle)


def _raw_to_host(ptr: int, n: int, device):
    """Copy n int32 from a raw device pointer to a numpy array (hipMemcpy through torch's HIP runtime)."""
    import numpy as np
    out = np.zeros(n, np.int32)
    if n == 0:
        return out
    hip = _hip_runtime()
    torch.cuda.synchronize(device)
    rc = hip.hipMemcpy(C.c_void_p(out.ctypes.data), C.c_void_p(ptr), C.c_size_t(4 * n), 2)
    if rc != 0:
        raise RuntimeError(f"hipMemcpy failed: {rc}")
    return out


_hip = None


def _hip_runtime():
    global _hip
    if _hip is None:
        for name in ("libamdhip64.so", "libamdhip64.so.7", "libamdhip64.so.6"):
            try:
                _hip = C.CDLL(name)
                break
            except OSError:
                continue
        if _hip is None:
            _hip = C.CDLL(os.path.join(os.environ.get("ROCM_PATH", "/opt/rocm"), "lib", "libamdhip64.so"))
        _hip.hipMemcpy.argtypes = [C.c_void_p, C.c_void_p, C.c_size_t, C.c_int]
        _hip.hipMemcpy.restype = C.c_int
    return _hip


def cb_sum_squared_diff(a_dev, b_dev, n: int, dtype: int, workspace_dev, stream=0) -> float:
    out = C.c_double()
    _check(lib().cb_sum_squared_diff(_ptr(a_dev), _ptr(b_dev), n, dtype, _ptr(workspace_dev), C.byref(out),
                                     stream or None), "cb_sum_squared_diff")
    return out.value


def cb_sum_squared_diff_noalloc(a_dev, b_dev, n: int, dtype: int, stream=0) -> float:
    out = C.c_double()
    _check(lib().cb_sum_squared_diff_noalloc(_ptr(a_dev), _ptr(b_dev), n, dtype, C.byref(out), stream or None),
           "cb_sum_squared_diff_noalloc")
    return out.value


class Network:
    """A chain of Layer objects, each optionally followed by its Pool (cb_stage array of the C ABI)."""

    def __init__(self, layers, pools=None):
        pools = pools if pools is not None else [None] * len(layers)
        assert len(pools) == len(layers)
        self.layers, self.pools = list(layers), list(pools)
        self.n = len(layers)
        self.stages = (cb_stage * self.n)()
        for s in range(self.n):
            self.stages[s].layer = self.layers[s].handle
            self.stages[s].pool = self.pools[s].handle if self.pools[s] is not None else None
        last = self.pools[-1] if self.pools[-1] is not None else self.layers[-1]
        self.out_shape = (last.O, last.Hp, last.Wp) if self.pools[-1] is not None else (last.O, last.Ho, last.Wo)
        for a, p, b in zip(self.layers, self.pools, self.layers[1:]):
            if p is None:
                b._fed_by(a)
        self._views = last._views
        self.dtype = self.layers[-1].dtype
        self.device = self.layers[0].device

    def reset(self):
        for L in self.layers:
            L.reset()

    def forward(self, x: torch.Tensor, taus) -> torch.Tensor:
        assert x.is_cuda and x.is_contiguous() and len(taus) == self.n
        t = (C.c_float * self.n)(*[float(v) for v in taus])
        out = C.c_void_p()
        _check(lib().cb_network_forward(self.stages, self.n, _ptr(x), t, C.byref(out)), "cb_network_forward")
        return self._views(out.value, self.out_shape)

    def select_thresholds(self, sequences, tau0: float, factor: float, max_loss, max_steps: int = 200):
        """Sec. III-F threshold selection over `sequences` (lists of equally many device frames).
        Returns (thresholds, loss at each selected threshold, thresholds tried per stage)."""
        n_seq, n_frames = len(sequences), len(sequences[0])
        assert all(len(sq) == n_frames for sq in sequences) and len(max_loss) == self.n
        ptrs = (C.c_void_p * (n_seq * n_frames))(*[_ptr(f) for sq in sequences for f in sq])
        nbytes = C.c_size_t()
        _check(lib().cb_select_workspace_bytes(self.stages, self.n, n_seq, C.byref(nbytes)),
               "cb_select_workspace_bytes")
        ws = _alloc(nbytes.value, self.device)
        prm = cb_select_params(float(tau0), float(factor), int(max_steps), 0)
        ml = (C.c_double * self.n)(*[float(v) for v in max_loss])
        taus, loss, steps = (C.c_float * self.n)(), (C.c_double * self.n)(), (C.c_int32 * self.n)()
        _check(lib().cb_select_thresholds(self.stages, self.n, ptrs, n_seq, n_frames, C.byref(prm), ml, _ptr(ws),
                                          nbytes.value, taus, loss, steps), "cb_select_thresholds")
        return list(taus), list(loss), list(steps)


class Pool:
    """A cb_pool fed by a Layer."""

    def __init__(self, producer: Layer, window: int = 2):
        self.producer = producer
        nbytes = cb_pool_workspace_bytes(producer.handle, window)
        self.state_buf = _alloc(nbytes, producer.device)
        self.handle = cb_pool_create(producer.handle, window, self.state_buf, self.state_buf.numel(),
                                     producer.stream_handle)
        self.O, self.Hp, self.Wp = cb_pool_out_shape(self.handle)
        self.dtype = producer.dtype
        self.stream_handle = producer.stream_handle
        self.device = producer.device
        self._views = _Views(self.state_buf, _TORCH_DT[self.dtype])

    def close(self):
        if getattr(self, "handle", None):
            cb_pool_destroy(self.handle)
            self.handle = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def process(self) -> torch.Tensor:
        p = cb_pool_process(self.handle)
        return self._views(p, (self.O, self.Hp, self.Wp))

    def changes(self) -> torch.Tensor:
        return _view(self.state_buf, cb_pool_changes(self.handle), (self.Hp, self.Wp), torch.uint8)


# ---------------------------------------------------------------- tokens of a stream
# (What keeps addresses of the wrong kind from the GPU is raised, not asserted: it holds under python -O too.)
_CB_DT = {torch.float32: CB_F32, torch.bfloat16: CB_BF16}
_E4M3 = torch.float8_e4m3fn
_BYTE_BLOCK = 16                   # tokens that share a scale of a cache in 8 bits
# The structures of one call, packed anew for it (a call may run while another thread packs its own).  A call's work on the host is
# part of a small call's time: packing takes 0.2 us a structure, filling a ctypes one 0.5 us.
_pack_heads = struct.Struct("@Pqqii").pack
_pack_attend = struct.Struct("@fffii").pack
_pack_evict = struct.Struct("@iiPPP").pack
_pack_two = struct.Struct("@PP").pack
_pack_choose = struct.Struct("@iiii").pack
assert struct.calcsize("@Pqqii") == C.sizeof(cb_heads) and struct.calcsize("@fffii") == C.sizeof(cb_attend_params)
assert struct.calcsize("@iiPPP") == C.sizeof(cb_evict_params) and struct.calcsize("@iiii") == C.sizeof(cb_choose_params)
assert 3 * struct.calcsize("@Pqqii") + 2 * struct.calcsize("@P") == C.sizeof(cb_norm_back)
_NO_HEADS = _pack_heads(0, 0, 0, 0, 0)
_raw_stream = torch._C._cuda_getCurrentRawStream if hasattr(torch._C, "_cuda_getCurrentRawStream") else \
    (lambda index: torch.cuda.current_stream(index).cuda_stream)
# (Kernels go to the current device, whose default stream has the same address as every other's: calls on tensors of another one make that one current first.)
_current_device = torch._C._cuda_getDevice if hasattr(torch._C, "_cuda_getDevice") else torch.cuda.current_device


def _heads(t: torch.Tensor, what: str, dtype, index: int, dim: int, heads: Optional[int] = None, tokens: Optional[int] = None) -> bytes:
    """A tokens x heads x head_dim tensor whose heads are contiguous, as the ABI takes it (cb_heads)."""
    shape, stride = t.shape, t.stride()
    if not (t.dtype is dtype and t.get_device() == index and len(shape) == 3 and shape[2] == dim and
            (stride[2] == 1 or t.numel() == 0) and (heads is None or shape[1] == heads) and (tokens is None or shape[0] == tokens)):
        raise AssertionError(f"{what}: {t.dtype} {tuple(shape)}, strides {stride}, on {t.device}; needed: {dtype} "
                             f"({'tokens' if tokens is None else tokens}, {'heads' if heads is None else heads}, {dim}), "
                             f"contiguous heads, on GPU {index}")
    return _pack_heads(t.data_ptr(), stride[0], stride[1], shape[1], 0)


def _fresh(t: torch.Tensor, dim: int) -> bytes:
    """... of a dense one that was made for the call."""
    heads = t.shape[1]
    return _pack_heads(t.data_ptr(), heads * dim, dim, heads, 0)


def _dense(t: Optional[torch.Tensor], what: str, dtype, index: int, shape) -> Optional[int]:
    """Address of a dense array of that type and shape (None: not given)."""
    if t is None:
        return None
    if not (t.dtype is dtype and t.get_device() == index and t.shape == shape and t.is_contiguous()):
        raise AssertionError(f"{what}: {t.dtype} {tuple(t.shape)}, strides {t.stride()}, on {t.device}; needed: dense {dtype} {tuple(shape)} on GPU {index}")
    return t.data_ptr()


def _given(*outs) -> tuple:
    """Those outputs that are given.  One that wants a gradient is refused where it would be part of a graph: what is written to it carries none."""
    given = tuple(t for t in outs if t is not None)
    if torch.is_grad_enabled() and any(t.requires_grad for t in given):
        raise AssertionError("an output that is given carries no gradient: give a detached one, or call under torch.no_grad()")
    return given


# Kernels write through addresses, past torch, whose graphs go by a tensor's version to find that what they have saved is still there: outputs that were
# given, which may be an input that a graph has saved, get a new one.  (0.7 us, for calls that give some.)
_written = torch.autograd.graph.increment_version


# Forward-mode derivatives live beside tensors at a level that is entered (torch.autograd.forward_ad.dual_level), and kernels see the values alone.
_dual = torch.autograd.forward_ad


def _refuse_tangents(*tensors) -> None:
    if any(t is not None and _dual.unpack_dual(t).tangent is not None for t in tensors):
        raise AssertionError("token operators carry no forward-mode derivatives: give them tensors without a tangent")


def _refuse_grad(where: str) -> None:
    if torch.is_grad_enabled():
        raise AssertionError(f"{where} carries no gradient: give it detached tensors, or call it under torch.no_grad()")


# A leaf's gradient is added up on the stream that was current when the first graph of the leaf was made, as long as one is alive.  A backward pass that is
# recorded into a HIP graph would have that stream wait for the recording one, which ends the process: so graphs leave their stream with their leaves.
# (Those that are made here: torch does not tell the stream of a graph that other operations made first.)
_MADE_ON = "stream of the first rotation"


def _is_leaf(node) -> bool:
    # (by name: the type is not to be had without a tensor that wants a gradient, which an import in inference mode cannot make)
    return type(node).__name__ == "AccumulateGrad"


def _mark_leaves(out: torch.Tensor) -> None:
    for node, _ in out.grad_fn.next_functions:
        if _is_leaf(node):
            node.metadata.setdefault(_MADE_ON, _raw_stream(out.get_device()))


def _check_leaves(nodes, need, index: int) -> None:
    here = _raw_stream(index)
    for (node, _), wanted in zip(nodes, need):
        if wanted and _is_leaf(node) and node.metadata.get(_MADE_ON, here) != here:
            raise AssertionError("a backward pass is recorded into a HIP graph while a graph of the same leaves, made on another stream, is alive: drop that one first")


class _Rotation(torch.autograd.Function):
    """Rotary.rotate in a graph: the gradient of a rotation is the rotation back."""

    @staticmethod
    def forward(ctx, rotary, inverse, positions, q, k):
        ctx.rotary, ctx.inverse = rotary, inverse
        ctx.save_for_backward(positions)
        ctx.set_materialize_grads(False)
        out = rotary.rotate(q, positions, k, inverse)
        q_out, k_out = (out, None) if k is None else out
        ctx.mark_non_differentiable(*(y for x, y in ((q, q_out), (k, k_out)) if x is not None and not x.requires_grad))
        return q_out, k_out

    @staticmethod
    def backward(ctx, *grads):
        positions, = ctx.saved_tensors
        if torch.cuda.is_current_stream_capturing():
            _check_leaves(ctx.next_functions, ctx.needs_input_grad[2:], positions.get_device())
        # (a gradient comes in any strides: a sum's is one value, repeated)
        back = [None if g is None else ctx.rotary.rotate(g.contiguous(), positions, inverse=not ctx.inverse) for g in grads]
        return None, None, None, back[0], back[1]


class _NormRotation(torch.autograd.Function):
    """Rotary.norm_rotate in a graph."""

    @staticmethod
    def forward(ctx, rotary, eps, positions, q, q_weight, k, k_weight):
        ctx.rotary, ctx.eps = rotary, eps
        ctx.save_for_backward(positions, q, q_weight, k, k_weight)
        ctx.set_materialize_grads(False)
        out = rotary.norm_rotate(q, positions, q_weight, k, k_weight, eps)
        q_out, k_out = (out, None) if k is None else out
        ctx.mark_non_differentiable(*(y for x, w, y in ((q, q_weight, q_out), (k, k_weight, k_out)) if x is not None and not (x.requires_grad or w.requires_grad)))
        return q_out, k_out

    @staticmethod
    def _gradients(ctx, q_grad, k_grad):
        positions, q, q_weight, k, k_weight = ctx.saved_tensors
        need = ctx.needs_input_grad
        if torch.cuda.is_current_stream_capturing():
            _check_leaves(ctx.next_functions, need[2:], q.get_device())
        return (None, None, None) + ctx.rotary._norm_back(positions, ctx.eps, (q, q_weight, q_grad, need[3], need[4]), (k, k_weight, k_grad, need[5], need[6]))

    # (what refuses gradients of gradients takes 4 us of the host's time: only where there may be some)
    _gradients_once = staticmethod(torch.autograd.function.once_differentiable(_gradients.__func__))

    @staticmethod
    def backward(ctx, q_grad, k_grad):
        return (_NormRotation._gradients_once if torch.is_grad_enabled() else _NormRotation._gradients)(ctx, q_grad, k_grad)


class Rotary:
    """Rotary positions with several axes: pairs[a] pairs of a head turn with a token's position on axis a."""

    def __init__(self, head_dim: int, pairs, base: float = 10000.0, layout: int = CB_PAIRS_HALVES, ladder: int = CB_LADDER_SHARED):
        pairs = [int(n) for n in pairs]
        if len(pairs) > CB_ROTARY_MAX_AXES:
            raise AssertionError(f"{len(pairs)} axes: {CB_ROTARY_MAX_AXES} at most")
        d = cb_rotary_desc()
        d.head_dim, d.n_axes, d.layout, d.ladder, d.base = head_dim, len(pairs), layout, ladder, base
        for a, n in enumerate(pairs):
            d.pairs[a] = n
        self.head_dim, self.n_axes = head_dim, len(pairs)
        self.plan = cb_rotary()
        _check(lib().cb_rotary_init(C.byref(d), C.byref(self.plan)), "cb_rotary_init")
        nbytes = C.c_size_t()
        _check(lib().cb_norm_rotate_back_scratch_bytes(C.byref(self.plan), C.byref(nbytes)), "cb_norm_rotate_back_scratch_bytes")
        self._back_bytes = nbytes.value

    def rotate(self, q: torch.Tensor, positions: torch.Tensor, k: Optional[torch.Tensor] = None, inverse: bool = False,
               q_out: Optional[torch.Tensor] = None, k_out: Optional[torch.Tensor] = None):
        """q (tokens x heads x head_dim) turned by positions (tokens x axes, int32), and k with it: q_out, or (q_out, k_out).
        inverse: turned back, which is also the gradient of q from that of q_out: q and k may be parts of a graph, if their outputs are not
        given.  An output may be its input, and is changed for torch's graphs too: one that has saved it finds out in its backward pass.  Forward-mode
        derivatives are refused, and so is a backward pass that is recorded into a HIP graph while a graph of the same leaves is alive that a rotate or norm_rotate on another
        stream made; of graphs that other operations made there the caller has to take care: torch waits for their stream, which ends the process."""
        if (q.requires_grad or (k is not None and k.requires_grad)) and torch.is_grad_enabled():
            if q_out is not None or k_out is not None:
                raise AssertionError("outputs that are given carry no gradient: rotate without them, or under torch.no_grad()")
            q_out, k_out = _Rotation.apply(self, inverse, positions, q, k)
            _mark_leaves(q_out if q_out.requires_grad else k_out)
            return q_out if k is None else (q_out, k_out)
        if k is None and k_out is not None:
            raise AssertionError("k_out without k")
        if _dual._current_level >= 0:
            _refuse_tangents(q, k, q_out, k_out)
        given = () if q_out is None and k_out is None else _given(q_out, k_out)
        n, dtype, index, dim = q.shape[0], q.dtype, q.get_device(), self.head_dim
        if index < 0 or dtype not in _CB_DT:
            raise AssertionError(f"q: {dtype} on {q.device}; needed: float32 or bfloat16 on a GPU")
        if index != _current_device():
            with torch.cuda.device(index):
                return self.rotate(q, positions, k, inverse, q_out, k_out)
        a, c, d = _heads(q, "q", dtype, index, dim), None, None
        if q_out is None:
            q_out = torch.empty_like(q, memory_format=torch.contiguous_format)
            b = _fresh(q_out, dim)
        else:
            b = _heads(q_out, "q_out", dtype, index, dim, q.shape[1], n)
        if k is not None:
            c = _heads(k, "k", dtype, index, dim, None, n)
            if k_out is None:
                k_out = torch.empty_like(k, memory_format=torch.contiguous_format)
                d = _fresh(k_out, dim)
            else:
                d = _heads(k_out, "k_out", dtype, index, dim, k.shape[1], n)
        status = lib().cb_rotate(C.byref(self.plan), _CB_DT[dtype], n, _dense(positions, "positions", torch.int32, index, (n, self.n_axes)),
                                 a, b, c, d, 1 if inverse else 0, _raw_stream(index))
        if status:
            _check(status, "cb_rotate")
        if given:
            _written(given)
        return q_out if k is None else (q_out, k_out)

    def norm_rotate(self, q: torch.Tensor, positions: torch.Tensor, q_weight: torch.Tensor, k: Optional[torch.Tensor] = None,
                    k_weight: Optional[torch.Tensor] = None, eps: float = 1e-6, q_out: Optional[torch.Tensor] = None, k_out: Optional[torch.Tensor] = None):
        """Every head of q over the root of its mean square (and eps), times q_weight (head_dim values, float32 or bfloat16), turned by positions as by
        rotate; k with it by k_weight: q_out, or (q_out, k_out).  q, k and the weights may be parts of a graph (once: gradients of gradients are
        refused), if their outputs are not given.  An output may be its input, and what is refused in recorded backward
        passes and forward mode is so, as with rotate."""
        if (k is None) != (k_weight is None):
            raise AssertionError("k and k_weight are given together")
        if torch.is_grad_enabled() and (q.requires_grad or q_weight.requires_grad or (k is not None and (k.requires_grad or k_weight.requires_grad))):
            if q_out is not None or k_out is not None:
                raise AssertionError("outputs that are given carry no gradient: norm_rotate without them, or under torch.no_grad()")
            q_out, k_out = _NormRotation.apply(self, eps, positions, q, q_weight, k, k_weight)
            _mark_leaves(q_out if q_out.requires_grad else k_out)
            return q_out if k is None else (q_out, k_out)
        if k is None and k_out is not None:
            raise AssertionError("k_out without k")
        if _dual._current_level >= 0:
            _refuse_tangents(q, q_weight, k, k_weight, q_out, k_out)
        given = () if q_out is None and k_out is None else _given(q_out, k_out)
        n, dtype, index, dim, wdtype = q.shape[0], q.dtype, q.get_device(), self.head_dim, q_weight.dtype
        if index < 0 or dtype not in _CB_DT or wdtype not in _CB_DT:
            raise AssertionError(f"q: {dtype} on {q.device}, q_weight: {wdtype}; needed: float32 or bfloat16 on a GPU")
        if index != _current_device():
            with torch.cuda.device(index):
                return self.norm_rotate(q, positions, q_weight, k, k_weight, eps, q_out, k_out)
        a, c, d, w = _heads(q, "q", dtype, index, dim), None, None, None
        if q_out is None:
            q_out = torch.empty_like(q, memory_format=torch.contiguous_format)
            b = _fresh(q_out, dim)
        else:
            b = _heads(q_out, "q_out", dtype, index, dim, q.shape[1], n)
        if k is not None:
            c, w = _heads(k, "k", dtype, index, dim, None, n), _dense(k_weight, "k_weight", wdtype, index, (dim,))
            if k_out is None:
                k_out = torch.empty_like(k, memory_format=torch.contiguous_format)
                d = _fresh(k_out, dim)
            else:
                d = _heads(k_out, "k_out", dtype, index, dim, k.shape[1], n)
        status = lib().cb_norm_rotate(C.byref(self.plan), _CB_DT[dtype], n, _dense(positions, "positions", torch.int32, index, (n, self.n_axes)), eps, _CB_DT[wdtype],
                                      a, _dense(q_weight, "q_weight", wdtype, index, (dim,)), b, c, w, d, _raw_stream(index))
        if status:
            _check(status, "cb_norm_rotate")
        if given:
            _written(given)
        return q_out if k is None else (q_out, k_out)

    def _norm_back(self, positions, eps, *sides):
        """Gradients of (x, weight) of each side: (x, weight, gradient of the output or None, whether x's is wanted, the weight's)."""
        # (this runs in a thread of its own, where every step takes longer than elsewhere)
        grads, packed, scratch = [], [], None
        dim, index, first, weight = self.head_dim, positions.get_device(), sides[0][0], sides[0][1]
        n, dtype, wdtype = first.shape[0], first.dtype, weight.dtype
        for x, weight, out_grad, of_x, of_weight in sides:
            if x is None or out_grad is None or not (of_x or of_weight):
                grads += (None, None)
                packed.append(None)
                continue
            if not out_grad.is_contiguous():                     # (a gradient comes in any strides)
                out_grad = out_grad.contiguous()
            x_grad = weight_grad = None
            if of_x:
                x_grad = torch.empty_like(x, memory_format=torch.contiguous_format)
            if of_weight:
                weight_grad = torch.empty_like(weight)
                if scratch is None:
                    scratch = positions.new_empty(self._back_bytes // 4)
            packed.append(_heads(x, "x", dtype, index, dim) + _heads(out_grad, "gradient", dtype, index, dim, x.shape[1], n) +
                          (_fresh(x_grad, dim) if of_x else _NO_HEADS) + _pack_two(weight.data_ptr(), weight_grad.data_ptr() if of_weight else 0))
            grads += (x_grad, weight_grad)
        if any(p is not None for p in packed):
            status = lib().cb_norm_rotate_back(C.byref(self.plan), _CB_DT[dtype], n, positions.data_ptr(), eps, _CB_DT[wdtype], packed[0], packed[1],
                                               None if scratch is None else scratch.data_ptr(), self._back_bytes, _raw_stream(index))
            if status:
                _check(status, "cb_norm_rotate_back")
        return tuple(grads)


class TokenCache:
    """A paged key-value cache (cb_cache) over tensors of the caller's, and its scratch buffer.

    k_pages, v_pages: pages x key heads x page_tokens x head_dim; table: sequences x pages of a sequence, int32; lengths:
    sequences, int32; weight (float32) and time (int32): sequences x key heads x capacity, needed to evict.  Pages of torch.float8_e4m3fn hold values in 8 bits
    with k_scale and v_scale (float32: pages x key heads x page_tokens / 16); what comes and goes is float32 or bfloat16 then, call by call.  bounds (pages x key
    heads x 2 x head_dim, of the pages' type, with 8 bits bfloat16): needed to choose pages.  scratch, if
    it is given (caches may share one): dense uint8, 256-byte aligned, scratch_bytes(query heads) long, and zeroed before the first call.  Calls run on
    the current stream; calls that share a cache or a scratch buffer have to be on one stream, or ordered.  A graph that
    has recorded calls needs the object as long as it is replayed: its scratch buffers stay until then.  Calls write the cache's own tensors past torch's
    autograd, which does not notice: what has saved them for a backward pass (other code's attention over the pages, say) has to be through with it before."""

    def __init__(self, k_pages: torch.Tensor, v_pages: torch.Tensor, table: torch.Tensor, lengths: torch.Tensor,
                 weight: Optional[torch.Tensor] = None, time: Optional[torch.Tensor] = None,
                 scratch: Optional[torch.Tensor] = None, k_scale: Optional[torch.Tensor] = None, v_scale: Optional[torch.Tensor] = None,
                 bounds: Optional[torch.Tensor] = None):
        in_bytes = k_pages.dtype == _E4M3
        if not (k_pages.is_cuda and k_pages.dim() == 4 and (k_pages.dtype in _CB_DT or in_bytes) and table.dim() == 2):
            raise AssertionError(f"k_pages: {k_pages.dtype} {tuple(k_pages.shape)} on {k_pages.device}, table: {tuple(table.shape)}; needed: float32, bfloat16 or "
                                 f"float8_e4m3fn (pages, key heads, page_tokens, head_dim) on a GPU, and (sequences, pages of a sequence)")
        if (k_scale is not None) != in_bytes or (v_scale is not None) != in_bytes:
            raise AssertionError(f"k_scale and v_scale belong to pages of float8_e4m3fn, and to no others: these are {k_pages.dtype}")
        n_pages, heads, page, dim = k_pages.shape
        self.n_seq, self.n_kv_heads, self.head_dim, self.capacity = table.shape[0], heads, dim, table.shape[1] * page
        self.device, self.dtype, self._index = k_pages.device, k_pages.dtype, k_pages.get_device()
        self._slots = (self.n_seq, heads, self.capacity)
        i = self._index
        self.desc = d = cb_cache()
        d.n_seq, d.n_kv_heads, d.head_dim, d.page_tokens = self.n_seq, heads, dim, page
        d.max_pages, d.n_pages, d.dtype = table.shape[1], n_pages, CB_E4M3 if in_bytes else _CB_DT[self.dtype]
        d.k_pages_dev = _dense(k_pages, "k_pages", self.dtype, i, k_pages.shape)
        d.v_pages_dev = _dense(v_pages, "v_pages", self.dtype, i, k_pages.shape)
        d.table_dev = _dense(table, "table", torch.int32, i, table.shape)
        d.lengths_dev = _dense(lengths, "lengths", torch.int32, i, (self.n_seq,))
        d.weight_dev = _dense(weight, "weight", torch.float32, i, self._slots)
        d.time_dev = _dense(time, "time", torch.int32, i, self._slots)
        blocks = (n_pages, heads, page // _BYTE_BLOCK)
        d.k_scale_dev, d.v_scale_dev = _dense(k_scale, "k_scale", torch.float32, i, blocks), _dense(v_scale, "v_scale", torch.float32, i, blocks)
        d.bounds_dev = _dense(bounds, "bounds", torch.bfloat16 if in_bytes else self.dtype, i, (n_pages, heads, 2, dim))
        self.k_pages, self.v_pages, self.table, self.lengths, self.weight, self.time = k_pages, v_pages, table, lengths, weight, time
        self.k_scale, self.v_scale, self.bounds = k_scale, v_scale, bounds
        # a structure for each type of what comes and goes (with 8 bits there are two)
        self._descs = {self.dtype: d}
        if in_bytes:
            other = cb_cache.from_buffer_copy(d)
            d.values_dtype, other.values_dtype = CB_BF16, CB_F32
            self._descs = {torch.bfloat16: d, torch.float32: other}
        self._address = C.addressof(d)
        self._addresses = {t: C.addressof(x) for t, x in self._descs.items()}
        self._room = -1                    # query heads that the scratch buffer has room for
        self._outgrown = []                # scratch buffers that graphs and other streams may still use
        self._lse = {}                     # by query heads: what an lse is like
        self._scratch(0, scratch)

    def __reduce_ex__(self, protocol):
        # (copy, deepcopy and pickle come here; the structure would be shared, or hold addresses of another process)
        raise TypeError("a TokenCache is not copied: make another one of tensors, or of copies of them")

    @classmethod
    def create(cls, n_seq: int, n_kv_heads: int, head_dim: int, capacity: int, dtype=torch.bfloat16, page_tokens: int = 64,
               device="cuda", evictable: Optional[bool] = None, bounded: bool = False):
        """An empty cache whose pages belong to the sequences in order.  dtype: float32, bfloat16 or float8_e4m3fn.  evictable: with weight and time (not
        given: where it can be cut back, that is, not in 8 bits); bounded: with bounds, so that pages can be chosen."""
        pages = -(-capacity // page_tokens)
        shape = (n_seq * pages, n_kv_heads, page_tokens, head_dim)
        table = torch.arange(n_seq * pages, dtype=torch.int32, device=device).view(n_seq, pages)
        slots = (n_seq, n_kv_heads, pages * page_tokens)
        in_bytes = dtype == _E4M3
        evictable = not in_bytes if evictable is None else evictable
        if in_bytes and evictable:
            raise AssertionError("a cache in 8 bits is not cut back: evictable has to be left out, or False")
        blocks = shape[:2] + (page_tokens // _BYTE_BLOCK,)
        scales = [torch.ones(blocks, dtype=torch.float32, device=device) if in_bytes else None for _ in range(2)]
        return cls(torch.zeros(shape, dtype=dtype, device=device), torch.zeros(shape, dtype=dtype, device=device), table,
                   torch.zeros(n_seq, dtype=torch.int32, device=device),
                   torch.zeros(slots, dtype=torch.float32, device=device) if evictable else None,
                   torch.zeros(slots, dtype=torch.int32, device=device) if evictable else None, None, *scales,
                   torch.zeros(shape[:2] + (2, head_dim), dtype=torch.bfloat16 if in_bytes else dtype, device=device) if bounded else None)

    def scratch_bytes(self, n_q_heads: int) -> int:
        n = C.c_size_t()
        _check(lib().cb_cache_scratch_bytes(self._address, n_q_heads, C.byref(n)), "cb_cache_scratch_bytes")
        return n.value

    def _scratch(self, n_q_heads: int, given: Optional[torch.Tensor] = None):
        nbytes = self.scratch_bytes(n_q_heads)
        if given is None and self._room >= 0 and self.scratch.numel() >= nbytes:
            given = self.scratch
        if given is None:
            # its counters are cleared once, now: a recorded clearing would only come with the graph's first replay
            if torch.cuda.is_current_stream_capturing():
                raise AssertionError(f"a scratch buffer for {n_q_heads} query heads has to be made before a graph is recorded: attend once before, or give one")
            given = _alloc(nbytes, self.device)
            given.zero_()
            if self._room >= 0:
                self._outgrown.append(self.scratch)
        if not (given.dtype == torch.uint8 and given.device == self.device and given.is_contiguous()):
            raise AssertionError(f"scratch: {given.dtype}, strides {given.stride()}, on {given.device}; needed: dense uint8 on {self.device}")
        self.scratch, self._room = given, n_q_heads
        self.desc.scratch_dev, self.desc.scratch_bytes = given.data_ptr(), given.numel()
        for d in getattr(self, "_descs", {}).values():
            d.scratch_dev, d.scratch_bytes = self.desc.scratch_dev, self.desc.scratch_bytes

    def _values(self, t: torch.Tensor, what: str):
        """Type of what a call brings, and the structure for it."""
        address = self._addresses.get(t.dtype)
        if address is None:
            raise AssertionError(f"{what}: {t.dtype}; needed: {' or '.join(str(x) for x in self._addresses)}")
        return t.dtype, address

    def append(self, k: torch.Tensor, v: torch.Tensor, positions: Optional[torch.Tensor] = None, rotary: Optional[Rotary] = None,
               q: Optional[torch.Tensor] = None, offsets: Optional[torch.Tensor] = None, start: Optional[torch.Tensor] = None,
               q_out: Optional[torch.Tensor] = None) -> Optional[torch.Tensor]:
        """Rows offsets[s] .. offsets[s + 1] - 1 of k and v (without offsets row s) behind the tokens of sequence s, or from
        slot start[s] on; keys rotated if there is a rotary, and q (row for row), which is returned (rows behind the last
        sequence's are not written).  Tensors that want a gradient are refused."""
        if k.requires_grad or v.requires_grad or (q is not None and q.requires_grad):
            _refuse_grad("append")
        if _dual._current_level >= 0:
            _refuse_tangents(k, v, q, q_out)
        given = () if q_out is None else _given(q_out)
        n, i, dim = k.shape[0], self._index, self.head_dim
        if i != _current_device():
            with torch.cuda.device(i):
                return self.append(k, v, positions, rotary, q, offsets, start, q_out)
        dtype, address = self._values(k, "k")
        a = _heads(k, "k", dtype, i, dim, self.n_kv_heads)
        b = _heads(v, "v", dtype, i, dim, self.n_kv_heads, n)
        c = d = None
        if q is not None:
            c = _heads(q, "q", dtype, i, dim, None, n)
            if q_out is None:
                q_out = torch.empty_like(q, memory_format=torch.contiguous_format)
                d = _fresh(q_out, dim)
            else:
                d = _heads(q_out, "q_out", dtype, i, dim, q.shape[1], n)
        elif q_out is not None:
            raise AssertionError("q_out without q")
        status = lib().cb_cache_append(
            address, None if rotary is None else C.byref(rotary.plan), n if n < 2 ** 31 else -1,
            _dense(positions, "positions", torch.int32, i, (n, 1 if rotary is None else rotary.n_axes)),
            _dense(offsets, "offsets", torch.int32, i, (self.n_seq + 1,)), _dense(start, "start", torch.int32, i, (self.n_seq,)),
            a, b, c, d, _raw_stream(i))
        if status:
            _check(status, "cb_cache_append")
        if given:
            _written(given)
        return q_out

    def attend(self, q: torch.Tensor, scale: Optional[float] = None, softcap: float = 0.0, accumulate: bool = False,
               decay: float = 1.0, out: Optional[torch.Tensor] = None, lse: Optional[torch.Tensor] = None, chosen=None):
        """(out, lse) of one query token per sequence (q: sequences x query heads x head_dim).  scale: 1 / sqrt(head_dim) if not
        given.  accumulate: the cache's weight becomes decay * weight + the weights of this call.  chosen: (chosen, count) as choose gives them, to read
        those pages alone (and not to accumulate).  A q that wants a gradient is refused."""
        if q.requires_grad:
            _refuse_grad("attend")
        if _dual._current_level >= 0:
            _refuse_tangents(q, out, lse)
        given = () if out is None and lse is None else _given(out, lse)
        i, dim = self._index, self.head_dim
        if i != _current_device():
            with torch.cuda.device(i):
                return self.attend(q, scale, softcap, accumulate, decay, out, lse, chosen)
        dtype, address = self._values(q, "q")
        a = _heads(q, "q", dtype, i, dim, None, self.n_seq)
        heads = q.shape[1]
        if chosen is not None:
            pages, count = chosen
            pairs = (self.n_seq, self.n_kv_heads)
            if pages.dim() != 3:
                raise AssertionError(f"chosen: {tuple(pages.shape)}; needed: sequences x key heads x budget")
            pages_at = _dense(pages, "chosen", torch.int32, i, pairs + (pages.shape[2],))
            count_at = _dense(count, "count", torch.int32, i, pairs)
        if heads > self._room:
            self._scratch(heads)
        if out is None:
            out = torch.empty_like(q, memory_format=torch.contiguous_format)
            b = _fresh(out, dim)
        else:
            b = _heads(out, "out", dtype, i, dim, heads, self.n_seq)
        if lse is None:
            like = self._lse.get(heads)
            if like is None:
                like = self._lse[heads] = torch.empty((self.n_seq, heads), dtype=torch.float32, device=self.device)
            lse = torch.empty_like(like)
        else:
            _dense(lse, "lse", torch.float32, i, (self.n_seq, heads))
        params = _pack_attend(dim ** -0.5 if scale is None else scale, softcap, decay, 1 if accumulate else 0, 0)
        if chosen is None:
            status = lib().cb_cache_attend(address, params, a, b, lse.data_ptr(), _raw_stream(i))
        else:
            status = lib().cb_cache_attend_chosen(address, params, a, b, lse.data_ptr(), pages_at, count_at, pages.shape[2], _raw_stream(i))
        if status:
            _check(status, "cb_cache_attend" if chosen is None else "cb_cache_attend_chosen")
        if given:
            _written(given)
        return out, lse

    def bound(self, since: Optional[torch.Tensor] = None) -> None:
        """Bring the bounds up to date, of the pages with slots from since[s] (int32; not given: 0) to the last token of sequence s: after an append
        from what it started at, after an eviction all."""
        i = self._index
        if i != _current_device():
            with torch.cuda.device(i):
                return self.bound(since)
        status = lib().cb_cache_bound(self._address, _dense(since, "since", torch.int32, i, (self.n_seq,)), _raw_stream(i))
        if status:
            _check(status, "cb_cache_bound")

    def choose(self, q: torch.Tensor, budget: int, first: int = 0, recent: int = 0):
        """(chosen, count): for every sequence and key head up to `budget` pages that q can matter to most (q as for attend), by the bounds: the
        `first` first and the `recent` last ones, then the highest scores; places in the sequence's table, ascending, -1 behind them, and how many."""
        if q.requires_grad:
            _refuse_grad("choose")
        if _dual._current_level >= 0:
            _refuse_tangents(q)
        i = self._index
        if i != _current_device():
            with torch.cuda.device(i):
                return self.choose(q, budget, first, recent)
        dtype, address = self._values(q, "q")
        a = _heads(q, "q", dtype, i, self.head_dim, None, self.n_seq)
        if not 1 <= budget <= 2 ** 30:
            raise AssertionError(f"budget: {budget}; needed: 1 .. 2^30")
        chosen = torch.empty((self.n_seq, self.n_kv_heads, budget), dtype=torch.int32, device=self.device)
        count = torch.empty((self.n_seq, self.n_kv_heads), dtype=torch.int32, device=self.device)
        status = lib().cb_cache_choose(address, _pack_choose(budget, first, recent, 0), a, chosen.data_ptr(), count.data_ptr(), _raw_stream(i))
        if status:
            _check(status, "cb_cache_choose")
        return chosen, count

    def evict(self, budget: int, window: int = 0, weight: Optional[torch.Tensor] = None, time: Optional[torch.Tensor] = None,
              lengths: Optional[torch.Tensor] = None) -> None:
        """Cut every sequence back to `budget` tokens a key head: those of the newest `window` steps of time, then those with the
        most weight.  weight, time, lengths: what to go by instead of the cache's own, which receive what is left."""
        i = self._index
        if i != _current_device():
            with torch.cuda.device(i):
                return self.evict(budget, window, weight, time, lengths)
        status = lib().cb_cache_evict(self._address, _pack_evict(
            budget, window, _dense(weight, "weight", torch.float32, i, self._slots) or 0,
            _dense(time, "time", torch.int32, i, self._slots) or 0, _dense(lengths, "lengths", torch.int32, i, (self.n_seq,)) or 0),
            _raw_stream(i))
        if status:
            _check(status, "cb_cache_evict")
