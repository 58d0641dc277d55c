"""ctypes binding of libbalancekv.so: argument marshalling only.

Every step of the hot path runs inside the CUDA library; this module converts torch tensors
to device pointers and error codes to exceptions.  There is no CPU fallback: a missing
library or a failing CUDA call raises.
"""
from __future__ import annotations

import ctypes as C
import functools
import os

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libbalancekv.so")
_lib = None

OK, E_INVAL, E_NOMEM, E_STATE, E_CUDA, E_TIMEOUT = 0, -1, -2, -3, -4, -5

EXPORTS = [
    "balancekv_create", "balancekv_destroy", "balancekv_stream_append", "balancekv_stream_append_layer",
    "balancekv_stream_append_layer_host", "balancekv_compress", "balancekv_compress_layer",
    "balancekv_decode_attn", "balancekv_decode_attn_host", "balancekv_cache_load_level",
    "balancekv_cache_view", "balancekv_level_sizes", "balancekv_debug_enable", "balancekv_debug_call",
    "balancekv_stats", "balancekv_strerror", "balancekv_plan_calls", "balancekv_reset",
    "balancekv_profile_enable", "balancekv_profile_sample", "balancekv_profile_read", "balancekv_decode_attn_static",
    "balancekv_stream_step", "balancekv_stream_step_host", "balancekv_stream_append_layer_keys",
    "balancekv_decode_attn_two", "balancekv_decode_attn_merged", "balancekv_stream_append_bucketed",
    "balancekv_stream_append_layer_bucketed", "balancekv_stream_append_layer_preserving", "balancekv_debug_set_status", "balancekv_decode_attn_static_status", "balancekv_debug_scratch_used",
    "balancekv_debug_late_split",
    "balancekv_attn_scored", "balancekv_attn_scored_workspace", "balancekv_cache_evict", "balancekv_cache_evict_workspace",
    "balancekv_decode_attn_prefix", "balancekv_decode_attn_prefix_workspace",
]
PROFILE_CLASSES = ("append", "radii", "gram_walk", "compact", "decode", "bookkeeping")


class BalanceKVError(RuntimeError):
    def __init__(self, code: int, what: str):
        self.code = code
        msg = load().balancekv_strerror(code).decode() if _lib is not None else str(code)
        super().__init__(f"{what}: {msg} ({code})")


class Config(C.Structure):
    """Mirror of ``balancekv_config``."""

    _fields_ = [
        ("n_seqs", C.c_int32), ("n_layers", C.c_int32), ("n_kv_heads", C.c_int32), ("n_q_heads", C.c_int32),
        ("head_dim", C.c_int32), ("dtype", C.c_int32), ("block", C.c_int32), ("levels", C.c_int32),
        ("max_tokens", C.c_int32), ("max_pending", C.c_int32), ("recent_window", C.c_int32),
        ("center_keys", C.c_int32), ("gram_path", C.c_int32), ("decode_splits", C.c_int32),
        ("seed", C.c_uint64), ("delta", C.c_float), ("c_override", C.c_float), ("r_key", C.c_float),
        ("r_value", C.c_float),
    ]


class Stats(C.Structure):
    _fields_ = [(n, C.c_int64) for n in ("tokens_appended", "tokens_stored", "calls_run", "walk_fails",
                                         "device_status", "bytes_resident", "kernels_launched", "walk_kernel",
                                         "decode_kernel")]


def load():
    """Load the shared library (building it with nvcc if it is absent); raises on failure."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(LIB_PATH):
        from . import build as _build

        _build.build()
    lib = C.CDLL(LIB_PATH)
    vp, ci = C.c_void_p, C.c_int
    lib.balancekv_create.argtypes = [C.POINTER(Config), C.POINTER(vp)]
    lib.balancekv_destroy.argtypes = [vp]
    lib.balancekv_stream_append.argtypes = [vp, ci, ci, ci, vp, vp, ci, vp]
    lib.balancekv_stream_append_layer.argtypes = [vp, ci, vp, vp, ci, vp]
    lib.balancekv_stream_append_layer_host.argtypes = [vp, ci, vp, vp, ci, vp]
    lib.balancekv_compress.argtypes = [vp, ci, vp]
    lib.balancekv_compress_layer.argtypes = [vp, ci, ci, vp]
    lib.balancekv_decode_attn.argtypes = [vp, ci, vp, vp, vp]
    lib.balancekv_decode_attn_host.argtypes = [vp, ci, vp, vp, vp]
    lib.balancekv_cache_load_level.argtypes = [vp, ci, ci, vp, vp, vp, ci, vp]
    lib.balancekv_cache_view.argtypes = [vp, ci, ci, ci] + [C.POINTER(vp)] * 4 + [C.POINTER(ci)]
    lib.balancekv_level_sizes.argtypes = [vp, ci, ci, ci, vp]
    lib.balancekv_debug_enable.argtypes = [vp, ci]
    lib.balancekv_debug_call.argtypes = [vp, ci, ci, ci, ci, ci] + [C.POINTER(vp)] * 3 + [C.POINTER(ci)]
    lib.balancekv_stats.argtypes = [vp, C.POINTER(Stats)]
    lib.balancekv_strerror.argtypes = [ci]
    lib.balancekv_strerror.restype = C.c_char_p
    lib.balancekv_plan_calls.argtypes = [ci, ci, ci, vp, ci, vp, ci]
    lib.balancekv_reset.argtypes = [vp, vp]
    lib.balancekv_stream_step.argtypes = [vp, ci, vp, vp, vp, vp, vp]
    lib.balancekv_stream_step_host.argtypes = [vp, ci, vp, vp, vp, vp, vp]
    lib.balancekv_profile_enable.argtypes = [vp, ci]
    lib.balancekv_profile_sample.argtypes = [vp, ci, ci]
    lib.balancekv_stream_append_layer_keys.argtypes = [vp, ci, vp, ci, vp]
    lib.balancekv_decode_attn_two.argtypes = [vp, ci, ci, vp, vp, vp]
    lib.balancekv_decode_attn_merged.argtypes = [vp, vp, ci, vp, ci, vp, vp, vp]
    lib.balancekv_profile_read.argtypes = [vp, vp]
    lib.balancekv_stream_append_bucketed.argtypes = [vp, ci, ci, ci, ci, ci, vp, vp, ci, C.c_float, vp, vp, vp]
    lib.balancekv_stream_append_layer_bucketed.argtypes = [vp, ci, ci, ci, vp, vp, ci, C.c_float, vp, vp, vp]
    lib.balancekv_stream_append_layer_preserving.argtypes = [vp, ci, vp, vp, ci, C.c_float, vp, vp, vp]
    lib.balancekv_decode_attn_static.argtypes = [vp, vp, ci, ci, ci, ci, vp, vp, ci, ci, ci, vp]
    lib.balancekv_decode_attn_static_status.argtypes = [vp, vp]
    lib.balancekv_debug_set_status.argtypes = [vp, ci]
    lib.balancekv_debug_late_split.argtypes = [vp, ci]
    lib.balancekv_debug_scratch_used.argtypes = [vp, C.POINTER(C.c_int64)]
    size, flt = C.c_size_t, C.c_float
    lib.balancekv_attn_scored.argtypes = [vp, vp, vp, ci, ci, vp, vp, ci, ci, ci, ci, vp, vp, ci, flt, vp, size, vp]
    lib.balancekv_attn_scored_workspace.argtypes = [ci] * 7 + [C.POINTER(size)]
    lib.balancekv_cache_evict.argtypes = [vp] * 5 + [ci, ci] + [vp] * 5 + [ci] * 6 + [vp, size, vp]
    lib.balancekv_cache_evict_workspace.argtypes = [ci] * 6 + [C.POINTER(size)]
    lib.balancekv_decode_attn_prefix.argtypes = [vp, vp, vp, ci, vp, vp, vp, ci, vp, vp, ci, ci, ci, ci, ci, vp, size, vp]
    lib.balancekv_decode_attn_prefix_workspace.argtypes = [ci] * 7 + [C.POINTER(size)]
    for name in EXPORTS:
        if name != "balancekv_strerror":
            getattr(lib, name).restype = ci
    _lib = lib
    return lib


def _check(code: int, what: str):
    if code != OK:
        raise BalanceKVError(code, what)


def _stream_ptr(stream):
    """The cudaStream_t as an integer: of a torch stream, a raw one, or (None) the current stream of the current device."""
    if isinstance(stream, int):          # a raw cudaStream_t
        return stream
    if stream is not None:
        return stream.cuda_stream
    import torch

    # torch.cuda.current_stream() builds a stream object: 3.3 us of every call against 0.3 us for the handle alone, which a
    # torch without these two functions, not initialised yet, or forked since, does not give
    if torch.cuda.is_initialized():
        try:
            return torch._C._cuda_getCurrentRawStream(torch._C._cuda_getDevice())
        except AttributeError:
            pass
    return torch.cuda.current_stream().cuda_stream


def _torch_dtype(dtype_code: int):
    import torch

    return torch.bfloat16 if dtype_code == 1 else torch.float32


def plan_calls(block: int, levels: int, recent_window: int, appended_after_event):
    """Host-only bookkeeping of Algorithm 3: list of (event, level, ordinal) per call."""
    import numpy as np

    ev = np.ascontiguousarray(appended_after_event, dtype=np.int32)
    cap = 4 * (int(ev[-1]) // block + 1) + 8 if len(ev) else 8
    out = np.zeros((cap, 3), np.int32)
    n = load().balancekv_plan_calls(block, levels, recent_window, ev.ctypes.data_as(C.c_void_p), len(ev),
                                    out.ctypes.data_as(C.c_void_p), cap)
    _check(min(n, 0), "balancekv_plan_calls")
    assert n <= cap
    return [tuple(int(x) for x in r) for r in out[:n]]


class Context:
    """Owns one ``balancekv_ctx``.  Tensor arguments are CUDA torch tensors of the context's dtype.

    A call with ``stream=`` (a torch stream or a raw cudaStream_t) runs there and waits for no other stream: the caller orders it behind what makes
    its tensors and keeps them until it is over."""

    def __init__(self, n_seqs=1, n_layers=1, n_kv_heads=1, n_q_heads=None, head_dim=128, dtype="bf16", block=1024,
                 levels=2, max_tokens=32768, max_pending=0, recent_window=0, center_keys=0, gram_path=0, seed=0,
                 decode_splits=0, delta=0.0, c_override=0.0, r_key=0.0, r_value=0.0):
        import torch

        if not torch.cuda.is_available():
            raise RuntimeError("balancekv needs a CUDA device; there is no CPU fallback")
        self.lib = load()
        self.cfg = Config(n_seqs, n_layers, n_kv_heads, n_q_heads if n_q_heads else n_kv_heads, head_dim,
                          1 if dtype == "bf16" else 0, block, levels, max_tokens, max_pending, recent_window,
                          center_keys, gram_path, decode_splits, seed, delta, c_override, r_key, r_value)
        self.dtype = _torch_dtype(self.cfg.dtype)
        self._h = C.c_void_p()
        _check(self.lib.balancekv_create(C.byref(self.cfg), C.byref(self._h)), "balancekv_create")

    def close(self):
        if getattr(self, "_h", None) and self._h.value:
            self.lib.balancekv_destroy(self._h)
            self._h = C.c_void_p()

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def _dev(self, t, name):
        if not t.is_cuda or t.dtype != self.dtype or not t.is_contiguous():
            raise ValueError(f"{name}: expected a contiguous CUDA tensor of dtype {self.dtype}")
        return t.data_ptr()

    def stream_append(self, seq, layer, kv_head, K_blk, V_blk, stream=None):
        assert K_blk.shape == V_blk.shape and K_blk.shape[-1] == self.cfg.head_dim
        _check(self.lib.balancekv_stream_append(self._h, seq, layer, kv_head, self._dev(K_blk, "K_blk"),
                                                self._dev(V_blk, "V_blk"), K_blk.shape[0], _stream_ptr(stream)),
               "balancekv_stream_append")

    def stream_append_layer(self, layer, K, V, stream=None):
        c = self.cfg
        assert tuple(K.shape) == tuple(V.shape) and K.shape[0] == c.n_seqs and K.shape[1] == c.n_kv_heads
        assert K.shape[3] == c.head_dim
        _check(self.lib.balancekv_stream_append_layer(self._h, layer, self._dev(K, "K"), self._dev(V, "V"),
                                                      K.shape[2], _stream_ptr(stream)),
               "balancekv_stream_append_layer")

    def stream_append_layer_host(self, layer, K_host, V_host, stream=None):
        c = self.cfg
        assert not K_host.is_cuda and K_host.dtype == self.dtype and K_host.is_contiguous() and V_host.is_contiguous()
        assert tuple(K_host.shape) == tuple(V_host.shape) and K_host.shape[:2] == (c.n_seqs, c.n_kv_heads)
        _check(self.lib.balancekv_stream_append_layer_host(self._h, layer, C.c_void_p(K_host.data_ptr()),
                                                           C.c_void_p(V_host.data_ptr()), K_host.shape[2],
                                                           _stream_ptr(stream)),
               "balancekv_stream_append_layer_host")

    def compress(self, T=None, stream=None):
        _check(self.lib.balancekv_compress(self._h, self.cfg.levels if T is None else T, _stream_ptr(stream)),
               "balancekv_compress")

    def compress_layer(self, layer, T=None, stream=None):
        _check(self.lib.balancekv_compress_layer(self._h, layer, self.cfg.levels if T is None else T,
                                                 _stream_ptr(stream)), "balancekv_compress_layer")

    def decode_attn(self, layer, q, out=None, stream=None):
        import torch

        c = self.cfg
        assert tuple(q.shape) == (c.n_seqs, c.n_q_heads, c.head_dim)
        if out is None:
            out = torch.empty_like(q)
        _check(self.lib.balancekv_decode_attn(self._h, layer, self._dev(q, "q"), self._dev(out, "out"),
                                              _stream_ptr(stream)), "balancekv_decode_attn")
        return out

    def stream_step(self, layer, q, k_new, v_new, out, stream=None):
        """Append one token per stream of the layer and decode: q, out [B, Hq, d]; k_new, v_new [B, H, d]."""
        _check(self.lib.balancekv_stream_step(self._h, layer, self._dev(q, "q"), self._dev(k_new, "k_new"),
                                              self._dev(v_new, "v_new"), self._dev(out, "out"), _stream_ptr(stream)),
               "balancekv_stream_step")
        return out

    def stream_append_layer_keys(self, layer, K, stream=None):
        """Denominator instance of Algorithm 1: append (k_j, 1); K [B, H, n, d] on the device."""
        _check(self.lib.balancekv_stream_append_layer_keys(self._h, layer, self._dev(K, "K"), K.shape[2],
                                                           _stream_ptr(stream)), "balancekv_stream_append_layer_keys")

    def stream_append_layer_bucketed(self, layer0, n_buckets, i_top, K, V, erase_ratio=0.0, want_slots=False,
                                     stream=None):
        """Algorithm 1's bucketing step for every stream of a layer: K, V [B, H, n, d] on the device;
        slot layer0 + b receives the rows with 2^(i_top-b-1) < ||v|| <= 2^(i_top-b).  Returns the
        per-stream counts [B*H, n_buckets + 1] (last column: dropped rows) and, if asked, the int8
        slot of every row [B, H, n]."""
        import numpy as np
        import torch

        assert K.shape == V.shape and K.dim() == 4
        counts = np.zeros((K.shape[0] * K.shape[1], n_buckets + 1), np.int32)
        slots = torch.empty(K.shape[:3], dtype=torch.int8, device=K.device) if want_slots else None
        _check(self.lib.balancekv_stream_append_layer_bucketed(
            self._h, layer0, n_buckets, i_top, self._dev(K, "K"), self._dev(V, "V"), K.shape[2], float(erase_ratio),
            slots.data_ptr() if want_slots else None, counts.ctypes.data, _stream_ptr(stream)),
            "balancekv_stream_append_layer_bucketed")
        return (counts, slots) if want_slots else counts

    def stream_append_layer_preserving(self, layer0, K, V, tau, want_slots=False, stream=None):
        """Section 4.3's augmented variant: rows whose key has cosine <= tau with the block's mean key go to slot
        layer0 (kept exactly), the rest to slot layer0 + 1.  Returns counts [B*H, 3] (preserved, rest, dropped)
        and, if asked, the int8 slot of every row [B, H, n]."""
        import numpy as np
        import torch

        assert K.shape == V.shape and K.dim() == 4
        counts = np.zeros((K.shape[0] * K.shape[1], 3), np.int32)
        slots = torch.empty(K.shape[:3], dtype=torch.int8, device=K.device) if want_slots else None
        _check(self.lib.balancekv_stream_append_layer_preserving(
            self._h, layer0, self._dev(K, "K"), self._dev(V, "V"), K.shape[2], float(tau),
            slots.data_ptr() if want_slots else None, counts.ctypes.data, _stream_ptr(stream)),
            "balancekv_stream_append_layer_preserving")
        return (counts, slots) if want_slots else counts

    def stream_append_bucketed(self, seq, layer0, n_buckets, i_top, kv_head, K, V, erase_ratio=0.0, want_slots=False,
                               stream=None):
        """Same for one stream: K, V [n, d] on the device."""
        import numpy as np
        import torch

        assert K.shape == V.shape and K.dim() == 2
        counts = np.zeros((1, n_buckets + 1), np.int32)
        slots = torch.empty(K.shape[0], dtype=torch.int8, device=K.device) if want_slots else None
        _check(self.lib.balancekv_stream_append_bucketed(
            self._h, seq, layer0, n_buckets, i_top, kv_head, self._dev(K, "K"), self._dev(V, "V"), K.shape[0],
            float(erase_ratio), slots.data_ptr() if want_slots else None, counts.ctypes.data, _stream_ptr(stream)),
            "balancekv_stream_append_bucketed")
        return (counts[0], slots) if want_slots else counts[0]

    def decode_attn_two(self, layer_num, layer_den, q, out=None, stream=None):
        """Algorithm 1's output ratio: numerator from slot layer_num, denominator from slot layer_den."""
        import torch

        if out is None:
            out = torch.empty_like(q)
        _check(self.lib.balancekv_decode_attn_two(self._h, layer_num, layer_den, self._dev(q, "q"), self._dev(out, "out"),
                                                  _stream_ptr(stream)), "balancekv_decode_attn_two")
        return out

    def decode_attn_merged(self, layers_num, layers_den, q, out=None, stream=None):
        """Value sums of the slots layers_num over weight sums of the slots layers_den (see balancekv.h)."""
        import torch

        if out is None:
            out = torch.empty_like(q)
        ln = (C.c_int32 * len(layers_num))(*layers_num)
        ld = (C.c_int32 * len(layers_den))(*layers_den)
        _check(self.lib.balancekv_decode_attn_merged(self._h, ln, len(layers_num), ld, len(layers_den), self._dev(q, "q"),
                                                     self._dev(out, "out"), _stream_ptr(stream)), "balancekv_decode_attn_merged")
        return out

    def stream_step_host(self, layer, q_host, k_host, v_host, out_host, stream=None):
        _check(self.lib.balancekv_stream_step_host(self._h, layer, q_host.data_ptr(),
                                                   k_host.data_ptr(), v_host.data_ptr(),
                                                   out_host.data_ptr(), _stream_ptr(stream)),
               "balancekv_stream_step_host")
        return out_host

    def decode_attn_host(self, layer, q_host, out_host, stream=None):
        assert not q_host.is_cuda and not out_host.is_cuda and q_host.dtype == self.dtype
        _check(self.lib.balancekv_decode_attn_host(self._h, layer, q_host.data_ptr(),
                                                   out_host.data_ptr(), _stream_ptr(stream)),
               "balancekv_decode_attn_host")
        return out_host

    def cache_load_level(self, layer, level, K, V, orig_idx=None, stream=None):
        import torch

        idx_p = None
        if orig_idx is not None:
            assert orig_idx.is_cuda and orig_idx.dtype == torch.int32 and orig_idx.is_contiguous()
            idx_p = C.c_void_p(orig_idx.data_ptr())
        _check(self.lib.balancekv_cache_load_level(self._h, layer, level, self._dev(K, "K"), self._dev(V, "V"),
                                                   idx_p, K.shape[2], _stream_ptr(stream)),
               "balancekv_cache_load_level")

    def level_sizes(self, seq, layer, kv_head):
        import numpy as np

        s = np.zeros(self.cfg.levels + 1, np.int32)
        _check(self.lib.balancekv_level_sizes(self._h, seq, layer, kv_head, s.ctypes.data_as(C.c_void_p)),
               "balancekv_level_sizes")
        return s

    def cache_view(self, seq, layer, kv_head):
        """Copies of the stream's weighted set as torch tensors: K, V [len,d], w [len], idx [len]."""
        import torch

        pk, pv, pw, pi = C.c_void_p(), C.c_void_p(), C.c_void_p(), C.c_void_p()
        n = C.c_int()
        _check(self.lib.balancekv_cache_view(self._h, seq, layer, kv_head, C.byref(pk), C.byref(pv), C.byref(pw),
                                             C.byref(pi), C.byref(n)), "balancekv_cache_view")
        n = n.value
        d = self.cfg.head_dim
        K = _from_ptr(pk.value, (n, d), self.dtype)
        V = _from_ptr(pv.value, (n, d), self.dtype)
        w = _from_ptr(pw.value, (n,), torch.float32)
        idx = _from_ptr(pi.value, (n,), torch.int32)
        return K, V, w, idx

    def debug_enable(self, on=True):
        _check(self.lib.balancekv_debug_enable(self._h, 1 if on else 0), "balancekv_debug_enable")

    def debug_call(self, seq, layer, kv_head, level, ordinal):
        import torch

        pe, ps, pp = C.c_void_p(), C.c_void_p(), C.c_void_p()
        m = C.c_int()
        _check(self.lib.balancekv_debug_call(self._h, seq, layer, kv_head, level, ordinal, C.byref(pe), C.byref(ps),
                                             C.byref(pp), C.byref(m)), "balancekv_debug_call")
        torch.cuda.synchronize()
        return (_from_ptr(pe.value, (m.value,), torch.int8), _from_ptr(ps.value, (m.value,), torch.float32),
                _from_ptr(pp.value, (m.value,), torch.float32))

    def debug_scratch_used(self) -> int:
        """Words of the split-K decode scratch that are not empty (0 between launches)."""
        n = C.c_int64(0)
        _check(self.lib.balancekv_debug_scratch_used(self._h, C.byref(n)), "balancekv_debug_scratch_used")
        return int(n.value)

    def debug_late_split(self, missing):
        """Testing aid: combine a head whose split ``missing`` (-1: none) arrives after the bounded wait has run out."""
        _check(self.lib.balancekv_debug_late_split(self._h, int(missing)), "balancekv_debug_late_split")

    def debug_set_status(self, value):
        """Testing aid: overwrite the device status word (1 = a bounded wait gave up)."""
        _check(self.lib.balancekv_debug_set_status(self._h, int(value)), "balancekv_debug_set_status")

    def reset(self, stream=None):
        _check(self.lib.balancekv_reset(self._h, _stream_ptr(stream)), "balancekv_reset")

    def profile_enable(self, on=True, classes=None):
        """Time every kernel class, or only the named ones (see PROFILE_CLASSES)."""
        flag = 1 if on else 0
        if on and classes is not None:
            flag = sum(2 << PROFILE_CLASSES.index(n) for n in classes)
        _check(self.lib.balancekv_profile_enable(self._h, flag), "balancekv_profile_enable")

    def profile_sample(self, kernel_class, every):
        """Time only every `every`-th launch of one class (name from PROFILE_CLASSES)."""
        _check(self.lib.balancekv_profile_sample(self._h, PROFILE_CLASSES.index(kernel_class), int(every)),
               "balancekv_profile_sample")

    def profile_read(self):
        """{class name: (launches, total ms)} since the last read."""
        buf = (C.c_double * (2 * len(PROFILE_CLASSES)))()
        _check(self.lib.balancekv_profile_read(self._h, buf), "balancekv_profile_read")
        return {n: (int(buf[2 * i]), float(buf[2 * i + 1])) for i, n in enumerate(PROFILE_CLASSES)}

    def stats(self):
        s = Stats()
        code = self.lib.balancekv_stats(self._h, C.byref(s))
        if code != E_TIMEOUT:               # a timed-out wait is reported through device_status; the record is filled
            _check(code, "balancekv_stats")
        return {n: getattr(s, n) for n, _ in Stats._fields_}


def decode_attn_static(K, V, n_heavy, level, q, out=None, stream=None):
    """Allocation-free decode attention over caller-owned caches (see balancekv.h).

    K, V: CUDA tensors [n_streams, cache_len, d]; q: [n_streams, group, d]; the first
    ``n_heavy`` rows of every stream weigh 2**level, the rest 1.  ``out`` must be supplied by
    callers that may not allocate; when it is None a tensor is created for convenience."""
    import torch

    assert K.is_cuda and V.is_cuda and q.is_cuda and K.is_contiguous() and V.is_contiguous() and q.is_contiguous()
    assert K.shape == V.shape and K.dtype == V.dtype == q.dtype and q.shape[0] == K.shape[0] and q.shape[2] == K.shape[2]
    if out is None:
        out = torch.empty_like(q)
    dtype_code = 1 if K.dtype == torch.bfloat16 else {torch.float32: 0}[K.dtype]
    _check(load().balancekv_decode_attn_static(K.data_ptr(), V.data_ptr(), K.shape[0],
                                               K.shape[1], n_heavy, level, q.data_ptr(),
                                               out.data_ptr(), q.shape[1], K.shape[2], dtype_code,
                                               _stream_ptr(stream)), "balancekv_decode_attn_static")
    return out


def decode_attn_static_status(stream=None):
    """Status word of the allocation-free entry point on the current device: 0, or 1 if a bounded
    wait of one of its launches gave up since the last read (reading clears it).  Synchronises the stream."""
    v = C.c_int(0)
    _check(load().balancekv_decode_attn_static_status(C.byref(v), _stream_ptr(stream)), "balancekv_decode_attn_static_status")
    return v.value


def _is(t, dtype, shape, device):
    """A contiguous tensor of this dtype and shape on CUDA device number ``device``, or None."""
    return t is None or (t.dtype is dtype and t.shape == shape and t.get_device() == device and t.is_contiguous())


def _expect(what, device, **tensors):
    """Says which of the tensors (each with its dtype and shape) is not what it should be."""
    for name, (t, dtype, shape) in tensors.items():
        if t is None:
            continue
        if t.dtype is not dtype or t.shape != shape:
            raise ValueError(f"{what}: {name}: expected dtype {dtype} and shape {tuple(shape)}, got {t.dtype} and {tuple(t.shape)}")
        if t.get_device() != device or not t.is_contiguous():
            raise ValueError(f"{what}: {name}: expected a contiguous tensor on the device of the first")


def _on_current(what, device, t):
    """The call runs on a stream of the current CUDA device, which has to be the tensors'."""
    if device < 0 or device != _torch()._C._cuda_getDevice():
        raise ValueError(f"{what}: the tensors are on {t.device}, not on the current CUDA device")


def _torch():
    global _torch_module
    if _torch_module is None:
        import torch

        _torch_module = torch
    return _torch_module


_torch_module = None


def _dtype_code(what, dtype):
    torch = _torch()
    if dtype is torch.bfloat16:
        return 1
    if dtype is torch.float32:
        return 0
    raise ValueError(f"{what}: dtype {dtype} is neither torch.bfloat16 nor torch.float32")


def _ptr(t):
    return None if t is None else t.data_ptr()


def _on_stream(stream, call, *tensors, **more):
    """A call on a stream other than the current one.  Tensors made inside belong to that stream, and those given are recorded on it, so that the
    memory of neither is handed on while the call still runs.  (A raw stream, or torch's ExternalStream of one, may be gone by the time that a
    tensor's memory is freed: there the caller keeps the tensors.)"""
    torch = _torch()
    raw = isinstance(stream, (int, torch.cuda.ExternalStream))
    if isinstance(stream, int):
        stream = torch.cuda.ExternalStream(stream) if stream else torch.cuda.default_stream()
    with torch.cuda.stream(stream):
        result = call(*tensors, **more)
    if not raw:
        out = more.get("out")
        for t in (*tensors, *more.values(), *(out.values() if isinstance(out, dict) else ())):
            if isinstance(t, torch.Tensor):
                t.record_stream(stream)
    return result


@functools.lru_cache(maxsize=1024)
def _workspace_bytes(name, *sizes):
    """What ``name``_workspace asks for: a function of the sizes alone."""
    size = C.c_size_t(0)
    _check(getattr(load(), name + "_workspace")(*sizes, C.byref(size)), name + "_workspace")
    return size.value


def _workspace(device, size):
    torch = _torch()
    return torch.empty(size, dtype=torch.uint8, device=device) if size else None


def _in_32_bits(what, *numbers):
    """ctypes would cut the upper bits off."""
    for n in numbers:
        if not -(1 << 31) <= n < 1 << 31:
            raise ValueError(f"{what}: {n} does not fit 32 bits")


def attn_scored(K, V, q, lens=None, score=None, score_out=None, n_scored=None, decay=1.0, out=None, stream=None):
    """Attention of every stream's newest tokens over its cache, and the weight that each cached row receives (see balancekv.h).

    K, V: CUDA tensors [n_streams, capacity, d]; q: [n_streams, group, n_queries, d] or, for one query, [n_streams, group, d];
    lens: int32 [n_streams], rows in use (None: all).  The newest ``n_scored`` queries (None: all) add their weights to ``decay`` times
    ``score`` (float32 [n_streams, capacity]; None: zeros); the result goes to ``score_out``, by default ``score`` itself or a
    new tensor of zeros.  Returns (out, score_out); with n_scored = 0 the second is ``score_out`` as it was.

    ``stream``: a torch stream or a raw cudaStream_t to run on in place of the current one.  The call does not wait for other streams: the caller orders
    it behind what makes its tensors, and what uses its results behind it.  The tensors given may be let go once a call on a torch stream has
    returned; for a raw one (an ExternalStream too) the caller keeps them until it is over.  (The same holds for cache_evict and decode_attn_prefix.)"""
    if stream is not None:
        return _on_stream(stream, attn_scored, K, V, q, lens, score, score_out, n_scored=n_scored, decay=decay, out=out)
    what, torch = "balancekv_attn_scored", _torch()
    ks, qs = K.shape, q.shape
    if len(ks) != 3 or len(qs) not in (3, 4):
        raise ValueError(f"{what}: expected K [n_streams, capacity, d] and q [n_streams, group, (n_queries,) d]")
    (S, cap, d), group, m = ks, qs[1], qs[2] if len(qs) == 4 else 1
    dtype, device, ss, f32 = K.dtype, K.get_device(), (S, cap), torch.float32
    code = _dtype_code(what, dtype)
    if n_scored is None:
        n_scored = m
    _in_32_bits(what, n_scored)
    if not (qs[0] == S and qs[-1] == d and _is(K, dtype, ks, device) and _is(V, dtype, ks, device) and _is(q, dtype, qs, device) and _is(out, dtype, qs, device)
            and _is(lens, torch.int32, (S,), device) and _is(score, f32, ss, device) and _is(score_out, f32, ss, device)):
        _expect(what, device, K=(K, dtype, ks), V=(V, dtype, ks), q=(q, dtype, (S, *qs[1:-1], d)), out=(out, dtype, qs), lens=(lens, torch.int32, (S,)),
                score=(score, f32, ss), score_out=(score_out, f32, ss))
    _on_current(what, device, K)
    if out is None:
        out = torch.empty_like(q)
    if score_out is None and n_scored:
        score_out = torch.zeros(S, cap, device=K.device) if score is None else score
    size = _workspace_bytes(what, S, cap, m, group, d, code, n_scored)
    ws = _workspace(K.device, size)
    _check(load().balancekv_attn_scored(K.data_ptr(), V.data_ptr(), _ptr(lens), S, cap, q.data_ptr(), out.data_ptr(), m, group, d, code,
                                        _ptr(score), _ptr(score_out), n_scored, decay, _ptr(ws), size, _stream_ptr(None)), what)
    return out, score_out


def cache_evict(K, V, score, n_keep, lens=None, pos=None, n_first=0, n_recent=0, out=None, in_place=False, stream=None):
    """Keep the ``n_keep`` rows of every stream that received the most weight, and the first and newest positions (see balancekv.h).

    K, V: CUDA tensors [n_streams, capacity, d]; score: float32, pos (None: the rows' numbers): int32, both [n_streams, capacity];
    lens: int32 [n_streams] (None: all rows are in use).  ``out``: a dict of "k", "v", "score" and, if they are wanted, "pos" and "lens" to
    fill, by default new tensors of min(n_keep, capacity) rows whose unused ones are zero; with ``in_place`` the cache itself, of which only
    the rows that fill a hole move (``pos`` and ``lens`` are updated if given, ``lens`` is made if not).  Returns that dict."""
    if stream is not None:
        return _on_stream(stream, cache_evict, K, V, score, n_keep, lens, pos, n_first=n_first, n_recent=n_recent, out=out, in_place=in_place)
    what, torch = "balancekv_cache_evict", _torch()
    ks = K.shape
    if len(ks) != 3:
        raise ValueError(f"{what}: expected K [n_streams, capacity, d]")
    _in_32_bits(what, n_keep, n_first, n_recent)
    S, cap, d = ks
    dtype, device, ss, i32, f32 = K.dtype, K.get_device(), (S, cap), torch.int32, torch.float32
    code = _dtype_code(what, dtype)
    if not (score is not None and _is(K, dtype, ks, device) and _is(V, dtype, ks, device) and _is(score, f32, ss, device) and _is(pos, i32, ss, device)
            and _is(lens, i32, (S,), device)):
        _expect(what, device, K=(K, dtype, ks), V=(V, dtype, ks), score=(score, f32, ss), pos=(pos, i32, ss), lens=(lens, i32, (S,)))
    _on_current(what, device, K)
    if in_place:
        if out is not None:
            raise ValueError(f"{what}: either out or in_place")
        out = {"k": K, "v": V, "score": score, "pos": pos, "lens": torch.empty(S, dtype=i32, device=K.device) if lens is None else lens}
        Ko, Vo, so, po, lo, rows = K, V, score, pos, out["lens"], cap
    else:
        if out is None:
            rows = min(n_keep, cap)
            if rows < 1:
                raise ValueError(f"{what}: n_keep and the capacity are at least 1")
            out = {"k": K.new_zeros(S, rows, d), "v": V.new_zeros(S, rows, d), "score": score.new_zeros(S, rows),
                   "pos": torch.zeros(S, rows, dtype=i32, device=K.device), "lens": torch.empty(S, dtype=i32, device=K.device)}
        Ko, Vo, so, po, lo = out["k"], out["v"], out["score"], out.get("pos"), out.get("lens")
        rows = Ko.shape[1] if Ko.dim() == 3 else 0
        os = (S, rows)
        if not (_is(Ko, dtype, (S, rows, d), device) and _is(Vo, dtype, (S, rows, d), device) and _is(so, f32, os, device) and _is(po, i32, os, device)
                and _is(lo, i32, (S,), device)):
            _expect(what, device, out_k=(Ko, dtype, (S, rows, d)), out_v=(Vo, dtype, (S, rows, d)), out_score=(so, f32, os), out_pos=(po, i32, os),
                    out_lens=(lo, i32, (S,)))
    k, ko = K.data_ptr(), Ko.data_ptr()
    size = _workspace_bytes(what, S, cap, n_keep, d, code, int(ko == k))
    ws = _workspace(K.device, size)
    _check(load().balancekv_cache_evict(k, V.data_ptr(), _ptr(score), _ptr(pos), _ptr(lens), S, cap, ko, Vo.data_ptr(), _ptr(so), _ptr(po), _ptr(lo), rows,
                                        n_keep, n_first, n_recent, d, code, _ptr(ws), size, _stream_ptr(None)), what)
    return out


def decode_attn_prefix(K_prefix, V_prefix, K, V, q, lens=None, weight=None, out=None, stream=None):
    """Decode attention of a batch over a shared prefix and every sequence's own rows (see balancekv.h).

    K_prefix, V_prefix: CUDA tensors [n_kv_heads, prefix_len, d]; weight: float32 [n_kv_heads, prefix_len] (None: ones);
    K, V: [n_seqs, n_kv_heads, capacity, d], or None where the sequences have no rows of their own; lens: int32 [n_seqs] (None: all rows
    are in use); q: [n_seqs, n_kv_heads * group, d]."""
    if stream is not None:
        return _on_stream(stream, decode_attn_prefix, K_prefix, V_prefix, K, V, q, lens, weight, out=out)
    what, torch = "balancekv_decode_attn_prefix", _torch()
    ps, qs = K_prefix.shape, q.shape
    if len(ps) != 3 or len(qs) != 3 or (K is None) != (V is None) or (K is not None and K.dim() != 4):
        raise ValueError(f"{what}: expected K_prefix [n_kv_heads, prefix_len, d], K [n_seqs, n_kv_heads, capacity, d] and q [n_seqs, n_q_heads, d]")
    (H, P, d), (B, Hq, _), cap = ps, qs, 0 if K is None else K.shape[2]
    if H < 1 or Hq % H:
        raise ValueError(f"{what}: {Hq} query heads do not share {H} KV heads")
    dtype, device, ks, f32 = K_prefix.dtype, K_prefix.get_device(), (B, H, cap, d), torch.float32
    code = _dtype_code(what, dtype)
    if not (qs[2] == d and _is(K_prefix, dtype, ps, device) and _is(V_prefix, dtype, ps, device) and _is(K, dtype, ks, device) and _is(V, dtype, ks, device)
            and _is(q, dtype, qs, device) and _is(out, dtype, qs, device) and _is(weight, f32, (H, P), device) and _is(lens, torch.int32, (B,), device)):
        _expect(what, device, K_prefix=(K_prefix, dtype, ps), V_prefix=(V_prefix, dtype, ps), K=(K, dtype, ks), V=(V, dtype, ks), q=(q, dtype, (B, Hq, d)),
                out=(out, dtype, qs), weight=(weight, f32, (H, P)), lens=(lens, torch.int32, (B,)))
    _on_current(what, device, K_prefix)
    if out is None:
        out = torch.empty_like(q)
    size = _workspace_bytes(what, P, cap, B, H, Hq // H, d, code)
    ws = _workspace(q.device, size)
    _check(load().balancekv_decode_attn_prefix(K_prefix.data_ptr(), V_prefix.data_ptr(), _ptr(weight), P, _ptr(K), _ptr(V), _ptr(lens), cap,
                                               q.data_ptr(), out.data_ptr(), B, H, Hq // H, d, code, _ptr(ws), size, _stream_ptr(None)), what)
    return out


class _RawDevice:
    def __init__(self, ptr, shape, typestr):
        self.__cuda_array_interface__ = {"data": (ptr, False), "shape": tuple(shape), "typestr": typestr,
                                         "version": 2}


def _from_ptr(ptr, shape, dtype):
    """Copy ``shape`` elements of ``dtype`` from a raw device pointer into a new torch tensor."""
    import torch

    n = 1
    for s in shape:
        n *= s
    if n == 0 or not ptr:
        return torch.empty(shape, dtype=dtype, device="cuda")
    typestr = {torch.float32: "<f4", torch.int32: "<i4", torch.int8: "|i1", torch.bfloat16: "<i2"}[dtype]
    raw = torch.as_tensor(_RawDevice(ptr, shape, typestr), device="cuda")
    if dtype == torch.bfloat16:
        raw = raw.view(torch.bfloat16)
    out = raw.clone()
    torch.cuda.synchronize()
    return out
