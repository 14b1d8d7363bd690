"""Thin ctypes binding of the C ABI in include/lazyev.h.

Argument marshalling only: every step of the decode path runs in the HIP library.  torch is
used for device memory and the stream.  Importing this module fails if the library has not
been built (python -m paper_2506_15969_amd.build); there is no fallback path.
"""
from __future__ import annotations

import ctypes as C
import os

import torch

# (LAZYEV_LIBRARY names another build of the same library in lib/, e.g. the instrumented
# liblazyev_timeline.so that bench.py --timeline measures with)
_LIB_PATH = os.path.join(os.path.dirname(os.path.abspath(__file__)), "lib",
                         os.path.basename(os.environ.get("LAZYEV_LIBRARY", "liblazyev.so")))
if not os.path.exists(_LIB_PATH):
    raise ImportError("liblazyev.so is not built: run `python -m paper_2506_15969_amd.build` "
                      "(expected at %s)" % _LIB_PATH)
lib = C.CDLL(_LIB_PATH)

OK, EINVAL, ECAPACITY, EWORKSPACE, EHIP, ENOMEM, ESCRATCH, EEXCHANGE = 0, -1, -2, -3, -4, -5, -6, -7
DTYPE_FP32, DTYPE_BF16 = 0, 1
SCORE_H1, SCORE_H2 = 1, 2
SCORE_H2_DECREASING = 16
SCORE_CURRENT_ATTENTION = 32
MAX_HIST_BINS = 8192
LDS_CANDIDATES = 8192
ROPE_NONE, ROPE_HALVES, ROPE_PAIRS = 0, 1, 2


class Config(C.Structure):
    _fields_ = [("n_layers", C.c_int32), ("batch", C.c_int32), ("n_q_heads", C.c_int32),
                ("n_kv_heads", C.c_int32), ("head_dim", C.c_int32), ("budget", C.c_int32),
                ("window", C.c_int32), ("prompt_len", C.c_int32), ("alpha", C.c_float),
                ("softmax_scale", C.c_float), ("dtype", C.c_int32), ("score_flags", C.c_int32),
                ("k_cache", C.c_void_p), ("v_cache", C.c_void_p), ("ts", C.c_void_p),
                ("mri", C.c_void_p), ("pos", C.c_void_p), ("workspace", C.c_void_p),
                ("workspace_bytes", C.c_size_t), ("stream", C.c_void_p)]


class Stats(C.Structure):
    _fields_ = [("n_layers", C.c_int32), ("len", C.POINTER(C.c_int32)),
                ("last_step", C.POINTER(C.c_int32)), ("n_evict_events", C.POINTER(C.c_int64)),
                ("n_evicted", C.POINTER(C.c_int64)), ("n_activations", C.POINTER(C.c_int64)),
                ("n_rows_moved", C.POINTER(C.c_int64))]


class Heads(C.Structure):
    _fields_ = [("rows", C.c_void_p), ("to", C.c_void_p), ("seq_stride", C.c_int64),
                ("token_stride", C.c_int64), ("head_stride", C.c_int64), ("to_seq_stride", C.c_int64),
                ("to_token_stride", C.c_int64), ("to_head_stride", C.c_int64),
                ("weight", C.c_void_p), ("n_heads", C.c_int32)]


class Rotation(C.Structure):
    _fields_ = [("layout", C.c_int32), ("dims", C.c_int32), ("inv_freq", C.c_void_p), ("eps", C.c_float)]


class Pages(C.Structure):
    _fields_ = [("n_kv_heads", C.c_int32), ("head_dim", C.c_int32), ("dtype", C.c_int32),
                ("n_pages", C.c_int32), ("page_size", C.c_int32), ("n_seqs", C.c_int32),
                ("table_stride", C.c_int32), ("k_pages", C.c_void_p), ("v_pages", C.c_void_p),
                ("table", C.c_void_p)]


# what include/lazyev.h declares (the contract) ...
EXPORTS = ["lazyev_capacity", "lazyev_workspace_size", "lazyev_init", "lazyev_decode_step",
           "lazyev_prefill_track", "lazyev_prefill_track_seq", "lazyev_evict", "lazyev_evict_all",
           "lazyev_evict_static", "lazyev_stats", "lazyev_admit", "lazyev_retire",
           "lazyev_cached_before_step", "lazyev_mri_histogram", "lazyev_window_from_histogram",
           "lazyev_score_pairs", "lazyev_norm_rope", "lazyev_pages_append", "lazyev_pages_attend",
           "lazyev_pages_attend_workspace", "lazyev_decode_step_shared", "lazyev_destroy", "lazyev_strerror", "lazyev_last_hip_error"]
# ... and include/lazyev_bench.h (knobs and the per-kernel timer in the same library; the plain
# streaming probes in liblazyev_bench.so, loaded by bench_lib() when somebody measures)
BENCH_EXPORTS = ["lazyev_set_chunk", "lazyev_set_target_blocks", "lazyev_set_variant", "lazyev_set_spin_ticks",
                 "lazyev_profile_arm", "lazyev_profile_read", "lazyev_log_words", "lazyev_log_peek"]
BENCH_LIB_EXPORTS = ["lazyev_stream_probe", "lazyev_stream_read_probe", "lazyev_event_overhead"]
_BENCH_LIB_PATH = os.path.join(os.path.dirname(_LIB_PATH), "liblazyev_bench.so")
_bench_lib = None


def bench_lib():
    """liblazyev_bench.so (plain streaming probes, event-pair cost), loaded on first use."""
    global _bench_lib
    if _bench_lib is None:
        if not os.path.exists(_BENCH_LIB_PATH):
            raise ImportError("liblazyev_bench.so is not built: run `python -m paper_2506_15969_amd.build`")
        b = C.CDLL(_BENCH_LIB_PATH)
        b.lazyev_stream_probe.restype = C.c_int
        b.lazyev_stream_probe.argtypes = [C.c_void_p, C.c_void_p, C.c_size_t, C.c_int32, C.c_void_p]
        b.lazyev_stream_read_probe.restype = C.c_int
        b.lazyev_stream_read_probe.argtypes = [C.c_void_p, C.c_size_t, C.c_int32, C.c_void_p, C.c_void_p]
        b.lazyev_event_overhead.restype = C.c_int
        b.lazyev_event_overhead.argtypes = [C.c_int32, C.c_void_p, C.POINTER(C.c_double)]
        _bench_lib = b
    return _bench_lib


lib.lazyev_capacity.restype = C.c_int32
lib.lazyev_capacity.argtypes = [C.POINTER(Config)]
lib.lazyev_workspace_size.restype = C.c_size_t
lib.lazyev_workspace_size.argtypes = [C.POINTER(Config)]
lib.lazyev_init.restype = C.c_int
lib.lazyev_init.argtypes = [C.POINTER(Config), C.POINTER(C.c_void_p)]
lib.lazyev_prefill_track.restype = C.c_int
lib.lazyev_prefill_track.argtypes = [C.c_void_p, C.c_int32, C.c_void_p, C.c_void_p, C.c_void_p]
lib.lazyev_prefill_track_seq.restype = C.c_int
lib.lazyev_prefill_track_seq.argtypes = [C.c_void_p, C.c_int32, C.c_int32, C.c_void_p, C.c_void_p, C.c_void_p]
lib.lazyev_decode_step.restype = C.c_int
lib.lazyev_decode_step.argtypes = [C.c_void_p, C.c_int32, C.c_int32, C.c_void_p, C.c_void_p,
                                   C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p]
lib.lazyev_evict.restype = C.c_int
lib.lazyev_evict.argtypes = [C.c_void_p, C.c_int32, C.c_int32, C.POINTER(C.c_int32)]
lib.lazyev_evict_all.restype = C.c_int
lib.lazyev_evict_all.argtypes = [C.c_void_p, C.c_int32, C.POINTER(C.c_int32)]
lib.lazyev_evict_static.restype = C.c_int
lib.lazyev_evict_static.argtypes = [C.c_void_p, C.c_int32, C.c_int32, C.POINTER(C.c_int32)]
lib.lazyev_window_from_histogram.restype = C.c_int
lib.lazyev_window_from_histogram.argtypes = [C.POINTER(C.c_int64), C.c_int32, C.c_double, C.POINTER(C.c_int32)]
lib.lazyev_stats.restype = C.c_int
lib.lazyev_stats.argtypes = [C.c_void_p, C.POINTER(Stats)]
lib.lazyev_admit.restype = C.c_int
lib.lazyev_admit.argtypes = [C.c_void_p, C.c_int32, C.c_int32, C.c_int32]
lib.lazyev_retire.restype = C.c_int
lib.lazyev_cached_before_step.restype = C.c_int32
lib.lazyev_cached_before_step.argtypes = [C.c_int32] * 4
lib.lazyev_retire.argtypes = [C.c_void_p, C.c_int32]
lib.lazyev_mri_histogram.restype = C.c_int
lib.lazyev_mri_histogram.argtypes = [C.c_void_p, C.c_int32, C.c_int32, C.POINTER(C.c_int64)]
lib.lazyev_score_pairs.restype = C.c_int
lib.lazyev_score_pairs.argtypes = [C.c_void_p, C.c_void_p, C.c_void_p, C.c_int64, C.c_int32,
                                   C.c_void_p]
lib.lazyev_norm_rope.restype = C.c_int
lib.lazyev_norm_rope.argtypes = [C.c_int32, C.c_int32, C.c_int32, C.c_int32, C.POINTER(Heads), C.POINTER(Heads),
                                 C.POINTER(Rotation), C.c_void_p, C.c_int32, C.c_void_p]
lib.lazyev_pages_append.restype = C.c_int
lib.lazyev_pages_append.argtypes = [C.POINTER(Pages), C.c_int32, C.c_int32, C.POINTER(Heads), C.POINTER(Heads),
                                    C.POINTER(Rotation), C.c_int32, C.c_void_p]
lib.lazyev_pages_attend_workspace.restype = C.c_size_t
lib.lazyev_pages_attend_workspace.argtypes = [C.POINTER(Pages), C.c_int32, C.c_int32, C.c_int32]
lib.lazyev_pages_attend.restype = C.c_int
lib.lazyev_pages_attend.argtypes = [C.POINTER(Pages), C.c_int32, C.c_int32, C.c_int32, C.c_void_p, C.c_void_p,
                                    C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p, C.c_float, C.c_void_p,
                                    C.c_size_t, C.c_void_p]
lib.lazyev_decode_step_shared.restype = C.c_int
lib.lazyev_decode_step_shared.argtypes = [C.c_void_p, C.c_int32, C.c_int32, C.c_void_p, C.c_void_p, C.c_void_p,
                                          C.c_void_p, C.POINTER(Pages), C.c_int32, C.c_void_p, C.c_size_t,
                                          C.c_void_p, C.c_void_p]
lib.lazyev_set_chunk.restype = C.c_int
lib.lazyev_set_chunk.argtypes = [C.c_void_p, C.c_int32]
lib.lazyev_set_target_blocks.restype = C.c_int
lib.lazyev_set_target_blocks.argtypes = [C.c_void_p, C.c_int32]
lib.lazyev_set_variant.restype = C.c_int
lib.lazyev_set_variant.argtypes = [C.c_void_p, C.c_int32]
lib.lazyev_set_spin_ticks.restype = C.c_int
lib.lazyev_set_spin_ticks.argtypes = [C.c_void_p, C.c_uint32]
lib.lazyev_profile_arm.restype = C.c_int
lib.lazyev_profile_arm.argtypes = [C.c_void_p, C.c_int32]
lib.lazyev_log_words.restype = C.c_int32
lib.lazyev_log_words.argtypes = [C.c_void_p]
lib.lazyev_log_peek.restype = C.c_int
lib.lazyev_log_peek.argtypes = [C.c_void_p, C.c_int32, C.c_int32, C.c_int32, C.POINTER(C.c_uint32), C.POINTER(C.c_int32)]
lib.lazyev_profile_read.restype = C.c_int
lib.lazyev_profile_read.argtypes = [C.c_void_p, C.POINTER(C.c_double), C.POINTER(C.c_int64)]
lib.lazyev_destroy.restype = None
lib.lazyev_destroy.argtypes = [C.c_void_p]
lib.lazyev_strerror.restype = C.c_char_p
lib.lazyev_strerror.argtypes = [C.c_int]
lib.lazyev_last_hip_error.restype = C.c_int
lib.lazyev_last_hip_error.argtypes = [C.c_void_p]


class LazyevError(RuntimeError):
    def __init__(self, code: int, where: str):
        self.code = code
        super().__init__("%s: %s (code %d)" % (where, lib.lazyev_strerror(code).decode(), code))


def _check(code: int, where: str):
    if code != OK:
        raise LazyevError(code, where)


def _ptr(t):
    return None if t is None else C.c_void_p(t.data_ptr())


def score_pairs(delta_t: torch.Tensor, mri: torch.Tensor, score_flags: int = SCORE_H1 | SCORE_H2):
    """lazyev_score_pairs on int32 device tensors; returns a float64 device tensor."""
    assert delta_t.is_cuda and mri.is_cuda and delta_t.dtype == torch.int32 and mri.dtype == torch.int32
    delta_t, mri = delta_t.contiguous(), mri.contiguous()
    out = torch.empty(delta_t.numel(), dtype=torch.float64, device=delta_t.device)
    stream = torch.cuda.current_stream(delta_t.device).cuda_stream
    _check(lib.lazyev_score_pairs(_ptr(delta_t), _ptr(mri), _ptr(out), delta_t.numel(),
                                  score_flags, C.c_void_p(stream)), "lazyev_score_pairs")
    return out.view(delta_t.shape)


def window_from_histogram(hist, quantile: float = 0.8) -> int:
    """lazyev_window_from_histogram on a sequence of counts (host only)."""
    n = len(hist)
    arr = (C.c_int64 * n)(*[int(x) for x in hist])
    w = C.c_int32(0)
    _check(lib.lazyev_window_from_histogram(arr, n, quantile, C.byref(w)), "lazyev_window_from_histogram")
    return w.value


_DTYPES = {torch.float32: DTYPE_FP32, torch.bfloat16: DTYPE_BF16}


def _need(ok, what: str):
    if not ok:
        raise ValueError(what)


# (torch.cuda.current_stream(device).cuda_stream without the Stream object around it: 0.1 instead of 1.9 us)
_raw_stream = torch._C._cuda_getCurrentRawStream


def _launch(device, call, *args):
    """call(*args, the device's current stream) with the device as the current one: a launch and its stream belong to it."""
    index = device.index
    if index == torch.cuda.current_device():
        return call(*args, _raw_stream(index))
    with torch.cuda.device(device):
        return call(*args, _raw_stream(index))


class NormRope:
    """Norms of the query and key heads of a layer and the rotation by the token's position (lazyev_norm_rope).  For serving, as everything
    here: results carry no gradients, whether the inputs ask for them or not.

    q_weight, k_weight [head_dim] of the rows' type, or None: not normed.  inv_freq [dims / 2] fp32, or None: not
    rotated; layout ROPE_HALVES (elements j and j + dims / 2 form a pair) or ROPE_PAIRS (2 j and 2 j + 1).
    """

    def __init__(self, head_dim, dtype=torch.bfloat16, q_weight=None, k_weight=None, eps=1e-6, inv_freq=None,
                 layout=ROPE_HALVES):
        _need(dtype in _DTYPES and head_dim in (64, 128), "rows of 64 or 128 elements, fp32 or bf16")
        self.device = None
        for w in (q_weight, k_weight):
            _need(w is None or (w.dtype == dtype and w.shape == (head_dim,) and w.is_contiguous()),
                  "a norm's weight is [head_dim], contiguous, of the rows' type")
        _need(inv_freq is None or (inv_freq.dtype == torch.float32 and inv_freq.dim() == 1 and inv_freq.is_contiguous()),
              "inv_freq is [dims / 2], contiguous, fp32")
        for x in (q_weight, k_weight, inv_freq):
            if x is None:
                continue
            _need(x.is_cuda and self.device in (None, x.device), "weights and frequencies are on one GPU")
            self.device = x.device
        dims = 0 if inv_freq is None else 2 * inv_freq.numel()
        _need(inv_freq is None or (dims >= 16 and dims % 16 == 0 and dims <= head_dim and layout in (ROPE_HALVES, ROPE_PAIRS)),
              "rotated elements: a multiple of 16, at most head_dim")
        self.head_dim, self.dtype = head_dim, dtype
        self.q_weight, self.k_weight, self.inv_freq = q_weight, k_weight, inv_freq
        self.rotation = Rotation(ROPE_NONE if inv_freq is None else layout, dims, 0 if inv_freq is None else inv_freq.data_ptr(), eps)

    def heads(self, x, to, weight):
        """lazyev_heads of x [S,n,H,d] or [n,H,d] (any strides, the last one 1) with its result at `to` (the same shape)."""
        shape, a, b = x.shape, x.stride(), to.stride()
        if (x.dtype is not self.dtype or to.dtype is not self.dtype or to.shape != shape or len(shape) not in (3, 4) or
                shape[-1] != self.head_dim or not x.is_cuda or (a[-1] != 1 or b[-1] != 1) and x.numel() != 0):
            raise ValueError("heads are [S, n, H, head_dim] or [n, H, head_dim] of the rows' type on a GPU, their elements side by side")
        device = x.device
        if to.device != device or self.device is not None and self.device != device:
            raise ValueError("one GPU for everything in a call")
        w = None if weight is None else weight.data_ptr()
        if len(shape) == 3:
            return Heads(x.data_ptr(), to.data_ptr(), 0, a[0], a[1], 0, b[0], b[1], w, shape[1])
        return Heads(x.data_ptr(), to.data_ptr(), a[0], a[1], a[2], b[0], b[1], b[2], w, shape[2])

    def __call__(self, q=None, k=None, positions=None, start=0, q_out=None, k_out=None):
        """q, k [S,n,H,d] or [n,H,d] (either may be None) -> (q_out, k_out), new tensors where none are given (in place:
        the same tensor).  positions int32 [S,n] or [n]: token i is at start + positions[i]; None: at start + i."""
        first = q if q is not None else k
        _need(first is not None, "queries, keys or both")
        hq = hk = None
        if q is not None:
            if q_out is None:
                q_out = torch.empty_like(q, memory_format=torch.contiguous_format)
            hq = self.heads(q, q_out, self.q_weight)
        if k is not None:
            if k_out is None:
                k_out = torch.empty_like(k, memory_format=torch.contiguous_format)
            hk = self.heads(k, k_out, self.k_weight)
        shape, device, at = first.shape, first.device, None
        n_seqs, n_tokens = (1, shape[0]) if len(shape) == 3 else (shape[0], shape[1])
        if hk is not None and hq is not None:
            _need(k.shape[:-2] == shape[:-2] and k.device == device, "queries and keys of the same tokens")
        if positions is not None:
            _need(positions.dtype is torch.int32 and positions.shape == shape[:-2] and positions.is_contiguous() and
                  positions.device == device, "positions are int32, one for each token, contiguous, on the rows' GPU")
            at = positions.data_ptr()
        _need(-1 << 31 <= start < 1 << 31, "start is a 32-bit number")
        code = _launch(device, lib.lazyev_norm_rope, n_seqs, n_tokens, self.head_dim, _DTYPES[self.dtype], hq, hk, self.rotation, at,
                       start)
        _check(code, "lazyev_norm_rope")
        return q_out, k_out


class PagedCache:
    """Keys and values of one layer in pages: k_pages, v_pages [n_pages,Hkv,page_size,d] and table [S,m] int32 (entry i of row s is
    place i % page_size of page table[s, i // page_size]), all the caller's tensors.  A layer's caches of a LazyEviction are such
    pages too: PagedCache(eng.k_cache[l], eng.v_cache[l], table) with one page per sequence, a page number = a sequence.  Results carry no gradients."""

    def __init__(self, k_pages, v_pages, table, n_q_heads=None):
        for x in (k_pages, v_pages):
            _need(x.is_cuda and x.dtype in _DTYPES and x.dim() == 4 and x.is_contiguous() and x.shape == k_pages.shape and
                  x.dtype == k_pages.dtype and x.device == k_pages.device and x.numel() > 0,
                  "pages are [n_pages, Hkv, page_size, head_dim], contiguous, fp32 or bf16, on a GPU")
        _need(table.dtype == torch.int32 and table.dim() == 2 and table.numel() > 0 and table.device == k_pages.device and
              table.stride(1) == 1 and (table.shape[0] == 1 or table.shape[1] <= table.stride(0) < 1 << 31),
              "the table is [S, pages of a row], int32, rows side by side, on the pages' GPU")
        n_pages, heads, page_size, d = k_pages.shape
        _need(d in (64, 128), "rows of 64 or 128 elements")
        self.k_pages, self.v_pages, self.table = k_pages, v_pages, table
        self.n_q_heads, self.device, self.dtype = n_q_heads, k_pages.device, k_pages.dtype
        self.entries = min(table.shape[1] * page_size, 1 << 30)   # of a row: entries have 32-bit numbers
        self.pages = Pages(heads, d, _DTYPES[self.dtype], n_pages, page_size, table.shape[0],
                           table.stride(0) if table.shape[0] > 1 else table.shape[1], k_pages.data_ptr(), v_pages.data_ptr(), table.data_ptr())

    def append(self, start, k, v, rope=None, position0=None):
        """lazyev_pages_append: k, v [S,n,Hkv,d] (or [n,Hkv,d] of a single row; any strides, the last one 1) become the entries
        start .. start + n - 1, the keys normed and rotated by `rope` (a NormRope, None: as they are) on the way, token i by
        the position position0 + i (None: its entry's number)."""
        pg = self.pages
        if rope is None:
            rope = NormRope(pg.head_dim, self.dtype)
        _need(rope.dtype is self.dtype and rope.head_dim == pg.head_dim, "the rotation's rows are the pages'")
        shape = k.shape
        _need((len(shape) == 4 and shape[0] == pg.n_seqs or len(shape) == 3 and pg.n_seqs == 1) and shape[-2] == pg.n_kv_heads and
              v.shape == shape and k.device == self.device and v.device == self.device,
              "keys and values are [S, n, Hkv, head_dim] of the table's rows")
        n = shape[-3]
        _need(0 <= start and start + n <= self.entries, "entries beyond the table's row")
        if position0 is None:
            position0 = start
        _need(-1 << 31 <= position0 < 1 << 31, "position0 is a 32-bit number")
        hk, hv = rope.heads(k, k, rope.k_weight), rope.heads(v, v, None)
        code = _launch(self.device, lib.lazyev_pages_append, pg, start, n, hk, hv, rope.rotation, position0)
        _check(code, "lazyev_pages_append")

    def workspace_bytes(self, length, n_tokens, n_q_heads=None) -> int:
        _need(0 <= length <= self.entries, "entries beyond the table's row")
        return lib.lazyev_pages_attend_workspace(self.pages, length, n_tokens, n_q_heads or self.n_q_heads or self.pages.n_kv_heads)

    def attend(self, length, q, visible=None, joined=None, out=None, lse=None, scale=0.0, workspace=None):
        """lazyev_pages_attend: q [S,n,Hq,d] (or [n,Hq,d] of a single row) over the first `length` entries -> (out like q,
        lse [S,n,Hq] fp32).  visible int32 [S,n]: entries that a token sees (None: all).  joined: (out, lse) of the same queries
        over other entries, to be joined.  workspace: uint8, at least workspace_bytes(length, n) (None: allocated)."""
        pg, shape, device = self.pages, q.shape, self.device
        _need(q.dtype is self.dtype and (len(shape) == 4 and shape[0] == pg.n_seqs or len(shape) == 3 and pg.n_seqs == 1) and
              shape[-1] == pg.head_dim and q.is_contiguous() and q.device == device,
              "queries are [S, n, Hq, head_dim] of the table's rows, contiguous, of the pages' type, on their GPU")
        n, n_q_heads, rows = shape[-3], shape[-2], shape[:-1]
        _need(self.n_q_heads in (None, n_q_heads), "another number of query heads")
        _need(0 <= length <= self.entries, "entries beyond the table's row")
        if out is None:
            out = torch.empty_like(q)
        else:
            _need(out.shape == shape and out.dtype is q.dtype and out.is_contiguous() and out.device == device, "out is like q")
        if lse is None:
            lse = q.new_empty(rows, dtype=torch.float32)
        other = []
        for o, l in ((None, lse),) if joined is None else ((None, lse), joined):
            _need((o is None or o.shape == shape and o.dtype is q.dtype and o.is_contiguous() and o.device == device) and
                  l.shape == rows and l.dtype is torch.float32 and l.is_contiguous() and l.device == device,
                  "outputs are like q, log-sum-exps fp32, one for each row of q")
            other = [None if o is None else o.data_ptr(), l.data_ptr()]
        seen = None
        if visible is not None:
            _need(visible.dtype is torch.int32 and visible.shape == shape[:-2] and visible.is_contiguous() and visible.device == device,
                  "visible is int32, one for each token, contiguous, on the pages' GPU")
            seen = visible.data_ptr()
        workspace, n_bytes = self._workspace(length, n, n_q_heads, workspace)
        code = _launch(device, lib.lazyev_pages_attend, pg, length, n, n_q_heads, seen, q.data_ptr(), other[0],
                       None if joined is None else other[1], out.data_ptr(), lse.data_ptr(), scale,
                       None if workspace is None else workspace.data_ptr(), n_bytes)
        _check(code, "lazyev_pages_attend")
        return out, lse

    def _workspace(self, length, n_tokens, n_q_heads, given):
        """(workspace, its bytes) for a call: the given one, or one from torch's allocator for the current stream."""
        _need(-1 << 31 <= length < 1 << 31, "a length is a 32-bit number")
        if given is not None:
            _need(given.dtype == torch.uint8 and given.is_contiguous() and given.device == self.device, "a workspace is bytes on the pages' GPU")
            return given, given.numel()
        n = lib.lazyev_pages_attend_workspace(self.pages, length, n_tokens, n_q_heads)
        return (self.k_pages.new_empty(n, dtype=torch.uint8), n) if n else (None, 0)


class LazyEviction:
    """Owns the device buffers (as torch tensors) and a library context for them.

    k_cache / v_cache [L,S,Hkv,C,d], ts / mri / pos [L,S,Hkv,C] are attributes; fill the prompt
    rows with `load_prompt` (or write them directly) BEFORE `init()`.
    """

    def __init__(self, n_layers, batch, n_q_heads, n_kv_heads, head_dim, budget, window,
                 prompt_len, alpha, dtype=torch.bfloat16, softmax_scale=0.0,
                 score_flags=SCORE_H1 | SCORE_H2, device="cuda:0", stream=None):
        if not torch.cuda.is_available():
            raise RuntimeError("lazyev needs a GPU: no CPU fallback exists")
        self.device = torch.device(device)
        self.dtype = dtype
        self.cfg = Config(n_layers=n_layers, batch=batch, n_q_heads=n_q_heads,
                          n_kv_heads=n_kv_heads, head_dim=head_dim, budget=budget, window=window,
                          prompt_len=prompt_len, alpha=alpha, softmax_scale=softmax_scale,
                          dtype=DTYPE_FP32 if dtype == torch.float32 else DTYPE_BF16,
                          score_flags=score_flags)
        cap = lib.lazyev_capacity(C.byref(self.cfg))
        if cap <= 0:
            raise LazyevError(EINVAL, "lazyev_capacity")
        self.capacity = cap
        L, S, H, d = n_layers, batch, n_kv_heads, head_dim
        self.k_cache = torch.zeros((L, S, H, cap, d), dtype=dtype, device=self.device)
        self.v_cache = torch.zeros((L, S, H, cap, d), dtype=dtype, device=self.device)
        self.ts = torch.zeros((L, S, H, cap), dtype=torch.int32, device=self.device)
        self.mri = torch.zeros((L, S, H, cap), dtype=torch.int32, device=self.device)
        self.pos = torch.zeros((L, S, H, cap), dtype=torch.int32, device=self.device)
        ws_bytes = lib.lazyev_workspace_size(C.byref(self.cfg))
        self.workspace = torch.zeros(ws_bytes, dtype=torch.uint8, device=self.device)
        self.stream = stream if stream is not None else torch.cuda.current_stream(self.device)
        self.cfg.k_cache, self.cfg.v_cache = self.k_cache.data_ptr(), self.v_cache.data_ptr()
        self.cfg.ts, self.cfg.mri, self.cfg.pos = (self.ts.data_ptr(), self.mri.data_ptr(),
                                                  self.pos.data_ptr())
        self.cfg.workspace, self.cfg.workspace_bytes = self.workspace.data_ptr(), ws_bytes
        self.cfg.stream = self.stream.cuda_stream
        self._ctx = C.c_void_p()

    def load_prompt(self, layer: int, k: torch.Tensor, v: torch.Tensor):
        """k, v [S,Hkv,P,d] -> entries 0..P-1 of the layer."""
        P = self.cfg.prompt_len
        self.k_cache[layer, :, :, :P].copy_(k)
        self.v_cache[layer, :, :, :P].copy_(v)

    def init(self):
        if self._ctx:
            lib.lazyev_destroy(self._ctx)
            self._ctx = C.c_void_p()
        _check(lib.lazyev_init(C.byref(self.cfg), C.byref(self._ctx)), "lazyev_init")
        return self

    def set_chunk(self, chunk: int):
        _check(lib.lazyev_set_chunk(self._ctx, chunk), "lazyev_set_chunk")

    def decode_step(self, layer, t, q, k_new, v_new, out, p_out=None, p_override=None):
        code = lib.lazyev_decode_step(self._ctx, layer, t, q.data_ptr(), k_new.data_ptr(),
                                      v_new.data_ptr(), out.data_ptr(), _ptr(p_out),
                                      _ptr(p_override))
        if code != OK:
            raise LazyevError(code, "lazyev_decode_step")

    def decode_step_shared(self, layer, t, q, k_new, v_new, out, prefix, prefix_len, p_out=None, p_override=None,
                           workspace=None):
        """lazyev_decode_step_shared: decode_step over the first prefix_len entries of `prefix` (a PagedCache of one
        table row) and the sequences' own caches."""
        cfg = self.cfg
        _need(prefix.k_pages.get_device() == self.k_cache.get_device(), "the prefix is on the context's GPU")
        with torch.cuda.stream(self.stream):
            workspace, n_bytes = prefix._workspace(prefix_len, cfg.batch, cfg.n_q_heads, workspace)
            code = lib.lazyev_decode_step_shared(self._ctx, layer, t, q.data_ptr(), k_new.data_ptr(), v_new.data_ptr(),
                                                 out.data_ptr(), prefix.pages, prefix_len, _ptr(workspace), n_bytes,
                                                 _ptr(p_out), _ptr(p_override))
        if code != OK:
            raise LazyevError(code, "lazyev_decode_step_shared")

    def prefill_track(self, layer, q_prompt, p_out=None, p_override=None):
        """lazyev_prefill_track.  q_prompt [S,P,Hq,d]; p_out / p_override [S,Hq,P,P] fp32."""
        code = lib.lazyev_prefill_track(self._ctx, layer, q_prompt.data_ptr(), _ptr(p_out), _ptr(p_override))
        if code != OK:
            raise LazyevError(code, "lazyev_prefill_track")

    def prefill_track_seq(self, layer, seq, q_prompt, p_out=None, p_override=None):
        """lazyev_prefill_track_seq.  q_prompt [P,Hq,d]; p_out / p_override [Hq,P,P] fp32."""
        code = lib.lazyev_prefill_track_seq(self._ctx, layer, seq, q_prompt.data_ptr(), _ptr(p_out),
                                            _ptr(p_override))
        if code != OK:
            raise LazyevError(code, "lazyev_prefill_track_seq")

    def evict(self, layer, t) -> int:
        n = C.c_int32(0)
        code = lib.lazyev_evict(self._ctx, layer, t, C.byref(n))
        if code != OK:
            raise LazyevError(code, "lazyev_evict")
        return n.value

    def evict_static(self, layer, t) -> int:
        """lazyev_evict_static: lazyev_evict with the gather list in the library's own static
        device array instead of the workspace."""
        n = C.c_int32(0)
        code = lib.lazyev_evict_static(self._ctx, layer, t, C.byref(n))
        if code != OK:
            raise LazyevError(code, "lazyev_evict_static")
        return n.value

    def evict_all(self, t) -> int:
        """lazyev_evict_all: the eviction check of every layer after step t."""
        n = C.c_int32(0)
        code = lib.lazyev_evict_all(self._ctx, t, C.byref(n))
        if code != OK:
            raise LazyevError(code, "lazyev_evict_all")
        return n.value

    def stats(self) -> dict:
        L = self.cfg.n_layers
        a32 = lambda: (C.c_int32 * L)()
        a64 = lambda: (C.c_int64 * L)()
        bufs = dict(len=a32(), last_step=a32(), n_evict_events=a64(), n_evicted=a64(),
                    n_activations=a64(), n_rows_moved=a64())
        st = Stats(n_layers=L, **{k: C.cast(v, C.POINTER(C.c_int32 if k in ("len", "last_step")
                                                         else C.c_int64)) for k, v in bufs.items()})
        _check(lib.lazyev_stats(self._ctx, C.byref(st)), "lazyev_stats")
        return {k: list(v) for k, v in bufs.items()}

    def admit(self, seq: int, prompt_len: int, t0: int, k=None, v=None):
        """lazyev_admit.  k, v [L,Hkv,prompt_len,d] (optional): the prompt rows, copied into the
        slot's units of every layer first."""
        if k is not None:
            self.k_cache[:, seq, :, :prompt_len].copy_(k)
            self.v_cache[:, seq, :, :prompt_len].copy_(v)
        _check(lib.lazyev_admit(self._ctx, seq, prompt_len, t0), "lazyev_admit")

    def retire(self, seq: int):
        _check(lib.lazyev_retire(self._ctx, seq), "lazyev_retire")

    def mri_histogram(self, layer: int = -1, n_bins: int = MAX_HIST_BINS):
        """lazyev_mri_histogram: counts of cached entries by MRI (last bin: MRI >= n_bins - 1)
        over the units of `layer` (-1: all layers), as a list of ints."""
        hist = (C.c_int64 * n_bins)()
        _check(lib.lazyev_mri_histogram(self._ctx, layer, n_bins, hist), "lazyev_mri_histogram")
        return list(hist)

    def set_target_blocks(self, n_blocks: int):
        _check(lib.lazyev_set_target_blocks(self._ctx, n_blocks), "lazyev_set_target_blocks")

    def set_variant(self, variant: int):
        _check(lib.lazyev_set_variant(self._ctx, variant), "lazyev_set_variant")

    def set_spin_ticks(self, ticks: int):
        _check(lib.lazyev_set_spin_ticks(self._ctx, ticks), "lazyev_set_spin_ticks")

    def log_peek(self, layer: int, units, back: int = 0):
        """lazyev_log_peek for the (sequence, kv_head) pairs in `units`: (step, bool array
        [len(units), 32 * log_words]) of a logged call, or None if the layer has no such call in
        its activation log."""
        import numpy as np
        words = lib.lazyev_log_words(self._ctx)
        if words <= 0:
            return None
        buf = (C.c_uint32 * words)()
        t = C.c_int32(0)
        rows = []
        for (seq, kvh) in units:
            if lib.lazyev_log_peek(self._ctx, layer, back, seq * self.cfg.n_kv_heads + kvh, buf, C.byref(t)) != 0:
                return None
            a = np.frombuffer(buf, dtype=np.uint32).copy()
            rows.append(np.unpackbits(a.view(np.uint8), bitorder="little").astype(bool))
        return t.value, np.stack(rows)

    def profile_arm(self, n_calls: int):
        _check(lib.lazyev_profile_arm(self._ctx, n_calls), "lazyev_profile_arm")

    def profile_read(self) -> dict:
        """{kernel: (total ms, launches)} of the armed calls since the last read."""
        ms, n = (C.c_double * 4)(), (C.c_int64 * 4)()
        _check(lib.lazyev_profile_read(self._ctx, ms, n), "lazyev_profile_read")
        names = ("split", "combine", "select", "move")
        return {k: (ms[i], n[i]) for i, k in enumerate(names)}

    def close(self):
        if self._ctx:
            lib.lazyev_destroy(self._ctx)
            self._ctx = C.c_void_p()

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass
