"""ctypes binding of the C ABI in include/rd.h.  Argument marshalling only: every step of the path
runs inside the CUDA library.  There is no CPU fallback: a missing or unloadable library raises."""
from __future__ import annotations

import ctypes as C
import os

import numpy as np

HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(HERE, "librd_b200.so")

RD_F32, RD_BF16 = 0, 1
RD_OK, RD_E_INVALID_ARG, RD_E_STATE, RD_E_CAPACITY, RD_E_OOM, RD_E_CUDA, RD_E_TIMEOUT = 0, -1, -2, -3, -4, -5, -6
RD_DBG_LATENTS, RD_DBG_DELTA, RD_DBG_DRAFTS, RD_DBG_LOGITS, RD_DBG_EMBED = 0, 1, 2, 3, 4

EXPORTS = ["rd_load", "rd_free", "rd_session_create", "rd_session_destroy", "rd_prefill", "rd_ar_step",
           "rd_df_step", "rd_sync", "rd_committed", "rd_get_tokens", "rd_last_step_rows", "rd_debug_read",
           "rd_debug_force_tokens", "rd_debug_read_kv", "rd_stats", "rd_set_gemm_path", "rd_strerror",
           "rd_last_cuda_error", "rd_profile_enable", "rd_profile_read", "rd_debug_read_kv_noalloc", "rd_set_launch_chaining",
           "rd_debug_expire_next_wait", "rd_set_fused_swiglu", "rd_set_attention_path", "rd_poll_begin", "rd_poll_end",
           "rd_debug_gemm_sequence", "rd_prefill_sliced", "rd_prefill_advance", "rd_prefill_pending",
           "rd_set_prefill_units", "rd_paged_create", "rd_paged_destroy", "rd_paged_pages", "rd_paged_append", "rd_paged_attend",
           "rd_paged_sync", "rd_session_create_paged", "rd_session_release"]


class RdConfig(C.Structure):
    _fields_ = [(n, C.c_int32) for n in ("hidden", "n_heads", "head_dim", "mlp_inner", "n_prelude", "n_core",
                                         "n_coda", "vocab", "dtype", "tie_embeddings")] + \
               [(n, C.c_float) for n in ("rope_base", "norm_eps", "init_sigma")]


class RdSessionConfig(C.Structure):
    _fields_ = [(n, C.c_int32) for n in ("batch", "max_context", "max_window", "max_iters_per_pos",
                                         "max_new_tokens", "keep_logits")] + \
               [("temperature", C.c_float), ("seed", C.c_uint64), ("eta", C.c_float), ("beta", C.c_float),
                ("top_p", C.c_float), ("latent_slots", C.c_int32)]


class RdPagedConfig(C.Structure):
    _fields_ = [(n, C.c_int32) for n in ("n_heads", "n_kv_heads", "head_dim", "dtype", "page_size", "n_pages", "n_layers",
                                         "max_context", "max_rows")] + [("rope_base", C.c_float)]


class RdPagedRows(C.Structure):
    _fields_ = [("n_rows", C.c_int32), ("n_groups", C.c_int32), ("group_start", C.c_void_p), ("max_group_rows", C.c_int32),
                ("row_pos", C.c_void_p), ("table", C.c_void_p), ("table_stride", C.c_int32)]


class RdPagedSessionConfig(C.Structure):
    _fields_ = [(n, C.c_int32) for n in ("page_size", "n_pages", "window", "sinks")]


class RdStats(C.Structure):
    _fields_ = [(n, C.c_uint64) for n in ("df_steps", "ar_steps", "rows_prelude", "rows_core", "rows_coda",
                                          "tokens_committed", "kernel_launches", "tc_gemm_launches",
                                          "weight_bytes", "kv_bytes", "flops")] + [("commit_hist", C.c_uint64 * 16)]


class RdProfile(C.Structure):
    _fields_ = [("gemm_launches", C.c_uint64), ("gemm_ms", C.c_double), ("gemm_weight_bytes", C.c_uint64),
                ("attn_launches", C.c_uint64), ("attn_ms", C.c_double), ("attn_kv_bytes", C.c_uint64),
                ("other_launches", C.c_uint64), ("other_ms", C.c_double)]


class RdError(RuntimeError):
    def __init__(self, code, where, detail=""):
        self.code = code
        super().__init__(f"{where}: {code} ({detail})")


_lib = None


def lib():
    """The loaded library (raises if it is missing: build it with paper_2510_14961_b200.build)."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise RuntimeError(f"{LIB_PATH} is missing: run `python -m paper_2510_14961_b200.build`")
        L = C.CDLL(LIB_PATH)
        vp, i32, f32 = C.c_void_p, C.c_int32, C.c_float
        L.rd_load.argtypes = [C.POINTER(RdConfig), C.POINTER(vp), i32, i32, C.POINTER(vp)]
        L.rd_free.argtypes = [vp]
        L.rd_free.restype = None
        L.rd_session_create.argtypes = [vp, C.POINTER(RdSessionConfig), vp, C.POINTER(vp)]
        L.rd_session_destroy.argtypes = [vp]
        L.rd_session_destroy.restype = None
        L.rd_prefill.argtypes = [vp, i32, vp, i32, i32]
        L.rd_prefill_sliced.argtypes = [vp, i32, vp, i32, i32]
        L.rd_prefill_advance.argtypes = [vp, i32]
        L.rd_prefill_pending.argtypes = [vp]
        L.rd_set_prefill_units.argtypes = [vp, i32]
        L.rd_ar_step.argtypes = [vp, i32]
        L.rd_df_step.argtypes = [vp, i32, i32, f32]
        L.rd_sync.argtypes = [vp]
        L.rd_committed.argtypes = [vp, i32, C.POINTER(i32), C.POINTER(i32)]
        L.rd_get_tokens.argtypes = [vp, i32, vp, i32, C.POINTER(i32)]
        L.rd_last_step_rows.argtypes = [vp, i32, C.POINTER(i32), C.POINTER(i32)]
        L.rd_debug_read.argtypes = [vp, i32, i32, vp, C.c_size_t]
        L.rd_debug_force_tokens.argtypes = [vp, i32, i32, vp, i32]
        L.rd_debug_read_kv.argtypes = [vp, i32, i32, i32, i32, i32, i32, vp]
        L.rd_debug_read_kv_noalloc.argtypes = [vp, i32, i32, i32, i32, i32, i32, vp]
        L.rd_stats.argtypes = [vp, C.POINTER(RdStats)]
        L.rd_set_gemm_path.argtypes = [vp, i32]
        L.rd_set_launch_chaining.argtypes = [vp, i32]
        L.rd_debug_expire_next_wait.argtypes = [vp]
        L.rd_set_fused_swiglu.argtypes = [vp, i32]
        L.rd_set_attention_path.argtypes = [vp, i32]
        L.rd_debug_gemm_sequence.argtypes = [vp, i32, i32, C.POINTER(C.c_uint64), C.POINTER(i32)]
        L.rd_poll_begin.argtypes = [vp, C.POINTER(i32)]
        L.rd_poll_end.argtypes = [vp, i32, i32, C.POINTER(i32), C.POINTER(i32)]
        L.rd_profile_enable.argtypes = [vp, i32]
        L.rd_profile_read.argtypes = [vp, C.POINTER(RdProfile)]
        i64 = C.c_int64
        L.rd_session_create_paged.argtypes = [vp, C.POINTER(RdSessionConfig), C.POINTER(RdPagedSessionConfig), vp, C.POINTER(vp)]
        L.rd_session_release.argtypes = [vp, i32]
        L.rd_paged_create.argtypes = [C.POINTER(RdPagedConfig), vp, vp, C.POINTER(vp)]
        L.rd_paged_destroy.argtypes = [vp]
        L.rd_paged_destroy.restype = None
        L.rd_paged_pages.argtypes = [vp, C.POINTER(vp), C.POINTER(vp)]
        L.rd_paged_append.argtypes = [vp, C.POINTER(RdPagedRows), i32, vp, i64, vp, i64, vp, i64, vp, i64, vp]
        L.rd_paged_attend.argtypes = [vp, C.POINTER(RdPagedRows), i32, vp, i64, vp, i64, vp, i32, i32, f32, vp]
        L.rd_paged_sync.argtypes = [vp, vp]
        L.rd_strerror.argtypes = [C.c_int]
        L.rd_strerror.restype = C.c_char_p
        L.rd_last_cuda_error.restype = C.c_char_p
        _lib = L
    return _lib


def _check(rc, where):
    if rc != RD_OK:
        L = lib()
        detail = L.rd_strerror(rc).decode()
        if rc in (RD_E_CUDA, RD_E_OOM):
            detail += "; " + L.rd_last_cuda_error().decode()
        raise RdError(rc, where, detail)


def _ptr(x):
    """Address of a numpy array (host) or of anything exposing data_ptr() (a torch tensor)."""
    if x is None:
        return None
    if hasattr(x, "data_ptr"):
        return x.data_ptr()
    return x.ctypes.data


class Model:
    """rd_load: device copy of the weights of P, R and C."""

    def __init__(self, hidden, n_heads, head_dim, mlp_inner, n_prelude, n_core, n_coda, vocab, tensors,
                 dtype=RD_F32, tie_embeddings=True, rope_base=10000.0, norm_eps=1e-6, init_sigma=1.0,
                 elem_bytes=4):
        """`tensors`: sequence of arrays in the order include/rd.h states (numpy on the host or torch
        tensors on the device); gains float32, matrices float32 (elem_bytes 4) or bf16 bits (2)."""
        self.cfg = RdConfig(hidden, n_heads, head_dim, mlp_inner, n_prelude, n_core, n_coda, vocab, dtype,
                            1 if tie_embeddings else 0, rope_base, norm_eps, init_sigma)
        self._keep = list(tensors)
        arr = (C.c_void_p * len(self._keep))(*[_ptr(t) for t in self._keep])
        self.handle = C.c_void_p()
        _check(lib().rd_load(C.byref(self.cfg), arr, len(self._keep), elem_bytes, C.byref(self.handle)), "rd_load")
        self._keep = None

    def close(self):
        if self.handle:
            lib().rd_free(self.handle)
            self.handle = C.c_void_p()

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


class Session:
    """rd_session_create and the per-session calls.  page_size > 0: rd_session_create_paged with pools of n_pages
    pages (attn_window, attn_sinks: the positions a row attends)."""

    def __init__(self, model: Model, batch=1, max_context=1024, max_window=1, max_iters_per_pos=64,
                 max_new_tokens=64, keep_logits=False, temperature=0.0, seed=0, stream=None, eta=0.0, beta=0.0,
                 top_p=0.0, latent_slots=0, page_size=0, n_pages=0, attn_window=0, attn_sinks=0):
        self.model = model
        self.sc = RdSessionConfig(batch, max_context, max_window, max_iters_per_pos, max_new_tokens,
                                  1 if keep_logits else 0, temperature, seed, eta, beta, top_p, latent_slots)
        self.handle = C.c_void_p()
        if page_size or n_pages or attn_window or attn_sinks:
            pc = RdPagedSessionConfig(page_size, n_pages, attn_window, attn_sinks)
            _check(lib().rd_session_create_paged(model.handle, C.byref(self.sc), C.byref(pc), C.c_void_p(stream or 0),
                                                 C.byref(self.handle)), "rd_session_create_paged")
            return
        _check(lib().rd_session_create(model.handle, C.byref(self.sc), C.c_void_p(stream or 0),
                                       C.byref(self.handle)), "rd_session_create")

    def close(self):
        if self.handle:
            lib().rd_session_destroy(self.handle)
            self.handle = C.c_void_p()

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def prefill(self, seq, prompt, r):
        p = np.ascontiguousarray(prompt, dtype=np.int32)
        _check(lib().rd_prefill(self.handle, seq, p.ctypes.data, len(p), r), "rd_prefill")

    def release(self, seq):
        """Paged sessions: stops the sequence and returns its pages to the pool."""
        _check(lib().rd_session_release(self.handle, seq), "rd_session_release")

    def prefill_sliced(self, seq, prompt, r):
        p = np.ascontiguousarray(prompt, dtype=np.int32)
        _check(lib().rd_prefill_sliced(self.handle, seq, p.ctypes.data, len(p), r), "rd_prefill_sliced")

    def prefill_advance(self, units):
        _check(lib().rd_prefill_advance(self.handle, units), "rd_prefill_advance")

    def prefill_pending(self):
        n = lib().rd_prefill_pending(self.handle)
        if n < 0:
            _check(n, "rd_prefill_pending")
        return n

    def set_prefill_units(self, units_per_step):
        _check(lib().rd_set_prefill_units(self.handle, units_per_step), "rd_set_prefill_units")

    def ar_step(self, r):
        _check(lib().rd_ar_step(self.handle, r), "rd_ar_step")

    def df_step(self, window, inner_iters, exit_threshold=0.0):
        _check(lib().rd_df_step(self.handle, window, inner_iters, exit_threshold), "rd_df_step")

    def sync(self):
        _check(lib().rd_sync(self.handle), "rd_sync")

    def committed(self, seq=0):
        n, d = C.c_int32(), C.c_int32()
        _check(lib().rd_committed(self.handle, seq, C.byref(n), C.byref(d)), "rd_committed")
        return n.value, bool(d.value)

    def poll_begin(self):
        t = C.c_int32()
        _check(lib().rd_poll_begin(self.handle, C.byref(t)), "rd_poll_begin")
        return t.value

    def poll_end(self, ticket, seq=-1):
        n, d = C.c_int32(), C.c_int32()
        _check(lib().rd_poll_end(self.handle, ticket, seq, C.byref(n), C.byref(d)), "rd_poll_end")
        return n.value, bool(d.value)

    def tokens(self, seq=0, out=None):
        cap = self.sc.max_context + 1
        buf = out if out is not None else np.empty(cap, dtype=np.int32)
        n = C.c_int32()
        _check(lib().rd_get_tokens(self.handle, seq, _ptr(buf), len(buf), C.byref(n)), "rd_get_tokens")
        return buf[: n.value]

    def last_step_rows(self, seq=0):
        f, n = C.c_int32(), C.c_int32()
        _check(lib().rd_last_step_rows(self.handle, seq, C.byref(f), C.byref(n)), "rd_last_step_rows")
        return f.value, n.value

    def debug_read(self, what, seq=0):
        _, n = self.last_step_rows(seq)
        c = self.model.cfg
        shape, dt = {RD_DBG_LATENTS: ((n, c.hidden), np.float32), RD_DBG_EMBED: ((n, c.hidden), np.float32),
                     RD_DBG_DELTA: ((n,), np.float32), RD_DBG_DRAFTS: ((n,), np.int32),
                     RD_DBG_LOGITS: ((n, c.vocab), np.float32)}[what]
        out = np.empty(shape, dtype=dt)
        _check(lib().rd_debug_read(self.handle, what, seq, out.ctypes.data, out.nbytes), "rd_debug_read")
        return out

    def force_tokens(self, seq, first_pos, tokens):
        t = np.ascontiguousarray(tokens, dtype=np.int32)
        _check(lib().rd_debug_force_tokens(self.handle, seq, first_pos, t.ctypes.data, len(t)),
               "rd_debug_force_tokens")

    def read_kv(self, block, layer, which, seq, pos0, n):
        out = np.empty((n, self.model.cfg.hidden), dtype=np.float32)
        _check(lib().rd_debug_read_kv(self.handle, block, layer, which, seq, pos0, n, out.ctypes.data),
               "rd_debug_read_kv")
        return out

    def read_kv_noalloc(self, block, layer, which, seq, pos0, n):
        """read_kv through the library's fixed staging array: no device allocation is made.  For
        callers that cannot allocate (device memory fully committed, or other streams must not be
        stalled); at most 1,048,576 values per call, calls on one device must not overlap."""
        out = np.empty((n, self.model.cfg.hidden), dtype=np.float32)
        _check(lib().rd_debug_read_kv_noalloc(self.handle, block, layer, which, seq, pos0, n, out.ctypes.data),
               "rd_debug_read_kv_noalloc")
        return out

    def stats(self):
        st = RdStats()
        _check(lib().rd_stats(self.handle, C.byref(st)), "rd_stats")
        out = {k: getattr(st, k) for k, _ in RdStats._fields_}
        out["commit_hist"] = [int(v) for v in st.commit_hist]
        return out

    def set_gemm_path(self, path):
        _check(lib().rd_set_gemm_path(self.handle, path), "rd_set_gemm_path")

    def set_launch_chaining(self, on):
        _check(lib().rd_set_launch_chaining(self.handle, 1 if on else 0), "rd_set_launch_chaining")

    def set_attention_path(self, path):
        _check(lib().rd_set_attention_path(self.handle, path), "rd_set_attention_path")

    def set_fused_swiglu(self, on):
        _check(lib().rd_set_fused_swiglu(self.handle, 1 if on else 0), "rd_set_fused_swiglu")

    def gemm_sequence(self, n_rows, reps=1):
        """Measurement aid: the GEMM launches of a decode step, back to back; returns (weight bytes, launches)."""
        b, n = C.c_uint64(), C.c_int32()
        _check(lib().rd_debug_gemm_sequence(self.handle, n_rows, reps, C.byref(b), C.byref(n)), "rd_debug_gemm_sequence")
        return b.value, n.value

    def expire_next_wait(self):
        """Test aid: the next tensor-core GEMM launch lets one bounded wait run out (RD_E_TIMEOUT at the next sync)."""
        _check(lib().rd_debug_expire_next_wait(self.handle), "rd_debug_expire_next_wait")

    def profile_enable(self, on=True):
        _check(lib().rd_profile_enable(self.handle, 1 if on else 0), "rd_profile_enable")

    def profile_read(self):
        pr = RdProfile()
        _check(lib().rd_profile_read(self.handle, C.byref(pr)), "rd_profile_read")
        return {k: getattr(pr, k) for k, _ in RdProfile._fields_}


class PagedRows:
    """The rows of a paged call (rd_paged_rows): device tensors of int32.

    row_pos [n_rows]: position of every row in its sequence, negative: no row.  table [n_groups, pages]: the
    sequences' pages in order.  group_start [n_groups + 1]: group i holds rows group_start[i] ..; None: every
    group holds `max_group_rows` rows.  The tensors are read when the kernels run: keep them alive (this object
    does) and change them only behind the calls that use them."""

    def __init__(self, row_pos, table, group_start=None, max_group_rows=0):
        for name, t, dims in (("row_pos", row_pos, 1), ("table", table, 2), ("group_start", group_start, 1)):
            if t is None and name == "group_start":
                continue
            if t.dim() != dims or t.element_size() != 4 or t.is_floating_point() or not t.is_cuda:
                raise ValueError(f"{name}: a device tensor of int32 with {dims} dimension(s)")
            if t.numel() and t.stride(-1) != 1:
                raise ValueError(f"{name}: not contiguous")
        n_groups, pages = table.shape
        if group_start is not None and group_start.numel() != n_groups + 1:
            raise ValueError("group_start: one entry per group and one more")
        self.row_pos, self.table, self.group_start = row_pos, table, group_start
        self.c = RdPagedRows(row_pos.numel(), n_groups, _ptr(group_start), max_group_rows, _ptr(row_pos), _ptr(table),
                             table.stride(0) if n_groups > 1 else pages)
        self.ref = C.byref(self.c)


class PagedCache:
    """rd_paged_create and the calls on a paged K/V cache.

    k_pages, v_pages: device tensors [n_layers, n_pages, n_kv_heads, page_size, head_dim] of the cache's type, or
    None: the library allocates them.  stream: the CUDA stream of calls that name none (None: the legacy default
    stream).  Calls of one cache run one after another; see include/rd.h."""

    def __init__(self, n_heads, n_kv_heads, head_dim, page_size, n_pages, n_layers=1, max_context=4096, dtype=RD_BF16,
                 rope_base=10000.0, max_rows=0, k_pages=None, v_pages=None, stream=None):
        self.cfg = RdPagedConfig(n_heads, n_kv_heads, head_dim, dtype, page_size, n_pages, n_layers, max_context, max_rows, rope_base)
        self.handle = C.c_void_p()
        self.stream = stream
        self._dtype = None                   # the cache's torch type, once a tensor of it has been seen
        for name, t in (("k_pages", k_pages), ("v_pages", v_pages)):
            if t is None:
                continue
            self._typed(name, t)
            if t.numel() != n_layers * n_pages * n_kv_heads * page_size * head_dim or not t.is_contiguous():
                raise ValueError(f"{name}: contiguous [n_layers, n_pages, n_kv_heads, page_size, head_dim]")
        self._keep = (k_pages, v_pages)
        _check(lib().rd_paged_create(C.byref(self.cfg), _ptr(k_pages), _ptr(v_pages), C.byref(self.handle)), "rd_paged_create")

    def _typed(self, name, t):
        if not t.is_cuda or not str(t.dtype).endswith("bfloat16" if self.cfg.dtype == RD_BF16 else "float32"):
            raise ValueError(f"{name}: a device tensor of the cache's type")
        self._dtype = t.dtype

    def _rows(self, name, t, n_rows, heads):
        """Address and row stride of [n_rows, heads, head_dim] (or [n_rows, heads * head_dim])."""
        if t.dtype is not self._dtype or not t.is_cuda:
            self._typed(name, t)
        d, shape, stride = self.cfg.head_dim, t.shape, t.stride()
        if len(shape) == 3:
            ok = shape[0] == n_rows and shape[1] == heads and shape[2] == d
            flat = stride[2] == 1 and (heads == 1 or stride[1] == d)
        else:
            ok = len(shape) == 2 and shape[0] == n_rows and shape[1] == heads * d
            flat = ok and stride[1] == 1
        if not ok:
            raise ValueError(f"{name}: shape {tuple(shape)}, wanted ({n_rows}, {heads}, {d})")
        if not flat and n_rows:
            raise ValueError(f"{name}: heads and features must be contiguous")
        return t.data_ptr(), (stride[0] if n_rows > 1 else heads * d)

    def append(self, rows, q, k, v, q_out, layer=0, stream=None):
        n, c = rows.c.n_rows, self.cfg
        h, g = c.n_heads, c.n_kv_heads
        rc = lib().rd_paged_append(self.handle, rows.ref, layer, *self._rows("q", q, n, h), *self._rows("k", k, n, g),
                                   *self._rows("v", v, n, g), *self._rows("q_out", q_out, n, h), self.stream if stream is None else stream)
        if rc:
            _check(rc, "rd_paged_append")

    def attend(self, rows, q, out, lse=None, layer=0, window=0, sinks=0, scale=0.0, stream=None):
        n, h = rows.c.n_rows, self.cfg.n_heads
        if lse is not None and (lse.shape != (n, h) or lse.element_size() != 4 or not lse.is_contiguous() or not lse.is_cuda):
            raise ValueError(f"lse: contiguous float32 ({n}, {h})")
        rc = lib().rd_paged_attend(self.handle, rows.ref, layer, *self._rows("q", q, n, h), *self._rows("out", out, n, h),
                                   None if lse is None else lse.data_ptr(), window, sinks, scale, self.stream if stream is None else stream)
        if rc:
            _check(rc, "rd_paged_attend")

    def pages(self):
        """Device addresses of the K and the V pages."""
        k, v = C.c_void_p(), C.c_void_p()
        _check(lib().rd_paged_pages(self.handle, C.byref(k), C.byref(v)), "rd_paged_pages")
        return k.value, v.value

    def sync(self, stream=None):
        _check(lib().rd_paged_sync(self.handle, self.stream if stream is None else stream), "rd_paged_sync")

    def close(self):
        if self.handle:
            lib().rd_paged_destroy(self.handle)
            self.handle = C.c_void_p()

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass
