"""ctypes binding of libsk.so: the same entry points as include/sk.h, argument marshalling
only.  PyTorch appears here for device memory and streams, nothing else; every step of the
path runs in the library's HIP kernels.  There is no CPU fallback: if libsk.so is missing or
a call fails, an exception is raised.
"""
import array
import ctypes
import os
import numpy as np

import torch

from . import _build

SK_F32, SK_BF16 = 0, 1
SK_OP_APPEND, SK_OP_QUERY_A, SK_OP_QUERY_B = 0, 1, 2
SK_POOL_METADATA_ONLY = 1

SK_SITE_RING, SK_SITE_UPLOAD, SK_SITE_BLOCK_COPY, SK_SITE_SCATTER, SK_SITE_ATTENTION, SK_SITE_COMBINE, SK_SITE_PLAN = 1, 2, 3, 4, 5, 6, 7
SK_SITE_EVICT_SELECT, SK_SITE_EVICT_MOVE = 8, 9
SK_TOP2_STATIC_BYTES = 1 << 20
SK_LOGPROBS_MAX_TOP, SK_LOGPROBS_MAX_ROWS, SK_LOGPROBS_MAX_VOCAB = 32, 1 << 20, 1 << 21
SK_VERIFY_MAX_DRAFT, SK_VERIFY_MAX_ROWS, SK_VERIFY_MAX_VOCAB = 32, 1 << 20, 1 << 21

SK_OK = 0
SK_E_INVAL, SK_E_SHAPE, SK_E_DTYPE, SK_E_NOMEM, SK_E_BADSESSION = -1, -2, -3, -4, -5
SK_E_EMPTY, SK_E_WORKSPACE, SK_E_HIP, SK_E_NODEVICE = -6, -7, -8, -9


class SkError(RuntimeError):
    def __init__(self, status, where):
        self.status = status
        msg = "%s: %s (%d)" % (where, lib().sk_strerror(status).decode(), status)
        if status == SK_E_HIP:
            msg += " hipError=%d" % lib().sk_last_hip_error()
        super().__init__(msg)


class sk_pool_desc(ctypes.Structure):
    _fields_ = [
        ("dtype", ctypes.c_int32), ("n_q_heads", ctypes.c_int32), ("n_kv_heads", ctypes.c_int32),
        ("head_dim", ctypes.c_int32), ("block_tokens", ctypes.c_int32), ("max_sessions", ctypes.c_int32),
        ("n_blocks", ctypes.c_int64), ("max_session_tokens", ctypes.c_int64),
        ("max_batch_tokens", ctypes.c_int32), ("flags", ctypes.c_int32),
        ("softmax_scale", ctypes.c_float), ("reserved", ctypes.c_int32),
        ("kv_mem", ctypes.c_void_p), ("kv_bytes", ctypes.c_size_t),
        ("workspace", ctypes.c_void_p), ("workspace_bytes", ctypes.c_size_t),
    ]


class sk_pool_stats(ctypes.Structure):
    _fields_ = [("tokens_appended", ctypes.c_int64), ("tokens_queried", ctypes.c_int64),
                ("launches", ctypes.c_int64), ("kv_bytes_streamed", ctypes.c_int64),
                ("tokens_evicted", ctypes.c_int64), ("forks", ctypes.c_int64)]


class sk_launch_info(ctypes.Structure):
    _fields_ = [("workgroups", ctypes.c_int32), ("n_splits", ctypes.c_int32),
                ("row_tiles", ctypes.c_int32), ("kernel_variant", ctypes.c_int32),
                ("fused_merge", ctypes.c_int32), ("reserved", ctypes.c_int32 * 3)]


class sk_profile(ctypes.Structure):
    _fields_ = [("calls", ctypes.c_int64), ("attention_ms", ctypes.c_double), ("combine_ms", ctypes.c_double)]


EXPORTS = [
    "sk_pool_kv_bytes", "sk_pool_workspace_bytes", "sk_pool_create", "sk_pool_destroy",
    "sk_pool_blocks_free", "sk_pool_set_alloc_order", "sk_session_create", "sk_session_destroy",
    "sk_session_length", "sk_session_block_table", "sk_session_append", "sk_session_query",
    "sk_batch_step", "sk_session_query_shared_prefix", "sk_session_gather",
    "sk_session_truncate", "sk_session_freeze", "sk_session_evict_oldest", "sk_session_fork",
    "sk_pool_set_profiling", "sk_pool_read_profile",
    "sk_pool_element_offset", "sk_pool_get_stats", "sk_pool_last_launch", "sk_strerror",
    "sk_last_hip_error", "sk_version", "sk_top2_workspace_bytes", "sk_top2", "sk_top2_static",
    "sk_session_evict_lowest", "sk_session_attention_mass", "sk_batch_attention_mass",
    "sk_logprobs_workspace_bytes", "sk_logprobs", "sk_verify_workspace_bytes", "sk_verify",
    "sk_pool_set_rotation", "sk_rotate", "sk_session_append_rotated", "sk_batch_step_rotated", "sk_session_shift",
    "sk_pool_inject_failure", "sk_probe_read", "sk_probe_mfma",
]

_lib = None


def lib_path():
    return _build.LIB


def lib():
    """Loads libsk.so (building it only if no built library is there)."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(_build.LIB):
        _build.build(force=True)
    elif _build.is_stale():
        import warnings
        warnings.warn("%s is older than its sources; run paper_2605_13784_amd._build.build()" % _build.LIB, RuntimeWarning)
    L = ctypes.CDLL(_build.LIB)
    vp, i32, i64, sz = ctypes.c_void_p, ctypes.c_int32, ctypes.c_int64, ctypes.c_size_t
    P = ctypes.POINTER
    L.sk_pool_kv_bytes.restype = sz
    L.sk_pool_kv_bytes.argtypes = [P(sk_pool_desc)]
    L.sk_pool_workspace_bytes.restype = sz
    L.sk_pool_workspace_bytes.argtypes = [P(sk_pool_desc)]
    L.sk_pool_create.argtypes = [P(sk_pool_desc), P(vp)]
    L.sk_pool_destroy.argtypes = [vp]
    L.sk_pool_blocks_free.argtypes = [vp, P(i64)]
    L.sk_pool_set_alloc_order.argtypes = [vp, P(i32), i64]
    L.sk_session_create.argtypes = [vp, P(i32)]
    L.sk_session_destroy.argtypes = [vp, i32]
    L.sk_session_length.argtypes = [vp, i32, P(i64)]
    L.sk_session_block_table.argtypes = [vp, i32, P(P(i32)), P(i64)]
    L.sk_session_append.argtypes = [vp, i32, vp, vp, vp, i32, vp, ctypes.c_int, vp, vp]
    L.sk_session_query.argtypes = [vp, i32, vp, vp, vp, i32, vp, ctypes.c_int, vp, i32, vp]
    L.sk_batch_step.argtypes = [vp, i32, P(i32), P(i32), P(i32), vp, vp, vp, vp, ctypes.c_int, vp, vp]
    L.sk_session_query_shared_prefix.argtypes = [vp, i32, vp, vp, vp, i32, vp, vp, vp, i32, i32,
                                                 vp, vp, ctypes.c_int, vp, vp, vp]
    L.sk_session_gather.argtypes = [vp, i32, i64, i64, vp, vp, vp]
    L.sk_session_truncate.argtypes = [vp, i32, i64]
    L.sk_session_freeze.argtypes = [vp, i32, i64]
    L.sk_session_evict_oldest.argtypes = [vp, i32, i64, vp]
    L.sk_session_fork.argtypes = [vp, i32, i64, P(i32), vp]
    L.sk_top2_workspace_bytes.restype = ctypes.c_size_t
    L.sk_top2_workspace_bytes.argtypes = [i32, i32]
    L.sk_top2.argtypes = [vp, i32, i32, i64, vp, ctypes.c_size_t, vp, vp, vp, vp, vp, vp]
    L.sk_top2_static.argtypes = [vp, i32, i32, i64, vp, vp, vp, vp, vp, vp]
    L.sk_session_evict_lowest.argtypes = [vp, i32, vp, i64, i64, i64, i32, vp, i64, vp]
    L.sk_session_attention_mass.argtypes = [vp, i32, vp, vp, i32, i32, vp, i64, ctypes.c_float, vp, i64, vp]
    L.sk_batch_attention_mass.argtypes = [vp, i32, P(i32), P(i32), P(i32), vp, vp, P(vp), P(i64), ctypes.c_float, P(vp), P(i64), vp]
    L.sk_logprobs_workspace_bytes.restype = ctypes.c_size_t
    L.sk_logprobs_workspace_bytes.argtypes = [i32, i32, i32]
    L.sk_logprobs.argtypes = [vp, ctypes.c_int, i32, i32, i64, vp, i32, i32, vp, ctypes.c_size_t, vp, vp, vp, vp, vp, vp]
    L.sk_pool_set_rotation.argtypes = [vp, i32, i32, P(ctypes.c_double), ctypes.c_float]
    L.sk_rotate.argtypes = [vp, vp, vp, i32, vp, i32, vp, vp, vp]
    L.sk_session_append_rotated.argtypes = [vp, i32, vp, vp, vp, i32, vp, i32, vp, vp, ctypes.c_int, vp, vp]
    L.sk_batch_step_rotated.argtypes = [vp, i32, vp, vp, vp, vp, vp, vp, vp, vp, vp, ctypes.c_int, vp, vp]
    L.sk_session_shift.argtypes = [vp, i32, i64, i64, i32, vp, i64, vp]
    L.sk_verify_workspace_bytes.restype = ctypes.c_size_t
    L.sk_verify_workspace_bytes.argtypes = [i32, i32, i32]
    L.sk_verify.argtypes = [vp, i64, vp, i64, ctypes.c_int, i32, i32, i32, vp, vp, vp, vp, ctypes.c_size_t, vp, vp, vp, vp]
    L.sk_pool_inject_failure.argtypes = [vp, i32, i32]
    L.sk_probe_read.argtypes = [vp, ctypes.c_size_t, i32, i32, vp, vp]
    L.sk_probe_mfma.argtypes = [i32, i32, vp, ctypes.c_size_t, vp, P(ctypes.c_double), vp]
    L.sk_pool_set_profiling.argtypes = [vp, ctypes.c_int]
    L.sk_pool_read_profile.argtypes = [vp, P(sk_profile), P(ctypes.c_float), P(ctypes.c_float), i32]
    L.sk_pool_element_offset.restype = i64
    L.sk_pool_element_offset.argtypes = [vp, i64, i32, i32, i32, i32]
    L.sk_pool_get_stats.argtypes = [vp, P(sk_pool_stats)]
    L.sk_pool_last_launch.argtypes = [vp, P(sk_launch_info)]
    L.sk_strerror.restype = ctypes.c_char_p
    L.sk_strerror.argtypes = [ctypes.c_int]
    L.sk_last_hip_error.argtypes = []
    L.sk_version.argtypes = []
    for name in EXPORTS:
        fn = getattr(L, name)
        if fn.restype is ctypes.c_int:
            fn.restype = ctypes.c_int
    _lib = L
    return L


def _dt(dtype):
    if dtype in ("f32", torch.float32, SK_F32):
        return SK_F32
    if dtype in ("bf16", torch.bfloat16, SK_BF16):
        return SK_BF16
    raise ValueError(dtype)


def _p(t):
    if t is None:
        return None
    assert t.is_contiguous()
    return t.data_ptr()


# The current stream's handle.  torch.cuda.current_stream() makes a Stream object on every call (2.9 us; the handle alone
# 0.1); with it and a pointer object per argument a decoded token at 2,600 cached tokens took the host 8.6 us, as
# long as the GPU, of which the library's call is 3.8.
_raw_stream, _device = getattr(torch._C, "_cuda_getCurrentRawStream", None), getattr(torch._C, "_cuda_getDevice", None)


def _stream(stream):
    if stream is None:
        if _raw_stream is not None and _device is not None:
            return _raw_stream(_device())
        return torch.cuda.current_stream().cuda_stream
    if isinstance(stream, torch.cuda.Stream):
        return stream.cuda_stream
    return stream


def _made(stream, *tensors):
    """Tensors that a call makes here, as outputs or scratch, for a stream that is named: their memory came from the current one, and the
    allocator may not hand it out again, however early they are dropped, before that stream has come to here."""
    if stream is not None:
        if not isinstance(stream, torch.cuda.Stream):
            stream = torch.cuda.ExternalStream(getattr(stream, "value", stream) or 0)
        for t in tensors:
            if t is not None:
                t.record_stream(stream)


def _ck(status, where):
    if status != SK_OK:
        raise SkError(status, where)


def make_desc(dtype, n_q_heads, n_kv_heads, head_dim, block_tokens, n_blocks, max_sessions=1,
              max_session_tokens=0, max_batch_tokens=0, softmax_scale=0.0, flags=0):
    d = sk_pool_desc()
    d.dtype = _dt(dtype)
    d.n_q_heads, d.n_kv_heads, d.head_dim = n_q_heads, n_kv_heads, head_dim
    d.block_tokens, d.n_blocks, d.max_sessions = block_tokens, n_blocks, max_sessions
    d.max_session_tokens, d.max_batch_tokens = max_session_tokens, max_batch_tokens
    d.softmax_scale, d.flags = softmax_scale, flags
    return d


def sk_pool_kv_bytes(desc):
    return int(lib().sk_pool_kv_bytes(ctypes.byref(desc)))


def sk_pool_workspace_bytes(desc):
    return int(lib().sk_pool_workspace_bytes(ctypes.byref(desc)))


class Pool:
    """A pool handle plus the torch tensors that back it (allocation only)."""

    def __init__(self, dtype, n_q_heads, n_kv_heads, head_dim, block_tokens, n_blocks, max_sessions=1,
                 max_session_tokens=0, max_batch_tokens=0, softmax_scale=0.0, metadata_only=False,
                 device="cuda:0", kv_fill=None):
        self.desc = make_desc(dtype, n_q_heads, n_kv_heads, head_dim, block_tokens, n_blocks, max_sessions,
                              max_session_tokens, max_batch_tokens, softmax_scale,
                              SK_POOL_METADATA_ONLY if metadata_only else 0)
        self.dtype = "f32" if self.desc.dtype == SK_F32 else "bf16"
        self.torch_dtype = torch.float32 if self.desc.dtype == SK_F32 else torch.bfloat16
        self.Hq, self.Hkv, self.d = n_q_heads, n_kv_heads, head_dim
        self.device = device
        kvb, wsb = sk_pool_kv_bytes(self.desc), sk_pool_workspace_bytes(self.desc)
        if kvb == 0 or wsb == 0:
            raise SkError(SK_E_SHAPE, "pool description")
        self.kv_mem = self.workspace = None
        if not metadata_only:
            self.kv_mem = torch.empty(kvb, dtype=torch.uint8, device=device)
            if kv_fill is not None:
                self.kv_mem.fill_(kv_fill)
            self.workspace = torch.empty(wsb, dtype=torch.uint8, device=device)
            self.desc.kv_mem, self.desc.kv_bytes = self.kv_mem.data_ptr(), kvb
            self.desc.workspace, self.desc.workspace_bytes = self.workspace.data_ptr(), wsb
        h = ctypes.c_void_p()
        _ck(lib().sk_pool_create(ctypes.byref(self.desc), ctypes.byref(h)), "sk_pool_create")
        self.h = h
        self._len = ctypes.c_int64()
        self._len_ref = ctypes.byref(self._len)

    def close(self):
        if self.h:
            if self.kv_mem is not None:
                torch.cuda.synchronize()
            lib().sk_pool_destroy(self.h)
            self.h = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    # -- bookkeeping -----------------------------------------------------------------------
    def sk_pool_blocks_free(self):
        out = ctypes.c_int64()
        _ck(lib().sk_pool_blocks_free(self.h, ctypes.byref(out)), "sk_pool_blocks_free")
        return out.value

    def sk_pool_set_alloc_order(self, perm):
        arr = np.ascontiguousarray(perm, dtype=np.int32)
        _ck(lib().sk_pool_set_alloc_order(self.h, arr.ctypes.data_as(ctypes.POINTER(ctypes.c_int32)), arr.size),
            "sk_pool_set_alloc_order")

    def sk_session_create(self):
        out = ctypes.c_int32()
        _ck(lib().sk_session_create(self.h, ctypes.byref(out)), "sk_session_create")
        return out.value

    def sk_session_destroy(self, sid):
        _ck(lib().sk_session_destroy(self.h, sid), "sk_session_destroy")

    def sk_session_length(self, sid):
        out = ctypes.c_int64()
        _ck(lib().sk_session_length(self.h, sid, ctypes.byref(out)), "sk_session_length")
        return out.value

    def sk_session_block_table(self, sid):
        tbl = ctypes.POINTER(ctypes.c_int32)()
        n = ctypes.c_int64()
        _ck(lib().sk_session_block_table(self.h, sid, ctypes.byref(tbl), ctypes.byref(n)), "sk_session_block_table")
        return [tbl[i] for i in range(n.value)]

    def sk_session_truncate(self, sid, new_length):
        _ck(lib().sk_session_truncate(self.h, sid, int(new_length)), "sk_session_truncate")

    def sk_session_freeze(self, sid, n_frozen):
        _ck(lib().sk_session_freeze(self.h, sid, int(n_frozen)), "sk_session_freeze")

    def sk_session_fork(self, src, n_prefix, stream=None):
        out = ctypes.c_int32()
        _ck(lib().sk_session_fork(self.h, src, int(n_prefix), ctypes.byref(out),
                                  _stream(stream) if self.kv_mem is not None else None), "sk_session_fork")
        return out.value

    def sk_session_evict_oldest(self, sid, n_tokens, stream=None):
        _ck(lib().sk_session_evict_oldest(self.h, sid, int(n_tokens), _stream(stream) if self.kv_mem is not None else None),
            "sk_session_evict_oldest")

    def sk_pool_set_profiling(self, enable):
        _ck(lib().sk_pool_set_profiling(self.h, int(bool(enable))), "sk_pool_set_profiling")

    def sk_pool_read_profile(self):
        """-> (sums dict, per-call attention ms list, per-call combine ms list)"""
        s = sk_profile()
        cap = 4096
        a = (ctypes.c_float * cap)()
        c = (ctypes.c_float * cap)()
        _ck(lib().sk_pool_read_profile(self.h, ctypes.byref(s), a, c, cap), "sk_pool_read_profile")
        n = min(cap, s.calls)
        return {k: getattr(s, k) for k, _ in s._fields_}, list(a[:n]), list(c[:n])

    def sk_pool_get_stats(self):
        s = sk_pool_stats()
        _ck(lib().sk_pool_get_stats(self.h, ctypes.byref(s)), "sk_pool_get_stats")
        return {k: getattr(s, k) for k, _ in s._fields_}

    def sk_pool_last_launch(self):
        s = sk_launch_info()
        _ck(lib().sk_pool_last_launch(self.h, ctypes.byref(s)), "sk_pool_last_launch")
        return {k: getattr(s, k) for k, _ in s._fields_ if k != "reserved"}

    def sk_pool_inject_failure(self, site, countdown=1):
        _ck(lib().sk_pool_inject_failure(self.h, int(site), int(countdown)), "sk_pool_inject_failure")

    def sk_pool_element_offset(self, block, kv_head, is_v, slot, dim):
        return int(lib().sk_pool_element_offset(self.h, block, kv_head, int(is_v), slot, dim))

    # -- compute ---------------------------------------------------------------------------
    def _out(self, T, out_dtype, want_lse, stream):
        odt = torch.float32 if _dt(out_dtype) == SK_F32 else torch.bfloat16
        out = torch.empty((T, self.Hq, self.d), dtype=odt, device=self.device)
        lse = torch.empty((T, self.Hq), dtype=torch.float32, device=self.device) if want_lse else None
        _made(stream, out, lse)
        return out, lse

    def sk_session_append(self, sid, q, k, v, out=None, lse=None, out_dtype="f32", want_lse=True, stream=None,
                          n_tokens=None):
        L = int(k.shape[0]) if n_tokens is None else int(n_tokens)
        if q is not None and out is None and self.kv_mem is not None:
            out, lse = self._out(L, out_dtype, want_lse, stream)
        _ck(lib().sk_session_append(self.h, sid, _p(q), _p(k), _p(v), L, _p(out), _dt(out_dtype), _p(lse),
                                    _stream(stream) if self.kv_mem is not None else None), "sk_session_append")
        return out, lse

    def reserve(self, sid, n_tokens):
        """Metadata-only pools: the allocation half of an append."""
        _ck(lib().sk_session_append(self.h, sid, None, None, None, int(n_tokens), None, SK_F32, None, None),
            "sk_session_append")

    def sk_session_query(self, sid, q, k=None, v=None, out=None, lse=None, out_dtype="f32", want_lse=True,
                         n_splits=0, stream=None):
        nq = int(q.shape[0])
        if out is None:
            out, lse = self._out(nq, out_dtype, want_lse, stream)
        _ck(lib().sk_session_query(self.h, sid, _p(q), _p(k), _p(v), nq, _p(out), _dt(out_dtype), _p(lse),
                                   int(n_splits), _stream(stream)), "sk_session_query")
        return out, lse

    def sk_batch_step(self, session_ids, ops, cu_tokens, q, k, v, out=None, lse=None, out_dtype="f32",
                      want_lse=True, stream=None):
        n = len(session_ids)
        T = int(cu_tokens[-1])
        if out is None:
            out, lse = self._out(T, out_dtype, want_lse, stream)
        sid = (ctypes.c_int32 * n)(*[int(x) for x in session_ids])
        op = (ctypes.c_int32 * n)(*[int(x) for x in ops])
        cu = (ctypes.c_int32 * (n + 1))(*[int(x) for x in cu_tokens])
        _ck(lib().sk_batch_step(self.h, n, sid, op, cu, _p(q), _p(k), _p(v), _p(out), _dt(out_dtype), _p(lse),
                                _stream(stream)), "sk_batch_step")
        return out, lse

    def sk_session_query_shared_prefix(self, sid, qp, kp, vp, qs, ks, vs, out_dtype="f32", want_lse=True,
                                       stream=None):
        P = 0 if qp is None else int(qp.shape[0])
        NQ, Sfx = int(qs.shape[0]), int(qs.shape[1])
        out_p, lse_p = self._out(P, out_dtype, want_lse, stream)
        out_s, lse_s = self._out(NQ * Sfx, out_dtype, want_lse, stream)
        _ck(lib().sk_session_query_shared_prefix(self.h, sid, _p(qp), _p(kp), _p(vp), P, _p(qs), _p(ks), _p(vs),
                                                 NQ, Sfx, _p(out_p), _p(out_s), _dt(out_dtype), _p(lse_p),
                                                 _p(lse_s), _stream(stream)), "sk_session_query_shared_prefix")
        out_s = out_s.view(NQ, Sfx, self.Hq, self.d)
        if lse_s is not None:
            lse_s = lse_s.view(NQ, Sfx, self.Hq)
        return out_p, lse_p, out_s, lse_s

    def _length(self, sid):
        _ck(lib().sk_session_length(self.h, sid, self._len_ref), "sk_session_length")
        return self._len.value

    def _mass(self, t, n):
        """Checks an array of accumulated weights: float32 [Hkv, >= n], entries of a row next to each other.  -> address, row stride"""
        rows, cols = t.shape
        stride, step = t.stride()
        assert t.dtype is torch.float32 and rows == self.Hkv and cols >= n and (step == 1 or cols <= 1) and t.is_cuda
        return t.data_ptr(), (stride if rows > 1 else max(n, 1))

    def sk_session_attention_mass(self, sid, q, lse, causal=False, mass_in=None, keep=1.0, mass_out=None, stream=None):
        """q [tokens, Hq, d], lse [tokens, Hq] of a call's rows; mass_in, mass_out: float32 [Hkv, capacity]; mass_out left out: mass_in in
        place, or a new [Hkv, length]."""
        n, n_tok = self._length(sid), 0 if q is None else q.shape[0]
        if mass_out is None:
            mass_out = mass_in
            if mass_in is None:
                mass_out = torch.empty((self.Hkv, n), dtype=torch.float32, device=self.device)
                _made(stream, mass_out)
        assert q is None or (q.dtype is self.torch_dtype and lse.dtype is torch.float32 and q.numel() == n_tok * self.Hq * self.d and lse.numel() == n_tok * self.Hq)
        po, so = self._mass(mass_out, n)
        pi, si = (None, 0) if mass_in is None or keep == 0 else (po, so) if mass_in is mass_out else self._mass(mass_in, n)
        _ck(lib().sk_session_attention_mass(self.h, sid, _p(q), _p(lse), n_tok, int(bool(causal)), pi, si, keep, po, so, _stream(stream)),
            "sk_session_attention_mass")
        return mass_out

    def sk_session_evict_lowest(self, sid, mass_in, n_evict, n_recent=0, per_head=True, mass_out=None, stream=None):
        """mass_in: float32 [Hkv, capacity]; the sums of what stays go to mass_out, left out: mass_in in place; False: they are not kept, and
        mass_in stays as it is.  Metadata-only pools: mass_in None."""
        pi, si, po, so = None, 0, None, 0
        mass_out = mass_in if mass_out is None else None if mass_out is False else mass_out
        if self.kv_mem is not None:
            n = self._length(sid)
            pi, si = self._mass(mass_in, n)
            if mass_out is not None:
                po, so = self._mass(mass_out, n)
        _ck(lib().sk_session_evict_lowest(self.h, sid, pi, si, int(n_evict), int(n_recent), int(bool(per_head)), po, so,
                                          _stream(stream) if self.kv_mem is not None else None), "sk_session_evict_lowest")
        return mass_out

    def sk_batch_attention_mass(self, session_ids, cu_tokens, q, lse, causal=None, mass_in=None, keep=1.0, mass_out=None, stream=None):
        """The same for a ragged step: mass_in and mass_out are lists of arrays, one a session."""
        n = len(session_ids)
        lengths = [self._length(s) for s in session_ids]
        if mass_out is None:
            mass_out = mass_in
            if mass_in is None:
                mass_out = [torch.empty((self.Hkv, m), dtype=torch.float32, device=self.device) for m in lengths]
                _made(stream, *mass_out)
        assert q.dtype is self.torch_dtype and lse.dtype is torch.float32 and q.numel() >= cu_tokens[-1] * self.Hq * self.d and lse.numel() >= cu_tokens[-1] * self.Hq

        def host(arrays):
            got = [self._mass(t, m) for t, m in zip(arrays, lengths, strict=True)]
            return (ctypes.c_void_p * n)(*[x for x, _ in got]), (ctypes.c_int64 * n)(*[x for _, x in got])

        pi, si = host(mass_in) if mass_in is not None and keep != 0 else (None, None)
        po, so = host(mass_out)
        _ck(lib().sk_batch_attention_mass(self.h, n, (ctypes.c_int32 * n)(*session_ids), None if causal is None else (ctypes.c_int32 * n)(*map(int, causal)),
                                          (ctypes.c_int32 * (n + 1))(*cu_tokens), _p(q), _p(lse), pi, si, keep, po, so, _stream(stream)),
            "sk_batch_attention_mass")
        return mass_out

    # -- position rotation -------------------------------------------------------------------
    def sk_pool_set_rotation(self, inv_freq, interleaved=False, factor=1.0):
        """inv_freq: an angle a position for each pair (rotary_dim / 2 numbers, float64 on the host)."""
        f = np.ascontiguousarray(inv_freq, dtype=np.float64)
        assert f.ndim == 1
        _ck(lib().sk_pool_set_rotation(self.h, 2 * f.size, int(bool(interleaved)), f.ctypes.data_as(ctypes.POINTER(ctypes.c_double)), float(factor)),
            "sk_pool_set_rotation")

    def _turns(self, q, q_out, heads, n, positions, stream):
        """Checks rows that are turned, and their positions; makes the output that was left out."""
        assert positions is None or (positions.dtype is torch.int32 and positions.is_cuda and positions.numel() == n)
        if q is None:
            return None
        size = n * heads * self.d
        assert q.dtype is self.torch_dtype and q.is_cuda and q.numel() == size
        if q_out is None:
            q_out = torch.empty_like(q, memory_format=torch.contiguous_format)
            _made(stream, q_out)
        else:
            assert q_out.dtype is self.torch_dtype and q_out.is_cuda and q_out.numel() == size
        return q_out

    def _own(self, x, n):
        """Checks k or v of a call that reads n tokens of it."""
        assert x.dtype is self.torch_dtype and x.is_cuda and x.numel() >= n * self.Hkv * self.d

    def _results(self, out, lse, out_dtype, n):
        """Checks a caller's outputs of a call of n tokens (which may have room for more)."""
        rows = n * self.Hq
        assert out is None or (out.dtype is (torch.float32 if _dt(out_dtype) == SK_F32 else torch.bfloat16) and out.is_cuda and out.numel() >= rows * self.d)
        assert lse is None or (lse.dtype is torch.float32 and lse.is_cuda and lse.numel() >= rows)

    def sk_rotate(self, q, k=None, positions=None, pos0=0, q_out=None, k_out=None, stream=None):
        """q [tokens, Hq, d] and k [tokens, Hkv, d] (either None) turned by int32 positions [tokens], or pos0, pos0 + 1, ..: of no session, so
        that rows that an append would put at its session's length need pos0=sk_session_length(sid).  -> (q_out, k_out)"""
        n = int((k if q is None else q).shape[0])
        q_out = self._turns(q, q_out, self.Hq, n, positions, stream)
        k_out = self._turns(k, k_out, self.Hkv, n, positions, stream)
        _ck(lib().sk_rotate(self.h, _p(q), _p(k), n, _p(positions), int(pos0), _p(q_out), _p(k_out), _stream(stream)), "sk_rotate")
        return q_out, k_out

    def sk_session_append_rotated(self, sid, q, k, v, positions=None, pos0=None, q_out=None, out=None, lse=None, attend=True, out_dtype="f32",
                                  want_lse=True, stream=None):
        """sk_session_append with q and k turned on the way.  attend=False: q is turned, nothing attends.  -> (q_out, out, lse)

        positions and pos0 left out: the new tokens' positions follow the session's length, the right ones where the cached tokens' are 0, 1, ..  They are not where
        tokens have left the session (sk_session_evict_oldest, sk_session_evict_lowest) and sk_session_shift has not moved what stays: there the
        length is a position that a cached key has, and the caller gives its own.  Nor are they where earlier appends got other positions."""
        L = int(k.shape[0])
        if pos0 is None:
            pos0 = 0 if positions is not None else self._length(sid)
        if self.kv_mem is not None:
            q_out = self._turns(q, q_out, self.Hq, L, positions, stream)
            self._own(k, L), self._own(v, L)
            assert k.numel() == v.numel() == L * self.Hkv * self.d
            if q is not None and attend and out is None:
                out, lse = self._out(L, out_dtype, want_lse, stream)
            else:
                self._results(out, lse, out_dtype, L)
        _ck(lib().sk_session_append_rotated(self.h, sid, _p(q), _p(k), _p(v), L, _p(positions), int(pos0), _p(q_out), _p(out), _dt(out_dtype), _p(lse),
                                            _stream(stream) if self.kv_mem is not None else None), "sk_session_append_rotated")
        return q_out, out, lse

    def sk_batch_step_rotated(self, session_ids, ops, cu_tokens, positions, q, k, v, q_out=None, out=None, lse=None, out_dtype="f32", want_lse=True,
                              stream=None):
        """sk_batch_step with q and k turned on the way by int32 positions [tokens] -> (q_out, out, lse)"""
        n, T = len(session_ids), int(cu_tokens[-1])
        q_out = self._turns(q, q_out, self.Hq, T, positions, stream)
        sid, op, cu = array.array("i", session_ids), array.array("i", ops), array.array("i", cu_tokens)
        assert len(op) == n and len(cu) == n + 1
        read = n                                             # behind the last item whose k and v are read
        while read and op[read - 1] == SK_OP_QUERY_A:
            read -= 1
        if cu[read]:
            for x in (k, v):
                if x is not None:                            # (left out: refused by the call)
                    self._own(x, cu[read])
        if out is None:
            out, lse = self._out(T, out_dtype, want_lse, stream)
        else:
            self._results(out, lse, out_dtype, T)
        _ck(lib().sk_batch_step_rotated(self.h, n, sid.buffer_info()[0], op.buffer_info()[0], cu.buffer_info()[0], _p(positions), _p(q), _p(k), _p(v),
                                        _p(q_out), _p(out), _dt(out_dtype), _p(lse), _stream(stream)), "sk_batch_step_rotated")
        return q_out, out, lse

    def sk_session_shift(self, sid, delta, first=0, count=None, stream=None):
        """Turns the cached keys of retained tokens first .. first + count - 1 on by delta positions: a number, or CUDA int32 [count] or
        [Hkv, count] (rows may be strided)."""
        count = self._length(sid) - first if count is None else int(count)
        deltas, stride, by = None, 0, 0
        if isinstance(delta, torch.Tensor):
            assert delta.dtype is torch.int32 and delta.is_cuda and delta.dim() in (1, 2) and delta.shape[-1] == count and (delta.stride(-1) == 1 or count <= 1)
            assert delta.dim() == 1 or delta.shape[0] == self.Hkv
            deltas = delta.data_ptr() if count else None
            # (one row, or one that stands for all: any stride)
            stride = delta.stride(0) if delta.dim() == 2 and self.Hkv > 1 else 0
        else:
            by = int(delta)
        _ck(lib().sk_session_shift(self.h, sid, int(first), count, by, deltas, stride, _stream(stream) if self.kv_mem is not None else None),
            "sk_session_shift")

    def sk_session_gather(self, sid, first=0, count=None, stream=None):
        if count is None:
            count = self.sk_session_length(sid) - first
        k = torch.empty((count, self.Hkv, self.d), dtype=self.torch_dtype, device=self.device)
        v = torch.empty_like(k)
        _made(stream, k, v)
        _ck(lib().sk_session_gather(self.h, sid, first, count, _p(k), _p(v), _stream(stream)), "sk_session_gather")
        return k, v


def top2_outputs(rows, device):
    """Output tensors of sk_top2 / sk_top2_static for `rows` rows: (idx1, idx2, val1, val2, gap)."""
    idx1 = torch.empty(rows, dtype=torch.int32, device=device)
    val1 = torch.empty(rows, dtype=torch.float32, device=device)
    return idx1, torch.empty_like(idx1), val1, torch.empty_like(val1), torch.empty_like(val1)


def sk_top2_static(logits, outputs=None, stream=None):
    """sk_top2 through the entry point that allocates nothing: `outputs` (see top2_outputs) are the
    caller's; they are only made here when left out."""
    assert logits.is_cuda and logits.dtype == torch.float32 and logits.dim() == 2 and logits.stride(1) == 1
    rows, vocab = logits.shape
    if outputs is None:
        outputs = top2_outputs(rows, logits.device)
        _made(stream, *outputs)
    idx1, idx2, val1, val2, gap = outputs
    _ck(lib().sk_top2_static(logits.data_ptr() if rows else None, rows, vocab,
                             logits.stride(0) if rows else vocab, _p(idx1), _p(idx2), _p(val1), _p(val2), _p(gap),
                             _stream(stream)), "sk_top2_static")
    return outputs


def sk_top2(logits, stream=None, workspace=None, outputs=None):
    """logits: CUDA float32 tensor [rows, vocab] (rows may be strided by a multiple of 4 elements).
    Returns (idx1, idx2, val1, val2, gap), each [rows]."""
    assert logits.is_cuda and logits.dtype == torch.float32 and logits.dim() == 2 and logits.stride(1) == 1
    rows, vocab = logits.shape
    if workspace is None:
        workspace = torch.empty(max(lib().sk_top2_workspace_bytes(rows, vocab), 16), dtype=torch.uint8, device=logits.device)
        _made(stream, workspace)
    if outputs is None:
        outputs = top2_outputs(rows, logits.device)
        _made(stream, *outputs)
    idx1, idx2, val1, val2, gap = outputs
    _ck(lib().sk_top2(logits.data_ptr() if rows else None, rows, vocab, logits.stride(0) if rows else vocab, _p(workspace),
                      workspace.numel(), _p(idx1), _p(idx2), _p(val1), _p(val2), _p(gap), _stream(stream)), "sk_top2")
    return idx1, idx2, val1, val2, gap


def logprobs_outputs(rows, n_tokens, n_top, device):
    """Output tensors of sk_logprobs: (logprob [rows, n_tokens], lse [rows], entropy [rows], top_idx [rows, n_top], top_logprob)."""
    f32 = dict(dtype=torch.float32, device=device)
    return (torch.empty((rows, n_tokens), **f32), torch.empty(rows, **f32), torch.empty(rows, **f32),
            torch.empty((rows, n_top), dtype=torch.int32, device=device), torch.empty((rows, n_top), **f32))


def sk_logprobs(logits, tokens=None, n_top=0, workspace=None, outputs=None, stream=None):
    """logits: CUDA float32 or bfloat16 tensor [rows, vocab] (rows may be strided); tokens: CUDA int32 [rows, n_tokens] (or [rows]) or
    None.  Returns (logprob [rows, n_tokens], lse [rows], entropy [rows], top_idx [rows, n_top], top_logprob [rows, n_top])."""
    assert logits.is_cuda and logits.dtype in (torch.float32, torch.bfloat16) and logits.dim() == 2 and (logits.stride(1) == 1 or logits.shape[1] == 1)
    rows, vocab = logits.shape
    n_tokens = 0
    if tokens is not None:
        tokens = tokens.view(rows, 1) if tokens.dim() == 1 else tokens
        assert tokens.dtype == torch.int32 and tokens.device == logits.device and tokens.shape[0] == rows and tokens.dim() == 2
        n_tokens = tokens.shape[1]
    if outputs is None:
        outputs = logprobs_outputs(rows, n_tokens, n_top, logits.device)
        _made(stream, *outputs)
    logprob, lse, entropy, top_idx, top_logprob = outputs
    assert top_idx is None or (top_idx.dtype is torch.int32 and top_idx.numel() == rows * n_top and top_idx.is_cuda)
    for t, n in ((logprob, rows * n_tokens), (lse, rows), (entropy, rows), (top_logprob, rows * n_top)):
        assert t is None or (t.dtype is torch.float32 and t.numel() == n and t.is_cuda)
    if workspace is None:
        workspace = torch.empty(max(lib().sk_logprobs_workspace_bytes(rows, vocab, n_top), 16), dtype=torch.uint8, device=logits.device)
        _made(stream, workspace)
    # (a single row may have any stride)
    _ck(lib().sk_logprobs(logits.data_ptr() if rows else None, _dt(logits.dtype), rows, vocab, logits.stride(0) if rows > 1 else vocab, _p(tokens), n_tokens,
                          n_top, _p(workspace), workspace.numel() * workspace.element_size(), _p(logprob), _p(lse), _p(entropy), _p(top_idx), _p(top_logprob),
                          _stream(stream)), "sk_logprobs")
    return outputs


def verify_outputs(n_seq, n_draft, device):
    """Output tensors of sk_verify: (n_accepted [n_seq], tokens [n_seq, n_draft + 1], logprob [n_seq, n_draft + 1])."""
    i32 = dict(dtype=torch.int32, device=device)
    return torch.empty(n_seq, **i32), torch.empty((n_seq, n_draft + 1), **i32), torch.empty((n_seq, n_draft + 1), dtype=torch.float32, device=device)


def sk_verify(target, tokens, uniform, draft=None, temperature=None, workspace=None, outputs=None, stream=None):
    """target: CUDA float32 or bfloat16 logits [n_seq, n_draft + 1, vocab]; tokens: int32 [n_seq, n_draft]; uniform: float32 [n_seq, n_draft + 1];
    draft: the logits that the tokens were drawn from [n_seq, n_draft, vocab], or None; temperature: float32 [n_seq] or None.  Rows of logits may be
    strided, evenly over sequences and places.  Returns (n_accepted [n_seq], tokens [n_seq, n_draft + 1], logprob [n_seq, n_draft + 1])."""
    assert target.is_cuda and target.dtype in (torch.float32, torch.bfloat16) and target.dim() == 3
    n_seq, places, vocab = target.shape
    n_draft, on = places - 1, target.get_device()

    def rows(x, n):                                          # address and row stride of [n_seq, n, vocab]
        s0, s1, s2 = x.stride()
        stride = s1 if n > 1 else s0 if n_seq > 1 else vocab
        assert (s2 == 1 or vocab == 1) and (n <= 1 or n_seq <= 1 or s0 == n * stride)
        return x.data_ptr() if n_seq else None, stride

    pt, st = rows(target, places)
    pd, sd = None, 0
    if draft is not None:
        assert draft.dtype is target.dtype and draft.shape == (n_seq, n_draft, vocab) and draft.get_device() == on
        pd, sd = rows(draft, n_draft) if n_draft else (None, 0)
    assert tokens.dtype is torch.int32 and tokens.shape == (n_seq, n_draft) and tokens.get_device() == on
    assert uniform.dtype is torch.float32 and uniform.shape == (n_seq, places) and uniform.get_device() == on
    assert temperature is None or (temperature.dtype is torch.float32 and temperature.shape == (n_seq,) and temperature.get_device() == on)
    if outputs is None:
        outputs = verify_outputs(n_seq, n_draft, target.device)
        _made(stream, *outputs)
        n_accepted, out_tokens, logprob = outputs
    else:
        n_accepted, out_tokens, logprob = outputs
        assert n_accepted.dtype is torch.int32 and n_accepted.numel() == n_seq and n_accepted.get_device() == on
        assert out_tokens.dtype is torch.int32 and out_tokens.numel() == n_seq * places and out_tokens.get_device() == on
        assert logprob is None or (logprob.dtype is torch.float32 and logprob.numel() == n_seq * places and logprob.get_device() == on)
    L = lib()
    if workspace is None:
        workspace = torch.empty(max(L.sk_verify_workspace_bytes(n_seq, n_draft, vocab), 16), dtype=torch.uint8, device=target.device)
        _made(stream, workspace)
    _ck(L.sk_verify(pt, st, pd, sd, SK_F32 if target.dtype is torch.float32 else SK_BF16, n_seq, n_draft, vocab, _p(tokens), _p(uniform), _p(temperature),
                    _p(workspace), workspace.numel() * workspace.element_size(), _p(n_accepted), _p(out_tokens), _p(logprob), _stream(stream)), "sk_verify")
    return outputs


def sk_probe_read(buf, n_workgroups, sink, stream=None, nbytes=None, non_temporal=False):
    """Plain streaming read of a CUDA tensor (measurement probe)."""
    nbytes = buf.numel() * buf.element_size() if nbytes is None else int(nbytes)
    _ck(lib().sk_probe_read(_p(buf), nbytes, int(n_workgroups), int(bool(non_temporal)), _p(sink), _stream(stream)), "sk_probe_read")


def sk_probe_mfma(n_workgroups, iters, sink, operands=None, stream=None):
    """Back-to-back bf16 matrix products on register operands (measurement probe), the operands taken
    from the bf16 CUDA tensor `operands` if given; returns the flops of the launch."""
    f = ctypes.c_double()
    nb = 0 if operands is None else operands.numel() * operands.element_size()
    _ck(lib().sk_probe_mfma(int(n_workgroups), int(iters), _p(operands), nb, _p(sink), ctypes.byref(f), _stream(stream)),
        "sk_probe_mfma")
    return f.value
