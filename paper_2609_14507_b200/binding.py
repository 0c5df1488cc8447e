"""Thin ctypes binding of the C-ABI library (``include/ipkv.h``): argument marshalling only.

Every step of the path runs in the library's CUDA kernels; there is no Python or CPU fallback.
If ``libipkv.so`` is missing or cannot be loaded, :func:`lib` raises.

Tensors are passed as ``torch`` tensors (device or host); this module only takes their
``data_ptr()`` and the current CUDA stream.
"""
import ctypes as C
import os
import struct

HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(HERE, "libipkv.so")

GQA, MLA = 0, 1
REGION_U, REGION_P, REGION_W = 0, 1, 2
LAYOUT_PLAIN, LAYOUT_TILE = 0, 1
FLAG_NO_HOST_U, FLAG_NO_HOST_P, FLAG_GROW_P = 1, 2, 4
ATTEND_STATIC_SCHEDULE, ATTEND_BALANCE = 1, 2
OK = 0
STATUS_NAMES = {0: "OK", 1: "EINVAL", 2: "ENOMEM", 3: "ERANGE", 4: "ESTATE", 5: "ECUDA", 6: "ETIMEOUT", 7: "EINTERNAL"}

EXPORTS = [
    "ipkv_query_sizes", "ipkv_create", "ipkv_destroy", "ipkv_set_share", "ipkv_reset", "ipkv_append_bulk",
    "ipkv_append", "ipkv_flush", "ipkv_attend_gpu", "ipkv_attend_gpu_sparse", "ipkv_attend_cpu", "ipkv_merge", "ipkv_views", "ipkv_locate", "ipkv_counts",
    "ipkv_read_token", "ipkv_get_stats", "ipkv_profile_enable", "ipkv_profile_read", "ipkv_attend_scratch_bytes", "ipkv_attend_runs", "ipkv_pack_blocks",
    "ipkv_attend_runs_noalloc", "ipkv_noalloc_scratch_limit", "ipkv_roofline_share", "ipkv_roofline_step_time",
    "ipkv_policy_create", "ipkv_policy_destroy", "ipkv_policy_observe", "ipkv_policy_update", "ipkv_policy_prefill_share",
    "ipkv_block_bytes", "ipkv_status_str", "ipkv_last_error", "ipkv_version", "ipkv_probe_read_bandwidth",
    "ipkv_selftest_expire_wait", "ipkv_selftest_fail_next_launch", "ipkv_selftest_declare_bounds", "ipkv_probe_umma",
    "ipkv_norm_rope", "ipkv_nibble_block_bytes", "ipkv_nibble_pack", "ipkv_nibble_unpack",
    "ipkv_nibble_scratch_bytes", "ipkv_nibble_attend",
]


class Config(C.Structure):
    _fields_ = [
        ("struct_size", C.c_uint32), ("kind", C.c_int32), ("n_layers", C.c_int32), ("max_seqs", C.c_int32),
        ("n_q_heads", C.c_int32), ("n_kv_heads", C.c_int32), ("dim_qk", C.c_int32), ("dim_v", C.c_int32),
        ("block_tokens", C.c_int32), ("window_tokens", C.c_int32), ("chunk_tokens", C.c_int32), ("n_slots", C.c_int32),
        ("max_u_tokens_per_seq", C.c_int64), ("max_p_tokens_per_seq", C.c_int64), ("resident_tokens_per_seq", C.c_int64),
        ("p_initial_tokens_per_seq", C.c_int64),
        ("softmax_scale", C.c_float), ("share_num", C.c_int32), ("share_den", C.c_int32), ("device", C.c_int32),
        ("flags", C.c_uint32),
        ("u_host", C.c_void_p), ("u_bytes", C.c_size_t), ("p_host_pinned", C.c_void_p), ("p_bytes", C.c_size_t),
        ("w_dev", C.c_void_p), ("w_bytes", C.c_size_t), ("resident_dev", C.c_void_p), ("resident_bytes", C.c_size_t),
        ("pp_dev", C.c_void_p), ("pp_bytes", C.c_size_t),
        ("resident_tokens_by_seq", C.POINTER(C.c_int64)),
    ]


class AttendOpts(C.Structure):
    _fields_ = [("kv_splits", C.c_int32), ("flags", C.c_int32), ("side_stream", C.c_void_p),
                ("fold_o_dev", C.c_void_p), ("fold_lse_dev", C.c_void_p), ("append_k_dev", C.c_void_p), ("append_v_dev", C.c_void_p)]


class Extent(C.Structure):
    _fields_ = [("region", C.c_int32), ("layout", C.c_int32), ("first_token", C.c_int64), ("n_tokens", C.c_int64),
                ("region_block", C.c_int64), ("host_ptr", C.c_void_p), ("dev_ptr", C.c_void_p), ("block_bytes", C.c_int64)]


class Stats(C.Structure):
    _fields_ = [(n, C.c_uint64) for n in (
        "attend_calls", "attend_kernels", "reduce_kernels", "merge_kernels", "append_kernels", "pack_kernels",
        "kv_bytes_attended", "h2d_bytes", "d2h_bytes", "d2d_bytes", "flushes", "flushes_to_u", "fused_appends", "early_launches",
        "p_segments", "p_pinned_bytes", "p_pin_us", "p_grow_waits", "p_grow_wait_us",
        "p_register_us", "p_register_calls", "p_register_max_us")] + [("device_status", C.c_uint32)]


class AttnShape(C.Structure):
    _fields_ = [("kind", C.c_int32), ("n_q_heads", C.c_int32), ("n_kv_heads", C.c_int32), ("dim_qk", C.c_int32),
                ("dim_v", C.c_int32), ("block_tokens", C.c_int32), ("softmax_scale", C.c_float)]


class Run(C.Structure):
    _fields_ = [("blocks_dev", C.c_void_p), ("n_tokens", C.c_int64)]


class Rope(C.Structure):
    _fields_ = [("dim", C.c_int32), ("rot_dim", C.c_int32), ("n_axes", C.c_int32), ("interleaved", C.c_int32), ("eps", C.c_float),
                ("theta", C.c_double), ("inv_freq", C.c_void_p), ("pair_axis", C.c_char_p)]


class Heads(C.Structure):
    _fields_ = [("in_dev", C.c_void_p), ("out_dev", C.c_void_p), ("weight_dev", C.c_void_p), ("n_heads", C.c_int32),
                ("in_token_stride", C.c_int64), ("in_head_stride", C.c_int64), ("out_token_stride", C.c_int64), ("out_head_stride", C.c_int64)]


class Span(C.Structure):
    _fields_ = [("blocks_dev", C.c_void_p), ("first_token", C.c_int64), ("n_tokens", C.c_int64)]


class Roofline(C.Structure):
    _fields_ = [("A", C.c_double), ("B", C.c_double), ("C_cpu", C.c_double), ("C_gpu", C.c_double)]


class IpkvError(RuntimeError):
    def __init__(self, status, where, detail=""):
        self.status = status
        super().__init__(f"{where}: {STATUS_NAMES.get(status, status)} {detail}".strip())


_lib = None


def lib():
    """Load ``libipkv.so`` (built by ``paper_2609_14507_b200.build``); raises if it is absent.  With IPKV_LIB_VARIANT=checked
    in the environment the bounds-checked build ``libipkv_checked.so`` is loaded instead (same ABI)."""
    global _lib, LIB_PATH
    if _lib is not None:
        return _lib
    if os.environ.get("IPKV_LIB_VARIANT") == "checked":
        LIB_PATH = os.path.join(os.path.dirname(LIB_PATH), "libipkv_checked.so")
    if not os.path.exists(LIB_PATH):
        raise RuntimeError(f"{LIB_PATH} is missing: build it with `python -m paper_2609_14507_b200.build` "
                           "(there is no fallback path)")
    L = C.CDLL(LIB_PATH)
    vp, i32, i64 = C.c_void_p, C.c_int32, C.c_int64
    sig = {
        "ipkv_query_sizes": [C.POINTER(Config), C.POINTER(C.c_size_t)],
        "ipkv_create": [C.POINTER(Config), C.POINTER(vp)],
        "ipkv_destroy": [vp],
        "ipkv_set_share": [vp, i32],
        "ipkv_reset": [vp, i32],
        "ipkv_append_bulk": [vp, i32, i32, vp, vp, i64, i32, i32, vp],
        "ipkv_append": [vp, i32, C.POINTER(i32), i32, vp, vp, vp],
        "ipkv_flush": [vp, i32, i32, vp],
        "ipkv_attend_gpu": [vp, i32, C.POINTER(i32), i32, vp, C.POINTER(AttendOpts), vp, vp, vp],
        "ipkv_attend_gpu_sparse": [vp, i32, C.POINTER(i32), i32, vp, C.POINTER(i64), C.POINTER(i32), i32, C.POINTER(AttendOpts),
                                   vp, vp, vp],
        "ipkv_attend_cpu": [vp, i32, C.POINTER(i32), i32, vp, vp, vp, i32],
        "ipkv_merge": [vp, i32, i32, i32, C.POINTER(vp), C.POINTER(vp), vp, i32, vp, vp],
        "ipkv_views": [vp, i32, i32, C.POINTER(Extent), i32, C.POINTER(i32)],
        "ipkv_locate": [vp, i32, i32, i64, C.POINTER(i32), C.POINTER(i64), C.POINTER(i32)],
        "ipkv_counts": [vp, i32, i32, C.POINTER(i64)],
        "ipkv_read_token": [vp, i32, i32, i64, vp, vp],
        "ipkv_get_stats": [vp, C.POINTER(Stats)],
        "ipkv_selftest_expire_wait": [vp, C.c_uint32, vp],
        "ipkv_selftest_fail_next_launch": [vp],
        "ipkv_selftest_declare_bounds": [vp, i32, i64],
        "ipkv_profile_enable": [vp, i32],
        "ipkv_profile_read": [vp, C.POINTER(C.c_double), C.POINTER(i64), C.POINTER(i64)],
        "ipkv_attend_scratch_bytes": [C.POINTER(AttnShape), i32, i32, i64, i32, C.POINTER(C.c_size_t)],
        "ipkv_attend_runs": [C.POINTER(AttnShape), i32, C.POINTER(Run), C.POINTER(i32), vp, i32, vp, C.c_size_t, vp, vp, vp, vp],
        "ipkv_pack_blocks": [C.POINTER(AttnShape), i32, vp, vp, i64, vp, vp],
        "ipkv_norm_rope": [C.POINTER(Rope), i64, vp, i32, vp, vp],
        "ipkv_nibble_pack": [C.POINTER(AttnShape), i32, vp, i64, vp, vp, i64, i64, vp],
        "ipkv_nibble_unpack": [C.POINTER(AttnShape), i32, vp, i64, vp, vp, i64, i64, vp],
        "ipkv_nibble_scratch_bytes": [C.POINTER(AttnShape), i32, i32, C.POINTER(C.c_size_t)],
        "ipkv_nibble_attend": [C.POINTER(AttnShape), i32, vp, vp, vp, vp, C.c_size_t, vp, vp, vp, vp],
        "ipkv_attend_runs_noalloc": [C.POINTER(AttnShape), i32, C.POINTER(Run), C.POINTER(i32), vp, i32, vp, vp, vp, vp],
    }
    L.ipkv_version.restype = C.c_char_p
    L.ipkv_version_bytes = lambda: L.ipkv_version()
    for name, args in sig.items():
        f = getattr(L, name)
        f.argtypes = args
        f.restype = C.c_int
    L.ipkv_block_bytes.argtypes = [C.POINTER(AttnShape)]
    L.ipkv_block_bytes.restype = C.c_int64
    L.ipkv_nibble_block_bytes.argtypes = [C.POINTER(AttnShape)]
    L.ipkv_nibble_block_bytes.restype = C.c_int64
    L.ipkv_roofline_share.argtypes = [C.POINTER(Roofline), C.c_double]
    L.ipkv_roofline_share.restype = C.c_double
    L.ipkv_roofline_step_time.argtypes = [C.POINTER(Roofline), C.c_double, C.c_double, C.c_double, C.POINTER(C.c_double), C.POINTER(C.c_double)]
    L.ipkv_roofline_step_time.restype = C.c_double
    L.ipkv_policy_create.argtypes = [C.POINTER(Roofline), i32, i32, C.POINTER(vp)]
    L.ipkv_policy_destroy.argtypes = [vp]
    L.ipkv_policy_observe.argtypes = [vp, C.c_double, C.c_double]
    L.ipkv_policy_update.argtypes = [vp, C.POINTER(i32), C.POINTER(Roofline)]
    L.ipkv_policy_prefill_share.argtypes = [vp, C.c_double, C.POINTER(i32)]
    for name in ("ipkv_policy_create", "ipkv_policy_destroy", "ipkv_policy_observe", "ipkv_policy_update", "ipkv_policy_prefill_share"):
        getattr(L, name).restype = C.c_int
    L.ipkv_noalloc_scratch_limit.argtypes = []
    L.ipkv_noalloc_scratch_limit.restype = C.c_size_t
    L.ipkv_status_str.argtypes = [C.c_int]
    L.ipkv_status_str.restype = C.c_char_p
    L.ipkv_last_error.argtypes = [vp]
    L.ipkv_last_error.restype = C.c_char_p
    L.ipkv_version.argtypes = []
    L.ipkv_version.restype = C.c_char_p
    _lib = L
    return L


def _ptr(t):
    if t is None:
        return None
    if isinstance(t, int):
        return t
    return t.data_ptr()


def _stream(stream):
    if stream is None:
        import torch
        return torch.cuda.current_stream().cuda_stream
    if isinstance(stream, int):
        return stream
    return stream.cuda_stream


def _ids(seq_ids):
    if isinstance(seq_ids, tuple) and len(seq_ids) == 2 and isinstance(seq_ids[1], int) and not isinstance(seq_ids[0], int):
        return seq_ids                       # already marshalled by seq_id_array()
    arr = (C.c_int32 * len(seq_ids))(*[int(s) for s in seq_ids])
    return arr, len(seq_ids)


def seq_id_array(seq_ids):
    """Marshal a list of sequence ids once; the result can be passed wherever seq_ids is expected."""
    return (C.c_int32 * len(seq_ids))(*[int(s) for s in seq_ids]), len(seq_ids)


def make_config(kind, n_layers, max_seqs, n_q_heads, n_kv_heads, dim_qk, dim_v, *, block_tokens=64,
                window_tokens=256, chunk_tokens=512, n_slots=2, max_u_tokens_per_seq=0, max_p_tokens_per_seq=0,
                resident_tokens_per_seq=0, softmax_scale=0.0, share_num=0, share_den=1, device=0, flags=0,
                p_initial_tokens_per_seq=0, resident_tokens_by_seq=None):
    c = Config()
    c.struct_size = C.sizeof(Config)
    c.kind, c.n_layers, c.max_seqs = kind, n_layers, max_seqs
    c.n_q_heads, c.n_kv_heads, c.dim_qk, c.dim_v = n_q_heads, n_kv_heads, dim_qk, dim_v
    c.block_tokens, c.window_tokens, c.chunk_tokens, c.n_slots = block_tokens, window_tokens, chunk_tokens, n_slots
    c.max_u_tokens_per_seq, c.max_p_tokens_per_seq = max_u_tokens_per_seq, max_p_tokens_per_seq
    c.resident_tokens_per_seq = resident_tokens_per_seq
    c.p_initial_tokens_per_seq = p_initial_tokens_per_seq
    c.softmax_scale = softmax_scale
    c.share_num, c.share_den, c.device, c.flags = share_num, share_den, device, flags
    if resident_tokens_by_seq is not None:                  # per-sequence ring capacities (read by query_sizes / create only)
        if len(resident_tokens_by_seq) != max_seqs:
            raise ValueError("resident_tokens_by_seq needs one entry per sequence")
        c._ring_keepalive = (C.c_int64 * max_seqs)(*[int(x) for x in resident_tokens_by_seq])
        c.resident_tokens_by_seq = C.cast(c._ring_keepalive, C.POINTER(C.c_int64))
    return c


class UmmaTiming(C.Structure):
    _fields_ = [("m", C.c_int32), ("n", C.c_int32), ("n_mma", C.c_int32), ("accumulators", C.c_int32),
                ("issue_cycles", C.c_int64), ("total_cycles", C.c_int64)]


def ipkv_probe_umma(device=0, reps=5):
    """List of dicts: SM clocks for n back-to-back tcgen05.mma of small shapes (see ipkv.h)."""
    out = (UmmaTiming * 64)()
    n = C.c_int32()
    f = lib().ipkv_probe_umma
    f.argtypes = [C.c_int32, C.c_int32, C.POINTER(UmmaTiming), C.c_int32, C.POINTER(C.c_int32)]
    rc = f(device, reps, out, 64, C.byref(n))
    if rc != OK:
        raise IpkvError(rc, "ipkv_probe_umma")
    return [{k: getattr(out[i], k) for k, _ in UmmaTiming._fields_} for i in range(n.value)]


def ipkv_probe_read_bandwidth(device=0, nbytes=1 << 30, reps=10):
    """(best, mean) GB/s of a read-only stream through the attention kernels' copy ring, no arithmetic."""
    best, mean = C.c_double(), C.c_double()
    lib().ipkv_probe_read_bandwidth.argtypes = [C.c_int32, C.c_size_t, C.c_int32, C.POINTER(C.c_double), C.POINTER(C.c_double)]
    rc = lib().ipkv_probe_read_bandwidth(device, nbytes, reps, C.byref(best), C.byref(mean))
    if rc != OK:
        raise IpkvError(rc, "ipkv_probe_read_bandwidth")
    return best.value, mean.value


def ipkv_query_sizes(cfg):
    out = (C.c_size_t * 5)()
    rc = lib().ipkv_query_sizes(C.byref(cfg), out)
    if rc != OK:
        raise IpkvError(rc, "ipkv_query_sizes")
    return dict(u=out[0], p=out[1], w=out[2], resident=out[3], pp=out[4])


class Cache:
    """Owner of one ``ipkv_t`` handle; methods carry the C names without the prefix."""

    def __init__(self, cfg):
        self.cfg = cfg
        h = C.c_void_p()
        rc = lib().ipkv_create(C.byref(cfg), C.byref(h))
        if rc != OK:
            raise IpkvError(rc, "ipkv_create")
        self._h = h

    def close(self):
        if getattr(self, "_h", None):
            lib().ipkv_destroy(self._h)
            self._h = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def __enter__(self):
        return self

    def __exit__(self, *a):
        self.close()

    def _check(self, rc, where):
        if rc != OK:
            raise IpkvError(rc, where, lib().ipkv_last_error(self._h).decode())

    def set_share(self, num):
        self._check(lib().ipkv_set_share(self._h, num), "ipkv_set_share")

    def reset(self, seq=-1):
        self._check(lib().ipkv_reset(self._h, seq), "ipkv_reset")

    def append_bulk(self, layer, seq, k, v, n_tokens, num0, den0, stream=None):
        self._check(lib().ipkv_append_bulk(self._h, layer, seq, _ptr(k), _ptr(v), n_tokens, num0, den0, _stream(stream)),
                    "ipkv_append_bulk")

    def append(self, layer, seq_ids, k, v, stream=None):
        ids, n = _ids(seq_ids)
        self._check(lib().ipkv_append(self._h, layer, ids, n, _ptr(k), _ptr(v), _stream(stream)), "ipkv_append")

    def flush(self, layer=-1, seq=-1, stream=None):
        self._check(lib().ipkv_flush(self._h, layer, seq, _stream(stream)), "ipkv_flush")

    def attend_gpu(self, layer, seq_ids, q, o_part, lse_part, kv_splits=0, side_stream=None, stream=None,
                   fold_o=None, fold_lse=None, static_schedule=False, force_balance=False, append_k=None, append_v=None):
        """append_k / append_v: one new token per listed sequence, appended first (fused into the kernel where possible)."""
        ids, n = _ids(seq_ids)
        opts = AttendOpts(kv_splits, (ATTEND_STATIC_SCHEDULE if static_schedule else 0) | (ATTEND_BALANCE if force_balance else 0),
                          _stream(side_stream) if side_stream is not None else None, _ptr(fold_o), _ptr(fold_lse),
                          _ptr(append_k), _ptr(append_v))
        self._check(lib().ipkv_attend_gpu(self._h, layer, ids, n, _ptr(q), C.byref(opts), _ptr(o_part), _ptr(lse_part),
                                          _stream(stream)), "ipkv_attend_gpu")

    def attend_gpu_call(self, layer, seq_ids, q, o_part, lse_part, kv_splits=0, side_stream=None, stream=None,
                        fold_o=None, fold_lse=None, static_schedule=False, force_balance=False, append_k=None, append_v=None):
        """The same call as attend_gpu with its arguments marshalled once: returns a function of no arguments that issues
        ipkv_attend_gpu on the given buffers (for loops that call a layer with the same tensors every step)."""
        ids, n = _ids(seq_ids)
        opts = AttendOpts(kv_splits, (ATTEND_STATIC_SCHEDULE if static_schedule else 0) | (ATTEND_BALANCE if force_balance else 0),
                          _stream(side_stream) if side_stream is not None else None, _ptr(fold_o), _ptr(fold_lse),
                          _ptr(append_k), _ptr(append_v))
        fn, check = lib().ipkv_attend_gpu, self._check
        args = (self._h, layer, ids, n, _ptr(q), C.byref(opts), _ptr(o_part), _ptr(lse_part), _stream(stream))
        keep = (opts, ids, q, o_part, lse_part, fold_o, fold_lse, append_k, append_v)      # the buffers stay alive with the call

        def call(_keep=keep):
            rc = fn(*args)
            if rc != OK:
                check(rc, "ipkv_attend_gpu")
        return call

    def attend_gpu_sparse(self, layer, seq_ids, q, blocks_per_row, o_part, lse_part, include_window=True, kv_splits=0,
                          stream=None, fold_o=None, fold_lse=None, static_schedule=False):
        """Attention over the D-window plus the listed whole P blocks of every row (block ordinals in region P)."""
        ids, n = _ids(seq_ids)
        flat, start = [], [0]
        for row in blocks_per_row:
            flat += [int(b) for b in row]
            start.append(len(flat))
        blocks = (C.c_int64 * max(1, len(flat)))(*flat)
        starts = (C.c_int32 * len(start))(*start)
        opts = AttendOpts(kv_splits, ATTEND_STATIC_SCHEDULE if static_schedule else 0, None, _ptr(fold_o), _ptr(fold_lse))
        self._check(lib().ipkv_attend_gpu_sparse(self._h, layer, ids, n, _ptr(q), blocks, starts, 1 if include_window else 0,
                                                 C.byref(opts), _ptr(o_part), _ptr(lse_part), _stream(stream)), "ipkv_attend_gpu_sparse")

    def attend_cpu(self, layer, seq_ids, q_host, o_part_host, lse_part_host, n_threads=0):
        """CPU-side engine over the tokens routed to U; all tensors in host memory."""
        ids, n = _ids(seq_ids)
        self._check(lib().ipkv_attend_cpu(self._h, layer, ids, n, _ptr(q_host), _ptr(o_part_host), _ptr(lse_part_host), n_threads),
                    "ipkv_attend_cpu")

    def merge(self, n_rows, dim_v, o_parts, lse_parts, o_out, lse_out=None, out_is_bf16=False, stream=None):
        ipkv_merge(n_rows, dim_v, o_parts, lse_parts, o_out, lse_out, out_is_bf16, stream, handle=self)

    def views(self, layer, seq):
        n = C.c_int32()
        self._check(lib().ipkv_views(self._h, layer, seq, None, 0, C.byref(n)), "ipkv_views")
        arr = (Extent * max(1, n.value))()
        self._check(lib().ipkv_views(self._h, layer, seq, arr, n.value, C.byref(n)), "ipkv_views")
        return [arr[i] for i in range(n.value)]

    def locate(self, layer, seq, token):
        r, b, o = C.c_int32(), C.c_int64(), C.c_int32()
        self._check(lib().ipkv_locate(self._h, layer, seq, token, C.byref(r), C.byref(b), C.byref(o)), "ipkv_locate")
        return r.value, b.value, o.value

    def counts(self, layer, seq):
        c = (C.c_int64 * 6)()
        self._check(lib().ipkv_counts(self._h, layer, seq, c), "ipkv_counts")
        return dict(n_u=c[0], n_p=c[1], n_w=c[2], n_p_resident=c[3], n_flush=c[4], n_flush_cpu=c[5])

    def read_token(self, layer, seq, token):
        """(K [Hkv][dqk], V [Hkv][dv] or None) of one token as NumPy uint16 bf16 bits."""
        import numpy as np
        cfg = self.cfg
        k = np.zeros((cfg.n_kv_heads, cfg.dim_qk), dtype=np.uint16)
        v = None if cfg.kind == MLA else np.zeros((cfg.n_kv_heads, cfg.dim_v), dtype=np.uint16)
        self._check(lib().ipkv_read_token(self._h, layer, seq, token, k.ctypes.data, v.ctypes.data if v is not None else None),
                    "ipkv_read_token")
        return k, v

    def profile_enable(self, on=True, reduce=False, every=1):
        """Time every `every`-th attention-kernel launch (or, with reduce=True, split-reduce launch) with CUDA events."""
        self._check(lib().ipkv_profile_enable(self._h, ((2 if reduce else 1) + 256 * max(1, int(every))) if on else 0), "ipkv_profile_enable")

    def profile_read(self):
        """(summed attention-kernel milliseconds, launches timed, launches seen) since the last read."""
        ms, nt, nl = C.c_double(), C.c_int64(), C.c_int64()
        self._check(lib().ipkv_profile_read(self._h, C.byref(ms), C.byref(nt), C.byref(nl)), "ipkv_profile_read")
        return ms.value, nt.value, nl.value

    def get_stats(self):
        s = Stats()
        self._check(lib().ipkv_get_stats(self._h, C.byref(s)), "ipkv_get_stats")
        return {n: getattr(s, n) for n, _ in Stats._fields_}

    def selftest_declare_bounds(self, base_id, nbytes):
        self._check(lib().ipkv_selftest_declare_bounds(self._h, base_id, nbytes), "ipkv_selftest_declare_bounds")

    def selftest_fail_next_launch(self):
        self._check(lib().ipkv_selftest_fail_next_launch(self._h), "ipkv_selftest_fail_next_launch")

    def selftest_expire_wait(self, limit_us, stream=None):
        self._check(lib().ipkv_selftest_expire_wait(self._h, limit_us, _stream(stream)), "ipkv_selftest_expire_wait")


def ipkv_merge(n_rows, dim_v, o_parts, lse_parts, o_out, lse_out=None, out_is_bf16=False, stream=None, handle=None):
    n = len(o_parts)
    op = (C.c_void_p * n)(*[_ptr(t) for t in o_parts])
    lp = (C.c_void_p * n)(*[_ptr(t) for t in lse_parts])
    h = handle._h if handle is not None else None
    rc = lib().ipkv_merge(h, n_rows, dim_v, n, op, lp, _ptr(o_out), 1 if out_is_bf16 else 0, _ptr(lse_out), _stream(stream))
    if rc != OK:
        raise IpkvError(rc, "ipkv_merge", lib().ipkv_last_error(h).decode() if h else "")


def ipkv_roofline_share(A, B, C_cpu, C_gpu, L):
    """Eq. 2: the CPU share that balances the two engines at placed length L."""
    return float(lib().ipkv_roofline_share(C.byref(Roofline(A, B, C_cpu, C_gpu)), L))


def ipkv_roofline_step_time(A, B, C_cpu, C_gpu, r, L, t_merge=0.0):
    """Eq. 1: (T, T_CPU, T_GPU) at share r."""
    tc, tg = C.c_double(), C.c_double()
    t = lib().ipkv_roofline_step_time(C.byref(Roofline(A, B, C_cpu, C_gpu)), r, L, t_merge, C.byref(tc), C.byref(tg))
    return float(t), tc.value, tg.value


class Policy:
    """Owner of one ``ipkv_policy_t``: sliding-window feedback on the CPU cost A, marginal share p = B/(A+B)."""

    def __init__(self, A, B, C_cpu, C_gpu, window_steps=256, share_den=64):
        h = C.c_void_p()
        rc = lib().ipkv_policy_create(C.byref(Roofline(A, B, C_cpu, C_gpu)), window_steps, share_den, C.byref(h))
        if rc != OK:
            raise IpkvError(rc, "ipkv_policy_create")
        self._h = h

    def __del__(self):
        if getattr(self, "_h", None):
            lib().ipkv_policy_destroy(self._h)
            self._h = None

    def observe(self, cpu_seconds, cpu_tokens):
        rc = lib().ipkv_policy_observe(self._h, cpu_seconds, cpu_tokens)
        if rc != OK:
            raise IpkvError(rc, "ipkv_policy_observe")

    def update(self):
        """(share numerator, dict of the current model)."""
        num, m = C.c_int32(), Roofline()
        rc = lib().ipkv_policy_update(self._h, C.byref(num), C.byref(m))
        if rc != OK:
            raise IpkvError(rc, "ipkv_policy_update")
        return num.value, dict(A=m.A, B=m.B, C_cpu=m.C_cpu, C_gpu=m.C_gpu)

    def prefill_share(self, L0):
        num = C.c_int32()
        rc = lib().ipkv_policy_prefill_share(self._h, L0, C.byref(num))
        if rc != OK:
            raise IpkvError(rc, "ipkv_policy_prefill_share")
        return num.value


def make_shape(kind, n_q_heads, n_kv_heads, dim_qk, dim_v, block_tokens, softmax_scale=0.0):
    return AttnShape(kind, n_q_heads, n_kv_heads, dim_qk, dim_v, block_tokens, softmax_scale)


def ipkv_block_bytes(shape):
    return int(lib().ipkv_block_bytes(C.byref(shape)))


def ipkv_attend_scratch_bytes(shape, n_rows, n_runs, total_tokens, kv_splits=0):
    out = C.c_size_t()
    rc = lib().ipkv_attend_scratch_bytes(C.byref(shape), n_rows, n_runs, total_tokens, kv_splits, C.byref(out))
    if rc != OK:
        raise IpkvError(rc, "ipkv_attend_scratch_bytes")
    return out.value


def ipkv_attend_runs(shape, runs_per_row, q, scratch, o_part, lse_part, kv_splits=0, status=None, stream=None):
    """runs_per_row: list (one entry per row) of lists of (device pointer or tensor, n_tokens)."""
    flat, start = [], [0]
    for row in runs_per_row:
        for ptr, n in row:
            flat.append(Run(_ptr(ptr), int(n)))
        start.append(len(flat))
    runs = (Run * max(1, len(flat)))(*flat)
    starts = (C.c_int32 * len(start))(*start)
    rc = lib().ipkv_attend_runs(C.byref(shape), len(runs_per_row), runs, starts, _ptr(q), kv_splits, _ptr(scratch),
                                scratch.numel() * scratch.element_size(), _ptr(o_part), _ptr(lse_part), _ptr(status),
                                _stream(stream))
    if rc != OK:
        raise IpkvError(rc, "ipkv_attend_runs")


def _marshal_runs(runs_per_row):
    flat, start = [], [0]
    for row in runs_per_row:
        for ptr, n in row:
            flat.append(Run(_ptr(ptr), int(n)))
        start.append(len(flat))
    return (Run * max(1, len(flat)))(*flat), (C.c_int32 * len(start))(*start)


def ipkv_noalloc_scratch_limit():
    return int(lib().ipkv_noalloc_scratch_limit())


def ipkv_attend_runs_noalloc(shape, runs_per_row, q, o_part, lse_part, kv_splits=0, status=None, stream=None):
    """ipkv_attend_runs for callers that cannot allocate device memory at the call site: same arguments minus the
    scratch buffer, which is a fixed 16 MiB array inside the library (shared by all calls on a device; calls that
    overlap on the GPU race on it).  Raises IpkvError(ERANGE) when the call would need more than that."""
    runs, starts = _marshal_runs(runs_per_row)
    rc = lib().ipkv_attend_runs_noalloc(C.byref(shape), len(runs_per_row), runs, starts, _ptr(q), kv_splits,
                                        _ptr(o_part), _ptr(lse_part), _ptr(status), _stream(stream))
    if rc != OK:
        raise IpkvError(rc, "ipkv_attend_runs_noalloc")


def ipkv_pack_blocks(shape, layout, k, v, n_tokens, dst, stream=None):
    rc = lib().ipkv_pack_blocks(C.byref(shape), layout, _ptr(k), _ptr(v), n_tokens, _ptr(dst), _stream(stream))
    if rc != OK:
        raise IpkvError(rc, "ipkv_pack_blocks")


# ---- operators beside the cache -------------------------------------------------------------------------------------
# A decode step calls these once a layer, so what they check is checked with few attribute reads, and tables go to the
# library as packed bytes.

_torch = _np = _bf16 = _f32 = _i32 = _int64 = _int32 = _current_device = _current_stream = None


def _modules():
    global _torch, _np, _bf16, _f32, _i32, _int64, _int32, _current_device, _current_stream
    import numpy
    import torch
    _np, _bf16, _f32, _i32, _int64, _int32 = numpy, torch.bfloat16, torch.float32, torch.int32, numpy.dtype(numpy.int64), numpy.dtype(numpy.int32)
    # torch's own short ways to the current device and stream; where a release lacks them, the public ones
    _current_device = getattr(torch._C, "_cuda_getDevice", None) or torch.cuda.current_device
    _current_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None) or (lambda dev: torch.cuda.current_stream(dev).cuda_stream)
    _torch = torch                                       # last: a call that finds it, in another thread, uses the others


def _call_stream(stream, dev):
    """The stream of a stateless call on tensors of CUDA device `dev`, as a number: the given one, or the current device's current
    one.  The call runs on the current device, so the tensors have to live there."""
    if dev < 0 or dev != _current_device():
        raise ValueError(f"the tensors are on device {dev} (-1: the host), the call runs on the current CUDA device")
    if stream is None:
        return _current_stream(dev)
    return stream if isinstance(stream, int) else stream.cuda_stream


# ---- head norm and rotation ----

_HEADS_FORMAT = struct.Struct("<QQQi4xqqqq")         # ipkv_heads
_AXIS = (b"\0", b"\1", b"\2", b"\3")


def make_rope(dim, rot_dim=None, *, theta=10000.0, sections=None, interleaved=False, eps=1e-6, inv_freq=None, pair_axis=None):
    """What ipkv_norm_rope does to a head.  sections: how many pairs of columns follow each axis, in order (their sum is
    rot_dim / 2); pair_axis: the axis of every pair instead, for other arrangements; neither: one axis."""
    rot_dim = dim if rot_dim is None else rot_dim
    pairs = rot_dim // 2
    n_axes = 1
    if sections is not None:
        if pair_axis is not None:
            raise ValueError("sections and pair_axis exclude each other")
        n_axes = len(sections)
        if n_axes > 1:
            pair_axis = b""
            for a, n in enumerate(sections):
                if n < 0:
                    raise ValueError(f"a section has {n} pairs")
                pair_axis += _AXIS[a] * n if a < 4 else bytes((a,)) * n
            total = len(pair_axis)
        else:
            total = sections[0] if n_axes else 0
        if total != pairs:
            raise ValueError(f"{total} pairs have an axis, {pairs} are rotated")
    elif pair_axis is not None:
        if len(pair_axis) != pairs:
            raise ValueError(f"{len(pair_axis)} pairs have an axis, {pairs} are rotated")
        n_axes = max(pair_axis, default=0) + 1
        pair_axis = bytes(pair_axis)
    r = Rope(dim, rot_dim, n_axes, 1 if interleaved else 0, eps, theta, None, pair_axis or None)         # the field keeps the bytes
    if inv_freq is not None:
        if len(inv_freq) != pairs:
            raise ValueError(f"{len(inv_freq)} frequencies, {pairs} pairs are rotated")
        r._freq = (C.c_double * max(1, pairs))(*[float(f) for f in inv_freq])
        r.inv_freq = C.cast(r._freq, C.c_void_p)
    return r


def ipkv_norm_rope(rope, parts, positions, stream=None):
    """parts: 1..4 tuples (x, weight or None, out or None): x and out [n_tokens, heads, dim] bf16 with any token and head
    strides, out None means in place.  positions: int32 [n_axes, n_tokens] (or flat), contiguous; None without a rotation."""
    if _torch is None:
        _modules()
    if not parts:
        raise ValueError("a call takes 1 to 4 parts")
    bf16, dim = _bf16, rope.dim
    x = parts[0][0]
    n_tokens, dev = x.shape[0], x.get_device()
    packed = b""
    for x, w, out in parts:
        shape = x.shape
        if x.dtype is not bf16 or len(shape) != 3 or shape[0] != n_tokens or shape[2] != dim:
            raise ValueError(f"heads are bfloat16 [{n_tokens}, n_heads, {dim}]: got {x.dtype} {tuple(shape)}")
        n_heads, (it, ih, ic), at = shape[1], x.stride(), x.data_ptr()
        if out is None:
            ot, oh, oc, to = it, ih, ic, at
        else:
            if out.dtype is not bf16 or out.shape != shape:
                raise ValueError(f"an output is like its input: got {out.dtype} {tuple(out.shape)} for {tuple(shape)}")
            (ot, oh, oc), to = out.stride(), out.data_ptr()
            if out.get_device() != dev:
                oc = 0
        if ic != 1 or oc != 1 or x.get_device() != dev:
            raise ValueError("the columns of a head are contiguous, and all tensors are on one device")
        if n_tokens <= 1:                                # the stride of a dimension of one is never used
            it = ot = 0
        if n_heads <= 1:
            ih = oh = 0
        if w is None:
            wp = 0
        else:
            if w.dtype is not bf16 or w.numel() != dim or not w.is_contiguous() or w.get_device() != dev:
                raise ValueError(f"a weight is contiguous bfloat16 [{dim}] on the device of the heads")
            wp = w.data_ptr()
        packed += _HEADS_FORMAT.pack(at, to, wp, n_heads, it, ih, ot, oh)
    if positions is not None:
        axes = rope.n_axes
        if (positions.dtype is not _i32 or positions.numel() != axes * n_tokens or not positions.is_contiguous() or positions.get_device() != dev
                or (axes > 1 and positions.dim() > 1 and positions.shape[-1] != n_tokens)):
            raise ValueError(f"positions are contiguous int32 [{axes}, {n_tokens}] on the device of the heads: got {positions.dtype} {tuple(positions.shape)}")
        positions = positions.data_ptr()
    rc = (_lib or lib()).ipkv_norm_rope(C.byref(rope), n_tokens, packed, len(parts), positions, _call_stream(stream, dev))
    if rc != OK:
        raise IpkvError(rc, "ipkv_norm_rope")


# ---- a cache held in 4 bits ----

def ipkv_nibble_block_bytes(shape):
    """Bytes of one NIBBLE block (grouped-query shapes, dim 64 or 128, block_tokens a multiple of 64)."""
    n = int(lib().ipkv_nibble_block_bytes(C.byref(shape)))
    if n < 0:
        raise IpkvError(1, "ipkv_nibble_block_bytes")
    return n


def _table(rows, width, dev):
    """A host table of 64-bit words, [n][width]: a NumPy int64 array as it is, or rows whose first entry may be a tensor on device dev."""
    if not isinstance(rows, _np.ndarray):
        for r in (rows, *rows):                          # a tensor's own entries would count as blocks
            if isinstance(r, _torch.Tensor):
                raise ValueError("a table of blocks is a list or a NumPy int64 array")
        for r in rows:
            if hasattr(r[0], "get_device") and r[0].get_device() != dev:
                raise ValueError(f"blocks on device {r[0].get_device()} (-1: the host), the other tensors are on {dev}")
        rows = _np.array([[_ptr(r[0]) or 0, *r[1:]] for r in rows], dtype=_np.int64).reshape(-1, width)
    shape = rows.shape
    if rows.dtype != _int64 or len(shape) != 2 or shape[1] != width or not rows.flags.c_contiguous:
        raise ValueError(f"expected a contiguous int64 array [n][{width}]: got {rows.dtype} {shape}")
    return rows


def _move(name, shape, spans, k, v, stream):
    if _torch is None:
        _modules()
    heads, dim, size, dev, bf16 = shape.n_kv_heads, shape.dim_qk, k.shape, k.get_device(), _bf16
    t = _table(spans, 3, dev)
    n = size[0]
    if k.dtype is not bf16 or v.dtype is not bf16 or len(size) != 3 or size[1] != heads or size[2] != dim or v.shape != size:
        raise ValueError(f"K and V are bfloat16 [tokens, {heads}, {dim}]: got {k.dtype} {tuple(size)}, {v.dtype} {tuple(v.shape)}")
    (kt, kh, kc), (vt, vh, vc) = k.stride(), v.stride()
    if n <= 1:                                           # the stride of a dimension of one is never used
        kt = vt = 0
    elif kt == 0 or vt == 0:
        kc = 0
    if kc != 1 or vc != 1 or (heads > 1 and (kh != dim or vh != dim)) or v.get_device() != dev:
        raise ValueError("the heads of a token lie side by side, its tokens apart, and K and V are on one device")
    rc = getattr(_lib or lib(), name)(C.byref(shape), len(t), t.tobytes(), n, k.data_ptr(), v.data_ptr(), kt, vt, _call_stream(stream, dev))
    if rc != OK:
        raise IpkvError(rc, name)


def ipkv_nibble_pack(shape, spans, k, v, stream=None):
    """Write the tokens of k and v [tokens][n_kv_heads][dim] into NIBBLE blocks: spans is a list of (blocks, first token, tokens),
    or an int64 array [n][3] of addresses and counts; the tokens of one span follow those of the one before."""
    _move("ipkv_nibble_pack", shape, spans, k, v, stream)


def ipkv_nibble_unpack(shape, spans, k, v, stream=None):
    """The inverse of ipkv_nibble_pack: the values that the spans' codes stand for, into k and v."""
    _move("ipkv_nibble_unpack", shape, spans, k, v, stream)


def ipkv_nibble_scratch_bytes(shape, n_rows, n_runs):
    out = C.c_size_t()
    rc = lib().ipkv_nibble_scratch_bytes(C.byref(shape), n_rows, n_runs, C.byref(out))
    if rc != OK:
        raise IpkvError(rc, "ipkv_nibble_scratch_bytes")
    return out.value


def ipkv_nibble_attend(shape, runs, row_start, q, scratch, o_part, lse_part, status=None, stream=None):
    """Attention of one query per row over runs of NIBBLE blocks.  runs: int64 array [n][2] of (address, tokens) with row_start,
    an int32 array [rows + 1]; or, with row_start None, one list per row of (blocks, tokens) as for ipkv_attend_runs."""
    if _torch is None:
        _modules()
    dev = q.get_device()
    if row_start is None:
        if isinstance(runs, _torch.Tensor):
            raise ValueError("the table of runs is a list per row, or a NumPy int64 array with row_start")
        row_start = _np.cumsum([0] + [len(r) for r in runs]).astype(_np.int32)
        runs = _table([x for r in runs for x in r], 2, dev)
    else:
        runs = _table(runs, 2, dev)
        if not isinstance(row_start, _np.ndarray) or row_start.dtype != _int32 or row_start.ndim != 1 or not row_start.flags.c_contiguous:
            raise ValueError("row_start is a contiguous int32 array [rows + 1]")
    rows = len(row_start) - 1
    if rows < 1 or row_start.item(-1) > len(runs):
        raise ValueError(f"row_start names runs that are not there: there are {len(runs)}")
    heads, f32 = shape.n_q_heads, _f32
    want = (rows, heads, shape.dim_qk)
    if (q.dtype is not _bf16 or o_part.dtype is not f32 or lse_part.dtype is not f32 or q.shape != want or o_part.shape != want
            or lse_part.shape != (rows, heads) or not (q.is_contiguous() and o_part.is_contiguous() and lse_part.is_contiguous())
            or o_part.get_device() != dev or lse_part.get_device() != dev):
        raise ValueError(f"q is contiguous bfloat16 {want}, o_part float32 {want} and lse_part float32 {want[:2]} on one device: got "
                         + ", ".join(f"{x.dtype} {tuple(x.shape)} {x.device}" for x in (q, o_part, lse_part)))
    if scratch.get_device() != dev or not scratch.is_contiguous() or (status is not None and (status.get_device() != dev or status.dtype not in (_i32, _torch.uint32))):
        raise ValueError("scratch and the status word (32 bits) are on the device of q")
    rc = (_lib or lib()).ipkv_nibble_attend(C.byref(shape), rows, runs.tobytes(), row_start.tobytes(), q.data_ptr(), scratch.data_ptr(), scratch.nbytes,
                                            o_part.data_ptr(), lse_part.data_ptr(), _ptr(status), _call_stream(stream, dev))
    if rc != OK:
        raise IpkvError(rc, "ipkv_nibble_attend")
