"""MI355X-native similarity join (Ahle & Silvestri, "Similarity Search with
Tensor Core Units", Section 4, brute-force method): Python binding of libsj.so.

The raw C-ABI entry points are exposed under their C names (sj_create,
sj_join_ip, sj_join_l2, sj_count, sj_join_noalloc, sj_normalize,
sj_join_hamming, sj_join_lsh, sj_lsh_sort, sj_lsh_collision, sj_lsh_plan, sj_jl, sj_destroy,
sj_get_stats, sj_last_error) with plain integer pointers; `join_ip`, `join_l2`, `count` and
`join_lsh` (the LSH-bucketed join of Theorem 3) are conveniences over PyTorch
device tensors, as are `rotary`, `cache_append`, `attend` and `cache_evict` around a
cache of key and value rows (`kv_cache`).  This module only marshals
arguments: every step of the join runs in the library's HIP kernels.  Import
fails when libsj.so has not been built (python paper_2006_12608_amd/build.py).
"""
from __future__ import annotations

import ctypes
import functools
import os

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libsj.so")

SJ_F16, SJ_BF16, SJ_I8 = 1, 2, 3
SJ_IP, SJ_L2 = 0, 1
SJ_OK, SJ_E_INVAL, SJ_E_OVERFLOW, SJ_E_NOMEM, SJ_E_HIP, SJ_E_UNSUPPORTED = 0, -1, -2, -3, -4, -5
SJ_FLAG_TWO_PASS, SJ_FLAG_TIMING, SJ_FLAG_RECOMPUTE, SJ_FLAG_COSINE = 1, 2, 4, 8
SJ_FLAG_INVERSE = 16
SJ_HALF, SJ_INTERLEAVED = 0, 1

STATUS_NAMES = {0: "SJ_OK", -1: "SJ_E_INVAL", -2: "SJ_E_OVERFLOW", -3: "SJ_E_NOMEM",
                -4: "SJ_E_HIP", -5: "SJ_E_UNSUPPORTED"}


class SjError(RuntimeError):
    def __init__(self, status: int, message: str, n_out: int | None = None):
        super().__init__(f"{STATUS_NAMES.get(status, status)}: {message}")
        self.status = status
        self.n_out = n_out


class sj_stats(ctypes.Structure):
    _fields_ = [("total", ctypes.c_uint64), ("ms_norms", ctypes.c_double),
                ("ms_join", ctypes.c_double), ("ms_count", ctypes.c_double),
                ("ms_scan", ctypes.c_double), ("ms_emit", ctypes.c_double),
                ("kernel", ctypes.c_uint32), ("timed", ctypes.c_uint32),
                ("emit_from_bits", ctypes.c_uint32), ("lsh_rows", ctypes.c_uint64)]


class sj_cache(ctypes.Structure):
    _fields_ = [("dtype", ctypes.c_int), ("heads", ctypes.c_uint32), ("d", ctypes.c_uint32),
                ("pages", ctypes.c_uint32), ("page", ctypes.c_uint32), ("batch", ctypes.c_uint32),
                ("width", ctypes.c_uint32), ("table_row", ctypes.c_int64),
                ("table", ctypes.c_void_p), ("k", ctypes.c_void_p), ("v", ctypes.c_void_p),
                ("k_page", ctypes.c_int64), ("k_row", ctypes.c_int64), ("k_head", ctypes.c_int64),
                ("v_page", ctypes.c_int64), ("v_row", ctypes.c_int64), ("v_head", ctypes.c_int64)]


# allocation of an output half-way through a call, once its size is known
# (csrc/sj_sized.h): (user, number of pairs) -> device pointer
_ALLOC = ctypes.CFUNCTYPE(ctypes.c_void_p, ctypes.c_void_p, ctypes.c_uint64)


def _load():
    if not os.path.exists(LIB_PATH):
        raise ImportError(f"{LIB_PATH} is missing: build it with "
                          "`python paper_2006_12608_amd/build.py` (hipcc, gfx950)")
    lib = ctypes.CDLL(LIB_PATH)
    vp, u32, u64, dbl, i32 = (ctypes.c_void_p, ctypes.c_uint32, ctypes.c_uint64, ctypes.c_double,
                              ctypes.c_int)
    lib.sj_create.argtypes = [ctypes.POINTER(vp), i32, vp]
    lib.sj_create.restype = i32
    join_args = [vp, i32, vp, u32, vp, u32, u32, dbl, vp, u64, ctypes.POINTER(u64), ctypes.c_uint]
    lib.sj_join_ip.argtypes = join_args
    lib.sj_join_ip.restype = i32
    lib.sj_join_l2.argtypes = join_args
    lib.sj_join_l2.restype = i32
    lib.sj_count.argtypes = [vp, i32, i32, vp, u32, vp, u32, u32, dbl, ctypes.POINTER(u64)]
    lib.sj_count.restype = i32
    lib.sj_join_noalloc.argtypes = [vp, i32, i32, vp, u32, vp, u32, u32, dbl, vp, u64,
                                    ctypes.POINTER(u64), ctypes.c_uint]
    lib.sj_join_noalloc.restype = i32
    lib.sj_normalize.argtypes = [vp, i32, vp, u32, u32, vp]
    lib.sj_normalize.restype = i32
    lib.sj_join_hamming.argtypes = [vp, vp, u32, vp, u32, u32, dbl, vp, u64,
                                    ctypes.POINTER(u64), ctypes.c_uint]
    lib.sj_join_hamming.restype = i32
    lib.sj_join_lsh.argtypes = [vp, i32, i32, vp, u32, vp, u32, u32, dbl, u32, u32, vp, vp,
                                ctypes.c_int32, vp, u64, ctypes.POINTER(u64),
                                ctypes.POINTER(u64)]
    lib.sj_join_lsh.restype = i32
    lib.sji_join_sized.argtypes = [vp, i32, i32, vp, u32, vp, u32, u32, dbl, _ALLOC, vp,
                                   ctypes.POINTER(u64), ctypes.c_uint]
    lib.sji_join_sized.restype = i32
    lib.sji_lsh_sized.argtypes = [vp, i32, i32, vp, u32, vp, u32, u32, dbl, u32, u32, vp, vp,
                                  ctypes.c_int32, _ALLOC, vp, ctypes.POINTER(u64),
                                  ctypes.POINTER(u64)]
    lib.sji_lsh_sized.restype = i32
    lib.sj_lsh_sort.argtypes = [vp, vp, u32, u32, u32, vp]
    lib.sj_lsh_sort.restype = i32
    lib.sj_lsh_collision.argtypes = [ctypes.c_int32, dbl, dbl]
    lib.sj_lsh_collision.restype = dbl
    lib.sj_lsh_plan.argtypes = [dbl, dbl, u64, u32, dbl, ctypes.POINTER(u32), ctypes.POINTER(u32),
                                ctypes.POINTER(u32)]
    lib.sj_lsh_plan.restype = i32
    lib.sj_jl.argtypes = [vp, i32, vp, u32, u32, u32, vp, vp, vp]
    lib.sj_jl.restype = i32
    strides = ctypes.POINTER(ctypes.c_int64)
    cache = ctypes.POINTER(sj_cache)
    lib.sj_rotary.argtypes = [vp, i32, vp, strides, vp, strides, u32, u32, u32, vp, vp, u32, i32,
                              dbl, ctypes.c_uint]
    lib.sj_rotary.restype = i32
    lib.sj_cache_append.argtypes = [vp, cache, vp, vp, u32, vp, strides, vp, strides, vp, vp, u32,
                                    i32, dbl, vp, strides, u32, vp, strides]
    lib.sj_cache_append.restype = i32
    lib.sj_attend.argtypes = [vp, cache, vp, vp, u32, vp, strides, u32, vp, strides, dbl, vp, vp,
                              vp, vp, u64]
    lib.sj_attend.restype = i32
    lib.sj_cache_evict.argtypes = [vp, cache, vp, vp, u32, u64, u32, u32, u32, cache, vp, vp, vp,
                                   u64]
    lib.sj_cache_evict.restype = i32
    lib.sj_destroy.argtypes = [vp]
    lib.sj_destroy.restype = None
    lib.sj_get_stats.argtypes = [vp, ctypes.POINTER(sj_stats)]
    lib.sj_get_stats.restype = i32
    lib.sj_last_error.argtypes = []
    lib.sj_last_error.restype = ctypes.c_char_p
    return lib


lib = _load()


# ------------------------------------------------------------ raw C-ABI names

def sj_last_error() -> str:
    return lib.sj_last_error().decode()


def sj_create(device: int = 0, stream: int | None = None) -> int:
    """Returns an opaque context handle (int)."""
    h = ctypes.c_void_p()
    st = lib.sj_create(ctypes.byref(h), device, stream or None)
    if st != SJ_OK:
        raise SjError(st, sj_last_error())
    return h.value


def sj_destroy(ctx: int | None) -> None:
    lib.sj_destroy(ctx)


def _join_raw(fn, ctx, dtype, P, n_p, Q, n_q, d, thr, pairs, cap, flags):
    n = ctypes.c_uint64(0)
    st = fn(ctx, dtype, P, n_p, Q, n_q, d, float(thr), pairs, cap, ctypes.byref(n), flags)
    return st, n.value


def sj_join_ip(ctx, dtype, P, n_p, Q, n_q, d, s, pairs, cap, flags=0):
    """Returns (status, n_out); pointers are integers (device addresses)."""
    return _join_raw(lib.sj_join_ip, ctx, dtype, P, n_p, Q, n_q, d, s, pairs, cap, flags)


def sj_join_l2(ctx, dtype, P, n_p, Q, n_q, d, r2, pairs, cap, flags=0):
    """Returns (status, n_out); pointers are integers (device addresses)."""
    return _join_raw(lib.sj_join_l2, ctx, dtype, P, n_p, Q, n_q, d, r2, pairs, cap, flags)


def sj_join_noalloc(ctx, metric, dtype, P, n_p, Q, n_q, d, thr, pairs, cap, flags=0):
    """The join without device allocation (fixed library scratch); returns
    (status, n_out); pointers are integers (device addresses)."""
    n = ctypes.c_uint64(0)
    st = lib.sj_join_noalloc(ctx, metric, dtype, P, n_p, Q, n_q, d, float(thr), pairs, cap,
                             ctypes.byref(n), flags)
    return st, n.value


def sj_normalize(ctx, dtype, X, n, d, Y):
    """Returns the status; pointers are integers (device addresses)."""
    return lib.sj_normalize(ctx, dtype, X, n, d, Y)


def sj_join_hamming(ctx, P, n_p, Q, n_q, d, r, pairs, cap, flags=0):
    """Returns (status, n_out); P and Q are device bit rows (ceil(d / 8) bytes)."""
    n = ctypes.c_uint64(0)
    st = lib.sj_join_hamming(ctx, P, n_p, Q, n_q, d, float(r), pairs, cap, ctypes.byref(n),
                             flags)
    return st, n.value


def sj_count(ctx, metric, dtype, P, n_p, Q, n_q, d, threshold):
    """Returns (status, count)."""
    n = ctypes.c_uint64(0)
    st = lib.sj_count(ctx, metric, dtype, P, n_p, Q, n_q, d, float(threshold), ctypes.byref(n))
    return st, n.value


def sj_join_lsh(ctx, metric, dtype, P, n_p, Q, n_q, d, thr, L, k, A, B, w, pairs, cap):
    """Returns (status, n_out, n_cand); pointers are integers (device addresses)."""
    n = ctypes.c_uint64(0)
    nc = ctypes.c_uint64(0)
    st = lib.sj_join_lsh(ctx, metric, dtype, P, n_p, Q, n_q, d, float(thr), L, k, A, B, int(w),
                         pairs, cap, ctypes.byref(n), ctypes.byref(nc))
    return st, n.value, nc.value


def sj_lsh_sort(ctx, keys, n, L, bits, perm) -> int:
    return lib.sj_lsh_sort(ctx, keys, n, L, bits, perm)


def sj_lsh_collision(w: int, sigma: float, dist: float) -> float:
    return lib.sj_lsh_collision(int(w), float(sigma), float(dist))


def sj_lsh_plan(p1: float, p2: float, n: int, tile: int, recall: float):
    """Returns (status, k, L_inst, reps)."""
    k, L, r = ctypes.c_uint32(), ctypes.c_uint32(), ctypes.c_uint32()
    st = lib.sj_lsh_plan(float(p1), float(p2), int(n), int(tile), float(recall), ctypes.byref(k),
                         ctypes.byref(L), ctypes.byref(r))
    return st, k.value, L.value, r.value


def sj_jl(ctx, dtype, X, n, d, levels, shape, A, Y):
    """Returns the status; shape is a sequence of (k_i, c_i, r_i), pointers
    are integers (device addresses)."""
    flat = [int(v) for s in shape for v in s]
    arr = (ctypes.c_uint32 * max(len(flat), 1))(*flat)
    return lib.sj_jl(ctx, dtype, X, n, d, levels, arr, A, Y)


@functools.lru_cache(maxsize=4096)
def _strides(*values):
    """Element strides as the C array the calls on caches take (which only read it)."""
    return (ctypes.c_int64 * len(values))(*values)


def sj_rotary(ctx, dtype, x, x_stride, y, y_stride, n, heads, d, pos, turns, n_pairs, layout,
              factor, flags=0):
    """Returns the status; strides are sequences of element strides, the other
    arrays device addresses."""
    return lib.sj_rotary(ctx, dtype, x, _strides(*x_stride), y, _strides(*y_stride), n, heads, d,
                         pos, turns, n_pairs, layout, factor, flags)


def sj_cache_append(ctx, cache, length, count, t, key, key_stride, value, value_stride, pos, turns,
                    n_pairs, layout, factor, q=None, q_stride=(0, 0, 0), q_heads=0, q_out=None,
                    q_out_stride=(0, 0, 0)):
    """Returns the status; cache is an sj_cache structure (or None)."""
    return lib.sj_cache_append(ctx, None if cache is None else ctypes.byref(cache), length, count,
                               t, key, _strides(*key_stride), value, _strides(*value_stride), pos,
                               turns, n_pairs, layout, factor, q, _strides(*q_stride), q_heads,
                               q_out, _strides(*q_out_stride))


def sj_attend(ctx, cache, length, count, t, q, q_stride, q_heads, tree, tree_stride, scale, out,
              lse, w_in=None, w_out=None, w_cols=0):
    """Returns the status; cache is an sj_cache structure (or None)."""
    return lib.sj_attend(ctx, None if cache is None else ctypes.byref(cache), length, count, t, q,
                         _strides(*q_stride), q_heads, tree, _strides(*tree_stride), scale, out,
                         lse, w_in, w_out, w_cols)


def sj_cache_evict(ctx, src, length, weight, sets, w_cols, keep, sink, recent, dst, index, new_len,
                   w_out=None, w_out_cols=0):
    """Returns the status; src and dst are sj_cache structures (or None)."""
    return lib.sj_cache_evict(ctx, None if src is None else ctypes.byref(src), length, weight,
                              sets, w_cols, keep, sink, recent,
                              None if dst is None else ctypes.byref(dst), index, new_len, w_out,
                              w_out_cols)


def sj_get_stats(ctx) -> sj_stats:
    out = sj_stats()
    st = lib.sj_get_stats(ctx, ctypes.byref(out))
    if st != SJ_OK:
        raise SjError(st, sj_last_error())
    return out


# ------------------------------------------------------ torch conveniences

_contexts: dict = {}


def context(device: int | None = None, stream=None) -> int:
    """A cached context bound to (device, stream); defaults to torch's
    current device and stream.  Threads that share a stream share its context:
    their calls wait for one another."""
    import torch
    dev = torch.cuda.current_device() if device is None else int(device)
    if stream is None:
        stream = torch.cuda.current_stream(dev)
    handle = int(stream.cuda_stream) if hasattr(stream, "cuda_stream") else int(stream or 0)
    key = (dev, handle)
    known = _contexts.get(key)
    if known is None:
        made = sj_create(dev, handle)
        known = _contexts.setdefault(key, made)
        if known != made:       # (another thread's came first)
            sj_destroy(made)
    return known


def dtype_code(t) -> int:
    import torch
    codes = {torch.float16: SJ_F16, torch.bfloat16: SJ_BF16, torch.int8: SJ_I8}
    if t.dtype not in codes:
        raise TypeError(f"unsupported dtype {t.dtype}; use float16, bfloat16 or int8")
    return codes[t.dtype]


def _metric_code(metric: str) -> int:
    if metric not in ("ip", "l2"):
        raise ValueError(f"metric must be 'ip' or 'l2', not {metric!r}")
    return SJ_IP if metric == "ip" else SJ_L2


def _check_pair(P, Q):
    if P.dim() != 2 or Q.dim() != 2 or P.shape[1] != Q.shape[1]:
        raise ValueError("P and Q must be 2-D with the same number of columns")
    if P.dtype != Q.dtype:
        raise ValueError("P and Q must have the same dtype")
    if not (P.is_cuda and Q.is_cuda):
        raise ValueError("P and Q must be device tensors")
    if not (P.is_contiguous() and Q.is_contiguous()):
        raise ValueError("P and Q must be contiguous")


def count(P, Q, threshold: float, metric: str = "ip", ctx=None) -> int:
    """Number of matching pairs (sj_count)."""
    _check_pair(P, Q)
    m = _metric_code(metric)
    ctx = ctx or context(P.device.index)
    st, n = sj_count(ctx, m, dtype_code(P), P.data_ptr(), P.shape[0], Q.data_ptr(), Q.shape[0],
                     P.shape[1], threshold)
    if st != SJ_OK:
        raise SjError(st, sj_last_error())
    return n


def _own_output(call, device):
    """Runs call(alloc) -> status, which sizes its output itself and asks for
    it half-way (the product, or the hashing and sorting, runs once).  Returns
    the pairs."""
    import torch
    out, failed = None, None

    def alloc(_, n):
        nonlocal out, failed
        try:
            out = torch.empty((n, 2), dtype=torch.int32, device=device)
            return out.data_ptr()
        except BaseException as e:      # nothing may pass through the C call
            failed = e
            return None
    st = call(_ALLOC(alloc))
    if failed is not None:
        raise failed
    if st != SJ_OK:
        raise SjError(st, sj_last_error(), 0 if out is None else out.shape[0])
    return torch.empty((1, 2), dtype=torch.int32, device=device)[:0] if out is None else out


def _join_sized(kind, ctx, dtype, P, Q, d, thr, flags):
    """A join without a capacity: count-then-emit into an output of the size
    that the count gives (kind 0: inner product, 1: L2, 2: Hamming)."""
    n = ctypes.c_uint64(0)
    return _own_output(lambda alloc: lib.sji_join_sized(
        ctx, kind, dtype, P.data_ptr(), P.shape[0], Q.data_ptr(), Q.shape[0], d, float(thr), alloc,
        None, ctypes.byref(n), flags), P.device)


def _sized_call(call, flags, cap, out, device):
    """Runs call(pairs_ptr, cap, flags) -> (status, n); with neither a
    capacity nor an output buffer, a first count-then-emit call with no room
    sizes the output (it stops after the count) and a second one fills it."""
    import torch
    if cap is None and out is None:
        st, n = call(None, 0, flags | SJ_FLAG_TWO_PASS)
        if st not in (SJ_OK, SJ_E_OVERFLOW):
            raise SjError(st, sj_last_error(), n)
        cap = n
    if out is None:
        out = torch.empty((max(int(cap), 1), 2), dtype=torch.int32, device=device)
        cap = int(cap)
    else:
        cap = out.shape[0] if cap is None else int(cap)
    st, n = call(out.data_ptr() if cap else None, cap, flags)
    if st != SJ_OK:
        raise SjError(st, sj_last_error(), n)
    return out[:n]


def _join(metric, P, Q, thr, cap, two_pass, timing, ctx, out, recompute=False, cosine=False):
    import torch
    _check_pair(P, Q)
    ctx = ctx or context(P.device.index)
    unsized = cap is None and out is None
    if two_pass is None:
        # no capacity given: count-then-emit sizes the output exactly
        two_pass = unsized
    flags = ((SJ_FLAG_TWO_PASS if two_pass else 0) | (SJ_FLAG_TIMING if timing else 0)
             | (SJ_FLAG_RECOMPUTE if recompute else 0) | (SJ_FLAG_COSINE if cosine else 0))
    if unsized and two_pass:
        return _join_sized(0 if metric == "ip" else 1, ctx, dtype_code(P), P, Q, P.shape[1], thr,
                           flags)
    if cosine:
        def call(ptr, c, f):
            return sj_join_ip(ctx, dtype_code(P), P.data_ptr(), P.shape[0], Q.data_ptr(),
                              Q.shape[0], P.shape[1], thr, ptr, c, f)
        return _sized_call(call, flags, cap, out, P.device)
    if unsized:
        cap = count(P, Q, thr, metric, ctx)
    if out is None:
        out = torch.empty((max(int(cap), 1), 2), dtype=torch.int32, device=P.device)
        cap = int(cap)
    else:
        cap = out.shape[0] if cap is None else int(cap)
    fn = sj_join_ip if metric == "ip" else sj_join_l2
    st, n = fn(ctx, dtype_code(P), P.data_ptr(), P.shape[0], Q.data_ptr(), Q.shape[0], P.shape[1],
               thr, out.data_ptr() if cap else None, cap, flags)
    if st != SJ_OK:
        raise SjError(st, sj_last_error(), n)
    return out[:n]


def join_ip(P, Q, s: float, cap: int | None = None, two_pass: bool | None = None,
            timing: bool = False, ctx=None, out=None, recompute: bool = False,
            cosine: bool = False):
    """All (i, j) with <P_i, Q_j> >= s as an (n, 2) int32 tensor of uint32
    indices.  With cap=None (and no `out`) the output is sized by the counting
    pass of count-then-emit (deterministic order) unless two_pass=False asks
    for the single pass (sized by sj_count); with a capacity the single pass runs unless
    two_pass=True.  recompute makes the second pass of count-then-emit repeat
    the product even where the first pass's match bits would be kept.
    cosine=True normalises the rows in the library first (SJ_FLAG_COSINE)."""
    return _join("ip", P, Q, s, cap, two_pass, timing, ctx, out, recompute, cosine)


def join_l2(P, Q, r2: float, cap: int | None = None, two_pass: bool | None = None,
            timing: bool = False, ctx=None, out=None, recompute: bool = False):
    """All (i, j) with ||P_i - Q_j||^2 <= r2 (see join_ip)."""
    return _join("l2", P, Q, r2, cap, two_pass, timing, ctx, out, recompute)


def normalize(X, ctx=None):
    """Section 4's cosine front end (sj_normalize): the rows of X (float16,
    bfloat16 or int8 device tensor) divided by their norms, rounded to
    float16 (bfloat16 for bfloat16 input)."""
    import torch
    if X.dim() != 2 or not X.is_cuda or not X.is_contiguous():
        raise ValueError("X must be a contiguous 2-D device tensor")
    ctx = ctx or context(X.device.index)
    Y = torch.empty(X.shape, dtype=torch.bfloat16 if X.dtype == torch.bfloat16 else torch.float16,
                    device=X.device)
    st = sj_normalize(ctx, dtype_code(X), X.data_ptr(), X.shape[0], X.shape[1], Y.data_ptr())
    if st != SJ_OK:
        raise SjError(st, sj_last_error())
    return Y


def join_hamming(P, Q, d: int, r: float, cap: int | None = None, two_pass: bool | None = None,
                 timing: bool = False, ctx=None, out=None):
    """Section 4's Hamming join (sj_join_hamming): all (i, j) whose d-bit rows
    differ in at most r coordinates.  P and Q are (n, ceil(d / 8)) uint8
    device tensors of bit rows (coordinate m in bit m % 8 of byte m / 8).
    Sizing and modes as join_ip."""
    import torch
    for X in (P, Q):
        if X.dtype != torch.uint8 or X.dim() != 2 or X.shape[1] != (d + 7) // 8 or \
                not X.is_cuda or not X.is_contiguous():
            raise ValueError(f"bit rows must be contiguous (n, {(d + 7) // 8}) uint8 device "
                             "tensors")
    ctx = ctx or context(P.device.index)
    if two_pass is None:
        two_pass = cap is None and out is None
    flags = (SJ_FLAG_TWO_PASS if two_pass else 0) | (SJ_FLAG_TIMING if timing else 0)
    if cap is None and out is None and two_pass:
        return _join_sized(2, ctx, 0, P, Q, d, r, flags)

    def call(ptr, c, f):
        return sj_join_hamming(ctx, P.data_ptr(), P.shape[0], Q.data_ptr(), Q.shape[0], d, r,
                               ptr, c, f)
    return _sized_call(call, flags, cap, out, P.device)


def join_lsh(P, Q, thr: float, metric: str = "ip", *, L: int, k: int, A, B=None, w: int = 0,
             cap: int | None = None, ctx=None, out=None):
    """LSH-bucketed join (sj_join_lsh): the pairs that share a bucket in one
    of L tables (k concatenated random projections each: signs when w == 0,
    quantised with offsets B when w > 0) and pass the exact test of `metric`.
    A is an (L*k, d) int8 device tensor, B an (L*k,) int32 device tensor (or
    None for sign hashes).  With cap=None the library sizes the output.
    Returns (pairs as an (n, 2) int32 tensor of uint32 indices, number of pair
    evaluations made)."""
    import torch
    _check_pair(P, Q)
    if A.dtype != torch.int8 or not A.is_cuda or not A.is_contiguous() or \
            tuple(A.shape) != (L * k, P.shape[1]):
        raise ValueError(f"A must be a contiguous ({L * k}, {P.shape[1]}) int8 device tensor")
    if B is not None and (B.dtype != torch.int32 or not B.is_cuda or not B.is_contiguous()
                          or B.numel() != L * k):
        raise ValueError(f"B must be a contiguous ({L * k},) int32 device tensor")
    m = _metric_code(metric)
    ctx = ctx or context(P.device.index)
    args = (ctx, m, dtype_code(P), P.data_ptr(), P.shape[0], Q.data_ptr(), Q.shape[0],
            P.shape[1], thr, L, k, A.data_ptr() if A.numel() else None,
            None if B is None else B.data_ptr(), w)
    if out is None and cap is None:
        n, nc = ctypes.c_uint64(0), ctypes.c_uint64(0)
        pairs = _own_output(lambda alloc: lib.sji_lsh_sized(
            *args[:8], float(thr), *args[9:], alloc, None, ctypes.byref(n), ctypes.byref(nc)),
            P.device)
        return pairs, nc.value
    if out is None:
        out = torch.empty((max(int(cap), 1), 2), dtype=torch.int32, device=P.device)
        cap = int(cap)
    else:
        cap = out.shape[0] if cap is None else int(cap)
    st, n, nc = sj_join_lsh(*args, out.data_ptr() if cap else None, cap)
    if st != SJ_OK:
        raise SjError(st, sj_last_error(), n)
    return out[:n], nc


def lsh_sort(keys, bits: int, ctx=None):
    """The LSH join's grouping step (sj_lsh_sort): keys is an (L, n) int64
    device tensor of bucket keys (read as uint64, each below 2**bits).  Returns
    an (L, n) int32 tensor: per table the rows with equal keys contiguous and
    in increasing order, the groups in an order fixed by the key values."""
    import torch
    if keys.dim() != 2 or keys.dtype != torch.int64 or not keys.is_cuda or \
            not keys.is_contiguous():
        raise ValueError("keys must be a contiguous (L, n) int64 device tensor")
    L, n = keys.shape
    perm = torch.empty((L, n), dtype=torch.int32, device=keys.device)
    ctx = ctx or context(keys.device.index)
    st = sj_lsh_sort(ctx, keys.data_ptr() if keys.numel() else None, n, L, int(bits),
                     perm.data_ptr() if perm.numel() else None)
    if st != SJ_OK:
        raise SjError(st, sj_last_error())
    return perm


def jl_transform(X, shapes, As, ctx=None):
    """TCU Johnson-Lindenstrauss transform (sj_jl): the rows of X (n x d device
    tensor: float16, bfloat16 or int8) reduced by M = (I_{r_l} (x) A_l) ...
    (I_{r_1} (x) A_1); shapes is the list of (k_i, c_i, r_i), As the list of
    k_i x c_i float32 device tensors.  Returns an (n, r_l k_l) float32 tensor."""
    import torch
    if X.dim() != 2 or not X.is_cuda or not X.is_contiguous():
        raise ValueError("X must be a contiguous 2-D device tensor")
    shapes = [tuple(int(v) for v in s) for s in shapes]
    if len(As) != len(shapes):
        raise ValueError("one factor per level")
    for (k, c, r), A in zip(shapes, As):
        if tuple(A.shape) != (k, c) or A.dtype != torch.float32 or not A.is_cuda:
            raise ValueError(f"factor of shape {(k, c)} float32 on the device expected")
    Acat = torch.cat([A.reshape(-1) for A in As]).contiguous()
    out_dim = shapes[-1][0] * shapes[-1][2]
    Y = torch.empty((X.shape[0], out_dim), dtype=torch.float32, device=X.device)
    ctx = ctx or context(X.device.index)
    st = sj_jl(ctx, dtype_code(X), X.data_ptr(), X.shape[0], X.shape[1], len(shapes), shapes,
               Acat.data_ptr(), Y.data_ptr())
    if st != SJ_OK:
        raise SjError(st, sj_last_error())
    return Y


# ------------------------------------------- a cache of key and value rows

_LAYOUTS = {"half": SJ_HALF, "interleaved": SJ_INTERLEAVED}


def _current(device) -> int:
    """The cached context of the device's current stream (context() without the stream
    object, which costs more than the rest)."""
    import torch
    dev = device.index
    handle = torch._C._cuda_getCurrentRawStream(dev)
    return _contexts.get((dev, handle)) or context(dev)


def _layout_code(layout: str) -> int:
    if layout not in _LAYOUTS:
        raise ValueError(f"layout must be 'half' or 'interleaved', not {layout!r}")
    return _LAYOUTS[layout]


def _refuse(name, x, shape, dtype, device):
    if x.dtype != dtype or x.device != device or x.dim() != len(shape) or \
            any(s is not None and s != n for s, n in zip(shape, x.shape)):
        raise ValueError(f"{name}: {tuple(x.shape)} {x.dtype} on {x.device}, expected "
                         f"{tuple('any' if s is None else s for s in shape)} {dtype} on {device}")
    if x.shape[-1] > 1 and x.stride(-1) != 1:
        raise ValueError(f"{name}: the elements of its last dimension must be adjacent")


def _check_rows(name, x, shape, dtype, device):
    """x: a device tensor of `shape` (None: any size) and dtype whose last
    dimension is adjacent."""
    if x.shape != shape or x.dtype is not dtype or x.device != device or x.stride(-1) != 1:
        _refuse(name, x, shape, dtype, device)


def _check_whole(name, x, shape, dtype, device):
    if x.shape != shape or x.dtype is not dtype or x.device != device or not x.is_contiguous():
        _refuse(name, x, shape, dtype, device)
        if not x.is_contiguous():
            raise ValueError(f"{name} must be contiguous")


def _ptr(x):
    """The address of a tensor's first element (None for none or an empty one)."""
    return None if x is None else (x.data_ptr() or None)


def _follows(*tensors) -> bool:
    """Whether one of the tensors (None: not given) requires grad."""
    for t in tensors:
        if t is not None and t.requires_grad:
            return True
    return False


def _lost(name):
    raise ValueError(f"{name}: a tensor requires grad, which the call would lose; "
                     "call it under torch.no_grad() or detach the tensor")


@functools.lru_cache(maxsize=None)
def _functions():
    """The calls as autograd sees them."""
    import torch

    class Rotary(torch.autograd.Function):
        @staticmethod
        def forward(ctx, x, pos, turns, kw, handle):
            ctx.save_for_backward(pos, turns)
            ctx.kw = kw
            return rotary(x, pos, turns, ctx=handle, **kw)

        @staticmethod
        def backward(ctx, grad):
            if grad.stride(-1) != 1:        # (a broadcast gradient, or another order)
                grad = grad.contiguous()
            back = dict(ctx.kw, inverse=not ctx.kw["inverse"])
            return rotary(grad, *ctx.saved_tensors, **back), None, None, None, None

    class NoGradient(torch.autograd.Function):
        @staticmethod
        def forward(ctx, name, call, *inputs):
            ctx.name = name
            return call()

        @staticmethod
        def backward(ctx, *grads):
            raise RuntimeError(f"{ctx.name} has no gradient")

    return Rotary, NoGradient


class kv_cache:
    """A cache of key and value rows over tensors the caller owns: k and v are
    (pages, page, heads, d) float16 or bfloat16 device tensors, views of any strides with
    adjacent elements in a row; table is a (sequences, pages of a sequence)
    int32 device tensor of page numbers (rows of a page number that does not
    exist, as -1, do not exist), or None when sequence b is page b.  Row n of
    sequence b is row n % page of page table[b, n // page].  Another tensor may be
    assigned to k, v or table; it is checked as here, together with the others."""

    def __init__(self, k, v, table=None):
        self._describe(k, v, table)

    k = property(lambda self: self._k, lambda self, x: self._describe(x, self._v, self._table))
    v = property(lambda self: self._v, lambda self, x: self._describe(self._k, x, self._table))
    table = property(lambda self: self._table, lambda self, x: self._describe(self._k, self._v, x))

    def _describe(self, k, v, table):
        import torch
        if k.dtype not in (torch.float16, torch.bfloat16) or not k.is_cuda:
            raise ValueError("k must be a float16 or bfloat16 device tensor")
        _check_rows("k", k, (None,) * 4, k.dtype, k.device)
        _check_rows("v", v, tuple(k.shape), k.dtype, k.device)
        pages, page, heads, d = k.shape
        if table is not None:
            _check_rows("table", table, (None, None), torch.int32, k.device)
        self._k, self._v, self._table = k, v, table
        self.follows = _follows(k, v)
        self.dtype, self.device = k.dtype, k.device
        self.heads, self.d, self.page = heads, d, page
        self.batch, self.width = (pages, 1) if table is None else table.shape
        # (a table without columns has no address, but NULL would mean that there is none;
        # nothing is read of it)
        self.raw = sj_cache(dtype_code(k), heads, d, pages, page, self.batch, self.width,
                            0 if table is None else table.stride(0),
                            None if table is None else (_ptr(table) or _ptr(k)),
                            _ptr(k), _ptr(v), *k.stride()[:3], *v.stride()[:3])

    @property
    def room(self) -> int:
        """Rows a sequence may hold."""
        return self.width * self.page


def rotary_turns(rot: int, base: float = 10000.0, *, linear: float = 1.0, ramp=None, device="cuda"):
    """The frequencies of rotary positions over the first `rot` elements of a
    head, as the calls below take them: an int64 tensor of rot / 2 fixed-point
    fractions, turns a position in units of 2^-64.  Pair i has base^(-2 i / rot)
    radians a position.  Long contexts: `linear` divides every frequency;
    ramp = (s, length, low, high) divides by s the pairs that turn less than
    `low` times within `length` positions, leaves those that turn more than `high`
    times, and blends linearly between."""
    import math
    import torch
    if rot < 0 or rot % 2 or not base > 0 or not linear > 0:
        raise ValueError("rot must be even, base and linear positive")
    out = []
    for i in range(rot // 2):
        f = base ** (-2.0 * i / rot) / linear
        if ramp is not None:
            s, length, low, high = ramp
            g = min(max((length * f / (2 * math.pi) - low) / (high - low), 0.0), 1.0)
            f = f / s * (1.0 - g) + f * g
        out.append(round(f / (2 * math.pi) * 2.0 ** 64) % 2 ** 64)
    return torch.tensor([t - 2 ** 64 if t >= 2 ** 63 else t for t in out], dtype=torch.int64,
                        device=device)


def rotary(x, pos, turns, *, layout: str = "half", factor: float = 1.0, inverse: bool = False,
           out=None, ctx=None):
    """Rotary positions (sj_rotary): x (tokens, heads, d) with the first
    2 len(turns) elements of every head turned by the token's position (pos: int32
    per token) and scaled by `factor`; layout "half" pairs elements i and i +
    len(turns), "interleaved" 2 i and 2 i + 1.  inverse=True turns back: the
    gradient with respect to x of the call without it, given the gradient of its result;
    autograd takes it where x requires grad.  out may be x."""
    import torch
    if x.requires_grad or _follows(out):
        if torch.is_grad_enabled():
            if out is not None:
                _lost("rotary with out")
            return _functions()[0].apply(x, pos, turns, dict(layout=layout, factor=factor,
                                                             inverse=inverse), ctx)
    code = _layout_code(layout)
    if x.dtype not in (torch.float16, torch.bfloat16) or not x.is_cuda:
        raise ValueError("x must be a float16 or bfloat16 device tensor")
    dev = x.device
    if x.dim() != 3 or x.stride(-1) != 1:
        _refuse("x", x, (None,) * 3, x.dtype, dev)
    n, heads, d = x.shape
    _check_whole("pos", pos, (n,), torch.int32, dev)
    _check_whole("turns", turns, (turns.numel(),), torch.int64, dev)
    if out is None:
        out = x.new_empty(x.shape)
    else:
        _check_rows("out", out, x.shape, x.dtype, dev)
    st = sj_rotary(ctx or _current(dev), dtype_code(x), _ptr(x), x.stride()[:2], _ptr(out),
                   out.stride()[:2], n, heads, d, _ptr(pos), _ptr(turns), turns.shape[0], code,
                   factor, SJ_FLAG_INVERSE if inverse else 0)
    if st != SJ_OK:
        raise SjError(st, sj_last_error())
    return out


def cache_append(cache, lengths, key, value, *, pos=None, turns=None, q=None, layout: str = "half",
                 factor: float = 1.0, counts=None, q_out=None, ctx=None):
    """Appends rows to a cache (sj_cache_append): row lengths[b] + u of sequence
    b receives key[b, u], turned by position pos[b, u] where turns are given (see
    rotary), and value[b, u]; with counts only u < counts[b].  key and value
    are (sequences, tokens, heads, d); lengths and counts int32 per sequence, pos
    int32 (sequences, tokens).  q (sequences, tokens, query heads, d), when
    given, is turned by the same positions and returned (in q_out, which may be
    q).  There is no gradient: a backward pass through the result raises.  May be
    captured into a HIP graph, as rotary may."""
    import torch
    if cache.follows or key.requires_grad or value.requires_grad or _follows(q, q_out):
        if torch.is_grad_enabled():
            if q is None or q_out is not None or cache.follows:
                _lost("cache_append")
            return _functions()[1].apply("cache_append", functools.partial(
                cache_append, cache, lengths, key, value, pos=pos, turns=turns, q=q, layout=layout,
                factor=factor, counts=counts, ctx=ctx), q, key, value)
    code = _layout_code(layout)
    B, dev = cache.batch, cache.device
    if key.dim() != 4:
        _refuse("key", key, (B, None, cache.heads, cache.d), cache.dtype, dev)
    _check_rows("key", key, (B, key.shape[1], cache.heads, cache.d), cache.dtype, dev)
    _check_rows("value", value, key.shape, cache.dtype, dev)
    _check_whole("lengths", lengths, (B,), torch.int32, dev)
    if counts is not None:
        _check_whole("counts", counts, (B,), torch.int32, dev)
    t = key.shape[1]
    if (pos is None) != (turns is None):
        raise ValueError("pos and turns go together")
    if turns is not None:
        _check_whole("pos", pos, (B, t), torch.int32, dev)
        _check_whole("turns", turns, (turns.numel(),), torch.int64, dev)
    args = ()
    if q is not None:
        if q.dim() != 4:
            _refuse("q", q, (B, t, None, cache.d), cache.dtype, dev)
        _check_rows("q", q, (B, t, q.shape[2], cache.d), cache.dtype, dev)
        if q_out is None:
            q_out = q.new_empty(q.shape)
        else:
            _check_rows("q_out", q_out, q.shape, q.dtype, dev)
        if q.numel():
            args = (q.data_ptr(), q.stride()[:3], q.shape[2], q_out.data_ptr(), q_out.stride()[:3])
    st = sj_cache_append(ctx or _current(dev), cache.raw, _ptr(lengths), _ptr(counts), t,
                         _ptr(key), key.stride()[:3], _ptr(value), value.stride()[:3], _ptr(pos),
                         _ptr(turns), 0 if turns is None else turns.shape[0], code, factor, *args)
    if st != SJ_OK:
        raise SjError(st, sj_last_error())
    return q_out


def attend(cache, lengths, q, tree=None, *, scale: float | None = None, counts=None, weight=None,
           weight_out=None, out=None, ctx=None):
    """Attention of a few tokens of every sequence over its rows in the cache
    (sj_attend).  q is (sequences, tokens, query heads, d); query head i reads cache head
    i // (query heads / cache heads).  Token u of sequence b sees the
    lengths[b] rows before the call's tokens and, of the tokens' own rows (which
    follow them, appended beforehand), those that its mask names: bit w % 64 of
    tree[b, u, w // 64] for token w (tree: int64 (sequences or 1, tokens,
    ceil(tokens / 64))), or tokens up to itself without a tree.  counts (int32
    per sequence): tokens that exist.  scale defaults to 1 / sqrt(d).
    Returns (out, lse): out as q, lse (sequences, tokens, query heads) float32; a
    token that sees nothing has out 0 and lse -inf.  With weight (float32
    (sequences, cache heads, columns)) the softmax weight that every row drew from all
    tokens and query heads is added to it in place; weight_out receives the sum instead
    where given (with weight None, of this call alone).  There is no gradient: a backward
    pass through the results raises.
    In a HIP graph: a capture cannot grow the context's scratch, and contexts belong to
    streams, so make the call once on the stream that captures, which torch.cuda.graph
    has to be told:
        with torch.cuda.stream(side): attend(...)
        with torch.cuda.graph(g, stream=side): attend(...)"""
    import torch
    if cache.follows or q.requires_grad or _follows(out, weight, weight_out):
        if torch.is_grad_enabled():
            if out is not None or _follows(weight, weight_out):
                _lost("attend")
            return _functions()[1].apply("attend", functools.partial(
                attend, cache, lengths, q, tree, scale=scale, counts=counts, weight=weight,
                weight_out=weight_out, ctx=ctx), q, cache.k, cache.v)
    B, dev = cache.batch, cache.device
    if q.dim() != 4:
        _refuse("q", q, (B, None, None, cache.d), cache.dtype, dev)
    t, q_heads = q.shape[1], q.shape[2]
    _check_rows("q", q, (B, t, q_heads, cache.d), cache.dtype, dev)
    _check_whole("lengths", lengths, (B,), torch.int32, dev)
    if counts is not None:
        _check_whole("counts", counts, (B,), torch.int32, dev)
    tree_stride = (0, 0)
    if tree is not None:
        words = (t + 63) // 64
        _check_rows("tree", tree, (1 if tree.shape[0] == 1 else B, t, words), torch.int64, dev)
        tree_stride = (0 if tree.shape[0] == 1 else tree.stride(0), tree.stride(1))
    if weight is not None:
        _check_whole("weight", weight, (B, cache.heads, weight.shape[-1]), torch.float32, dev)
        if weight_out is None:
            weight_out = weight
    cols = 0
    if weight_out is not None:
        cols = weight_out.shape[-1]
        _check_whole("weight_out", weight_out, (B, cache.heads, cols if weight is None else
                                                weight.shape[2]), torch.float32, dev)
    if out is None:
        out = q.new_empty(q.shape)
    else:
        _check_whole("out", out, q.shape, cache.dtype, dev)
    lse = q.new_empty((B, t, q_heads), dtype=torch.float32)
    st = sj_attend(ctx or _current(dev), cache.raw, _ptr(lengths), _ptr(counts), t, _ptr(q),
                   q.stride()[:3], q_heads, _ptr(tree), tree_stride,
                   cache.d ** -0.5 if scale is None else scale, _ptr(out), _ptr(lse),
                   _ptr(weight), _ptr(weight_out), cols)
    if st != SJ_OK:
        raise SjError(st, sj_last_error())
    return out, lse


def cache_evict(cache, lengths, weight, into, *, keep: int, sink: int = 0, recent: int = 0,
                weight_out=None, ctx=None):
    """Eviction by accumulated weight (sj_cache_evict): of every sequence's rows
    the first `sink`, the last `recent` and the heaviest of the others stay, `keep`
    in all; they are copied, closed up and in order, into the cache `into` (other
    pages).  weight is (sequences, 1 or heads, columns) float32: one choice for
    all heads, or one for each.  Returns (index, lengths, weight): index
    (sequences, 1 or heads, keep) int32, the kept rows in ascending order, then
    -1; the new lengths (int32); and the kept weights, then zeros (weight_out where
    given, else as wide as index).  In a HIP graph: see attend."""
    import torch
    if cache.follows or into.follows or _follows(weight, weight_out):
        if torch.is_grad_enabled():
            _lost("cache_evict")
    B, dev = cache.batch, cache.device
    _check_whole("lengths", lengths, (B,), torch.int32, dev)
    if weight.dim() != 3:
        _refuse("weight", weight, (B, None, None), torch.float32, dev)
    _check_whole("weight", weight, (B, *weight.shape[1:]), torch.float32, dev)
    sets = weight.shape[1]
    if keep < 0 or sink < 0 or recent < 0:
        raise ValueError("keep, sink and recent must not be negative")
    index = lengths.new_empty((B, sets, keep))
    new = lengths.new_empty((B,))
    if weight_out is None:
        weight_out = weight.new_empty((B, sets, keep))
    else:
        _check_whole("weight_out", weight_out, (B, sets, weight_out.shape[-1]), torch.float32, dev)
    st = sj_cache_evict(ctx or _current(dev), cache.raw, _ptr(lengths), _ptr(weight), sets,
                        weight.shape[2], keep, sink, recent, into.raw, _ptr(index), _ptr(new),
                        _ptr(weight_out), weight_out.shape[2])
    if st != SJ_OK:
        raise SjError(st, sj_last_error())
    return index, new, weight_out
