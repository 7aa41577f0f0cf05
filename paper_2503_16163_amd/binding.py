"""Thin ctypes binding of libspecache.so: argument marshalling only.

Every step of the decode path runs in the HIP kernels behind the C ABI declared
in include/specache.h; the functions here carry the same names.  Tensors are
PyTorch tensors on the GPU (PyTorch provides device memory and streams) or raw
integer device addresses.  There is no CPU fallback: if the library is missing
or a call fails, an exception is raised.
"""
import ctypes as C
import os
import struct
import threading

from . import build as _build

FP16, BF16 = 0, 1
OK, EINVAL, ECAPACITY, ENOMEM, EHIP, ESTATE = 0, -1, -2, -3, -4, -5
_NAMES = {EINVAL: "EINVAL", ECAPACITY: "ECAPACITY", ENOMEM: "ENOMEM", EHIP: "EHIP", ESTATE: "ESTATE"}

EXPORTS = ["specache_create", "specache_destroy", "specache_last_error", "specache_counts",
           "specache_plan_append", "specache_quantize_append", "specache_score_topk", "specache_gather",
           "specache_score", "specache_select_gather", "specache_append_score",
           "specache_attend", "specache_score_attend", "specache_append_score_attend", "specache_decode_step", "specache_attend_static", "specache_debug_poison_slot", "specache_debug_fail_alloc", "specache_debug_scored_by_word", "specache_order_by_events", "specache_debug_kernel_choice", "specache_debug_merger_polls", "specache_export_quantized", "specache_export_rows", "specache_debug_logits",
           "specache_timing", "specache_measure_hbm_read", "specache_measure_link",
           "specache_rotary_plan", "specache_rotate", "specache_window_scratch", "specache_window_attend",
           "specache_sample_scratch", "specache_sample",
           "specache_paged_append", "specache_paged_scratch", "specache_paged_attend",
           "specache_block_scratch", "specache_block_select", "specache_block_attend"]


class Config(C.Structure):
    _fields_ = [(n, C.c_int32) for n in ("n_layers", "batch", "n_q_heads", "n_kv_heads", "head_dim", "bits",
                                         "group", "residual", "max_seq", "topk", "dtype")] + [("sm_scale", C.c_float),
                                                                                 ("one_bit_form", C.c_int32), ("select_form", C.c_int32),
                                                                                 ("select_cache", C.c_int32), ("async_select", C.c_int32)]


class View(C.Structure):
    _fields_ = [("data", C.c_void_p), ("batch", C.c_int64), ("head", C.c_int64), ("token", C.c_int64)]


ROTARY_HALF, ROTARY_INTERLEAVED = 0, 1
ROTARY_UNSCALED, ROTARY_LINEAR, ROTARY_BASE, ROTARY_BANDS, ROTARY_RAMP = range(5)
FP32 = 2   # a type of logits only


class RotaryConfig(C.Structure):
    _fields_ = [(n, C.c_int32) for n in ("rotary_dim", "layout", "scaling", "original_tokens")] + \
               [(n, C.c_double) for n in ("base", "factor", "low", "high", "gain")]


class Rotary(C.Structure):
    _fields_ = [("turns", C.c_uint64 * 64), ("gain", C.c_float), ("rotary_dim", C.c_int32), ("layout", C.c_int32)]


class WindowConfig(C.Structure):
    _fields_ = [(n, C.c_int32) for n in ("batch", "n_q_heads", "n_kv_heads", "head_dim", "q_tokens", "kv_tokens", "window", "sinks",
                                         "dtype")] + [("sm_scale", C.c_float)]


class SampleConfig(C.Structure):
    _fields_ = [("rows", C.c_int32), ("vocab", C.c_int32), ("dtype", C.c_int32), ("row_stride", C.c_int64)]


class PagesConfig(C.Structure):
    _fields_ = [("k", View), ("v", View), ("bounds", View), ("table", C.c_void_p), ("table_stride", C.c_int64)] + \
               [(n, C.c_int32) for n in ("n_pages", "n_kv_heads", "page_tokens", "table_pages", "head_dim", "dtype")]


class PagedConfig(C.Structure):
    _fields_ = [(n, C.c_int32) for n in ("batch", "n_q_heads", "q_tokens", "kv_tokens", "shared_tokens")] + [("sm_scale", C.c_float)]


class BlockConfig(C.Structure):
    _fields_ = [(n, C.c_int32) for n in ("batch", "n_q_heads", "q_tokens", "kv_tokens", "top", "first", "recent")] + [("sm_scale", C.c_float)]


class SpeCacheError(RuntimeError):
    def __init__(self, code, msg):
        super().__init__(f"specache: {_NAMES.get(code, code)}: {msg}")
        self.code = code


_lib = None


def lib():
    """Load libspecache.so.  It is built first if it was never built; a library older than its
    sources is an error (build again: python -m paper_2503_16163_amd.build), so that tests and
    timings never run on a stale build unnoticed."""
    global _lib
    if _lib is None:
        if not os.path.exists(_build.LIB):
            _build.build()
        elif not _build.is_built():
            raise RuntimeError("libspecache.so is older than its sources under csrc/ or include/specache.h: "
                               "run `python -m paper_2503_16163_amd.build` (or __graft_entry__.build())")
        L = C.CDLL(_build.LIB)
        vp, i32 = C.c_void_p, C.c_int32
        L.specache_create.argtypes = [C.POINTER(Config), C.POINTER(vp)]
        L.specache_destroy.argtypes = [vp]
        L.specache_last_error.argtypes = [vp]
        L.specache_last_error.restype = C.c_char_p
        L.specache_counts.argtypes = [vp, i32, C.POINTER(i32), C.POINTER(i32)]
        L.specache_plan_append.argtypes = [i32, i32, i32, i32, i32, C.POINTER(i32)]
        L.specache_quantize_append.argtypes = [vp, i32, vp, vp, i32, vp]
        L.specache_score_topk.argtypes = [vp, i32, vp, i32, vp, vp]
        L.specache_gather.argtypes = [vp, i32, vp, i32, vp]
        L.specache_score.argtypes = [vp, i32, vp, i32, vp]
        L.specache_select_gather.argtypes = [vp, i32, vp, i32, vp]
        L.specache_append_score.argtypes = [vp, i32, vp, vp, vp, i32, vp]
        L.specache_attend.argtypes = [vp, i32, vp, i32, vp, vp, i32, vp, vp]
        L.specache_attend_static.argtypes = [vp, i32, vp, i32, vp, vp, i32, vp, vp]
        L.specache_score_attend.argtypes = [vp, i32, vp, i32, vp, vp, i32, vp, vp]
        L.specache_append_score_attend.argtypes = [vp, i32, vp, vp, vp, i32, vp, vp, i32, vp, vp]
        L.specache_decode_step.argtypes = [vp, i32, vp, vp, vp, vp, vp, i32, vp, vp, vp, i32, vp]
        L.specache_debug_poison_slot.argtypes = [vp, i32, i32, vp]
        L.specache_debug_kernel_choice.argtypes = [i32]
        L.specache_debug_merger_polls.argtypes = [i32]
        L.specache_debug_fail_alloc.argtypes = [i32]
        L.specache_debug_scored_by_word.argtypes = [vp, i32, C.POINTER(i32)]
        L.specache_order_by_events.argtypes = [vp, i32]
        L.specache_export_quantized.argtypes = [vp, i32] + [vp] * 6
        L.specache_export_rows.argtypes = [vp, i32, i32, i32, vp]
        L.specache_debug_logits.argtypes = [vp, vp]
        L.specache_timing.argtypes = [vp, i32, vp, vp]
        L.specache_measure_hbm_read.argtypes = [C.c_int64, i32, C.POINTER(C.c_double)]
        L.specache_measure_link.argtypes = [C.c_int64, i32, C.POINTER(C.c_double), C.POINTER(C.c_double)]
        view, i64 = vp, C.c_int64      # (addresses of View structures)
        L.specache_rotary_plan.argtypes = [C.POINTER(RotaryConfig), C.POINTER(Rotary)]
        L.specache_rotate.argtypes = [C.POINTER(Rotary), i32, i32, i32, i32, view, view, i32, view, view, view, view, vp, i32, vp]
        L.specache_window_scratch.argtypes = [C.POINTER(WindowConfig), C.POINTER(i64)]
        L.specache_window_attend.argtypes = [C.POINTER(WindowConfig), view, view, view, view, vp, vp, vp, i64, vp]
        L.specache_sample_scratch.argtypes = [C.POINTER(SampleConfig), C.POINTER(i64)]
        L.specache_sample.argtypes = [C.POINTER(SampleConfig), vp, vp, vp, vp, vp, vp, vp, vp, i64, vp]
        pages, cfg = vp, vp            # (addresses of PagesConfig, PagedConfig and BlockConfig structures)
        L.specache_paged_append.argtypes = [pages, C.POINTER(Rotary), i32, i32, i32, view, view, view, view, vp, vp, vp, vp]
        L.specache_paged_scratch.argtypes = [pages, cfg, C.POINTER(i64)]
        L.specache_paged_attend.argtypes = [pages, cfg, view, view, vp, vp, vp, i64, vp]
        L.specache_block_scratch.argtypes = [pages, cfg, C.POINTER(i64)]
        L.specache_block_select.argtypes = [pages, cfg, view, vp, vp, vp, vp, i64, vp]
        L.specache_block_attend.argtypes = [pages, cfg, view, view, vp, vp, vp, vp, i64, vp]
        for name in EXPORTS:
            if name != "specache_last_error":
                getattr(L, name).restype = C.c_int
        _lib = L
    return _lib


def _ptr(x):
    """Device (or host) address of a tensor / numpy array / int / None."""
    if x is None:
        return None
    if isinstance(x, int):
        return x
    if hasattr(x, "data_ptr"):
        return x.data_ptr()
    return x.ctypes.data


def _stream(s):
    if s is None:
        return None
    if isinstance(s, int):
        return s
    return s.cuda_stream  # torch.cuda.Stream


def plan_append(residual, group, n_tokens, n_quantized, n_new):
    out = C.c_int32()
    rc = lib().specache_plan_append(residual, group, n_tokens, n_quantized, n_new, C.byref(out))
    if rc != OK:
        raise SpeCacheError(rc, "plan_append: inconsistent arguments")
    return out.value


SCORE_ON_VECTOR_ALU, ATTEND_ON_VECTOR_ALU, KEEP_ONE_PASS_LOGITS = 1, 2, 4


def debug_fail_alloc(nth):
    """The nth allocating call of the next specache_create fails (0: off)."""
    rc = lib().specache_debug_fail_alloc(nth)
    if rc != OK:
        raise SpeCacheError(rc, "specache_debug_fail_alloc")


def debug_kernel_choice(flags):
    """Process-wide: send the shapes the integer-matrix-core kernels take to the vector-ALU kernels (A/B timing)."""
    rc = lib().specache_debug_kernel_choice(flags)
    if rc != OK:
        raise SpeCacheError(rc, "debug_kernel_choice: unknown flag")


def debug_merger_polls(polls):
    """Process-wide: looks of a merging workgroup before it leaves its share to the last chunk (0: at once, -1: the default)."""
    rc = lib().specache_debug_merger_polls(polls)
    if rc != OK:
        raise SpeCacheError(rc, "debug_merger_polls: below -1")


def measure_hbm_read(nbytes=1 << 30, reps=10):
    """GB/s of a plain 128-bit streaming read of `nbytes` of device memory (median of `reps` launches)."""
    out = C.c_double()
    rc = lib().specache_measure_hbm_read(nbytes, reps, C.byref(out))
    if rc != OK:
        raise SpeCacheError(rc, "measure_hbm_read failed")
    return out.value


def measure_link(nbytes=256 << 20, reps=5):
    """(memcpy GB/s, zero-copy read kernel GB/s) of the host link over `nbytes` of pinned host memory."""
    a, b = C.c_double(), C.c_double()
    rc = lib().specache_measure_link(nbytes, reps, C.byref(a), C.byref(b))
    if rc != OK:
        raise SpeCacheError(rc, "measure_link failed")
    return a.value, b.value


# ---- calls without a context: torch tensors, strided where the C call takes views ------------------------------------
# Without a stream they go to torch's current one.  They have no backward pass: inputs that require gradients are read like any others, and
# the outputs carry none.

def _done(rc):
    if rc != OK:
        raise SpeCacheError(rc, lib().specache_last_error(None).decode())


def _refuse(what):
    raise SpeCacheError(EINVAL, what)


_torch, _TYPES = None, {}


def _with_torch():
    """Imports torch on the first call (the package itself needs none)."""
    global _torch
    if _torch is None:
        import torch
        _TYPES.update({torch.float16: FP16, torch.bfloat16: BF16, torch.float32: FP32})
        _torch = torch
    return _torch


def _here():
    return _with_torch().cuda.current_device()


def _current(stream, device):
    # (the device is known here: torch takes 1.5 us to find it)
    return _torch.cuda.current_stream(device).cuda_stream if stream is None else _stream(stream)


def _type_of(t):
    _with_torch()
    return _TYPES.get(t.dtype, -1)


class _Views(threading.local):
    """Room for the specache_views of one call (the call is over before the thread makes another)."""

    def __init__(self):
        self.room = (C.c_int64 * 24)()
        at = C.addressof(self.room)
        self.at = tuple(at + 32 * i for i in range(6))


_room = _Views()
_PACK = {n: struct.Struct(f"{4 * n}q").pack_into for n in (3, 4, 6)}


def _views(device, dtype, names, tensors, shapes):
    """Addresses of the specache_views of [batch, heads, tokens, 128] tensors (or None) of the given type and shapes on the current device,
    the channels side by side.  (Packed at once: a ctypes structure for each cost a call 6 of its 12 us.)"""
    fields = []
    for t, shape in zip(tensors, shapes):
        if t is None:
            fields += (0, 0, 0, 0)
            continue
        if t.shape != shape or t.dtype is not dtype or t.get_device() != device:
            _refuse(f"{names[len(fields) // 4]} must be a {tuple(shape)} tensor of q's type on the current device")
        b, h, n, c = t.stride()
        if c != 1:
            _refuse(f"{names[len(fields) // 4]}: the channels must lie side by side")
        # (any stride goes with a single one)
        fields += (t.data_ptr(), b if shape[0] > 1 else 0, h if shape[1] > 1 else 0, n if shape[2] > 1 else 0)
    _PACK[len(tensors)](_room.room, 0, *fields)
    return _room.at


def _flat(t, shape, kind, device, name):
    """Address of a contiguous tensor of the given shape and type on the current device, or None."""
    if t is None:
        return None
    if t.shape != shape or t.dtype is not kind or t.get_device() != device or not t.is_contiguous():
        _refuse(f"{name} must be a contiguous {tuple(shape)} tensor of {kind} on the current device")
    return t.data_ptr()


def _scratch(t, device):
    if t is None:
        return None, 0
    if t.get_device() != device or not t.is_contiguous():
        _refuse("scratch must be contiguous and on the current device")
    return t.data_ptr(), t.nbytes


def rotary_plan(rotary_dim=128, base=10000.0, layout=ROTARY_HALF, scaling=ROTARY_UNSCALED, factor=1.0, original_tokens=0,
                low=0.0, high=0.0, gain=0.0):
    """A worked-out rotary configuration for rotate (host only)."""
    out = Rotary()
    _done(lib().specache_rotary_plan(C.byref(RotaryConfig(rotary_dim, layout, scaling, original_tokens, base, factor, low, high, gain)),
                                     C.byref(out)))
    return out


def rotate(plan, q, q_out, k=None, k_out=None, v=None, v_out=None, positions=None, first_position=0, stream=None):
    """q [B, Hq, n, 128] and k [B, Hkv, n, 128] turned by their positions, v as it is, each into its output, in one launch."""
    shape = q.shape
    B, Hq, n, _ = shape
    kv = v if k is None else k
    kv_shape = None if kv is None else (B, kv.shape[1], n, 128)
    if (k is None) != (k_out is None) or (v is None) != (v_out is None):
        _refuse("a tensor and its output are given or left out together")
    device = _here()
    if shape[3] != 128:
        _refuse("a head has 128 channels")
    a = _views(device, q.dtype, ("q", "q_out", "k", "k_out", "v", "v_out"), (q, q_out, k, k_out, v, v_out),
               (shape, shape, kv_shape, kv_shape, kv_shape, kv_shape))
    _done(lib().specache_rotate(C.byref(plan), _type_of(q), B, n, Hq, a[0], a[1], 0 if kv is None else kv_shape[1],
                                None if k is None else a[2], None if k is None else a[3], None if v is None else a[4], None if v is None else a[5],
                                _flat(positions, (B, n), _torch.int32, device, "positions"), first_position, _current(stream, device)))


def window_scratch(batch, n_q_heads, n_kv_heads, q_tokens, kv_tokens, window=0, sinks=0):
    """Bytes of scratch memory that window_attend needs for these counts (0: none)."""
    out = C.c_int64()
    _done(lib().specache_window_scratch(C.byref(WindowConfig(batch, n_q_heads, n_kv_heads, 128, q_tokens, kv_tokens, window, sinks)),
                                        C.byref(out)))
    return out.value


def window_attend(q, k, v, out, window=0, sinks=0, q_lengths=None, kv_lengths=None, sm_scale=0.0, scratch=None, stream=None):
    """Attention of q [B, Hq, n, 128] over k, v [B, Hkv, N, 128] with a sliding window and sinks, into out (q's shape)."""
    rows, pairs = q.shape, k.shape
    B, Hq, n, D = rows
    device = _here()
    if pairs[0] != B or D != 128 or pairs[3] != 128:
        _refuse("q is [B, Hq, n, 128], k and v are [B, Hkv, N, 128]")
    a = _views(device, q.dtype, ("q", "k", "v", "out"), (q, k, v, out), (rows, pairs, pairs, rows))
    cfg = WindowConfig(B, Hq, pairs[1], D, n, pairs[2], window, sinks, _type_of(q), sm_scale)
    address, size = _scratch(scratch, device)
    _done(lib().specache_window_attend(C.byref(cfg), a[0], a[1], a[2], a[3], _flat(q_lengths, (B,), _torch.int32, device, "q_lengths"),
                                       _flat(kv_lengths, (B,), _torch.int32, device, "kv_lengths"), address, size, _current(stream, device)))


def sample_scratch(rows, vocab, dtype):
    """Bytes of scratch memory that sample needs (0: none); dtype: the logits' torch type or FP16, BF16, FP32."""
    if not isinstance(dtype, int):
        _with_torch()
        dtype = _TYPES.get(dtype, -1)
    out = C.c_int64()
    _done(lib().specache_sample_scratch(C.byref(SampleConfig(rows, vocab, dtype, vocab)), C.byref(out)))
    return out.value


def sample(logits, u, tokens, temperature=None, top_k=None, top_p=None, min_p=None, scratch=None, stream=None):
    """tokens[r] from logits [rows, vocab] (rows may lie apart) and the random numbers u [rows]."""
    R, V = logits.shape
    device = _here()
    if logits.get_device() != device or (V > 1 and logits.stride(1) != 1):
        _refuse("logits must be on the current device, a row's side by side")
    cfg = SampleConfig(R, V, _type_of(logits), logits.stride(0) if R > 1 else V)
    f32, i32, shape = _torch.float32, _torch.int32, (R,)
    address, size = _scratch(scratch, device)
    _done(lib().specache_sample(C.byref(cfg), logits.data_ptr(), _flat(u, shape, f32, device, "u"),
                                _flat(temperature, shape, f32, device, "temperature"), _flat(top_k, shape, i32, device, "top_k"),
                                _flat(top_p, shape, f32, device, "top_p"), _flat(min_p, shape, f32, device, "min_p"),
                                _flat(tokens, shape, i32, device, "tokens"), address, size, _current(stream, device)))


class _Room(threading.local):
    """Room for two specache_views and a configuration behind them, packed at once."""

    def __init__(self):
        self.room = (C.c_int64 * 12)()
        self.q = C.addressof(self.room)
        self.out, self.cfg = self.q + 32, self.q + 64


_call = _Room()
_PACK_PAGED = struct.Struct("8q5if").pack_into
_PACK_BLOCKS = struct.Struct("8q7if").pack_into
_PACK_PAGED_COUNTS = struct.Struct("5if").pack_into
_PACK_BLOCK_COUNTS = struct.Struct("7if").pack_into
_WIDE = "counts must be whole numbers of 32 bits, sm_scale a number"
_MOST = 2 ** 31 - 1    # (ctypes would cut a longer count off without a word)


def _rows(t, shape, kind, device, name):
    """The fields of a [B, H, n, 128] tensor's specache_view."""
    if t.shape != shape or t.dtype is not kind or t.get_device() != device:
        _refuse(f"{name} must be a {tuple(shape)} tensor of the cache's type on the current device")
    b, h, n, c = t.stride()
    if c != 1:
        _refuse(f"{name}: the channels must lie side by side")
    return t.data_ptr(), b if shape[0] > 1 else 0, h if shape[1] > 1 else 0, n if shape[2] > 1 else 0


class Pages:
    """A layer's paged cache for the calls below: k, v [pages, Hkv, page_tokens, 128] and bounds [pages, Hkv, 2, 128] (views as they are), table [B, table_pages]
    int32 (a row's entries side by side).  It keeps the tensors; what is in them may change between calls."""

    def __init__(self, k, v, table, bounds=None):
        self.device, self.kind, self.k, self.v, self.table, self.bounds = _here(), k.dtype, k, v, table, bounds
        if k.dim() != 4 or k.shape[3] != 128 or _type_of(k) not in (FP16, BF16):
            _refuse("k must be a [pages, KV heads, page_tokens, 128] tensor of a 16-bit type")
        P, H, T, _ = k.shape
        views = _views(self.device, k.dtype, ("k", "v", "bounds"), (k, v, bounds), (k.shape, k.shape, (P, H, 2, 128)))
        if table.dim() != 2 or table.dtype is not _torch.int32 or table.get_device() != self.device or (table.shape[1] > 1 and table.stride(1) != 1):
            _refuse("table must be a [batch, pages] tensor of int32 on the current device, a row's entries side by side")
        if max(P, H, T, table.shape[1]) > _MOST:
            _refuse(_WIDE)
        self.batch, self.kv_heads, self.places = table.shape[0], H, table.shape[1] * T
        self.config = PagesConfig(*(View.from_address(at) for at in views[:3]), table.data_ptr(), table.stride(0) if table.shape[0] > 1 else table.shape[1],
                                  P, H, T, table.shape[1], 128, _type_of(k))
        self.at = C.addressof(self.config)

    def _shape(self, q):
        """q's shape and the device, checked against the cache's."""
        shape, device = q.shape, _here()
        if device != self.device:
            _refuse("the cache is not on the current device")
        if len(shape) != 4 or shape[3] != 128 or shape[0] != self.batch:
            _refuse("q is [B, Hq, n, 128], with as many sequences as the table has")
        return shape, device


def paged_append(cache, plan, k, v, q=None, q_out=None, starts=None, lengths=None, positions=None, stream=None):
    """k, v [B, Hkv, n, 128] to positions starts[b] .. of the cache, k turned by plan (None: as it is); q [B, Hq, n, 128] turned into q_out."""
    B, _, n, _ = k.shape
    device, H, kind = _here(), cache.kv_heads, cache.kind
    if device != cache.device or B != cache.batch:
        _refuse("the cache is not on the current device, or has other sequences")
    if n > _MOST or B > _MOST or (q is not None and q.shape[1] > _MOST):
        _refuse(_WIDE)
    if (q is None) != (q_out is None):
        _refuse("a tensor and its output are given or left out together")
    if q is None:
        heads, rows, out = 0, (0, 0, 0, 0), (0, 0, 0, 0)
    else:
        heads = q.shape[1]
        shape = (B, heads, n, 128)
        rows, out = _rows(q, shape, kind, device, "q"), _rows(q_out, shape, kind, device, "q_out")
    shape = (B, H, n, 128)
    _PACK[4](_room.room, 0, *rows, *out, *_rows(k, shape, kind, device, "k"), *_rows(v, shape, kind, device, "v"))
    a, i32 = _room.at, _torch.int32
    _done(lib().specache_paged_append(cache.at, None if plan is None else C.byref(plan), B, n, heads, a[0], a[1], a[2], a[3],
                                      _flat(starts, (B,), i32, device, "starts"), _flat(lengths, (B,), i32, device, "lengths"),
                                      _flat(positions, (B, n), i32, device, "positions"), _current(stream, device)))


def paged_scratch(cache, batch, n_q_heads, q_tokens, kv_tokens, shared_tokens=0):
    """Bytes of scratch memory that paged_attend needs for these counts (0: none)."""
    out, c = C.c_int64(), _call
    try:
        _PACK_PAGED_COUNTS(c.room, 64, batch, n_q_heads, q_tokens, kv_tokens, shared_tokens, 0.0)
    except struct.error:
        _refuse(_WIDE)
    _done(lib().specache_paged_scratch(cache.at, c.cfg, C.byref(out)))
    return out.value


def paged_attend(cache, q, out, kv_tokens=None, shared_tokens=0, q_lengths=None, kv_lengths=None, sm_scale=0.0, scratch=None, stream=None):
    """Attention of q [B, Hq, n, 128] over the cache's positions (kv_tokens at most; None: what the table holds), whose first shared_tokens the sequences
    share, into out (q's shape)."""
    shape, device = cache._shape(q)
    B, Hq, n, _ = shape
    kind, i32, c = cache.kind, _torch.int32, _call
    try:
        _PACK_PAGED(c.room, 0, *_rows(q, shape, kind, device, "q"), *_rows(out, shape, kind, device, "out"),
                    B, Hq, n, cache.places if kv_tokens is None else kv_tokens, shared_tokens, sm_scale)
    except struct.error:
        _refuse(_WIDE)
    address, size = _scratch(scratch, device)
    _done(lib().specache_paged_attend(cache.at, c.cfg, c.q, c.out, _flat(q_lengths, (B,), i32, device, "q_lengths"),
                                      _flat(kv_lengths, (B,), i32, device, "kv_lengths"), address, size, _current(stream, device)))


def block_scratch(cache, batch, n_q_heads, q_tokens, kv_tokens, top, first=0, recent=0):
    """Bytes of scratch memory that block_select and block_attend need for these counts (0: none)."""
    out, c = C.c_int64(), _call
    try:
        _PACK_BLOCK_COUNTS(c.room, 64, batch, n_q_heads, q_tokens, kv_tokens, top, first, recent, 0.0)
    except struct.error:
        _refuse(_WIDE)
    _done(lib().specache_block_scratch(cache.at, c.cfg, C.byref(out)))
    return out.value


def block_select(cache, q, blocks, kv_tokens=None, top=0, first=0, recent=0, q_lengths=None, kv_lengths=None, scratch=None, stream=None):
    """blocks [B, Hkv, n, first + top + recent] of int32: the blocks of the cache (its pages) that the rows of q [B, Hq, n, 128] see."""
    shape, device = cache._shape(q)
    B, Hq, n, _ = shape
    i32, c = _torch.int32, _call
    if cache.bounds is None and top > 0:
        _refuse("the cache keeps no bounds")
    lists = _flat(blocks, (B, cache.kv_heads, n, first + top + recent), i32, device, "blocks")
    try:
        _PACK_BLOCKS(c.room, 0, *_rows(q, shape, cache.kind, device, "q"), 0, 0, 0, 0,
                     B, Hq, n, cache.places if kv_tokens is None else kv_tokens, top, first, recent, 0.0)
    except struct.error:
        _refuse(_WIDE)
    address, size = _scratch(scratch, device)
    _done(lib().specache_block_select(cache.at, c.cfg, c.q, lists, _flat(q_lengths, (B,), i32, device, "q_lengths"),
                                      _flat(kv_lengths, (B,), i32, device, "kv_lengths"), address, size, _current(stream, device)))


def block_attend(cache, q, out, blocks, kv_tokens=None, q_lengths=None, kv_lengths=None, sm_scale=0.0, scratch=None, stream=None):
    """Attention of q [B, Hq, n, 128] over the listed blocks [B, Hkv, n, entries] of the cache, into out (q's shape)."""
    shape, device = cache._shape(q)
    B, Hq, n, _ = shape
    kind, i32, c = cache.kind, _torch.int32, _call
    if blocks.dim() != 4:
        _refuse("blocks is [B, Hkv, n, entries]")
    slots = blocks.shape[3]
    lists = _flat(blocks, (B, cache.kv_heads, n, slots), i32, device, "blocks")
    try:
        _PACK_BLOCKS(c.room, 0, *_rows(q, shape, kind, device, "q"), *_rows(out, shape, kind, device, "out"),
                     B, Hq, n, cache.places if kv_tokens is None else kv_tokens, slots, 0, 0, sm_scale)
    except struct.error:
        _refuse(_WIDE)
    address, size = _scratch(scratch, device)
    _done(lib().specache_block_attend(cache.at, c.cfg, c.q, c.out, lists, _flat(q_lengths, (B,), i32, device, "q_lengths"),
                                      _flat(kv_lengths, (B,), i32, device, "kv_lengths"), address, size, _current(stream, device)))


class SpeCache:
    """Owner of a specache_ctx; methods mirror the C calls one to one."""

    def __init__(self, n_layers, batch, n_q_heads, n_kv_heads, bits, group, max_seq, topk, dtype,
                 residual=64, head_dim=128, sm_scale=0.0, one_bit_form=0, select_form=0, select_cache=0, async_select=0):
        self.cfg = Config(n_layers, batch, n_q_heads, n_kv_heads, head_dim, bits, group, residual, max_seq,
                          topk, dtype, sm_scale, one_bit_form, select_form, select_cache, async_select)
        self._ctx = C.c_void_p()
        rc = lib().specache_create(C.byref(self.cfg), C.byref(self._ctx))
        if rc != OK:
            raise SpeCacheError(rc, lib().specache_last_error(None).decode())

    def close(self):
        if getattr(self, "_ctx", None):
            lib().specache_destroy(self._ctx)
            self._ctx = None

    def __del__(self):
        self.close()

    def _check(self, rc):
        if rc != OK:
            raise SpeCacheError(rc, lib().specache_last_error(self._ctx).decode())

    def counts(self, layer):
        n, nq = C.c_int32(), C.c_int32()
        self._check(lib().specache_counts(self._ctx, layer, C.byref(n), C.byref(nq)))
        return n.value, nq.value

    def quantize_append(self, layer, k_new, v_new, n_new, stream=None):
        self._check(lib().specache_quantize_append(self._ctx, layer, _ptr(k_new), _ptr(v_new), n_new, _stream(stream)))

    def score_topk(self, layer, q, n_rows, topk_idx_out, stream=None):
        self._check(lib().specache_score_topk(self._ctx, layer, _ptr(q), n_rows, _ptr(topk_idx_out), _stream(stream)))

    def score(self, layer, q, n_rows, stream=None):
        self._check(lib().specache_score(self._ctx, layer, _ptr(q), n_rows, _stream(stream)))

    def append_score(self, layer, k_new, v_new, q, n_rows, stream=None):
        self._check(lib().specache_append_score(self._ctx, layer, _ptr(k_new), _ptr(v_new), _ptr(q), n_rows, _stream(stream)))

    def select_gather(self, layer, topk_idx_out, slot, side_stream=None):
        self._check(lib().specache_select_gather(self._ctx, layer, _ptr(topk_idx_out), slot, _stream(side_stream)))

    def gather(self, layer, idx, slot, side_stream=None):
        self._check(lib().specache_gather(self._ctx, layer, _ptr(idx), slot, _stream(side_stream)))

    def attend(self, layer, q, n_rows, k_spec, v_spec, slot, out, stream=None):
        self._check(lib().specache_attend(self._ctx, layer, _ptr(q), n_rows, _ptr(k_spec), _ptr(v_spec), slot,
                                          _ptr(out), _stream(stream)))

    def score_attend(self, layer, q, n_rows, k_spec, v_spec, slot, out, stream=None):
        self._check(lib().specache_score_attend(self._ctx, layer, _ptr(q), n_rows, _ptr(k_spec), _ptr(v_spec), slot,
                                                _ptr(out), _stream(stream)))

    def append_score_attend(self, layer, k_new, v_new, q, n_rows, k_spec, v_spec, slot, out, stream=None):
        self._check(lib().specache_append_score_attend(self._ctx, layer, _ptr(k_new), _ptr(v_new), _ptr(q), n_rows,
                                                       _ptr(k_spec), _ptr(v_spec), slot, _ptr(out), _stream(stream)))

    def decode_step(self, layer, k_new, v_new, q, k_spec, v_spec, read_slot, out, stream, topk_idx_out, fill_slot, side_stream):
        self._check(lib().specache_decode_step(self._ctx, layer, _ptr(k_new), _ptr(v_new), _ptr(q), _ptr(k_spec), _ptr(v_spec),
                                               read_slot, _ptr(out), _stream(stream), _ptr(topk_idx_out), fill_slot,
                                               _stream(side_stream)))

    def attend_static(self, layer, q, n_rows, k_spec, v_spec, slot, out, stream=None):
        self._check(lib().specache_attend_static(self._ctx, layer, _ptr(q), n_rows, _ptr(k_spec), _ptr(v_spec), slot,
                                                 _ptr(out), _stream(stream)))

    def debug_poison_slot(self, layer, slot, stream=None):
        self._check(lib().specache_debug_poison_slot(self._ctx, layer, slot, _stream(stream)))

    def order_by_events(self, enable):
        self._check(lib().specache_order_by_events(self._ctx, int(bool(enable))))

    def debug_scored_by_word(self, layer):
        out = C.c_int32()
        self._check(lib().specache_debug_scored_by_word(self._ctx, layer, C.byref(out)))
        return bool(out.value)

    KERNELS = ("flush", "append_copy", "score", "topk", "gather", "attend", "attend_combine", "score_attend")

    def timing(self, enable):
        """Collect and reset per-kernel event timings; returns {kernel: (total_us, launches)}."""
        us = (C.c_double * len(self.KERNELS))()
        n = (C.c_int64 * len(self.KERNELS))()
        self._check(lib().specache_timing(self._ctx, int(bool(enable)), us, n))
        return {k: (us[i], n[i]) for i, k in enumerate(self.KERNELS)}

    # ---- parity hooks (host numpy arrays) ------------------------------------
    def export_quantized(self, layer):
        import numpy as np
        c = self.cfg
        rows, (_, nq), g, D = c.batch * c.n_kv_heads, self.counts(layer), c.group, c.head_dim
        shp = (c.batch, c.n_kv_heads)
        r = dict(k_codes=np.zeros(shp + (nq, D), np.uint8), k_mnmx=np.zeros(shp + (nq // g, D, 2), np.uint16),
                 k_sz=np.zeros(shp + (nq // g, D, 2), np.float32), v_codes=np.zeros(shp + (nq, D), np.uint8),
                 v_mnmx=np.zeros(shp + (nq, D // g, 2), np.uint16), v_sz=np.zeros(shp + (nq, D // g, 2), np.float32))
        self._check(lib().specache_export_quantized(self._ctx, layer, _ptr(r["k_codes"]), _ptr(r["k_mnmx"]),
                                                    _ptr(r["k_sz"]), _ptr(r["v_codes"]), _ptr(r["v_mnmx"]),
                                                    _ptr(r["v_sz"])))
        return r

    def export_rows(self, layer, first, count):
        import numpy as np
        c = self.cfg
        out = np.zeros((c.batch, c.n_kv_heads, count, 2, c.head_dim), np.uint16)
        self._check(lib().specache_export_rows(self._ctx, layer, first, count, _ptr(out)))
        return out

    def debug_logits(self, layer, n_rows):
        import numpy as np
        c = self.cfg
        _, nq = self.counts(layer)
        out = np.zeros((c.batch, c.n_q_heads, n_rows, nq), np.float32)
        self._check(lib().specache_debug_logits(self._ctx, _ptr(out)))
        return out
