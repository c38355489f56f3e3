"""Python binding of the eosq C-ABI library (argument marshalling only).

Every step of the compression path runs inside ``libeosq.so`` (hand-written CUDA for
sm_100a); PyTorch is used here for device memory and streams.  The functions carry the
names of the C entry points declared in ``include/eosq.h``.  There is no CPU fallback:
if the library has not been built the first call raises.
"""
from __future__ import annotations

import ctypes
from dataclasses import dataclass
from pathlib import Path
from typing import Optional

import numpy as np

_PKG = Path(__file__).resolve().parent
LIB_PATH = _PKG / "libeosq.so"

EOSQ_OK, EOSQ_ERR_INVALID_ARG, EOSQ_ERR_UNSUPPORTED, EOSQ_ERR_BUFFER_TOO_SMALL, EOSQ_ERR_CUDA, EOSQ_WARN_BLOCK_STATUS = range(6)
EOSQ_F16, EOSQ_F32, EOSQ_BF16 = 0, 1, 2
EOSQ_KV_INT8, EOSQ_KV_E4M3 = 0, 1
EOSQ_KV8_NO_PAGE, EOSQ_KV8_TOO_LONG, EOSQ_KV8_BAD_SEQ, EOSQ_KV8_BAD_PAGE = 1, 2, 4, 8
EOSQ_RMAX = 16
STATUS_NAMES = {0: "OK", 1: "INVALID_ARG", 2: "UNSUPPORTED", 3: "BUFFER_TOO_SMALL", 4: "CUDA", 5: "BLOCK_STATUS"}

EXPORTS = [
    "eosq_pilot_k", "eosq_codebook", "eosq_rotation", "eosq_layout", "eosq_bits_per_entry",
    "eosq_workspace_bytes", "eosq_create", "eosq_destroy", "eosq_last_cuda_error", "eosq_encode",
    "eosq_decode", "eosq_scores", "eosq_encode_host_arena_bytes", "eosq_encode_host",
    "eosq_check_status", "eosq_launch_count", "eosq_profile_enable", "eosq_profile_select", "eosq_profile_read",
    "eosq_encode_static", "eosq_encode_static_max_blocks", "eosq_selftest_wait_timeout",
    "eosq_kv8_workspace_bytes", "eosq_kv8_reserve", "eosq_kv8_store", "eosq_kv8_attend", "eosq_kv8_fork", "eosq_kv8_free",
    "eosq_kv8_compact", "eosq_kv8_copy_pages", "eosq_kv8_check",
]
STAGES = ["gram", "tridiag_a", "tridiag_b", "tridiag_c", "eigvals", "spectral", "quant", "decode", "scores", "redo", "other"]


class EosqError(RuntimeError):
    def __init__(self, code, what, detail=""):
        super().__init__(f"{what}: EOSQ_{STATUS_NAMES.get(code, code)}" + (f" ({detail})" if detail else ""))
        self.code = code


class _CacheStruct(ctypes.Structure):
    _fields_ = [(name, ctypes.c_void_p) for name in
                ("codes", "norms", "rank", "sigma", "phi", "P", "V", "status", "eig", "lambda_plus", "vr32", "coef")]


class _LayoutStruct(ctypes.Structure):
    _fields_ = [("k", ctypes.c_int32), ("rmax", ctypes.c_int32), ("row_bytes", ctypes.c_int32),
                ("reserved", ctypes.c_int32)] + [
        (name, ctypes.c_int64) for name in
        ("codes_bytes", "norms_bytes", "P_bytes", "V_bytes", "sigma_bytes", "phi_bytes", "eig_bytes", "stored_bytes")]


class _Kv8Struct(ctypes.Structure):
    _fields_ = [(name, ctypes.c_void_p) for name in ("k", "v", "k_scale", "v_scale", "table", "lengths", "refs", "flags")] + [
        (name, ctypes.c_int32) for name in ("layers", "num_pages", "kv_heads", "page_size", "d", "format", "max_seqs", "max_pages")]


_lib = None


def lib():
    """The loaded shared library; raises if it has not been built (no fallback exists)."""
    global _lib
    if _lib is None:
        if not LIB_PATH.exists():
            raise RuntimeError(
                f"{LIB_PATH} is missing: build it with `python -m paper_2605_02905_b200.build` "
                "(nvcc, sm_100a).  There is no CPU fallback.")
        L = ctypes.CDLL(str(LIB_PATH))
        L.eosq_bits_per_entry.restype = ctypes.c_double
        L.eosq_bits_per_entry.argtypes = [ctypes.c_int, ctypes.c_double, ctypes.c_int, ctypes.c_int, ctypes.c_double, ctypes.c_int]
        L.eosq_workspace_bytes.restype = ctypes.c_size_t
        L.eosq_workspace_bytes.argtypes = [ctypes.c_int64, ctypes.c_int, ctypes.c_int]
        L.eosq_encode_host_arena_bytes.restype = ctypes.c_size_t
        L.eosq_encode_host_arena_bytes.argtypes = [ctypes.c_int64, ctypes.c_int, ctypes.c_int, ctypes.c_int, ctypes.c_int]
        L.eosq_last_cuda_error.restype = ctypes.c_char_p
        L.eosq_last_cuda_error.argtypes = [ctypes.c_void_p]
        L.eosq_launch_count.restype = ctypes.c_int64
        L.eosq_launch_count.argtypes = [ctypes.c_void_p]
        L.eosq_rotation.argtypes = [ctypes.c_int, ctypes.c_uint64, ctypes.c_void_p]
        L.eosq_codebook.argtypes = [ctypes.c_int, ctypes.c_int, ctypes.c_void_p, ctypes.c_void_p]
        L.eosq_layout.argtypes = [ctypes.c_int, ctypes.c_int, ctypes.c_int, ctypes.c_void_p]
        L.eosq_create.argtypes = [ctypes.c_void_p]
        L.eosq_destroy.argtypes = [ctypes.c_void_p]
        L.eosq_encode.argtypes = [ctypes.c_void_p, ctypes.c_void_p, ctypes.c_int, ctypes.c_int64, ctypes.c_int, ctypes.c_int,
                                  ctypes.c_int, ctypes.c_uint64, ctypes.c_void_p, ctypes.c_void_p, ctypes.c_size_t, ctypes.c_void_p]
        L.eosq_encode_static.argtypes = [ctypes.c_void_p, ctypes.c_void_p, ctypes.c_int, ctypes.c_int64, ctypes.c_int, ctypes.c_int,
                                         ctypes.c_int, ctypes.c_uint64, ctypes.c_void_p, ctypes.c_void_p]
        L.eosq_encode_static_max_blocks.restype = ctypes.c_int64
        L.eosq_encode_static_max_blocks.argtypes = []
        L.eosq_decode.argtypes = [ctypes.c_void_p, ctypes.c_void_p, ctypes.c_int64, ctypes.c_int, ctypes.c_int, ctypes.c_int,
                                  ctypes.c_uint64, ctypes.c_void_p, ctypes.c_int, ctypes.c_void_p]
        L.eosq_scores.argtypes = [ctypes.c_void_p, ctypes.c_void_p, ctypes.c_int64, ctypes.c_int64, ctypes.c_int64, ctypes.c_int,
                                  ctypes.c_int, ctypes.c_int, ctypes.c_uint64, ctypes.c_void_p, ctypes.c_int, ctypes.c_float,
                                  ctypes.c_void_p, ctypes.c_void_p]
        L.eosq_encode_host.argtypes = [ctypes.c_void_p, ctypes.c_void_p, ctypes.c_int, ctypes.c_int64, ctypes.c_int, ctypes.c_int,
                                       ctypes.c_int, ctypes.c_uint64, ctypes.c_void_p, ctypes.c_void_p, ctypes.c_size_t, ctypes.c_void_p]
        L.eosq_selftest_wait_timeout.argtypes = [ctypes.c_void_p, ctypes.c_uint32, ctypes.c_void_p]
        L.eosq_profile_enable.argtypes = [ctypes.c_void_p, ctypes.c_int]
        L.eosq_profile_select.argtypes = [ctypes.c_void_p, ctypes.c_uint32]
        L.eosq_profile_read.argtypes = [ctypes.c_void_p, ctypes.c_void_p, ctypes.c_void_p]
        L.eosq_check_status.argtypes = [ctypes.c_void_p, ctypes.c_void_p, ctypes.c_int64, ctypes.c_void_p, ctypes.c_void_p]
        p, i32, i64 = ctypes.c_void_p, ctypes.c_int, ctypes.c_int64
        L.eosq_kv8_workspace_bytes.restype = ctypes.c_size_t
        L.eosq_kv8_workspace_bytes.argtypes = [p, i32]
        L.eosq_kv8_reserve.argtypes = [p, p, p, p, i32, p, p]
        L.eosq_kv8_store.argtypes = [p, p, i32, p, p, i32, i64, i64, i64, i64, i64, p, p, p, i32, i32, p]
        L.eosq_kv8_attend.argtypes = [p, p, i32, p, i32, i64, i64, i64, p, p, i32, i32, i32, ctypes.c_float, i32, i32, p, i64, i64, p, p,
                                      ctypes.c_size_t, p]
        L.eosq_kv8_fork.argtypes = [p, p, p, p, i32, p, ctypes.c_size_t, p]
        L.eosq_kv8_free.argtypes = [p, p, p, i32, p]
        L.eosq_kv8_compact.argtypes = [p, p, p, p, ctypes.c_size_t, p]
        L.eosq_kv8_copy_pages.argtypes = [p, p, p, p, p, i32, p]
        L.eosq_kv8_check.argtypes = [p, p, p, p]
        _lib = L
    return _lib


def _check(rc, what, ctx=None):
    if rc != EOSQ_OK:
        detail = ""
        if rc == EOSQ_ERR_CUDA and ctx is not None:
            detail = lib().eosq_last_cuda_error(ctx._h).decode()
        raise EosqError(rc, what, detail)


# ---- host-side pure functions ------------------------------------------------------------

def eosq_pilot_k(d: int) -> int:
    return int(lib().eosq_pilot_k(int(d)))


def eosq_codebook(bits: int, d: int):
    cen = np.zeros(1 << bits, dtype=np.float64)
    thr = np.zeros((1 << bits) - 1, dtype=np.float64)
    _check(lib().eosq_codebook(int(bits), int(d), cen.ctypes.data, thr.ctypes.data), "eosq_codebook")
    return cen, thr


def eosq_rotation(d: int, seed: int):
    pi = np.zeros((d, d), dtype=np.float64)
    _check(lib().eosq_rotation(int(d), ctypes.c_uint64(seed), pi.ctypes.data), "eosq_rotation")
    return pi


def eosq_layout(n: int, d: int, bits: int) -> dict:
    s = _LayoutStruct()
    _check(lib().eosq_layout(int(n), int(d), int(bits), ctypes.addressof(s)), "eosq_layout")
    return {name: int(getattr(s, name)) for name, _ in _LayoutStruct._fields_ if name != "reserved"}


def eosq_bits_per_entry(bits: int, rank: float, n: int, d: int, b_s: float, prod: bool = False) -> float:
    return float(lib().eosq_bits_per_entry(int(bits), float(rank), int(n), int(d), float(b_s), int(bool(prod))))


def eosq_workspace_bytes(num_blocks: int, n: int, d: int) -> int:
    return int(lib().eosq_workspace_bytes(int(num_blocks), int(n), int(d)))


def eosq_encode_host_arena_bytes(num_blocks: int, n: int, d: int, bits: int, in_dtype: int) -> int:
    return int(lib().eosq_encode_host_arena_bytes(int(num_blocks), int(n), int(d), int(bits), int(in_dtype)))


# ---- context and compressed cache ----------------------------------------------------------

class Context:
    """Owner of an ``eosq_ctx`` on the current CUDA device."""

    def __init__(self):
        h = ctypes.c_void_p()
        _check(lib().eosq_create(ctypes.byref(h)), "eosq_create")
        self._h = h

    def close(self):
        if getattr(self, "_h", None):
            lib().eosq_destroy(self._h)
            self._h = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def selftest_wait_timeout(self, polls: int = 64, stream=None):
        """Launches the kernel whose bounded wait runs out; the next check_status reports it."""
        _check(lib().eosq_selftest_wait_timeout(self._h, int(polls), _stream_ptr(stream)), "eosq_selftest_wait_timeout", self)

    @property
    def launch_count(self) -> int:
        return int(lib().eosq_launch_count(self._h))

    def profile_enable(self, on: bool = True):
        _check(lib().eosq_profile_enable(self._h, int(bool(on))), "eosq_profile_enable", self)

    def profile_select(self, stages):
        """Times only the named stages (see STAGES)."""
        mask = 0
        for name in stages:
            mask |= 1 << STAGES.index(name)
        _check(lib().eosq_profile_select(self._h, mask), "eosq_profile_select", self)

    def profile_read(self) -> dict:
        """{stage: (milliseconds, launches)} accumulated since the last read (synchronises)."""
        ms = (ctypes.c_float * len(STAGES))()
        cnt = (ctypes.c_int64 * len(STAGES))()
        _check(lib().eosq_profile_read(self._h, ms, cnt), "eosq_profile_read", self)
        return {STAGES[i]: (float(ms[i]), int(cnt[i])) for i in range(len(STAGES))}


@dataclass
class Cache:
    """Structure-of-arrays compressed cache (``eosq_cache_t``) held in torch tensors."""
    num_blocks: int
    n: int
    d: int
    bits: int
    codes: "object"
    norms: "object"
    rank: "object"
    sigma: "object"
    phi: "object"
    P: "object"
    V: "object"
    status: "object"
    eig: Optional["object"] = None
    lambda_plus: Optional["object"] = None
    vr32: Optional["object"] = None
    coef: Optional["object"] = None

    @staticmethod
    def allocate(num_blocks, n, d, bits, device="cuda", diagnostics=True, pinned=False):
        import torch
        kw = dict(device=device) if not pinned else dict(device="cpu", pin_memory=True)
        B = max(int(num_blocks), 0)
        c = Cache(
            B, n, d, bits,
            codes=torch.empty((B, n, d * bits // 8), dtype=torch.uint8, **kw),
            norms=torch.empty((B, n), dtype=torch.float16, **kw),
            rank=torch.empty((B,), dtype=torch.int32, **kw),
            sigma=torch.empty((B, EOSQ_RMAX), dtype=torch.float32, **kw),
            phi=torch.empty((B, EOSQ_RMAX), dtype=torch.float32, **kw),
            P=torch.empty((B, EOSQ_RMAX, n), dtype=torch.float16, **kw),
            V=torch.empty((B, EOSQ_RMAX, d), dtype=torch.float16, **kw),
            status=torch.empty((B,), dtype=torch.int32, **kw),
        )
        # diagnostics: True = every optional array; "staged" = all but the full spectrum `eig`
        # (asking for `eig` makes eosq_encode resolve all d eigenvalues instead of the 3k + 2 it needs)
        if diagnostics and diagnostics != "staged":
            c.eig = torch.empty((B, d), dtype=torch.float32, **kw)
        if diagnostics:
            c.lambda_plus = torch.empty((B,), dtype=torch.float32, **kw)
            c.vr32 = torch.empty((B, EOSQ_RMAX, d), dtype=torch.float32, **kw)
            c.coef = torch.empty((B, EOSQ_RMAX), dtype=torch.float32, **kw)
        return c

    def struct(self) -> _CacheStruct:
        s = _CacheStruct()
        for name, _ in _CacheStruct._fields_:
            t = getattr(self, name)
            setattr(s, name, t.data_ptr() if t is not None and t.numel() > 0 else None)
        return s

    def stored_bytes(self) -> int:
        """Bytes eosq_scores / eosq_decode read per pass: codes, norms and the kept factor rows."""
        r = int(self.rank.sum().item())
        return int(self.codes.numel() + 2 * self.norms.numel() + 2 * r * (self.n + self.d))


def _stream_ptr(stream):
    import torch
    s = stream if stream is not None else torch.cuda.current_stream()
    return ctypes.c_void_p(s.cuda_stream)


def _dtype_code(t):
    import torch
    if t.dtype == torch.float16:
        return EOSQ_F16
    if t.dtype == torch.float32:
        return EOSQ_F32
    raise TypeError(f"blocks must be float16 or float32, got {t.dtype}")


def eosq_encode(ctx: Context, blocks, bits: int, seed: int, out: Optional[Cache] = None, workspace=None, stream=None) -> Cache:
    """blocks: CUDA tensor [B][n][d] fp16/fp32, contiguous.  Returns (and fills) the cache."""
    import torch
    assert blocks.is_cuda and blocks.is_contiguous() and blocks.dim() == 3
    B, n, d = blocks.shape
    if out is None:
        out = Cache.allocate(B, n, d, bits, device=blocks.device)
    if workspace is None:
        workspace = torch.empty(max(eosq_workspace_bytes(B, n, d), 256), dtype=torch.uint8, device=blocks.device)
    st = out.struct()
    rc = lib().eosq_encode(ctx._h, blocks.data_ptr() if B else None, _dtype_code(blocks), B, n, d, bits,
                           ctypes.c_uint64(seed), ctypes.addressof(st), workspace.data_ptr(), workspace.numel(),
                           _stream_ptr(stream))
    _check(rc, "eosq_encode", ctx)
    return out


def eosq_encode_static_max_blocks() -> int:
    return int(lib().eosq_encode_static_max_blocks())


def eosq_encode_static(ctx: Context, blocks, bits: int, seed: int, out: Cache, stream=None) -> Cache:
    """``eosq_encode`` for callers that may not allocate device memory: no workspace argument, the
    library's fixed device array serves as scratch.  ``out`` must be allocated by the caller
    beforehand; at most ``eosq_encode_static_max_blocks()`` blocks per call.  This wrapper itself
    creates no tensor."""
    assert blocks.is_cuda and blocks.is_contiguous() and blocks.dim() == 3
    B, n, d = blocks.shape
    st = out.struct()
    rc = lib().eosq_encode_static(ctx._h, blocks.data_ptr() if B else None, _dtype_code(blocks), B, n, d, bits,
                                  ctypes.c_uint64(seed), ctypes.addressof(st), _stream_ptr(stream))
    if rc == EOSQ_ERR_BUFFER_TOO_SMALL:
        raise EosqError(rc, "eosq_encode_static", lib().eosq_last_cuda_error(ctx._h).decode())
    _check(rc, "eosq_encode_static", ctx)
    return out


def eosq_decode(ctx: Context, cache: Cache, seed: int, out_dtype=None, out=None, stream=None):
    import torch
    out_dtype = out_dtype or torch.float32
    if out is None:
        out = torch.empty((cache.num_blocks, cache.n, cache.d), dtype=out_dtype, device=cache.codes.device)
    st = cache.struct()
    rc = lib().eosq_decode(ctx._h, ctypes.addressof(st), cache.num_blocks, cache.n, cache.d, cache.bits,
                           ctypes.c_uint64(seed), out.data_ptr() if cache.num_blocks else None, _dtype_code(out),
                           _stream_ptr(stream))
    _check(rc, "eosq_decode", ctx)
    return out


def eosq_scores(ctx: Context, kcache: Cache, q, num_kv_heads: int, blocks_per_head: int, head_stride_blocks: int,
                seed: int, scale: Optional[float] = None, out=None, stream=None):
    """q: CUDA fp16 [num_kv_heads][G][d].  Returns fp32 [num_kv_heads][G][blocks_per_head*n]."""
    import torch
    assert q.is_cuda and q.dtype == torch.float16 and q.is_contiguous()
    G = q.shape[1]
    if scale is None:
        scale = 1.0 / float(np.sqrt(kcache.d))
    if out is None:
        out = torch.empty((num_kv_heads, G, blocks_per_head * kcache.n), dtype=torch.float32, device=q.device)
    st = kcache.struct()
    rc = lib().eosq_scores(ctx._h, ctypes.addressof(st), num_kv_heads, blocks_per_head, head_stride_blocks, kcache.n,
                           kcache.d, kcache.bits, ctypes.c_uint64(seed), q.data_ptr(), G, ctypes.c_float(scale),
                           out.data_ptr(), _stream_ptr(stream))
    _check(rc, "eosq_scores", ctx)
    return out


def eosq_encode_host(ctx: Context, host_blocks, bits: int, seed: int, host_out: Cache, arena, stream=None) -> Cache:
    """host_blocks: CPU tensor [B][n][d] (pinned preferred); host_out: Cache of CPU tensors;
    arena: CUDA uint8 tensor of at least eosq_encode_host_arena_bytes()."""
    assert not host_blocks.is_cuda and host_blocks.is_contiguous()
    B, n, d = host_blocks.shape
    st = host_out.struct()
    rc = lib().eosq_encode_host(ctx._h, host_blocks.data_ptr(), _dtype_code(host_blocks), B, n, d, bits,
                                ctypes.c_uint64(seed), ctypes.addressof(st), arena.data_ptr(), arena.numel(),
                                _stream_ptr(stream))
    _check(rc, "eosq_encode_host", ctx)
    return host_out


def eosq_check_status(ctx: Context, cache: Cache, stream=None) -> int:
    """Number of blocks whose status word is non-zero (synchronises the stream)."""
    flagged = ctypes.c_int64(0)
    rc = lib().eosq_check_status(ctx._h, cache.status.data_ptr() if cache.num_blocks else None, cache.num_blocks,
                                 ctypes.byref(flagged), _stream_ptr(stream))
    if rc not in (EOSQ_OK, EOSQ_WARN_BLOCK_STATUS):
        _check(rc, "eosq_check_status", ctx)
    return int(flagged.value)


# ---- 8-bit paged cache ---------------------------------------------------------------------

# These calls are a serving loop's, one per layer and token, so what surrounds the C call is kept short: sizes that follow from the cache are worked
# out with the handle, tensors are checked by single attributes, and the stream is asked for as a number.

_torch = None   # set by the first Kv8Cache: an import statement in every call would cost as much as one of its checks


class Kv8Cache:
    """``eosq_kv8_t`` over torch tensors: keys and values of the tokens that no compressed block holds, a byte per number, in
    pages that sequences own through a table in device memory.

    k, v [layers][num_pages][kv_heads][page_size][d] uint8; k_scale, v_scale [layers][num_pages][kv_heads] float32; table
    [max_seqs][max_pages], lengths [max_seqs], refs [num_pages] and flags [1] int32.  The attributes are the handle: they are set
    once and cannot be replaced.  A new cache is empty: table -1, lengths, refs and flags 0."""

    __slots__ = ("k", "v", "k_scale", "v_scale", "table", "lengths", "refs", "flags", "format", "layers", "num_pages", "kv_heads",
                 "page_size", "d", "max_seqs", "max_pages", "device", "_struct", "_address", "_index", "_scratch", "_scale")

    def __init__(self, *, k, v, k_scale, v_scale, table, lengths, refs, format, flags=None):
        global _torch
        import torch
        _torch = torch
        if k.dim() != 5 or table.dim() != 2:
            raise ValueError("k is [layers][num_pages][kv_heads][page_size][d], table [max_seqs][max_pages]")
        layers, num_pages, kv_heads, page_size, d = k.shape
        max_seqs, max_pages = table.shape
        if flags is None:
            flags = torch.zeros(1, dtype=torch.int32, device=k.device)
        want = dict(k=(k, torch.uint8, tuple(k.shape)), v=(v, torch.uint8, tuple(k.shape)),
                    k_scale=(k_scale, torch.float32, (layers, num_pages, kv_heads)), v_scale=(v_scale, torch.float32, (layers, num_pages, kv_heads)),
                    table=(table, torch.int32, (max_seqs, max_pages)), lengths=(lengths, torch.int32, (max_seqs,)),
                    refs=(refs, torch.int32, (num_pages,)), flags=(flags, torch.int32, (1,)))
        st = _Kv8Struct()
        for name, (t, dtype, shape) in want.items():
            if t.dtype != dtype or tuple(t.shape) != shape or not t.is_contiguous() or t.device != k.device:
                raise ValueError(f"{name}: {dtype} {list(shape)} contiguous on {k.device} is wanted, not {t.dtype} {list(t.shape)} on {t.device}")
            object.__setattr__(self, name, t)
            setattr(st, name, t.data_ptr())
        for name, value in (("layers", layers), ("num_pages", num_pages), ("kv_heads", kv_heads), ("page_size", page_size), ("d", d),
                            ("format", int(format)), ("max_seqs", max_seqs), ("max_pages", max_pages)):
            object.__setattr__(self, name, value)
            setattr(st, name, value)
        object.__setattr__(self, "device", k.device)
        object.__setattr__(self, "_index", k.get_device())
        object.__setattr__(self, "_scratch", {})
        object.__setattr__(self, "_scale", 1.0 / float(np.sqrt(d)))
        object.__setattr__(self, "_struct", st)
        object.__setattr__(self, "_address", ctypes.addressof(st))

    def __setattr__(self, name, value):
        raise AttributeError(f"{name}: a Kv8Cache is made once; write into its tensors, or make another")

    @staticmethod
    def allocate(layers, num_pages, kv_heads, page_size, d, format, max_seqs, max_pages, device="cuda"):
        import torch
        shape = (layers, num_pages, kv_heads, page_size, d)
        i32 = dict(dtype=torch.int32, device=device)
        return Kv8Cache(k=torch.empty(shape, dtype=torch.uint8, device=device), v=torch.empty(shape, dtype=torch.uint8, device=device),
                        k_scale=torch.ones(shape[:3], dtype=torch.float32, device=device), v_scale=torch.ones(shape[:3], dtype=torch.float32, device=device),
                        table=torch.full((max_seqs, max_pages), -1, **i32), lengths=torch.zeros(max_seqs, **i32), refs=torch.zeros(num_pages, **i32),
                        format=format)


def _kv8_list(cache, t, n, what):
    if t.dtype is not _torch.int32 or t.dim() != 1 or not t.is_contiguous() or t.get_device() != cache._index or (n is not None and t.size(0) != n):
        raise ValueError(f"{what}: int32 [{n if n is not None else 'n'}] contiguous on {cache.device} is wanted, not {t.dtype} {list(t.shape)} on {t.device}")
    return t.data_ptr()


def _kv8_rows(cache, t, heads, what):
    """Data pointer and strides of [total][heads][d], d contiguous; 0 for the stride of a dimension of one, which torch gives any value."""
    stride = t.stride()
    if len(stride) != 3 or stride[2] != 1 or t.size(1) != heads or t.size(2) != cache.d or t.get_device() != cache._index:
        raise ValueError(f"{what}: [total][{heads}][{cache.d}] with contiguous rows on {cache.device} is wanted, not {list(t.shape)} on {t.device}")
    return t.data_ptr(), stride[0] if t.size(0) > 1 else 0, stride[1] if heads > 1 else 0


def _any_dtype_code(t):
    dtype = t.dtype
    return EOSQ_F16 if dtype is _torch.float16 else EOSQ_BF16 if dtype is _torch.bfloat16 else _dtype_code(t)


def _kv8_stream(cache, stream):
    """The stream to launch on.  The memory is the current device's: a kernel of another device must not be given it."""
    if cache._index < 0 or _torch._C._cuda_getDevice() != cache._index:
        raise ValueError(f"the cache is on {cache.device}, which is not the current CUDA device")
    return stream.cuda_stream if stream is not None else _torch._C._cuda_getCurrentRawStream(cache._index)


def _new(like, shape, dtype, stream):
    """Memory on `like`'s device that belongs to the stream it is used on: freed, it goes back to that stream's later work."""
    if stream is None:
        return like.new_empty(shape) if like.dtype is dtype else like.new_empty(shape, dtype=dtype)
    with _torch.cuda.stream(stream):
        return like.new_empty(shape, dtype=dtype)


def _kv8_workspace(cache, rows, workspace, stream):
    """(tensor, address, bytes)"""
    if workspace is None:
        need = cache._scratch.get(rows)
        if need is None:
            if len(cache._scratch) > 64:
                cache._scratch.clear()
            need = cache._scratch[rows] = max(eosq_kv8_workspace_bytes(cache, rows), 256)
        workspace = _new(cache.k, need, _torch.uint8, stream)
        return workspace, workspace.data_ptr(), need
    if workspace.get_device() != cache._index or not workspace.is_contiguous():
        raise ValueError(f"workspace: contiguous memory on {cache.device} is wanted")
    return workspace, workspace.data_ptr(), workspace.numel() * workspace.element_size()


def eosq_kv8_workspace_bytes(cache: Kv8Cache, query_rows: int = 0) -> int:
    return int(lib().eosq_kv8_workspace_bytes(cache._address, int(query_rows)))


def eosq_kv8_reserve(ctx: Context, cache: Kv8Cache, seqs, add, first=None, stream=None):
    """Room for add[i] more tokens of sequence seqs[i].  Returns the position of each one's first new token, -1 where refused."""
    n = seqs.shape[0]
    if first is None:
        first = _new(seqs, n, _torch.int32, stream)
    rc = lib().eosq_kv8_reserve(ctx._h, cache._address, _kv8_list(cache, seqs, None, "seqs"), _kv8_list(cache, add, n, "add"), n,
                                _kv8_list(cache, first, n, "first"), _kv8_stream(cache, stream))
    _check(rc, "eosq_kv8_reserve", ctx)
    return first


def eosq_kv8_store(ctx: Context, cache: Kv8Cache, layer: int, k, v, seqs, first, cu, max_new: int, stream=None) -> None:
    """k, v: [total][kv_heads][d] fp16, bf16 or fp32, any token and head strides that are multiples of 16 bytes."""
    n = seqs.shape[0]
    if k.dtype != v.dtype or k.shape[0] != v.shape[0]:
        raise ValueError("k and v differ in type or number of tokens")
    kp, kt, kh = _kv8_rows(cache, k, cache.kv_heads, "k")
    vp, vt, vh = _kv8_rows(cache, v, cache.kv_heads, "v")
    rc = lib().eosq_kv8_store(ctx._h, cache._address, layer, kp, vp, _any_dtype_code(k), k.shape[0], kt, kh, vt, vh, _kv8_list(cache, seqs, None, "seqs"),
                              _kv8_list(cache, first, n, "first"), _kv8_list(cache, cu, n + 1, "cu"), n, max_new, _kv8_stream(cache, stream))
    _check(rc, "eosq_kv8_store", ctx)


def eosq_kv8_attend(ctx: Context, cache: Kv8Cache, layer: int, q, seqs, cu, max_q: int, scale: Optional[float] = None, causal: bool = True,
                    window: int = 0, out=None, lse=None, want_lse: bool = False, workspace=None, stream=None):
    """q: [total][kv_heads * G][d] fp16 or bf16.  Returns out, or (out, lse) with want_lse (or with an lse to write to)."""
    if q.dim() != 3:
        raise ValueError(f"q: [total][heads][{cache.d}] is wanted, not {list(q.shape)}")
    n = seqs.size(0)
    total, H, _ = q.size()
    G = H // cache.kv_heads
    if H == 0 or G * cache.kv_heads != H:
        raise ValueError(f"q has {H} heads, not a multiple of {cache.kv_heads}")
    qp, qt, qh = _kv8_rows(cache, q, H, "q")
    if out is None:
        out = _torch.empty_like(q) if stream is None and q.is_contiguous() else _new(q, (total, H, cache.d), q.dtype, stream)
        op, ot, oh = out.data_ptr(), H * cache.d, cache.d
    else:
        if out.dtype is not q.dtype or out.size(0) != total:
            raise ValueError(f"out: {q.dtype} [{total}][{H}][{cache.d}] is wanted")
        op, ot, oh = _kv8_rows(cache, out, H, "out")
    if want_lse and lse is None:
        lse = _new(q, (total, H), _torch.float32, stream)
    if lse is not None and (lse.dtype != _torch.float32 or tuple(lse.shape) != (total, H) or not lse.is_contiguous() or lse.device != cache.device):
        raise ValueError(f"lse: float32 [{total}][{H}] contiguous on {cache.device} is wanted")
    workspace, ws, ws_bytes = _kv8_workspace(cache, min(max_q, total) * G, workspace, stream)
    if scale is None:
        scale = cache._scale
    rc = lib().eosq_kv8_attend(ctx._h, cache._address, layer, qp, _any_dtype_code(q), total, qt, qh, _kv8_list(cache, seqs, None, "seqs"),
                               _kv8_list(cache, cu, n + 1, "cu"), n, max_q, G, scale, int(causal), window, op, ot, oh,
                               None if lse is None else lse.data_ptr(), ws, ws_bytes, _kv8_stream(cache, stream))
    _check(rc, "eosq_kv8_attend", ctx)
    return out if lse is None else (out, lse)


def eosq_kv8_fork(ctx: Context, cache: Kv8Cache, src, dst, workspace=None, stream=None) -> None:
    """Sequence dst[i], empty before, becomes a copy of sequence src[i]; they share whole pages."""
    n = src.shape[0]
    workspace, ws, ws_bytes = _kv8_workspace(cache, 0, workspace, stream)
    rc = lib().eosq_kv8_fork(ctx._h, cache._address, _kv8_list(cache, src, None, "src"), _kv8_list(cache, dst, n, "dst"), n, ws, ws_bytes, _kv8_stream(cache, stream))
    _check(rc, "eosq_kv8_fork", ctx)


def eosq_kv8_free(ctx: Context, cache: Kv8Cache, seqs, stream=None) -> None:
    rc = lib().eosq_kv8_free(ctx._h, cache._address, _kv8_list(cache, seqs, None, "seqs"), seqs.shape[0], _kv8_stream(cache, stream))
    _check(rc, "eosq_kv8_free", ctx)


def eosq_kv8_compact(ctx: Context, cache: Kv8Cache, remap=None, workspace=None, stream=None):
    """Moves the used pages to the front of the pool.  Returns where each page went, -1 for one that was free."""
    if remap is None:
        remap = _new(cache.refs, cache.num_pages, _torch.int32, stream)
    workspace, ws, ws_bytes = _kv8_workspace(cache, 0, workspace, stream)
    rc = lib().eosq_kv8_compact(ctx._h, cache._address, _kv8_list(cache, remap, cache.num_pages, "remap"), ws, ws_bytes, _kv8_stream(cache, stream))
    _check(rc, "eosq_kv8_compact", ctx)
    return remap


def eosq_kv8_copy_pages(ctx: Context, from_cache: Kv8Cache, to_cache: Kv8Cache, src_pages, dst_pages, stream=None) -> None:
    """Pages src_pages[i] of one cache to dst_pages[i] of another of the same geometry (or of itself)."""
    n = src_pages.shape[0]
    if from_cache.device != to_cache.device:
        raise ValueError("the caches are on different devices")
    rc = lib().eosq_kv8_copy_pages(ctx._h, from_cache._address, to_cache._address, _kv8_list(from_cache, src_pages, None, "src_pages"),
                                   _kv8_list(from_cache, dst_pages, n, "dst_pages"), n, _kv8_stream(from_cache, stream))
    _check(rc, "eosq_kv8_copy_pages", ctx)


def eosq_kv8_check(ctx: Context, cache: Kv8Cache, stream=None) -> int:
    """The EOSQ_KV8_* flags that calls on this cache have raised, which are then cleared (synchronises the stream)."""
    flags = ctypes.c_uint32(0)
    rc = lib().eosq_kv8_check(ctx._h, cache._address, ctypes.byref(flags), _kv8_stream(cache, stream))
    if rc not in (EOSQ_OK, EOSQ_WARN_BLOCK_STATUS):
        _check(rc, "eosq_kv8_check", ctx)
    return int(flags.value)
