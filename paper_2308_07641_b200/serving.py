"""Torch-tensor front of include/tsvd_serving.h: 8-bit rows, the 8-bit linear layer, and the 4-bit key/value cache
with its attention.  Argument checks and marshalling only; the arithmetic runs in the library, on torch's current
stream.
"""
from __future__ import annotations

import math

from . import binding
from .binding import DTYPES, TSVD_BF16, TSVD_F32, TSVD_I8, TSVDError

# torch is loaded with the first call: the package's other parts do without it.  These calls last microseconds, so the front
# looks up as little as it can: the raw stream (a Stream object costs 2 us to make), the library's functions directly.
_CODES: dict = {}          # torch dtype -> the library's number
_empty = _quick = _raw_stream = _device = _i32 = _f32 = _i8 = _bf16 = None


def _load() -> None:
    global _empty, _quick, _raw_stream, _device, _i32, _f32, _i8, _bf16
    import torch
    from torch._C import _cuda_getCurrentRawStream, _cuda_getDevice
    _raw_stream, _device = _cuda_getCurrentRawStream, _cuda_getDevice
    # torch's own short way to memory of the current device (0.8 us in place of 1.6), where this torch has it
    _quick = getattr(getattr(getattr(torch._C, "_dynamo", None), "guards", None), "_empty_strided_cuda", None)
    _empty = _empty_here if _quick else torch.empty_strided
    _i32, _f32, _i8, _bf16 = torch.int32, torch.float32, torch.int8, torch.bfloat16
    _CODES.update({torch.float32: TSVD_F32, torch.bfloat16: TSVD_BF16, torch.int8: TSVD_I8})


def _empty_here(shape, strides, dtype, device):
    """torch.empty_strided on the current device: the one that every call's tensors were checked to lie on."""
    return _quick(shape, strides, dtype)


def _code(dtype, what: str) -> int:
    """The library's number of a torch dtype (float32, bfloat16 or int8)."""
    if not _CODES:
        _load()
    code = _CODES.get(dtype)
    if code is None:
        raise TSVDError(binding.TSVD_E_DTYPE, what)
    return code


def _stream(what: str, x, *others) -> int:
    """torch's current stream, after a check that all tensors (or None) of a call lie on the current device: the library
    launches there, whatever the pointers."""
    index = x.get_device()
    if index != _device():
        raise TSVDError(binding.TSVD_E_CUDA, what)
    for t in others:
        if t is not None and t.get_device() != index:
            raise TSVDError(binding.TSVD_E_CUDA if t.is_cuda else binding.TSVD_E_SHAPE, what)
    return _raw_stream(index)


def _count(n, what: str) -> None:
    """A number of the caller's that the library takes in 32 bits: ctypes would cut a larger one without a word."""
    if not -0x80000000 <= n <= 0x7fffffff:
        raise TSVDError(binding.TSVD_E_SHAPE, what)


def _rows(x, what: str):
    """A CUDA tensor [rows, cols] with contiguous rows; returns (rows, cols, row stride).  The stride of a single row says
    nothing and is taken as cols; any other is handed on as it is, and the library refuses one below cols (rows that overlap,
    as expand and unfold make them)."""
    if not x.is_cuda or x.dim() != 2:
        raise TSVDError(binding.TSVD_E_SHAPE, what)
    rows, cols = x.shape
    ld, one = x.stride()
    if one != 1 and cols > 1:
        raise TSVDError(binding.TSVD_E_SHAPE, what)
    return rows, cols, ld if rows > 1 else cols


def quantize(x):
    """8-bit integers with one scale per row: x float32 or bfloat16 [rows, cols] (row stride >= cols) ->
    (q int8 [rows, cols], its rows 16-byte aligned; scale float32 [rows]); x is about q * scale[:, None]."""
    rows, cols, ldx = _rows(x, "quantize")
    code, device = _code(x.dtype, "quantize"), x.device
    stream = _stream("quantize", x)
    ldq = (cols + 15) & ~15
    q = _empty((rows, cols), (ldq, 1), dtype=_i8, device=device)
    scale = _empty((rows,), (1,), dtype=_f32, device=device)
    err = binding.lib().tsvd_quantize(x.data_ptr(), code, rows, cols, ldx, q.data_ptr(), ldq, scale.data_ptr(), stream)
    if err:
        raise TSVDError(err, "tsvd_quantize")
    return q, scale


def dequantize(q, scale, dtype=None):
    """q * scale[:, None] as float32 (default) or bfloat16."""
    rows, cols, ldq = _rows(q, "dequantize")
    if _code(q.dtype, "dequantize") != TSVD_I8 or scale.dtype != _f32:
        raise TSVDError(binding.TSVD_E_DTYPE, "dequantize")
    if scale.shape != (rows,) or not scale.is_cuda or not scale.is_contiguous():
        raise TSVDError(binding.TSVD_E_SHAPE, "dequantize")
    dtype = dtype or _f32
    code = _code(dtype, "dequantize")
    stream = _stream("dequantize", q, scale)
    y = _empty((rows, cols), (cols, 1), dtype=dtype, device=q.device)
    err = binding.lib().tsvd_dequantize(q.data_ptr(), ldq, scale.data_ptr(), rows, cols, y.data_ptr(), code, cols, stream)
    if err:
        raise TSVDError(err, "tsvd_dequantize")
    return y


def _norm(x, weight, eps: float, residual, bits8: bool, what: str):
    """Both norms: their checks, and the call; returns (y, None, h) or (q, scale, h)."""
    rows, cols, ldx = _rows(x, what)
    code, weight_code = _code(x.dtype, what), _code(weight.dtype, what)
    if weight.shape != (cols,) or not weight.is_contiguous() or not weight.is_cuda:
        raise TSVDError(binding.TSVD_E_SHAPE, what)
    device, dtype = x.device, x.dtype
    if residual is None:
        stream = _stream(what, x, weight)
        h = r_ptr = h_ptr = None
        ldr = 0
    else:
        if residual.dtype != dtype or residual.shape != x.shape:
            raise TSVDError(binding.TSVD_E_DTYPE if residual.dtype != dtype else binding.TSVD_E_SHAPE, what)
        ldr = _rows(residual, what)[2]
        stream = _stream(what, x, weight, residual)
        h = _empty((rows, cols), (cols, 1), dtype=dtype, device=device)
        r_ptr, h_ptr = residual.data_ptr(), h.data_ptr()
    if bits8:
        ldq = (cols + 15) & ~15
        y, scale = _empty((rows, cols), (ldq, 1), dtype=_i8, device=device), _empty((rows,), (1,), dtype=_f32, device=device)
        err = binding.lib().tsvd_rms_norm(x.data_ptr(), code, rows, cols, ldx, r_ptr, ldr, h_ptr, cols, weight.data_ptr(), weight_code, eps,
                                          None, 0, y.data_ptr(), ldq, scale.data_ptr(), stream)
    else:
        y, scale = _empty((rows, cols), (cols, 1), dtype=dtype, device=device), None
        err = binding.lib().tsvd_rms_norm(x.data_ptr(), code, rows, cols, ldx, r_ptr, ldr, h_ptr, cols, weight.data_ptr(), weight_code, eps,
                                          y.data_ptr(), cols, None, 0, None, stream)
    if err:
        raise TSVDError(err, "tsvd_rms_norm")
    return y, scale, h


def rms_norm(x, weight, eps: float = 1e-6, residual=None):
    """Root-mean-square norm of rows: x float32 or bfloat16 [rows, cols] (row stride >= cols), weight float32 or bfloat16 [cols].
    With a residual (like x), h = x + residual is normalised, and the call returns (y, h); else y.  y and h like x."""
    y, _, h = _norm(x, weight, eps, residual, False, "rms_norm")
    return y if h is None else (y, h)


def rms_norm_quantize(x, weight, eps: float = 1e-6, residual=None):
    """The same with the result in 8-bit rows, as quantize makes them: (q int8 [rows, cols], its rows 16-byte aligned, scale
    float32 [rows]), and h behind them where there is a residual.  Int8Linear and LowRankAdapters take q with its scale."""
    q, scale, h = _norm(x, weight, eps, residual, True, "rms_norm_quantize")
    return (q, scale) if h is None else (q, scale, h)


def rotary_table(positions: int, turned: int, base: float = 10000.0, rates=None, amplitude: float = 1.0, device=None):
    """Cosines and sines for KV4Cache.append_rotated: float32 [positions, turned], for each position turned / 2 cosines and then as
    many sines of position * rate, the angles in 64 bits.  rates: float64 [turned / 2]; without them base ** (-2 i / turned)."""
    import torch
    if not _CODES:
        _load()
    _count(positions, "rotary_table")
    if positions < 1 or turned < 2 or turned % 2:
        raise TSVDError(binding.TSVD_E_SHAPE, "rotary_table")
    device = torch.device(device if device is not None else "cuda")
    if rates is None:
        rates = base ** (-torch.arange(0, turned, 2, dtype=torch.float64) / turned)
    if rates.dtype != torch.float64:
        raise TSVDError(binding.TSVD_E_DTYPE, "rotary_table")
    if rates.shape != (turned // 2,):
        raise TSVDError(binding.TSVD_E_SHAPE, "rotary_table")
    rates = rates.to(device).contiguous()
    table = _empty((positions, turned), (turned, 1), dtype=_f32, device=device)
    stream = _stream("rotary_table", table, rates)
    err = binding.lib().tsvd_rotary_table(table.data_ptr(), positions, turned, rates.data_ptr(), amplitude, stream)
    if err:
        raise TSVDError(err, "tsvd_rotary_table")
    return table


class Int8Linear:
    """y = x W^T + bias with W in 8 bits (one scale per output channel) and x in 8 bits (one scale per token)."""

    def __init__(self, w8, w_scale, bias=None):
        """w8: int8 [M, N], w_scale: float32 [M], bias: float32 [M] or None; torch tensors on the host or the device.
        `Int8Linear(*quantize(W), bias)` takes a float matrix W [M, N] on the device."""
        import torch
        if w8.dtype != torch.int8 or w_scale.dtype != torch.float32 or (bias is not None and bias.dtype != torch.float32):
            raise TSVDError(binding.TSVD_E_DTYPE, "Int8Linear")
        if w8.dim() != 2 or (w8.shape[1] > 1 and w8.stride(1) != 1) or w_scale.shape != (w8.shape[0],) or not w_scale.is_contiguous() or (
                bias is not None and (bias.shape != w_scale.shape or not bias.is_contiguous())):
            raise TSVDError(binding.TSVD_E_SHAPE, "Int8Linear")
        self.M, self.N = w8.shape
        for device in {t.device for t in (w8, w_scale, bias) if t is not None and t.is_cuda}:
            torch.cuda.current_stream(device).synchronize()      # the copy runs on another stream
        self.handle = binding.tsvd_i8_pack(w8.data_ptr(), w8.stride(0) if self.M > 1 else self.N, w_scale.data_ptr(),
                                           bias.data_ptr() if bias is not None else 0, self.M, self.N)

    def reserve(self, B_max: int, x_dtype: str) -> None:
        binding.tsvd_i8_reserve(self.handle, B_max, DTYPES[x_dtype])

    def forward(self, x, x_scale=None, out=None, flags: int = 0):
        """x: CUDA tensor [B, N], row stride >= N: float32 or bfloat16 (quantised on the way), or int8 with x_scale
        float32 [B] (None: ones).  Returns [B, M]: bfloat16 for bfloat16 x, else float32, unless flags say otherwise."""
        B, N, ldx = _rows(x, "Int8Linear.forward")
        dt = _code(x.dtype, "Int8Linear.forward")
        if N != self.N:
            raise TSVDError(binding.TSVD_E_SHAPE, "Int8Linear.forward")
        if x_scale is not None:
            if x_scale.shape != (B,) or not x_scale.is_contiguous() or not x_scale.is_cuda:
                raise TSVDError(binding.TSVD_E_SHAPE, "Int8Linear.forward")
            if x_scale.dtype != _f32:
                raise TSVDError(binding.TSVD_E_DTYPE, "Int8Linear.forward")
        stream = _stream("Int8Linear.forward", x, x_scale, out)
        want = _bf16 if (flags & binding.TSVD_FLAG_OUT_BF16 or (dt == TSVD_BF16 and not flags & binding.TSVD_FLAG_OUT_F32)) else _f32
        ldy = self.M
        if out is None:
            out = _empty((B, ldy), (ldy, 1), dtype=want, device=x.device)
        elif out.dtype != want or out.shape != (B, ldy):
            raise TSVDError(binding.TSVD_E_DTYPE if out.dtype != want else binding.TSVD_E_SHAPE, "Int8Linear.forward")
        else:
            ldy = _rows(out, "Int8Linear.forward")[2]
        err = binding.lib().tsvd_i8_forward(self.handle, x.data_ptr(), ldx, x_scale.data_ptr() if x_scale is not None else None,
                                            out.data_ptr(), ldy, B, dt, flags, stream)
        if err:
            raise TSVDError(err, "tsvd_i8_forward")
        return out

    __call__ = forward

    def status(self) -> int:
        return binding.tsvd_i8_last_status(self.handle)

    def close(self):
        if getattr(self, "handle", None):
            binding.tsvd_i8_destroy(self.handle)
            self.handle = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


class LowRankAdapters:
    """Low-rank adapters of many requests beside one projection from N to M numbers (an Int8Linear, a TSVDLinear, any other):
    row i of a batch gets scale * B (A x_i) of its sequence's adapter added.  Weights are kept in bfloat16."""

    def __init__(self, N: int, M: int, max_rank: int, n_slots: int):
        self.handle = binding.tsvd_adapters_create(N, M, max_rank, n_slots)
        self.N, self.M, self.max_rank, self.n_slots = N, M, max_rank, n_slots

    def set(self, slot: int, A, B, scale: float = 1.0) -> None:
        """An adapter into a slot, on torch's current stream: A [rank, N], B [M, rank], CUDA tensors, both float32 or both
        bfloat16."""
        what = "LowRankAdapters.set"
        if A.dtype != B.dtype or _code(A.dtype, what) == TSVD_I8:
            raise TSVDError(binding.TSVD_E_DTYPE, what)
        (rank, N, lda), (M, rank_b, ldb) = _rows(A, what), _rows(B, what)
        if N != self.N or M != self.M or rank != rank_b or not 0 < rank <= self.max_rank:
            raise TSVDError(binding.TSVD_E_SHAPE, what)
        self._slot(slot, what)
        stream = _stream(what, A, B)
        err = binding.lib().tsvd_adapters_set(self.handle, slot, A.data_ptr(), lda, B.data_ptr(), ldb, _code(A.dtype, what), rank, scale, stream)
        if err:
            raise TSVDError(err, "tsvd_adapters_set")

    def _slot(self, slot: int, what: str) -> None:
        if not 0 <= slot < self.n_slots:
            raise TSVDError(binding.TSVD_E_INDEX, what)

    def clear(self, slot: int) -> None:
        """Empty a slot, on torch's current stream."""
        self._slot(slot, "LowRankAdapters.clear")
        if not _CODES:
            _load()
        err = binding.lib().tsvd_adapters_set(self.handle, slot, None, 0, None, 0, TSVD_BF16, 0, 0.0, _raw_stream(_device()))
        if err:
            raise TSVDError(err, "tsvd_adapters_set")

    def reserve(self, rows_max: int) -> None:
        _count(rows_max, "LowRankAdapters.reserve")
        binding.tsvd_adapters_reserve(self.handle, rows_max)

    def forward(self, x, base, slots, q_start=None, x_scale=None, out=None, flags: int = 0):
        """base + scale * B (A x) for every row: x [rows, N] float32, bfloat16, or int8 with x_scale float32 [rows] (None: ones),
        base [rows, M] float32 or bfloat16 (None: zeros, float32 unless x is bfloat16), slots int32 [n_seq] (-1: no adapter),
        q_start int32 [n_seq + 1] (None: one row per sequence); all CUDA tensors, rows with any stride.  out may be base.
        Returns [rows, M] of base's type; rows of no sequence are not written."""
        what = "LowRankAdapters.forward"
        rows, N, ldx = _rows(x, what)
        code = _code(x.dtype, what)
        if N != self.N:
            raise TSVDError(binding.TSVD_E_SHAPE, what)
        if x_scale is not None:
            if x_scale.shape != (rows,) or not x_scale.is_contiguous() or not x_scale.is_cuda:
                raise TSVDError(binding.TSVD_E_SHAPE, what)
            if x_scale.dtype != _f32:
                raise TSVDError(binding.TSVD_E_DTYPE, what)
        if slots.dtype != _i32 or (q_start is not None and q_start.dtype != _i32):
            raise TSVDError(binding.TSVD_E_DTYPE, what)
        if slots.dim() != 1 or not slots.is_cuda or not slots.is_contiguous():
            raise TSVDError(binding.TSVD_E_SHAPE, what)
        n_seq, start = slots.shape[0], None
        if q_start is not None:
            if q_start.shape != (n_seq + 1,) or not q_start.is_cuda or not q_start.is_contiguous():
                raise TSVDError(binding.TSVD_E_SHAPE, what)
            start = q_start.data_ptr()
        stream = _stream(what, x, base, slots, q_start, x_scale, out)
        ldb, dtype = 0, _bf16 if code == TSVD_BF16 else _f32
        if base is not None:
            if base.shape != (rows, self.M):
                raise TSVDError(binding.TSVD_E_SHAPE, what)
            ldb, dtype = _rows(base, what)[2], base.dtype
        ldo = self.M
        if out is None:
            out = _empty((rows, ldo), (ldo, 1), dtype=dtype, device=x.device)
        elif out.dtype != dtype or out.shape != (rows, ldo):
            raise TSVDError(binding.TSVD_E_DTYPE if out.dtype != dtype else binding.TSVD_E_SHAPE, what)
        else:
            ldo = _rows(out, what)[2]
        err = binding.lib().tsvd_adapters_forward_ex(self.handle, x.data_ptr(), ldx, x_scale.data_ptr() if x_scale is not None else None, code,
                                                     base.data_ptr() if base is not None else None, ldb, out.data_ptr(), ldo,
                                                     _code(dtype, what), slots.data_ptr(), start, n_seq, rows, flags, stream)
        if err:
            raise TSVDError(err, "tsvd_adapters_forward")
        return out

    __call__ = forward

    def status(self) -> int:
        return binding.tsvd_adapters_last_status(self.handle)

    def close(self):
        if getattr(self, "handle", None):
            binding.tsvd_adapters_destroy(self.handle)
            self.handle = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


class KV4Cache:
    """Keys and values in 4 bits, in pages; the caller hands out the pages.

    Every call takes page_table int32 [n_seq, max_pages], seq_len int32 [n_seq] (positions in the cache, the call's rows
    included) and q_start int32 [n_seq + 1] (the rows of each sequence; None: one row per sequence), all CUDA tensors that
    are read on the device."""

    def __init__(self, n_kv_heads: int, head_dim: int, n_pages: int, page_tokens: int = 64):
        self.handle = binding.tsvd_kv4_create(n_kv_heads, head_dim, page_tokens, n_pages)
        self.n_kv_heads, self.head_dim, self.n_pages, self.page_tokens = n_kv_heads, head_dim, n_pages, page_tokens

    def _heads(self, x, what: str):
        """A CUDA tensor [rows, heads, head_dim] whose rows lie in one piece; returns (rows, heads, row stride), the stride
        as in _rows."""
        if not x.is_cuda or x.dim() != 3:
            raise TSVDError(binding.TSVD_E_SHAPE, what)
        rows, heads, dim = x.shape
        ld, per_head, one = x.stride()
        if dim != self.head_dim or one != 1 or (heads > 1 and per_head != dim):
            raise TSVDError(binding.TSVD_E_SHAPE, what)
        return rows, heads, ld if rows > 1 else heads * dim

    def _batch(self, page_table, seq_len, q_start, rows: int, what: str):
        if not _CODES:
            _load()
        if page_table.dtype != _i32 or seq_len.dtype != _i32 or (q_start is not None and q_start.dtype != _i32):
            raise TSVDError(binding.TSVD_E_DTYPE, what)
        if page_table.dim() != 2 or seq_len.dim() != 1 or not (page_table.is_cuda and seq_len.is_cuda) or not (
                page_table.is_contiguous() and seq_len.is_contiguous()):
            raise TSVDError(binding.TSVD_E_SHAPE, what)
        n_seq, max_pages = page_table.shape
        if seq_len.shape[0] != n_seq:
            raise TSVDError(binding.TSVD_E_SHAPE, what)
        start = None
        if q_start is not None:
            if q_start.dim() != 1 or q_start.shape[0] != n_seq + 1 or not q_start.is_cuda or not q_start.is_contiguous():
                raise TSVDError(binding.TSVD_E_SHAPE, what)
            start = q_start.data_ptr()
        return page_table.data_ptr(), max_pages, seq_len.data_ptr(), start, n_seq, rows

    def append(self, k, v, page_table, seq_len, q_start=None) -> None:
        """Put k, v [rows, n_kv_heads, head_dim] (float32 or bfloat16) at the last positions of their sequences."""
        if k.dtype != v.dtype or k.shape != v.shape:
            raise TSVDError(binding.TSVD_E_DTYPE if k.dtype != v.dtype else binding.TSVD_E_SHAPE, "KV4Cache.append")
        (rows, heads, ldk), (_, _, ldv) = self._heads(k, "KV4Cache.append"), self._heads(v, "KV4Cache.append")
        if heads != self.n_kv_heads:
            raise TSVDError(binding.TSVD_E_SHAPE, "KV4Cache.append")
        batch = self._batch(page_table, seq_len, q_start, rows, "KV4Cache.append")
        err = binding.lib().tsvd_kv4_append(self.handle, k.data_ptr(), ldk, v.data_ptr(), ldv, _code(k.dtype, "KV4Cache.append"), *batch,
                                            _stream("KV4Cache.append", k, v, page_table, seq_len, q_start))
        if err:
            raise TSVDError(err, "tsvd_kv4_append")

    def append_rotated(self, q, k, v, rotary, page_table, seq_len, q_start=None, interleaved: bool = False):
        """append with the rotation by position: the first rotary.shape[1] numbers of every head of q and k are turned by the
        angles of the row's position (rotary float32 [positions, turned], see rotary_table), in pairs (p, p + turned / 2), or
        (2 p, 2 p + 1) where interleaved.  Keys go into the cache turned; q [rows, n_heads, head_dim], of the same type, is
        returned turned, as a new tensor (None: no queries)."""
        what = "KV4Cache.append_rotated"
        if k.dtype != v.dtype or k.shape != v.shape or (q is not None and q.dtype != k.dtype):
            raise TSVDError(binding.TSVD_E_DTYPE if k.dtype != v.dtype or k.shape == v.shape else binding.TSVD_E_SHAPE, what)
        (rows, heads, ldk), (_, _, ldv) = self._heads(k, what), self._heads(v, what)
        n_heads = ldq = 0
        if q is not None:
            q_rows, n_heads, ldq = self._heads(q, what)
            if q_rows != rows:
                raise TSVDError(binding.TSVD_E_SHAPE, what)
        if heads != self.n_kv_heads or rotary.dim() != 2 or not rotary.is_cuda or not rotary.is_contiguous():
            raise TSVDError(binding.TSVD_E_SHAPE, what)
        batch = self._batch(page_table, seq_len, q_start, rows, what)
        if rotary.dtype != _f32:
            raise TSVDError(binding.TSVD_E_DTYPE, what)
        code, stream = _code(k.dtype, what), _stream(what, k, v, q, rotary, page_table, seq_len, q_start)
        ldo, out = n_heads * self.head_dim, None
        if q is not None:
            out = _empty((rows, n_heads, self.head_dim), (ldo, self.head_dim, 1), dtype=q.dtype, device=q.device)
        positions, turned = rotary.shape
        err = binding.lib().tsvd_kv4_append_rotated(self.handle, q.data_ptr() if n_heads else None, ldq, out.data_ptr() if n_heads else None, ldo,
                                                    n_heads, k.data_ptr(), ldk, v.data_ptr(), ldv, code, rotary.data_ptr(), positions,
                                                    turned, int(interleaved), *batch, stream)
        if err:
            raise TSVDError(err, "tsvd_kv4_append_rotated")
        return out

    def read(self, rows: int, page_table, seq_len, q_start=None, dtype=None):
        """(k, v) [rows, n_kv_heads, head_dim] as the cache holds them: float32 (default) or bfloat16."""
        batch = self._batch(page_table, seq_len, q_start, rows, "KV4Cache.read")
        dtype, device, ld = dtype or _f32, seq_len.device, self.n_kv_heads * self.head_dim
        code = _code(dtype, "KV4Cache.read")
        stream = _stream("KV4Cache.read", seq_len, page_table, q_start)
        shape, strides = (rows, self.n_kv_heads, self.head_dim), (ld, self.head_dim, 1)
        k = _empty(shape, strides, dtype=dtype, device=device)
        v = _empty(shape, strides, dtype=dtype, device=device)
        err = binding.lib().tsvd_kv4_read(self.handle, k.data_ptr(), ld, v.data_ptr(), ld, code, *batch, stream)
        if err:
            raise TSVDError(err, "tsvd_kv4_read")
        return k, v

    def attend(self, q, page_table, seq_len, q_start=None, max_q=None, max_kv=None, causal=True, window=0, scale=None, out=None,
               flags: int = 0, sinks: int = 0):
        """Attention of q [rows, n_heads, head_dim] (bfloat16 or float32) over the cached keys and values; the rows are the
        last positions of their sequences (append their keys first).  max_q, max_kv: bounds on the rows and the positions
        of one sequence, where the caller knows them; with q_start and without max_q a sequence may have all the rows, and
        the call takes the kernel for that (single tokens take far longer in it).  sinks: first positions of a sequence that a
        window does not hide.  Returns a tensor like q."""
        rows, n_heads, ldq = self._heads(q, "KV4Cache.attend")
        batch = self._batch(page_table, seq_len, q_start, rows, "KV4Cache.attend")
        stream = _stream("KV4Cache.attend", q, out, page_table, seq_len, q_start)
        if max_q is None:
            max_q = 1 if q_start is None else max(1, rows)
        if (max_q | (max_kv or 0) | window | sinks) >> 31 not in (0, -1):    # (_count of all four; the library refuses those below 0)
            raise TSVDError(binding.TSVD_E_SHAPE, "KV4Cache.attend")
        if out is None:
            ldo = n_heads * self.head_dim
            out = _empty((rows, n_heads, self.head_dim), (ldo, self.head_dim, 1), dtype=q.dtype, device=q.device)
        elif out.dtype != q.dtype or out.shape != q.shape:
            raise TSVDError(binding.TSVD_E_DTYPE if out.dtype != q.dtype else binding.TSVD_E_SHAPE, "KV4Cache.attend")
        else:
            ldo = self._heads(out, "KV4Cache.attend")[2]
        if scale is None:
            scale = 1.0 / math.sqrt(self.head_dim)
        if causal:
            flags |= binding.TSVD_FLAG_CAUSAL
        err = binding.lib().tsvd_kv4_attend_sinks(self.handle, q.data_ptr(), ldq, out.data_ptr(), ldo, n_heads,
                                                  _code(q.dtype, "KV4Cache.attend"), *batch, max_q, max_kv or 0, scale, window, sinks, flags,
                                                  stream)
        if err:
            raise TSVDError(err, "tsvd_kv4_attend")
        return out

    def status(self) -> int:
        return binding.tsvd_kv4_last_status(self.handle)

    def close(self):
        if getattr(self, "handle", None):
            binding.tsvd_kv4_destroy(self.handle)
            self.handle = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass
