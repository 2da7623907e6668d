"""Torch-tensor front of include/tsvd_serving.h: 8-bit rows, the 8-bit linear layer, and the 4-bit key/value cache
with its attention.  Argument checks and marshalling only; the arithmetic runs in the library, on torch's current
stream.
"""
from __future__ import annotations

import math

from . import binding
from .binding import DTYPES, TSVD_BF16, TSVD_F32, TSVD_I8, TSVDError

_CODES: dict = {}


def _code(dtype, what: str) -> int:
    """The library's number of a torch dtype (float32, bfloat16 or int8)."""
    if not _CODES:
        import torch
        _CODES.update({torch.float32: TSVD_F32, torch.bfloat16: TSVD_BF16, torch.int8: TSVD_I8})
    try:
        return _CODES[dtype]
    except KeyError:
        raise TSVDError(binding.TSVD_E_DTYPE, what) from None


def _stream(x) -> int:
    import torch
    return torch.cuda.current_stream(x.device).cuda_stream


def _rows(x, what: str):
    """A CUDA tensor [rows, cols] with contiguous rows; returns its row stride."""
    if not x.is_cuda or x.dim() != 2 or (x.shape[1] > 1 and x.stride(1) != 1):
        raise TSVDError(binding.TSVD_E_SHAPE, what)
    return max(x.stride(0), x.shape[1])


def quantize(x):
    """8-bit integers with one scale per row: x float32 or bfloat16 [rows, cols] (row stride >= cols) ->
    (q int8 [rows, cols], its rows 16-byte aligned; scale float32 [rows]); x is about q * scale[:, None]."""
    import torch
    ldx = _rows(x, "quantize")
    rows, cols = x.shape
    ldq = (cols + 15) & ~15
    q = torch.empty((rows, ldq), dtype=torch.int8, device=x.device)
    scale = torch.empty(rows, dtype=torch.float32, device=x.device)
    binding.tsvd_quantize(x.data_ptr(), _code(x.dtype, "quantize"), rows, cols, ldx, q.data_ptr(), ldq, scale.data_ptr(), _stream(x))
    return q[:, :cols] if ldq != cols else q, scale


def dequantize(q, scale, dtype=None):
    """q * scale[:, None] as float32 (default) or bfloat16."""
    import torch
    ldq = _rows(q, "dequantize")
    if q.dtype != torch.int8 or scale.dtype != torch.float32:
        raise TSVDError(binding.TSVD_E_DTYPE, "dequantize")
    rows, cols = q.shape
    if scale.shape != (rows,) or not scale.is_cuda or not scale.is_contiguous():
        raise TSVDError(binding.TSVD_E_SHAPE, "dequantize")
    y = torch.empty((rows, cols), dtype=dtype or torch.float32, device=q.device)
    binding.tsvd_dequantize(q.data_ptr(), ldq, scale.data_ptr(), rows, cols, y.data_ptr(), _code(y.dtype, "dequantize"), cols, _stream(q))
    return y


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
        if w8.is_cuda or w_scale.is_cuda or (bias is not None and bias.is_cuda):
            torch.cuda.current_stream().synchronize()      # the copy runs on another stream
        self.handle = binding.tsvd_i8_pack(w8.data_ptr(), max(w8.stride(0), self.N), w_scale.data_ptr(),
                                           bias.data_ptr() if bias is not None else 0, self.M, self.N)

    def reserve(self, B_max: int, x_dtype: str) -> None:
        binding.tsvd_i8_reserve(self.handle, B_max, DTYPES[x_dtype])

    def forward(self, x, x_scale=None, out=None, flags: int = 0):
        """x: CUDA tensor [B, N], row stride >= N: float32 or bfloat16 (quantised on the way), or int8 with x_scale
        float32 [B] (None: ones).  Returns [B, M]: bfloat16 for bfloat16 x, else float32, unless flags say otherwise."""
        import torch
        ldx = _rows(x, "Int8Linear.forward")
        B = x.shape[0]
        dt = _code(x.dtype, "Int8Linear.forward")
        if x.shape[1] != self.N or (x_scale is not None and (x_scale.shape != (B,) or not x_scale.is_contiguous() or not x_scale.is_cuda)):
            raise TSVDError(binding.TSVD_E_SHAPE, "Int8Linear.forward")
        if x_scale is not None and x_scale.dtype != torch.float32:
            raise TSVDError(binding.TSVD_E_DTYPE, "Int8Linear.forward")
        want = torch.bfloat16 if (flags & binding.TSVD_FLAG_OUT_BF16 or (dt == TSVD_BF16 and not flags & binding.TSVD_FLAG_OUT_F32)) \
            else torch.float32
        if out is None:
            out = torch.empty((B, self.M), dtype=want, device=x.device)
        elif out.dtype != want or out.shape != (B, self.M):
            raise TSVDError(binding.TSVD_E_DTYPE if out.dtype != want else binding.TSVD_E_SHAPE, "Int8Linear.forward")
        binding.tsvd_i8_forward(self.handle, x.data_ptr(), ldx, x_scale.data_ptr() if x_scale is not None else 0, out.data_ptr(),
                                _rows(out, "Int8Linear.forward"), B, dt, flags, _stream(x))
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


class KV4Cache:
    """Keys and values in 4 bits, in pages; the caller hands out the pages.

    Every call takes page_table int32 [n_seq, max_pages], seq_len int32 [n_seq] (positions in the cache, the call's rows
    included) and q_start int32 [n_seq + 1] (the rows of each sequence; None: one row per sequence), all CUDA tensors that
    are read on the device."""

    def __init__(self, n_kv_heads: int, head_dim: int, n_pages: int, page_tokens: int = 64):
        self.handle = binding.tsvd_kv4_create(n_kv_heads, head_dim, page_tokens, n_pages)
        self.n_kv_heads, self.head_dim, self.n_pages, self.page_tokens = n_kv_heads, head_dim, n_pages, page_tokens

    def _heads(self, x, heads: int, what: str) -> int:
        """A CUDA tensor [rows, heads, head_dim] whose rows lie in one piece; returns the row stride."""
        if not x.is_cuda or x.dim() != 3 or x.shape[1] != heads or x.shape[2] != self.head_dim or x.stride(2) != 1 or (
                heads > 1 and x.stride(1) != self.head_dim):
            raise TSVDError(binding.TSVD_E_SHAPE, what)
        return max(x.stride(0), heads * self.head_dim)

    def _batch(self, page_table, seq_len, q_start, rows: int, what: str):
        import torch
        for t in (page_table, seq_len) + ((q_start,) if q_start is not None else ()):
            if t.dtype != torch.int32:
                raise TSVDError(binding.TSVD_E_DTYPE, what)
            if not t.is_cuda or not t.is_contiguous():
                raise TSVDError(binding.TSVD_E_SHAPE, what)
        if page_table.dim() != 2 or seq_len.shape != (page_table.shape[0],) or (
                q_start is not None and q_start.shape != (page_table.shape[0] + 1,)):
            raise TSVDError(binding.TSVD_E_SHAPE, what)
        n_seq, max_pages = page_table.shape
        return (page_table.data_ptr(), max_pages, seq_len.data_ptr(), q_start.data_ptr() if q_start is not None else 0, n_seq, rows)

    def append(self, k, v, page_table, seq_len, q_start=None) -> None:
        """Put k, v [rows, n_kv_heads, head_dim] (float32 or bfloat16) at the last positions of their sequences."""
        if k.dtype != v.dtype or k.shape != v.shape:
            raise TSVDError(binding.TSVD_E_DTYPE if k.dtype != v.dtype else binding.TSVD_E_SHAPE, "KV4Cache.append")
        ldk, ldv = self._heads(k, self.n_kv_heads, "KV4Cache.append"), self._heads(v, self.n_kv_heads, "KV4Cache.append")
        batch = self._batch(page_table, seq_len, q_start, k.shape[0], "KV4Cache.append")
        binding.tsvd_kv4_append(self.handle, k.data_ptr(), ldk, v.data_ptr(), ldv, _code(k.dtype, "KV4Cache.append"), *batch, _stream(k))

    def read(self, rows: int, page_table, seq_len, q_start=None, dtype=None):
        """(k, v) [rows, n_kv_heads, head_dim] as the cache holds them: float32 (default) or bfloat16."""
        import torch
        shape = (rows, self.n_kv_heads, self.head_dim)
        k = torch.empty(shape, dtype=dtype or torch.float32, device=seq_len.device)
        v = torch.empty_like(k)
        batch = self._batch(page_table, seq_len, q_start, rows, "KV4Cache.read")
        ld = self.n_kv_heads * self.head_dim
        binding.tsvd_kv4_read(self.handle, k.data_ptr(), ld, v.data_ptr(), ld, _code(k.dtype, "KV4Cache.read"), *batch, _stream(k))
        return k, v

    def attend(self, q, page_table, seq_len, q_start=None, max_q=None, max_kv=None, causal=True, window=0, scale=None, out=None,
               flags: int = 0):
        """Attention of q [rows, n_heads, head_dim] (bfloat16 or float32) over the cached keys and values; the rows are the
        last positions of their sequences (append their keys first).  max_q, max_kv: bounds on the rows and the positions
        of one sequence, where the caller knows them.  Returns a tensor like q."""
        import torch
        n_heads = q.shape[1] if q.dim() == 3 else 0
        ldq = self._heads(q, n_heads, "KV4Cache.attend")
        batch = self._batch(page_table, seq_len, q_start, q.shape[0], "KV4Cache.attend")
        if max_q is None:
            max_q = 1 if q_start is None else max(1, q.shape[0])
        if out is None:
            out = torch.empty(q.shape, dtype=q.dtype, device=q.device)
        elif out.dtype != q.dtype or out.shape != q.shape:
            raise TSVDError(binding.TSVD_E_DTYPE if out.dtype != q.dtype else binding.TSVD_E_SHAPE, "KV4Cache.attend")
        ldo = self._heads(out, n_heads, "KV4Cache.attend")
        if scale is None:
            scale = 1.0 / math.sqrt(self.head_dim)
        if causal:
            flags |= binding.TSVD_FLAG_CAUSAL
        binding.tsvd_kv4_attend(self.handle, q.data_ptr(), ldq, out.data_ptr(), ldo, n_heads, _code(q.dtype, "KV4Cache.attend"), *batch,
                                max_q, max_kv or 0, scale, window, flags, _stream(q))
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
