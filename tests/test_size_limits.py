"""Counts that the serving kernels could not hold in 32 bits are refused on the host, before any device call."""
import ctypes

import pytest

from tests.test_layer_front import _adapters, binding  # noqa: F401
from tests.test_serving_front import OnCard, _cache, _status, front  # noqa: F401

torch = pytest.importorskip("torch")
MOST = 2 ** 31 - 2 ** 16           # of columns, sequences and rows
P = ctypes.c_void_p(64)            # never dereferenced


@pytest.mark.parametrize("cols", [MOST + 1, 2 ** 31 - 1])
def test_rows_too_wide(binding, cols):  # noqa: F811
    L, b = binding.lib(), binding
    for dtype in (b.TSVD_F32, b.TSVD_BF16):
        assert L.tsvd_quantize(P, dtype, 1, cols, cols, P, cols, P, None) == b.TSVD_E_TOOBIG
        assert L.tsvd_dequantize(P, cols, P, 1, cols, P, dtype, cols, None) == b.TSVD_E_TOOBIG
        for h in (None, P):
            assert L.tsvd_rms_norm(P, dtype, 1, cols, cols, h, cols, h, cols, P, b.TSVD_F32, 1e-6, P, cols, None, 0, None, None) == b.TSVD_E_TOOBIG
            assert L.tsvd_rms_norm(P, dtype, 1, cols, cols, h, cols, h, cols, P, b.TSVD_F32, 1e-6, None, 0, P, cols, P, None) == b.TSVD_E_TOOBIG


def test_more_rows_or_sequences_than_are_counted(front):  # noqa: F811
    b, serving = front
    a, cache, L = _adapters(serving), _cache(serving), b.lib()
    many = 2 ** 30 + 1
    for call in (L.tsvd_adapters_forward, lambda *p: L.tsvd_adapters_forward_ex(*p[:-1], 0, p[-1])):
        assert call(a.handle, P, 8, None, b.TSVD_F32, P, 6, P, 6, b.TSVD_F32, P, P, 1, many, None) == b.TSVD_E_TOOBIG
        assert call(a.handle, P, 8, None, b.TSVD_F32, P, 6, P, 6, b.TSVD_F32, P, P, many, 1, None) == b.TSVD_E_TOOBIG
        assert call(a.handle, P, 8, None, b.TSVD_F32, P, 6, P, 6, b.TSVD_F32, P, None, many, many, None) == b.TSVD_E_TOOBIG
    assert L.tsvd_adapters_reserve(a.handle, many) == b.TSVD_E_TOOBIG
    for n_seq, n_rows in ((MOST + 1, 1), (1, MOST + 1), (2 ** 31 - 1, 2 ** 31 - 1)):
        batch = (P, 1, P, P, n_seq, n_rows)
        assert L.tsvd_kv4_append(cache.handle, P, 128, P, 128, b.TSVD_F32, *batch, None) == b.TSVD_E_TOOBIG
        assert L.tsvd_kv4_read(cache.handle, P, 128, P, 128, b.TSVD_F32, *batch, None) == b.TSVD_E_TOOBIG
        assert L.tsvd_kv4_append_rotated(cache.handle, None, 0, None, 0, 0, P, 128, P, 128, b.TSVD_F32, P, 9, 64, 0, *batch, None) == b.TSVD_E_TOOBIG
        assert L.tsvd_kv4_attend(cache.handle, P, 128, P, 128, 2, b.TSVD_F32, *batch, 1, 0, 1.0, 0, 0, None) == b.TSVD_E_TOOBIG
        assert L.tsvd_kv4_attend_sinks(cache.handle, P, 128, P, 128, 2, b.TSVD_F32, *batch, 1, 0, 1.0, 5, 1, 0, None) == b.TSVD_E_TOOBIG


@pytest.mark.parametrize("beyond", [2 ** 31, 2 ** 32, 2 ** 32 + 1, -2 ** 32 + 1, 2 ** 40])
def test_numbers_that_32_bits_would_cut(front, beyond):  # noqa: F811
    """2^32 first positions are not none of them, and slot 2^32 is not slot 0."""
    b, serving = front
    a, cache = _adapters(serving), _cache(serving)
    card = lambda *s, dtype=torch.float32: OnCard(torch.zeros(*s, dtype=dtype))  # noqa: E731
    assert _status(b, a.set, beyond, card(3, 8), card(6, 3)) == b.TSVD_E_INDEX
    assert _status(b, a.clear, beyond) == b.TSVD_E_INDEX
    assert _status(b, a.reserve, beyond) == b.TSVD_E_SHAPE
    assert _status(b, serving.rotary_table, beyond, 64) == b.TSVD_E_SHAPE
    args = card(3, 2, 64), card(3, 1, dtype=torch.int32), card(3, dtype=torch.int32)
    for name in ("sinks", "window", "max_q", "max_kv"):
        assert _status(b, cache.attend, *args, **{"window": 5, name: beyond}) == b.TSVD_E_SHAPE
