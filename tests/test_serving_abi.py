"""include/tsvd_serving.h without a GPU: constants, and arguments that are refused on the host before any device call."""
import ctypes
import os
import re

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def binding():
    from paper_2308_07641_b200 import build
    build.build()
    from paper_2308_07641_b200 import binding as b
    return b


def test_constants_match_the_header(binding):
    hdr = open(os.path.join(ROOT, "include", "tsvd_serving.h")).read()
    for name in ("TSVD_I8_MAX_N", "TSVD_FLAG_OUT_BF16", "TSVD_FLAG_CAUSAL"):
        value = int(re.search(r"#define\s+" + name + r"\s+(0x[0-9a-fA-F]+|\d+)", hdr).group(1), 0)
        assert value == getattr(binding, name)
    # a sum of that many products of two 8-bit values fits 32 bits, one more would not
    assert 128 * 128 * binding.TSVD_I8_MAX_N < 2 ** 31 <= 128 * 128 * (binding.TSVD_I8_MAX_N + 1)
    text = open(os.path.join(ROOT, "include", "tsvd.h")).read()
    assert int(re.search(r"TSVD_E_INDEX\s*=\s*(\d+)", text).group(1)) == binding.TSVD_E_INDEX
    assert binding.tsvd_strerror(binding.TSVD_E_INDEX) != "unknown status"


def test_flags_do_not_overlap(binding):
    flags = [binding.TSVD_FLAG_OUT_F32, binding.TSVD_FLAG_OUT_BF16, binding.TSVD_FLAG_CAUSAL, binding.TSVD_FLAG_PATH_SIMPLE,
             binding.TSVD_FLAG_TEST_STALL]
    assert sum(flags) == flags[0] | flags[1] | flags[2] | flags[3] | flags[4]


def test_rows(binding):
    L, b = binding.lib(), binding
    p = ctypes.c_void_p(64)       # never dereferenced
    odd = ctypes.c_void_p(65)
    assert L.tsvd_quantize(None, b.TSVD_F32, 1, 4, 4, p, 4, p, None) == b.TSVD_E_NULL
    assert L.tsvd_quantize(p, b.TSVD_F32, 1, 4, 4, None, 4, p, None) == b.TSVD_E_NULL
    assert L.tsvd_quantize(p, b.TSVD_F32, 1, 4, 4, p, 4, None, None) == b.TSVD_E_NULL
    assert L.tsvd_quantize(None, b.TSVD_F32, 0, 4, 4, None, 4, None, None) == b.TSVD_OK      # no rows: nothing to do
    assert L.tsvd_quantize(p, b.TSVD_F32, -1, 4, 4, p, 4, p, None) == b.TSVD_E_SHAPE
    assert L.tsvd_quantize(p, b.TSVD_F32, 1, 0, 4, p, 4, p, None) == b.TSVD_E_SHAPE
    assert L.tsvd_quantize(p, b.TSVD_F32, 1, 4, 3, p, 4, p, None) == b.TSVD_E_SHAPE
    assert L.tsvd_quantize(p, b.TSVD_F32, 1, 4, 4, p, 3, p, None) == b.TSVD_E_SHAPE
    assert L.tsvd_quantize(p, b.TSVD_I8, 1, 4, 4, p, 4, p, None) == b.TSVD_E_DTYPE
    assert L.tsvd_quantize(odd, b.TSVD_BF16, 1, 4, 4, p, 4, p, None) == b.TSVD_E_ALIGN
    assert L.tsvd_dequantize(None, 4, p, 1, 4, p, b.TSVD_F32, 4, None) == b.TSVD_E_NULL
    assert L.tsvd_dequantize(p, 4, p, 1, 4, p, b.TSVD_F32, 3, None) == b.TSVD_E_SHAPE
    assert L.tsvd_dequantize(p, 4, p, 1, 4, p, b.TSVD_I8, 4, None) == b.TSVD_E_DTYPE
    assert L.tsvd_dequantize(p, 4, p, 1, 4, odd, b.TSVD_F32, 4, None) == b.TSVD_E_ALIGN


def test_layer(binding):
    L, b = binding.lib(), binding
    p, h = ctypes.c_void_p(64), ctypes.c_void_p()
    assert L.tsvd_i8_pack(p, 4, p, None, 2, 4, 0, None) == b.TSVD_E_NULL
    assert L.tsvd_i8_pack(None, 4, p, None, 2, 4, 0, ctypes.byref(h)) == b.TSVD_E_NULL
    assert L.tsvd_i8_pack(p, 4, None, None, 2, 4, 0, ctypes.byref(h)) == b.TSVD_E_NULL
    assert L.tsvd_i8_pack(p, 4, p, None, 0, 4, 0, ctypes.byref(h)) == b.TSVD_E_SHAPE
    assert L.tsvd_i8_pack(p, 3, p, None, 2, 4, 0, ctypes.byref(h)) == b.TSVD_E_SHAPE
    assert L.tsvd_i8_pack(p, 4, p, None, 2, 4, 1, ctypes.byref(h)) == b.TSVD_E_DTYPE
    big = b.TSVD_I8_MAX_N + 1
    assert L.tsvd_i8_pack(p, big, p, None, 2, big, 0, ctypes.byref(h)) == b.TSVD_E_TOOBIG
    assert h.value is None
    assert L.tsvd_i8_forward(None, p, 4, None, p, 4, 1, 0, 0, None) == b.TSVD_E_NULL
    assert L.tsvd_i8_reserve(None, 1, 0) == b.TSVD_E_NULL
    assert L.tsvd_i8_info(None, None, None, None) == b.TSVD_E_NULL
    assert L.tsvd_i8_last_status(None) == b.TSVD_E_NULL
    L.tsvd_i8_destroy(None)


def test_cache(binding):
    L, b = binding.lib(), binding
    p, h = ctypes.c_void_p(64), ctypes.c_void_p()
    assert L.tsvd_kv4_create(1, 64, 16, 1, None) == b.TSVD_E_NULL
    for heads, dim, page, n in ((0, 64, 16, 1), (1, 80, 16, 1), (1, 64, 8, 1), (1, 64, 24, 1), (1, 64, 0, 1), (1, 64, 16, 0)):
        assert L.tsvd_kv4_create(heads, dim, page, n, ctypes.byref(h)) == b.TSVD_E_SHAPE
    assert L.tsvd_kv4_create(1, 64, 16, 1 << 28, ctypes.byref(h)) == b.TSVD_E_TOOBIG
    assert h.value is None
    assert L.tsvd_kv4_append(None, p, 64, p, 64, 0, p, 1, p, None, 1, 1, None) == b.TSVD_E_NULL
    assert L.tsvd_kv4_read(None, p, 64, p, 64, 0, p, 1, p, None, 1, 1, None) == b.TSVD_E_NULL
    assert L.tsvd_kv4_attend(None, p, 64, p, 64, 1, 0, p, 1, p, None, 1, 1, 1, 0, 1.0, 0, 0, None) == b.TSVD_E_NULL
    assert L.tsvd_kv4_info(None, None, None, None, None, None) == b.TSVD_E_NULL
    assert L.tsvd_kv4_last_status(None) == b.TSVD_E_NULL
    L.tsvd_kv4_destroy(None)


def test_wrappers_refuse_host_tensors(binding):
    import torch
    from paper_2308_07641_b200 import Int8Linear, dequantize, quantize
    with pytest.raises(binding.TSVDError) as e:
        quantize(torch.zeros(2, 4))
    assert e.value.status == binding.TSVD_E_SHAPE
    with pytest.raises(binding.TSVDError) as e:
        dequantize(torch.zeros(2, 4, dtype=torch.int8), torch.zeros(2))
    assert e.value.status == binding.TSVD_E_SHAPE
    with pytest.raises(binding.TSVDError) as e:
        Int8Linear(torch.zeros(2, 4), torch.zeros(2))
    assert e.value.status == binding.TSVD_E_DTYPE
    with pytest.raises(binding.TSVDError) as e:
        Int8Linear(torch.zeros(2, 4, dtype=torch.int8), torch.zeros(3))
    assert e.value.status == binding.TSVD_E_SHAPE
