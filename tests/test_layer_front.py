"""What the norm, the adapters, the rotated append and the attention with first positions refuse, without a GPU: constants, the C
calls (arguments are checked on the host before any device call) and the torch front (host tensors that say they lie on a GPU)."""
import ctypes
import os
import re

import pytest

from tests.test_serving_front import OnCard, ROWS, _cache, _status, front  # noqa: F401
from tests.test_tensor_memory_order import CSRC

torch = pytest.importorskip("torch")
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def binding():
    from paper_2308_07641_b200 import build
    build.build()
    from paper_2308_07641_b200 import binding as b
    return b


def test_constants_match_the_header(binding):
    hdr = open(os.path.join(ROOT, "include", "tsvd_serving.h")).read()
    assert int(re.search(r"#define\s+TSVD_ADAPTERS_MAX_RANK\s+(\d+)", hdr).group(1)) == binding.TSVD_ADAPTERS_MAX_RANK
    assert f"MAX_RANK = {binding.TSVD_ADAPTERS_MAX_RANK};" in open(os.path.join(CSRC, "adapters.cu")).read()


def test_norm_refusals(binding):
    b, p, odd = binding, ctypes.c_void_p(64), ctypes.c_void_p(65)
    ok = dict(x=p, dtype=b.TSVD_F32, rows=1, cols=4, ldx=4, r=None, ldr=0, h=None, ldh=0, w=p, wd=b.TSVD_F32, eps=1e-6, y=p, ldy=4, q=None, ldq=0,
              scale=None)

    def status(**kw):
        return b.lib().tsvd_rms_norm(*{**ok, **kw}.values(), None)

    assert status(rows=0, x=None, y=None, w=None) == b.TSVD_OK                    # nothing to do
    for kw in (dict(x=None), dict(w=None), dict(y=None), dict(q=p, ldq=4, scale=p), dict(y=None, q=p, ldq=4), dict(scale=p),
               dict(r=p, ldr=4, ldh=4), dict(h=p, ldh=4)):
        assert status(**kw) == b.TSVD_E_NULL, kw
    for kw in (dict(rows=-1), dict(rows=1 << 31), dict(cols=0), dict(ldx=3), dict(ldy=3), dict(y=None, q=p, ldq=3, scale=p),
               dict(r=p, h=p, ldr=3, ldh=4), dict(r=p, h=p, ldr=4, ldh=3)):
        assert status(**kw) == b.TSVD_E_SHAPE, kw
    for kw in (dict(dtype=b.TSVD_I8), dict(wd=b.TSVD_I8), dict(dtype=7)):
        assert status(**kw) == b.TSVD_E_DTYPE, kw
    for eps in (0.0, -1.0, 1e-13, float("nan"), float("inf")):
        assert status(eps=eps) == b.TSVD_E_VALUE
    for kw in (dict(x=odd), dict(w=odd), dict(y=odd), dict(y=None, q=odd, ldq=4, scale=odd), dict(r=odd, h=p, ldr=4, ldh=4), dict(r=p, h=odd, ldr=4, ldh=4)):
        assert status(**kw) == b.TSVD_E_ALIGN, kw


def test_adapter_refusals(binding):
    L, b, p, h = binding.lib(), binding, ctypes.c_void_p(64), ctypes.c_void_p()
    assert L.tsvd_adapters_create(4, 4, 1, 1, None) == b.TSVD_E_NULL
    for a in ((0, 4, 1, 1), (4, 0, 1, 1), (4, 4, 0, 1), (4, 4, 1, 0), (-1, 4, 1, 1)):
        assert L.tsvd_adapters_create(*a, ctypes.byref(h)) == b.TSVD_E_SHAPE
    for a in ((4, 4, b.TSVD_ADAPTERS_MAX_RANK + 1, 1), ((1 << 24) + 1, 4, 1, 1), (4, (1 << 21) + 1, 1, 1)):
        assert L.tsvd_adapters_create(*a, ctypes.byref(h)) == b.TSVD_E_TOOBIG
    assert h.value is None
    assert L.tsvd_adapters_set(None, 0, p, 4, p, 4, 0, 1, 1.0, None) == b.TSVD_E_NULL
    assert L.tsvd_adapters_forward(None, p, 4, None, 0, p, 4, p, 4, 0, p, None, 1, 1, None) == b.TSVD_E_NULL
    assert L.tsvd_adapters_reserve(None, 1) == b.TSVD_E_NULL
    assert L.tsvd_adapters_info(None, None, None, None, None, None) == b.TSVD_E_NULL
    assert L.tsvd_adapters_last_status(None) == b.TSVD_E_NULL
    L.tsvd_adapters_destroy(None)


def _adapters(serving, N=8, M=6, max_rank=4, n_slots=2):
    """An object without device memory: its handle is a host block that the refused calls read no further than their checks."""
    a = serving.LowRankAdapters.__new__(serving.LowRankAdapters)
    block = ctypes.create_string_buffer(512)
    # struct tsvd_adapters_s: int device, sms, N, M, max_rank, n_slots; ...
    for i, value in enumerate((N, M, max_rank, n_slots)):
        ctypes.cast(block, ctypes.POINTER(ctypes.c_int))[2 + i] = value
    a._block, a.handle, a.close = block, ctypes.addressof(block), lambda: None
    a.N, a.M, a.max_rank, a.n_slots = N, M, max_rank, n_slots
    return a


def test_adapter_front(front):  # noqa: F811
    binding, serving = front
    a = _adapters(serving)
    card = lambda *s, dtype=torch.float32: OnCard(torch.zeros(*s, dtype=dtype))  # noqa: E731
    A, B = card(3, 8), card(6, 3)
    E = binding
    for bad_A, bad_B in ((card(3, 7), B), (A, card(5, 3)), (A, card(6, 2)), (card(5, 8), card(6, 5)), (card(0, 8), card(6, 0)),
                         (OnCard(torch.zeros(8, 3).t()), B), (OnCard(torch.zeros(1, 8).expand(3, 8)), B), (torch.zeros(3, 8), B)):
        assert _status(binding, a.set, 0, bad_A, bad_B) == E.TSVD_E_SHAPE
    assert _status(binding, a.set, 0, A, card(6, 3, dtype=torch.bfloat16)) == E.TSVD_E_DTYPE
    assert _status(binding, a.set, 0, card(3, 8, dtype=torch.int8), card(6, 3, dtype=torch.int8)) == E.TSVD_E_DTYPE
    assert _status(binding, a.set, 2, A, B) == E.TSVD_E_INDEX and _status(binding, a.set, -1, A, B) == E.TSVD_E_INDEX
    assert _status(binding, a.set, 0, OnCard(torch.zeros(3, 8), 1), B) == E.TSVD_E_CUDA
    assert _status(binding, a.set, 0, A, OnCard(torch.zeros(6, 3), 1)) == E.TSVD_E_CUDA
    x, base, slots = card(5, 8), card(5, 6), card(5, dtype=torch.int32)
    starts = card(6, dtype=torch.int32)
    for bad in (dict(x=card(5, 7)), dict(base=card(5, 5)), dict(base=card(4, 6)), dict(slots=card(4, dtype=torch.int32)), dict(q_start=card(5, dtype=torch.int32)),
                dict(slots=torch.zeros(5, dtype=torch.int32)), dict(out=card(5, 5)), dict(x=card(5, 8, dtype=torch.int8), x_scale=card(4)),
                dict(x=OnCard(torch.zeros(1, 8).expand(5, 8))), dict(base=OnCard(torch.zeros(1, 6).expand(5, 6))),
                dict(out=OnCard(torch.zeros(1, 6).expand(5, 6))), dict(slots=OnCard(torch.zeros(10, dtype=torch.int32)[::2]))):
        args = {**dict(x=x, base=base, slots=slots), **bad}
        assert _status(binding, a, **args) == E.TSVD_E_SHAPE, bad
    for bad in (dict(x=card(5, 8, dtype=torch.float64)), dict(base=card(5, 6, dtype=torch.int8)), dict(slots=card(5, dtype=torch.int64)),
                dict(q_start=card(6, dtype=torch.int64)), dict(out=card(5, 6, dtype=torch.bfloat16)), dict(x_scale=card(5)),
                dict(x=card(5, 8, dtype=torch.int8), x_scale=card(5, dtype=torch.bfloat16))):
        args = {**dict(x=x, base=base, slots=slots), **bad}
        assert _status(binding, a, **args) == E.TSVD_E_DTYPE, bad
    far = lambda t: OnCard(t.tensor, 1)  # noqa: E731
    for bad in (dict(x=far(x)), dict(base=far(base)), dict(slots=far(slots)), dict(q_start=far(starts)), dict(out=far(base))):
        args = {**dict(x=x, base=base, slots=slots), **bad}
        assert _status(binding, a, **args) == E.TSVD_E_CUDA, bad


@pytest.mark.parametrize("name", ["rms_norm", "rms_norm_quantize"])
def test_norm_front(front, name):  # noqa: F811
    binding, serving = front
    norm = getattr(serving, name)
    card = lambda *s, dtype=torch.float32: OnCard(torch.zeros(*s, dtype=dtype))  # noqa: E731
    x, w = card(5, 8), card(8)
    for a in ((x, card(7)), (x, card(1, 8)), (card(8), w), (torch.zeros(5, 8), w), (x, torch.zeros(8)), (x, OnCard(torch.zeros(16)[::2])),
              (x, w, 1e-6, card(5, 7)), (x, w, 1e-6, card(4, 8)), (OnCard(torch.zeros(8, 5).t()), w)):
        assert _status(binding, norm, *a) == binding.TSVD_E_SHAPE
    for view in ROWS.values():
        overlap = OnCard(view(torch.zeros(6, 8)))
        assert _status(binding, norm, overlap, w) == binding.TSVD_E_SHAPE
        assert _status(binding, norm, x, w, residual=overlap) == binding.TSVD_E_SHAPE
    for a in ((card(5, 8, dtype=torch.float16), w), (x, card(8, dtype=torch.float16)), (x, w, 1e-6, card(5, 8, dtype=torch.bfloat16)),
              (card(5, 8, dtype=torch.int8), w)):
        assert _status(binding, norm, *a) == binding.TSVD_E_DTYPE
    assert _status(binding, norm, x, w, 0.0) == binding.TSVD_E_VALUE
    far = OnCard(torch.zeros(5, 8), 1)
    assert _status(binding, norm, far, w) == binding.TSVD_E_CUDA
    assert _status(binding, norm, x, OnCard(torch.zeros(8), 1)) == binding.TSVD_E_CUDA
    assert _status(binding, norm, x, w, residual=far) == binding.TSVD_E_CUDA


def test_rotated_front(front):  # noqa: F811
    binding, serving = front
    cache = _cache(serving)
    card = lambda *s, dtype=torch.float32: OnCard(torch.zeros(*s, dtype=dtype))  # noqa: E731
    ok = dict(q=card(3, 4, 64), k=card(3, 2, 64), v=card(3, 2, 64), rotary=card(9, 64), page_table=card(3, 1, dtype=torch.int32),
              seq_len=card(3, dtype=torch.int32))
    status = lambda **kw: _status(binding, cache.append_rotated, **{**ok, **kw})  # noqa: E731
    bf16 = dict(dtype=torch.bfloat16)
    for kw in (dict(q=card(2, 4, 64)), dict(q=card(3, 4, 32)), dict(k=card(3, 3, 64), v=card(3, 3, 64)), dict(v=card(3, 1, 64)), dict(rotary=card(9)),
               dict(rotary=card(9, 63)), dict(rotary=card(9, 66)), dict(rotary=card(9, 0)), dict(rotary=card(0, 64)), dict(rotary=torch.zeros(9, 64)),
               dict(rotary=OnCard(torch.zeros(9, 65)[:, :64])), dict(q=OnCard(torch.zeros(1, 4, 64).expand(3, 4, 64))),
               dict(seq_len=card(2, dtype=torch.int32))):
        assert status(**kw) == binding.TSVD_E_SHAPE, kw
    for kw in (dict(q=card(3, 4, 64, **bf16)), dict(k=card(3, 2, 64, **bf16)), dict(rotary=card(9, 64, **bf16)), dict(seq_len=card(3, dtype=torch.int64))):
        assert status(**kw) == binding.TSVD_E_DTYPE, kw
    for name in ok:
        assert status(**{name: OnCard(ok[name].tensor, 1)}) == binding.TSVD_E_CUDA
    p = ctypes.c_void_p(64)
    L, b = binding.lib(), binding
    rest = (p, 1, p, None, 1, 1, None)
    assert L.tsvd_kv4_append_rotated(None, p, 64, p, 64, 1, p, 64, p, 64, 0, p, 9, 64, 0, *rest) == b.TSVD_E_NULL
    call = lambda *a: L.tsvd_kv4_append_rotated(cache.handle, *a, *rest)  # noqa: E731
    assert call(p, 256, p, 256, 2, p, 128, p, 128, 0, p, 9, 64, 0) == b.TSVD_E_VALUE                 # onto q itself
    other = ctypes.c_void_p(4096)
    for a in ((None, 256, other, 256, 2), (p, 256, None, 256, 2)):
        assert call(*a, p, 128, p, 128, 0, p, 9, 64, 0) == b.TSVD_E_NULL
    assert call(p, 256, other, 256, 2, p, 128, p, 128, 0, None, 9, 64, 0) == b.TSVD_E_NULL
    for a in ((p, 127, other, 256, 2), (p, 256, other, 127, 2), (p, 256, other, 256, -1)):
        assert call(*a, p, 128, p, 128, 0, p, 9, 64, 0) == b.TSVD_E_SHAPE
    assert call(p, 256, other, 256, 2, p, 128, p, 128, b.TSVD_I8, p, 9, 64, 0) == b.TSVD_E_DTYPE
    assert call(p, 256, other, 256, 2, p, 128, p, 128, 0, ctypes.c_void_p(66), 9, 64, 0) == b.TSVD_E_ALIGN
    assert call(p, 256, ctypes.c_void_p(4097), 256, 2, p, 128, p, 128, 0, p, 9, 64, 0) == b.TSVD_E_ALIGN
    for a in ((None, 9, 64, p), (p, 9, 64, None)):
        assert L.tsvd_rotary_table(*a, 1.0, None) == b.TSVD_E_NULL
    for positions, turned in ((0, 64), (9, 63), (9, 0)):
        assert L.tsvd_rotary_table(p, positions, turned, p, 1.0, None) == b.TSVD_E_SHAPE
    assert L.tsvd_rotary_table(p, 9, 64, ctypes.c_void_p(68), 1.0, None) == b.TSVD_E_ALIGN


def test_sinks_front(front):  # noqa: F811
    binding, serving = front
    cache = _cache(serving)
    q, table, n = OnCard(torch.zeros(3, 2, 64)), OnCard(torch.zeros(3, 1, dtype=torch.int32)), OnCard(torch.ones(3, dtype=torch.int32))
    assert _status(binding, cache.attend, q, table, n, window=5, sinks=-1) == binding.TSVD_E_SHAPE
    assert _status(binding, cache.attend, q, table, n, window=-5, sinks=1) == binding.TSVD_E_SHAPE
    p = ctypes.c_void_p(64)
    assert binding.lib().tsvd_kv4_attend_sinks(None, p, 64, p, 64, 1, 0, p, 1, p, None, 1, 1, 1, 0, 1.0, 5, 1, 0, None) == binding.TSVD_E_NULL


def _body(path, name):
    """The text of a kernel, without comments."""
    text = re.sub(r"//[^\n]*", "", open(os.path.join(CSRC, path)).read())
    start = re.search(name + r"\([^{;]*\)\s*\{", text).end()
    depth, i = 1, start
    while depth:
        depth += {"{": 1, "}": -1}.get(text[i], 0)
        i += 1
    return text[start:i]


def test_dependents_do_not_promise_that_their_inputs_stay():
    """As the other serving kernels: no read-only loads of what a kernel ahead may have written."""
    for path in ("norm.cu", "adapters.cu"):
        text = re.sub(r"//[^\n]*", "", open(os.path.join(CSRC, path)).read())
        assert "__ldg(" not in text and "ld.global.nc" not in text and not re.search(r"const\s+[\w<>]+\s*\*\s*__restrict__", text), path
    body = _body("norm.cu", "rms_norm_kernel")
    assert body.index("pdl_wait()") < body.index("p.load(")


def test_what_is_read_ahead_of_the_wait_is_there():
    """The adapters' second kernel reads slots, weights and base before its wait.  That is sound because the first one lets it start
    only behind its own wait (what came before has ended), and the kernel that writes weights lets nothing start early."""
    down, up, put = (_body("adapters.cu", f"adapter_{n}_kernel") for n in ("down", "up", "set"))
    assert down.index("pdl_wait()") < down.index("pdl_launch_dependents()") < down.index("find_slots<")
    assert "return" not in re.sub(r"auto \w+ = \[&\].*?\n    \};", "", up[:up.index("pdl_wait()")], flags=re.S)      # every block waits
    assert up.index("pdl_wait()") < up.index("p.z +") and up.index("pdl_wait()") < up.index("pdl_launch_dependents()")
    assert "pdl_launch_dependents" not in put and "pdl_wait" not in put


def test_the_same_for_many_rows():
    down, up = _body("adapters.cu", "adapter_down_many_kernel"), _body("adapters.cu", "adapter_many_kernel")
    for body in (down, up):                  # the whole block has its tensor memory, not only the warp that asks for it
        assert body.index("tmem_alloc(") < body.index("__syncthreads()") < body.index("pdl_launch_dependents()")
    assert down.index("tmem_alloc(") < down.index("pdl_wait()") < down.index("find_tile(") and down.index("pdl_wait()") < down.index("pdl_launch_dependents()")
    assert up.index("pdl_wait();\n    if (real)") < up.index("p.z +")
    early = [m.start() for m in re.finditer(r"\breturn;", up)]
    assert len(early) == 1 and "pdl_wait();" in up[early[0] - 200:early[0]]                                            # every block waits
    # every wait of theirs has a limit, and what was under way has ended before a block does
    for body in (down, up):
        assert "mbar_try_wait" not in body and body.count("mbar_wait") >= 3 and "mbar_drain(&drained" in body and "KV4_DEV_TIMEOUT" in body


def test_lanes_that_read_what_others_copied_wait_for_them():
    """The adapters' rings: a lane's wait covers its own copies only, so the warp meets before it reads (and with that before the place
    read last is filled again)."""
    for name, waits in (("adapter_down_kernel", 1), ("adapter_few_kernel", 2)):
        after = re.findall(r"(?:arrived\(\)|copies_wait<STAGES - 2>\(\));\s*(\S+)", _body("adapters.cu", name))
        assert after == ["__syncwarp();"] * waits, name
    many = re.findall(r"copies_wait<L::kStages - 2>\(\);\s*(\S+)", _body("adapters.cu", "adapter_many_kernel"))
    assert many == ["__syncwarp();"]
