"""What the torch front of the serving operators refuses, without a GPU: the library checks these arguments on the host, before
any device call, so host tensors that say they lie on a GPU do."""
import pytest

torch = pytest.importorskip("torch")


class OnCard:
    """A host tensor that presents itself as one of GPU `index`."""

    is_cuda = True

    def __init__(self, tensor, index=0):
        self.tensor, self.index = tensor, index

    def __getattr__(self, name):
        return getattr(self.tensor, name)

    def get_device(self):
        return self.index


@pytest.fixture()
def front(monkeypatch):
    from paper_2308_07641_b200 import build
    build.build()
    from paper_2308_07641_b200 import binding, serving
    serving._load()
    monkeypatch.setattr(serving, "_raw_stream", lambda index: 0)
    monkeypatch.setattr(serving, "_device", lambda: 0, raising=False)

    def empty(shape, strides, dtype=None, device=None):
        return OnCard(torch.empty_strided(shape, strides, dtype=dtype))

    monkeypatch.setattr(serving, "_empty", empty)
    return binding, serving


def _status(binding, f, *a, **kw):
    with pytest.raises(binding.TSVDError) as e:
        f(*a, **kw)
    return e.value.status


def _cache(serving, heads=2, dim=64):
    """A cache object without a pool: its handle is a host block that the refused calls read no further than their checks."""
    import ctypes
    cache = serving.KV4Cache.__new__(serving.KV4Cache)
    fields = (ctypes.c_int * 64)()
    block = ctypes.create_string_buffer(bytes(fields), 1024)
    # struct tsvd_kv4_s: int device; { uint8_t* pool; int heads, dim, page_tokens, n_pages; ... }
    ints = ctypes.cast(block, ctypes.POINTER(ctypes.c_int))
    ints[4], ints[5], ints[6], ints[7] = heads, dim, 16, 4
    cache._block, cache.handle = block, ctypes.addressof(block)
    cache.n_kv_heads, cache.head_dim, cache.n_pages, cache.page_tokens = heads, dim, 4, 16
    cache.close = lambda: None
    return cache


# Views whose rows overlap: every row the same one (expand), and rows that start two numbers apart (unfold).
ROWS = {"expand": lambda t: t[:1].expand(5, t.shape[1]), "unfold": lambda t: t.flatten().unfold(0, t.shape[1], 2)[:5]}


@pytest.mark.parametrize("view", sorted(ROWS))
def test_rows_that_overlap(front, view):
    binding, serving = front
    overlap = lambda dtype, cols=8: OnCard(ROWS[view](torch.zeros(6, cols, dtype=dtype)))  # noqa: E731
    assert overlap(torch.float32).shape == (5, 8) and overlap(torch.float32).stride(0) < 8
    assert _status(binding, serving.quantize, overlap(torch.float32)) == binding.TSVD_E_SHAPE
    assert _status(binding, serving.quantize, overlap(torch.bfloat16)) == binding.TSVD_E_SHAPE
    assert _status(binding, serving.dequantize, overlap(torch.int8), OnCard(torch.ones(5))) == binding.TSVD_E_SHAPE
    # weights are refused on the host as well
    assert _status(binding, serving.Int8Linear, ROWS[view](torch.zeros(6, 8, dtype=torch.int8)), torch.ones(5)) == binding.TSVD_E_SHAPE


@pytest.mark.parametrize("view", sorted(ROWS))
def test_layer_rows_that_overlap(front, view):
    binding, serving = front
    import ctypes
    layer = serving.Int8Linear.__new__(serving.Int8Linear)
    block = ctypes.create_string_buffer(1024)            # struct tsvd_i8_s: int device, sms, M, N, ...
    ints = ctypes.cast(block, ctypes.POINTER(ctypes.c_int))
    ints[2], ints[3] = 8, 8
    layer.M, layer.N, layer.handle = 8, 8, ctypes.addressof(block)
    layer.close = lambda: None
    overlap = OnCard(ROWS[view](torch.zeros(6, 8)))
    dense = OnCard(torch.zeros(5, 8))
    assert _status(binding, layer, overlap) == binding.TSVD_E_SHAPE
    assert _status(binding, layer, dense, out=overlap) == binding.TSVD_E_SHAPE


@pytest.mark.parametrize("view", sorted(ROWS))
def test_cache_rows_that_overlap(front, view):
    binding, serving = front
    cache = _cache(serving)
    wide = torch.zeros(6, 128, dtype=torch.bfloat16)
    overlap = OnCard(ROWS[view](wide).unflatten(1, (2, 64)))
    dense = OnCard(torch.zeros(5, 2, 64, dtype=torch.bfloat16))
    table, n = OnCard(torch.zeros(5, 2, dtype=torch.int32)), OnCard(torch.ones(5, dtype=torch.int32))
    assert _status(binding, cache.append, overlap, dense, table, n) == binding.TSVD_E_SHAPE
    assert _status(binding, cache.append, dense, overlap, table, n) == binding.TSVD_E_SHAPE
    assert _status(binding, cache.attend, overlap, table, n) == binding.TSVD_E_SHAPE
    assert _status(binding, cache.attend, dense, table, n, out=overlap) == binding.TSVD_E_SHAPE


def test_a_single_row_has_any_stride(front):
    """Its stride says nothing: such a row is not refused for it."""
    _, serving = front
    assert serving._rows(OnCard(torch.zeros(1, 8).expand(1, 8)), "") == (1, 8, 8)
    assert serving._rows(OnCard(torch.zeros(40).as_strided((1, 8), (3, 1))), "") == (1, 8, 8)
    assert serving._rows(OnCard(torch.zeros(4, 10)[:, :8]), "") == (4, 8, 10)
    assert _cache(serving)._heads(OnCard(torch.zeros(200).as_strided((1, 2, 64), (7, 64, 1))), "") == (1, 2, 128)


def test_tensors_of_another_device(front, monkeypatch):
    """The library launches on the current device: tensors of another one, or of two, are refused before any call of it."""
    import types
    binding, serving = front
    monkeypatch.setattr(serving, "_device", lambda: 0)

    def called(*a):
        raise AssertionError("the library was called")

    monkeypatch.setattr(binding, "lib", lambda: types.SimpleNamespace(
        tsvd_strerror=lambda status: b"", **{f: called for f in ("tsvd_quantize", "tsvd_dequantize", "tsvd_i8_forward", "tsvd_kv4_append", "tsvd_kv4_read", "tsvd_kv4_attend")}))
    x, far = OnCard(torch.zeros(3, 8)), OnCard(torch.zeros(3, 8), 1)
    q, qfar = OnCard(torch.zeros(3, 8, dtype=torch.int8)), OnCard(torch.zeros(3, 8, dtype=torch.int8), 1)
    s, sfar = OnCard(torch.ones(3)), OnCard(torch.ones(3), 1)
    E = binding.TSVD_E_CUDA
    assert _status(binding, serving.quantize, far) == E
    assert _status(binding, serving.dequantize, qfar, sfar) == E
    assert _status(binding, serving.dequantize, q, sfar) == E
    layer = serving.Int8Linear.__new__(serving.Int8Linear)
    layer.M, layer.N, layer.handle, layer.close = 8, 8, 1, lambda: None
    assert _status(binding, layer, far) == E
    assert _status(binding, layer, q, sfar) == E
    assert _status(binding, layer, x, out=far) == E
    assert _status(binding, layer, x, out=torch.zeros(3, 8)) == binding.TSVD_E_SHAPE        # on the host
    cache = _cache(serving)
    at = lambda d: (OnCard(torch.zeros(3, 2, 64), d), OnCard(torch.zeros(3, 2, dtype=torch.int32), d),  # noqa: E731
                    OnCard(torch.ones(3, dtype=torch.int32), d), OnCard(torch.arange(4, dtype=torch.int32), d))
    (k, table, n, start), (kf, tf, nf, sf) = at(0), at(1)
    for a in ((kf, kf, tf, nf, sf), (kf, k, table, n), (k, kf, table, n), (k, k, tf, n), (k, k, table, nf), (k, k, table, n, sf)):
        assert _status(binding, cache.append, *a) == E
    for a in ((3, tf, nf), (3, tf, n), (3, table, nf), (3, table, n, sf)):
        assert _status(binding, cache.read, *a) == E
    for a in ((kf, tf, nf, sf), (kf, table, n), (k, tf, n), (k, table, nf), (k, table, n, sf)):
        assert _status(binding, cache.attend, *a) == E
    assert _status(binding, cache.attend, k, table, n, out=kf) == E
