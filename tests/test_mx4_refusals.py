"""Calls of the 4-bit operators that are refused on the host, before anything is launched, and the pins of their plain implementation."""
import math

import numpy as np
import pytest

from paper_2506_10848_b200 import binding as sfs
import mx4_reference as R

A = 1 << 20                                                 # an aligned address that no refused call reads


def refused(status, fn, *args, **kw):
    with pytest.raises(sfs.SfsError) as e:
        fn(*args, stream=0, **kw)
    assert e.value.status == status, str(e.value)
    return str(e.value)


def cache(**kw):
    d = dict(k_codes=A, k_scales=A, v_codes=A, v_scales=A, batch=2, capacity=8, n_kv_heads=2, head_dim=64)
    d.update(kw)
    return sfs.Cache4(**d)


@pytest.mark.parametrize("change", [dict(x=None), dict(codes=None), dict(scales=None), dict(rows=0), dict(cols=0), dict(rows=-1), dict(in_dtype=2),
                                    dict(ldx=63), dict(x=A + 1), dict(codes=A + 8), dict(scales=A + 4), dict(ld_codes=40), dict(ld_codes=16)])
def test_quantize_and_dequantize(change):
    kw = dict(x=A, ldx=64, in_dtype=0, rows=4, cols=64, codes=A, ld_codes=32, scales=A)
    kw.update(change)
    refused(sfs.ERR_INVALID_ARG, sfs.sfs_mx4_quantize, **kw)
    kw["out_dtype"] = kw.pop("in_dtype")
    refused(sfs.ERR_INVALID_ARG, sfs.sfs_mx4_dequantize, **kw)


def test_sizes_beyond_the_index_types():
    refused(sfs.ERR_UNSUPPORTED, sfs.sfs_mx4_quantize, A, 64, 0, (1 << 30) + 1, 64, A, 32, A)
    refused(sfs.ERR_UNSUPPORTED, sfs.sfs_linear_mx4, A, 32, A, A, 32, A, A, 64, (1 << 30) + 1, 64, 64)
    refused(sfs.ERR_INVALID_ARG, sfs.sfs_cache4_store, cache(batch=1 << 20, capacity=1 << 12), A, 128, A, 128, 0, None, 1)


@pytest.mark.parametrize("change", [dict(A=None), dict(A_scales=None), dict(Bm=None), dict(B_scales=None), dict(C=None), dict(M=0), dict(N=0), dict(K=0),
                                    dict(out_dtype=2), dict(lda=24), dict(ldb=16), dict(A=A + 8), dict(B_scales=A + 8), dict(ldc=63), dict(C=A + 1)])
def test_linear(change):
    kw = dict(A=A, lda=32, A_scales=A, Bm=A, ldb=32, B_scales=A, C=A, ldc=64, M=4, N=64, K=64)
    kw.update(change)
    refused(sfs.ERR_INVALID_ARG, sfs.sfs_linear_mx4, **kw)


@pytest.mark.parametrize("bad, status", [(dict(k_codes=None), -1), (dict(v_scales=None), -1), (dict(v_codes=A + 8), -1), (dict(batch=0), -1),
                                         (dict(capacity=0), -1), (dict(n_kv_heads=0), -1), (dict(head_dim=96), -2), (dict(n_kv_heads=2048), -2)])
def test_caches(bad, status):
    c = cache(**bad)
    refused(status, sfs.sfs_cache4_store, c, A, 1 << 18, A, 1 << 18, 0, None, 1)
    refused(status, sfs.sfs_cache4_load, c, None, 1, A, 1 << 18, A, 1 << 18, 0)
    refused(status, sfs.sfs_attention_cache4, c, A, 1 << 18, A, 1 << 18, 2, 1)


@pytest.mark.parametrize("change", [dict(k=None), dict(v=None), dict(in_dtype=7), dict(n_rows=-1), dict(ld_k=127), dict(ld_v=64), dict(k=A + 1), dict(slots=A + 2)])
def test_store_and_load(change):
    kw = dict(cache=cache(), k=A, ld_k=128, v=A, ld_v=128, in_dtype=0, slots=A, n_rows=1)
    kw.update(change)
    refused(sfs.ERR_INVALID_ARG, sfs.sfs_cache4_store, **kw)
    if kw["k"] is not None and kw["v"] is not None:         # (the load may leave keys or values out)
        kw["out_dtype"] = kw.pop("in_dtype")
        refused(sfs.ERR_INVALID_ARG, sfs.sfs_cache4_load, **kw)


@pytest.mark.parametrize("change", [dict(q=None), dict(out=None), dict(n_heads=3), dict(n_heads=0), dict(n_q=-1), dict(sinks=-1), dict(ld_q=120), dict(ld_q=132),
                                    dict(ld_out=100), dict(q=A + 8), dict(out=A + 2), dict(lengths=A + 1), dict(positions=A + 2), dict(n_q=1 << 30)])
def test_attention(change):
    kw = dict(cache=cache(), q=A, ld_q=128, out=A, ld_out=128, n_heads=2, n_q=1)
    kw.update(change)
    refused(sfs.ERR_INVALID_ARG, sfs.sfs_attention_cache4, **kw)


def test_sizes_that_would_pass_an_index():
    refused(sfs.ERR_UNSUPPORTED, sfs.sfs_attention_cache4, cache(batch=1, capacity=(1 << 30) + 1), A, 128, A, 128, 2, 1)
    refused(sfs.ERR_UNSUPPORTED, sfs.sfs_attention_cache4, cache(batch=1, n_kv_heads=1), A, 1 << 22, A, 1 << 22, 65535, 1 << 16)


def test_more_rows_than_an_index_of_them_holds():
    refused(sfs.ERR_UNSUPPORTED, sfs.sfs_cache4_store, cache(), A, 128, A, 128, 0, A, (1 << 30) + 1)
    refused(sfs.ERR_UNSUPPORTED, sfs.sfs_cache4_load, cache(), A, (1 << 30) + 1, A, 128, A, 128, 0)


def test_tensors_of_the_host_are_refused():
    torch = pytest.importorskip("torch")
    t, b = torch.zeros(1 << 12, dtype=torch.bfloat16), torch.zeros(1 << 12, dtype=torch.uint8)
    refused(sfs.ERR_INVALID_ARG, sfs.sfs_mx4_quantize, t, 64, 0, 4, 64, A, 32, A)
    refused(sfs.ERR_INVALID_ARG, sfs.sfs_mx4_dequantize, b, 32, A, 4, 64, A, 64, 0)
    refused(sfs.ERR_INVALID_ARG, sfs.sfs_linear_mx4, A, 32, A, A, 32, b, A, 64, 4, 64, 64)
    refused(sfs.ERR_INVALID_ARG, sfs.sfs_cache4_store, cache(), A, 128, t, 128, 0, None, 1)
    refused(sfs.ERR_INVALID_ARG, sfs.sfs_cache4_load, cache(), None, 1, t, 128, A, 128, 0)
    refused(sfs.ERR_INVALID_ARG, sfs.sfs_attention_cache4, cache(), A, 128, A, 128, 2, 1, lengths=b)
    for bad in (b, torch.zeros(8, dtype=torch.uint8), torch.zeros(1 << 12, dtype=torch.int32)):
        with pytest.raises(sfs.SfsError):
            cache(k_codes=bad)


class OnDevice:
    """What the binding asks of a CUDA tensor."""
    is_cuda = True

    def __init__(self, index):
        self.index, self.device = index, f"cuda:{index}"

    def get_device(self): return self.index
    def data_ptr(self): return A
    def element_size(self): return 1
    def is_contiguous(self): return True
    def numel(self): return 1 << 20


def test_cache_of_another_device(monkeypatch):
    """A cache made on one device does not follow the program to another."""
    import torch
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 0)
    parts = dict(zip(("k_codes", "k_scales", "v_codes", "v_scales"), (OnDevice(0),) * 4))
    c, t = cache(**parts), OnDevice(0)
    sfs.sfs_attention_cache4(c, t, 128, t, 128, 2, 0, stream=0)
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 1)
    for here in (OnDevice(1), A):
        refused(sfs.ERR_INVALID_ARG, sfs.sfs_attention_cache4, c, here, 128, here, 128, 2, 0)
        refused(sfs.ERR_INVALID_ARG, sfs.sfs_cache4_store, c, here, 128, here, 128, 0, None, 0)
        refused(sfs.ERR_INVALID_ARG, sfs.sfs_cache4_load, c, None, 0, here, 128, here, 128, 0)
    with pytest.raises(sfs.SfsError):
        cache(**{**parts, "v_scales": OnDevice(1)})


class Indexes(OnDevice):
    """A CUDA tensor of integers, by what the binding asks of it."""
    def __init__(self, size=4, floating=False, contiguous=True, count=16):
        super().__init__(0)
        self.size, self.floating, self.contiguous, self.count = size, floating, contiguous, count

    def element_size(self): return self.size
    def is_floating_point(self): return self.floating
    def is_contiguous(self): return self.contiguous
    def numel(self): return self.count


@pytest.mark.parametrize("bad", [dict(size=8), dict(size=2), dict(floating=True), dict(contiguous=False), dict(count=3)])
def test_indexes_of_another_type_or_too_few(bad, monkeypatch):
    """Slots, lengths and positions are int32: of int64, torch's default, every second would be read as 0."""
    import torch
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 0)
    c, t = cache(batch=4), OnDevice(0)
    refused(sfs.ERR_INVALID_ARG, sfs.sfs_cache4_store, c, t, 128, t, 128, 0, Indexes(**bad), 4)
    refused(sfs.ERR_INVALID_ARG, sfs.sfs_cache4_load, c, Indexes(**bad), 4, t, 128, t, 128, 0)
    refused(sfs.ERR_INVALID_ARG, sfs.sfs_attention_cache4, c, t, 128, t, 128, 2, 1, lengths=Indexes(**bad))
    refused(sfs.ERR_INVALID_ARG, sfs.sfs_attention_cache4, c, t, 128, t, 128, 2, 1, positions=Indexes(**bad))
    # the right ones pass, to calls that have nothing to do
    sfs.sfs_cache4_store(c, t, 128, t, 128, 0, Indexes(), 0, stream=0)
    sfs.sfs_attention_cache4(c, t, 128, t, 128, 2, 0, Indexes(), Indexes(), stream=0)


def test_nothing_to_do_is_no_error():
    sfs.sfs_cache4_store(cache(), A, 128, A, 128, 0, None, 0, stream=0)
    sfs.sfs_cache4_load(cache(), None, 0, A, 128, A, 128, 0, stream=0)
    sfs.sfs_cache4_load(cache(), None, 5, None, 0, None, 0, 0, stream=0)
    sfs.sfs_attention_cache4(cache(), A, 128, A, 128, 2, 0, stream=0)


def test_sizes_of_the_buffers():
    assert sfs.mx4_code_bytes(1) == 16 and sfs.mx4_code_bytes(32) == 16 and sfs.mx4_code_bytes(33) == 32
    for rows, cols in ((1, 1), (128, 128), (129, 128), (5, 700)):
        assert sfs.mx4_scale_bytes(rows, cols) == R.tile_scales(np.zeros((rows, (cols + 31) // 32), np.uint8)).size


def test_plain_rounding():
    """Half-way points go to the even code, everything above 5 to 6, signs are kept."""
    y = np.array([0.25, 0.2500001, 0.75, 1.25, 1.75, 2.5, 2.4999, 3.5, 5.0, 5.0001, 7.9, -0.75, -5.0])
    assert R.nearest_code(y).tolist() == [0, 1, 2, 2, 4, 4, 4, 6, 6, 7, 7, 10, 14]


def test_plain_scales():
    x = np.zeros((6, 64))
    x[0, 3] = 4.0; x[1, 40] = 7.99; x[2, 0] = 2.0 ** -127; x[3, 1] = np.nan; x[4, 32] = -np.inf; x[5, 5] = 2.0 ** 127
    codes, scales = R.quantize(x, R.MATRIX)
    assert scales.tolist() == [[127, 0], [0, 127], [0, 0], [255, 0], [0, 255], [252, 0]]
    assert codes[0, 3] == 6 and codes[1, 40] == 7 and codes[2, 0] == 2 and not codes[3].any() and codes[5, 5] == 6
    assert R.quantize(x, R.CACHE)[1].tolist() == [[127, 65], [65, 127], [65, 65], [255, 65], [65, 255], [192, 65]]
    assert np.isnan(R.values(codes, scales)[3, :32]).all() and (R.values(codes, scales)[3, 32:] == 0).all()
    assert (R.unpack(R.pack(codes)) == codes).all()


def test_plain_attention():
    rng = np.random.default_rng(0)
    q, k, v = rng.normal(size=(3, 8)), rng.normal(size=(5, 8)), rng.normal(size=(5, 8))
    mask = np.array([[1, 1, 1, 1, 1], [0, 0, 0, 0, 0], [0, 1, 0, 0, 0]], dtype=bool)
    out, bound = R.attention(q, k, v, mask)
    w = [math.exp(sum(q[0, d] * k[j, d] for d in range(8)) / math.sqrt(8)) for j in range(5)]
    assert np.allclose(out[0], sum(w[j] * v[j] for j in range(5)) / sum(w), rtol=1e-12)
    assert (out[1] == 0).all() and (out[2] == v[1]).all() and (bound[0] > 0).all()
    assert R.seen(6, 3, 1, 1, 1).tolist() == [True, False, True, True, True, False]
    assert R.seen(4, 9, 2, -1, 0).tolist() == [False] * 4 and R.seen(3, 0, -1, 0, 3).tolist() == [True, False, False]
