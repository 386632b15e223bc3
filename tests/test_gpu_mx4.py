"""Microscaled 4-bit matrices and caches against the plain 64-bit implementation: codes, scales and values exactly, products within
32-bit sums."""
import numpy as np
import pytest
import torch

import mx4_reference as R
from paper_2506_10848_b200 import binding as sfs

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
TYPES = {"bf16": (torch.bfloat16, sfs.LOGITS_BF16), "f32": (torch.float32, sfs.LOGITS_F32)}
GUARD = 0xA5


def dev(a):
    return torch.from_numpy(np.ascontiguousarray(a)).to(DEV)


def matrix(rows, cols, seed, spread=3.0):
    """Normal values whose blocks differ in size by powers of two."""
    rng = np.random.default_rng(seed)
    x = rng.normal(size=(rows, cols))
    return x * 2.0 ** np.repeat(rng.integers(-spread, spread + 1, size=(rows, (cols + 31) // 32)), 32, 1)[:, :cols]


def as_input(x, dtype):
    t = torch.from_numpy(x).to(TYPES[dtype][0])
    return t, t.double().numpy()


def quantize_on_gpu(t, dtype, ld=None, offset=0, pad=0):
    """-> (codes uint8 [rows, bytes + pad], scales, as written into buffers filled with GUARD bytes)."""
    rows, cols = t.shape
    ld = ld or cols
    buf = torch.zeros(rows * ld + offset, dtype=t.dtype, device=DEV)
    x = buf[offset:].view(rows, ld)
    x[:, :cols] = t.to(DEV)
    codes = torch.full((rows, sfs.mx4_code_bytes(cols) + pad), GUARD, dtype=torch.uint8, device=DEV)
    scales = torch.full((sfs.mx4_scale_bytes(rows, cols) + 64,), GUARD, dtype=torch.uint8, device=DEV)
    sfs.sfs_mx4_quantize(x, ld, TYPES[dtype][1], rows, cols, codes, codes.stride(0), scales)
    torch.cuda.synchronize()
    return codes, scales


SHAPES = [(1, 1), (1, 32), (3, 40), (128, 128), (129, 96), (5, 688), (130, 257), (33, 4096), (257, 1000), (7, 3), (1000, 20), (700, 64), (3000, 33), (261, 256), (300, 200), (9, 519), (6, 1021), (4, 1031), (5, 2047), (3, 3706)]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("rows,cols", SHAPES)
def test_quantize_gives_the_formats_codes_and_scales(rows, cols, dtype):
    t, x = as_input(matrix(rows, cols, rows * 7 + cols), dtype)
    want_codes, want_scales = R.quantize(x, R.MATRIX)
    # aligned rows, and rows at every other address, beside a guard
    for ld, offset, pad in ((cols, 0, 0), (cols + 3, 1, 16), (cols + 1, 3, 0), (cols + 2, 6, 32), (cols, 5, 0)):
        codes, scales = quantize_on_gpu(t, dtype, ld, offset, pad)
        n = sfs.mx4_code_bytes(cols)
        assert (codes[:, :n].cpu().numpy() == R.pack(want_codes)).all()
        assert (codes[:, n:] == GUARD).all() and (scales[-64:] == GUARD).all()
        assert (scales[:-64].cpu().numpy() == R.tile_scales(want_scales)).all()       # the tiles' padding holds zeros


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("quads", [3, 4, 5, 6, 7, 8, 9, 10, 11, 13, 14, 17, 18, 21, 27])
def test_rows_of_every_length_in_aligned_places(quads, dtype):
    """Every length of a warp's segment, its last one full or in part, rows that end inside a vector."""
    for cols in (quads * 128, quads * 128 - 37, quads * 128 - 96, quads * 128 - 127):
        rows, ld, blocks = 70, quads * 128 + 16, (cols + 31) // 32
        t, x = as_input(matrix(rows, cols, cols), dtype)
        codes, scales = quantize_on_gpu(t, dtype, ld, 0, 16)
        want_codes, want_scales = R.quantize(x, R.MATRIX)
        assert (codes[:, :blocks * 16].cpu().numpy() == R.pack(want_codes)).all() and (codes[:, blocks * 16:] == GUARD).all()
        assert (scales[:-64].cpu().numpy() == R.tile_scales(want_scales)).all() and (scales[-64:] == GUARD).all()
        out = torch.full((rows, ld), 77.0, dtype=TYPES[dtype][0], device=DEV)
        sfs.sfs_mx4_dequantize(codes, codes.stride(0), scales, rows, cols, out, ld, TYPES[dtype][1])
        got = out.double().cpu().numpy()
        assert np.array_equal(got[:, :cols], R.values(want_codes, want_scales)[:, :cols], equal_nan=True) and (got[:, cols:] == 77.0).all()


def test_quantize_at_the_edges_of_the_numbers():
    x = np.zeros((12, 96))
    x[0, :8] = [0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, 6.0]         # half-way points under a scale of 1
    x[1, :8] = [-0.25, -0.75, -1.25, -1.75, -2.5, -3.5, -5.0, -7.9]
    x[2, 0], x[2, 40], x[2, 70] = 3.0e38, -3.38e38, 2.0 ** 127
    x[3, 5] = np.nan
    x[4, 33], x[4, 64] = np.inf, -np.inf
    x[5, 0], x[5, 1] = 2.0 ** -126, 2.0 ** -133                     # the smallest normal number and a bf16 subnormal
    x[6, 0] = 2.0 ** -133
    x[7, :2] = [4.0, 2.0 ** -40]
    x[8, 31], x[8, 32] = 1.0, 1.0                                   # last of one block, first of the next
    x[9] = -0.0
    x[10] = 7.99
    x[11, 95] = 1e-30
    for dtype in ("bf16", "f32"):
        t, y = as_input(x, dtype)
        codes, scales = quantize_on_gpu(t, dtype)
        want_codes, want_scales = R.quantize(y, R.MATRIX)
        got = R.unpack(codes.cpu().numpy())
        same = (got == want_codes) | ((got & 7 == 0) & (want_codes & 7 == 0))         # (either zero)
        assert same.all(), np.argwhere(~same)
        assert (scales[:-64].cpu().numpy() == R.tile_scales(want_scales)).all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("rows,cols", SHAPES)
def test_dequantize_gives_the_values(rows, cols, dtype):
    rng = np.random.default_rng(rows + cols)
    blocks = (cols + 31) // 32
    codes = rng.integers(0, 16, size=(rows, blocks * 32)).astype(np.uint8)
    scales = rng.integers(90, 160, size=(rows, blocks)).astype(np.uint8)
    scales[0, 0] = 255
    scales[-1, -1] = 0 if dtype == "f32" else 30
    want = R.values(codes, scales)[:, :cols]
    for ld, offset in ((cols, 0), (cols + 5, 1), (cols, 3), (cols + 1, 2), (cols + 2, 7)):
        buf = torch.full((rows * ld + offset,), 77.0, dtype=TYPES[dtype][0], device=DEV)
        out = buf[offset:].view(rows, ld)
        sfs.sfs_mx4_dequantize(dev(R.pack(codes)), blocks * 16, dev(R.tile_scales(scales)), rows, cols, out, ld, TYPES[dtype][1])
        got = out.double().cpu().numpy()
        assert np.array_equal(got[:, :cols], want, equal_nan=True) and (got[:, cols:] == 77.0).all()


def test_rows_behind_two_to_the_32_values():
    """Rows that lie far apart: the last ones begin behind 2^32 elements of the matrix, and of what it becomes again."""
    rows, ld = 20, 1 << 28
    if torch.cuda.mem_get_info()[0] < 16 * 2 ** 30:
        pytest.skip("needs 16 GB of device memory")
    for cols in (40, 700):
        t, x = as_input(matrix(rows, cols, cols), "bf16")
        buf = torch.zeros((rows - 1) * ld + cols, dtype=torch.bfloat16, device=DEV)
        view = buf.as_strided((rows, cols), (ld, 1))
        view.copy_(t)
        codes = torch.full((rows, sfs.mx4_code_bytes(cols)), GUARD, dtype=torch.uint8, device=DEV)
        scales = torch.full((sfs.mx4_scale_bytes(rows, cols),), GUARD, dtype=torch.uint8, device=DEV)
        sfs.sfs_mx4_quantize(buf, ld, 0, rows, cols, codes, codes.stride(0), scales)
        want_codes, want_scales = R.quantize(x, R.MATRIX)
        assert (codes.cpu().numpy() == R.pack(want_codes)).all() and (scales.cpu().numpy() == R.tile_scales(want_scales)).all()
        view.fill_(77.0)
        sfs.sfs_mx4_dequantize(codes, codes.stride(0), scales, rows, cols, buf, ld, 0)
        assert np.array_equal(view.double().cpu().numpy(), R.values(want_codes, want_scales)[:, :cols], equal_nan=True)


# ---- the product --------------------------------------------------------------------------------------------------------------------

def operand(rows, cols, seed):
    codes, scales = R.quantize(matrix(rows, cols, seed), R.MATRIX)
    return dev(R.pack(codes)), dev(R.tile_scales(scales)), R.values(codes, scales)


def check_linear(M, N, K, out="bf16", scale=1.0, seed=0, ld_pad=0, ldc_pad=0, offset=0):
    a, a_s, av = operand(M, K, seed + 1)
    b, b_s, bv = operand(N, K, seed + 2)
    if ld_pad:
        a, b = (torch.nn.functional.pad(t, (0, ld_pad), value=0x77) for t in (a, b))       # codes behind the rows that nothing may read as values
    dtype, code = TYPES[out]
    buf = torch.full((M * (N + ldc_pad) + offset,), 77.0, dtype=dtype, device=DEV)
    c = buf[offset:].view(M, N + ldc_pad)
    sfs.sfs_linear_mx4(a, a.stride(0), a_s, b, b.stride(0), b_s, c, N + ldc_pad, M, N, K, code, scale)
    sfs.sfs_check_device_status()
    want = scale * (torch.from_numpy(av).to(DEV) @ torch.from_numpy(bv).to(DEV).T).cpu().numpy()           # in 64 bits
    # products are exact; every addition of a 32-bit sum is off by at most 2^-23 of the terms' magnitudes, whichever way it rounds.
    # In any order no term passes through more additions than there are blocks of 64 columns, four levels inside them and the joining
    # of up to 16 parts and the scale.
    steps = (K + 63) // 64 + 4 + 16 + 1
    bound = steps * 2.0 ** -23 * abs(scale) * (torch.from_numpy(np.abs(av)).to(DEV) @ torch.from_numpy(np.abs(bv)).to(DEV).T).cpu().numpy()
    if out == "bf16":
        bound = bound * (1 + 2.0 ** -8) + 2.0 ** -8 * np.abs(want)
    got = c.double().cpu().numpy()
    err = np.abs(got[:, :N] - want)
    assert (err <= bound).all(), (float((err / np.maximum(bound, 1e-300)).max()), np.argwhere(err > bound)[:4])
    assert (got[:, N:] == 77.0).all() and (buf[:offset] == 77.0).all()


@pytest.mark.parametrize("M", [1, 2, 7, 16, 17, 33, 64, 100, 128, 129, 200, 257, 300])
def test_linear_rows(M):
    check_linear(M, 384, 512, seed=M)


@pytest.mark.parametrize("N", [1, 8, 31, 127, 128, 129, 250, 256, 700, 2048])
def test_linear_columns(N):
    for M in (3, 140):
        check_linear(M, N, 256, seed=N + M)


@pytest.mark.parametrize("K", [1, 16, 32, 48, 64, 96, 128, 160, 250, 256, 320, 688, 1024, 1056, 4096])
def test_linear_depths(K):
    for M in (5, 150):
        check_linear(M, 136, K, seed=K + M)


@pytest.mark.parametrize("M,N,K", [(1, 4096, 4096), (8, 4096, 12288), (128, 1024, 4096), (640, 1536, 2048), (16, 12288, 64), (1000, 1000, 1000)])
def test_linear_larger(M, N, K):
    check_linear(M, N, K, seed=5)


# enough tiles for pairs of CTAs: whole and ragged ones in either direction, one or several for each pair, short and long rows
@pytest.mark.parametrize("M,N,K", [(256, 192, 4096), (512, 384, 1024), (2048, 4096, 512), (300, 20000, 96), (5000, 1000, 352), (777, 2500, 1056), (129, 24576, 64), (4100, 8200, 32), (1537, 3001, 688)])
def test_linear_many_rows(M, N, K):
    check_linear(M, N, K, seed=M)
    if M * N < 4e6:
        check_linear(M, N, K, out="f32", scale=-0.75, ldc_pad=4, seed=N)
        check_linear(M, N, K, ld_pad=32, ldc_pad=3, offset=1, seed=K)
        check_linear(M, N, K, ldc_pad=-N % 8, seed=K + 1)           # aligned rows whose last columns are no whole store


def test_linear_many_rows_does_not_let_a_nan_leave_its_row_or_column():
    M, N, K = 1030, 6000, 512
    a, a_s, _ = operand(M, K, 1)
    b, b_s, _ = operand(N, K, 2)
    a_s[int(R.scale_places(M, 16)[1029, 15])] = 255
    b_s[int(R.scale_places(N, 16)[777, 3])] = 255
    out = torch.zeros((M, N), dtype=torch.float32, device=DEV)
    sfs.sfs_linear_mx4(a, 256, a_s, b, 256, b_s, out, N, M, N, K, 1)
    bad = out.isnan()
    assert bad[1029].all() and bad[:, 777].all()
    bad[1029], bad[:, 777] = False, False
    assert not bad.any()
    sfs.sfs_check_device_status()


@pytest.mark.parametrize("M,N", [(4, 100), (150, 257), (300, 512)])
def test_linear_types_strides_and_scale(M, N):
    check_linear(M, N, 352, out="f32", ldc_pad=-N % 4)
    check_linear(M, N, 352, out="bf16", ldc_pad=-N % 8)
    check_linear(M, N, 352, out="f32", scale=0.375, ld_pad=16, ldc_pad=3, offset=1)
    check_linear(M, N, 352, out="bf16", scale=-2.5, ld_pad=48, ldc_pad=5, offset=1)
    check_linear(M, N, 352, out="bf16", ldc_pad=8)


def test_linear_does_not_let_a_nan_leave_its_row():
    a, a_s, av = operand(150, 256, 1)
    b, b_s, bv = operand(70, 256, 2)
    places = R.scale_places(150, 8)
    a_s[int(places[149, 7])] = 255
    out = torch.zeros((150, 70), dtype=torch.float32, device=DEV)
    sfs.sfs_linear_mx4(a, 128, a_s, b, 128, b_s, out, 70, 150, 70, 256, 1)
    assert out[149].isnan().all() and not out[:149].isnan().any()
    sfs.sfs_check_device_status()


def test_quantise_and_multiply_in_a_graph_on_another_stream():
    """Two projections captured in one graph, replayed on new inputs: no state is kept between calls."""
    M, N, K = 40, 512, 1024
    b, b_s, bv = operand(N, K, 9)
    x = torch.zeros((M, K), dtype=torch.bfloat16, device=DEV)
    codes = torch.zeros((M, K // 2), dtype=torch.uint8, device=DEV)
    scales = torch.zeros(sfs.mx4_scale_bytes(M, K), dtype=torch.uint8, device=DEV)
    out = torch.zeros((M, N), dtype=torch.float32, device=DEV)

    def step():
        sfs.sfs_mx4_quantize(x, K, 0, M, K, codes, K // 2, scales)
        sfs.sfs_linear_mx4(codes, K // 2, scales, b, K // 2, b_s, out, N, M, N, K, 1)
    step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for seed in (1, 2):
        t, xv = as_input(matrix(M, K, seed), "bf16")
        x.copy_(t)
        with torch.cuda.stream(torch.cuda.Stream()):
            torch.cuda.current_stream().wait_stream(torch.cuda.default_stream())
            graph.replay()
        torch.cuda.synchronize()
        av = R.values(*R.quantize(xv, R.MATRIX))
        bound = (16 + 4 + 16) * 2.0 ** -23 * (np.abs(av) @ np.abs(bv).T)
        assert (np.abs(out.double().cpu().numpy() - av @ bv.T) <= bound).all()


FIRST_CALL = """
import torch
from paper_2506_10848_b200 import binding as sfs
z = lambda *s: torch.zeros(s, dtype=torch.uint8, device="cuda:0")
a, b, sa, sb = z(40, 64), z(96, 64), z(sfs.mx4_scale_bytes(40, 128)), z(sfs.mx4_scale_bytes(96, 128))
out = torch.full((40, 96), 7.0, device="cuda:0")
call = lambda: sfs.sfs_linear_mx4(a, 64, sa, b, 64, sb, out, 96, 40, 96, 128, 1)
graph, status = torch.cuda.CUDAGraph(), None
with torch.cuda.graph(graph):
    try:
        call()
    except sfs.SfsError as e:
        status = e.status
    out.add_(1.0)                                           # the capture goes on
assert status == sfs.ERR_INVALID_ARG, status
call()
torch.cuda.synchronize()
assert not out.any()
graph.replay()
graph = torch.cuda.CUDAGraph()
with torch.cuda.graph(graph):
    call()
out.fill_(3.0)
graph.replay()
torch.cuda.synchronize()
assert not out.any()
"""


def test_the_first_call_of_a_process_is_not_captured():
    import os
    import subprocess
    import sys
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    r = subprocess.run([sys.executable, "-c", FIRST_CALL], cwd=root, capture_output=True, text=True, timeout=300)
    assert r.returncode == 0, r.stderr[-2000:]


def test_two_products_at_once():
    """Divided over clusters and not, on two streams that overlap."""
    cases = [(9, 512, 8192), (16, 256, 12288), (128, 640, 8192), (300, 4096, 512)]
    ops = [(operand(m, k, m), operand(n, k, n)) for m, n, k in cases]
    outs = [[torch.zeros((m, n), dtype=torch.float32, device=DEV) for m, n, k in cases] for _ in range(2)]
    torch.cuda.synchronize()
    for out in outs:
        with torch.cuda.stream(torch.cuda.Stream()):
            for _ in range(20):
                for (m, n, k), ((a, a_s, _), (b, b_s, _)), o in zip(cases, ops, out):
                    sfs.sfs_linear_mx4(a, k // 2, a_s, b, k // 2, b_s, o, n, m, n, k, 1)
    torch.cuda.synchronize()
    sfs.sfs_check_device_status()
    for (m, n, k), ((_, _, av), (_, _, bv)), x, y in zip(cases, ops, *outs):
        assert torch.equal(x, y)
        bound = ((k + 63) // 64 + 21) * 2.0 ** -23 * (np.abs(av) @ np.abs(bv).T)
        assert (np.abs(x.double().cpu().numpy() - av @ bv.T) <= bound).all()


def test_two_host_threads_with_products_of_different_depth():
    """Short and long rings of one kernel's instance, launched by two threads at once: neither takes shared memory from the other."""
    import threading
    cases = [(16, 128, 64), (16, 128, 24576), (300, 512, 512), (300, 512, 8192)]
    for short, deep in (cases[:2], cases[2:]):
        work = []
        for m, n, k in (short, deep):
            a, a_s, av = operand(m, k, m)
            b, b_s, bv = operand(n, k, n)
            work.append((m, n, k, a, a_s, b, b_s, torch.zeros((m, n), dtype=torch.float32, device=DEV), torch.cuda.Stream(), av @ bv.T, np.abs(av) @ np.abs(bv).T))
        torch.cuda.synchronize()
        failed, start = [], threading.Barrier(2)

        def calls(m, n, k, a, a_s, b, b_s, out, stream, *_):
            torch.cuda.set_device(0)
            start.wait()
            try:
                for _ in range(4000):
                    sfs.sfs_linear_mx4(a, k // 2, a_s, b, k // 2, b_s, out, n, m, n, k, 1, stream=stream.cuda_stream)
            except sfs.SfsError as e:
                failed.append(str(e))
        threads = [threading.Thread(target=calls, args=w) for w in work]
        for t in threads:
            t.start()
        for t in threads:
            t.join()
        torch.cuda.synchronize()
        sfs.sfs_check_device_status()
        assert not failed, failed
        for m, n, k, *_, out, _, want, size in work:
            assert (np.abs(out.double().cpu().numpy() - want) <= ((k + 63) // 64 + 21) * 2.0 ** -23 * size).all()


# ---- the cache ------------------------------------------------------------------------------------------------------------------------

def new_cache(batch, capacity, heads, dim):
    slots = batch * capacity
    full = lambda *s: torch.full(s, GUARD, dtype=torch.uint8, device=DEV)  # noqa: E731
    return sfs.Cache4(full(slots, heads, dim // 2), full(slots, heads, dim // 32), full(slots, heads, dim // 2), full(slots, heads, dim // 32),
                      batch, capacity, heads, dim)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("heads,dim", [(1, 64), (3, 64), (4, 128), (5, 128)])
def test_store_and_load(heads, dim, dtype):
    batch, capacity, n = 2, 37, 21
    width = heads * dim
    c = new_cache(batch, capacity, heads, dim)
    rng = np.random.default_rng(heads + dim)
    slots = rng.permutation(batch * capacity)[:n].astype(np.int32)
    slots[3], slots[4], slots[5] = -1, batch * capacity, -2 ** 31   # rows that are left out
    t, kv = as_input(matrix(n, 2 * width + 3, 3), dtype)
    t = t.to(DEV)
    k, v = t[:, :width], t[:, width + 3:]                           # rows of keys and values side by side, at odd addresses
    sfs.sfs_cache4_store(c, k, t.stride(0), v, t.stride(0), TYPES[dtype][1], dev(slots), n)
    torch.cuda.synchronize()
    kept = (slots >= 0) & (slots < batch * capacity)
    for x, codes, scales in ((kv[:, :width], c._tensors[0], c._tensors[1]), (kv[:, width + 3:], c._tensors[2], c._tensors[3])):
        want_codes, want_scales = R.quantize(x, R.CACHE)
        all_codes = np.full((batch * capacity, width // 2), GUARD, np.uint8)
        all_scales = np.full((batch * capacity, width // 32), GUARD, np.uint8)
        all_codes[slots[kept]], all_scales[slots[kept]] = R.pack(want_codes)[kept], want_scales[kept]
        assert (codes.cpu().numpy().reshape(all_codes.shape) == all_codes).all() and (scales.cpu().numpy().reshape(all_scales.shape) == all_scales).all()
    out = torch.full((n, 2, width + 1), 77.0, dtype=TYPES[dtype][0], device=DEV)
    sfs.sfs_cache4_load(c, dev(slots), n, out, out.stride(0), out[:, 1], out.stride(0), TYPES[dtype][1])
    got = out.double().cpu().numpy()
    for i, x in enumerate((kv[:, :width], kv[:, width + 3:])):
        want = R.values(*R.quantize(x, R.CACHE))
        assert (got[kept, i, :width] == want[kept]).all() and (got[~kept, i] == 77.0).all() and (got[:, i, width:] == 77.0).all()
    only = torch.full((n, width), 77.0, dtype=TYPES[dtype][0], device=DEV)
    sfs.sfs_cache4_load(c, dev(slots), n, None, 0, only, width, TYPES[dtype][1])    # values alone
    assert torch.equal(only.cpu(), out[:, 1, :width].cpu())


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("heads,dim", [(3, 128), (6, 128), (9, 128), (11, 64), (13, 64), (13, 128), (21, 128)])
def test_store_and_load_of_many_heads(heads, dim, dtype):
    n, width = 300, heads * dim
    c = new_cache(1, n, heads, dim)
    t, x = as_input(matrix(n, width, heads), dtype)
    t = t.to(DEV)
    sfs.sfs_cache4_store(c, t, width, t.flip(0).contiguous(), width, TYPES[dtype][1], None, n)
    out = torch.full((2, n, width), 77.0, dtype=TYPES[dtype][0], device=DEV)
    sfs.sfs_cache4_load(c, None, n, out[0], width, out[1], width, TYPES[dtype][1])
    want = R.values(*R.quantize(x, R.CACHE))
    assert np.array_equal(out[0].double().cpu().numpy(), want, equal_nan=True) and np.array_equal(out[1].double().cpu().numpy(), want[::-1], equal_nan=True)


def test_of_rows_with_one_slot_the_last_counts():
    heads, dim, n, slots_n = 2, 64, 1000, 7
    c = new_cache(1, slots_n, heads, dim)
    slots = (np.arange(n) * 31 % slots_n).astype(np.int32)
    t, x = as_input(matrix(n, heads * dim, 1), "bf16")
    t = t.to(DEV)
    for _ in range(3):
        sfs.sfs_cache4_store(c, t, heads * dim, t, heads * dim, 0, dev(slots), n)
    out = torch.zeros((slots_n, heads * dim), dtype=torch.bfloat16, device=DEV)
    sfs.sfs_cache4_load(c, None, slots_n, out, heads * dim, None, 0, 0)
    last = [max(r for r in range(n) if slots[r] == s) for s in range(slots_n)]
    assert (out.double().cpu().numpy() == R.values(*R.quantize(x[last], R.CACHE))).all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("n,slots_n,kind", [(8192, 5000, "any"), (8193, 7, "few"), (20001, 30000, "any"), (20001, 40000, "once"), (30000, 1, "few"), (50000, 3000, "far"), (9000, 9000, "reversed"),
                                            (310000, 400000, "any"), (12345, 100000, "crowded")])
def test_the_last_of_many_rows_counts(n, slots_n, kind, dtype):
    """More rows than the scan of small calls takes, beside guards: random slots with repetitions, few slots, none twice, repetitions far apart,
    slots that share the head of a table, and slots outside of the cache."""
    heads, dim = (1, 64) if dtype == "bf16" else (3, 64)
    if n > 100000 and dtype == "f32":
        heads = 1
    width = heads * dim
    rng = np.random.default_rng(n + slots_n)
    if kind == "once":
        slots = rng.permutation(slots_n)[:n]
    elif kind == "reversed":
        slots = np.arange(n)[::-1]
    elif kind == "far":
        slots = np.arange(n) * 17 % slots_n
    elif kind == "crowded":                                 # multiples of 2^10, whose products with an odd number agree in the lower bits
        slots = rng.integers(0, slots_n // 1024, size=n) * 1024
    else:
        slots = rng.integers(0, slots_n, size=n)
    slots = slots.astype(np.int32)
    out = rng.random(n) < 0.03
    slots[out] = rng.choice([-1, slots_n, 2 ** 31 - 1, -2 ** 31, -7], size=int(out.sum()))
    c = new_cache(1, slots_n, heads, dim)
    t, x = as_input(np.random.default_rng(5).normal(size=(n, 2 * width)).astype(np.float32).astype(np.float64), dtype)
    t = t.to(DEV)
    sfs.sfs_cache4_store(c, t, 2 * width, t[:, width:], 2 * width, TYPES[dtype][1], dev(slots), n)
    kept = np.flatnonzero((slots >= 0) & (slots < slots_n))
    last = np.full(slots_n, -1)
    last[slots[kept]] = kept                                # (numpy assigns in order: the last one stays)
    assert all(last[s] == r for r, s in zip(kept[-50:], slots[kept[-50:]]) if (slots[r + 1:] != s).all())
    named = np.flatnonzero(last >= 0)
    for part, codes, scales in ((0, c._tensors[0], c._tensors[1]), (1, c._tensors[2], c._tensors[3])):
        want_codes, want_scales = R.quantize(x[last[named], part * width:(part + 1) * width], R.CACHE)
        codes, scales = codes.cpu().numpy().reshape(slots_n, -1), scales.cpu().numpy().reshape(slots_n, -1)
        assert (codes[named] == R.pack(want_codes)).all() and (scales[named] == want_scales).all()
        rest = np.setdiff1d(np.arange(slots_n), named)
        assert (codes[rest] == GUARD).all() and (scales[rest] == GUARD).all()


def test_many_rows_at_odd_places_and_of_many_heads():
    heads, dim, n, slots_n = 13, 128, 8500, 9001
    width = heads * dim
    rng = np.random.default_rng(3)
    slots = rng.integers(-3, slots_n, size=n).astype(np.int32)
    c = new_cache(1, slots_n, heads, dim)
    x = torch.randn((n, 2 * width + 3), generator=torch.Generator().manual_seed(2)).to(torch.bfloat16)
    t = x.to(DEV)
    sfs.sfs_cache4_store(c, t, t.stride(0), t[:, width + 3:], t.stride(0), 0, dev(slots), n)
    kept = np.flatnonzero(slots >= 0)
    last = np.full(slots_n, -1)
    last[slots[kept]] = kept
    named = np.flatnonzero(last >= 0)
    at, row = torch.from_numpy(named).to(torch.int32).to(DEV), torch.from_numpy(last[named]).to(DEV)
    out = torch.zeros((2, named.size, width), dtype=torch.bfloat16, device=DEV)
    sfs.sfs_cache4_load(c, at, named.size, out[0], width, out[1], width, 0)
    # the same rows stored by a small call each: no slot twice, no table
    ref, want = new_cache(1, 4096, heads, dim), torch.zeros((2, named.size, width), dtype=torch.bfloat16, device=DEV)
    for i in range(0, named.size, 4096):
        part = t[row[i:i + 4096]].contiguous()
        sfs.sfs_cache4_store(ref, part, part.stride(0), part[:, width + 3:], part.stride(0), 0, None, part.shape[0])
        sfs.sfs_cache4_load(ref, None, part.shape[0], want[0, i:], width, want[1, i:], width, 0)
    assert torch.equal(out, want)


def test_many_rows_in_a_captured_graph_on_another_stream():
    """Slots and rows are read when the graph runs; two replays at once on caches of their own."""
    heads, dim, n, slots_n = 2, 64, 7000, 3000
    width = heads * dim
    caches = [new_cache(1, slots_n, heads, dim) for _ in range(2)]
    t, slots = torch.zeros((n, 2 * width), dtype=torch.bfloat16, device=DEV), torch.full((n,), -1, dtype=torch.int32, device=DEV)
    graphs = []
    for c in caches:
        graphs.append(torch.cuda.CUDAGraph())
        with torch.cuda.graph(graphs[-1]):
            sfs.sfs_cache4_store(c, t, 2 * width, t[:, width:], 2 * width, 0, slots, n)
    rng = np.random.default_rng(1)
    for _ in range(2):
        x = torch.randn((n, 2 * width), generator=torch.Generator().manual_seed(int(rng.integers(100)))).to(torch.bfloat16)
        at = rng.integers(-10, slots_n, size=n).astype(np.int32)
        t.copy_(x)
        slots.copy_(torch.from_numpy(at))
        torch.cuda.synchronize()
        for g in graphs:
            with torch.cuda.stream(torch.cuda.Stream()):
                g.replay()
        torch.cuda.synchronize()
        kept = np.flatnonzero(at >= 0)
        last = np.full(slots_n, -1)
        last[at[kept]] = kept
        named = np.flatnonzero(last >= 0)
        want = R.pack(R.quantize(x.double().numpy()[last[named], width:], R.CACHE)[0])
        for c in caches:
            assert (c._tensors[2].cpu().numpy().reshape(slots_n, -1)[named] == want).all()


def test_many_rows_of_which_none_is_in_the_cache():
    c = new_cache(2, 10, 2, 64)
    t = torch.ones((9000, 128), dtype=torch.bfloat16, device=DEV)
    for slot in (-1, 20, 2 ** 31 - 1):
        sfs.sfs_cache4_store(c, t, 128, t, 128, 0, torch.full((9000,), slot, dtype=torch.int32, device=DEV), 9000)
    assert all((p == GUARD).all() for p in c._tensors)


def test_slots_in_order_and_scales_at_the_ends_of_their_range():
    heads, dim = 1, 128
    x = np.ones((4, 128))
    x[0] *= 2.0 ** 100; x[1] *= 2.0 ** -100; x[2, 7] = np.nan; x[3, 64:] = 0.0
    c = new_cache(1, 5, heads, dim)
    t, y = as_input(x, "bf16")
    sfs.sfs_cache4_store(c, t.to(DEV), dim, t.to(DEV), dim, 0, None, 4)
    out = torch.full((5, dim), 77.0, dtype=torch.float32, device=DEV)
    sfs.sfs_cache4_load(c, None, 4, out, dim, None, 0, 1)
    want = R.values(*R.quantize(y, R.CACHE))
    assert want[0, 0] == 6 * 2.0 ** 65 and want[1, 0] == 0 and np.isnan(want[2, :32]).all()
    got = out.double().cpu().numpy()
    assert np.array_equal(got[:4], want, equal_nan=True) and (got[4] == 77.0).all()
