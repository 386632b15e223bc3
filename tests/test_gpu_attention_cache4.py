"""Attention over a 4-bit cache against the plain 64-bit implementation, row by row within bounds taken from the arithmetic."""
import numpy as np
import pytest
import torch

import mx4_reference as R
from paper_2506_10848_b200 import binding as sfs

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def dev(a):
    return torch.from_numpy(np.ascontiguousarray(a)).to(DEV)


class Case:
    """A cache filled with random codes (every slot, also those that no length covers) and queries."""

    def __init__(self, batch, capacity, heads, kv, dim, n_q, seed=0, sharp=1.0, scale_span=2):
        rng = np.random.default_rng(seed)
        self.batch, self.capacity, self.heads, self.kv, self.dim, self.n_q = batch, capacity, heads, kv, dim, n_q
        slots = batch * capacity
        self.codes = [rng.integers(0, 16, size=(slots, kv, dim)).astype(np.uint8) for _ in range(2)]
        self.scales = [(126 + rng.integers(-scale_span, scale_span + 1, size=(slots, kv, dim // 32))).astype(np.uint8) for _ in range(2)]
        self.q = (torch.from_numpy(rng.normal(size=(batch * n_q, heads * dim)) * sharp)).to(torch.bfloat16)
        self.rng = rng

    def run(self, lengths=None, positions=None, left=-1, right=-1, sinks=0, ld_pad=0, stream=None):
        c = sfs.Cache4(dev(R.pack(self.codes[0])), dev(self.scales[0]), dev(R.pack(self.codes[1])), dev(self.scales[1]), self.batch, self.capacity, self.kv, self.dim)
        width = self.heads * self.dim
        rows = self.batch * self.n_q
        q = torch.full((rows, width + ld_pad), float("nan"), dtype=torch.bfloat16, device=DEV)
        q[:, :width] = self.q.to(DEV)
        out = torch.full((rows + 1, width + ld_pad), 77.0, dtype=torch.bfloat16, device=DEV)
        n = None if lengths is None else dev(np.asarray(lengths, np.int32))
        p = None if positions is None else dev(np.asarray(positions, np.int32))
        sfs.sfs_attention_cache4(c, q, width + ld_pad, out, width + ld_pad, self.heads, self.n_q, n, p, left, right, sinks, stream=stream)
        sfs.sfs_check_device_status(stream)
        got = out.double().cpu().numpy()
        assert (got[rows] == 77.0).all() and (got[:, width:] == 77.0).all()
        return got[:rows, :width]

    def check(self, lengths=None, positions=None, left=-1, right=-1, sinks=0, ld_pad=0):
        got = self.run(lengths, positions, left, right, sinks, ld_pad)
        k, v = (R.values(c, s, nan_above=192).reshape(self.batch, self.capacity, self.kv, self.dim) for c, s in zip(self.codes, self.scales))
        q = self.q.double().numpy().reshape(self.batch, self.n_q, self.heads, self.dim)
        got = got.reshape(self.batch, self.n_q, self.heads, self.dim)
        for b in range(self.batch):
            n = self.capacity if lengths is None else min(max(int(lengths[b]), 0), self.capacity)
            at = [int(np.asarray(positions).reshape(self.batch, self.n_q)[b, i]) if positions is not None else n - self.n_q + i for i in range(self.n_q)]
            computed = np.array([positions is None or p >= 0 for p in at])
            mask = np.stack([R.seen(n, p, left, right, sinks) for p in at])
            for h in range(self.heads):
                g = h // (self.heads // self.kv)
                want, bound = R.attention(q[b, :, h], k[b, :n, g], v[b, :n, g], mask)
                bound = bound + 2.0 ** -8 * (np.abs(want) + bound)
                with np.errstate(invalid="ignore"):
                    fine = np.abs(got[b, :, h] - want) <= bound
                fine |= np.isnan(want) & np.isnan(got[b, :, h])
                fine[~computed] = got[b, ~computed, h] == 77.0
                assert fine.all(), (b, h, np.argwhere(~fine)[:4], float(np.nanmax(np.abs(got[b, computed, h] - want[computed]) / np.maximum(bound[computed], 1e-300))))


@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("capacity", [1, 2, 7, 16, 31, 63, 64, 65, 127, 128, 129, 200, 500])
def test_single_tokens_over_every_length(capacity, dim):
    Case(2, capacity, 3, 3, dim, 1, seed=capacity).check()


@pytest.mark.parametrize("n_q", [1, 2, 5, 15, 16, 17, 31, 33, 64, 65, 127, 128, 129, 200, 260])
def test_query_counts(n_q):
    Case(1, 300, 2, 2, 128, n_q, seed=n_q).check()
    Case(2, 150, 1, 1, 64, n_q, seed=n_q).check(lengths=[150, 97])


@pytest.mark.parametrize("heads,kv", [(1, 1), (4, 1), (6, 2), (8, 8), (10, 2), (16, 1), (24, 3), (40, 2), (7, 7)])
@pytest.mark.parametrize("n_q", [1, 3, 40])
def test_shared_key_heads(heads, kv, n_q):
    Case(2, 100, heads, kv, 128 if kv % 2 else 64, n_q, seed=heads + n_q).check(lengths=[100, 41])


@pytest.mark.parametrize("n_q", [1, 4, 70, 150])
@pytest.mark.parametrize("left,right,sinks", [(0, 0, 0), (5, 5, 0), (16, -1, 3), (-1, 0, 0), (20, 0, 4), (0, 0, 1), (64, 64, 130), (-1, 7, 2), (1000, 1000, 5), (3, 200, 64)])
def test_windows(left, right, sinks, n_q):
    c = Case(2, 333, 2, 1, 64, n_q, seed=left + 3 * right + n_q)
    c.check(left=left, right=right, sinks=sinks)
    c.check(lengths=[333, 180], positions=c.rng.integers(0, 333, size=(2, n_q)), left=left, right=right, sinks=sinks)


@pytest.mark.parametrize("n_q", [1, 3, 130])
def test_rows_that_see_nothing_rows_left_out_and_lengths_out_of_range(n_q):
    c = Case(4, 90, 2, 2, 128, n_q, seed=1)
    pos = c.rng.integers(0, 90, size=(4, n_q))
    pos[:, -1] = -1                                         # left as it was
    pos[1, 0] = 2 ** 31 - 1
    c.check(lengths=[0, 90, 1000, -5], positions=pos)
    c.check(lengths=[0, 90, 1, 37], positions=pos, left=4, right=4)
    c.check(lengths=[10, 0, 1, 37], left=2, right=0)       # positions below zero, derived from a length shorter than the queries


@pytest.mark.parametrize("n_q", [1, 20, 140])
def test_what_is_masked_may_hold_anything(n_q):
    c = Case(2, 200, 2, 2, 128, n_q, seed=4)
    lengths = np.array([120, 33])
    for part in range(2):
        s = c.scales[part].reshape(2, 200, 2, 4)
        s[0, 120:], s[1, 33:] = 255, 255
        s[0, 20:60, :, 1] = 255                             # behind the window, inside the length
        s[1, 5:7, 0] = 193
    pos = np.stack([np.full(n_q, 110), np.full(n_q, 30)])
    c.check(lengths=lengths, positions=pos, left=40, right=30, sinks=2)
    # and where some rows of a tile see it, those alone are NaN
    pos = np.stack([np.arange(n_q) % 100 + 10, np.arange(n_q) % 30])
    c.check(lengths=lengths, positions=pos, left=9, right=2, sinks=3)


# Enough rows and heads for the tensor-memory kernel, which few rows of a small case do not reach: one row tile per key head, pairs of them,
# and key tiles divided over clusters of two to eight.
MANY = [(8, 500, 8, 8, 128, 130), (4, 300, 20, 20, 64, 128), (1, 700, 40, 40, 128, 200), (2, 260, 96, 96, 64, 140), (1, 1100, 64, 2, 128, 60), (1, 2000, 8, 1, 64, 300),
        (2, 900, 10, 2, 128, 400), (1, 3000, 16, 1, 128, 60), (1, 1500, 6, 6, 128, 1000), (3, 129, 50, 50, 128, 129), (1, 4000, 12, 4, 64, 350)]


@pytest.mark.parametrize("batch,capacity,heads,kv,dim,n_q", MANY)
def test_many_rows(batch, capacity, heads, kv, dim, n_q):
    c = Case(batch, capacity, heads, kv, dim, n_q, seed=capacity)
    c.check()
    c.check(lengths=c.rng.integers(0, capacity + 1, size=batch), ld_pad=8)


@pytest.mark.parametrize("batch,capacity,heads,kv,dim,n_q", MANY)
@pytest.mark.parametrize("left,right,sinks", [(-1, 0, 0), (100, 100, 5), (300, 20, 0), (200, -1, 130)])
def test_many_rows_with_windows(batch, capacity, heads, kv, dim, n_q, left, right, sinks):
    c = Case(batch, capacity, heads, kv, dim, n_q, seed=capacity + left)
    pos = c.rng.integers(0, capacity, size=(batch, n_q))
    pos[:, 3] = -1
    c.check(left=left, right=right, sinks=sinks)
    c.check(lengths=c.rng.integers(capacity // 2, capacity + 1, size=batch), positions=pos, left=left, right=right, sinks=sinks)


@pytest.mark.parametrize("batch,capacity,heads,kv,dim,n_q", [MANY[0], MANY[3], MANY[4], MANY[6]])
def test_many_rows_beside_nan_and_infinite_values(batch, capacity, heads, kv, dim, n_q):
    c = Case(batch, capacity, heads, kv, dim, n_q, seed=7)
    v, k = (x.reshape(batch, capacity, kv, dim // 32) for x in (c.scales[1], c.scales[0]))
    v[:, 40:44, 0, 1], v[:, capacity // 2, :, 0], v[0, capacity - 1] = 255, 200, 255
    k[:, 90, 0], k[0, capacity - 1] = 255, 193
    width = 20
    pos = c.rng.integers(0, capacity, size=(batch, n_q))
    pos[:, :4] = 300 % capacity
    c.check(positions=pos, left=width, right=width, sinks=2)
    lengths = np.full(batch, capacity - 1)                  # the last token hidden by the length
    c.check(lengths=lengths, left=200, right=0)


# Two row tiles that share every decoded key tile, over more key tiles than the ring has places; the last pair with one tile, or a part of
# its second.
PAIRS = [(3, 700, 25, 25, 128, 200), (3, 450, 50, 25, 128, 101), (3, 650, 25, 25, 64, 190), (2, 400, 30, 30, 128, 300)]


@pytest.mark.parametrize("batch,capacity,heads,kv,dim,n_q", PAIRS)
def test_pairs_of_row_tiles(batch, capacity, heads, kv, dim, n_q):
    c = Case(batch, capacity, heads, kv, dim, n_q, seed=capacity)
    c.check()
    c.check(lengths=[0, capacity, capacity // 3][:batch], ld_pad=8)
    pos = c.rng.integers(0, capacity, size=(batch, n_q))
    pos[:, 3], pos[0, -1], pos[-1, : n_q // 2] = -1, -1, capacity - 1
    c.check(lengths=[capacity, capacity - 5, 129][:batch], positions=pos, left=100, right=30, sinks=5)
    c.check(left=-1, right=0)


@pytest.mark.parametrize("batch,capacity,heads,kv,dim,n_q", PAIRS)
def test_pairs_of_row_tiles_beside_nan_and_infinite_values(batch, capacity, heads, kv, dim, n_q):
    c = Case(batch, capacity, heads, kv, dim, n_q, seed=7)
    v, k = (x.reshape(batch, capacity, kv, dim // 32) for x in (c.scales[1], c.scales[0]))
    v[:, 40:44, 0, 1], v[:, capacity // 2, :, 0], v[0, capacity - 1] = 255, 200, 255
    k[:, 90, 0], k[0, capacity - 1] = 255, 193
    pos = c.rng.integers(0, capacity, size=(batch, n_q))
    pos[:, :4] = 300 % capacity
    c.check(positions=pos, left=20, right=20, sinks=2)
    c.check(lengths=np.full(batch, capacity - 1), left=200, right=0)


def test_the_same_bits_whatever_runs_beside():
    """Row tiles in pairs, alone and over clusters: two streams at once, and a captured graph replayed, give what one call gives."""
    for shape in (PAIRS[0], PAIRS[2], MANY[0], MANY[4], MANY[7]):
        batch, capacity, heads, kv, dim, n_q = shape
        c = Case(*shape, seed=11)
        cache = sfs.Cache4(dev(R.pack(c.codes[0])), dev(c.scales[0]), dev(R.pack(c.codes[1])), dev(c.scales[1]), batch, capacity, kv, dim)
        q, width = c.q.to(DEV), heads * dim
        outs = [torch.zeros_like(q) for _ in range(4)]

        def call(i): sfs.sfs_attention_cache4(cache, q, width, outs[i], width, heads, n_q)
        call(0)
        torch.cuda.synchronize()
        streams = [torch.cuda.Stream() for _ in range(2)]
        for _ in range(5):
            for i, stream in enumerate(streams):
                with torch.cuda.stream(stream):
                    call(1 + i)
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            call(3)
        for _ in range(3):
            graph.replay()
        torch.cuda.synchronize()
        sfs.sfs_check_device_status()
        for out in outs[1:]:
            assert torch.equal(out.view(torch.int16), outs[0].view(torch.int16))


def test_many_rows_that_see_nothing():
    c = Case(8, 400, 8, 8, 128, 130, seed=1)
    pos = c.rng.integers(0, 400, size=(8, 130))
    pos[:, -1] = -1
    pos[2] = -1                                             # a whole sequence left as it was
    c.check(lengths=[0, 400, 100, 1, 0, 399, 1000, -3], positions=pos)
    c.check(lengths=[0, 400, 100, 1, 0, 399, 1000, -3], positions=pos, left=4, right=4)
    c = Case(1, 1100, 64, 2, 128, 60, seed=1)               # clusters, some of whose CTAs have no tile
    c.check(lengths=[0])
    c.check(lengths=[130])


@pytest.mark.parametrize("sharp", [0.0, 30.0])
def test_many_rows_with_flat_and_peaked_scores(sharp):
    Case(8, 500, 8, 8, 128, 130, seed=2, sharp=sharp).check()
    Case(1, 1100, 64, 2, 64, 60, seed=2, sharp=sharp).check()


def test_many_rows_with_scales_over_their_whole_range():
    c = Case(8, 300, 8, 8, 128, 140, seed=8)
    c.scales[1][:] = c.rng.integers(65, 193, size=c.scales[1].shape)
    c.scales[0][:] = 127 - 10
    c.check()


def test_many_rows_with_infinite_and_nan_queries():
    c = Case(8, 300, 8, 8, 64, 140, seed=3)
    c.codes[0][:, :, 0] = 2
    q = c.q.clone()
    q[1, 0], q[2, 5] = float("inf"), float("nan")
    c.q = q
    got = c.run()
    assert np.isnan(got[1, :64]).all() and np.isnan(got[2, :64]).all() and not np.isnan(got[1:3, 64:]).any()
    assert not np.isnan(np.delete(got, [1, 2], 0)).any()
    assert np.array_equal(got, c.run(), equal_nan=True)


@pytest.mark.parametrize("sharp", [0.0, 30.0])
def test_flat_and_peaked_scores(sharp):
    for n_q in (1, 130):
        Case(1, 257, 2, 2, 64, n_q, seed=2, sharp=sharp).check()


def test_infinite_and_nan_queries_stay_in_their_rows():
    for n_q in (4, 140):
        c = Case(1, 70, 1, 1, 64, n_q, seed=3)
        c.codes[0][:, :, 0] = 2                             # the first component of every key is positive
        q = c.q.clone()
        q[1, 0], q[2, 5] = float("inf"), float("nan")
        c.q = q
        got = c.run()
        assert np.isnan(got[1]).all() and np.isnan(got[2]).all()
        assert not np.isnan(np.delete(got, [1, 2], 0)).any()


@pytest.mark.parametrize("n_q", [1, 130])
def test_scales_over_their_whole_range(n_q):
    c = Case(1, 120, 2, 2, 128, n_q, seed=8)
    c.scales[1][:] = c.rng.integers(65, 193, size=c.scales[1].shape)                 # values of 2^-63 .. 6 2^65 side by side
    c.scales[0][:] = 127 - 10
    c.check()
    c.q = (c.q.double() * 2.0 ** -60).to(torch.bfloat16)
    c.scales[0][:] = 127 + 60
    c.check()


def test_strided_queries_and_repeatability():
    for n_q in (1, 9, 150):
        c = Case(3, 140, 4, 2, 128, n_q, seed=5)
        c.check(lengths=[140, 3, 77], ld_pad=8)
        assert np.array_equal(c.run(), c.run())


def test_long_cache_with_offsets_beyond_32_bits():
    """Code bytes of the last sequence lie behind 2^32."""
    batch, capacity, kv, dim = 3, 1 << 17, 128, 128
    slots = batch * capacity
    if torch.cuda.mem_get_info()[0] < 10 * 2 ** 30:
        pytest.skip("needs 10 GB of device memory")
    z = lambda w: torch.zeros((slots, kv, w), dtype=torch.uint8, device=DEV)  # noqa: E731
    kc, ks, vc, vs = z(dim // 2), z(dim // 32), z(dim // 2), z(dim // 32)
    assert kc.numel() < 2 ** 32 and slots * kv * dim // 2 == 3 * 2 ** 30
    c = sfs.Cache4(kc, ks, vc, vs, batch, capacity, kv, dim)
    # a few tokens at the end of the last sequence, seen through a window
    n, width = 40, kv * dim
    x = torch.randn((n, 2 * width), generator=torch.Generator().manual_seed(0)).to(torch.bfloat16)
    first = slots - n
    sfs.sfs_cache4_store(c, x.to(DEV), 2 * width, x.to(DEV)[:, width:], 2 * width, 0, torch.arange(first, slots, dtype=torch.int32, device=DEV), n)
    q = torch.randn((batch, width), generator=torch.Generator().manual_seed(1)).to(torch.bfloat16)
    out = torch.zeros((batch, width), dtype=torch.bfloat16, device=DEV)
    sfs.sfs_attention_cache4(c, q.to(DEV), width, out, width, kv, 1, None, None, n - 1, 0, 0)
    sfs.sfs_check_device_status()
    kq, vq = (R.values(*R.quantize(t.double().numpy(), R.CACHE)).reshape(n, kv, dim) for t in (x[:, :width], x[:, width:]))
    for h in (0, 77, 127):
        want, bound = R.attention(q[2].double().numpy().reshape(kv, dim)[h:h + 1], kq[:, h], vq[:, h], np.ones((1, n), bool))
        got = out[2].double().cpu().numpy().reshape(kv, dim)[h]
        assert (np.abs(got - want[0]) <= bound[0] + 2.0 ** -8 * (np.abs(want[0]) + bound[0])).all(), h
    assert (out[:2] == 0).all()                             # the other sequences hold zeros


def test_a_layer_of_4_bit_operators_in_a_captured_graph():
    """Projection, cache, attention and output projection as a program runs them, captured once and replayed: the values are those of the
    plain implementation fed with the device's own projections."""
    B, n, cap, H, dim = 2, 24, 64, 4, 64
    d = H * dim
    gen = torch.Generator().manual_seed(11)
    rand = lambda *s: torch.randn(s, generator=gen)  # noqa: E731
    w_qkv, w_o = (rand(3 * d, d) * 0.06).to(torch.bfloat16).to(DEV), (rand(d, d) * 0.06).to(torch.bfloat16).to(DEV)
    u8 = lambda *s: torch.zeros(s, dtype=torch.uint8, device=DEV)  # noqa: E731

    def weight(w):
        codes, scales = u8(w.shape[0], w.shape[1] // 2), u8(sfs.mx4_scale_bytes(*w.shape))
        sfs.sfs_mx4_quantize(w, w.shape[1], 0, w.shape[0], w.shape[1], codes, w.shape[1] // 2, scales)
        return codes, scales
    wq, wo = weight(w_qkv), weight(w_o)
    c = sfs.Cache4(u8(B * cap, H, dim // 2), u8(B * cap, H, dim // 32), u8(B * cap, H, dim // 2), u8(B * cap, H, dim // 32), B, cap, H, dim)
    x = torch.zeros((B * n, d), dtype=torch.bfloat16, device=DEV)
    xc, xs = u8(B * n, d // 2), u8(sfs.mx4_scale_bytes(B * n, d))
    qkv, att, y = (torch.zeros((B * n, w), dtype=torch.bfloat16, device=DEV) for w in (3 * d, d, d))
    first = torch.zeros(1, dtype=torch.int32, device=DEV)
    row = torch.arange(n, dtype=torch.int32, device=DEV)
    slots, positions, lengths = (torch.zeros(s, dtype=torch.int32, device=DEV) for s in (B * n, B * n, B))

    def step():
        positions.copy_((first + row).repeat(B))
        slots.copy_(positions + cap * torch.arange(B, dtype=torch.int32, device=DEV).repeat_interleave(n))
        lengths.copy_((first + n).repeat(B))
        sfs.sfs_mx4_quantize(x, d, 0, B * n, d, xc, d // 2, xs)
        sfs.sfs_linear_mx4(xc, d // 2, xs, wq[0], d // 2, wq[1], qkv, 3 * d, B * n, 3 * d, d)
        sfs.sfs_cache4_store(c, qkv[:, d:], 3 * d, qkv[:, 2 * d:], 3 * d, 0, slots, B * n)
        sfs.sfs_attention_cache4(c, qkv, 3 * d, att, d, H, n, lengths, positions, 20, -1, 2)
        sfs.sfs_mx4_quantize(att, d, 0, B * n, d, xc, d // 2, xs)
        sfs.sfs_linear_mx4(xc, d // 2, xs, wo[0], d // 2, wo[1], y, d, B * n, d, d)
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        step()
    side.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    keys, vals = np.zeros((B, cap, H, dim)), np.zeros((B, cap, H, dim))
    wov = R.values(*R.quantize(w_o.double().cpu().numpy(), R.MATRIX))
    for t in range(2):
        x.copy_(rand(B * n, d).to(torch.bfloat16))
        first.fill_(t * n)
        graph.replay()
        torch.cuda.synchronize()
        now = qkv.double().cpu().numpy().reshape(B, n, 3, H, dim)
        lo, hi = t * n, t * n + n
        for to, part in ((keys, 1), (vals, 2)):
            to[:, lo:hi] = R.values(*R.quantize(now[:, :, part].reshape(-1, d), R.CACHE)).reshape(B, n, H, dim)
        got = att.double().cpu().numpy().reshape(B, n, H, dim)
        mask = np.stack([R.seen(hi, lo + i, 20, -1, 2) for i in range(n)])
        for b in range(B):
            for h in range(H):
                want, bound = R.attention(now[b, :, 0, h], keys[b, :hi, h], vals[b, :hi, h], mask)
                assert (np.abs(got[b, :, h] - want) <= bound + 2.0 ** -8 * (np.abs(want) + bound)).all()
        av = R.values(*R.quantize(att.double().cpu().numpy(), R.MATRIX))
        want = av @ wov.T
        bound = (4 + 4 + 16) * 2.0 ** -23 * (np.abs(av) @ np.abs(wov).T)
        assert (np.abs(y.double().cpu().numpy() - want) <= bound + 2.0 ** -8 * (np.abs(want) + bound)).all()
    sfs.sfs_check_device_status()


@pytest.mark.parametrize("batch,capacity,heads,kv,dim,n_q", PAIRS + [(4, 300, 32, 32, 128, 256), (24, 300, 32, 32, 128, 256), (24, 300, 32, 32, 64, 256)])
def test_sequences_without_keys_among_pairs_of_row_tiles(batch, capacity, heads, kv, dim, n_q):
    """Row tiles of a sequence of which no row sees a key, beside others that do, by queries that come from memory at a time of their own:
    zeros every time, whichever warp has its queries last."""
    c = Case(batch, capacity, heads, kv, dim, n_q, seed=17)
    cache = sfs.Cache4(dev(R.pack(c.codes[0])), dev(c.scales[0]), dev(R.pack(c.codes[1])), dev(c.scales[1]), batch, capacity, kv, dim)
    width, rows = heads * dim, batch * n_q
    queries = [torch.randn((rows, width), generator=torch.Generator(device=DEV).manual_seed(i), device=DEV).to(torch.bfloat16) for i in range(1 + 2 ** 28 // (2 * rows * width))]
    out = torch.empty((rows, width), dtype=torch.bfloat16, device=DEV)
    empty = torch.ones(rows, dtype=torch.bool, device=DEV)
    empty[n_q:2 * n_q] = False                              # the second sequence has its keys
    wrong = torch.zeros((), dtype=torch.int64, device=DEV)
    lengths = torch.zeros(batch, dtype=torch.int32, device=DEV)
    lengths[1] = capacity
    behind = torch.full((batch, n_q), 2 * capacity, dtype=torch.int32, device=DEV)         # windows behind every key
    behind[1] = torch.arange(n_q, device=DEV) % capacity
    for i in range(400):
        q = queries[i % len(queries)]
        out.fill_(77.0)
        if i % 2:
            sfs.sfs_attention_cache4(cache, q, width, out, width, heads, n_q, lengths)
        else:
            sfs.sfs_attention_cache4(cache, q, width, out, width, heads, n_q, None, behind, 50, 20, 0)
        wrong += (out[empty].view(torch.int16) != 0).sum() + (out[~empty] == 77.0).all(1).sum()
    sfs.sfs_check_device_status()
    assert int(wrong) == 0


FIRST_CALLS = """
import torch
from paper_2506_10848_b200 import binding as sfs
B, cap, H, dim, n_q = 8, 500, 8, 128, 130
z = lambda *s: torch.zeros(s, dtype=torch.uint8, device="cuda:0")
cache = sfs.Cache4(z(B * cap, H, dim // 2), z(B * cap, H, dim // 32), z(B * cap, H, dim // 2), z(B * cap, H, dim // 32), B, cap, H, dim)
q = torch.zeros((B * n_q, H * dim), dtype=torch.bfloat16, device="cuda:0")
out = torch.full((B * n_q, H * dim), 7.0, dtype=torch.bfloat16, device="cuda:0")
call = lambda rows: sfs.sfs_attention_cache4(cache, q, H * dim, out, H * dim, H, rows)
if CAPTURED_FIRST:                                          # few rows take no status word: nothing to refuse
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call(1)
    graph.replay()
call(1)                                                     # the first call outside a capture
torch.cuda.synchronize()
assert not out[:B].any() and (out[B:] == 7.0).all()
graph = torch.cuda.CUDAGraph()
with torch.cuda.graph(graph):
    call(n_q)
graph.replay()
torch.cuda.synchronize()
assert not out.any()
sfs.sfs_check_device_status()
"""


@pytest.mark.parametrize("captured_first", [False, True])
def test_a_first_call_of_few_rows_serves_a_captured_call_of_many(captured_first):
    import os
    import subprocess
    import sys
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    r = subprocess.run([sys.executable, "-c", FIRST_CALLS.replace("CAPTURED_FIRST", str(captured_first))], cwd=root, capture_output=True, text=True, timeout=300)
    assert r.returncode == 0, r.stderr[-2000:]


@pytest.mark.parametrize("batch,capacity,heads,kv,dim,n_q", [(2, 200, 2, 2, 128, 1), (1, 70, 1, 1, 64, 6), PAIRS[0], PAIRS[2], MANY[0], MANY[4], MANY[7]])
def test_a_row_whose_scores_are_all_minus_infinity_is_not_one_that_sees_nothing(batch, capacity, heads, kv, dim, n_q):
    """exp(-inf - -inf) is no number: such a row is NaN, as it is with one score of infinity, and only a row without keys is zeros."""
    c = Case(batch, capacity, heads, kv, dim, n_q, seed=23)
    c.codes[0][:] = 2 + c.codes[0] % 4                      # keys positive, so that no product with an infinity is NaN by itself
    q = c.q.clone().abs()
    q[n_q - 1, :dim] = float("-inf")                        # first head of the first sequence's last row
    c.q = q
    got = c.run()
    assert np.isnan(got[n_q - 1, :dim]).all()
    got[n_q - 1, :dim] = 0.0
    assert np.isfinite(got).all()
    lengths = np.full(batch, capacity)
    lengths[0] = 0
    assert (c.run(lengths=lengths)[:n_q] == 0).all()


@pytest.mark.parametrize("n_q", [1, 100, 200])
def test_sequences_behind_two_to_the_32_bytes_of_codes(n_q):
    """The last sequence's codes begin at byte 2^32: single tokens, one row tile and pairs of them, keys and values at the end of every
    sequence, those of the last one read back too."""
    batch, capacity, kv, dim = 5, 1 << 17, 128, 128
    if torch.cuda.mem_get_info()[0] < 20 * 2 ** 30:
        pytest.skip("needs 20 GB of device memory")
    slots, width, n = batch * capacity, kv * dim, 240
    z = lambda w: torch.zeros((slots, kv, w), dtype=torch.uint8, device=DEV)  # noqa: E731
    c = sfs.Cache4(z(dim // 2), z(dim // 32), z(dim // 2), z(dim // 32), batch, capacity, kv, dim)
    assert (batch - 1) * capacity * kv * dim // 2 == 2 ** 32
    x = torch.randn((n, 2 * width), generator=torch.Generator().manual_seed(0)).to(torch.bfloat16)
    xd = x.to(DEV)
    at = torch.arange(slots - n, slots, dtype=torch.int32, device=DEV)
    sfs.sfs_cache4_store(c, xd, 2 * width, xd[:, width:], 2 * width, 0, at, n)
    back = torch.zeros((2, n, width), dtype=torch.float32, device=DEV)
    sfs.sfs_cache4_load(c, at, n, back[0], width, back[1], width, 1)
    kq, vq = (R.values(*R.quantize(t.double().numpy(), R.CACHE)).reshape(n, kv, dim) for t in (x[:, :width], x[:, width:]))
    assert (back[0].double().cpu().numpy() == kq.reshape(n, width)).all() and (back[1].double().cpu().numpy() == vq.reshape(n, width)).all()
    q = torch.randn((batch * n_q, width), generator=torch.Generator().manual_seed(1)).to(torch.bfloat16)
    out = torch.full((batch * n_q, width), 77.0, dtype=torch.bfloat16, device=DEV)
    left = n - n_q                                          # row i sees the keys i .. n - n_q + i of the last n
    sfs.sfs_attention_cache4(c, q.to(DEV), width, out, width, kv, n_q, None, None, left, 0, 0)
    sfs.sfs_check_device_status()
    mask = np.stack([(np.arange(n) >= i) & (np.arange(n) <= n - n_q + i) for i in range(n_q)])
    for h in (0, 77, 127):
        want, bound = R.attention(q[-n_q:].double().numpy().reshape(n_q, kv, dim)[:, h], kq[:, h], vq[:, h], mask)
        got = out[-n_q:].double().cpu().numpy().reshape(n_q, kv, dim)[:, h]
        assert (np.abs(got - want) <= bound + 2.0 ** -8 * (np.abs(want) + bound)).all(), h
    assert (out[:-n_q] == 0).all()                          # the other sequences hold zeros


def test_attention_over_clusters_beside_products_on_other_streams():
    """Row tiles of 64 features over clusters leave room on their SMs for products, which take tensor memory too: what runs beside changes
    no bit of either, and all of it ends."""
    att = []
    for shape in ((1, 1100, 64, 2, 64, 60), (1, 4000, 12, 4, 64, 350), (1, 1100, 64, 2, 128, 60)):
        batch, capacity, heads, kv, dim, n_q = shape
        c = Case(*shape, seed=3)
        cache = sfs.Cache4(dev(R.pack(c.codes[0])), dev(c.scales[0]), dev(R.pack(c.codes[1])), dev(c.scales[1]), batch, capacity, kv, dim)
        att.append((cache, c.q.to(DEV), heads, n_q, heads * dim))
    gen = torch.Generator(device=DEV).manual_seed(0)
    prod = []
    for m, n, k in ((16, 4096, 12288), (9, 512, 8192), (128, 1024, 4096), (300, 2048, 512)):
        ops = []
        for r in (m, n):
            x = torch.randn((r, k), generator=gen, device=DEV).to(torch.bfloat16)
            codes, scales = torch.zeros((r, k // 2), dtype=torch.uint8, device=DEV), torch.zeros(sfs.mx4_scale_bytes(r, k), dtype=torch.uint8, device=DEV)
            sfs.sfs_mx4_quantize(x, k, 0, r, k, codes, k // 2, scales)
            ops.append((x, codes, scales))
        prod.append((m, n, k, ops))

    def attentions(outs):
        for (cache, q, heads, n_q, width), out in zip(att, outs):
            sfs.sfs_attention_cache4(cache, q, width, out, width, heads, n_q)

    def products(outs):
        for (m, n, k, ((_, a, a_s), (_, b, b_s))), out in zip(prod, outs):
            sfs.sfs_linear_mx4(a, k // 2, a_s, b, k // 2, b_s, out, n, m, n, k, 1)

    def plain(outs):
        for (m, n, k, ((x, _, _), (y, _, _))), out in zip(prod, outs):
            sfs.sfs_linear(x, k, y, k, out, n, m, n, k, 1)
    new = {attentions: lambda: [torch.zeros_like(q) for _, q, *_ in att], products: lambda: [torch.zeros((m, n), device=DEV) for m, n, *_ in prod]}
    new[plain] = new[products]
    alone, beside = ({f: new[f]() for f in new} for _ in range(2))
    for f in new:
        f(alone[f])
    torch.cuda.synchronize()
    streams = {f: torch.cuda.Stream() for f in new}
    for _ in range(60):
        for f, stream in streams.items():
            with torch.cuda.stream(stream):
                f(beside[f])
    torch.cuda.synchronize()
    sfs.sfs_check_device_status()
    for f in new:
        for x, y in zip(alone[f], beside[f]):
            assert torch.equal(x, y), f.__name__
