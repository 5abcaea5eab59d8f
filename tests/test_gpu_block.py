"""The operators of a block together, as a serving program calls them: norm to codes, query,
key and value products, rotary positions, the eight-bit cache and its attention, the output
product, the norm between, routing, experts and their sum; eagerly, captured and replayed with
another step's values, and on two streams at once."""
import math
import os
import re

import pytest
import torch

from paper_2608_29809_gb300 import synth
from tests import block_ref as B
from tests import eight_bit_ref as E

pytestmark = pytest.mark.gpu

BF, F32 = torch.bfloat16, torch.float32


@pytest.fixture(scope="module")
def lib():
    from paper_2608_29809_gb300 import build
    build.build()
    from paper_2608_29809_gb300 import regioncache as R
    d = synth.Dims(hidden=128, heads=2, mlp=128, layers=1, grid_h=4, grid_w=4, timesteps=1)
    ctx = R.rc_create(R.dims_struct(d))
    yield R, ctx
    R.rc_destroy(ctx)


def _rand(*shape, seed=0, scale=1.0):
    return synth.randn(shape, synth.tensor_seed(seed, *shape), "cuda", scale)
COLS, HEADS, KV, DH, EXPERTS, TOP_K, MLP = 256, 4, 2, 64, 8, 2, 200
ROWS, ITEMS, TABLE = 40, 3, 4


class Block:
    """The buffers of a block over up to ROWS rows of ITEMS requests; what a step reads is in
    x, positions, lengths and counts, and its rows are those that row_offsets says."""

    def __init__(self, lib):
        R, ctx = self.R, self.ctx = lib
        qkv = (HEADS + 2 * KV) * DH

        def weight(rows, cols, seed):
            m = R.Fp8Matrix(rows, cols, 128)
            w = _rand(rows, cols, seed=seed, scale=1 / math.sqrt(cols))
            R.rc_fp8_quantize(ctx, w, cols, R.RC_F32, m)
            return m

        def zeros(*shape, dtype=F32):
            return torch.zeros(shape, dtype=dtype, device="cuda")

        ints = torch.int32
        self.Wqkv, self.Wo = weight(qkv, COLS, 1), weight(COLS, HEADS * DH, 2)
        self.Wr = weight(EXPERTS, COLS, 3)
        self.W1 = weight(EXPERTS * 512, COLS, 4)   # (of which 2 * MLP rows count)
        self.W2 = weight(EXPERTS * COLS, MLP, 5)
        self.b1 = _rand(EXPERTS, 2 * MLP, seed=6, scale=0.1)
        self.mod = _rand(ITEMS, 3 * COLS, seed=7, scale=0.5)
        self.gate, self.scale, self.shift = self.mod.split(COLS, 1)
        self.w_norm = (1 + _rand(COLS, seed=8, scale=0.2))
        self.lengths, self.counts = zeros(ITEMS, dtype=ints), zeros(ITEMS, dtype=ints)
        self.positions = zeros(ROWS, 1, dtype=ints)
        self.offsets, self.slots = zeros(ITEMS + 1, dtype=ints), zeros(ROWS, dtype=ints)
        self.table, self.used = zeros(ITEMS, TABLE, dtype=ints), zeros(1, dtype=ints)
        self.free = torch.arange(ITEMS * TABLE, dtype=ints, device="cuda")
        self.pool = R.Kv8Pool(ITEMS * TABLE, KV, DH)
        self.x, self.out = zeros(ROWS, COLS), torch.full((ROWS, COLS), 7.0, device="cuda")
        self.x1 = zeros(ROWS, COLS)
        self.n1, self.n2 = R.Fp8Matrix(ROWS, COLS), R.Fp8Matrix(ROWS, COLS)
        self.qkv, self.qk = zeros(ROWS, qkv, dtype=BF), zeros(ROWS, (HEADS + KV) * DH, dtype=BF)
        self.o, self.o8 = zeros(ROWS, HEADS * DH, dtype=BF), R.Fp8Matrix(ROWS, HEADS * DH)
        self.h, self.z = zeros(ROWS, COLS, dtype=BF), zeros(ROWS, EXPERTS)
        self.ids, self.w = zeros(ROWS, TOP_K, dtype=ints), zeros(ROWS, TOP_K)
        self.first = zeros(EXPERTS + 1, dtype=ints)
        self.source, self.places = zeros(ROWS * TOP_K, dtype=ints), zeros(ROWS, TOP_K, dtype=ints)
        self.u8, self.d = R.Fp8Matrix(ROWS * TOP_K, MLP), zeros(ROWS * TOP_K, COLS, dtype=BF)
        self.rotary = R.Rotary(DH)
        self.routing = R.Routing(EXPERTS, TOP_K)
        norm = R.Norm(R.RC_NORM_RMS, 1e-6, self.w_norm)
        self.enter = R.ResidualNorm(COLS, x=self.x, y=self.n1, pre=norm, scale=self.scale,
                                    shift=self.shift, row_offsets=self.offsets)
        self.between = R.ResidualNorm(COLS, x=self.x, h=self.h, x_out=self.x1, y=self.n2, pre=norm,
                                      gate=self.gate, row_offsets=self.offsets)
        self.join = R.ResidualNorm(COLS, x=self.x1, h=self.d, x_out=self.out, places=self.places,
                                   weights=self.w, gate=self.gate, row_offsets=self.offsets)
        R.rc_sync(ctx)

    def feed(self, seed, lengths, counts):
        n = sum(counts)
        at = torch.cat([torch.arange(a - c, a) for a, c in zip(lengths, counts)])
        self.x.copy_(_rand(ROWS, COLS, seed=seed))
        self.positions.fill_(-2 ** 31)  # (of rows that there are not)
        self.positions[:n, 0] = at.int().cuda()
        self.lengths.copy_(torch.tensor(lengths, dtype=torch.int32))
        self.counts.copy_(torch.tensor(counts, dtype=torch.int32))
        self.live = n

    def step(self, stream=None):
        R, ctx, live = self.R, self.ctx, self.offsets[ITEMS:]
        qkv = self.qkv.shape[1]
        R.rc_kv8_tables(ctx, self.lengths, self.counts, None, ITEMS, self.free, ITEMS * TABLE,
                        self.table, TABLE, self.offsets, self.slots, ROWS, self.used, stream)
        R.rc_norm_residual(ctx, self.enter, stream)
        R.rc_fp8_linear(ctx, self.n1, self.Wqkv, None, self.qkv, qkv, R.RC_BF16, stream)
        R.rc_rotary_apply(ctx, self.rotary, self.qkv, qkv, R.RC_BF16, ROWS, HEADS + KV, DH,
                          self.positions, live, False, self.qk, self.qk.shape[1], stream)
        v = self.qkv[:, (HEADS + KV) * DH:]
        k = self.qkv[:, HEADS * DH:(HEADS + KV) * DH]  # (beside its values: turned in place)
        R.rc_rotary_apply(ctx, self.rotary, k, qkv, R.RC_BF16, ROWS, KV, DH,
                          self.positions, live, False, k, qkv, stream)
        R.rc_kv8_store(ctx, self.pool, k, v, qkv, R.RC_BF16, self.slots, ROWS, live,
                       R.RC_KV8_APPEND, stream)
        R.rc_kv8_attention(ctx, self.pool, self.qk, self.qk.shape[1], ROWS, self.offsets,
                           self.lengths, ITEMS, ROWS, self.table, TABLE, HEADS, True, self.o,
                           HEADS * DH, stream)
        R.rc_fp8_quantize(ctx, self.o, HEADS * DH, R.RC_BF16, self.o8, stream)
        R.rc_fp8_linear(ctx, self.o8, self.Wo, None, self.h, COLS, R.RC_BF16, stream)
        R.rc_norm_residual(ctx, self.between, stream)
        R.rc_fp8_linear(ctx, self.n2, self.Wr, None, self.z, EXPERTS, R.RC_F32, stream)
        R.rc_experts_route(ctx, self.routing, self.z, EXPERTS, R.RC_F32, ROWS, live, self.ids,
                           self.w, stream)
        R.rc_experts_sort(ctx, self.ids, ROWS, TOP_K, EXPERTS, live, self.first, self.source,
                          self.places, stream)
        pairs = ROWS * TOP_K
        R.rc_experts_linear(ctx, self.n2, self.W1, self.b1, EXPERTS, MLP, self.first, self.source,
                            pairs, R.RC_ACT_GATED_SILU, None, 0, 0, self.u8, stream)
        R.rc_experts_linear(ctx, self.u8, self.W2, None, EXPERTS, COLS, self.first, None, pairs,
                            R.RC_ACT_NONE, self.d, COLS, R.RC_BF16, None, stream)
        R.rc_norm_residual(ctx, self.join, stream)

    def results(self):
        self.R.rc_sync(self.ctx)
        n = self.live
        return [t.clone() for t in (self.out, self.qk[:n], self.o[:n], self.x1[:n], self.ids,
                                    self.w, self.first, self.places, self.offsets, self.table,
                                    self.pool.k, self.pool.k_scale)]


FILL, MORE = ([5, 1, 20], [5, 1, 20]), ([6, 2, 21], [1, 1, 1])


def _same(got, want):
    for i, (a, b) in enumerate(zip(got, want)):
        assert torch.equal(a, b), i


def _codes_close(m, want, tol, n):
    """Codes of f64 values known up to tol: half a step of e4m3, or of its least value with the
    scale, a power of two of which the largest of the group takes more than a quarter."""
    rows, cols = want.shape
    got = E.values(m.codes, m.scales, 1, cols)[:n]
    for c in range(0, cols, 128):
        w, t = want[:, c:c + 128], tol[:, c:c + 128]
        top = (w.abs() + t).amax(1, keepdim=True)
        limit = t + 2.0 ** -4 * (w.abs() + t) + 2.0 ** -10 * top / 112
        assert bool(((got[:, c:c + 128] - w).abs() <= limit).all())


def test_each_stage_of_a_step(lib):
    """A first fill of 26 rows in a batch padded to 40, each stage from what it was given."""
    R, ctx = lib
    b = Block(lib)
    b.feed(30, *FILL)
    b.step()
    R.rc_sync(ctx)
    n = b.live
    item = torch.repeat_interleave(torch.arange(ITEMS), torch.tensor(FILL[1]))
    x, w = b.x[:n].cpu().double(), b.w_norm
    gate, scale, shift = (t.cpu().double()[item] for t in (b.gate, b.scale, b.shift))
    none = ("none", 0, None, None)
    _, _, y, dy = B.residual(x, None, None, None, 1.0, none, ("rms", 1e-6, w, None), scale, shift)
    _codes_close(b.n1, y, dy, n)
    at = torch.cat([torch.arange(c) for c in FILL[1]])[:, None]
    f, axis = B.frequencies([DH // 2], 1e4)
    # (the queries' and keys' heads; the keys beside the values have been turned in place)
    raw = torch.zeros(ROWS, b.qkv.shape[1], dtype=BF, device="cuda")
    R.rc_fp8_linear(ctx, b.n1, b.Wqkv, None, raw, raw.shape[1], R.RC_BF16)
    R.rc_sync(ctx)
    heads = raw[:n, :(HEADS + KV) * DH].cpu().double().view(n, HEADS + KV, DH)
    # as test_gpu_rotary.py: the angle, the series and three roundings
    tol = (2.0 ** -22 + 3 * B.F32_HALF + 16 * 20 * 2.0 ** -53) * 2 * \
        heads.abs().amax(-1, keepdim=True)
    B.close(b.qk[:n].view(n, HEADS + KV, DH), B.rotate(heads, at, f, axis, 0, True),
            tol.expand_as(heads), BF, "turned")
    assert torch.equal(b.qkv[:n, HEADS * DH:(HEADS + KV) * DH], b.qk[:n, HEADS * DH:])
    x1, dx, y, dy = B.residual(x, b.h[:n].cpu().double(), torch.zeros(n, COLS).double(), gate, 1.0,
                               none, ("rms", 1e-6, w, None), None, None)
    B.close(b.x1[:n], x1, dx, F32, "between")
    _codes_close(b.n2, y, dy, n)
    ids, weights = B.route(b.z[:n], "softmax", TOP_K)
    assert torch.equal(b.ids[:n].cpu(), ids) and bool((b.ids[n:] == -1).all())
    # exponentials and their sum, f32
    assert bool(((b.w[:n].cpu().double() - weights).abs() <= 2.0 ** -20 * weights).all())
    first, source, places = B.sort(ids, EXPERTS)
    assert torch.equal(b.first.cpu(), first) and torch.equal(b.places[:n].cpu(), places)
    assert torch.equal(b.source[:n * TOP_K].cpu(), source) and bool((b.places[n:] == -1).all())
    n2 = E.values(b.n2.codes, b.n2.scales, 1, COLS)
    w1 = E.values(b.W1.codes, b.W1.scales, 128, COLS).view(EXPERTS, 512, COLS)
    w2 = E.values(b.W2.codes, b.W2.scales, 128, MLP).view(EXPERTS, COLS, MLP)
    u8 = E.values(b.u8.codes, b.u8.scales, 1, MLP)
    for e in range(EXPERTS):
        lo, hi = int(first[e]), int(first[e + 1])
        if lo == hi:
            continue
        rows, wide = n2[source[lo:hi].long()], w1[e, :2 * MLP]
        s = rows @ wide.t() + b.b1[e].cpu().double()
        # COLS additions and the bias's, 2^-23 of the magnitudes each
        ds = (COLS + 1) * 2.0 ** -23 * (rows.abs() @ wide.abs().t() + b.b1[e].cpu().double().abs())
        g, c = s[:, :MLP], s[:, MLP:]
        act = g * torch.sigmoid(g)
        tol = (1.1 * ds[:, :MLP] + 2.0 ** -16 * act.abs() + 2.0 ** -25) * \
            (c.abs() + ds[:, MLP:]) + act.abs() * ds[:, MLP:]
        part = R.Fp8Matrix(hi - lo, MLP)
        part.codes.copy_(b.u8.codes[lo:hi]), part.scales.copy_(b.u8.scales[:, lo:hi])
        _codes_close(part, act * c, tol, hi - lo)
        d = u8[lo:hi] @ w2[e].t()
        B.close(b.d[lo:hi], d, MLP * 2.0 ** -23 * (u8[lo:hi].abs() @ w2[e].abs().t()), BF, "d")
    part = b.d.cpu().double()[places.long()] * b.w[:n].cpu().double()[:, :, None]
    out, dout, _, _ = B.residual(b.x1[:n].cpu().double(), part.sum(1),
                                 TOP_K * B.F32_HALF * part.abs().sum(1), gate, 1.0, none, none,
                                 None, None)
    B.close(b.out[:n], out, dout, F32, "joined")
    assert bool((b.out[n:] == 7).all())


def test_captured_and_replayed(lib):
    """A fill and a step of one token each, of which the second replays the first's graph."""
    eager, graph = Block(lib), Block(lib)
    want = []
    for seed, step in ((30, FILL), (31, MORE)):
        eager.feed(seed, *step)
        eager.step()
        want.append(eager.results())
    graph.feed(5, *FILL)
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=stream):
        graph.step(stream.cuda_stream)
    for i, (seed, step) in enumerate(((30, FILL), (31, MORE))):
        graph.feed(seed, *step)
        g.replay()
        torch.cuda.synchronize()
        _same(graph.results(), want[i])


def test_two_streams_at_once(lib):
    blocks = [Block(lib) for _ in range(3)]
    for b, seed in zip(blocks, (30, 40, 30)):
        b.feed(seed, *FILL)
    blocks[2].step()
    want = blocks[2].results()
    streams = [torch.cuda.Stream() for _ in range(2)]
    torch.cuda.synchronize()
    for _ in range(20):
        for b, s in zip(blocks, streams):
            b.step(s.cuda_stream)
    torch.cuda.synchronize()
    # (blocks of the cache that hold nothing yet may be taken anew; the rest is the first step's)
    _same(blocks[0].results()[:9], want[:9])
    other = Block(lib)
    other.feed(40, *FILL)
    other.step()
    _same(blocks[1].results()[:9], other.results()[:9])


def test_the_readmes_block_of_experts_runs(lib):
    R, ctx = lib
    readme = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "README.md")
    code = re.findall(r"```python\n(.*?)```", open(readme).read(), re.S)[1]
    rows = 7

    def weight(n, cols, seed):
        m = R.Fp8Matrix(n, cols, 128)
        R.rc_fp8_quantize(ctx, _rand(n, cols, seed=seed, scale=1 / math.sqrt(cols)), cols, R.RC_F32,
                          m)
        return m

    def ints(*shape):
        return torch.zeros(shape, dtype=torch.int32, device="cuda")

    x = _rand(rows, 1152, seed=1)
    x0 = x.cpu().double()
    names = dict(R=R, ctx=ctx, rows=rows, x=x, norm_weight=1 + _rand(1152, seed=2, scale=0.1),
                 w_router=weight(16, 1152, 3), w_up=weight(16 * 4608, 1152, 4),
                 w_down=weight(16 * 1152, 2304, 5), logits=torch.zeros(rows, 16, device="cuda"),
                 ids=ints(rows, 2), weights=torch.zeros(rows, 2, device="cuda"), first=ints(17),
                 source=ints(2 * rows), places=ints(rows, 2),
                 d=torch.zeros(2 * rows, 1152, dtype=BF, device="cuda"))
    exec(code, names)
    R.rc_sync(ctx)
    ids, weights = B.route(names["logits"], "softmax", 2)
    assert torch.equal(names["ids"].cpu(), ids)
    first, source, places = B.sort(ids, 16)
    assert torch.equal(names["first"].cpu(), first) and torch.equal(names["places"].cpu(), places)
    u8, w = names["u8"], names["w_down"]
    uv = E.values(u8.codes, u8.scales, 1, 2304)
    wv = E.values(w.codes, w.scales, 128, 2304).view(16, 1152, 2304)
    of = torch.repeat_interleave(torch.arange(16), (first[1:] - first[:-1]).long())
    d = torch.stack([wv[e] @ v for e, v in zip(of, uv)])
    mag = torch.stack([wv[e].abs() @ v.abs() for e, v in zip(of, uv)])
    B.close(names["d"], d, 2304 * 2.0 ** -23 * mag, BF, "down")
    part = names["d"].cpu().double()[places.long()] * names["weights"].cpu().double()[:, :, None]
    none = ("none", 0, None, None)
    want, tol, _, _ = B.residual(x0, part.sum(1), 2 * B.F32_HALF * part.abs().sum(1), None, 1.0,
                                 none, none, None, None)
    B.close(x, want, tol, F32, "joined")


def test_calls_of_several_threads(lib):
    """Two host threads at once, each with its stream and its sizes of shared memory."""
    import threading
    R, ctx = lib
    jobs = []
    for cols, cols8 in ((1152, 256), (2304, 4608)):
        x, h, y = (_rand(64, cols, seed=i) for i in range(3))
        x8, W = R.Fp8Matrix(4, cols8), R.Fp8Matrix(2 * 128, cols8, 128)
        R.rc_fp8_quantize(ctx, _rand(4, cols8, seed=4), cols8, R.RC_F32, x8)
        R.rc_fp8_quantize(ctx, _rand(256, cols8, seed=5), cols8, R.RC_F32, W)
        jobs.append(dict(op=R.ResidualNorm(cols, x=x, h=h, x_out=torch.empty_like(x), y=y,
                                           pre=R.Norm(R.RC_NORM_RMS, 1e-6)), y=y, x8=x8, W=W,
                         first=torch.tensor([0, 1, 4], dtype=torch.int32, device="cuda"),
                         z=torch.zeros(4, 128, device="cuda"), stream=torch.cuda.Stream(),
                         errors=[]))

    def work(j, n):
        try:
            for _ in range(n):
                R.rc_norm_residual(ctx, j["op"], j["stream"].cuda_stream)
                R.rc_experts_linear(ctx, j["x8"], j["W"], None, 2, 128, j["first"], None, 4,
                                    R.RC_ACT_GELU, j["z"], 128, R.RC_F32, None,
                                    j["stream"].cuda_stream)
        except Exception as e:  # noqa: BLE001
            j["errors"].append(e)

    torch.cuda.synchronize()
    want = []
    for j in jobs:
        work(j, 1)
        R.rc_sync(ctx)
        want.append((j["y"].clone(), j["z"].clone()))
    torch.cuda.synchronize()
    threads = [threading.Thread(target=work, args=(j, 300)) for j in jobs]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    R.rc_sync(ctx)
    for j, (y, z) in zip(jobs, want):
        assert not j["errors"]
        assert torch.equal(j["y"], y) and torch.equal(j["z"], z)


def _far(rows, cols, ld, dtype):
    """A matrix whose last rows lie beyond 2^31 elements."""
    assert (rows - 1) * ld > 2 ** 31
    buf = torch.empty((rows - 1) * ld + cols, dtype=dtype, device="cuda")
    return buf.as_strided((rows, cols), (ld, 1))


def test_offsets_beyond_32_bits(lib):
    R, ctx = lib
    ld, cols = 1_200_000_008, 128
    near = _rand(3, cols, seed=1).to(BF)
    for align in (0, 1):  # (whole vectors, and the general way)
        x = _far(3, cols, ld - align, BF)
        x.copy_(near)
        outs = []
        for t in (x, near.clone()):
            y = torch.zeros(3, cols, device="cuda")
            R.rc_norm_residual(ctx, R.ResidualNorm(cols, x=t, x_out=t, h=near, y=y,
                                                   pre=R.Norm(R.RC_NORM_RMS, 1e-6)))
            R.rc_rotary_apply(ctx, R.Rotary(64), t, t.stride(0), R.RC_BF16, 3, 2, 64, None, None,
                              False, t, t.stride(0))
            ids = torch.zeros(3, 4, dtype=torch.int32, device="cuda")
            w = torch.zeros(3, 4, device="cuda")
            R.rc_experts_route(ctx, R.Routing(cols, 4), t, t.stride(0), R.RC_BF16, 3, None, ids, w)
            R.rc_sync(ctx)
            outs.append((t.clone(), y, ids, w))
        for a, b in zip(*outs):
            assert torch.equal(a, b)
        del x, outs, t, y


@pytest.mark.parametrize("rows,ld", [(3, 1_200_000_008), (40, 60_000_000), (40, 60_000_001)])
def test_experts_results_beyond_32_bits(lib, rows, ld):
    R, ctx = lib
    x, W = R.Fp8Matrix(rows, 200), R.Fp8Matrix(128, 200, 128)
    R.rc_fp8_quantize(ctx, _rand(rows, 200, seed=1), 200, R.RC_F32, x)
    R.rc_fp8_quantize(ctx, _rand(128, 200, seed=2), 200, R.RC_F32, W)
    first = torch.tensor([0, rows], dtype=torch.int32, device="cuda")
    far, near = _far(rows, 100, ld, BF), torch.zeros(rows, 100, dtype=BF, device="cuda")
    for y in (far, near):
        R.rc_experts_linear(ctx, x, W, None, 1, 100, first, None, rows, R.RC_ACT_SILU, y,
                            y.stride(0), R.RC_BF16)
    R.rc_sync(ctx)
    assert torch.equal(far, near)
