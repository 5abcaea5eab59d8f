"""rc_experts_linear against float64: shares of the experts, sizes at the edges of
its tiles, activations, codes, gathered rows, strides and bad indexes."""
import math

import pytest
import torch

from paper_2608_29809_gb300 import synth
from tests import eight_bit_ref as E

pytestmark = pytest.mark.gpu

BF, F32 = torch.bfloat16, torch.float32
ACTS = ("none", "gelu", "silu", "gated_silu")


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


def _quantized(R, ctx, x, group):
    m = R.Fp8Matrix(x.shape[0], x.shape[1], group)
    R.rc_fp8_quantize(ctx, x, x.shape[1], R.RC_F32, m)
    return m


def _shares(experts, pairs, seed):
    """Uneven shares, some of nothing."""
    g = torch.Generator().manual_seed(seed)
    w = torch.rand(experts, generator=g) ** 2 * (torch.rand(experts, generator=g) > 0.2)
    if float(w.sum()) == 0:
        w[0] = 1
    return torch.bincount(torch.multinomial(w, pairs, replacement=True, generator=g) if pairs else
                          torch.zeros(0, dtype=torch.long), minlength=experts)


def _gelu(v):
    return v * torch.sigmoid(2 * math.sqrt(2 / math.pi) * (v + 0.044715 * v ** 3))


class Problem:
    """Operands of experts with `shares` rows each, and the result in f64 with how far the sums
    before the activation may be off: cols additions in f32 and the bias's, each by at most 2^-23
    of the magnitudes added."""

    def __init__(self, lib, shares, cols, n, act="none", bias=True, gather=True, pad_rows=0, seed=1,
                 scale=1.0):
        R, ctx = self.R, self.ctx = lib
        self.experts, self.n, self.act = len(shares), n, act
        self.pairs = int(shares.sum())
        wide = 2 * n if act == "gated_silu" else n
        per = -(-wide // 128) * 128 + 128 * pad_rows
        rows = max(1, self.pairs // 2) if gather else self.pairs
        g = torch.Generator().manual_seed(seed)
        self.x = _quantized(R, ctx, _rand(rows, cols, seed=seed) *
                            torch.exp(_rand(rows, 1, seed=seed + 1)), 1)
        w = _rand(self.experts * per, cols, seed=seed + 2) * (scale / math.sqrt(cols))
        w.view(self.experts, per, cols)[:, wide:] = math.nan  # (what is behind an expert's rows)
        self.W = _quantized(R, ctx, w.nan_to_num(0.0), 128)
        self.W.codes.view(self.experts, per, -1)[:, wide:] = 0x7f
        self.b = _rand(self.experts, wide, seed=seed + 3, scale=0.3) if bias else None
        self.offsets = torch.cat([torch.zeros(1).long(), shares.cumsum(0)]).int()
        self.source = torch.randint(0, rows, (self.pairs,), generator=g).int() if gather else None
        xv = E.values(self.x.codes, self.x.scales, 1, cols)
        wv = E.values(self.W.codes, self.W.scales, 128, cols)
        wv = wv.view(self.experts, per, cols)[:, :wide]
        xv = xv[self.source.long()] if gather else xv
        y, mag = torch.zeros(self.pairs, wide).double(), torch.zeros(self.pairs, wide).double()
        for e in range(self.experts):
            at = slice(int(self.offsets[e]), int(self.offsets[e + 1]))
            y[at], mag[at] = xv[at] @ wv[e].t(), xv[at].abs() @ wv[e].abs().t()
            if bias:
                be = self.b[e].cpu().double()
                y[at] += be
                mag[at] += be.abs()
        tol = (cols + 1) * 2.0 ** -23 * mag
        # slopes of the activations are at most 1.13; their powers are off by up to 2^-16 of the
        # result (exponents up to 126 rounded to f32, and twice multiplied)
        if act == "gelu":
            y, tol = _gelu(y), 1.13 * tol + 2.0 ** -16 * _gelu(y).abs()
        elif act == "silu":
            y, tol = y * torch.sigmoid(y), 1.1 * tol + 2.0 ** -16 * (y * torch.sigmoid(y)).abs()
        elif act == "gated_silu":
            a, c = y.chunk(2, 1)
            ta, tc = tol.chunk(2, 1)
            s = a * torch.sigmoid(a)
            y = s * c
            tol = (1.1 * ta + 2.0 ** -16 * s.abs()) * (c.abs() + tc) + s.abs() * tc
        self.y, self.tol = y, tol

    def call(self, y, ldy, type, y8=None, offsets=None, source=None, stream=None):
        R = self.R
        off = (self.offsets if offsets is None else offsets).cuda()
        src = self.source if source is None else source
        R.rc_experts_linear(self.ctx, self.x, self.W, self.b, self.experts, self.n, off,
                            None if src is None else src.cuda(), self.pairs,
                            ACTS.index(self.act), y, ldy, type, y8, stream)

    def check(self, dtype, pad=0, off=0):
        R = self.R
        wide = self.n + pad
        buf = torch.full((off + self.pairs * wide + 64,), 7.0, dtype=dtype, device="cuda")
        y = buf[off:off + self.pairs * wide].view(self.pairs, wide)
        self.call(y, wide, R.DTYPES[dtype])
        R.rc_sync(self.ctx)
        got = y[:, :self.n].cpu().double()
        limit = self.tol + torch.finfo(dtype).eps / 2 * (self.y.abs() + self.tol) + 1e-37
        bad = ~((got - self.y).abs() <= limit)
        assert not bool(bad.any()), (
            int(bad.sum()), bad.numel(), bad.nonzero()[:5].tolist(), got[bad][:5], self.y[bad][:5])
        assert bool((buf[:off] == 7).all()) and bool((y[:, self.n:] == 7).all())
        assert bool((buf[off + self.pairs * wide:] == 7).all())
        return y

    def check_codes(self):
        R, n = self.R, self.n
        m = R.Fp8Matrix(self.pairs + 2, n)
        m.codes.fill_(0x55)
        m.scales.fill_(0x33)
        self.call(None, 0, 0, m)
        R.rc_sync(self.ctx)
        assert bool((m.codes[self.pairs:] == 0x55).all()) and bool((m.codes[:, n:] == 0x55).all())
        assert bool((m.scales[:, self.pairs:] == 0x33).all())
        for g in range(-(-n // 128)):
            at = slice(128 * g, min(n, 128 * g + 128))
            y, tol = self.y[:, at], self.tol[:, at]
            top, most = y.abs().amax(1), tol.amax(1)
            lo = E.scale_exponent((top - most).clamp(min=0))
            hi = E.scale_exponent(top + most)
            b = m.scales[g, :self.pairs].cpu().double() - 127
            assert bool(((b >= lo) & (b <= hi)).all())
            scale = torch.exp2(b)[:, None]
            got = m.codes[:self.pairs, at].cpu().view(E.F8).double() * scale
            # half a step of e4m3: 2^-4 of the value, and of the least normal (2^-6) below it
            limit = tol + 2.0 ** -4 * (y.abs() + tol) + 2.0 ** -10 * scale
            assert bool(((got - y).abs() <= limit).all())
        return m


@pytest.mark.parametrize("pairs,experts", [(1, 1), (2, 8), (5, 64), (31, 3), (128, 1), (129, 1),
                                           (300, 64), (257, 2), (1000, 5), (700, 1), (640, 1024)])
@pytest.mark.parametrize("cols,n", [(128, 128), (70, 33), (1152, 200)])
@pytest.mark.parametrize("gather", [True, False])
def test_shares(lib, pairs, experts, cols, n, gather):
    if experts == 1024 and cols > 128:
        cols = 144
    p = Problem(lib, _shares(experts, pairs, pairs), cols, n, gather=gather)
    p.check(BF)
    p.check(F32)
    p.check_codes()


@pytest.mark.parametrize("shares", [[1], [127], [128], [129], [255, 1], [256], [257, 0, 33],
                                    [0, 0, 31, 32], [500, 3, 0, 400]])
@pytest.mark.parametrize("act", ACTS)
@pytest.mark.parametrize("n", [31, 64, 129, 400])
def test_activations(lib, shares, act, n):
    p = Problem(lib, torch.tensor(shares), 300, n, act, scale=3.0)
    p.check(F32)
    p.check(BF)
    p.check_codes()


@pytest.mark.parametrize("cols,n", [(1, 1), (16, 8), (129, 256), (1000, 1152), (4608, 130),
                                    (2100, 640), (8200, 65)])
@pytest.mark.parametrize("pairs", [3, 40, 400])
@pytest.mark.parametrize("bias", [True, False])
def test_sizes(lib, cols, n, pairs, bias):
    p = Problem(lib, _shares(3, pairs, 5), cols, n, "silu", bias, pad_rows=1)
    p.check(BF)
    p.check(F32)
    p.check_codes()


@pytest.mark.parametrize("shares,cols,n,act", [
    ([4000, 100, 2500, 0, 1411], 1152, 2304, "gated_silu"), ([2064, 2064], 1152, 1160, "gelu"),
    ([9000], 260, 1500, "none"), ([300] * 40, 400, 700, "gated_silu"),
    ([5] * 60, 1152, 1152, "none"), ([1, 1, 0, 0, 0, 0, 0, 0], 1152, 4608, "gelu"),
    ([1, 1, 0, 0, 0, 0, 0, 0], 4608, 1152, "none")])
@pytest.mark.parametrize("gather", [True, False])
def test_many_tiles(lib, shares, cols, n, act, gather):
    p = Problem(lib, torch.tensor(shares), cols, n, act, gather=gather)
    p.check(BF)
    p.check(F32)
    p.check_codes()


@pytest.mark.parametrize("pad,off", [(8, 8), (3, 1), (4, 0), (1, 0)])
@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("shares", [[200, 0, 57], [3, 2, 1]])
def test_strides(lib, pad, off, dtype, shares):
    Problem(lib, torch.tensor(shares), 200, 93, "gelu").check(dtype, pad, off)


def test_as_a_plain_layer(lib):
    """One expert without source, of f32 sums: rc_fp8_linear with an activation."""
    R, ctx = lib
    p = Problem(lib, torch.tensor([777]), 640, 512, gather=False)
    y = p.check(F32)
    z = torch.zeros(777, 512, device="cuda")
    W = R.Fp8Matrix.of(p.W.codes[:512], p.W.scales[:, :4], 640, 128)
    R.rc_fp8_linear(ctx, p.x, W, p.b, z, 512, R.RC_F32)
    R.rc_sync(ctx)
    assert float((y - z).abs().max()) <= float(2 * p.tol.max())


def test_places_outside_the_offsets_are_left(lib):
    R, ctx = lib
    p = Problem(lib, torch.tensor([40, 0, 30]), 200, 96)
    off = torch.tensor([5, 40, 40, 60], dtype=torch.int32)
    y = torch.full((70, 96), 7.0, device="cuda")
    m = R.Fp8Matrix(70, 96)
    m.codes.fill_(0x55)
    p.call(y, 96, R.RC_F32, offsets=off)
    p.call(None, 0, 0, m, offsets=off)
    R.rc_sync(ctx)
    for t, v in ((y, 7), (m.codes, 0x55)):
        assert bool((t[:5] == v).all()) and bool((t[60:] == v).all())
    got = y[5:40].cpu().double()
    assert bool(((got - p.y[5:40]).abs() <= p.tol[5:40] + 2.0 ** -22 * p.y[5:40].abs()).all())


@pytest.mark.parametrize("off", [[0, 50, 30, 70], [-1, 40, 40, 70], [0, 40, 71, 71],
                                 [0, 2 ** 31 - 1, -2 ** 31, 70], [70, 3, 2, 1]])
@pytest.mark.parametrize("codes", [True, False])
def test_bad_offsets_leave_their_experts_out(lib, off, codes):
    R, ctx = lib
    p = Problem(lib, torch.tensor([40, 0, 30]), 200, 96)
    y = torch.full((70, 96), 7.0, device="cuda")
    p.call(None if codes else y, 96, R.RC_F32, R.Fp8Matrix(70, 96) if codes else None,
           torch.tensor(off, dtype=torch.int32))
    with pytest.raises(R.RCError) as e:
        R.rc_sync(ctx)
    assert e.value.status == 6
    R.rc_sync(ctx)


@pytest.mark.parametrize("shares", [[3, 0, 2], [200, 0, 300]])
def test_bad_sources_are_reported(lib, shares):
    R, ctx = lib
    p = Problem(lib, torch.tensor(shares), 200, 96)
    for bad in (-1, p.x.c.rows, 2 ** 31 - 1, -2 ** 31):
        src = p.source.clone()
        src[1] = bad
        y = torch.zeros(p.pairs, 96, device="cuda")
        p.call(y, 96, R.RC_F32, source=src)
        with pytest.raises(R.RCError) as e:
            R.rc_sync(ctx)
        assert e.value.status == 6
        rest = torch.ones(p.pairs, dtype=torch.bool)
        rest[1] = False
        assert bool(((y.cpu().double() - p.y).abs() <= p.tol + 2.0 ** -22 * p.y.abs())[rest].all())


def test_what_is_not_finite_stays_in_its_row(lib):
    R, ctx = lib
    p = Problem(lib, torch.tensor([130, 70]), 300, 200, gather=False)
    p.x.scales[1, 57] = 255
    y, m = torch.zeros(200, 200, device="cuda"), R.Fp8Matrix(200, 200)
    p.call(y, 200, R.RC_F32)
    p.call(None, 0, 0, m)
    R.rc_sync(ctx)
    rest = torch.arange(200) != 57
    assert bool(y[57].isnan().all()) and bool(y[rest].isfinite().all())
    assert bool((m.scales[:, 57] == 255).all()) and bool((m.codes[57, :200] == 0x7f).all())
    assert bool((m.scales[:, rest] != 255).all())


@pytest.mark.parametrize("pairs", [5, 300])
@pytest.mark.parametrize("act", ACTS)
def test_sums_of_any_size(lib, pairs, act):
    """Activations far out, where they end, and beside columns that are not finite."""
    R, ctx = lib
    v = torch.tensor([math.nan, 1.0, -1.0, 0.5, math.inf, -2.0, 3.0, -math.inf, -1e30, 1e30, -1e4,
                      1e4, -100.0, -22.0, -21.0, -6.0, -5.5, -5.0, -0.0, 20.0, 0.0, 1e-20, -1e-20,
                      6.0, math.nan, math.nan, math.inf, 2.0, -math.inf, 4.0, -1e38, -3.0])
    v = torch.cat([v, v.flip(0), v[:5]])
    n = len(v)
    gated = act == "gated_silu"
    b = torch.cat([v, torch.linspace(0.5, 2.0, n)]) if gated else v
    x, W = R.Fp8Matrix(pairs, 128, 1), R.Fp8Matrix(256, 128, 128)
    R.rc_fp8_quantize(ctx, _rand(pairs, 128, seed=1), 128, R.RC_F32, x)
    R.rc_fp8_quantize(ctx, torch.zeros(256, 128, device="cuda"), 128, R.RC_F32, W)
    y = torch.zeros(pairs, n, device="cuda")
    R.rc_experts_linear(ctx, x, W, b.cuda()[None].contiguous(), 1, n,
                        torch.tensor([0, pairs], dtype=torch.int32, device="cuda"), None, pairs,
                        ACTS.index(act), y, n, R.RC_F32)
    R.rc_sync(ctx)
    u = v.double()
    want = u if act == "none" else _gelu(u) if act == "gelu" else u * torch.sigmoid(u)
    want = want * b[n:].double() if gated else want
    got = y.cpu().double()
    plain = want.isfinite()
    assert torch.equal(got.isnan(), want.isnan().expand_as(got))
    assert bool((got[:, want == math.inf] == math.inf).all())
    assert bool((got[:, want == -math.inf] == -math.inf).all())
    # the powers as in the sums' tolerance; 2^-25 for the 2^-31 that quotients are cut by, times
    # sums of 22 where they are not 0 and a factor of 2
    off = (got - want)[:, plain].abs()
    assert bool((off <= 2.0 ** -16 * want[plain].abs() + 2.0 ** -25).all())


def test_offsets_that_name_many_rows_again_and_again(lib):
    """2^32 tiles and more, were they counted as they stand: reported, and nothing else touched."""
    R, ctx = lib
    pairs, experts, guard = R.RC_EXPERTS_MAX_PAIRS, 1024, 4096
    x, W = R.Fp8Matrix(4, 16, 1), R.Fp8Matrix(experts * 128, 16, 128)
    R.rc_fp8_quantize(ctx, _rand(4, 16, seed=1), 16, R.RC_F32, x)
    R.rc_fp8_quantize(ctx, _rand(experts * 128, 16, seed=2), 16, R.RC_F32, W)
    off = torch.tensor([0, pairs] * (experts // 2) + [0], dtype=torch.int32, device="cuda")
    buf = torch.full((pairs + 2 * guard,), 7.0, dtype=BF, device="cuda")
    y = buf[guard:guard + pairs].view(pairs, 1)
    source = torch.zeros(pairs, dtype=torch.int32, device="cuda")
    R.rc_experts_linear(ctx, x, W, None, experts, 1, off, source, pairs, R.RC_ACT_NONE, y, 1,
                        R.RC_BF16)
    with pytest.raises(R.RCError) as e:
        R.rc_sync(ctx)
    assert e.value.status == 6
    R.rc_sync(ctx)
    assert bool((buf[:guard] == 7).all()) and bool((buf[guard + pairs:] == 7).all())


def test_captured_with_other_offsets(lib):
    """A graph follows the rows that its experts get later; two streams at once."""
    R, ctx = lib
    p = Problem(lib, torch.tensor([300, 20, 0, 180]), 512, 384, "gelu")
    y = torch.zeros(500, 384, dtype=BF, device="cuda")
    off, src = p.offsets.cuda(), p.source.cuda()

    def call(out, stream=None):
        R.rc_experts_linear(ctx, p.x, p.W, p.b, 4, 384, off, src, 500, R.RC_ACT_GELU, out, 384,
                            R.RC_BF16, None, stream)

    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        call(y)
    for cuts in ([0, 300, 320, 320, 500], [0, 0, 129, 500, 500], [0, 500, 500, 500, 500]):
        off.copy_(torch.tensor(cuts, dtype=torch.int32))
        y.zero_()
        g.replay()
        torch.cuda.synchronize()
        got = y.clone()
        streams = [torch.cuda.Stream(), torch.cuda.Stream()]
        outs = [torch.zeros_like(y) for _ in streams]
        torch.cuda.synchronize()
        for s, o in zip(streams, outs):
            call(o, s)
        torch.cuda.synchronize()
        R.rc_sync(ctx)
        assert all(torch.equal(o, got) for o in outs)
    # (the last cuts gave every row to the first expert)
    xv = E.values(p.x.codes, p.x.scales, 1, 512)[p.source.long()]
    wv = E.values(p.W.codes, p.W.scales, 128, 512)[:384]
    z = xv @ wv.t() + p.b[0].cpu().double()
    mag = xv.abs() @ wv.abs().t() + p.b[0].cpu().double().abs()
    limit = 1.13 * 513 * 2.0 ** -23 * mag + 2.0 ** -16 * _gelu(z).abs()
    limit = limit + 2.0 ** -8 * (_gelu(z).abs() + limit) + 1e-37
    assert bool(((got.cpu().double() - _gelu(z)).abs() <= limit).all())


@pytest.mark.parametrize("shares", [[3, 0, 2], [20, 11], [200, 0, 300]])
@pytest.mark.parametrize("up", [True, False])
@pytest.mark.parametrize("act", ["none", "gelu"])
def test_scales_far_from_one(lib, shares, up, act):
    """x at one end of f32 and W as far towards the other: the same results."""
    p = Problem(lib, torch.tensor(shares), 300, 90, act, scale=64.0)
    xs, ws = p.x.scales.int(), p.W.scales.int()
    assert int(xs.min()) > 0 and int(ws.min()) > 0
    by = min(247 - int(xs.max()), int(ws.min()) - 1) if up else \
        -min(int(xs.min()) - 1, 247 - int(ws.max()))
    assert abs(by) > 105
    p.x.scales.copy_((xs + by).to(torch.uint8))
    p.W.scales.copy_((ws - by).to(torch.uint8))
    p.check(F32)
    p.check(BF)
    p.check_codes()


@pytest.mark.parametrize("pairs", [5, 300])
@pytest.mark.parametrize("act", ACTS[1:])
def test_activations_far_below_zero(lib, pairs, act):
    """Small results keep their bits, in each type."""
    R, ctx = lib
    n = 300
    v = torch.linspace(-7.5, 2.0, n) if act == "gelu" else torch.linspace(-80.0, 2.0, n)
    gated = act == "gated_silu"
    b = torch.cat([v, torch.linspace(0.5, 2.0, n)]) if gated else v
    x, W = R.Fp8Matrix(pairs, 128, 1), R.Fp8Matrix(640, 128, 128)
    R.rc_fp8_quantize(ctx, _rand(pairs, 128, seed=1), 128, R.RC_F32, x)
    R.rc_fp8_quantize(ctx, torch.zeros(640, 128, device="cuda"), 128, R.RC_F32, W)
    m = R.Fp8Matrix(pairs, n)
    outs = {t: torch.zeros(pairs, n, dtype=t, device="cuda") for t in (F32, BF)}
    for t, y in list(outs.items()) + [(None, None)]:
        R.rc_experts_linear(ctx, x, W, b.cuda()[None].contiguous(), 1, n,
                            torch.tensor([0, pairs], dtype=torch.int32, device="cuda"), None,
                            pairs, ACTS.index(act), y, n, R.RC_F32 if t is None else R.DTYPES[t],
                            None if y is not None else m)
    R.rc_sync(ctx)
    u = v.double()
    want = _gelu(u) if act == "gelu" else u * torch.sigmoid(u)
    want = want * b[n:].double() if gated else want
    # the power of 2 that is taken, at most 116 (61 with GELU), is off by two roundings of f32
    # (five), and so is the result by 61 * 5 * 2^-24 of itself times log 2 at most; the powers'
    # and reciprocals' few steps
    tol = 2.0 ** -16 * want.abs()
    for t, y in outs.items():
        limit = tol + torch.finfo(t).eps / 2 * (want.abs() + tol) + 1e-37
        bad = ~((y.cpu().double() - want).abs() <= limit)
        assert not bool(bad.any()), (t, bad.nonzero()[:4].tolist(), y[bad.cuda()][:4])
    for g in range(-(-n // 128)):
        at = slice(128 * g, min(n, 128 * g + 128))
        w = want[at]
        scale = torch.exp2(m.scales[g].cpu().double() - 127)[:, None]
        e = E.scale_exponent((w.abs().max() * torch.tensor([1 - 2.0 ** -16, 1 + 2.0 ** -16])))
        assert bool(((scale >= 2.0 ** e[0]) & (scale <= 2.0 ** e[1])).all())
        got = m.codes[:, at].cpu().view(E.F8).double() * scale
        # half a step of e4m3: 2^-4 of the value, and of the least normal (2^-6) below it
        limit = tol[at] + 2.0 ** -4 * (w.abs() + tol[at]) + 2.0 ** -10 * scale
        assert bool(((got - w).abs() <= limit).all())


@pytest.mark.parametrize("shares,off", [
    ([40, 0, 30], [0, 50, 30, 60]), ([40, 0, 30], [-1, 40, 40, 70]), ([40, 0, 30], [0, 40, 71, 71]),
    ([40, 0, 30], [0, 2 ** 31 - 1, -2 ** 31, 70]), ([40, 0, 30], [70, 3, 2, 1]),
    ([400, 0, 300], [10, 400, 701, 700]), ([400, 0, 300], [700, 20, 0, 500]),
    ([3, 0, 2], [0, 4, 2, 3]), ([3, 0, 2], [-1, 3, 3, 5]), ([3, 0, 2], [0, 3, 6, 6]),
    ([3, 0, 2], [1, 2, 2 ** 31 - 1, -2 ** 31]), ([3, 0, 2], [5, 1, 0, 4])])
@pytest.mark.parametrize("gather", [True, False])
def test_what_bad_offsets_leave(lib, shares, off, gather):
    """Experts whose offsets are in order get their rows' results; the others' places, and those
    of no expert, are left as they were."""
    R, ctx = lib
    p = Problem(lib, torch.tensor(shares), 200, 96, gather=gather)
    off_t = torch.tensor(off, dtype=torch.int32)
    y = torch.full((p.pairs, 96), 7.0, device="cuda")
    m = R.Fp8Matrix(p.pairs, 96)
    m.codes.fill_(0x55)
    m.scales.fill_(0x33)
    for call in ((y, 96, R.RC_F32, None), (None, 0, 0, m)):
        p.call(*call, offsets=off_t)
        with pytest.raises(R.RCError) as e:
            R.rc_sync(ctx)
        assert e.value.status == 6
    xv = E.values(p.x.codes, p.x.scales, 1, 200)
    wv = E.values(p.W.codes, p.W.scales, 128, 200).view(3, -1, 200)[:, :96]
    of = [[] for _ in range(p.pairs)]
    for e, (lo, hi) in enumerate(zip(off, off[1:])):
        if 0 <= lo <= hi <= p.pairs:
            for r in range(lo, hi):
                of[r].append(e)
    codes = E.values(m.codes, m.scales, 1, 96)
    for r, experts in enumerate(of):
        if not experts:
            assert bool((y[r] == 7).all()) and bool((m.codes[r] == 0x55).all())
            assert bool((m.scales[:, r] == 0x33).all())
        elif len(experts) == 1:  # (a place of two experts: either's)
            x, w, b = xv[p.source[r] if gather else r], wv[experts[0]], p.b[experts[0]].cpu()
            want = w @ x + b.double()
            # as of Problem: 201 additions
            tol = 201 * 2.0 ** -23 * (w.abs() @ x.abs() + b.double().abs())
            assert bool(((y[r].cpu().double() - want).abs() <= tol + 2.0 ** -24 * want.abs()).all())
            # half a step of e4m3, of its least value with the scale a quarter of the largest's
            limit = tol + 2.0 ** -4 * (want.abs() + tol) + 2.0 ** -10 * want.abs().max() / 112
            assert bool(((codes[r] - want).abs() <= limit).all())
