"""Quantised matrices: rc_fp8_quantize bit for bit and rc_fp8_linear against
float64, at the edges of their tiles, types, strides and scales."""
import math

import pytest
import torch

from paper_2608_29809_gb300 import synth
from tests import eight_bit_ref as E

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def lib():
    from paper_2608_29809_gb300 import build as B
    B.build()
    from paper_2608_29809_gb300 import regioncache as R
    d = synth.Dims(hidden=128, heads=2, mlp=128, layers=1, grid_h=4, grid_w=4, timesteps=1)
    ctx = R.rc_create(R.dims_struct(d))
    yield R, ctx
    R.rc_destroy(ctx)


def _rand(*shape, seed=0, scale=1.0):
    return synth.randn(shape, synth.tensor_seed(seed, *shape), "cuda", scale)


def _quantized(R, ctx, x, group):
    m = R.Fp8Matrix(x.shape[0], x.shape[1], group)
    R.rc_fp8_quantize(ctx, x, x.stride(0), R.DTYPES[x.dtype], m)
    return m


def _same(m, x, group):
    codes, scales = E.quantize(x, group)
    got = m.codes[:, :x.shape[1]].cpu().view(E.F8).double()
    assert torch.equal(m.scales.cpu(), scales)
    assert torch.equal(got.isnan(), codes.isnan())
    assert torch.equal(got.nan_to_num(0.0), codes.nan_to_num(0.0))


@pytest.mark.parametrize("rows,cols", [(1, 1), (1, 1152), (3, 127), (129, 129), (16, 300),
                                       (257, 136), (128, 128), (40, 4608)])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("group", [1, 128])
@pytest.mark.parametrize("pad,off", [(0, 0), (8, 8), (3, 1)])
def test_quantize(lib, rows, cols, dtype, group, pad, off):
    R, ctx = lib
    wide = _rand(rows, cols + pad, seed=1) * torch.exp(2 * _rand(rows, 1, seed=2))
    buf = torch.zeros(off + wide.numel(), dtype=dtype, device="cuda")
    buf[off:] = wide.to(dtype).reshape(-1)
    x = buf[off:].view(rows, cols + pad)[:, :cols]
    m = R.Fp8Matrix(rows, cols, group)
    m.codes.fill_(0x55)
    R.rc_fp8_quantize(ctx, x, cols + pad, R.DTYPES[dtype], m)
    R.rc_sync(ctx)
    _same(m, x, group)
    assert bool((m.codes[:, cols:] == 0x55).all())


def test_quantize_scale_edges(lib):
    """Magnitudes at and next to 448 * 2^e, the least and the greatest ones, ties between codes."""
    R, ctx = lib
    tops = []
    for e in (-149, -135, -127, -126, -20, -1, 0, 1, 60, 119):
        t = torch.tensor(448.0 * 2.0 ** e, dtype=torch.float64).float()
        tops += [t, torch.nextafter(t, torch.tensor(math.inf)), torch.nextafter(t, torch.tensor(0.0))]
    tops += [torch.tensor(v) for v in (0.0, 1e-45, torch.finfo(torch.float32).max, 1.0)]
    x = torch.stack([torch.cat([t[None], t * (torch.arange(255) + 0.5) / 256]) for t in tops])
    x[:, 1::2] *= -1
    x = x[:, :200].cuda()
    for t in (x, x.bfloat16()):
        _same(_quantized(R, ctx, t, 1), t, 1)
    R.rc_sync(ctx)


@pytest.mark.parametrize("bad", [math.nan, math.inf, -math.inf])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("group", [1, 128])
def test_quantize_keeps_what_is_not_finite_to_its_block(lib, bad, dtype, group):
    R, ctx = lib
    x = _rand(150, 400, seed=3).to(dtype)
    x[130, 200] = bad
    m = _quantized(R, ctx, x, group)
    R.rc_sync(ctx)
    assert int((m.scales == 255).sum()) == 1
    _same(m, x, group)


def _product(R, ctx, xm, wm, b, dtype, pad=0, off=0):
    rows, n = xm.c.rows, wm.c.rows
    buf = torch.full((off + rows * (n + pad) + 16,), 7.0, dtype=dtype, device="cuda")
    y = buf[off:off + rows * (n + pad)].view(rows, n + pad)
    R.rc_fp8_linear(ctx, xm, wm, b, y, n + pad, R.DTYPES[dtype])
    R.rc_sync(ctx)
    assert bool((buf[:off] == 7).all()) and bool((y[:, n:] == 7).all())
    assert bool((buf[off + rows * (n + pad):] == 7).all())
    return y[:, :n].double().cpu()


def _linear_reference(xm, wm, b, dtype):
    """y in f64 and how far a result may be: k additions in f32, each off by at most 2^-23 of the
    magnitudes added, the bias's addition, and the rounding to the output's type (bf16: 2^-8)."""
    x = E.values(xm.codes, xm.scales, xm.c.group, xm.c.cols)
    w = E.values(wm.codes, wm.scales, wm.c.group, wm.c.cols)
    y, mag = x @ w.t(), x.abs() @ w.abs().t()
    if b is not None:
        y, mag = y + b.cpu().double(), mag + b.cpu().double().abs()
    tol = (xm.c.cols + 1) * 2.0 ** -23 * mag
    return y, tol + (2.0 ** -8 * (y.abs() + tol) if dtype == torch.bfloat16 else 0.0) + 1e-37


@pytest.mark.parametrize("rows,n,k", [
    (1, 1, 1), (1, 128, 128), (1, 1152, 4608), (5, 33, 70), (31, 384, 129), (64, 200, 1000),
    (128, 256, 256), (129, 193, 1152), (39, 3456, 1152), (257, 1152, 384), (300, 97, 16),
    (831, 640, 1152), (1500, 1152, 130), (2049, 320, 260), (831, 3500, 260), (700, 4608, 2100),
    (16384, 1160, 300), (9000, 2304, 1152)])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("bias", [True, False])
def test_linear(lib, rows, n, k, dtype, bias):
    R, ctx = lib
    x = (_rand(rows, k, seed=4) * torch.exp(_rand(rows, 1, seed=5))).bfloat16()
    w = _rand(n, k, seed=6, scale=k ** -0.5)
    xm, wm = _quantized(R, ctx, x, 1), _quantized(R, ctx, w, 128)
    b = _rand(n, seed=7) if bias else None
    want, tol = _linear_reference(xm, wm, b, dtype)
    for pad, off in ((0, 0), (3, 1), (8, 8)):
        got = _product(R, ctx, xm, wm, b, dtype, pad, off)
        assert bool(((got - want).abs() <= tol).all()), float(((got - want).abs() / tol).max())


@pytest.mark.parametrize("gx,gw", [(128, 1), (1, 1), (128, 128)])
def test_linear_takes_either_group(lib, gx, gw):
    R, ctx = lib
    xm = _quantized(R, ctx, _rand(200, 700, seed=8) * torch.exp(_rand(200, 1, seed=9)), gx)
    wm = _quantized(R, ctx, _rand(300, 700, seed=10) * torch.exp(_rand(300, 1, seed=11)), gw)
    want, tol = _linear_reference(xm, wm, None, torch.float32)
    got = _product(R, ctx, xm, wm, None, torch.float32)
    assert bool(((got - want).abs() <= tol).all())


def test_linear_far_scales(lib):
    """Blocks far apart in magnitude along k, and products near the ends of f32."""
    R, ctx = lib
    x, w = _rand(70, 640, seed=12), _rand(90, 640, seed=13)
    for b, e in enumerate((-30, 25, 0, -60, 12)):
        x[:, 128 * b:128 * b + 128] *= 2.0 ** e
        w[:, 128 * b:128 * b + 128] *= 2.0 ** (-e // 2)
    for s in (1.0, 2.0 ** 70, 2.0 ** -60):
        xm, wm = _quantized(R, ctx, x * s, 1), _quantized(R, ctx, w, 128)
        want, tol = _linear_reference(xm, wm, None, torch.float32)
        got = _product(R, ctx, xm, wm, None, torch.float32)
        assert bool(((got - want).abs() <= tol).all())


def test_linear_of_a_block_without_value(lib):
    """A NaN block makes NaN of the results that it enters and of no others."""
    R, ctx = lib
    x, w = _rand(140, 300, seed=14), _rand(260, 300, seed=15)
    x[131, 140] = math.inf
    xm, wm = _quantized(R, ctx, x, 1), _quantized(R, ctx, w, 128)
    got = _product(R, ctx, xm, wm, None, torch.float32)
    assert bool(got[131].isnan().all()) and int(got.isnan().sum()) == 260
    w[200, 5] = math.nan
    wm = _quantized(R, ctx, w, 128)
    got = _product(R, ctx, xm, wm, None, torch.bfloat16)
    assert bool(got[:, 128:256].isnan().all())
    assert not bool(got[:131, :128].isnan().any()) and not bool(got[:131, 256:].isnan().any())


def test_linear_gives_the_same_bits_again(lib):
    R, ctx = lib
    for rows, n, k in ((1, 1152, 4608), (60, 1152, 4608), (831, 4608, 1152)):
        xm, wm = (_quantized(R, ctx, _rand(rows, k, seed=16), 1),
                  _quantized(R, ctx, _rand(n, k, seed=17), 128))
        ys = [_product(R, ctx, xm, wm, None, torch.float32) for _ in range(3)]
        assert torch.equal(ys[0], ys[1]) and torch.equal(ys[0], ys[2])


def test_no_rows(lib):
    R, ctx = lib
    xm, wm = R.Fp8Matrix(0, 256), R.Fp8Matrix(128, 256, 128)
    n0 = R.rc_launch_count()
    R.rc_fp8_quantize(ctx, None, 256, R.RC_F32, xm)
    R.rc_fp8_linear(ctx, xm, wm, None, None, 128, R.RC_F32)
    assert R.rc_launch_count() == n0
    R.rc_sync(ctx)


def test_on_a_stream_of_its_own_and_captured(lib):
    """Quantise and product in order on a side stream, and replayed from a graph on new inputs."""
    R, ctx = lib
    x, w = _rand(100, 640, seed=18), _rand(256, 640, seed=19)
    wm = _quantized(R, ctx, w, 128)
    xm, y = R.Fp8Matrix(100, 640), torch.zeros(100, 256, device="cuda")
    torch.cuda.synchronize()
    st = torch.cuda.Stream()

    def go():
        R.rc_fp8_quantize(ctx, x, 640, R.RC_F32, xm)
        R.rc_fp8_linear(ctx, xm, wm, None, y, 256, R.RC_F32)

    with torch.cuda.stream(st):
        go()
    st.synchronize()
    first = y.clone()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        go()
    x.mul_(2.0)  # (exact: every result doubles)
    y.zero_()
    graph.replay()
    R.rc_sync(ctx)
    torch.cuda.synchronize()
    want, tol = _linear_reference(xm, wm, None, torch.float32)
    assert torch.equal(y, 2 * first)
    assert bool(((y.double().cpu() - want).abs() <= tol).all())
