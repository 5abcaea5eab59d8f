"""rc_norm_residual against float64: norms, gate, residual, modulation, sums of
expert rows, types, strides, codes, items and bad indexes."""
import math

import pytest
import torch

from paper_2608_29809_gb300 import synth
from tests import block_ref as B

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


def _matrix(rows, cols, dtype, pad=0, off=0, seed=0, scale=1.0, fill=None):
    """rows x cols with rows cols + pad apart, `off` elements into their buffer."""
    buf = torch.full((off + rows * (cols + pad) + 8,), 7.0, dtype=dtype, device="cuda")
    m = buf[off:off + rows * (cols + pad)].view(rows, cols + pad)[:, :cols]
    if fill is None:
        m.copy_(_rand(rows, cols, seed=seed, scale=scale))
    return m, buf


def _guarded(buf, off, rows, cols, pad):
    body = buf[off:off + rows * (cols + pad)].view(rows, cols + pad)
    assert bool((buf[:off] == 7).all()) and bool((body[:, cols:] == 7).all())
    assert bool((buf[off + rows * (cols + pad):] == 7).all())


KINDS = {"none": 0, "layer": 1, "rms": 2}


def _norm_of(R, kind, cols, seed, affine=True):
    w = 1 + _rand(cols, seed=seed, scale=0.3) if affine and kind != "none" else None
    b = _rand(cols, seed=seed + 1, scale=0.2) if affine and kind == "layer" else None
    return (R.Norm(KINDS[kind], 1e-5, w, b) if kind != "none" else None), (kind, 1e-5, w, b)


def _check(lib, rows, cols, types, post, pre, gate, mod, a=1.0, items=1, pad=0, off=0,
           affine=True, inplace=False):
    R, ctx = lib
    tx, th, ty = types
    x, xbuf = _matrix(rows, cols, tx, pad, off, 1, 2.0)
    x += 0.5
    h = _matrix(rows, cols, th, pad, off, 2)[0] if th else None
    x_out, obuf = (x, None) if inplace else _matrix(rows, cols, tx, pad, off, fill=0)
    y, ybuf = _matrix(rows, cols, ty, pad, off, fill=0)
    x0, h0 = x.cpu().double(), h.cpu().double() if th else None
    mods = _rand(items, 3 * cols + pad, seed=5, scale=0.5)
    ends = [0] + sorted(int(v) for v in
                        torch.randint(0, rows + 1, (items - 1,),
                                      generator=torch.Generator().manual_seed(rows))) + [rows]
    off_t = torch.tensor(ends, dtype=torch.int32, device="cuda") if items > 1 else None
    po, po64 = _norm_of(R, post if th else "none", cols, 11, affine)
    pr, pr64 = _norm_of(R, pre, cols, 21, affine)
    g = mods[:, :cols] if gate and th else None
    s, t = (mods[:, cols:2 * cols], mods[:, 2 * cols:3 * cols]) if mod else (None, None)
    R.rc_norm_residual(ctx, R.ResidualNorm(cols, x=x, h=h, x_out=x_out, y=y, post=po, pre=pr,
                                           gate=g, scale=s, shift=t, residual_scale=a,
                                           row_offsets=off_t))
    R.rc_sync(ctx)
    item = torch.bucketize(torch.arange(rows), torch.tensor(ends[1:]), right=True)
    of = lambda m: None if m is None else m.cpu().double()[item]
    x1, dx, out, dy = B.residual(x0, h0, torch.zeros_like(x0), of(g), a, po64, pr64, of(s), of(t))
    B.close(x_out, x1, dx, tx, "x'")
    B.close(y, out, dy, ty, "y")
    _guarded(ybuf, off, rows, cols, pad)
    _guarded(obuf if not inplace else xbuf, off, rows, cols, pad)


@pytest.mark.parametrize("rows,cols", [
    (1, 1), (1, 1152), (3, 7), (5, 129), (2, 2047), (4, 2304), (2, 4608), (3, 5120), (2, 5121),
    (2, 9000), (1, 16384), (1027, 1152), (1100, 1280), (1300, 40), (1025, 1001)])
@pytest.mark.parametrize("types", [(F32, BF, BF), (BF, BF, BF), (BF, F32, F32), (F32, None, F32)])
def test_sizes_and_types(lib, rows, cols, types):
    _check(lib, rows, cols, types, "none", "layer", True, True)
    _check(lib, rows, cols, types, "rms", "rms", False, False, a=0.5)


@pytest.mark.parametrize("post", ["none", "layer", "rms"])
@pytest.mark.parametrize("pre", ["none", "layer", "rms"])
@pytest.mark.parametrize("gate,mod", [(True, False), (False, True)])
@pytest.mark.parametrize("affine", [True, False])
def test_kinds(lib, post, pre, gate, mod, affine):
    _check(lib, 5, 300, (F32, BF, F32), post, pre, gate, mod, a=-1.25, affine=affine)


@pytest.mark.parametrize("pad,off", [(8, 8), (3, 1), (4, 4), (1, 0)])
@pytest.mark.parametrize("rows,cols", [(6, 136), (1030, 72), (3, 2312)])
@pytest.mark.parametrize("types", [(F32, BF, F32), (BF, F32, BF)])
def test_strides(lib, rows, cols, pad, off, types):
    _check(lib, rows, cols, types, "layer", "rms", True, True, items=3, pad=pad, off=off)
    _check(lib, rows, cols, types, "none", "layer", True, True, pad=pad, off=off, inplace=True)


@pytest.mark.parametrize("items", [2, 31, 32, 33, 64, 200, 1100])
@pytest.mark.parametrize("rows", [40, 1500])
def test_items(lib, items, rows):
    """Uneven items, empty ones among them."""
    _check(lib, rows, 64, (F32, BF, F32), "none", "rms", True, True, items=items)


def test_rows_of_no_item_are_left(lib):
    R, ctx = lib
    x, y = _rand(50, 72, seed=3), torch.full((50, 72), 9.0, device="cuda")
    out = torch.full_like(x, 8.0)
    off = torch.tensor([4, 4, 30, 41], dtype=torch.int32, device="cuda")
    R.rc_norm_residual(ctx, R.ResidualNorm(72, x=x, x_out=out, y=y, pre=R.Norm(2, 0.0),
                                           row_offsets=off))
    R.rc_sync(ctx)
    none = torch.ones(50, dtype=torch.bool)
    none[4:41] = False
    assert bool((y.cpu()[none] == 9).all()) and bool((out.cpu()[none] == 8).all())
    assert torch.equal(out[4:41], x[4:41]) and not bool((y[4:41] == 9).any())


@pytest.mark.parametrize("off", [[0, 30, 20, 50], [-1, 20, 50, 50], [0, 20, 51, 51],
                                 [60, 50, 3, 2], [0, 2 ** 31 - 1, -2 ** 31, 50]])
def test_bad_offsets_are_reported(lib, off):
    R, ctx = lib
    x, y = _rand(50, 72, seed=3), torch.full((50, 72), 9.0, device="cuda")
    m = _rand(3, 72, seed=4)
    R.rc_norm_residual(ctx, R.ResidualNorm(
        72, x=x, y=y, scale=m, row_offsets=torch.tensor(off, dtype=torch.int32, device="cuda")))
    with pytest.raises(R.RCError) as e:
        R.rc_sync(ctx)
    assert e.value.status == 6
    R.rc_sync(ctx)


@pytest.mark.parametrize("rows,cols,k", [(1, 1152, 2), (7, 130, 1), (1030, 96, 3), (5, 2304, 16),
                                         (2, 6000, 4)])
@pytest.mark.parametrize("th", [BF, F32])
def test_sums_of_expert_rows(lib, rows, cols, k, th):
    R, ctx = lib
    pairs = rows * k + 3
    h = _rand(pairs, cols, seed=6).to(th)
    g = torch.Generator().manual_seed(9)
    places = torch.stack([torch.randperm(pairs, generator=g)[:k] for _ in range(rows)]).int()
    w = torch.rand(rows, k, generator=g)
    places[torch.rand(rows, k, generator=g) < 0.2] = -1
    w[places < 0] = math.nan  # (passed over with its place)
    x, x_out = _rand(rows, cols, seed=7), torch.zeros(rows, cols, device="cuda")
    gate = _rand(1, cols, seed=8)
    R.rc_norm_residual(ctx, R.ResidualNorm(cols, x=x, h=h, x_out=x_out, gate=gate,
                                           places=places.cuda(), weights=w.cuda()))
    R.rc_sync(ctx)
    there = (places >= 0)[:, :, None]
    part = torch.where(there, h.cpu().double()[places.long().clamp(min=0)] *
                       w.double().nan_to_num(0.0)[:, :, None], 0.0)
    branch, db = part.sum(1), k * B.F32_HALF * part.abs().sum(1)
    x1, dx, _, _ = B.residual(x.cpu().double(), branch, db, gate.cpu().double(), 1.0,
                              ("none", 0, None, None), ("none", 0, None, None), None, None)
    B.close(x_out, x1, dx, F32)


@pytest.mark.parametrize("rows,cols,k", [(40000, 8, 16), (30001, 20, 11)])
def test_sums_where_many_rows_have_many_places(lib, rows, cols, k):
    """More of them than a CTA holds at once; whole sums of small numbers, so exact."""
    R, ctx = lib
    pairs = rows * k // 2
    g = torch.Generator(device="cuda").manual_seed(3)
    h = torch.randint(-8, 9, (pairs, cols), generator=g, device="cuda").float()
    x = torch.randint(-8, 9, (rows, cols), generator=g, device="cuda").float()
    places = torch.randint(-pairs // 8, pairs, (rows, k), generator=g, device="cuda").int()
    w = torch.randint(-4, 5, (rows, k), generator=g, device="cuda").float()
    want = x + torch.where((places >= 0)[:, :, None],
                           h[places.long().clamp(min=0)] * w[:, :, None], 0.0).sum(1)
    R.rc_norm_residual(ctx, R.ResidualNorm(cols, x=x, h=h, x_out=x, places=places, weights=w))
    R.rc_sync(ctx)
    assert torch.equal(x, want)


def test_places_of_rows_without_an_item_are_not_read_as_such(lib):
    R, ctx = lib
    h, x, out = _rand(4, 64, seed=1), _rand(5, 64, seed=2), torch.full((5, 64), 7.0, device="cuda")
    places = torch.tensor([[9], [2], [0], [2 ** 31 - 1], [4]], dtype=torch.int32, device="cuda")
    R.rc_norm_residual(ctx, R.ResidualNorm(
        64, x=x, h=h, x_out=out, places=places, weights=torch.ones(5, 1, device="cuda"),
        row_offsets=torch.tensor([1, 3], dtype=torch.int32, device="cuda")))
    R.rc_sync(ctx)
    assert torch.equal(out[1:3], x[1:3] + h[[2, 0]])
    assert bool((out[[0, 3, 4]] == 7).all())


def test_bad_places_are_passed_over_and_reported(lib):
    R, ctx = lib
    h, x = _rand(4, 64, seed=1), _rand(2, 64, seed=2)
    out = torch.zeros_like(x)
    places = torch.tensor([[1, 4], [2 ** 31 - 1, -2 ** 31]], dtype=torch.int32, device="cuda")
    R.rc_norm_residual(ctx, R.ResidualNorm(64, x=x, h=h, x_out=out, places=places,
                                           weights=torch.ones(2, 2, device="cuda")))
    with pytest.raises(R.RCError) as e:
        R.rc_sync(ctx)
    assert e.value.status == 6
    assert torch.equal(out[1], x[1])
    assert torch.equal(out[0], x[0] + h[1])


@pytest.mark.parametrize("rows,cols", [(1, 1152), (3, 130), (2, 4608), (1030, 1152), (1100, 77),
                                       (2, 9000)])
def test_codes_are_those_of_the_f32_values(lib, rows, cols):
    R, ctx = lib
    x = _rand(rows, cols, seed=3, scale=3.0).to(BF)
    x[0, cols // 2] = 0
    y, m = torch.zeros(rows, cols, device="cuda"), R.Fp8Matrix(rows + 2, cols)
    m.codes.fill_(0x55)
    n = R.Norm(R.RC_NORM_RMS, 1e-6, _rand(cols, seed=4))
    R.rc_norm_residual(ctx, R.ResidualNorm(cols, x=x, y=y, pre=n))
    R.rc_norm_residual(ctx, R.ResidualNorm(cols, x=x, y=m, pre=n))
    want = R.Fp8Matrix(rows, cols)
    R.rc_fp8_quantize(ctx, y, cols, R.RC_F32, want)
    R.rc_sync(ctx)
    assert torch.equal(m.codes[:rows, :cols], want.codes[:, :cols])
    assert torch.equal(m.scales[:, :rows], want.scales)
    assert bool((m.codes[rows:] == 0x55).all()) and bool((m.codes[:, cols:] == 0x55).all())


@pytest.mark.parametrize("rows,cols", [(1, 1152), (3, 130), (2, 4608), (1030, 1152), (900, 2056),
                                       (2, 9000)])
@pytest.mark.parametrize("tx,th", [(BF, BF), (F32, BF), (BF, F32), (F32, F32)])
def test_codes_beside_the_residual(lib, rows, cols, tx, th):
    """The same x' and, of the same f32 values, codes as with another kind of y."""
    R, ctx = lib
    x, h = _rand(rows, cols, seed=3, scale=3.0).to(tx), _rand(rows, cols, seed=5).to(th)
    off = torch.tensor([0, rows // 2, rows], dtype=torch.int32, device="cuda")
    mod = _rand(2, 3 * cols, seed=6)
    kw = dict(x=x, h=h, pre=R.Norm(R.RC_NORM_LAYER, 1e-6, _rand(cols, seed=4)), row_offsets=off,
              post=R.Norm(R.RC_NORM_RMS, 1e-6), gate=mod[:, :cols],
              scale=mod[:, cols:2 * cols], shift=mod[:, 2 * cols:])
    y, m = torch.zeros(rows, cols, device="cuda"), R.Fp8Matrix(rows + 2, cols)
    m.codes.fill_(0x55)
    outs = [torch.zeros_like(x) for _ in range(2)]
    R.rc_norm_residual(ctx, R.ResidualNorm(cols, x_out=outs[0], y=y, **kw))
    R.rc_norm_residual(ctx, R.ResidualNorm(cols, x_out=outs[1], y=m, **kw))
    want = R.Fp8Matrix(rows, cols)
    R.rc_fp8_quantize(ctx, y, cols, R.RC_F32, want)
    R.rc_sync(ctx)
    assert torch.equal(outs[0], outs[1])
    assert torch.equal(m.codes[:rows, :cols], want.codes[:, :cols])
    assert torch.equal(m.scales[:, :rows], want.scales)
    assert bool((m.codes[rows:] == 0x55).all()) and bool((m.codes[:, cols:] == 0x55).all())


@pytest.mark.parametrize("bad", [math.nan, math.inf])
def test_what_is_not_finite_stays_in_its_row(lib, bad):
    R, ctx = lib
    x = _rand(6, 200, seed=3)
    x[2, 50] = bad
    y = torch.zeros_like(x)
    m = R.Fp8Matrix(6, 200)
    for kind in (R.RC_NORM_LAYER, R.RC_NORM_RMS):
        R.rc_norm_residual(ctx, R.ResidualNorm(200, x=x, y=y, pre=R.Norm(kind, 1e-6)))
        R.rc_norm_residual(ctx, R.ResidualNorm(200, x=x, y=m, pre=R.Norm(kind, 1e-6)))
        R.rc_sync(ctx)
        assert not bool(y[2].isfinite().all()) and bool(y[[0, 1, 3, 4, 5]].isfinite().all())
        assert bool((m.scales[:, [0, 1, 3, 4, 5]] != 255).all()) and int(m.scales[0, 2]) == 255


def test_constant_and_zero_rows(lib):
    """A layer norm of a constant row is its bias (the differences are zero); of a zero row, rms
    gives zeros."""
    R, ctx = lib
    x = torch.full((2, 1000), 3.0, device="cuda")
    b, y = _rand(1000, seed=2), torch.zeros(2, 1000, device="cuda")
    R.rc_norm_residual(ctx, R.ResidualNorm(1000, x=x, y=y,
                                           pre=R.Norm(R.RC_NORM_LAYER, 1e-5, None, b)))
    R.rc_sync(ctx)
    assert torch.equal(y, b.expand(2, -1))
    x.zero_()
    R.rc_norm_residual(ctx, R.ResidualNorm(1000, x=x, y=y, pre=R.Norm(R.RC_NORM_RMS, 1e-5)))
    R.rc_sync(ctx)
    assert bool((y == 0).all())


def test_branch_alone(lib):
    """Without x the branch is the residual."""
    R, ctx = lib
    h, out = _rand(9, 88, seed=1).to(BF), torch.zeros(9, 88, dtype=BF, device="cuda")
    R.rc_norm_residual(ctx, R.ResidualNorm(88, h=h, x_out=out))
    R.rc_sync(ctx)
    assert torch.equal(out, h)


def test_captured_and_on_another_stream(lib):
    R, ctx = lib
    x, y = _rand(1200, 1152, seed=1), torch.zeros(1200, 1152, device="cuda")
    op = R.ResidualNorm(1152, x=x, x_out=x, h=_rand(1200, 1152, seed=2), y=y,
                        pre=R.Norm(R.RC_NORM_LAYER, 1e-6))
    x0 = x.clone()
    R.rc_norm_residual(ctx, op)
    want, want_x = y.clone(), x.clone()
    R.rc_sync(ctx)
    x.copy_(x0)
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=s):
        R.rc_norm_residual(ctx, op)
    y.zero_()
    g.replay()
    torch.cuda.synchronize()
    assert torch.equal(y, want) and torch.equal(x, want_x)
    with torch.cuda.stream(s):
        x.copy_(x0)
        R.rc_norm_residual(ctx, op)
    R.rc_sync(ctx, s)
    assert torch.equal(y, want) and torch.equal(x, want_x)


@pytest.mark.parametrize("rows,cols", [(1, 1000), (5, 1000), (3, 520), (2, 72), (2, 4616), (2, 77)])
@pytest.mark.parametrize("out", ["f32", "bf16", "codes"])
def test_large_constant_rows_beside_threads_without_columns(lib, rows, cols, out):
    """The branch's layer norm is its bias; its differences from the mean are nothing, whatever the
    mean times the root is.  (Sums of 2^115 are exact, and f32 holds 8191 of them.)"""
    R, ctx = lib
    x, h = _rand(rows, cols, seed=1), torch.full((rows, cols), 2.0 ** 115, device="cuda")
    b = _rand(cols, seed=2)
    x_out, m = torch.zeros_like(x), R.Fp8Matrix(rows, cols)
    y = torch.zeros(rows, cols, dtype=BF if out == "bf16" else F32, device="cuda")
    R.rc_norm_residual(ctx, R.ResidualNorm(
        cols, x=x, h=h, x_out=x_out, y=m if out == "codes" else y,
        post=R.Norm(R.RC_NORM_LAYER, 1e-12, None, b), pre=R.Norm(R.RC_NORM_LAYER, 1e-6)))
    R.rc_sync(ctx)
    assert torch.equal(x_out, x + b)
    x1 = x.cpu().double() + b.cpu().double()
    want, tol = B.norm("layer", 1e-6, None, None, x1, B.F32_HALF * x1.abs())
    if out == "codes":
        assert bool((m.scales != 255).all()) and bool(((m.codes[:, :cols] & 0x7f) != 0x7f).all())
    else:
        B.close(y, want, tol, y.dtype)


@pytest.mark.parametrize("top_k", [0, 1])
def test_as_many_rows_as_there_can_be(lib, top_k):
    """What is asked for ahead ends with the last row, where counting on would wrap."""
    R, ctx = lib
    rows = 2 ** 31 - 1
    buf = torch.ones(rows + 64, dtype=BF, device="cuda")
    buf[rows:] = 7.0
    x = buf[:rows].view(rows, 1)
    h = torch.full((1, 1) if top_k else (rows, 1), 3.0, dtype=BF, device="cuda")
    kw = dict(places=torch.zeros(rows, 1, dtype=torch.int32, device="cuda"),
              weights=torch.ones(rows, 1, device="cuda")) if top_k else {}
    R.rc_norm_residual(ctx, R.ResidualNorm(1, x=x, h=h, x_out=x, residual_scale=2.0, **kw))
    R.rc_sync(ctx)
    assert bool((buf[:rows] == 5).all()) and bool((buf[rows:] == 7).all())


@pytest.mark.parametrize("cols", [40, 129, 1000, 1152, 4608, 6000, 16384])
def test_constant_rows_of_any_value(lib, cols):
    """A layer norm of a constant row is its bias, whatever the sums' roundings."""
    R, ctx = lib
    c = torch.cat([torch.tensor([321.55563, 0.1, 1000.1, -77.77, 1e-3, 0.0, 16777215.0]),
                   1000 * torch.rand(60, generator=torch.Generator().manual_seed(1))])
    x = c[:, None].expand(-1, cols).contiguous().cuda()
    b, y = _rand(cols, seed=2), torch.zeros(len(c), cols, device="cuda")
    eps = 1e-6
    R.rc_norm_residual(ctx, R.ResidualNorm(cols, x=x, y=y,
                                           pre=R.Norm(R.RC_NORM_LAYER, eps, None, b)))
    R.rc_sync(ctx)
    # the mean is off by n / 32 + 16 roundings of c at most, its differences' mean by as many of
    # that and four more; the root is 1 / sqrt(eps) at most.  Means that the root does not bring
    # above 1 are left at that: c steps / sqrt(eps), of which c / sqrt(eps) is at most 1 (and a
    # few roundings)
    steps = (cols / 32 + 20) * B.F32_HALF
    far = c.double().abs()[:, None] / eps ** 0.5
    tol = far * steps * torch.where(far > 1 + 2.0 ** -20, steps, 1.0) + \
        B.F32_HALF * b.cpu().double().abs()
    off = (y.cpu().double() - b.cpu().double()).abs()
    assert bool((off <= tol + 1e-30).all()), (off.amax(1) / tol.amax(1)).max()


@pytest.mark.parametrize("cols", [40, 1000, 1152, 4608, 9000])
@pytest.mark.parametrize("far", [300.0, -4096.0])
def test_rows_far_from_zero(lib, cols, far):
    """Differences from the mean of rows whose mean is large against them."""
    R, ctx = lib
    x = _rand(40, cols, seed=3) + far
    y = torch.zeros_like(x)
    R.rc_norm_residual(ctx, R.ResidualNorm(cols, x=x, y=y, pre=R.Norm(R.RC_NORM_LAYER, 1e-6)))
    R.rc_sync(ctx)
    v = x.cpu().double()
    d = v - v.mean(1, keepdim=True)
    r = 1 / torch.sqrt((d * d).mean(1, keepdim=True) + 1e-6)
    # differences from a first mean, of numbers so close, are exact; their sums' and squares' sums
    # are off by n / 32 + 16 roundings, and some more of the statistics and the result (the first
    # mean's own error, below a fiftieth of the differences, in them)
    tol = 1.1 * (cols / 32 + 32) * B.F32_HALF * ((d * r).abs() + d.abs().mean(1, keepdim=True) * r)
    off = (y.cpu().double() - d * r).abs()
    assert bool((off <= tol).all()), (off / tol).max()


@pytest.mark.parametrize("cols", [72, 77, 1152, 4616])
@pytest.mark.parametrize("far", [1e4, math.nan, math.inf])
def test_rows_do_not_hang_on_their_neighbours(lib, cols, far):
    """A row gets the same bits alone, beside another, and beside one whose mean is far off."""
    R, ctx = lib
    n = R.Norm(R.RC_NORM_LAYER, 1e-6)
    rows = _rand(6, cols, seed=4) * torch.tensor([1, 1, 3, 0.01, 1, 1], device="cuda")[:, None]
    rows[4] += 2.0  # (itself one of a large mean)
    want = torch.zeros_like(rows)
    for i in range(6):
        R.rc_norm_residual(ctx, R.ResidualNorm(cols, x=rows[i:i + 1], y=want[i:i + 1], pre=n))
    for before in (0, 1):
        x = torch.cat([rows.new_full((before, cols), far), rows.repeat_interleave(2, 0)])
        x[before + 1::2] = x[before + 1::2] + far
        x = x.repeat(300, 1)  # (of which a CTA takes several)
        y = torch.zeros_like(x)
        R.rc_norm_residual(ctx, R.ResidualNorm(cols, x=x, y=y, pre=n))
        R.rc_sync(ctx)
        got = y.view(300, 12 + before, cols)[:, before::2]
        assert torch.equal(got, want.expand_as(got))
