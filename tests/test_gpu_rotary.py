"""rc_rotary_apply against float64: layouts, axes, parts of a head, types,
strides, far positions, the inverse and counts."""
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


def _rand(*shape, seed=0):
    return synth.randn(shape, synth.tensor_seed(seed, *shape), "cuda", 1.0)


def _check(lib, rows, heads, dh, rot, dtype, first=0, half=True, pairs=None, longest=5000, pad=0,
           off=0, inverse=False, amplitude=1.0, inplace=False, positions=True, low=0):
    R, ctx = lib
    wide = heads * dh
    buf = torch.full((off + rows * (wide + pad) + 16,), 7.0, dtype=dtype, device="cuda")
    x = buf[off:off + rows * (wide + pad)].view(rows, wide + pad)[:, :wide]
    x.copy_(_rand(rows, wide, seed=rot))
    x0 = x.cpu().double().reshape(rows, heads, dh)
    pairs = [rot // 2] if pairs is None else pairs
    plan = R.Rotary(rot, 1e4, pairs=pairs, first=first,
                    layout=R.RC_ROTARY_HALF if half else R.RC_ROTARY_PAIRS, amplitude=amplitude)
    at = torch.randint(low, longest, (rows, len(pairs)), dtype=torch.int32,
                       generator=torch.Generator().manual_seed(rows))
    obuf = buf if inplace else torch.full_like(buf, 7.0)
    y = obuf[off:off + rows * (wide + pad)].view(rows, wide + pad)
    R.rc_rotary_apply(ctx, plan, x, wide + pad, R.DTYPES[dtype], rows, heads, dh,
                      at.cuda() if positions else None, None, inverse, y, wide + pad)
    R.rc_sync(ctx)
    if not positions:
        at = torch.arange(rows, dtype=torch.int32)[:, None].expand(-1, len(pairs))
    f, axis = B.frequencies(pairs, 1e4)
    want = B.rotate(x0, at, f, axis, first, half, amplitude, inverse)
    # |a| + |b| times what cos and sin are off (2^-22: the angle's rounding, the series and its
    # Horner steps) and three roundings; the frequencies of f64 times far positions
    far = int(at.abs().max()) if at.numel() else 0
    tol = (2.0 ** -22 + 3 * B.F32_HALF + 16 * far * 2.0 ** -53) * amplitude * \
        x0.abs().amax(-1, keepdim=True) * 2
    B.close(y[:, :wide].reshape(rows, heads, dh), want, tol.expand_as(want), dtype)
    outside = torch.ones(dh, dtype=torch.bool)
    outside[first:first + rot] = False
    assert torch.equal(y[:, :wide].reshape(rows, heads, dh).cpu().double()[..., outside],
                       x0[..., outside])
    assert bool((obuf[:off] == 7).all()) and bool((y[:, wide:] == 7).all())
    assert bool((obuf[off + rows * (wide + pad):] == 7).all())


@pytest.mark.parametrize("rows,heads,dh,rot,first", [
    (1, 1, 2, 2, 0), (1, 40, 128, 128, 0), (48, 40, 128, 64, 0), (300, 32, 72, 72, 0),
    (5, 3, 72, 34, 0), (7, 5, 64, 30, 2), (9, 2, 65, 16, 48), (2, 200, 128, 128, 0),
    (33, 16, 64, 32, 32), (3, 1, 1024, 256, 700), (4, 2, 129, 62, 1), (20, 6, 80, 40, 40)])
@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("half", [True, False])
def test_heads(lib, rows, heads, dh, rot, first, dtype, half):
    _check(lib, rows, heads, dh, rot, dtype, first, half)
    _check(lib, rows, heads, dh, rot, dtype, first, half, inplace=True, inverse=True,
           amplitude=1.25)


@pytest.mark.parametrize("pad,off", [(8, 8), (5, 0), (3, 1), (4, 4), (1152, 0)])
@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("half", [True, False])
def test_strides(lib, pad, off, dtype, half):
    _check(lib, 37, 4, 72, 72, dtype, 0, half, [20, 16], pad=pad, off=off)
    _check(lib, 37, 4, 128, 96, dtype, 16, half, pad=pad, off=off, inplace=True)


@pytest.mark.parametrize("pairs", [[18, 18], [1, 35], [10, 12, 14], [1, 1, 34]])
@pytest.mark.parametrize("half", [True, False])
def test_axes(lib, pairs, half):
    _check(lib, 50, 4, 72, 72, BF, 0, half, pairs)
    _check(lib, 50, 4, 72, 72, F32, 0, half, pairs, positions=False)


@pytest.mark.parametrize("low,high", [(10 ** 6, 2 * 10 ** 6), (2 ** 31 - 100, 2 ** 31 - 1),
                                      (-2 ** 31, -2 ** 31 + 100), (-50, 50)])
def test_far_positions(lib, low, high):
    """Any position: the place within the turn is exact."""
    _check(lib, 64, 2, 128, 128, F32, longest=high, low=low)


def test_turned_back(lib):
    """The inverse is the transposed map: <R x, y> = <x, R^T y>, by differences as well (the map
    is linear)."""
    R, ctx = lib
    rows, heads, dh = 40, 3, 96
    plan = R.Rotary(64, first=8, amplitude=1.5)
    x, y = _rand(rows, heads * dh, seed=1), _rand(rows, heads * dh, seed=2)
    a, b = torch.empty_like(x), torch.empty_like(y)
    R.rc_rotary_apply(ctx, plan, x, heads * dh, R.RC_F32, rows, heads, dh, None, None, False, a,
                      heads * dh)
    R.rc_rotary_apply(ctx, plan, y, heads * dh, R.RC_F32, rows, heads, dh, None, None, True, b,
                      heads * dh)
    moved = torch.empty_like(x)
    step = _rand(rows, heads * dh, seed=3)
    xs = x + step
    R.rc_rotary_apply(ctx, plan, xs, heads * dh, R.RC_F32, rows, heads, dh, None, None, False,
                      moved, heads * dh)
    R.rc_sync(ctx)
    n = x.numel()
    left, right = (a.double() * y.double()).sum(), (x.double() * b.double()).sum()
    limit = n * 2.0 ** -20 * 1.5 * 4.0 * 4.0  # every product off by 2^-20 at most, |v| < 4 or so
    assert abs(float(left - right)) <= limit
    change = ((moved - a).double() * y.double()).sum()
    assert abs(float(change - (step.double() * b.double()).sum())) <= 4 * limit


@pytest.mark.parametrize("count", [0, 1, 17, 40])
def test_count(lib, count):
    R, ctx = lib
    x = _rand(40, 2 * 64, seed=1).to(BF)
    y = torch.full_like(x, 7.0)
    full = torch.empty_like(x)
    plan = R.Rotary(64)
    c = torch.tensor([count], dtype=torch.int32, device="cuda")
    R.rc_rotary_apply(ctx, plan, x, 128, R.RC_BF16, 40, 2, 64, None, c, False, y, 128)
    R.rc_rotary_apply(ctx, plan, x, 128, R.RC_BF16, 40, 2, 64, None, None, False, full, 128)
    R.rc_sync(ctx)
    assert torch.equal(y[:count], full[:count]) and bool((y[count:] == 7).all())


@pytest.mark.parametrize("count", [-1, 41, 2 ** 31 - 1])
def test_bad_counts_are_reported(lib, count):
    R, ctx = lib
    x = _rand(40, 128, seed=1).to(BF)
    y = torch.full_like(x, 7.0)
    c = torch.tensor([count], dtype=torch.int32, device="cuda")
    R.rc_rotary_apply(ctx, R.Rotary(64), x, 128, R.RC_BF16, 40, 2, 64, None, c, False, y, 128)
    with pytest.raises(R.RCError) as e:
        R.rc_sync(ctx)
    assert e.value.status == 6
    assert bool((y == 7).all())


@pytest.mark.parametrize("axes", [1, 2])
def test_a_callers_own_plan(lib, axes):
    """What stands behind the plan's axes is of no consequence."""
    R, ctx = lib
    pairs = [16, 16][:axes] if axes == 2 else [32]
    plan, x = R.Rotary(64, pairs=pairs), _rand(9, 64, seed=4)
    at = torch.randint(0, 5000, (9, axes), dtype=torch.int32,
                       generator=torch.Generator().manual_seed(2)).cuda()
    ys = [torch.zeros_like(x) for _ in range(2)]
    for i in range(2):
        R.rc_rotary_apply(ctx, plan, x, 64, R.RC_F32, 9, 1, 64, at, None, False, ys[i], 64)
        for a in range(axes, 3):
            plan.c.pairs[a] = -20 + a
    R.rc_sync(ctx)
    assert torch.equal(ys[0], ys[1])


def test_captured(lib):
    R, ctx = lib
    x, y = _rand(500, 16 * 72, seed=1).to(BF), torch.zeros(500, 16 * 72, dtype=BF, device="cuda")
    plan = R.Rotary(72, 100.0, pairs=[18, 18], layout=R.RC_ROTARY_PAIRS)
    at = torch.randint(0, 128, (500, 2), dtype=torch.int32, device="cuda")

    def call():
        R.rc_rotary_apply(ctx, plan, x, 1152, R.RC_BF16, 500, 16, 72, at, None, False, y, 1152)

    call()
    want = y.clone()
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        call()
    y.zero_()
    g.replay()
    R.rc_sync(ctx)
    assert torch.equal(y, want)
