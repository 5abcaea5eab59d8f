"""rc_experts_route and rc_experts_sort against float64: scores, biases, groups,
masks, ties and near ties, weights, counts and bad indexes."""
import math

import pytest
import torch

from paper_2608_29809_gb300 import synth
from tests import block_ref as B

pytestmark = pytest.mark.gpu

BF, F32 = torch.bfloat16, torch.float32
LOWEST = torch.finfo(torch.float32).min


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


def _route(lib, z, score, k, pad=0, count=None, **kw):
    R, ctx = lib
    rows, e = z.shape
    wide = torch.full((rows, e + pad), 99.0, dtype=z.dtype, device="cuda")
    wide[:, :e] = z
    ids = torch.full((rows, k), -7, dtype=torch.int32, device="cuda")
    w = torch.full((rows, k), 5.0, device="cuda")
    kw = {"top_groups" if n == "top" else "group_best" if n == "of_best" else n: v
          for n, v in kw.items()}
    routing = R.Routing(e, k, R.RC_SCORE_SOFTMAX if score == "softmax" else R.RC_SCORE_SIGMOID,
                        **kw)
    R.rc_experts_route(ctx, routing, wide, e + pad, R.DTYPES[z.dtype], rows, count, ids, w)
    R.rc_sync(ctx)
    return ids.cpu(), w.cpu()


def _check(lib, z, score, k, pad=0, **kw):
    ids, w = _route(lib, z, score, k, pad, **kw)
    names = {"top": "top_groups", "of_best": "group_best"}
    if "groups" in kw and "top" not in kw:
        kw["top"] = kw["groups"]
    want_ids, want_w = B.route(z, score, k, **{names.get(n, n): v for n, v in kw.items()})
    assert torch.equal(ids, want_ids)
    # exponents are rounded (2^-24 of differences up to the logits' range, cut where the result
    # vanishes), exponentials, sums (up to 48 additions), quotients and the scale
    spread = min(200.0, 2 * float(z.float().nan_to_num(0.0, 0.0, 0.0).abs().max()))
    tol = (2 * spread + 64) * B.F32_HALF * want_w.abs() + 1e-37
    bad = (w.double() - want_w).abs() > tol
    assert not bool(bad.any()), (w[bad][:4], want_w[bad][:4])


SIZES = [(1, 1, 1), (3, 4, 4), (5, 31, 3), (7, 32, 8), (2, 33, 16), (48, 64, 6), (33, 60, 10),
         (9, 100, 7), (21, 128, 2), (6, 160, 9), (70, 256, 8), (3, 257, 5), (5, 512, 16),
         (4, 1000, 4), (6, 1024, 8)]


@pytest.mark.parametrize("rows,e,k", SIZES)
@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("bias", [True, False])
def test_sizes(lib, rows, e, k, score, dtype, bias):
    z = _rand(rows, e, seed=1, scale=2.0).to(dtype)
    b = _rand(e, seed=2, scale=0.3) if bias else None
    _check(lib, z, score, k, bias=b)
    _check(lib, z, score, k, pad=3, bias=b, renormalise=False, scale=2.5)


@pytest.mark.parametrize("e,groups,top,k", [
    (256, 8, 4, 8), (64, 4, 1, 5), (60, 4, 2, 10), (60, 20, 7, 9), (1024, 32, 3, 16),
    (32, 32, 5, 5),
    (160, 2, 1, 6), (96, 3, 2, 8), (6, 2, 1, 3), (512, 1, 1, 10), (62, 31, 30, 4), (8, 4, 4, 8)])
@pytest.mark.parametrize("of_best", [1, 2])
@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
@pytest.mark.parametrize("bias", [True, False])
def test_groups(lib, e, groups, top, k, of_best, score, bias):
    z = _rand(40, e, seed=3, scale=1.5)
    z[::3, ::5] = -math.inf
    z[1, :e // 2] = -math.inf
    b = _rand(e, seed=4, scale=0.3) if bias else None
    _check(lib, z, score, k, bias=b, groups=groups, top=top, of_best=of_best)


@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("bias", [None, "zero", "some"])
@pytest.mark.parametrize("grouped", [False, True])
def test_ties_go_to_the_lower_index(lib, score, dtype, bias, grouped):
    z = torch.randint(-3, 4, (64, 128), generator=torch.Generator().manual_seed(5)).float()
    z[z == 0] = torch.where(torch.arange(int((z == 0).sum())) % 2 == 0, 0.0, -0.0)
    z = z.to(dtype).cuda()
    z[7] = 1.0
    b = None if bias is None else torch.zeros(128, device="cuda")
    if bias == "some":
        b[::2] = 0.25
    kw = dict(groups=8, top=3, of_best=2) if grouped else {}
    _check(lib, z, score, 9, bias=b, **kw)


@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
@pytest.mark.parametrize("grouped", [False, True])
def test_scores_that_f32_cannot_tell_apart(lib, score, grouped):
    """Logits a step or a few of f32 apart, with a bias: decided as in f64."""
    z = torch.ones(200, 64).mul_(0.7) + torch.randn(
        200, 1, generator=torch.Generator().manual_seed(1))
    steps = torch.randint(0, 5, (200, 64), generator=torch.Generator().manual_seed(2))
    z = (z.float().view(torch.int32) + steps.int()).view(torch.float32).cuda()
    kw = dict(groups=4, top=2, of_best=2) if grouped else {}
    _check(lib, z, score, 6, bias=torch.zeros(64, device="cuda"), **kw)
    _check(lib, z, score, 6, bias=torch.full((64,), 0.5, device="cuda"), **kw)
    _check(lib, z, score, 6, **kw)


@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
@pytest.mark.parametrize("bias", [True, False])
@pytest.mark.parametrize("renormalise", [True, False])
def test_masks(lib, score, bias, renormalise):
    """Rows that a mask leaves nothing, one or few experts; not-a-number, infinities, the lowest
    value; biases that mask an expert."""
    z = _rand(12, 40, seed=6)
    z[0] = -math.inf
    z[1] = math.nan
    z[2, 1:] = -math.inf
    z[3, :38] = math.nan
    z[4, 7] = math.inf
    z[5, 3:5] = math.inf
    z[6] = LOWEST
    z[7, 5:] = LOWEST
    z[8] = math.inf
    z[9, ::2] = -math.inf
    z[9, 1::4] = math.nan
    b = _rand(40, seed=7, scale=0.1) if bias else None
    if bias:
        b[11], b[12] = -math.inf, math.nan
    _check(lib, z, score, 5, bias=b, renormalise=renormalise)
    _check(lib, z, score, 5, bias=b, renormalise=renormalise, groups=5, top=2, of_best=2)
    if bias:
        b[20] = math.inf
        _check(lib, z, score, 5, bias=b, renormalise=renormalise)


@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
@pytest.mark.parametrize("shift", [-300.0, -120.0, 60.0])
def test_far_logits_keep_their_proportions(lib, score, shift):
    z = _rand(9, 32, seed=8) + shift
    if score == "sigmoid" and shift > 0:
        z = z - 55
    _check(lib, z, score, 4)


@pytest.mark.parametrize("rows", [1, 4, 5, 4096])
def test_many_rows(lib, rows):
    _check(lib, _rand(rows, 16, seed=9, scale=1.5).to(BF), "softmax", 2)
    _check(lib, _rand(min(rows, 600), 256, seed=9, scale=1.5), "sigmoid", 8,
           bias=_rand(256, seed=10, scale=0.2), groups=8, top=4, of_best=2)


@pytest.mark.parametrize("count", [0, 1, 30, 50])
def test_count(lib, count):
    z = _rand(50, 24, seed=1)
    full = _route(lib, z, "softmax", 3)
    c = torch.tensor([count], dtype=torch.int32, device="cuda")
    ids, w = _route(lib, z, "softmax", 3, count=c)
    assert torch.equal(ids[:count], full[0][:count]) and torch.equal(w[:count], full[1][:count])
    assert bool((ids[count:] == -1).all()) and bool((w[count:] == 0).all())


@pytest.mark.parametrize("count", [-1, 51])
def test_bad_counts_are_reported(lib, count):
    R, ctx = lib
    z = _rand(50, 24, seed=1)
    c = torch.tensor([count], dtype=torch.int32, device="cuda")
    with pytest.raises(R.RCError) as e:
        _route(lib, z, "softmax", 3, count=c)
    assert e.value.status == 6
    ids = torch.zeros(50, 3, dtype=torch.int32, device="cuda")
    off, src, at = (torch.full((n,), 9, dtype=torch.int32, device="cuda") for n in (25, 150, 150))
    R.rc_experts_sort(ctx, ids, 50, 3, 24, c, off, src, at)
    with pytest.raises(R.RCError) as e:
        R.rc_sync(ctx)
    assert e.value.status == 6
    assert bool((off == 0).all()) and bool((src == 9).all()) and bool((at == -1).all())


def _sort(lib, ids, experts, count=None):
    R, ctx = lib
    rows, k = ids.shape
    off = torch.full((experts + 3,), -9, dtype=torch.int32, device="cuda")
    src = torch.full((rows * k + 2,), -9, dtype=torch.int32, device="cuda")
    at = torch.full((rows * k + 2,), -9, dtype=torch.int32, device="cuda")
    R.rc_experts_sort(ctx, ids.cuda(), rows, k, experts, count, off, src, at)
    torch.cuda.synchronize()
    assert bool((off[experts + 1:] == -9).all()) and bool((at[rows * k:] == -9).all())
    return off[:experts + 1].cpu(), src.cpu(), at[:rows * k].view(rows, k).cpu()


@pytest.mark.parametrize("rows,k,experts", [
    (0, 2, 8), (1, 1, 1), (1, 16, 1024), (3, 5, 7), (48, 6, 64), (341, 3, 1000), (512, 2, 4),
    (513, 2, 4), (700, 3, 33), (4128, 2, 16), (16384, 8, 256), (16387, 5, 1024), (40000, 1, 3)])
@pytest.mark.parametrize("lean", [0.0, 3.0])
def test_sort(lib, rows, k, experts, lean):
    """Even and very uneven experts, and pairs without one."""
    R, ctx = lib
    g = torch.Generator().manual_seed(rows + k)
    ids = (torch.rand(rows, k, generator=g) ** (1 + lean) * experts).int().clamp(max=experts - 1)
    ids[torch.rand(rows, k, generator=g) < 0.05] = -1
    off, src, at = _sort(lib, ids, experts)
    R.rc_sync(ctx)
    want = B.sort(ids, experts)
    n = len(want[1])
    assert torch.equal(off, want[0]) and torch.equal(at, want[2])
    assert torch.equal(src[:n], want[1]) and bool((src[n:] == -9).all())


@pytest.mark.parametrize("rows,count", [(300, 0), (300, 1), (300, 299), (3000, 1234), (3000, 3000)])
def test_sort_count(lib, rows, count):
    R, ctx = lib
    ids = torch.randint(0, 20, (rows, 4), dtype=torch.int32)
    off, src, at = _sort(lib, ids, 20, torch.tensor([count], dtype=torch.int32, device="cuda"))
    R.rc_sync(ctx)
    ids[count:] = -1
    want = B.sort(ids, 20)
    assert torch.equal(off, want[0]) and torch.equal(at, want[2])
    assert torch.equal(src[:4 * count], want[1]) and bool((src[4 * count:] == -9).all())


def test_sort_reports_bad_ids(lib):
    R, ctx = lib
    ids = torch.tensor([[0, 3], [2, 4], [2 ** 31 - 1, -2 ** 31]], dtype=torch.int32)
    off, src, at = _sort(lib, ids, 4)
    with pytest.raises(R.RCError) as e:
        R.rc_sync(ctx)
    assert e.value.status == 6
    want = B.sort(ids, 4)
    assert torch.equal(off, want[0]) and torch.equal(at, want[2])
    assert torch.equal(src[:3], want[1])


def test_captured(lib):
    """Routing and sorting in a graph whose logits change between replays."""
    R, ctx = lib
    z = _rand(2000, 64, seed=1)
    routing = R.Routing(64, 6)
    ids = torch.zeros(2000, 6, dtype=torch.int32, device="cuda")
    w = torch.zeros(2000, 6, device="cuda")
    off, src, at = (torch.zeros(n, dtype=torch.int32, device="cuda") for n in (65, 12000, 12000))

    def call():
        R.rc_experts_route(ctx, routing, z, 64, R.RC_F32, 2000, None, ids, w)
        R.rc_experts_sort(ctx, ids, 2000, 6, 64, None, off, src, at)

    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        call()
    for seed in (2, 3):
        z.copy_(_rand(2000, 64, seed=seed))
        g.replay()
        torch.cuda.synchronize()
        got = [t.clone() for t in (ids, w, off, src, at)]
        call()
        R.rc_sync(ctx)
        assert all(torch.equal(a, b) for a, b in zip(got, (ids, w, off, src, at)))
        want = B.sort(ids.cpu(), 64)
        assert torch.equal(off.cpu(), want[0]) and torch.equal(src.cpu(), want[1])


@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
@pytest.mark.parametrize("experts,groups", [(8, 4), (64, 8), (12, 4), (256, 32)])
@pytest.mark.parametrize("value", [LOWEST, -LOWEST])
def test_biases_at_the_ends_of_f32_mask_nothing(lib, score, experts, groups, value):
    """Two of them add up to more than f32 holds; beside them groups that are masked."""
    size = experts // groups
    z = _rand(30, experts, seed=11)
    z[3, :size] = -math.inf
    z[4, size:2 * size] = -math.inf
    z[5] = -math.inf
    z[6, 1::size] = -math.inf
    b = torch.full((experts,), value, device="cuda")
    b[:size] = 0.25
    for top in (1, 2, groups - 1):
        for of_best in (1, 2):
            _check(lib, z, score, min(16, 2 * size), bias=b, groups=groups, top=top,
                   of_best=of_best)


@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
@pytest.mark.parametrize("grouped", [False, True])
@pytest.mark.parametrize("equal", [2, 3])
@pytest.mark.parametrize("steps", [1, 2])
def test_equal_experts_at_the_last_choice_hide_no_better_one(lib, score, grouped, equal, steps):
    """Experts of one logit for the last place, and one a step of f32 above them behind."""
    a = -0.5 - 6 * torch.rand(500, generator=torch.Generator().manual_seed(3))
    z = torch.full((500, 12), -20.0)
    z[:, 0] = 0.0
    z[:, 1:1 + equal] = a[:, None]
    z[:, 4] = (a.view(torch.int32) - steps).view(torch.float32)  # (towards zero)
    kw = dict(groups=3, top=2, of_best=1) if grouped else {}
    if grouped:  # (groups of three lanes: the general way)
        z = z[:, :9]
    assert bool((z[:, 4] > a).all())
    _check(lib, z.contiguous().cuda(), score, 2, bias=torch.zeros(z.shape[1], device="cuda"), **kw)
