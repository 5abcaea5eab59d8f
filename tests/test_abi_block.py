"""The structures of a block's row work and rotary positions match the header,
their wrappers check what they hold, bad arguments are refused before anything
is launched, and rotary plans hold their frequencies.  CPU only: no call here
reaches the GPU."""
import ctypes as C
import math
import os
import subprocess
import tempfile

import pytest
import torch

from tests import block_ref as B

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def R():
    from paper_2608_29809_gb300 import build
    build.build()
    from paper_2608_29809_gb300 import regioncache
    return regioncache


def test_structures_match_the_header(R):
    structs = (R.rc_norm, R.rc_residual, R.rc_rotary_spec, R.rc_rotary, R.rc_routing)
    lines = ["#include <stdio.h>", "#include <stddef.h>", '#include "regioncache.h"',
             "int main(void) {"]
    for s in structs:
        for f, _ in s._fields_:
            lines.append('printf("%%zu ", offsetof(%s, %s));' % (s.__name__, f))
        lines.append('printf("%%zu ", sizeof(%s));' % s.__name__)
    with tempfile.TemporaryDirectory(dir=os.path.join(ROOT, "tests")) as tmp:
        src, exe = os.path.join(tmp, "s.c"), os.path.join(tmp, "s")
        with open(src, "w") as f:
            f.write("\n".join(lines + ["return 0;", "}"]))
        subprocess.run(["gcc", "-std=c11", "-I", os.path.join(ROOT, "include"), src, "-o", exe],
                       check=True)
        out = subprocess.run([exe], check=True, capture_output=True, text=True).stdout.split()
    want = []
    for s in structs:
        want += [getattr(s, f).offset for f, _ in s._fields_] + [C.sizeof(s)]
    assert [int(v) for v in out] == want


# Checked before the context is looked at beyond its being there (nothing is dereferenced).
CTX = C.c_void_p(4096)
A, ODD = 1 << 20, (1 << 20) + 1


def _norm(R, kind=0, eps=0.0, weight=None, bias=None):
    return R.rc_norm(kind, eps, weight, bias)


def _residual(R, **kw):
    a = dict(rows=8, cols=256, n_items=1, top_k=0, row_offsets=None, x=A, x_out=A, h=A,
             places=None, weights=None, gate=None, scale=None, shift=None, y=A, y8=None, x_type=0,
             ldx=256, ldx_out=256, h_type=0, ldh=256, h_rows=8, ld_mod=256, y_type=0, ldy=256,
             residual_scale=1.0, post=_norm(R), pre=_norm(R))
    a.update(kw)
    return R.rc_residual(*[a[f] for f, _ in R.rc_residual._fields_])


def _codes(R, **kw):
    a = dict(codes=A, scales=A, rows=8, cols=256, ld=256, lds=8, group=1)
    a.update(kw)
    return C.pointer(R.rc_fp8(*[a[f] for f, _ in R.rc_fp8._fields_]))


def test_norm_residual_refusals(R):
    def call(ctx=CTX, **kw):
        return R._lib.rc_norm_residual(ctx, C.byref(_residual(R, **kw)), None)

    assert call(ctx=None) == 1 and R._lib.rc_norm_residual(CTX, None, None) == 1
    for kw in (dict(rows=-1), dict(cols=0), dict(cols=R.RC_NORM_MAX_COLS + 1), dict(n_items=0),
               dict(top_k=-1), dict(top_k=R.RC_EXPERTS_MAX_TOP_K + 1), dict(ldx=255),
               dict(ldx_out=255, x=None), dict(ldh=255), dict(ldy=255), dict(ldx=264),
               dict(top_k=2, places=A, weights=A, h_rows=-1),
               dict(n_items=2, row_offsets=A, gate=A, ld_mod=255),
               dict(y=None, y8=_codes(R, rows=7, lds=7)), dict(y=None, y8=_codes(R, cols=255)),
               dict(y=None, y8=_codes(R, group=128))):
        assert call(**kw) == 2, kw
    for kw in (dict(n_items=2), dict(x_out=None, y=None), dict(y8=_codes(R)), dict(x_type=2),
               dict(h_type=-1), dict(y_type=2), dict(x=ODD), dict(x=A + 2, x_type=1),
               dict(x_out=ODD), dict(h=ODD), dict(y=ODD), dict(y=A + 2, y_type=1),
               dict(top_k=2), dict(top_k=2, places=A), dict(top_k=2, weights=A),
               dict(h=None, top_k=2), dict(h=None, gate=A), dict(h=None, post=_norm(R, 2)),
               dict(gate=A + 2), dict(scale=ODD), dict(shift=A + 1), dict(row_offsets=A + 2),
               dict(top_k=1, places=A + 2, weights=A), dict(top_k=1, places=A, weights=A + 2),
               dict(residual_scale=math.nan), dict(residual_scale=math.inf),
               dict(pre=_norm(R, 3)), dict(pre=_norm(R, -1)), dict(pre=_norm(R, 1, -1.0)),
               dict(post=_norm(R, 1, math.nan)), dict(pre=_norm(R, 0, 0.0, A)),
               dict(pre=_norm(R, 0, 0.0, None, A)), dict(post=_norm(R, 2, 0.0, A + 2)),
               dict(y=None, y8=_codes(R, codes=A + 8))):
        assert call(**kw) == 1, kw
    assert call(rows=0) == 0


def test_rotary_plan_refusals(R):
    def call(rot=64, first=0, layout=0, axes=1, pairs=(32, 0, 0), scaling=0, theta=1e4,
             factor=2.0, native=4096.0, fast=4.0, slow=1.0, amplitude=1.0):
        s = R.rc_rotary_spec(rot, first, layout, axes, (C.c_int * 3)(*pairs), scaling, theta,
                             factor, native, fast, slow, amplitude)
        return R._lib.rc_rotary_plan(C.byref(s), C.byref(R.rc_rotary()))

    assert call() == 0
    assert R._lib.rc_rotary_plan(None, C.byref(R.rc_rotary())) == 1
    assert R._lib.rc_rotary_plan(C.byref(R.rc_rotary_spec()), None) == 1
    for kw in (dict(rot=0), dict(rot=63), dict(rot=258, pairs=(129, 0, 0)), dict(axes=0),
               dict(axes=4), dict(pairs=(31, 0, 0)), dict(axes=2), dict(axes=2, pairs=(33, -1, 0)),
               dict(axes=3, pairs=(2 ** 31 - 1, 2 ** 31 - 1, 34)), dict(first=-1),
               dict(first=R.RC_ROTARY_MAX_HEAD - 63), dict(first=2 ** 31 - 1)):
        assert call(**kw) == 2, kw
    for kw in (dict(layout=2), dict(layout=-1), dict(scaling=5), dict(scaling=-1), dict(theta=0.0),
               dict(theta=-2.0), dict(theta=math.nan), dict(theta=math.inf),
               dict(amplitude=math.inf), dict(amplitude=1e300), dict(scaling=1, factor=0.5),
               dict(scaling=1, factor=math.nan), dict(scaling=3, native=0.0),
               dict(scaling=3, slow=0.0), dict(scaling=3, fast=1.0), dict(scaling=4, fast=0.5),
               dict(scaling=4, theta=1.0), dict(scaling=3, fast=math.inf)):
        assert call(**kw) == 1, kw


@pytest.mark.parametrize("scaling", ["plain", "linear", "base", "bands", "ramp"])
@pytest.mark.parametrize("pairs,theta", [([64], 1e4), ([18, 18], 100.0), ([1], 1e4),
                                         ([5, 1, 10], 5e5)])
def test_rotary_plan_holds_its_frequencies(R, scaling, pairs, theta):
    kind = getattr(R, "RC_ROTARY_" + scaling.upper())
    p = R.Rotary(2 * sum(pairs), theta, pairs=pairs, scaling=kind, factor=4.0,
                 native_length=4096.0, fast=8.0, slow=1.0, amplitude=1.5)
    f, axis = B.frequencies(pairs, theta, scaling, 4.0, 4096.0, 8.0, 1.0)
    assert p.c.axes == len(pairs) and p.c.amplitude == 1.5
    for i, v in enumerate(f):
        want = v / (2 * math.pi)
        # a few roundings of f64 (powers and quotients) and the last place of 2^-64
        assert abs(p.c.turns[i] / 2.0 ** 64 - want) <= 16 * 2.0 ** -53 * want + 2.0 ** -63


def test_rotary_apply_refusals(R):
    plan = R.Rotary(64, first=8)

    def call(ctx=CTX, p=plan, x=A, ldx=192, type=0, rows=4, heads=2, dh=96, pos=None, count=None,
             y=A, ldy=192):
        return R._lib.rc_rotary_apply(ctx, p, x, ldx, type, rows, heads, dh, pos, count, 0, y,
                                      ldy, None)

    assert call(ctx=None) == 1 and call(p=None) == 1
    for kw in (dict(rows=-1), dict(heads=-1), dict(dh=71), dict(dh=1025), dict(ldx=191),
               dict(ldy=191), dict(ldy=200), dict(heads=2 ** 26, dh=96)):
        assert call(**kw) == 2, kw
    for kw in (dict(x=None), dict(y=None), dict(x=ODD), dict(y=ODD), dict(x=A + 2, type=1),
               dict(type=2), dict(pos=A + 2), dict(count=A + 1)):
        assert call(**kw) == 1, kw
    bad = R.Rotary(64)
    bad.c.rot = 62
    assert call(p=bad) == 2
    bad.c.rot, bad.c.layout = 64, 7
    assert call(p=bad) == 1
    assert call(rows=0, x=None, y=None) == 0 and call(heads=0, x=None, y=None) == 0


def test_route_refusals(R):
    def call(ctx=CTX, z=A, ld=64, type=0, rows=4, count=None, ids=A, w=A, **kw):
        a = dict(experts=64, top_k=2, score=0, groups=4, top_groups=2, group_best=1,
                 renormalise=1, scale=1.0, bias=None)
        a.update(kw)
        r = R.rc_routing(*[a[f] for f, _ in R.rc_routing._fields_])
        return R._lib.rc_experts_route(ctx, C.byref(r), z, ld, type, rows, count, ids, w, None)

    assert call(ctx=None) == 1
    assert R._lib.rc_experts_route(CTX, None, A, 64, 0, 4, None, A, A, None) == 1
    for kw in (dict(rows=-1), dict(experts=0), dict(experts=1025, ld=1025), dict(top_k=0),
               dict(top_k=17), dict(ld=63), dict(groups=0), dict(groups=3), dict(groups=64),
               dict(top_groups=0), dict(top_groups=5)):
        assert call(**kw) == 2, kw
    for kw in (dict(group_best=0), dict(group_best=3), dict(score=2), dict(score=-1),
               dict(scale=math.nan), dict(type=2), dict(z=ODD), dict(z=A + 2, type=1),
               dict(bias=A + 2), dict(count=A + 2), dict(ids=A + 2), dict(w=ODD), dict(z=None),
               dict(ids=None), dict(w=None)):
        assert call(**kw) == 1, kw
    assert call(rows=0, z=None, ids=None, w=None) == 0
    with pytest.raises(ValueError):
        R.Routing(8, 2, bias=torch.zeros(7))
    with pytest.raises(ValueError):
        R.Routing(8, 2, bias=torch.zeros(8, dtype=torch.double))


def test_sort_refusals(R):
    def call(ctx=CTX, ids=A, rows=4, k=2, e=8, count=None, off=A, src=A, at=A):
        return R._lib.rc_experts_sort(ctx, ids, rows, k, e, count, off, src, at, None)

    assert call(ctx=None) == 1
    for kw in (dict(rows=-1), dict(k=0), dict(k=17), dict(e=0), dict(e=1025),
               dict(rows=2 ** 30, k=2)):
        assert call(**kw) == 2, kw
    for kw in (dict(ids=None), dict(off=None), dict(src=None), dict(at=None), dict(ids=A + 2),
               dict(count=A + 1), dict(off=A + 2), dict(src=ODD), dict(at=A + 3)):
        assert call(**kw) == 1, kw


def _matrix(R, **kw):
    a = dict(codes=A, scales=A, rows=8, cols=256, ld=256, lds=2 ** 20, group=1)
    a.update(kw)
    return C.pointer(R.rc_fp8(*[a[f] for f, _ in R.rc_fp8._fields_]))


def test_experts_linear_refusals(R):
    def call(ctx=CTX, x=0, W=0, b=None, experts=3, n=200, off=A, src=None, pairs=8, act=0, y=A,
             ldy=200, type=0, y8=None):
        x = _matrix(R) if x == 0 else x
        W = _matrix(R, rows=768, group=128) if W == 0 else W
        return R._lib.rc_experts_linear(ctx, x, W, b, experts, n, off, src, pairs, act, y, ldy,
                                        type, y8, None)

    assert call(ctx=None) == 1 and call(x=None) == 1 and call(W=None) == 1
    for kw in (dict(x=_matrix(R, ld=248)), dict(W=_matrix(R, rows=768, group=128, lds=5)),
               dict(experts=0), dict(experts=1025), dict(n=0), dict(pairs=-1),
               dict(pairs=2 ** 30 + 1), dict(n=257, ldy=257), dict(act=3), dict(experts=4),
               dict(x=_matrix(R, cols=255)), dict(W=_matrix(R, rows=0, group=128)),
               dict(x=_matrix(R, rows=7)), dict(x=_matrix(R, rows=0, codes=None), src=A),
               dict(ldy=199), dict(y=None, y8=_matrix(R, rows=7, cols=200)),
               dict(y=None, y8=_matrix(R, cols=199)),
               dict(y=None, y8=_matrix(R, cols=200, group=128)),
               dict(x=_matrix(R, rows=2 ** 30, lds=2 ** 30), pairs=2 ** 30, experts=1, n=8192,
                    ldy=8192, W=_matrix(R, rows=8192, group=128))):
        assert call(**kw) == 2, kw
    for kw in (dict(x=_matrix(R, group=128)), dict(W=_matrix(R, rows=768)), dict(act=4),
               dict(act=-1), dict(y8=_matrix(R, cols=200)), dict(y=None), dict(off=None),
               dict(type=2), dict(y=ODD), dict(y=A + 2, type=1), dict(b=A + 2), dict(off=A + 2),
               dict(src=A + 1), dict(x=_matrix(R, codes=A + 8)), dict(x=_matrix(R, scales=None)),
               dict(W=_matrix(R, rows=768, group=128, codes=None))):
        assert call(**kw) == 1, kw
    assert call(pairs=0, off=None, y=None) == 0


def test_wrappers_refuse_tensors_that_do_not_fit(R):
    x = torch.zeros(6, 40)
    h = torch.zeros(6, 40, dtype=torch.bfloat16)
    ids, w = torch.zeros(6, 2, dtype=torch.int32), torch.zeros(6, 2)
    op = R.ResidualNorm(40, x=x, h=h, x_out=x, y=h, pre=R.Norm(R.RC_NORM_RMS, 1e-6, x[0]))
    assert (op.c.rows, op.c.cols, op.c.n_items, op.c.x_type, op.c.h_type) == (6, 40, 1, 1, 0)
    wide = torch.zeros(2, 120)
    op = R.ResidualNorm(40, x=x[:, :], y=x, gate=None, scale=wide[:, :40], shift=wide[:, 40:80],
                        row_offsets=torch.tensor([0, 2, 6], dtype=torch.int32))
    assert (op.c.n_items, op.c.ld_mod) == (2, 120)
    op = R.ResidualNorm(40, x=x, h=torch.zeros(9, 40), places=ids, weights=w, x_out=x)
    assert (op.c.rows, op.c.top_k, op.c.h_rows) == (6, 2, 9)
    off = torch.tensor([0, 2, 6], dtype=torch.int32)
    for kw in (dict(x=x[:5], y=x), dict(x=x.t(), y=x), dict(x=x.half(), y=x), dict(x=x, x_out=h),
               dict(x=x, h=h, places=ids), dict(x=x, places=ids, weights=w, y=x),
               dict(x=x, h=h, places=ids.long(), weights=w, y=x),
               dict(x=x, h=h, places=ids[:5], weights=w[:5], y=x),
               dict(x=x, y=x, scale=x[:2]), dict(x=x, y=x, scale=x[0]),
               dict(x=x, y=x, scale=wide[:, :39], row_offsets=off),
               dict(x=x, y=x, scale=wide[:, :40], shift=x[:2], row_offsets=off),
               dict(x=x, y=x, row_offsets=off.long()), dict(x=x, y=x, row_offsets=off[:1]),
               dict(x=x, y=x, pre=R.Norm(1, 0.0, x[0].double())),
               dict(x=x, y=x, pre=R.Norm(1, 0.0, x[0, :39])),
               dict(x=x, y=R.Fp8Matrix(5, 40, 1, device="cpu")),
               dict(x=x, y=R.Fp8Matrix(6, 39, 1, device="cpu")),
               dict(x=x, y=R.Fp8Matrix(6, 40, 128, device="cpu")),
               dict(x=x, y=x.to("meta"))):
        with pytest.raises(ValueError):
            R.ResidualNorm(40, **kw)
    with pytest.raises(R.RCError):
        R.Rotary(63)
    with pytest.raises(ValueError):
        R.Rotary(64, pairs=[8, 8, 8, 8])


@pytest.mark.parametrize("rot,theta,native,fast", [
    (128, 1e4, 4096.0, 32.0), (128, 1e4, 131072.0, 32.0), (36, 100.0, 4096.0, 64.0),
    (64, 10.0, 65536.0, 4096.0), (2, 1e4, 4096.0, 8.0), (2, 2.0, 4096.0, 8.0),
    (128, 5e5, 8192.0, 4.0)])
def test_ramp_of_one_axis_is_the_published_one(R, rot, theta, native, fast):
    """YaRN's: from the channel pair that turns `fast` times over the native length, rounded down,
    to the one that turns once, rounded up, between 0 and the turned channels less one, which may
    lie behind the last pair."""
    p = R.Rotary(rot, theta, scaling=R.RC_ROTARY_RAMP, factor=8.0, native_length=native, fast=fast,
                 slow=1.0)

    def dim(turns):
        return rot * math.log(native / (turns * 2 * math.pi)) / (2 * math.log(theta))

    lo, hi = max(math.floor(dim(fast)), 0), min(math.ceil(dim(1.0)), rot - 1)
    for i in range(rot // 2):
        f = theta ** (-2 * i / rot)
        stretched = min(max((i - lo) / (hi - lo if hi > lo else 0.001), 0.0), 1.0)
        want = (f / 8.0 * stretched + f * (1 - stretched)) / (2 * math.pi)
        # a few roundings of f64 (powers and quotients) and the last place of 2^-64
        assert abs(p.c.turns[i] / 2.0 ** 64 - want) <= 32 * 2.0 ** -53 * want + 2.0 ** -63
