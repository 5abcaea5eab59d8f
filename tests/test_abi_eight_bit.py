"""The structures of eight-bit serving match the header, their wrappers hold
what they name, and bad arguments are refused before anything is launched.
CPU only: no call here reaches the GPU."""
import ctypes as C
import os
import subprocess
import tempfile

import pytest
import torch

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def R():
    from paper_2608_29809_gb300 import build as B
    B.build()
    from paper_2608_29809_gb300 import regioncache
    return regioncache


def test_structures_match_the_header(R):
    lines = ["#include <stdio.h>", "#include <stddef.h>", '#include "regioncache.h"',
             "int main(void) {"]
    for s in (R.rc_fp8, R.rc_kv8):
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
    for s in (R.rc_fp8, R.rc_kv8):
        want += [getattr(s, f).offset for f, _ in s._fields_] + [C.sizeof(s)]
    assert [int(v) for v in out] == want
    assert (R.RC_BF16, R.RC_F32, R.RC_KV8_BLOCK) == (0, 1, 64)


def test_answers_of_devices_are_kept_apart():
    """What one device answered is no other's answer, and a failure is not kept."""
    source = r"""
#include <stdio.h>
#include "per_device.h"
static rc::PerDevice<9> known;
static int asked = 0;
static void show(int device, int kind, int answer) {
  printf("%d ", known.get(device, kind, [&] { ++asked; return answer; }));
}
int main() {
  show(0, 8, -1);  // fails: asked again
  show(0, 8, 19);
  show(0, 8, 5);   // kept
  show(1, 8, 12);  // another device's
  show(1, 8, 7);
  show(0, 7, 0);   // another question's (0 is an answer)
  show(0, 7, 3);
  show(-1, 8, 4);  // devices beyond those kept
  show(64, 8, 6);
  show(0, 8, 1);
  show(63, 0, 2);
  printf("%d\n", asked);
  return 0;
}
"""
    with tempfile.TemporaryDirectory(dir=os.path.join(ROOT, "tests")) as tmp:
        src, exe = os.path.join(tmp, "d.cpp"), os.path.join(tmp, "d")
        with open(src, "w") as f:
            f.write(source)
        subprocess.run(["g++", "-std=c++17", "-Wall", "-Werror", "-I",
                        os.path.join(ROOT, "paper_2608_29809_gb300", "csrc"), src, "-o", exe],
                       check=True)
        out = subprocess.run([exe], check=True, capture_output=True, text=True).stdout.split()
    assert [int(v) for v in out] == [-1, 19, 19, 12, 12, 0, 0, 4, 6, 19, 2, 7]


def test_wrappers(R):
    m = R.Fp8Matrix(130, 300, 128, device="cpu")
    assert m.codes.shape == (130, 304) and m.scales.shape == (3, 2)
    assert (m.c.rows, m.c.cols, m.c.ld, m.c.lds, m.c.group) == (130, 300, 304, 2, 128)
    m.codes.fill_(0x38)  # 1.0
    m.scales.fill_(128)
    m.scales[2, 1] = 255
    v = m.values()
    assert v.shape == (130, 300) and bool((v[:128] == 2).all()) and bool(v[128:, 256:].isnan().all())
    with pytest.raises(ValueError):
        R.Fp8Matrix.of(m.codes.t(), m.scales, 130, 1)
    with pytest.raises(ValueError):
        R.Fp8Matrix.of(m.codes.float(), m.scales, 300, 1)
    p = R.Kv8Pool(3, 2, 72, device="cpu")
    assert p.k.shape == (3, 2, 64, 72) and (p.c.blocks, p.c.kv_heads, p.c.head_dim) == (3, 2, 72)
    with pytest.raises(ValueError):
        R.Kv8Pool.of(p.k, p.v[:2], p.k_scale, p.v_scale)
    with pytest.raises(ValueError):
        R.Kv8Pool.of(p.k[:, :, :32].contiguous(), p.v[:, :, :32].contiguous(), p.k_scale,
                     p.v_scale)


# The entry points check everything below before they look at the context
# beyond its being there (nothing is dereferenced).
CTX = C.c_void_p(4096)
A, ODD = 1 << 20, (1 << 20) + 1


def _mat(R, **kw):
    a = dict(codes=A, scales=A, rows=8, cols=256, ld=256, lds=8, group=1)
    a.update(kw)
    return C.byref(R.rc_fp8(*[a[f] for f, _ in R.rc_fp8._fields_]))


BAD_MATRIX = [(dict(rows=-1), 2), (dict(rows=2 ** 30 + 1, lds=2 ** 31 - 1), 2), (dict(cols=0), 2),
              (dict(cols=4194305, ld=4194320), 2),
              (dict(group=64), 1), (dict(ld=248), 2), (dict(ld=260), 2), (dict(lds=7), 2),
              (dict(codes=None), 1), (dict(scales=None), 1), (dict(codes=A + 8), 1)]


@pytest.mark.parametrize("kw,status", BAD_MATRIX)
def test_matrix_refusals(R, kw, status):
    lib = R._lib
    assert lib.rc_fp8_quantize(CTX, A, 5000000, 0, _mat(R, **kw), None) == status
    assert "rc_fp8_quantize" in R.rc_last_error()
    assert lib.rc_fp8_linear(CTX, _mat(R, **kw), _mat(R), None, A, 64, 0, None) == status
    assert lib.rc_fp8_linear(CTX, _mat(R), _mat(R, **kw), None, A, 64, 0, None) == status


def test_quantize_and_linear_refusals(R):
    lib = R._lib
    assert lib.rc_fp8_quantize(None, A, 256, 0, _mat(R), None) == 1
    assert lib.rc_fp8_quantize(CTX, A, 256, 0, None, None) == 1
    assert lib.rc_fp8_quantize(CTX, None, 256, 0, _mat(R), None) == 1
    assert lib.rc_fp8_quantize(CTX, A, 255, 0, _mat(R), None) == 2
    assert lib.rc_fp8_quantize(CTX, A, 256, 2, _mat(R), None) == 1
    assert lib.rc_fp8_quantize(CTX, ODD, 256, 0, _mat(R), None) == 1
    assert lib.rc_fp8_quantize(CTX, A + 2, 256, 1, _mat(R), None) == 1
    assert lib.rc_fp8_quantize(CTX, None, 256, 0, _mat(R, rows=0), None) == 0

    def lin(x=None, w=None, b=None, y=A, ldy=8, type=0, ctx=CTX):
        return lib.rc_fp8_linear(ctx, x or _mat(R), w or _mat(R), b, y, ldy, type, None)

    assert lin(ctx=None) == 1
    assert lib.rc_fp8_linear(CTX, None, _mat(R), None, A, 8, 0, None) == 1
    assert lib.rc_fp8_linear(CTX, _mat(R), None, None, A, 8, 0, None) == 1
    assert lin(w=_mat(R, cols=255)) == 2
    assert lin(w=_mat(R, rows=0)) == 2
    assert lin(ldy=7) == 2
    assert lin(type=-1) == 1
    assert lin(y=None) == 1
    assert lin(y=ODD) == 1 and lin(y=A + 2, type=1) == 1 and lin(b=A + 2) == 1
    assert lin(x=_mat(R, rows=0), y=None) == 0


def test_tables_refusals(R):
    lib = R._lib

    def call(lengths=A, counts=A, positions=None, n=3, free=None, n_free=4, table=A, ld=2, off=A,
             slots=A, n_slots=5, used=A, ctx=CTX):
        return lib.rc_kv8_tables(ctx, lengths, counts, positions, n, free, n_free, table, ld, off,
                                 slots, n_slots, used, None)

    assert call(ctx=None) == 1
    for name in ("lengths", "table", "off", "slots", "used"):
        assert call(**{name: None}) == 1
        assert call(**{name: A + 2}) == 1
    assert call(positions=A + 1) == 1 and call(free=A + 2) == 1 and call(counts=A + 3) == 1
    for kw in (dict(n=0), dict(n=4097), dict(n_free=-1), dict(n_free=2 ** 26), dict(ld=0),
               dict(ld=2 ** 26), dict(n_slots=-1), dict(n_slots=2 ** 30 + 1)):
        assert call(**kw) == 2, kw


def _pool(R, **kw):
    a = dict(k=A, v=A, k_scale=A, v_scale=A, blocks=4, kv_heads=2, head_dim=72)
    a.update(kw)
    return C.byref(R.rc_kv8(*[a[f] for f, _ in R.rc_kv8._fields_]))


@pytest.mark.parametrize("kw,status", [
    (dict(k=None), 1), (dict(v=None), 1), (dict(k_scale=None), 1), (dict(v_scale=None), 1),
    (dict(k=A + 8), 1), (dict(v=A + 4), 1), (dict(blocks=0), 2), (dict(blocks=2 ** 25), 2),
    (dict(kv_heads=0), 2), (dict(kv_heads=1025), 2), (dict(head_dim=80), 2)])
def test_pool_refusals(R, kw, status):
    lib = R._lib
    assert lib.rc_kv8_store(CTX, _pool(R, **kw), A, A, 10 ** 6, 0, A, 3, None, 0, None) == status
    assert lib.rc_kv8_attention(CTX, _pool(R, **kw), A, 10 ** 6, 3, A, A, 1, 3, A, 2, 2, 0, A,
                                10 ** 6, None) == status


def test_store_refusals(R):
    def call(pool=None, k=A, v=A, ld=144, type=0, slots=A, n=3, count=None, mode=0, ctx=CTX):
        return R._lib.rc_kv8_store(ctx, pool or _pool(R), k, v, ld, type, slots, n, count, mode,
                                   None)

    assert call(ctx=None) == 1
    assert R._lib.rc_kv8_store(CTX, None, A, A, 144, 0, A, 3, None, 0, None) == 1
    assert call(type=2) == 1 and call(mode=2) == 1 and call(mode=-1) == 1
    assert call(n=-1) == 2 and call(ld=143) == 2
    assert call(k=None) == 1 and call(v=None) == 1 and call(slots=None) == 1
    assert call(k=ODD) == 1 and call(v=A + 2, type=1) == 1 and call(slots=A + 2) == 1
    assert call(count=A + 1) == 1
    assert call(n=0, k=None, v=None, slots=None) == 0


def test_attention_refusals(R):
    def call(q=A, ldq=288, rows=5, off=A, lens=A, n=2, max_q=3, table=A, ldt=4, heads=4, causal=0,
             o=A, ldo=288, ctx=CTX):
        return R._lib.rc_kv8_attention(ctx, _pool(R), q, ldq, rows, off, lens, n, max_q, table,
                                       ldt, heads, causal, o, ldo, None)

    assert call(ctx=None) == 1
    assert R._lib.rc_kv8_attention(CTX, None, A, 288, 5, A, A, 2, 3, A, 4, 4, 0, A, 288, None) == 1
    for kw in (dict(heads=3), dict(heads=0), dict(heads=34, ldq=9999 // 8 * 8, ldo=9992),
               dict(ldq=280), dict(ldo=280), dict(ldq=290), dict(ldo=292), dict(rows=-1),
               dict(max_q=-1), dict(n=-1), dict(n=4097), dict(ldt=0), dict(ldt=2 ** 26),
               dict(rows=2 ** 30 + 1)):
        assert call(**kw) == 2, kw
    for name in ("q", "off", "lens", "table", "o"):
        assert call(**{name: None}) == 1
        assert call(**{name: A + 2}) == 1
    assert call(q=A + 8) == 1 and call(o=A + 8) == 1
    for kw in (dict(rows=0), dict(max_q=0), dict(n=0)):
        assert call(q=None, o=None, **kw) == 0


def test_a_matrix_names_no_more_than_its_tensors_hold(R):
    """What the structure says is read and written by the kernels: tensors that hold less (or lie
    elsewhere) are refused where they are named."""
    def u8(*shape):
        return torch.zeros(*shape, dtype=torch.uint8)

    for group, wide in ((1, 130), (128, 2)):
        assert R.Fp8Matrix.of(u8(130, 304), u8(3, wide), 300, group).c.lds == wide
        assert R.Fp8Matrix.of(u8(130, 320)[:, :304], u8(4, wide + 6)[:, :wide], 300, group).c.lds \
            == wide + 6
        for codes, scales, cols in (
                (u8(130, 304), u8(2, wide), 300),                   # a block of columns short
                (u8(130, 304), u8(0, wide), 300),
                (u8(130, 304), u8(3, wide - 1), 300),               # a block of rows short
                (u8(130, 304), u8(3, wide + 6)[:, :wide - 1], 300),  # .. as the last row's are
                (u8(130, 288), u8(3, wide), 300),                   # columns short
                (u8(130, 320)[:, :288], u8(3, wide), 300),
                (u8(1, 288), u8(3, 1), 300),
                (u8(130, 304), u8(3, wide), 0),
                (u8(130, 304), u8(3, wide).to("meta"), 300)):
            with pytest.raises(ValueError):
                R.Fp8Matrix.of(codes, scales, cols, group)
    for group in (0, 2, -128):
        with pytest.raises(ValueError):
            R.Fp8Matrix.of(u8(130, 304), u8(3, 130), 300, group)
    assert R.Fp8Matrix.of(u8(0, 304), u8(3, 0), 300, 1).c.rows == 0
    p = R.Kv8Pool(3, 2, 72, device="cpu")
    with pytest.raises(ValueError):
        R.Kv8Pool.of(p.k, p.v.to("meta"), p.k_scale, p.v_scale)
    with pytest.raises(ValueError):
        R.Kv8Pool.of(p.k, p.v, p.k_scale, p.k_scale[:, :1].contiguous())
