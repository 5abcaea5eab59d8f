"""The README's Python example runs as it stands, and gives what its calls define."""
import os
import re

import pytest
import torch

from paper_2608_29809_gb300 import synth
from tests import eight_bit_ref as E

pytestmark = pytest.mark.gpu
README = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "README.md")


def _ints(v):
    return torch.tensor(v, dtype=torch.int32, device="cuda")


def test_the_example_runs():
    from paper_2608_29809_gb300 import build as B
    B.build()
    from paper_2608_29809_gb300 import regioncache as R
    code = re.search(r"```python\n(.*?)```", open(README).read(), re.S).group(1)
    d = synth.Dims(hidden=128, heads=2, mlp=128, layers=1, grid_h=4, grid_w=4, timesteps=1)
    ctx = R.rc_create(R.dims_struct(d))

    def rand(*shape, seed):
        return synth.randn(shape, synth.tensor_seed(seed, *shape), "cuda", 1.0, torch.bfloat16)

    lens, dirty, blocks, width = [130, 64], [5, 2], 6, 4
    rows, n = sum(dirty), 2
    table = torch.zeros(n, width, dtype=torch.int32)
    table[0, :3], table[1, 0] = torch.tensor([4, 0, 2], dtype=torch.int32), 5
    names = dict(
        rows=rows, blocks=blocks, ctx=ctx, n=n, width=width, max_rows=max(dirty),
        w=rand(3456, 1152, seed=1) * 0.03, x=rand(rows, 1152, seed=2),
        bias=rand(3456, seed=3).float(), lengths=_ints(lens), counts=_ints(dirty),
        qkv=torch.zeros(rows, 3456, dtype=torch.bfloat16, device="cuda"),
        positions=_ints([0, 63, 64, 65, 129, 7, 8]), table=table.cuda(),
        offsets=_ints([0] * (n + 1)), slots=_ints([0] * rows), used=_ints([0]),
        out=torch.zeros(rows, 1152, dtype=torch.bfloat16, device="cuda"))
    try:
        exec(code, names)
        R.rc_sync(ctx)
        assert names["offsets"].tolist() == [0, 5, 7]
        assert names["slots"].tolist() == [4 * 64, 4 * 64 + 63, 0, 1, 2 * 64 + 1, 5 * 64 + 7,
                                           5 * 64 + 8]
        x8, w8, pool, qkv = names["x8"], names["w8"], names["pool"], names["qkv"].double().cpu()
        xv, wv = E.values(x8.codes, x8.scales, 1, 1152), E.values(w8.codes, w8.scales, 128, 1152)
        want = xv @ wv.t() + names["bias"].double().cpu()
        # the result rounded to bf16, and 1152 additions in f32
        tol = 2.0 ** -8 * want.abs() + 1.01 * 1153 * 2.0 ** -23 * (
            xv.abs() @ wv.abs().t() + names["bias"].double().cpu().abs())
        assert bool(((qkv - want).abs() <= tol).all())
        k, v = E.cache_values(pool.k, pool.k_scale), E.cache_values(pool.v, pool.v_scale)
        out = names["out"].double().cpu()
        for r, (l, a, b) in enumerate(zip(lens, [0, 5], [5, 7])):
            pages = table[r, :-(-l // 64)].long()
            for h in range(16):
                cols = slice(72 * h, 72 * h + 72)
                o, pv, reach = E.attention(qkv[a:b, cols], k[pages, h].reshape(-1, 72)[:l],
                                           v[pages, h].reshape(-1, 72)[:l], False)
                assert bool(((out[a:b, cols] - o).abs() <=
                             E.attention_tolerance(o, pv, reach, 72)).all())
    finally:
        R.rc_destroy(ctx)
