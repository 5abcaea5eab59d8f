"""The first calls of a process, each of its kernels' first launch, captured into a graph."""
import os
import subprocess
import sys

import pytest

pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

SCRIPT = """
import torch
from paper_2608_29809_gb300 import regioncache as R, synth
d = synth.Dims(hidden=128, heads=2, mlp=128, layers=1, grid_h=4, grid_w=4, timesteps=1)
ctx = R.rc_create(R.dims_struct(d))
g = torch.Generator(device="cuda").manual_seed(1)

def ints(v):
    return torch.tensor(v, dtype=torch.int32, device="cuda")

def rand(*shape):
    return torch.randn(*shape, generator=g, device="cuda").bfloat16()

heads, dh = 4, 72
wide = heads * dh
# one long request of a row and one of many (a launch each), and a batch for both kernels at once
shapes = [([5000], [1]), ([5000], [300]), ([200] * 90, [1] * 80 + [100] * 10)]
runs = []
for lens, counts in shapes:
    n, rows, total = len(lens), sum(counts), sum(lens)
    width = -(-max(lens) // 64)
    pool = R.Kv8Pool(n * width, heads, dh)
    x, w = rand(total, 512), rand(3 * wide, 512)
    x8, w8 = R.Fp8Matrix(total, 512), R.Fp8Matrix(3 * wide, 512, 128)
    qkv = torch.zeros(total, 3 * wide, dtype=torch.bfloat16, device="cuda")
    table = torch.zeros(n, width, dtype=torch.int32, device="cuda")
    lengths, offsets, used, slots = ints(lens), ints([0] * (n + 1)), ints([0]), ints([0] * total)
    rows_at = ints([sum(counts[:i]) for i in range(n + 1)])
    out = torch.zeros(rows, wide, dtype=torch.bfloat16, device="cuda")

    def go(lens=lens, counts=counts, n=n, rows=rows, total=total, width=width, pool=pool, x=x, w=w,
           x8=x8, w8=w8, qkv=qkv, table=table, lengths=lengths, offsets=offsets, used=used,
           slots=slots, rows_at=rows_at, out=out):
        R.rc_fp8_quantize(ctx, x, 512, R.RC_BF16, x8)
        R.rc_fp8_quantize(ctx, w, 512, R.RC_BF16, w8)
        R.rc_fp8_linear(ctx, x8, w8, None, qkv, 3 * wide, R.RC_BF16)
        R.rc_kv8_tables(ctx, lengths, None, None, n, None, n * width, table, width, offsets, slots,
                        total, used)
        R.rc_kv8_store(ctx, pool, qkv[:, wide:], qkv[:, 2 * wide:], 3 * wide, R.RC_BF16, slots,
                       total, None, R.RC_KV8_APPEND)
        R.rc_kv8_attention(ctx, pool, qkv, 3 * wide, rows, rows_at, lengths, n, max(counts), table,
                           width, heads, True, out, wide)

    runs.append((go, out))
torch.cuda.synchronize()
graphs = []
for go, out in runs:
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        go()
    graphs.append(graph)
for graph, (go, out) in zip(graphs, runs):
    graph.replay()
    torch.cuda.synchronize()
    got = out.clone()
    assert bool(got.isfinite().all()) and bool((got != 0).any())
    out.zero_()
    go()
    R.rc_sync(ctx)
    assert torch.equal(out, got)
print("captured")
"""


def test_first_calls_of_a_process_are_captured():
    from paper_2608_29809_gb300 import build as B
    B.build()
    r = subprocess.run([sys.executable, "-c", SCRIPT], cwd=ROOT, capture_output=True, text=True,
                       timeout=300)
    assert r.returncode == 0 and r.stdout.split() == ["captured"], r.stderr[-2000:]
