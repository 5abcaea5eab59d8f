"""The paged eight-bit cache: block tables and slot maps and the store bit for
bit, the attention against float64, and all of them together."""
import math
import threading

import pytest
import torch

from paper_2608_29809_gb300 import synth
from tests import eight_bit_ref as E

pytestmark = pytest.mark.gpu
BLOCK = 64


@pytest.fixture(scope="module")
def lib():
    from paper_2608_29809_gb300 import build as B
    B.build()
    from paper_2608_29809_gb300 import regioncache as R
    d = synth.Dims(hidden=128, heads=2, mlp=128, layers=1, grid_h=4, grid_w=4, timesteps=1)
    ctx = R.rc_create(R.dims_struct(d))
    yield R, ctx
    R.rc_destroy(ctx)


def _rand(*shape, seed=0, dtype=torch.float32):
    return synth.randn(shape, synth.tensor_seed(seed, *shape), "cuda", 1.0, dtype)


def _ints(v):
    return torch.tensor(v, dtype=torch.int32, device="cuda")


def _perm(n, seed):
    g = torch.Generator()
    g.manual_seed(seed)
    return torch.randperm(n, generator=g).tolist()


def _blocks(n):
    return -(-n // BLOCK)


# ------------------------------------------------------------------ tables
def _tables(R, ctx, lengths, counts, positions, free, table, n_slots, free_list=True):
    n = len(lengths)
    offsets, used = _ints([9] * (n + 1)), _ints([9])
    slots = _ints([9] * (n_slots + 3))
    R.rc_kv8_tables(ctx, _ints(lengths), None if counts is None else _ints(counts),
                    None if positions is None else _ints(positions), n,
                    _ints(free) if free_list else None, len(free), table, table.shape[1],
                    offsets, slots, n_slots, used)
    torch.cuda.synchronize()
    assert slots[n_slots:].tolist() == [9] * 3
    return offsets.tolist(), slots[:n_slots].tolist(), used.tolist()[0]


@pytest.mark.parametrize("lengths,counts", [
    ([1], None), ([64], None), ([65, 0, 63, 128], None), ([0, 0, 0], None),
    ([1, 64, 65, 128, 129, 700], [1, 1, 1, 1, 1, 1]), ([500, 64, 10], [0, 64, 3]),
    ([4096] * 5, [130, 1, 4096, 0, 64]), ([7 + i % 130 for i in range(1200)], None),
    ([1 + i % 3 for i in range(4096)], None), ([16384, 3, 9000], [16384, 1, 8999])])
@pytest.mark.parametrize("free_list", [True, False])
def test_tables(lib, lengths, counts, free_list):
    R, ctx = lib
    cnt = lengths if counts is None else counts
    need = sum(map(_blocks, lengths))
    width = max(max(map(_blocks, lengths)), 1) + 2
    pages = _perm(2 * need + 5, 1)
    table = torch.full((len(lengths), width), -7, dtype=torch.int32)
    at = need
    for r, (l, c) in enumerate(zip(lengths, cnt)):  # blocks that are held already
        for j in range(_blocks(l - c)):
            table[r, j] = pages[at]
            at += 1
    free = pages[:need + 2] if free_list else list(range(need + 2))
    want, slots, used, offsets = table.clone(), [], 0, [0]
    for r, (l, c) in enumerate(zip(lengths, cnt)):
        for j in range(_blocks(l - c), _blocks(l)):
            want[r, j] = free[used]
            used += 1
        slots += [int(want[r, p // BLOCK]) * BLOCK + p % BLOCK for p in range(l - c, l)]
        offsets.append(offsets[-1] + c)
    dev = table.cuda()
    for _ in range(2):
        got = _tables(R, ctx, lengths, counts, None, free, dev, len(slots) + 70, free_list)
        assert got == (offsets, slots + [-1] * 70, used)
        assert torch.equal(dev.cpu(), want)
    R.rc_sync(ctx)


@pytest.mark.parametrize("n", [1023, 1024, 4074, 4075, 4095])
def test_tables_of_any_number_of_requests(lib, n):
    R, ctx = lib
    lengths = [(i * 5) % 66 for i in range(n)]
    need = sum(map(_blocks, lengths))
    table = torch.full((n, 2), -1, dtype=torch.int32, device="cuda")
    offsets, slots, used = _tables(R, ctx, lengths, None, None, range(need), table, sum(lengths),
                                   free_list=False)
    at, want = 0, []
    for l in lengths:
        want += [at * BLOCK + p for p in range(l)]
        at += _blocks(l)
    assert slots == want and used == need and offsets[-1] == len(want)
    R.rc_sync(ctx)


def test_tables_from_threads_at_once(lib):
    """Calls of different numbers of requests, whose shared memory differs, on streams and buffers
    of their own: none is refused because of another's."""
    R, ctx = lib
    errors = []

    def calls(n):
        try:
            stream = torch.cuda.Stream()
            with torch.cuda.stream(stream):
                table = torch.full((n, 1), -1, dtype=torch.int32, device="cuda")
                lengths, offsets, slots, used = (_ints([1] * n), _ints([0] * (n + 1)),
                                                 _ints([0] * n), _ints([0]))
                for _ in range(4000):
                    R.rc_kv8_tables(ctx, lengths, None, None, n, None, n, table, 1, offsets, slots,
                                    n, used, stream)
                stream.synchronize()
                assert slots.tolist() == [64 * i for i in range(n)]
        except Exception as e:  # noqa: BLE001  (told to the main thread)
            errors.append((n, e))

    threads = [threading.Thread(target=calls, args=(n,)) for n in (4096, 3500, 4000, 3600)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    assert not errors
    R.rc_sync(ctx)


def test_tables_report_sums_that_pass_the_integers(lib):
    """Rows and new blocks of all requests together beyond 2^32: the first rows as ever."""
    R, ctx = lib
    table = torch.full((4096, 16384), -1, dtype=torch.int32, device="cuda")
    offsets, slots, used = _tables(R, ctx, [2 ** 20] * 4096, None, None, [7, 3], table, 100)
    _reported(R, ctx)
    assert offsets[:3] == [0, 2 ** 20, 2 ** 21] and offsets[-1] == 2 ** 31 - 1
    assert offsets == sorted(offsets) and used == 4096 * 16384
    assert slots == [7 * 64 + i for i in range(64)] + [3 * 64 + i for i in range(36)]


@pytest.mark.parametrize("entry", [2 ** 25, 2 ** 26, 2 ** 31 - 1])
def test_tables_give_no_slot_in_a_block_that_no_pool_has(lib, entry):
    R, ctx = lib
    table = torch.full((1, 2), entry, dtype=torch.int32, device="cuda")
    assert _tables(R, ctx, [70], [2], None, [], table, 2)[1] == [-1, -1]
    _reported(R, ctx)
    assert _tables(R, ctx, [3], None, None, [entry], table, 3)[1] == [-1] * 3
    _reported(R, ctx)
    table.fill_(2 ** 25 - 1)
    assert _tables(R, ctx, [70], [2], None, [], table, 2)[1] == [2 ** 31 - 60, 2 ** 31 - 59]
    R.rc_sync(ctx)


def test_tables_of_dirty_tokens(lib):
    R, ctx = lib
    lengths, counts = [300, 64, 0, 1000], [3, 2, 0, 5]
    positions = [0, 64, 299, 63, 5, 999, 1, 2, 500, 512]
    table = torch.tensor(_perm(4 * 16, 2), dtype=torch.int32).view(4, 16).cuda()
    want = []
    at = 0
    for r, c in enumerate(counts):
        for p in positions[at:at + c]:
            want.append(int(table[r, p // BLOCK]) * BLOCK + p % BLOCK)
        at += c
    before = table.clone()
    got = _tables(R, ctx, lengths, counts, positions, [], table, 10)
    assert got == ([0, 3, 5, 5, 10], want, 0) and torch.equal(table, before)
    R.rc_sync(ctx)


def _reported(R, ctx):
    with pytest.raises(R.RCError) as e:
        R.rc_sync(ctx)
    assert e.value.status == 6
    R.rc_sync(ctx)  # (cleared)


def test_tables_report_what_is_wrong_and_stay_in_bounds(lib):
    R, ctx = lib

    def go(lengths, counts, free, width, n_slots, positions=None, fill=3):
        table = torch.full((len(lengths), width), fill, dtype=torch.int32, device="cuda")
        out = _tables(R, ctx, lengths, counts, positions, free, table, n_slots)
        _reported(R, ctx)
        return out, table.tolist()

    # the free blocks run out: rows without a block have no slot
    (off, slots, used), table = go([130, 64], None, [5, 6], 3, 194)
    assert off == [0, 130, 194] and used == 4
    assert slots == [5 * 64 + i for i in range(64)] + [6 * 64 + i for i in range(64)] + [-1] * 66
    assert table[0] == [5, 6, -1] and table[1][0] == -1
    # counts and lengths that cannot be: no rows, the other requests are served
    for bad in ((10, 11), (-1, 0), (5, -1), (300, 1)):
        (off, slots, used), _ = go([64, bad[0], 1], [64, bad[1], 1], [1, 2, 8], 4, 65)
        assert off == [0, 64, 64, 65] and slots == [64 + i for i in range(64)] + [128]
        assert used == 2
    # more rows than the slot map holds
    (off, slots, used), _ = go([100], None, [1, 2], 2, 70)
    assert off == [0, 100] and slots == [64 + i for i in range(64)] + [128 + i for i in range(6)]
    # positions out of range, and a missing block
    (off, slots, used), _ = go([100], [3], [], 2, 3, [-1, 100, 99])
    assert slots == [-1, -1, 3 * 64 + 35]
    (off, slots, used), _ = go([100], [2], [], 2, 2, [0, 99], fill=-1)
    assert slots == [-1, -1]


# ------------------------------------------------------------------- store
def _pool(R, blocks, heads, dh, seed=0):
    """A pool of random codes and scales near one another."""
    p = R.Kv8Pool(blocks, heads, dh)
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    for code, scale in ((p.k, p.k_scale), (p.v, p.v_scale)):
        code.copy_((_rand(*code.shape, seed=seed) * 100).clamp(-448, 448).to(E.F8).view(torch.uint8))
        scale.copy_(torch.randint(115, 123, scale.shape, generator=g, device="cuda"))
    return p


def _state(p):
    return [(c.cpu().view(E.F8).double(), s.cpu().clone())
            for c, s in ((p.k, p.k_scale), (p.v, p.v_scale))]


def _store_and_check(R, ctx, p, k, v, slots, append, count=None, ld=None):
    heads, dh, n = p.c.kv_heads, p.c.head_dim, len(slots)
    want = _state(p)
    live = n if count is None else count
    for (codes, scales), x in zip(want, (k, v)):
        x = x[:, :heads * dh].double().cpu().view(-1, heads, dh)
        E.store(codes, scales, x[:live], slots[:live], append)
    R.rc_kv8_store(ctx, p, k, v, k.stride(0) if ld is None else ld, R.DTYPES[k.dtype],
                   _ints(slots), n, None if count is None else _ints([count]),
                   R.RC_KV8_APPEND if append else R.RC_KV8_UPDATE)
    torch.cuda.synchronize()
    for (codes, scales), (gc, gs) in zip(want, _state(p)):
        assert torch.equal(scales, gs)
        assert torch.equal(codes.isnan(), gc.isnan())
        assert torch.equal(codes.nan_to_num(0.0), gc.nan_to_num(0.0))


SLOTS = {
    "one": [3 * 64 + 5],
    "first": [4 * 64],
    "block": list(range(128, 192)),
    "three": list(range(64 + 60, 64 + 64)) + list(range(5 * 64, 6 * 64)) + list(range(0, 17)),
    "singles": [64 * b + (7 * b) % 64 for b in _perm(40, 3)],
    "sparse": [64 * b + o for b in _perm(30, 4) for o in range(b % 5, 64, 1 + b % 7)],
    "skipped": [-1, -5] + list(range(64, 70)) + [-1] * 20 + list(range(200, 230)) + [-1],
    "backwards": list(range(319, 250, -1)),
}


@pytest.mark.parametrize("name", sorted(SLOTS))
@pytest.mark.parametrize("heads,dh", [(16, 72), (1, 64), (5, 128), (2, 72)])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("append", [False, True])
def test_store(lib, name, heads, dh, dtype, append):
    R, ctx = lib
    slots, wide = SLOTS[name], heads * dh
    p = _pool(R, 41, heads, dh, seed=1)
    for seed, pad in ((2, 0), (3, 3)):  # (rows that are, and are not, 16-byte aligned)
        kv = _rand(len(slots), 2 * wide + pad, seed=seed) * torch.exp(
            2 * _rand(len(slots), 1, seed=4))
        kv = kv.to(dtype)
        _store_and_check(R, ctx, p, kv, kv[:, wide:], slots, append)
    R.rc_sync(ctx)


def test_store_of_many_rows(lib):
    """A fill of 2500 tokens whose blocks lie scattered, then an edit of every third one."""
    R, ctx = lib
    heads, dh = 8, 72
    pages = _perm(40, 5)
    slots = [pages[t // 64] * 64 + t % 64 for t in range(2500)]
    p = R.Kv8Pool(41, heads, dh)
    kv = _rand(2500, 2 * heads * dh, seed=6, dtype=torch.bfloat16)
    _store_and_check(R, ctx, p, kv, kv[:, heads * dh:], slots, True)
    edit = slots[::3]
    kv = 3 * _rand(len(edit), 2 * heads * dh, seed=7, dtype=torch.bfloat16)
    _store_and_check(R, ctx, p, kv, kv[:, heads * dh:], edit, False)
    R.rc_sync(ctx)


def _holes(name):
    """Slots whose skipped rows (negative) lie among the rows of a block."""
    if name == "one":
        return [64, 65, -1, 67, 68]
    if name == "few":  # the run's first row skipped, its last, and all between
        return [-1, 129, -3, -1, 132, -1] + [5 * 64] + [-1] * 62 + [5 * 64 + 63] + [-2, 200, -1, 193]
    if name == "far":  # a block's rows 64 rows from end to end, in every place of a warp's rows
        return sum(([64 * b + 3] + [-1] * 62 + [64 * b + 60] + [-1] * (b % 5) for b in range(40)), [])
    keep = _perm(2560, 21)  # a scattered fill of which many rows are skipped
    pages = _perm(40, 22)
    return [pages[t // 64] * 64 + t % 64 if keep[t] % 7 < 4 else -1 - t for t in range(2560)]


@pytest.mark.parametrize("name", ["one", "few", "far", "fill"])
@pytest.mark.parametrize("heads,dh", [(1, 64), (16, 72), (5, 128)])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("append", [False, True])
def test_store_skips_rows_inside_a_block(lib, name, heads, dh, dtype, append):
    """One scale for all of a block's rows, whatever lies between them: each larger than those
    before it in turn, so that a second run of the block would raise the scale again."""
    R, ctx = lib
    slots, wide = _holes(name), heads * dh
    p = _pool(R, 41, heads, dh, seed=19)
    for seed, up in ((20, 1.0), (21, -1.0)):
        steps = torch.arange(len(slots), device="cuda") % 64 * 0.25
        kv = _rand(len(slots), 2 * wide, seed=seed) * torch.exp2(up * steps)[:, None]
        kv = kv.to(dtype)
        _store_and_check(R, ctx, p, kv, kv[:, wide:], slots, append)
    R.rc_sync(ctx)


def test_store_reports_a_slot_beyond_the_pool_inside_a_block(lib):
    """It is skipped as a negative one is: the block's other rows share their scale."""
    R, ctx = lib
    p = _pool(R, 4, 2, 72, seed=23)
    kv = _rand(5, 288, seed=24) * torch.exp2(4.0 * torch.arange(5, device="cuda"))[:, None]
    want = _state(p)
    for (codes, scales), x in zip(want, (kv, kv[:, 144:])):
        E.store(codes, scales, x[:, :144].double().cpu().view(5, 2, 72), [64, 65, -1, 67, 68], True)
    R.rc_kv8_store(ctx, p, kv, kv[:, 144:], 288, R.RC_F32, _ints([64, 65, 4 * 64, 67, 68]), 5, None,
                   R.RC_KV8_APPEND)
    _reported(R, ctx)
    for (codes, scales), (gc, gs) in zip(want, _state(p)):
        assert torch.equal(scales, gs) and torch.equal(codes, gc)


def test_store_scales_far_apart(lib):
    """Scales raised by up to the whole range, zero rows, and the greatest values."""
    R, ctx = lib
    p = R.Kv8Pool(3, 2, 64)
    slots = list(range(64, 74))
    for i, top in enumerate((0.0, 1e-42, 1e-30, 1e-3, 1.0, 500.0, 3e38)):
        x = _rand(10, 256, seed=8 + i).clamp(-4, 4) / 4 * top
        _store_and_check(R, ctx, p, x, x[:, 128:], [s + i for s in slots], False)
    R.rc_sync(ctx)


@pytest.mark.parametrize("byte", [248, 253, 254])
def test_store_under_scales_that_it_never_gives_itself(lib, byte):
    R, ctx = lib
    p = _pool(R, 2, 2, 64, seed=17)
    p.k_scale.fill_(byte)
    p.v_scale.fill_(byte)
    x = _rand(9, 256, seed=18).clamp(-4, 4) / 4 * 3e38
    _store_and_check(R, ctx, p, x, x[:, 128:], list(range(70, 79)), False)
    R.rc_sync(ctx)


def test_store_what_is_not_finite(lib):
    R, ctx = lib
    p = _pool(R, 4, 2, 64, seed=9)
    x = _rand(3, 256, seed=10)
    x[1, 70] = math.nan
    x[2, 128] = math.inf
    _store_and_check(R, ctx, p, x, x[:, 128:], [65, 66, 67], False)
    assert int((p.k_scale == 255).sum()) == 1 and int((p.v_scale == 255).sum()) == 1
    y = _rand(2, 256, seed=11)  # such a block stays so until it starts anew
    _store_and_check(R, ctx, p, y, y[:, 128:], [70, 71], True)
    _store_and_check(R, ctx, p, y, y[:, 128:], [64, 71], True)
    assert int((p.k_scale == 255).sum()) == 0
    R.rc_sync(ctx)


def test_store_counts_on_the_device(lib):
    R, ctx = lib
    p = _pool(R, 8, 4, 72, seed=12)
    kv = _rand(100, 2 * 288, seed=13, dtype=torch.bfloat16)
    for count in (0, 1, 37, 100):
        _store_and_check(R, ctx, p, kv, kv[:, 288:], list(range(100, 200)), False, count=count)
    R.rc_sync(ctx)
    before = _state(p)
    for bad in (-1, 101):
        R.rc_kv8_store(ctx, p, kv, kv[:, 288:], 576, R.RC_BF16, _ints(list(range(100, 200))), 100,
                       _ints([bad]), R.RC_KV8_UPDATE)
        _reported(R, ctx)
    for (a, b), (c, d) in zip(before, _state(p)):
        assert torch.equal(a, c) and torch.equal(b, d)


def test_store_drops_and_reports_bad_slots(lib):
    R, ctx = lib
    p = _pool(R, 4, 2, 64, seed=14)
    want = _state(p)
    x = _rand(5, 256, seed=15)
    slots = [64, 66, 66, 4 * 64, 2 ** 31 - 1]
    for (codes, scales), y in zip(want, (x, x[:, 128:])):
        E.store(codes, scales, y[:2, :128].double().cpu().view(-1, 2, 64), slots[:2], False)
    R.rc_kv8_store(ctx, p, x, x[:, 128:], 256, R.RC_F32, _ints(slots), 5, None, R.RC_KV8_UPDATE)
    _reported(R, ctx)
    for (codes, scales), (gc, gs) in zip(want, _state(p)):
        # (the dropped row may have raised the scale)
        assert bool((gs >= scales).all()) and torch.equal(gs, scales)
        assert torch.equal(codes, gc)
    # the same slot for more rows than a block has
    R.rc_kv8_store(ctx, p, _rand(90, 256, seed=16), _rand(90, 256, seed=16), 256, R.RC_F32,
                   _ints([70] * 90), 90, None, R.RC_KV8_UPDATE)
    _reported(R, ctx)


# --------------------------------------------------------------- attention
class Case:
    """Requests over a shuffled pool: queries, table, cache values in f64."""

    def __init__(self, R, lens, counts, heads, kvh, dh, seed, scale=1.0, spare=0):
        self.lens, self.counts, self.heads, self.kvh, self.dh = lens, counts, heads, kvh, dh
        need = sum(map(_blocks, lens))
        self.pool = _pool(R, need + 3, kvh, dh, seed)
        self.width = max(max(map(_blocks, lens)), 1) + spare
        self.table = torch.full((len(lens), self.width), 2 ** 31 - 1, dtype=torch.int32)
        pages, at = _perm(need + 3, seed), 0
        for r, l in enumerate(lens):
            for j in range(_blocks(l)):
                self.table[r, j] = pages[at]
                at += 1
        rows = sum(counts)
        self.q = (_rand(rows + 2, heads * dh + 8, seed=seed + 1) * scale).bfloat16()
        self.offsets = [0]
        for c in counts:
            self.offsets.append(self.offsets[-1] + c)

    def run(self, R, ctx, causal, max_q=None):
        wide, rows = self.heads * self.dh, sum(self.counts)
        out = torch.full((rows + 2, wide + 16), 7.0, dtype=torch.bfloat16, device="cuda")
        R.rc_kv8_attention(ctx, self.pool, self.q, wide + 8, rows + 2, _ints(self.offsets),
                           _ints(self.lens), len(self.lens),
                           max(self.counts) if max_q is None else max_q, self.table.cuda(),
                           self.width, self.heads, causal, out, wide + 16)
        torch.cuda.synchronize()
        assert bool((out[rows:] == 7).all()) and bool((out[:, wide:] == 7).all())
        return out[:rows, :wide].double().cpu()

    def check(self, got, causal, only=None):
        """only: (request, query head) pairs to look at (all of them where None)."""
        k = E.cache_values(self.pool.k, self.pool.k_scale)
        v = E.cache_values(self.pool.v, self.pool.v_scale)
        dh, q = self.dh, self.q.double().cpu()
        for r, (l, c) in enumerate(zip(self.lens, self.counts)):
            pages = self.table[r, :_blocks(l)].long()
            rows = slice(self.offsets[r], self.offsets[r + 1])
            for h in range(self.heads):
                if only is not None and (r, h) not in only:
                    continue
                g = h // (self.heads // self.kvh)
                o, pv, reach = E.attention(
                    q[rows, h * dh:(h + 1) * dh], k[pages, g].reshape(-1, dh)[:l],
                    v[pages, g].reshape(-1, dh)[:l], causal)
                tol = E.attention_tolerance(o, pv, reach, dh)
                err = (got[rows, h * dh:(h + 1) * dh] - o).abs()
                assert bool((err <= tol).all()), (r, h, float((err / tol).max()))


@pytest.mark.parametrize("lens,counts", [
    ([1], [1]), ([64], [1]), ([65], [2]), ([4096], [1]), ([1000], [3]), ([129, 0, 700], [1, 1, 1]),
    ([0], [5]), ([5, 2000, 63, 64, 128], [1, 2, 0, 4, 8]), ([300] * 20, [1] * 20),
    ([5000, 17], [16, 1]), ([777], [17]), ([100, 900], [40, 3])])
@pytest.mark.parametrize("heads,kvh,dh", [(4, 4, 72), (2, 2, 64), (8, 2, 128), (3, 1, 72),
                                          (16, 1, 64)])
@pytest.mark.parametrize("causal", [False, True])
def test_attention_few_rows(lib, lens, counts, heads, kvh, dh, causal):
    R, ctx = lib
    c = Case(R, lens, counts, heads, kvh, dh, 21)
    c.check(c.run(R, ctx, causal), causal)
    R.rc_sync(ctx)


@pytest.mark.parametrize("lens,counts", [
    ([64], [64]), ([200], [128]), ([257], [129]), ([1100], [300]), ([129, 0, 700], [130, 140, 260]),
    ([2000, 31, 500], [33, 700, 1]), ([100], [400]), ([4096], [200]), ([640, 640], [256, 255])])
@pytest.mark.parametrize("heads,kvh,dh", [(2, 2, 72), (1, 1, 64), (4, 2, 128), (3, 1, 72)])
@pytest.mark.parametrize("causal", [False, True])
def test_attention_many_rows(lib, lens, counts, heads, kvh, dh, causal):
    R, ctx = lib
    c = Case(R, lens, counts, heads, kvh, dh, 22, spare=1)
    c.check(c.run(R, ctx, causal), causal)
    R.rc_sync(ctx)


@pytest.mark.parametrize("lens,counts", [
    ([500] * 30, [1] * 10 + [300] + [2] * 10 + [17] + [16] * 7 + [0]),
    ([64, 3000] + [200] * 600, [1, 700] + [1] * 600), ([900, 300, 100], [40, 0, 200])])
@pytest.mark.parametrize("heads,kvh,dh", [(2, 2, 72), (4, 1, 64)])
@pytest.mark.parametrize("causal", [False, True])
def test_attention_few_and_many_rows_together(lib, lens, counts, heads, kvh, dh, causal):
    R, ctx = lib
    c = Case(R, lens, counts, heads, kvh, dh, 28)
    got = c.run(R, ctx, causal)
    c.check(got, causal, None if len(lens) < 40 else
            {(r, h) for r in (0, 1, 2, 300, 511, 512, 601) for h in (0, heads - 1)})
    R.rc_sync(ctx)


@pytest.mark.parametrize("n", [37, 40, 191, 192, 193])
def test_attention_of_many_single_rows(lib, n):
    """Requests of every length, some the same, some without a token or a row."""
    R, ctx = lib
    lens = [(i * 89) % 301 // 3 * 3 if i % 7 else 128 for i in range(n)]
    lens[3] = 0
    c = Case(R, lens, [0 if i % 11 == 5 else 1 for i in range(n)], 18, 9, 64, 32)
    got = c.run(R, ctx, True)
    c.check(got, True, {(r, h) for r in list(range(0, n, 5)) + [n - 1] for h in (0, 9, 17)})
    R.rc_sync(ctx)


@pytest.mark.parametrize("n", [63, 64, 65])
@pytest.mark.parametrize("causal", [False, True])
def test_attention_of_requests_of_every_size(lib, n, causal):
    """More units than SMs: whole and last ones of many lengths, some requests without any."""
    R, ctx = lib
    c = Case(R, [(i * 37) % 211 * (1 + i % 3) for i in range(n)],
             [0 if i % 9 == 4 else 1 + (i * 53) % 390 for i in range(n)], 6, 3, 64, 33)
    got = c.run(R, ctx, causal)
    c.check(got, causal, {(r, h) for r in list(range(0, n, 4)) + [n - 1] for h in (0, 3, 5)})
    R.rc_sync(ctx)


@pytest.mark.parametrize("lens,counts,heads,kvh,dh", [
    ([9000] * 4, [260, 300, 270, 290], 16, 16, 128), ([20000, 17000], [70, 500], 2, 2, 64),
    ([40000], [3], 2, 2, 72), ([3100], [1], 16, 16, 72), ([2900], [2], 22, 22, 64),
    ([2000, 3300], [4, 1], 12, 6, 128), ([2500], [1], 30, 30, 72)])
def test_attention_over_long_caches(lib, lens, counts, heads, kvh, dh):
    R, ctx = lib
    c = Case(R, lens, counts, heads, kvh, dh, 29)
    got = c.run(R, ctx, True)
    c.check(got, True, {(0, 0), (len(lens) - 1, heads - 1)})
    R.rc_sync(ctx)


@pytest.mark.parametrize("counts", [[1, 2], [150, 90]])
@pytest.mark.parametrize("scale", [8.0, 60.0])
def test_attention_scores_far_apart(lib, counts, scale):
    """Rows whose largest score grows along the keys, and falls, by far more than exp's range,
    with blocks whose scales differ by up to 2^60."""
    R, ctx = lib
    c = Case(R, [900, 700], counts, 2, 2, 72, 23, scale=scale)
    b = c.pool.k_scale.shape[0]
    ramp = torch.arange(b, device="cuda") % 11
    c.pool.k_scale.copy_((112 + ramp)[:, None].expand(-1, 2))
    c.pool.v_scale.copy_((80 + 6 * ramp.flip(0))[:, None].expand(-1, 2))
    c.check(c.run(R, ctx, False), False)
    c.check(c.run(R, ctx, True), True)
    R.rc_sync(ctx)


@pytest.mark.parametrize("counts", [[1], [200]])
def test_attention_extreme_queries_and_scales(lib, counts):
    """Queries and cache scales at opposite ends of their range."""
    R, ctx = lib
    for e, b in ((60, 60), (-60, 180), (100, 20), (-100, 220)):
        c = Case(R, [300], counts, 2, 2, 64, 24, scale=2.0 ** e)
        c.pool.k_scale.fill_(b)
        c.pool.v_scale.fill_(245 - b)
        c.check(c.run(R, ctx, False), False)
    R.rc_sync(ctx)


@pytest.mark.parametrize("counts", [[2, 1], [150, 40]])
@pytest.mark.parametrize("bad", [math.nan, math.inf])
def test_attention_of_a_query_without_value(lib, counts, bad):
    """Its row is NaN and no other."""
    R, ctx = lib
    c = Case(R, [300, 100], counts, 2, 2, 72, 30)
    want = c.run(R, ctx, False)
    c.q[1, 72 + 5] = bad
    got = c.run(R, ctx, False)
    assert bool(got[1, 72:].isnan().all())
    got[1, 72:] = want[1, 72:]
    assert torch.equal(got, want)
    R.rc_sync(ctx)


@pytest.mark.parametrize("counts", [[3], [200]])
def test_attention_value_scales_at_both_ends(lib, counts):
    """Rows that see one block with values of 2^100 times the others', before or behind them:
    what the others give is lost beside it where it counts, and whole where it does not."""
    R, ctx = lib
    for at in (0, 1, 4):
        c = Case(R, [300], counts, 2, 2, 64, 31)
        c.pool.v_scale.fill_(60)
        c.pool.v_scale[c.table[0, at].item()] = 160
        c.check(c.run(R, ctx, False), False)
        c.pool.v_scale.fill_(130)
        c.pool.v_scale[c.table[0, at].item()] = 0
        c.pool.v[c.table[0, at].item()] = 0
        c.check(c.run(R, ctx, True), True)
    R.rc_sync(ctx)


@pytest.mark.parametrize("lens,counts,heads,kvh,dh", [
    ([300], [3], 2, 2, 72), ([700, 64], [16, 2], 4, 2, 128), ([5000], [1], 2, 2, 64),
    ([300], [200], 2, 2, 64), ([260], [100], 1, 1, 128), ([3000], [150], 2, 2, 72),
    ([200] * 40, [45] * 40, 6, 6, 72)])
@pytest.mark.parametrize("byte", [3, 20, 240, 244])
def test_attention_of_the_smallest_and_largest_values(lib, lens, counts, heads, kvh, dh, byte):
    """A mean of values near f32's ends lies there too, whatever the sum of its weights (scores of
    up to some tens: the first blocks' may lie far below a row's largest)."""
    R, ctx = lib
    c = Case(R, lens, counts, heads, kvh, dh, 43, scale=0.5)
    c.pool.v_scale.fill_(byte)
    got = c.run(R, ctx, False)
    up = 2.0 ** (127 - byte)  # (the tolerance's floor is for values near 1)
    kept, c.pool.v_scale = c.pool.v_scale, torch.full_like(c.pool.v_scale, 127)
    assert bool(got.isfinite().all())
    c.check(got * up, False)
    c.pool.v_scale = kept
    R.rc_sync(ctx)


@pytest.mark.parametrize("tail", [15.5, 18.0, 21.0])
@pytest.mark.parametrize("up", [0, 3, 4, 5, 10, 13])
@pytest.mark.parametrize("count", [1, 5, 100])
def test_attention_long_tail_of_small_weights(lib, tail, up, count):
    """One key in 32 of the first 3200 outweighs all others but has no values; the next 3200 have
    values of 2^up times the last ones', but no weight; the last 8192, all about 2^-tail of the first
    ones, give the result.  No weight is off by more than 2^-8 of itself or 2^-25 of the largest."""
    R, ctx = lib
    head, length, dh = 3200, 2 * 3200 + 8192, 64
    c = Case(R, [length], [count], 1, 1, dh, 44)
    unit = tail * 8 / math.log2(math.e)  # a key of -1 has the score -tail, in base 2
    c.q.zero_()
    c.q[:, 0] = unit
    key = torch.full((length,), -16.0)
    key[:head:32] = 0.0
    key[2 * head:] = -1.0
    value = (_rand(length, dh, seed=45).abs().clamp(max=3.0).cpu() + 1.0) * 100
    value[:head:32] = 0.0
    codes = torch.zeros(length, dh)
    codes[:, 0] = key
    pages = c.table[0].long().cuda()
    c.pool.k[pages, 0] = codes.view(-1, 64, dh).to(E.F8).view(torch.uint8).cuda()
    c.pool.v[pages, 0] = value.view(-1, 64, dh).to(E.F8).view(torch.uint8).cuda()
    c.pool.k_scale.fill_(127)
    c.pool.v_scale.fill_(120)
    c.pool.v_scale[pages[head // 64:2 * head // 64]] = 120 + up
    got = c.run(R, ctx, False)
    k = E.cache_values(c.pool.k, c.pool.k_scale)[pages.cpu(), 0].reshape(-1, dh)
    v = E.cache_values(c.pool.v, c.pool.v_scale)[pages.cpu(), 0].reshape(-1, dh)
    o, pv, reach = E.attention(c.q[:count, :dh].double().cpu(), k, v, False)
    largest = 1 / (head // 32)  # (a little more than the largest weight)
    # weights of zero are exact; the block of no weight has no part in the bound
    small = 2.0 ** -25 * largest * v[2 * head:].abs().sum(0)
    tol = E.attention_tolerance(o, pv, reach, dh) + small
    err = (got - o).abs()
    assert bool((err <= tol).all()), float((err / tol).max())
    R.rc_sync(ctx)


@pytest.mark.parametrize("counts", [[1, 1], [3, 150]])
def test_attention_block_without_value(lib, counts):
    """NaN blocks reach the rows that see them and no others; behind the last token and in
    blocks of nobody they reach none."""
    R, ctx = lib
    c = Case(R, [190, 500], counts, 2, 1, 72, 25)
    used = c.table[0, 1].item()
    spare = (set(range(len(c.pool.k_scale))) - set(c.table[c.table < 2 ** 31 - 1].tolist())).pop()
    c.pool.k_scale[spare] = c.pool.v_scale[spare] = 255
    c.pool.k[c.table[0, 2].item(), :, 62:] = 0x7f  # behind token 189
    c.pool.v[c.table[0, 2].item(), :, 62:] = 0x7f
    clean = c.run(R, ctx, False)
    assert not bool(clean.isnan().any())
    for scale in (c.pool.k_scale, c.pool.v_scale):
        kept = scale[used].clone()
        scale[used] = 255
        got = c.run(R, ctx, False)
        assert bool(got[:counts[0]].isnan().all())
        assert torch.equal(got[counts[0]:], clean[counts[0]:])
        scale[used] = kept
    R.rc_sync(ctx)


def _causal_rows(c, got):
    """Causal rows against what each one sees, and nothing else: (its first and last visible block
    or None, result, definition, tolerance) of every row and query head."""
    k = E.cache_values(c.pool.k, c.pool.k_scale)
    v = E.cache_values(c.pool.v, c.pool.v_scale)
    q, dh = c.q.double().cpu(), c.dh
    for r, (l, n) in enumerate(zip(c.lens, c.counts)):
        pages = c.table[r, :_blocks(l)].long()
        for h in range(c.heads):
            g = h // (c.heads // c.kvh)
            kh, vh = k[pages, g].reshape(-1, dh), v[pages, g].reshape(-1, dh)
            for i in range(n):
                sees = max(0, l - n + i + 1)
                row, cols = c.offsets[r] + i, slice(h * dh, (h + 1) * dh)
                o, pv, reach = E.attention(q[row:row + 1, cols], kh[:sees], vh[:sees], False)
                yield (r, sees, got[row:row + 1, cols], o,
                       E.attention_tolerance(o, pv, reach, dh) if sees else None)


# few rows of one CTA and of clusters, many rows of one CTA (one tile and two) and of clusters,
# grouped heads, and requests whose first rows see nothing
LATER = [([66], [4], 2, 2, 72), ([66], [70], 1, 1, 64), ([130], [16], 2, 1, 128),
         ([20], [60], 1, 1, 72), ([5000], [13], 2, 2, 72), ([70, 200], [90, 160], 2, 2, 72),
         ([200], [230], 1, 1, 128), ([1500], [200], 4, 2, 64), ([700], [150], 1, 1, 64),
         ([100] * 40, [17, 45] * 20, 6, 6, 64)]


@pytest.mark.parametrize("lens,counts,heads,kvh,dh", LATER)
@pytest.mark.parametrize("side", ["k", "v"])
def test_attention_block_without_value_behind_causal_rows(lib, lens, counts, heads, kvh, dh, side):
    """A block that is not finite reaches the rows that see one of its tokens, and no others: with
    the codes that the store leaves there, and with any."""
    R, ctx = lib
    for codes in (False, True):
        c = Case(R, lens, counts, heads, kvh, dh, 41)
        scale, code = (c.pool.k_scale, c.pool.k) if side == "k" else (c.pool.v_scale, c.pool.v)
        first = [_blocks(l) - 1 for l in lens]
        for r, b in enumerate(first):
            scale[c.table[r, b].item()] = 255
            if codes:
                code[c.table[r, b].item()] = 0x7f
        rows = [0, 0]
        for r, sees, got, o, tol in _causal_rows(c, c.run(R, ctx, True)):
            if sees > first[r] * BLOCK:
                assert bool(got.isnan().all())
            elif sees == 0:
                assert bool((got == 0).all())
            else:
                assert bool(((got - o).abs() <= tol).all()), (r, sees)
            rows[sees > first[r] * BLOCK] += 1
        assert min(rows) > 0
    R.rc_sync(ctx)


@pytest.mark.parametrize("lens,counts,heads,kvh,dh", LATER)
def test_attention_value_scales_far_apart_behind_causal_rows(lib, lens, counts, heads, kvh, dh):
    """Values of 2^128 times the earlier blocks' in a later one: lost beside them for the rows that
    see both, and nothing to those that do not."""
    R, ctx = lib
    c = Case(R, lens, counts, heads, kvh, dh, 42)
    c.pool.v_scale -= 20  # (95 .. 102)
    for r, l in enumerate(lens):
        c.pool.v_scale[c.table[r, _blocks(l) - 1].item()] = 230
    for r, sees, got, o, tol in _causal_rows(c, c.run(R, ctx, True)):
        assert bool((got == 0).all() if sees == 0 else ((got - o).abs() <= tol).all()), (r, sees)
    R.rc_sync(ctx)


@pytest.mark.parametrize("counts", [[2, 3, 1], [200, 130, 5]])
def test_attention_leaves_out_and_reports_bad_requests(lib, counts):
    R, ctx = lib
    lens = [300, 128, 65]
    c = Case(R, lens, counts, 2, 2, 64, 26)
    want = c.run(R, ctx, False)
    a, b = c.offsets[1], c.offsets[2]

    def same_but_second(got):
        assert torch.equal(got[:a], want[:a]) and torch.equal(got[b:], want[b:])

    for bad in (-1, c.width * 64 + 1, 2 ** 31 - 1):
        c.lens = [300, bad, 65]
        got = c.run(R, ctx, False)
        _reported(R, ctx)
        same_but_second(got)
        assert bool((got[a:b] == 7).all())
    c.lens = lens
    # too many rows for max_q: that request alone
    got = c.run(R, ctx, False, max_q=max(counts) - 1)
    _reported(R, ctx)
    worst = counts.index(max(counts))
    for r in range(3):
        rows = slice(c.offsets[r], c.offsets[r + 1])
        assert bool((got[rows] == 7).all()) if r == worst else torch.equal(got[rows], want[rows])
    # a block outside the pool hides its tokens: as if the request ended before it
    entry = c.table[1, 1].item()
    for bad in (-1, 10 ** 6):
        c.table[1, 1] = bad
        got = c.run(R, ctx, False)
        _reported(R, ctx)
        same_but_second(got)
        c.table[1, 1] = entry
        c.lens = [300, 64, 65]
        c.check(got, False)
        c.lens = lens
    R.rc_sync(ctx)


@pytest.mark.parametrize("counts", [[1] * 60, [40] * 60, [3] * 99 + [900] + [30] * 20])
def test_attention_leaves_bad_requests_out_of_the_order(lib, counts):
    """Batches of more CTAs than places: the other requests' rows keep their bits."""
    R, ctx = lib
    n = len(counts)
    lens = [(i * 31) % 160 + 1 for i in range(n)]
    c = Case(R, lens, counts, 6, 6, 64, 34)
    want = c.run(R, ctx, False)
    for r in (0, 7, n - 1):
        for bad in (-1, c.width * 64 + 1):
            c.lens = lens[:r] + [bad] + lens[r + 1:]
            got = c.run(R, ctx, False)
            _reported(R, ctx)
            rows = slice(c.offsets[r], c.offsets[r + 1])
            assert bool((got[rows] == 7).all())
            got[rows] = want[rows]
            assert torch.equal(got, want)
    R.rc_sync(ctx)


def test_attention_gives_the_same_bits_again(lib):
    R, ctx = lib
    for lens, counts in (([5000, 300], [1, 1]), ([3000, 700], [130, 200])):
        c = Case(R, lens, counts, 4, 2, 72, 27)
        first = c.run(R, ctx, True)
        for _ in range(3):
            assert torch.equal(first, c.run(R, ctx, True))
    R.rc_sync(ctx)


def test_attention_captured_on_streams_at_once(lib):
    """Graphs of batches for either kernel and for both, replayed at once on streams of their own
    with other lengths than at capture."""
    R, ctx = lib
    cases = [Case(R, lens, counts, 8, 4, 64, 35 + len(lens)) for lens, counts in (
        ([900] * 3, [1] * 3), ([700] * 5, [90, 200, 3, 40, 150]),
        ([300] * 90, [1] * 80 + [100] * 10), ([5000], [300]))]
    runs = []
    for c in cases:
        wide, rows = 8 * 64, sum(c.counts)
        full, short = _ints(c.lens), _ints([l - 70 * (i % 3) for i, l in enumerate(c.lens)])
        lens, offsets, table = full.clone(), _ints(c.offsets), c.table.cuda()
        out = torch.zeros(rows, wide, dtype=torch.bfloat16, device="cuda")

        def go(c=c, lens=lens, offsets=offsets, table=table, out=out, rows=rows, wide=wide):
            R.rc_kv8_attention(ctx, c.pool, c.q, wide + 8, rows, offsets, lens, len(c.lens),
                               max(c.counts), table, c.width, c.heads, True, out, wide)

        want = []
        for l in (short, full):
            lens.copy_(l)
            go()
            want.append(out.clone())
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            go()
        runs.append((graph, torch.cuda.Stream(), go, lens, (short, full), out, want))
    for i in (0, 1, 0):
        for *_, lens, choice, out, want in runs:
            lens.copy_(choice[i])
            out.zero_()
        torch.cuda.synchronize()
        for _ in range(4):
            for graph, stream, *_ in runs:
                with torch.cuda.stream(stream):
                    graph.replay()
        torch.cuda.synchronize()
        for *_, out, want in runs:
            assert torch.equal(out, want[i])
    R.rc_sync(ctx)


# ---------------------------------------------------------------- together
def test_a_region_sublayer_in_eight_bits(lib):
    """Quantised q | k | v product, slot map of the dirty tokens, store, attention and quantised
    output product of three sessions, launched and replayed from a graph, each stage against its
    definition on what the stage before left."""
    R, ctx = lib
    heads, dh = 4, 72
    d = heads * dh
    lens, dirty = [300, 64, 1000], [70, 0, 129]
    rows, bound = sum(dirty), 220  # (padded rows: slots -1)
    wq, wo = (R.Fp8Matrix(3 * d, d, 128), R.Fp8Matrix(d, d, 128))
    for m, seed in ((wq, 31), (wo, 32)):
        w = _rand(m.c.rows, d, seed=seed) * d ** -0.5
        R.rc_fp8_quantize(ctx, w, d, R.RC_F32, m)
    pool = R.Kv8Pool(60, heads, dh)
    table = torch.full((3, 16), -1, dtype=torch.int32, device="cuda")
    offsets, used = _ints([0] * 4), _ints([0])
    # the first fill of the three sessions
    total = sum(lens)
    slots = _ints([0] * total)
    R.rc_kv8_tables(ctx, _ints(lens), None, None, 3, _ints(_perm(60, 33)), 60, table, 16, offsets,
                    slots, total, used)
    kv = _rand(total, 2 * d, seed=34, dtype=torch.bfloat16)
    R.rc_kv8_store(ctx, pool, kv, kv[:, d:], 2 * d, R.RC_BF16, slots, total, None, R.RC_KV8_APPEND)
    # an edit
    pos = []
    for l, c in zip(lens, dirty):
        pos += sorted(_perm(l, 35 + l)[:c])
    lengths, counts, positions = _ints(lens), _ints(dirty), _ints(pos + [0] * (bound - rows))
    x = _rand(bound, d, seed=36, dtype=torch.bfloat16)
    xm, om = R.Fp8Matrix(bound, d), R.Fp8Matrix(bound, d)
    qkv = torch.zeros(bound, 3 * d, dtype=torch.bfloat16, device="cuda")
    o, y = torch.zeros_like(x), torch.zeros(bound, d, device="cuda")
    slots = _ints([0] * bound)

    def step():
        R.rc_fp8_quantize(ctx, x, d, R.RC_BF16, xm)
        R.rc_fp8_linear(ctx, xm, wq, None, qkv, 3 * d, R.RC_BF16)
        R.rc_kv8_tables(ctx, lengths, counts, positions, 3, None, 0, table, 16, offsets, slots,
                        bound, used)
        R.rc_kv8_store(ctx, pool, qkv[:, d:], qkv[:, 2 * d:], 3 * d, R.RC_BF16, slots, bound, None,
                       R.RC_KV8_UPDATE)
        R.rc_kv8_attention(ctx, pool, qkv, 3 * d, bound, offsets, lengths, 3, 150, table, 16,
                           heads, 0, o, d)
        R.rc_fp8_quantize(ctx, o, d, R.RC_BF16, om)
        R.rc_fp8_linear(ctx, om, wo, None, y, d, R.RC_F32)

    def check(before):
        R.rc_sync(ctx)
        codes, scales = E.quantize(x, 1)
        assert torch.equal(xm.scales.cpu(), scales)
        w = E.values(wq.codes, wq.scales, 128, d)
        want = E.values(xm.codes, xm.scales, 1, d) @ w.t()
        mag = E.values(xm.codes, xm.scales, 1, d).abs() @ w.abs().t()
        got = qkv.double().cpu()
        assert bool(((got - want).abs() <= 2.0 ** -8 * want.abs() + 1.01 * d * 2.0 ** -23 * mag).all())
        for i, (codes, scales) in enumerate(before):
            part = got[:rows, d * (i + 1):d * (i + 2)].reshape(rows, heads, dh)
            E.store(codes, scales, part, slots[:rows].tolist(), False)
            after = _state(pool)[i]
            assert torch.equal(after[0], codes) and torch.equal(after[1], scales)
        assert slots[rows:].tolist() == [-1] * (bound - rows)
        c = Case.__new__(Case)
        c.lens, c.counts, c.heads, c.kvh, c.dh, c.pool = lens, dirty, heads, heads, dh, pool
        c.table, c.q, c.offsets = table.cpu(), qkv[:, :d], offsets.tolist()
        c.check(o[:rows].double().cpu(), False)
        w = E.values(wo.codes, wo.scales, 128, d)
        ov = E.values(om.codes, om.scales, 1, d)
        assert bool(((y.double().cpu() - ov @ w.t()).abs() <=
                     d * 2.0 ** -23 * (ov.abs() @ w.abs().t()) + 1e-37).all())

    before = _state(pool)
    step()
    check(before)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    x.copy_(_rand(bound, d, seed=37))
    x.mul_(3.0)
    before = _state(pool)
    torch.cuda.synchronize()
    graph.replay()
    check(before)
