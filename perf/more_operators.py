"""The operators around the quantised products and the eight-bit cache of a
transformer block, as cases to be timed.

  norm    rc_norm_residual   norm of a block's output, its gate, the scaled
                             residual and the norm before the next block
  rotary  rc_rotary_apply    rotary positions of query and key heads
  route   rc_experts_route,  experts of each row (softmax or sigmoid scores,
          rc_experts_sort    balance bias, groups, top-k) and the order of
                             the rows by expert
  linear  rc_experts_linear  each expert's quantised product of its rows
  ffn     all of them        a feed-forward block of experts: norm to codes,
                             routing, both products, weighted sum, residual

``run`` computes them with plain torch in 32 bits (scores that are compared
and angles in 64), or (``own``) through the public entry points.  ``exact``
restates them in float64.
"""
import math

import torch

own = False

DEV = "cuda"
GROUP = 128   # columns of a scale of a quantised matrix
E4M3 = torch.float8_e4m3fn
TYPES = {"bf16": torch.bfloat16, "f32": torch.float32}
SIZE = {"bf16": 2, "f32": 4}
BIG = torch.finfo(torch.float32).max


# ------------------------------------------------------------------- cases
def _norm(name, rows, cols, items=1, x="f32", h="bf16", y="bf16", post="none", pre="layer",
          gate=True, mod=True, scale=1.0):
    """h "": no branch, the norm before a block alone."""
    return {"name": name, "kind": "norm", "rows": rows, "cols": cols, "items": items, "x": x,
            "h": h, "y": y, "post": post, "pre": pre, "gate": gate, "mod": mod, "scale": scale}


def _rotary(name, rows, heads, dh, rot, dtype="bf16", layout="half", axes=1, longest=4096,
            scaling="none", factor=1.0, pad=0):
    return {"name": name, "kind": "rotary", "rows": rows, "heads": heads, "dh": dh, "rot": rot,
            "dtype": dtype, "layout": layout, "axes": axes, "longest": longest,
            "scaling": scaling, "factor": factor, "pad": pad}


def _route(name, rows, experts, k, score="softmax", dtype="f32", bias=False, groups=1, best=1,
           of_best=1, renorm=True, masked=0):
    """`groups` groups, of which the `best` by the sum of their `of_best` best scores count;
    `masked`: experts without a score in some rows."""
    return {"name": name, "kind": "route", "rows": rows, "experts": experts, "k": k,
            "score": score, "dtype": dtype, "bias": bias, "groups": groups, "best": best,
            "of_best": of_best, "renorm": renorm, "masked": masked}


def _linear(name, rows, k, experts, cols, n, act="none", out="bf16", bias=True, gather=True):
    """rows * k products of a row and an expert, cols -> n."""
    return {"name": name, "kind": "linear", "rows": rows, "k": k, "experts": experts,
            "cols": cols, "n": n, "act": act, "out": out, "bias": bias, "gather": gather}


def _ffn(name, rows, k, experts, cols, mlp, act="gelu", score="softmax"):
    return {"name": name, "kind": "ffn", "rows": rows, "k": k, "experts": experts, "cols": cols,
            "mlp": mlp, "act": act, "score": score}


def listed():
    return [
        # one token before its block: all latency
        _norm("norm_1x1152", 1, 1152, h=""),
        # eight sessions' edits at 1024 px between the attention and the MLP, modulated by item
        _norm("norm_8_edits", 4128, 1152, items=8),
        # every token of 2048 px at the MLP's width, norms on both sides of the block
        _norm("norm_16384x4608", 16384, 4608, x="bf16", post="rms", pre="rms", gate=False,
              mod=False, scale=0.5),
        # one token of 48 sequences, four query heads a key head, stretched to four times the length
        _rotary("rotary_48_tokens", 48, 40, 128, 128, longest=12000, scaling="bands", factor=4.0),
        # q | k of an image of 128 x 128 tokens as the projection leaves them, a half of a head
        # for each axis
        _rotary("rotary_16384", 16384, 32, 72, 72, layout="pairs", axes=2, longest=128, pad=1152),
        # one token of 48 sequences
        _route("route_48_of_64", 48, 64, 6),
        # every token of 1024 px, few experts
        _route("route_4096_of_16", 4096, 16, 2, dtype="bf16"),
        # every token of 2048 px, many small experts in groups
        _route("route_16384_of_256", 16384, 256, 8, score="sigmoid", bias=True, groups=8, best=4,
               of_best=2),
        # one token of 48 sequences, small experts: all weights are read for a few rows each
        _linear("linear_48x6_of_64", 48, 6, 64, 1152, 1152),
        # every token of 2048 px through two of eight MLPs
        _linear("linear_16384x2_of_8", 16384, 2, 8, 1152, 4608, act="gelu"),
        # a block of one new token
        _ffn("ffn_1x2_of_8", 1, 2, 8, 1152, 4608),
        # eight sessions' edits at 1024 px, gated experts
        _ffn("ffn_8_edits", 4128, 2, 16, 1152, 2304, act="gated_silu"),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    most = {}
    for c in listed():
        w = work(c)
        m = most.setdefault(c["kind"], [0.0, 0.0])
        most[c["kind"]] = [max(m[0], w["bytes"]), max(m[1], w["flops"])]
    while True:
        kind = rng.choice(["norm", "norm", "rotary", "rotary", "route", "route", "linear",
                           "linear", "ffn"])
        if kind == "norm":
            rows = _log_int(rng, 1, 16384)
            post, pre = rng.choice(["none", "rms", "layer"]), rng.choice(["rms", "layer"])
            cols = rng.choice([1152, 4608]) if rng.random() < 0.4 else _log_int(rng, 40, 9000)
            c = _norm("", rows, cols, rng.randint(1, min(rows, 64)), rng.choice(["f32", "bf16"]),
                      rng.choice(["bf16", "bf16", "f32", ""]), rng.choice(["bf16", "f32"]), post,
                      pre, rng.random() < 0.6, rng.random() < 0.6, rng.choice([1.0, 0.5, 1.25]))
        elif kind == "rotary":
            dh = rng.choice([64, 72, 128, 128])
            c = _rotary("", _log_int(rng, 1, 16384), rng.choice([1, 5, 16, 32, 40]), dh,
                        rng.choice([dh, dh, dh // 2, dh // 4 * 2 - 2]),
                        rng.choice(["bf16", "bf16", "f32"]), rng.choice(["half", "pairs"]),
                        rng.choice([1, 1, 2]), _log_int(rng, 100, 1000000),
                        rng.choice(["none", "linear", "base", "bands", "ramp"]),
                        rng.choice([2.0, 8.0]), rng.choice([0, 0, 1152, 5]))
        elif kind == "route":
            experts = rng.choice([4, 8, 16, 60, 64, 128, 160, 256, 512])
            groups = rng.choice([1, 1, 1, 2, 4])
            best = rng.randint(1, groups)
            c = _route("", _log_int(rng, 1, 16384), experts,
                       rng.randint(1, min(10, experts // groups * best)),
                       rng.choice(["softmax", "sigmoid"]), rng.choice(["f32", "bf16"]),
                       rng.random() < 0.5, groups, best, rng.choice([1, 2]) if groups > 1 else 1,
                       rng.random() < 0.6, rng.choice([0, 0, 3]))
        elif kind == "linear":
            wide = [1152, 2304, 4608]
            n, cols = ((rng.choice(wide), rng.choice(wide)) if rng.random() < 0.5 else
                       (_log_int(rng, 20, 4000), _log_int(rng, 20, 4000)))
            experts = rng.choice([1, 4, 8, 16, 60, 64])
            c = _linear("", _log_int(rng, 1, 16384), rng.randint(1, min(6, experts)), experts,
                        cols, n, rng.choice(["none", "none", "gelu", "silu", "gated_silu"]),
                        rng.choice(["bf16", "bf16", "f32"]), rng.random() < 0.6,
                        rng.random() < 0.5)
        else:
            experts = rng.choice([4, 8, 16, 60, 64])
            mlp = rng.choice([1152, 2304, 4608]) if rng.random() < 0.6 else _log_int(rng, 60, 4000)
            c = _ffn("", _log_int(rng, 1, 4128), rng.randint(1, min(6, experts)), experts,
                     rng.choice([1152, 1152, _log_int(rng, 60, 2304)]), mlp,
                     rng.choice(["gelu", "silu", "gated_silu"]), rng.choice(["softmax", "sigmoid"]))
        if kind in ("linear", "ffn"):
            # what the plain form holds: weights in 32 bits, each expert's rows as the most of one
            wide = c["cols"] + c.get("n", 0) + 3 * c.get("mlp", 0)
            if c["experts"] * wide * max(_cap(c), c["cols"]) > 8e8:
                continue
        del c["name"]
        w = work(c)
        if w["bytes"] <= most[kind][0] and w["flops"] <= most[kind][1]:
            return c


# ------------------------------------------------------------------- sizes
def _shares(c):
    """Rows of each expert: uneven, and the same for each seed."""
    pairs, e = c["rows"] * c["k"], c["experts"]
    weights = [1.0 / (1 + (7 * i) % e) ** 0.4 for i in range(e)]
    total, at, cuts = sum(weights), 0.0, [0]
    for w in weights:
        at += w
        cuts.append(int(round(pairs * at / total)))
    return [b - a for a, b in zip(cuts, cuts[1:])]


def _cap(c):
    if c["kind"] == "linear":
        return max(_shares(c))
    return min(c["rows"], 4 * c["rows"] * c["k"] // c["experts"] + 64)


def _item_rows(c):
    """First row of each item of a norm, and the end: uneven pieces."""
    n = c["items"]
    return [c["rows"] * (2 * i * n + i * i) // (3 * n * n) for i in range(n)] + [c["rows"]]


def _wide(act):
    """Columns of a product for each column after its activation."""
    return 2 if act == "gated_silu" else 1


def work(case):
    """Each input read once, each output written once; products and sums of the definition."""
    kind, rows = case["kind"], case["rows"]
    if kind == "norm":
        n = rows * case["cols"]
        per = SIZE[case["x"]] + SIZE[case["y"]] + (
            SIZE[case["h"]] + SIZE[case["x"]] if case["h"] else 0)
        mods = (1 if case["gate"] and case["h"] else 0) + (2 if case["mod"] else 0)
        return {"bytes": n * per + 4 * case["items"] * case["cols"] * mods, "flops": 10 * n}
    if kind == "rotary":
        n = rows * case["heads"] * case["dh"]
        return {"bytes": 2 * n * SIZE[case["dtype"]] + 4 * rows * case["axes"],
                "flops": 3 * rows * case["heads"] * case["rot"]}
    if kind == "route":
        n, pairs = rows * case["experts"], rows * case["k"]
        # logits; ids, weights, places and source rows; offsets
        return {"bytes": n * SIZE[case["dtype"]] + 16 * pairs + 4 * case["experts"],
                "flops": 8 * n}
    cols, e = case["cols"], case["experts"]
    if kind == "linear":
        pairs, n, used = rows * case["k"], case["n"], sum(1 for s in _shares(case) if s)
        wide = n * _wide(case["act"])
        read = rows if case["gather"] else pairs
        return {"bytes": read * (cols + cols // GROUP) + used * wide * cols +
                pairs * n * SIZE[case["out"]] + (4 * pairs if case["gather"] else 0) +
                (4 * used * wide if case["bias"] else 0), "flops": 2 * pairs * wide * cols}
    pairs, mlp, wide = rows * case["k"], case["mlp"], case["mlp"] * _wide(case["act"])
    used = e * (1 - (1 - case["k"] / e) ** rows)
    return {"bytes": 4 * rows * cols + 4 * rows * e + used * cols * (wide + mlp),
            "flops": 2 * pairs * cols * (wide + mlp)}


# ------------------------------------------------------------- preparation
def _randn(g, *shape):
    return torch.randn(*shape, generator=g, device=DEV)


def _ints(values):
    return torch.tensor(values, dtype=torch.int32, device=DEV)


def _logits(g, case):
    """Scores as a router's projection gives them: some experts are liked better than others."""
    z = 1.5 * _randn(g, case["rows"], case["experts"]) + 0.7 * _randn(g, case["experts"])
    if case.get("masked"):
        some = torch.rand(case["rows"], 1, generator=g, device=DEV) < 0.3
        z = torch.where(some & (torch.arange(case["experts"], device=DEV) < case["masked"]),
                        -math.inf, z)
    return z.to(TYPES[case.get("dtype", "f32")])


def _matrix(g, rows, cols, per, scale=0.0):
    """A quantised matrix: codes [rows][ld], scales [ceil(cols / 128)][ceil(rows / per)], of
    values of about 2^scale."""
    ld, kb = -(-cols // 16) * 16, -(-cols // GROUP)
    codes = torch.zeros(rows, ld, dtype=torch.uint8, device=DEV)
    codes[:, :cols] = (_randn(g, rows, cols) * 110).clamp_(-448, 448).to(E4M3).view(torch.uint8)
    mid = 127 - 7 + int(round(scale))
    scales = torch.randint(mid - 1, mid + 2, (kb, -(-rows // per)), generator=g, device=DEV,
                           dtype=torch.uint8)
    return codes, scales


def _expert_rows(n):
    """Rows that an expert's matrix takes in the stack: scales are of 128 whole rows."""
    return -(-n // GROUP) * GROUP


def _affine(g, kind, cols):
    """Weight and bias of a norm (rms: no bias)."""
    if kind == "none":
        return None, None
    w = 1 + 0.2 * _randn(g, cols)
    return w, (0.1 * _randn(g, cols) if kind == "layer" else None)


def prepare(case, seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    st = dict(case)
    {"norm": _prepare_norm, "rotary": _prepare_rotary, "route": _prepare_route,
     "linear": _prepare_linear, "ffn": _prepare_ffn}[case["kind"]](case, st, g)
    if own:
        _handles(st)
    return st


def _prepare_norm(case, st, g):
    rows, cols, items = case["rows"], case["cols"], case["items"]
    xt = TYPES[case["x"]]
    # residual streams grow a few large channels
    st["xin"] = (2 * _randn(g, rows, cols) * torch.exp(0.5 * _randn(g, cols))).to(xt)
    st["hin"] = (_randn(g, rows, cols) + 0.3).to(TYPES[case["h"]]) if case["h"] else None
    st["xout"] = torch.zeros(rows, cols, dtype=xt, device=DEV) if case["h"] else None
    st["yout"] = torch.zeros(rows, cols, dtype=TYPES[case["y"]], device=DEV)
    st["pw"], st["pb"] = _affine(g, case["post"] if case["h"] else "none", cols)
    st["nw"], st["nb"] = _affine(g, case["pre"], cols)
    # modulations of each item: gate | scale | shift in one row
    st["mods"] = 0.4 * _randn(g, items, 3 * cols)
    st["offsets"] = _ints(_item_rows(case))


def _prepare_rotary(case, st, g):
    rows, wide = case["rows"], case["heads"] * case["dh"]
    st["xin"] = _randn(g, rows, wide + case["pad"]).to(TYPES[case["dtype"]])[:, :wide]
    st["yout"] = torch.zeros(rows, wide, dtype=TYPES[case["dtype"]], device=DEV)
    st["at"] = torch.randint(0, case["longest"], (rows, case["axes"]), generator=g, device=DEV,
                             dtype=torch.int32)


def _outputs_of_routing(st, rows, k, experts):
    st["ids"] = torch.zeros(rows, k, dtype=torch.int32, device=DEV)
    st["w"] = torch.zeros(rows, k, device=DEV)
    st["first"] = torch.zeros(experts + 1, dtype=torch.int32, device=DEV)
    st["source"] = torch.zeros(rows * k, dtype=torch.int32, device=DEV)
    st["places"] = torch.zeros(rows, k, dtype=torch.int32, device=DEV)


def _prepare_route(case, st, g):
    st["z"] = _logits(g, case)
    st["balance"] = 0.2 * _randn(g, case["experts"]) if case["bias"] else None
    _outputs_of_routing(st, case["rows"], case["k"], case["experts"])


def _prepare_linear(case, st, g):
    pairs, e, cols, n = case["rows"] * case["k"], case["experts"], case["cols"], case["n"]
    wide = n * _wide(case["act"])
    st["x"], st["xs"] = _matrix(g, case["rows"] if case["gather"] else pairs, cols, 1)
    st["W"], st["Ws"] = _matrix(g, e * _expert_rows(wide), cols, GROUP, -0.5 * math.log2(cols))
    st["b"] = 0.3 * _randn(g, e, wide) if case["bias"] else None
    shares = _shares(case)
    st["first"] = torch.nn.functional.pad(_ints(shares).cumsum(0), (1, 0)).int()
    st["source"] = None
    if case["gather"]:  # each expert's rows in ascending order
        turn = torch.randperm(case["rows"], generator=g, device=DEV).repeat(case["k"])
        e_of = torch.repeat_interleave(torch.arange(e, device=DEV), _ints(shares).long(),
                                       output_size=pairs)
        st["source"] = turn[torch.argsort(e_of * case["rows"] + turn)].int()
    st["most"] = max(shares)
    st["y"] = torch.zeros(pairs, n, dtype=TYPES[case["out"]], device=DEV)


def _prepare_ffn(case, st, g):
    rows, k, e, cols, mlp = (case[i] for i in ("rows", "k", "experts", "cols", "mlp"))
    wide = mlp * _wide(case["act"])
    st["xin"] = (2 * _randn(g, rows, cols) * torch.exp(0.5 * _randn(g, cols))).bfloat16()
    st["xout"] = torch.zeros(rows, cols, dtype=torch.bfloat16, device=DEV)
    st["nw"] = 1 + 0.2 * _randn(g, cols)
    st["gate"] = 3 * _randn(g, 1, cols)
    st["z"] = _logits(g, case)
    st["W1"], st["W1s"] = _matrix(g, e * _expert_rows(wide), cols, GROUP, -0.5 * math.log2(cols))
    st["W2"], st["W2s"] = _matrix(g, e * _expert_rows(cols), mlp, GROUP, -0.5 * math.log2(mlp))
    st["b1"] = 0.3 * _randn(g, e, wide)
    _outputs_of_routing(st, rows, k, e)
    # the most rows of an expert, as large as the plain form lays each of them out
    ids, _ = _choose(st["z"], st, None)
    st["most"] = int(torch.bincount(ids.reshape(-1), minlength=e).max())


def _rotary_spec(c):
    """Rotations a position of each pair of channels, in radians (float64), and its axis."""
    pairs = c["rot"] // 2
    of = [pairs - pairs // 2, pairs // 2] if c["axes"] == 2 else [pairs]
    theta = 10000.0 if c["axes"] == 1 else 100.0
    return of, theta


EPS = 1e-6
NATIVE, FAST, SLOW = 4096.0, 4.0, 1.0   # of scaled rotary positions


def _handles(st):
    """The context, structures and buffers that a user's program keeps."""
    from paper_2608_29809_gb300 import regioncache as R
    from paper_2608_29809_gb300 import synth
    global _ctx
    if _ctx is None:
        _ctx = R.rc_create(R.dims_struct(synth.Dims(hidden=128, heads=2, mlp=128, layers=1,
                                                    grid_h=4, grid_w=4, timesteps=1)))
    st["R"], st["ctx"], kind = R, _ctx, st["kind"]
    norms = {"layer": R.RC_NORM_LAYER, "rms": R.RC_NORM_RMS}

    def norm(kind, w, b):
        return R.Norm(norms[kind], EPS, w, b) if kind != "none" else None

    if kind == "norm":
        cols, mods = st["cols"], st["mods"]
        st["op"] = R.ResidualNorm(
            cols, x=st["xin"], h=st["hin"], x_out=st["xout"], y=st["yout"],
            post=norm(st["post"], st["pw"], st["pb"]) if st["h"] else None,
            pre=norm(st["pre"], st["nw"], st["nb"]),
            gate=mods[:, :cols] if st["gate"] and st["h"] else None,
            scale=mods[:, cols:2 * cols] if st["mod"] else None,
            shift=mods[:, 2 * cols:] if st["mod"] else None,
            residual_scale=st["scale"], row_offsets=st["offsets"])
    elif kind == "rotary":
        of, theta = _rotary_spec(st)
        st["plan"] = R.Rotary(
            st["rot"], theta, pairs=of,
            layout=R.RC_ROTARY_HALF if st["layout"] == "half" else R.RC_ROTARY_PAIRS,
            scaling={"none": R.RC_ROTARY_PLAIN, "linear": R.RC_ROTARY_LINEAR,
                     "base": R.RC_ROTARY_BASE, "bands": R.RC_ROTARY_BANDS,
                     "ramp": R.RC_ROTARY_RAMP}[st["scaling"]],
            factor=st["factor"], native_length=NATIVE, fast=FAST, slow=SLOW,
            amplitude=_amplitude(st))
    scores = {"softmax": R.RC_SCORE_SOFTMAX, "sigmoid": R.RC_SCORE_SIGMOID}
    if kind == "route":
        st["routing"] = R.Routing(st["experts"], st["k"], scores[st["score"]],
                                  bias=st["balance"], groups=st["groups"],
                                  top_groups=st["best"], group_best=st["of_best"],
                                  renormalise=st["renorm"])
    acts = {"none": R.RC_ACT_NONE, "gelu": R.RC_ACT_GELU, "silu": R.RC_ACT_SILU,
            "gated_silu": R.RC_ACT_GATED_SILU}
    if kind == "linear":
        st["x8"] = R.Fp8Matrix.of(st["x"], st["xs"], st["cols"], 1)
        st["W8"] = R.Fp8Matrix.of(st["W"], st["Ws"], st["cols"], GROUP)
        st["act_"] = acts[st["act"]]
    if kind == "ffn":
        rows, k, cols, mlp = st["rows"], st["k"], st["cols"], st["mlp"]
        st["act_"] = acts[st["act"]]
        st["routing"] = R.Routing(st["experts"], k, scores[st["score"]])
        st["W18"] = R.Fp8Matrix.of(st["W1"], st["W1s"], cols, GROUP)
        st["W28"] = R.Fp8Matrix.of(st["W2"], st["W2s"], mlp, GROUP)
        st["n8"], st["u8"] = R.Fp8Matrix(rows, cols), R.Fp8Matrix(rows * k, mlp)
        st["d"] = torch.zeros(rows * k, cols, device=DEV)
        st["before"] = R.ResidualNorm(cols, x=st["xin"], y=st["n8"],
                                      pre=R.Norm(R.RC_NORM_RMS, EPS, st["nw"], None))
        st["after"] = R.ResidualNorm(cols, x=st["xin"], h=st["d"], places=st["places"],
                                     weights=st["w"], gate=st["gate"], x_out=st["xout"])


_ctx = None


# ------------------------------------------------------------------ a pass
def run(state):
    if own:
        return _run_own(state)
    return {"norm": _plain_norm, "rotary": _plain_rotary, "route": _plain_route,
            "linear": _plain_linear, "ffn": _plain_ffn}[state["kind"]](state)


def _run_own(st):
    R, ctx, kind = st["R"], st["ctx"], st["kind"]
    if kind == "norm":
        R.rc_norm_residual(ctx, st["op"])
        return [t for t in (st["xout"], st["yout"]) if t is not None]
    if kind == "rotary":
        R.rc_rotary_apply(ctx, st["plan"], st["xin"], st["xin"].stride(0),
                          R.DTYPES[st["xin"].dtype], st["rows"], st["heads"], st["dh"], st["at"],
                          None, False, st["yout"], st["heads"] * st["dh"])
        return st["yout"]
    if kind in ("route", "ffn"):
        rows, k, e = st["rows"], st["k"], st["experts"]
        if kind == "ffn":
            R.rc_norm_residual(ctx, st["before"])
        R.rc_experts_route(ctx, st["routing"], st["z"], e, R.DTYPES[st["z"].dtype], rows, None,
                           st["ids"], st["w"])
        R.rc_experts_sort(ctx, st["ids"], rows, k, e, None, st["first"], st["source"],
                          st["places"])
        if kind == "route":
            return st["ids"], st["w"], st["first"], st["source"], st["places"]
        R.rc_experts_linear(ctx, st["n8"], st["W18"], st["b1"], e, st["mlp"], st["first"],
                            st["source"], rows * k, st["act_"], None, 0, 0, st["u8"])
        R.rc_experts_linear(ctx, st["u8"], st["W28"], None, e, st["cols"], st["first"], None,
                            rows * k, R.RC_ACT_NONE, st["d"], st["cols"], R.RC_F32)
        R.rc_norm_residual(ctx, st["after"])
        return st["xout"]
    R.rc_experts_linear(ctx, st["x8"], st["W8"], st["b"], st["experts"], st["n"], st["first"],
                        st["source"], st["rows"] * st["k"], st["act_"], st["y"], st["n"],
                        R.DTYPES[st["y"].dtype])
    return st["y"]


def _plain_norm_of(kind, v, w, b):
    if kind == "none":
        return v
    if kind == "layer":
        v = v - v.mean(1, keepdim=True)
    v = v * torch.rsqrt((v * v).mean(1, keepdim=True) + EPS) * w
    return v if b is None else v + b


def _plain_norm(st):
    rows, cols = st["rows"], st["cols"]
    item = torch.searchsorted(st["offsets"][1:].contiguous(),
                              torch.arange(rows, device=DEV, dtype=torch.int32), right=True)
    x = st["xin"].float()
    out = []
    if st["h"]:
        r = _plain_norm_of(st["post"], st["hin"].float(), st["pw"], st["pb"])
        if st["gate"]:
            r = r * st["mods"][:, :cols][item]
        x = st["scale"] * x + r
        st["xout"].copy_(x)
        out.append(st["xout"])
    y = _plain_norm_of(st["pre"], x, st["nw"], st["nb"])
    if st["mod"]:
        y = y * (1 + st["mods"][:, cols:2 * cols][item]) + st["mods"][:, 2 * cols:][item]
    st["yout"].copy_(y)
    return out + [st["yout"]]


def _frequencies(c):
    """Radians a position of each pair (f64), and the axis whose position it takes."""
    of, theta = _rotary_spec(c)
    freq, axis = [], []
    for a, n in enumerate(of):
        i = torch.arange(n, dtype=torch.float64, device=DEV)
        base = theta
        if c["scaling"] == "base" and n > 1:
            base = theta * c["factor"] ** (n / (n - 1))
        f = base ** (-i / n)
        if c["scaling"] == "linear":
            f = f / c["factor"]
        if c["scaling"] in ("bands", "ramp"):
            if c["scaling"] == "bands":  # by the turns that a pair makes over the native length
                keep = (NATIVE * f / (2 * math.pi) - SLOW) / (FAST - SLOW)
            else:  # by the pair's index between those that make FAST and SLOW turns
                lo, hi = (n * math.log(NATIVE / (t * 2 * math.pi)) / math.log(theta)
                          for t in (FAST, SLOW))
                lo, hi = max(math.floor(lo), 0), min(math.ceil(hi), n - 1)
                keep = 1 - (i - lo) / max(hi - lo, 0.001)
            keep = keep.clamp(0, 1)
            f = keep * f + (1 - keep) * f / c["factor"]
        freq.append(f)
        axis += [a] * n
    return torch.cat(freq), torch.tensor(axis, device=DEV)


def _amplitude(c):
    return 0.1 * math.log(c["factor"]) + 1.0 if c["scaling"] == "ramp" else 1.0


def _plain_rotary(st):
    freq, axis = _frequencies(st)
    angle = st["at"].double()[:, axis] * freq
    cos = (torch.cos(angle) * _amplitude(st)).float()[:, None]
    sin = (torch.sin(angle) * _amplitude(st)).float()[:, None]
    x, rot = st["xin"].float().reshape(st["rows"], st["heads"], st["dh"]), st["rot"]
    y = x.clone()
    if st["layout"] == "half":
        a, b = slice(0, rot // 2), slice(rot // 2, rot)
    else:
        a, b = slice(0, rot, 2), slice(1, rot, 2)
    y[..., a] = x[..., a] * cos - x[..., b] * sin
    y[..., b] = x[..., b] * cos + x[..., a] * sin
    st["yout"].copy_(y.view(st["rows"], -1))
    return st["yout"]


def _choose(z, c, bias):
    """ids (-1: none) and weights (f64) of each row's experts."""
    rows, e, k = z.shape[0], c["experts"], c["k"]
    z = z.double().clamp(max=BIG)
    there = z > -math.inf
    if c["score"] == "softmax":
        s = torch.exp(z - z.amax(1, keepdim=True).clamp(min=-BIG))
        s = s / s.sum(1, keepdim=True)
    else:
        s = 1 / (1 + torch.exp(-z))
    choice = torch.where(there, s if bias is None else s + bias.double(), -math.inf)
    if c.get("groups", 1) > 1:
        parts = choice.view(rows, c["groups"], -1)
        top = torch.sort(parts, dim=2, descending=True).values[:, :, :c["of_best"]]
        value = torch.where(top > -math.inf, top, 0.0).sum(2)
        value = torch.where(top[:, :, 0] > -math.inf, value, -math.inf)
        order = torch.sort(value, dim=1, descending=True, stable=True).indices[:, :c["best"]]
        keep = torch.zeros_like(value, dtype=torch.bool).scatter_(1, order, True)
        choice = torch.where(keep[:, :, None], parts, -math.inf).view(rows, e)
    best, ids = torch.sort(choice, dim=1, descending=True, stable=True)
    best, ids = best[:, :k], ids[:, :k]
    w = torch.where(best > -math.inf, s.gather(1, ids), 0.0)
    if c.get("renorm", True):
        total = w.sum(1, keepdim=True)
        w = torch.where(total > 0, w / total, 0.0)
    return torch.where(best > -math.inf, ids, -1).int(), w


def _sorted_by_expert(ids, experts):
    """Rows of each expert (offsets), the row of each place, the place of each pair."""
    rows, k = ids.shape
    flat = ids.reshape(-1)
    order = torch.argsort(torch.where(flat < 0, experts, flat), stable=True)
    first = torch.searchsorted(torch.where(flat < 0, experts, flat)[order].contiguous(),
                               torch.arange(experts + 1, device=ids.device, dtype=torch.int32))
    places = torch.empty_like(flat).scatter_(
        0, order, torch.arange(rows * k, device=ids.device, dtype=torch.int32))
    return first.int(), (order // k).int(), torch.where(flat < 0, -1, places).view(rows, k)


def _plain_route(st):
    ids, w = _choose(st["z"], st, st["balance"])
    first, source, places = _sorted_by_expert(ids, st["experts"])
    st["ids"].copy_(ids)
    st["w"].copy_(w)
    st["first"].copy_(first)
    # (what stands behind the last place is left as it was)
    st["source"].copy_(torch.where(torch.arange(len(source), device=DEV) < first[-1], source,
                                   st["source"]))
    st["places"].copy_(places)
    return st["ids"], st["w"], st["first"], st["source"], st["places"]


def _power(byte):
    """2^(byte - 127) in f32 (bytes of 1 and more)."""
    return (byte.int() << 23).view(torch.float32)


def _dense(codes, scales, cols, per):
    s = _power(scales).t().repeat_interleave(per, 0)[:len(codes)]
    return codes.view(E4M3)[:, :cols].float() * s.repeat_interleave(GROUP, 1)[:, :cols]


def _coded(v):
    """v (f32) through e4m3 codes with a scale for each 128 columns, as the values they stand
    for."""
    rows, cols = v.shape
    kb = -(-cols // GROUP)
    tiles = torch.nn.functional.pad(v, (0, kb * GROUP - cols)).view(rows, kb, GROUP)
    bits = tiles.abs().amax(2).view(torch.int32)
    e = ((bits >> 23) - 8 + ((bits & 0x7FFFFF) > 0x600000).int()).clamp(min=1)
    q = (tiles * ((254 - e) << 23).view(torch.float32)[:, :, None]).to(E4M3).float()
    return (q * _power(e)[:, :, None]).view(rows, -1)[:, :cols]


def _act(name, v):
    if name == "gelu":
        return 0.5 * v * (1 + torch.tanh(math.sqrt(2 / math.pi) * (v + 0.044715 * v * v * v)))
    if name == "silu":
        return v / (1 + torch.exp(-v))
    if name == "gated_silu":
        a, b = v.chunk(2, -1)
        return a / (1 + torch.exp(-a)) * b
    return v


def _by_expert(x, W, b, first, most, experts, wide):
    """x [pairs][cols] in order of the experts times their matrices: [pairs][wide]."""
    at = torch.arange(len(x), device=DEV, dtype=torch.int32)
    e = torch.searchsorted(first[1:].contiguous(), at, right=True).clamp(max=experts - 1)
    i = at - first[e]
    rows = torch.zeros(experts, most, x.shape[1], device=DEV)
    rows[e, i] = x
    y = rows @ W.view(experts, -1, W.shape[1])[:, :wide].transpose(1, 2)
    return y[e, i] if b is None else y[e, i] + b[e]


def _plain_linear(st):
    x = _dense(st["x"], st["xs"], st["cols"], 1)
    x = x if st["source"] is None else x[st["source"].long()]
    W = _dense(st["W"], st["Ws"], st["cols"], GROUP)
    y = _by_expert(x, W, st["b"], st["first"], st["most"], st["experts"],
                   st["n"] * _wide(st["act"]))
    st["y"].copy_(_act(st["act"], y))
    return st["y"]


def _plain_ffn(st):
    rows, k, e, cols, mlp = (st[i] for i in ("rows", "k", "experts", "cols", "mlp"))
    x = st["xin"].float()
    n = _coded(_plain_norm_of("rms", x, st["nw"], None))
    ids, w = _choose(st["z"], st, None)
    first, source, places = _sorted_by_expert(ids, e)
    u = _by_expert(n[source.long()], _dense(st["W1"], st["W1s"], cols, GROUP), st["b1"], first,
                   st["most"], e, mlp * _wide(st["act"]))
    u = _coded(_act(st["act"], u))
    d = _by_expert(u, _dense(st["W2"], st["W2s"], mlp, GROUP), None, first, st["most"], e,
                   cols)
    r = (d[places.long()] * w.float()[:, :, None]).sum(1)
    st["xout"].copy_(x + st["gate"] * r)
    return st["xout"]


# ------------------------------------------------------ float64 definition
def exact(case, seed):
    global own
    was, own = own, False
    try:
        st = prepare(case, seed)
    finally:
        own = was
    return {"norm": _exact_norm, "rotary": _exact_rotary, "route": _exact_route,
            "linear": _exact_linear, "ffn": _exact_ffn}[case["kind"]](st)


def _exact_normed(kind, v, w, b):
    if kind == "none":
        return v
    if kind == "layer":
        var, mean = torch.var_mean(v, 1, correction=0, keepdim=True)
        return (v - mean) / torch.sqrt(var + EPS) * w.double() + b.double()
    return v / torch.sqrt(v.square().mean(1, keepdim=True) + EPS) * w.double()


def _exact_norm(st):
    cols, ends = st["cols"], st["offsets"].tolist()
    mods = st["mods"].double()
    outs = []
    for i, (a, b) in enumerate(zip(ends, ends[1:])):
        x = st["xin"][a:b].double()
        piece = []
        if st["h"]:
            r = _exact_normed(st["post"], st["hin"][a:b].double(), st["pw"], st["pb"])
            x = st["scale"] * x + (r * mods[i, :cols] if st["gate"] else r)
            piece.append(x)
        y = _exact_normed(st["pre"], x, st["nw"], st["nb"])
        if st["mod"]:
            y = y + y * mods[i, cols:2 * cols] + mods[i, 2 * cols:]
        outs.append(piece + [y])
    return [torch.cat(t) for t in zip(*outs)]


def _exact_rotary(st):
    """Each pair as a complex number times amplitude * e^(i position f)."""
    freq, axis = _frequencies(st)
    turn = torch.polar(torch.full((st["rows"], len(freq)), _amplitude(st), dtype=torch.float64,
                                  device=DEV), st["at"].double()[:, axis] * freq)
    x = st["xin"].double().reshape(st["rows"], st["heads"], st["dh"])
    head, rest = x[..., :st["rot"]], x[..., st["rot"]:]
    if st["layout"] == "half":
        z = torch.complex(*head.chunk(2, -1)) * turn[:, None]
        out = torch.cat([z.real, z.imag, rest], -1)
    else:
        z = torch.view_as_complex(head.unflatten(-1, (-1, 2)).contiguous()) * turn[:, None]
        out = torch.cat([torch.view_as_real(z).flatten(-2), rest], -1)
    return out.reshape(st["rows"], -1)


def _exact_route(st):
    """Row by row where that is quick: the scores as they are defined, a pick at a time."""
    z, c = st["z"].double().cpu(), st
    if z.numel() > 200000:
        return None
    bias = torch.zeros(c["experts"], dtype=torch.float64) if st["balance"] is None else \
        st["balance"].double().cpu()
    ids, weights = torch.full((c["rows"], c["k"]), -1, dtype=torch.int32), []
    for r in range(c["rows"]):
        p = torch.softmax(z[r], 0) if c["score"] == "softmax" else torch.sigmoid(z[r])
        there = [i for i in range(c["experts"]) if z[r, i] > -math.inf]
        pick = {i: float(p[i] + bias[i]) for i in there}
        if c["groups"] > 1:
            per = c["experts"] // c["groups"]
            value = {}
            for i in there:
                value.setdefault(i // per, []).append(pick[i])
            value = {q: sum(sorted(v)[::-1][:c["of_best"]]) for q, v in value.items()}
            kept = sorted(value, key=lambda q: (-value[q], q))[:c["best"]]
            pick = {i: v for i, v in pick.items() if i // per in kept}
        got = sorted(pick, key=lambda i: (-pick[i], i))[:c["k"]]
        w = torch.zeros(c["k"], dtype=torch.float64)
        for j, i in enumerate(got):
            ids[r, j], w[j] = i, p[i]
        weights.append(w / w.sum() if c["renorm"] and got else w)
    return ids, torch.stack(weights), None, None, None


def _two(byte):
    return torch.exp2(byte.double() - 127)


def _exact_values(codes, scales, cols, per):
    v = codes.view(E4M3)[:, :cols].double()
    for b in range(scales.shape[0]):
        v[:, b * GROUP:(b + 1) * GROUP] *= _two(scales[b]).repeat_interleave(per)[:len(v), None]
    return v


def _exact_codes(v):
    """v through e4m3 codes (nearest, ties to even) with the least scale of 128 columns."""
    out = torch.zeros_like(v)
    for b in range(0, v.shape[1], GROUP):
        part = v[:, b:b + GROUP]
        top = part.abs().amax(1, keepdim=True)
        e = torch.ceil(torch.log2((top / 448).clamp(min=2.0 ** -126)))
        e = torch.where(top <= 448 * torch.exp2(e - 1), e - 1, e)
        e = torch.where(top > 448 * torch.exp2(e), e + 1, e)
        q = part * torch.exp2(-e)
        step = torch.exp2(torch.floor(torch.log2(q.abs().clamp(min=2.0 ** -6))) - 3)
        out[:, b:b + GROUP] = torch.round(q / step) * step * torch.exp2(e)
    return out


def _exact_act(name, v):
    n = v.shape[1] // 2
    if name == "gelu":
        # 0.5 (1 + tanh a) = sigmoid(2 a)
        return v * torch.sigmoid(2 * math.sqrt(2 / math.pi) * (v + 0.044715 * v ** 3))
    if name == "silu":
        return v * torch.sigmoid(v)
    if name == "gated_silu":
        return v[:, :n] * torch.sigmoid(v[:, :n]) * v[:, n:]
    return v


def _exact_product(x, st, names, b, e, wide, cols):
    codes, scales = (st[n] for n in names)
    per = codes.shape[0] // st["experts"]
    W = _exact_values(codes[e * per:(e + 1) * per],
                      scales[:, e * per // GROUP:(e + 1) * per // GROUP], cols, GROUP)[:wide]
    y = x @ W.t()
    return y if b is None else y + b[e].double()


def _exact_linear(st):
    x = _exact_values(st["x"], st["xs"], st["cols"], 1)
    ends, parts = st["first"].tolist(), []
    for e, (a, b) in enumerate(zip(ends, ends[1:])):
        rows = x[a:b] if st["source"] is None else x[st["source"][a:b].long()]
        y = _exact_product(rows, st, ("W", "Ws"), st["b"], e, st["n"] * _wide(st["act"]),
                           st["cols"])
        parts.append(_exact_act(st["act"], y))
    return torch.cat(parts)


def _exact_ffn(st):
    cols, mlp = st["cols"], st["mlp"]
    x = st["xin"].double()
    n = _exact_codes(_exact_normed("rms", x, st["nw"], None))
    p = torch.softmax(st["z"].double(), 1) if st["score"] == "softmax" else \
        torch.sigmoid(st["z"].double())
    top = torch.topk(p, st["k"], 1)
    share = top.values / top.values.sum(1, keepdim=True)
    out = torch.zeros_like(x)
    for e in range(st["experts"]):
        row, j = torch.nonzero(top.indices == e, as_tuple=True)
        if not len(row):
            continue
        u = _exact_product(n[row], st, ("W1", "W1s"), st["b1"], e, mlp * _wide(st["act"]), cols)
        u = _exact_codes(_exact_act(st["act"], u))
        d = _exact_product(u, st, ("W2", "W2s"), None, e, cols, mlp)
        out.index_add_(0, row, d * share[row, j][:, None])
    return x + st["gate"].double() * out
