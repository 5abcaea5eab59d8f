"""The rest of a block in 64 bits, from the definitions of the header, on the
CPU: norms with gate and residual, rotary positions (test helper)."""
import math

import torch

F32_HALF = 2.0 ** -24  # half a step of f32, relative


def rounding(dtype):
    """Largest relative error of a rounding to the type."""
    return torch.finfo(dtype).eps / 2


def norm(kind, eps, w, b, v, dv):
    """A norm of the rows of v (f64), and how far f32 may be off where v is off by dv: sums of n
    terms in at most n / 32 + 16 steps (each 2^-24 of the magnitudes added), the difference and
    root of the statistics, three more roundings."""
    if kind == "none":
        return v, dv
    n = v.shape[1]
    steps = (n / 32 + 16) * F32_HALF
    mean = v.mean(1, keepdim=True) if kind == "layer" else torch.zeros(len(v), 1).double()
    dmean = steps * v.abs().mean(1, keepdim=True) + dv.mean(1, keepdim=True)
    d = v - mean
    dd = dv + (dmean if kind == "layer" else 0) + F32_HALF * d.abs()
    var = (d * d).mean(1, keepdim=True)
    r = 1 / torch.sqrt(var + eps)
    # of the variance, relative; a row whose differences are all error has none to speak of
    dvar = steps + ((2 * d.abs() * dd + dd * dd).mean(1, keepdim=True) / (var + eps))
    w = torch.ones(n).double() if w is None else w.cpu().double()
    b = torch.zeros(n).double() if b is None else b.cpu().double()
    y = d * r * w + b
    return y, (dd + d.abs() * (dvar + 8 * F32_HALF)) * r * w.abs() + 2 * F32_HALF * y.abs()


def residual(x, branch, dbranch, gate, a, post, pre, scale, shift):
    """x', y of rows (f64) and their tolerances before they are rounded.  branch None: none."""
    dx = torch.zeros_like(x)
    x1 = a * x
    if branch is not None:
        r, dr = norm(*post, branch, dbranch)
        g = torch.ones(x.shape[1]).double() if gate is None else gate
        x1 = x1 + g * r
        dx = 3 * F32_HALF * ((a * x).abs() + (g * r).abs()) + g.abs() * dr
    else:
        dx = F32_HALF * x1.abs()
    y, dy = norm(*pre, x1, dx)
    s = 0 if scale is None else scale
    t = torch.zeros(x.shape[1]).double() if shift is None else shift
    out = y * (1 + s) + t
    factor = (1 + s) if scale is not None else torch.ones(x.shape[1]).double()
    return x1, dx, out, dy * factor.abs() + 3 * F32_HALF * (y.abs() * (1 + abs(s)) + t.abs())


def close(got, want, tol, dtype, what=""):
    """Within tol before the rounding to dtype and half a step (and the least subnormal) after."""
    got = got.cpu().double()
    limit = tol + rounding(dtype) * (want.abs() + tol) + 1e-37
    bad = ~((got - want).abs() <= limit)
    most = float(((got - want).abs() / limit).max()) if got.numel() else 0.0
    assert not bool(bad.any()), \
        f"{what}: {int(bad.sum())} of {bad.numel()} off, at most {most:.2f} of the limit"


def frequencies(pairs, theta, scaling="plain", factor=1.0, native=0.0, fast=0.0, slow=0.0):
    """Radians a position of every pair, and its axis."""
    f, axis = [], []
    for a, n in enumerate(pairs):
        base = theta * factor ** (n / (n - 1)) if scaling == "base" and n > 1 else theta
        if scaling == "ramp":
            at = [n * math.log(native / (2 * math.pi * t)) / math.log(base) for t in (fast, slow)]
            lo, hi = max(math.floor(at[0]), 0), min(math.ceil(at[1]), n - 1)
        for i in range(n):
            v = base ** (-i / n)
            keep = 1.0
            if scaling == "linear":
                keep = 0.0
            if scaling == "bands":
                keep = (native * v / (2 * math.pi) - slow) / (fast - slow)
            if scaling == "ramp":
                keep = 1 - (i - lo) / max(hi - lo, 0.001)
            keep = min(max(keep, 0.0), 1.0)
            f.append(keep * v + (1 - keep) * v / factor)
            axis.append(a)
    return f, axis


def rotate(x, positions, f, axis, first, half_layout, amplitude=1.0, inverse=False):
    """x [rows][heads][head_dim] turned (f64), each pair as a complex number."""
    rot = 2 * len(f)
    at = positions.cpu().double()[:, axis] * torch.tensor(f, dtype=torch.float64)
    turn = amplitude * torch.exp(1j * (-at if inverse else at))[:, None]
    y = x.clone()
    part = x[..., first:first + rot]
    a, b = (part.chunk(2, -1)) if half_layout else (part[..., 0::2], part[..., 1::2])
    z = torch.complex(a.contiguous(), b.contiguous()) * turn
    if half_layout:
        y[..., first:first + rot] = torch.cat([z.real, z.imag], -1)
    else:
        y[..., first:first + rot] = torch.view_as_real(z).flatten(-2)
    return y


BIG = torch.finfo(torch.float32).max


def route(z, score, k, bias=None, groups=1, top_groups=1, group_best=1, renormalise=True,
          scale=1.0):
    """ids and weights (f64) of the rows' experts."""
    z = z.cpu().double().clamp(max=BIG)
    rows, e = z.shape
    b = torch.zeros(e).double() if bias is None else bias.cpu().double().clamp(max=BIG)
    there = (z > -math.inf) & (b > -math.inf)
    z = torch.where(there, z, -math.inf)
    if score == "softmax":
        s = torch.exp(z - z.amax(1, keepdim=True).clamp(min=-BIG))
        s = s / s.sum(1, keepdim=True)
    else:
        s = 1 / (1 + torch.exp(-z))
    ids, w = torch.full((rows, k), -1), torch.zeros(rows, k).double()
    # (without a bias larger logits have larger scores, also where f64 has them equal)
    plain = bias is None and (top_groups == groups or group_best == 1)
    value = z if plain else s + b
    size = e // groups
    for r in range(rows):
        left = [i for i in range(e) if there[r, i]]
        if top_groups < groups:
            of = {}
            for i in left:
                of.setdefault(i // size, []).append(float(value[r, i]))
            worth = {g: sum(sorted(v, reverse=True)[:group_best]) for g, v in of.items()}
            best = sorted(worth, key=lambda g: (-worth[g], g))[:top_groups]
            left = [i for i in left if i // size in best]
        chosen = sorted(left, key=lambda i: (-float(value[r, i]), i))[:k]
        for j, i in enumerate(chosen):
            ids[r, j], w[r, j] = i, s[r, i]
    if renormalise:
        total = w.sum(1, keepdim=True)
        w = torch.where(total > 0, w / total, 0.0)
    return ids.int(), w * scale


def sort(ids, experts):
    """Offsets, rows in order of the experts, places of the pairs."""
    rows, k = ids.shape
    pairs = [(e, i) for i, e in enumerate(ids.flatten().tolist()) if 0 <= e < experts]
    pairs.sort()
    offsets = [0] * (experts + 1)
    for e, _ in pairs:
        offsets[e + 1] += 1
    for e in range(experts):
        offsets[e + 1] += offsets[e]
    places = torch.full((rows * k,), -1, dtype=torch.int32)
    source = torch.zeros(len(pairs), dtype=torch.int32)
    for p, (_, i) in enumerate(pairs):
        places[i], source[p] = p, i // k
    return torch.tensor(offsets, dtype=torch.int32), source, places.view(rows, k)
