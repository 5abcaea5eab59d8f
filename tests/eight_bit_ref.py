"""Eight-bit serving in 64 bits, from the definitions of the header, on the
CPU: the quantiser, the cache store and the attention (test helper)."""
import math

import torch

F8 = torch.float8_e4m3fn
BLOCK = 64


def scale_exponent(top):
    """The least e >= -127 with top <= 448 * 2^e for every value of `top` (finite, f64)."""
    e = torch.full(top.shape, -127.0, dtype=torch.float64)
    m, x = torch.frexp(top / 448)  # m in [0.5, 1): top <= 448 * 2^x, less than half only at m = 0.5
    x = torch.where(m == 0.5, x - 1, x).double()
    return torch.where(top > 0, torch.maximum(x, e), e)


def e4m3(v):
    """Nearest e4m3 value, ties to the even mantissa (f64 in, f64 out)."""
    _, x = torch.frexp(v)
    step = torch.exp2((x.double() - 1).clamp(min=-6) - 3)
    return torch.round(v / step) * step


def quantize(x, group):
    """Values of the codes [rows][cols] (f64) and the scale bytes [kb][groups] of x."""
    x = x.cpu().double()
    rows, cols = x.shape
    kb, gs = -(-cols // 128), -(-rows // group)
    codes, scales = torch.zeros(rows, cols, dtype=torch.float64), torch.zeros(kb, gs).byte()
    for b in range(kb):
        for g in range(gs):
            part = x[g * group:(g + 1) * group, b * 128:(b + 1) * 128]
            at = codes[g * group:(g + 1) * group, b * 128:(b + 1) * 128]
            if not bool(torch.isfinite(part).all()):
                scales[b, g] = 255
                at.fill_(math.nan)
                continue
            e = scale_exponent(part.abs().max())
            scales[b, g] = int(e) + 127
            at.copy_(e4m3(part * torch.exp2(-e)))
    return codes, scales


def values(codes, scales, group, cols):
    """Codes times scales of a quantised matrix, f64."""
    c = codes[:, :cols].cpu().view(F8).double()
    s = torch.exp2(scales.cpu().double() - 127)
    s = torch.where(scales.cpu() == 255, math.nan, s).t()
    return c * s.repeat_interleave(group, 0)[:len(c)].repeat_interleave(128, 1)[:, :cols]


def cache_values(codes, scales):
    s = torch.where(scales.cpu() == 255, math.nan, torch.exp2(scales.cpu().double() - 127))
    return codes.cpu().view(F8).double() * s[:, :, None, None]


def store(codes, scales, x, slots, append):
    """One side of rc_kv8_store on f64 code values [blocks][heads][64][dh] and bytes, in place.
    x f64 [n][heads][dh]."""
    slots = [int(s) for s in slots]
    for block in sorted({s // BLOCK for s in slots if s >= 0}):
        rows = [i for i, s in enumerate(slots) if s >= 0 and s // BLOCK == block]
        offs = [slots[i] % BLOCK for i in rows]
        fresh = append and 0 in offs
        for h in range(codes.shape[1]):
            part = x[rows, h]
            old = 0 if fresh else int(scales[block, h])
            if bool(torch.isfinite(part).all()) and old != 255:
                b = max(old, int(scale_exponent(part.abs().max())) + 127)
            else:
                b = 255
            if not fresh and b > old:
                move = math.nan if b == 255 else 2.0 ** (old - b)
                codes[block, h] = e4m3(codes[block, h] * move)
            codes[block, h, offs] = e4m3(part * (math.nan if b == 255 else 2.0 ** (127 - b)))
            scales[block, h] = b


def attention(q, k, v, causal):
    """Of one request and head, f64: q [n][dh], k, v [len][dh].  The result and the sums of
    p |v| and of |q| |k| that its tolerance counts with."""
    n, length = len(q), len(k)
    s = q @ k.t() / math.sqrt(q.shape[1])
    if causal:
        s = s.masked_fill(torch.ones(n, length).triu(length - n + 1).bool(), -math.inf)
    top = s.amax(1, keepdim=True).clamp(min=-1e300) if length else s.new_zeros(n, 1)
    p = torch.exp(s - top)
    p = p / p.sum(1, keepdim=True).clamp(min=1e-300)
    reach = (q.abs() @ k.abs().t() / math.sqrt(q.shape[1])).amax(1) if length else s.new_zeros(n)
    return p @ v, p @ v.abs(), reach


def attention_tolerance(o, pv, reach, dh):
    """bf16 weights (half a step, 2^-8) against their own sum, the rounded result (2^-8), scores
    summed in f32 (dh additions of at most 2^-23 of the magnitudes; the same again for the row's
    largest) and an exponential good to 2^-18."""
    return 2.0 ** -8 * o.abs() + (2.0 ** -8 + 2 * (dh + 4) * 2.0 ** -23 * reach[:, None] +
                                  2.0 ** -18) * pv + 1e-30
