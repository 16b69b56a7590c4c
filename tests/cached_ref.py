"""Plain 64-bit forms of the cached layer's operators (CPU), for the tests."""
import math

import torch

E4M3, INT8 = "e4m3", "int8"
BF16 = 2.0 ** -8      # half a step of bf16, relative
F32 = 2.0 ** -24      # half a step of fp32, relative


def rope(x, dims, grid, theta, halves, positions, text=0, transpose=False):
    """[B, H, L, d] rotated in 64 bits; positions [B, L - text]."""
    y = x.double().clone()
    B, _, L, _ = x.shape
    _, height, width = grid
    p = positions
    place = (p // (height * width), p // width % height, p % width)
    base = 0
    for a, w in enumerate(dims):
        for j in range(w // 2):
            i0, i1 = (base + j, base + j + w // 2) if halves else (base + 2 * j, base + 2 * j + 1)
            ang = place[a].double() * theta ** (-2.0 * j / w)
            c, s = ang.cos()[:, None], ang.sin()[:, None] * (-1 if transpose else 1)
            x0, x1 = x[:, :, :L - text, i0].double(), x[:, :, :L - text, i1].double()
            y[:, :, :L - text, i0] = x0 * c - x1 * s
            y[:, :, :L - text, i1] = x1 * c + x0 * s
        base += w
    return y


def numbers(codes, fmt):
    return codes.view(torch.int8 if fmt == INT8 else torch.float8_e4m3fn).double()


def scale_of(amax, fmt):
    """amax: a Python float; the scale as a float."""
    if not math.isfinite(amax):
        return math.nan
    if amax == 0:
        return 0.0
    if fmt == INT8:
        return max(float(torch.tensor(amax / 127, dtype=torch.float64).float()), 2.0 ** -126)
    e = -126
    while amax > 448 * 2.0 ** e:
        e += 1
    return 2.0 ** e


def encode(x, s, fmt):
    """Codes of x / s (double), nearest, ties to even."""
    z = x / s if s > 0 else torch.zeros_like(x)
    if fmt == INT8:
        return z.round().clamp(-127, 127).to(torch.int8).view(torch.uint8)
    gap = torch.exp2((torch.frexp(z)[1] - 1).clamp(min=-6).double() - 3)
    return ((z / gap).round() * gap).float().to(torch.float8_e4m3fn).view(torch.uint8)


def write(codes, scales, x, block, fmt, starts, counts):
    """In place, sequence by sequence and block by block."""
    B, H, cap, _ = codes.shape
    for b in range(B):
        p0 = starts[b]
        if not 0 <= p0 < cap:
            continue
        p1 = min(cap, p0 + max(0, min(x.shape[2], counts[b])))
        for h in range(H):
            for j in range(p0 // block, -(-p1 // block)) if p1 > p0 else ():
                lo, hi = max(p0, j * block), min(p1, (j + 1) * block)
                new = x[b, h, lo - p0:hi - p0].double()
                s = scale_of(float(new.abs().max()) if new.isfinite().all() else math.nan, fmt)
                if lo > j * block:
                    old = float(scales[b, h, j])
                    if math.isnan(old) or math.isnan(s):
                        s = math.nan
                    elif old >= s:
                        s = old
                    else:
                        held = codes[b, h, j * block:lo]
                        codes[b, h, j * block:lo] = encode(numbers(held, fmt) * old, s, fmt)
                scales[b, h, j] = s
                codes[b, h, lo:hi] = encode(new, s, fmt) if not math.isnan(s) else 0


def dequant(codes, scales, fmt):
    block = -(-codes.shape[2] // scales.shape[2])
    return dequant_by(codes, scales, fmt, block)


def dequant_by(codes, scales, fmt, block):
    at = torch.arange(codes.shape[2]) // block
    return numbers(codes, fmt) * scales.double()[:, :, at, None]


def attention(q, k, v, lens, block, scale, lists=None):
    """q [B, Hq, Lq, d]; k, v [B, H, cap, d] in 64 bits; lists[b][h][i]: kept
    blocks.  Returns o, lse and the bounds of the kernel's error on both:
    scores are exact products summed in fp32 (at most (d + 8) fp32 roundings of
    the sum of magnitudes, with the factors and the exponential's argument),
    probabilities carry 2^-20 for the exponential and the sums' roundings and
    half a bf16 step, the output half a bf16 step more."""
    B, Hq, Lq, d = q.shape
    H = k.shape[1]
    o = torch.zeros(q.shape, dtype=torch.float64)
    lse = torch.full((B, Hq, Lq), -math.inf, dtype=torch.float64)
    eo, el = torch.zeros_like(o), torch.zeros_like(lse)
    for b in range(B):
        for h in range(Hq):
            kk, vv = k[b, h * H // Hq], v[b, h * H // Hq]
            for i in range(-(-Lq // block)):
                rows = slice(i * block, min(Lq, (i + 1) * block))
                if lists is None:
                    at = torch.arange(lens[b])
                else:
                    at = torch.cat([torch.arange(j * block, max(j * block, min((j + 1) * block, lens[b])))
                                    for j in lists[b][h][i]] + [torch.arange(0)])
                if at.numel() == 0:
                    continue
                x = q[b, h, rows].double()
                s = x @ kk[at].t() * scale
                mag = (x.abs() @ kk[at].abs().t()).amax(1) * scale
                ds = (d + 8) * F32 * mag + 8 * F32 * s.abs().amax(1)
                top = torch.logsumexp(s, 1)
                p = torch.exp(s - top[:, None])
                o[b, h, rows] = p @ vv[at]
                lse[b, h, rows] = top
                spread = p @ vv[at].abs()
                eo[b, h, rows] = BF16 * o[b, h, rows].abs() + (BF16 + 2 * ds[:, None] + 2.0 ** -20) * 1.01 * spread
                el[b, h, rows] = ds + 2.0 ** -20 + 4 * F32 * top.abs()
    return o, lse, eo, el
