"""Plain forms in 64 bits of the latent-cache operators, on the CPU, and the
error bounds that follow from the operators' stated roundings."""
import math

import torch

BLOCK, LATENT, ROPE = 32, 512, 64
MAGNITUDES = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)
HALF_ULP = 2.0 ** -8      # of bfloat16: largest relative error of a rounding
F32 = 2.0 ** -24          # of float32


def quantize(x):
    """(codes [..., K/2], scales [..., K/32]) of x, by the definition, value by value in float64."""
    x = x.double().reshape(*x.shape[:-1], -1, BLOCK)
    top = x.abs().amax(-1)
    bad = ~torch.isfinite(x).all(-1)
    part, power = torch.frexp(torch.where(bad, 0.0, top))      # top = part * 2^power, part in [0.5, 1)
    # the unit u = 2^e with top / u in [3.5, 7)
    e = torch.where(part >= 0.875, power - 2, power - 3)
    e = torch.where(top > 0, e, -125).clamp(-125, 125)
    a = x.abs() / torch.exp2(e.double()).unsqueeze(-1)
    a = torch.where(bad.unsqueeze(-1), 0.0, a)
    far = torch.stack([(a - m).abs() for m in MAGNITUDES], -1)
    near = far.amin(-1, keepdim=True)
    hit = far == near
    # of two equally near magnitudes the even code
    code = torch.where(hit, torch.tensor([0, 9, 2, 11, 4, 13, 6, 15]), 99).amin(-1) % 8
    code = code + 8 * torch.signbit(x)
    scale = torch.where(bad, 255, e + 127)
    code = code.reshape(*code.shape[:-2], -1, 2)
    return (code[..., 0] + 16 * code[..., 1]).to(torch.uint8), scale.to(torch.uint8)


def values(codes, scales):
    """float64 values of codes and scales."""
    codes, scales = codes.cpu(), scales.cpu().double()
    c = torch.stack((codes & 15, codes >> 4), -1).flatten(-2).long()
    v = torch.tensor(MAGNITUDES + tuple(-m for m in MAGNITUDES), dtype=torch.float64)[c]
    unit = torch.where(scales == 255, math.nan, torch.exp2(scales - 127))
    return v * unit.repeat_interleave(BLOCK, -1)


def rotate(x, angles, halves):
    """(values, largest error of float32 products and one rounding to bfloat16) of x [..., 64]."""
    x, t = x.cpu().double(), angles.cpu().double()
    a, b = (x[..., :32], x[..., 32:]) if halves else (x[..., 0::2], x[..., 1::2])
    c, s = t[..., 0], t[..., 1]
    u, v = a * c - b * s, a * s + b * c
    size = (a * c).abs() + (b * s).abs() + (a * s).abs() + (b * c).abs()
    if halves:
        y, size = torch.cat((u, v), -1), torch.cat((size, size), -1)
    else:
        y, size = torch.stack((u, v), -1).flatten(-2), torch.stack((size, size), -1).flatten(-2)
    return y, HALF_ULP * y.abs() + 4 * F32 * size


def row_values(raw, mx4):
    """float64 [..., 576] of rows in bytes."""
    raw = raw.cpu().contiguous()
    if not mx4:
        return raw.view(torch.bfloat16).double()
    rope = raw[..., 272:].contiguous().view(torch.bfloat16).double()
    return torch.cat((values(raw[..., :256], raw[..., 256:272]), rope), -1)


def attend(q, keys, counts, scale):
    """One query token: q [H][576], keys [K][576] float64, counts [K] bool.
    Returns out [H][512], lse [H] and the largest errors of both."""
    q = q.cpu().double()
    keys = keys[counts]
    if keys.shape[0] == 0:
        z = torch.zeros(q.shape[0], LATENT, dtype=torch.float64)
        return z, torch.full((q.shape[0],), -math.inf, dtype=torch.float64), z, torch.zeros(q.shape[0]).double()
    s = q @ keys.T * scale
    # a score's products are exact in float32 and are added in some order, then scaled
    off = ((q.abs() @ keys.abs().T) * abs(scale) * (keys.shape[1] + 4) * F32).amax(-1)
    p = torch.softmax(s, -1)
    out, size = p @ keys[:, :LATENT], p @ keys[:, :LATENT].abs()
    lse = torch.logsumexp(s, -1)
    # weights: rounded once, scores off by `off` at most (and the exponential's few ulps of its argument)
    weight = HALF_ULP + 2 * off + (keys.shape[0] + 64) * F32 + 4 * F32 * s.abs().amax(-1)
    return out, lse, HALF_ULP * out.abs() + weight.unsqueeze(-1) * size + 1e-30, \
        off + (keys.shape[0] + 64) * F32 + 4 * F32 * (lse.abs() + s.abs().amax(-1))
