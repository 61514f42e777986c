"""AdamW, its states in 8 bits, products with an epilogue and gated blocks in 64 bits on the CPU, for their tests."""
import math

import torch

BLOCK = 256


def _blocks(x):
    rows, cols = x.shape
    nb = (cols + BLOCK - 1) // BLOCK
    full = torch.zeros(rows, nb * BLOCK, dtype=x.dtype)
    full[:, :cols] = x
    return full.reshape(rows, nb, BLOCK)


def first_values():
    """What the 256 codes of a first state stand for, before their block's scale: sign, 4 bits of exponent, 3 of mantissa; two codes are NaN."""
    out = []
    for c in range(256):
        e, f = (c >> 3) & 15, c & 7
        v = f / 8 * 2.0 ** -6 if e == 0 else (1 + f / 8) * 2.0 ** (e - 7)
        out.append((-v if c & 128 else v) if c & 127 != 127 else math.nan)
    return torch.tensor(out, dtype=torch.float64)


def second_values():
    """What the 256 codes of a second state stand for."""
    return torch.tensor([0.0] + [(1 + (c + 1) % 8 / 8) * 2.0 ** ((c + 1) // 8 - 31) for c in range(1, 256)], dtype=torch.float64)


def encode(x, second):
    """(codes, exponents) of float32 values [rows x cols], code by code: the nearest value of the table, the even one of two that are as near."""
    rows, cols = x.shape
    full = _blocks(x.float())
    E = (full.view(torch.int32) & 0x7FFFFFFF).amax(2) >> 23
    scale = torch.ldexp(torch.ones((), dtype=torch.float64), (E.double() - (127 if second else 134)))
    y = full.double() / scale.unsqueeze(2)
    table = second_values() if second else first_values()[:128].nan_to_num(nan=math.inf)
    mids = (table[1:] + table[:-1]) / 2
    mag = y.abs().nan_to_num(nan=0.0, posinf=0.0).contiguous()
    up = torch.bucketize(mag, mids, right=True)        # mids[up - 1] <= mag < mids[up]
    tie = (up > 0) & (mag == mids[(up - 1).clamp(min=0)])
    code = torch.where(tie & (up % 2 == 1), up - 1, up)
    if second:
        # (mantissa and exponent run on from code to code, counted from 1 at an odd place: the even mantissa is that of an odd code)
        code = torch.where(tie, torch.where(up % 2 == 1, up, up - 1), up)
        code = torch.where(mag > 0, code.clamp(1, 255), torch.zeros_like(code))
    else:
        code = code + 128 * torch.signbit(y).long()
    dead = ((E == 0) | (E == 255)).unsqueeze(2)
    code = torch.where(dead, torch.zeros_like(code), code)
    return code.reshape(rows, full.shape[1] * BLOCK)[:, :cols].to(torch.uint8), E.to(torch.uint8)


def decode(codes, exps, second):
    """float64 values of codes."""
    table = second_values() if second else first_values()
    v = table[codes.long()]
    E = torch.repeat_interleave(exps.double(), BLOCK, dim=1)[:, :codes.shape[1]]
    v = torch.ldexp(v, E - (127 if second else 134))
    return torch.where(E == 255, torch.full_like(v, math.nan), v)


def adamw(p, g, m, v, t, lr, beta1, beta2, eps, weight_decay, c=1.0):
    """(p, m, v, |change of p|) in float64 after step t."""
    g = c * g.double()
    m = beta1 * m.double() + (1 - beta1) * g
    v = beta2 * v.double() + (1 - beta2) * g * g
    step = m / -math.expm1(t * math.log(beta1)) if beta1 else m
    root = torch.sqrt(v / -math.expm1(t * math.log(beta2)) if beta2 else v)
    step = step / (root + eps)
    p = p.double()
    return p - lr * (step + weight_decay * p), m, v, lr * (step.abs() + weight_decay * p.abs())


def act(name, g):
    """act(g) and its derivative."""
    if name == "none":
        return g, torch.ones_like(g)
    if name == "relu":
        return torch.relu(g), (g > 0).to(g.dtype)
    if name == "gelu":
        phi = 0.5 * torch.erfc(-g * math.sqrt(0.5))
        return g * phi, phi + g * torch.exp(-0.5 * g * g) / math.sqrt(2 * math.pi)
    s, rest = torch.sigmoid(g), torch.sigmoid(-g)
    return (s, s * rest) if name == "sigmoid" else (g * s, s * (1 + g * rest))
