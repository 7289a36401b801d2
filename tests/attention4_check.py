"""What the tests of the cache in 4 bits and of rotary positions share: the definitions in 64 bits on the CPU, with the bounds that the kernels'
roundings have against them.  Attention's own definition is attention_check.attend over the numbers that the cache stands for.
"""
import torch

import attention_check
from attention_check import F, HALF

LEVELS = torch.tensor([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0], dtype=torch.float64)


def sylvester(n=32):
    h = torch.ones(1, 1, dtype=torch.float64)
    while h.shape[0] < n:
        h = torch.cat((torch.cat((h, h), 1), torch.cat((h, -h), 1)), 0)
    return h


def transform(x, over):
    """H of every 32 elements / over."""
    return (x.double().unflatten(-1, (-1, 32)) @ sylvester() / over).flatten(-2)


def decode(codes, scales):
    """The numbers [..., D] of codes [..., D / 2] and scales [..., D / 32], float64."""
    codes, scales = codes.cpu().long(), scales.cpu()
    codes = torch.stack((codes & 15, codes >> 4), -1).flatten(-2)
    x = torch.where(codes >= 8, -LEVELS[codes % 8], LEVELS[codes % 8]).unflatten(-1, (-1, 32))
    scale = torch.where(scales >= 253, torch.nan, torch.pow(2.0, scales.double() - 127))
    return (x * scale[..., None]).flatten(-2)


def encode(x):
    """(codes, scales) of x [..., D] float64: the nearest level by distance, of two as near the even code; the least scale by trying."""
    block = x.unflatten(-1, (-1, 32))
    odd = ~torch.isfinite(block).all(-1)
    block = torch.where(odd[..., None], 0.0, block)
    most = block.abs().amax(-1)
    e = torch.full(most.shape, 125, dtype=torch.int64)
    for power in range(124, -125, -1):
        e = torch.where(most <= 6.0 * 2.0 ** power, power, e)
    away = ((block / torch.pow(2.0, e.double())[..., None]).abs()[..., None] - LEVELS).abs()
    even_first = torch.tensor([0, 2, 4, 6, 1, 3, 5, 7])
    code = even_first[away[..., even_first].argmin(-1)]
    code = torch.where((block < 0) & (code > 0), code + 8, code).flatten(-2)
    scale = torch.where(odd, 255, e + 127)
    return (code[..., 0::2] | code[..., 1::2] << 4).to(torch.uint8), scale.to(torch.uint8)


def make4(B, queries, lengths, heads, page, prefix=0, dtype=torch.bfloat16, order="head", seed=0, device="cuda:0"):
    """attention_check.make's batch, with a cache of 4 bits of the same numbers."""
    c = attention_check.make(B, queries, lengths, heads, page, prefix, dtype, "head", seed, device=device)
    back = {"head": lambda t: t, "token": lambda t: t.transpose(1, 2).contiguous().transpose(1, 2), "outer": lambda t: t.transpose(0, 1).contiguous().transpose(0, 1)}[order]
    for n in ("k", "v"):
        codes, scales = encode(c.pop(n + "_pages").cpu().double())
        c[n + "_pages"], c[n + "_scales"] = back(codes.to(device)), back(scales.to(device))
    return c


def attend4(c, transformed, **kw):
    """(out, lse, and their bounds) as attention_check.attend; the transform adds its five sums and moves the rounding behind them."""
    d = {**c, "k_pages": decode(c["k_pages"], c["k_scales"]), "v_pages": decode(c["v_pages"], c["v_scales"])}
    out, lse, tol, tol_lse = attention_check.attend(d, **kw)
    if not transformed:
        return out, lse, tol, tol_lse
    half = HALF[c["q"].dtype]
    tol = tol - half * out.abs() * 1.01
    size = lambda x: (x.unflatten(-1, (-1, 32)).sum(-1, keepdim=True) / 8).expand(*x.shape[:-1], x.shape[-1] // 32, 32).flatten(-2)
    bound = size(tol) + 8 * F * size(out.abs())
    out = transform(out, 8)
    return out, lse, bound + half * out.abs() * 1.01 + 1e-30, tol_lse


def turn(x, rope, place, interleaved, back=False):
    """(x turned, its bound): x [T, H, D], place [T, rotary / 2] rows of rope, -1 or past the table: NaN."""
    x, rope = x.detach().cpu().double(), rope.cpu().double()
    y, size, r = x.clone(), torch.zeros_like(x), rope.shape[1]
    ok = ((place >= 0) & (place < rope.shape[0])).all(-1)
    angle = rope[place.clamp(0, max(rope.shape[0] - 1, 0)), torch.arange(r)][:, None]
    c, s = angle[..., 0], angle[..., 1] * (-1 if back else 1)
    a, b = (slice(0, 2 * r, 2), slice(1, 2 * r, 2)) if interleaved else (slice(0, r), slice(r, 2 * r))
    y[..., a], y[..., b] = x[..., a] * c - x[..., b] * s, x[..., b] * c + x[..., a] * s
    size[..., a] = size[..., b] = x[..., a].abs() + x[..., b].abs()
    y[~ok] = torch.nan
    return y, 3 * F * size


def append4(c, rope, place, interleaved, transformed):
    """(q, its bound, k and v in 64 bits as they are to be stored) of every row; place [T, rotary / 2]."""
    q, k, v = (c[n].detach().cpu().double() for n in ("q", "k", "v"))
    bound = torch.zeros_like(q)
    if rope is not None:
        (q, bound), (k, _) = turn(q, rope, place, interleaved), turn(k, rope, place, interleaved)
    if transformed:
        size = lambda x: (x.unflatten(-1, (-1, 32)).sum(-1, keepdim=True) / 8).expand(*x.shape[:-1], x.shape[-1] // 32, 32).flatten(-2)
        bound = size(bound) + 8 * F * size(q.abs())
        q, k, v = transform(q, 8), transform(k, 4), transform(v, 4)
    return q, bound + HALF[c["q"].dtype] * q.abs() * 1.01 + 1e-38, k, v
