"""What the tests of the paged cache and its attention share: inputs, and the definition in 64 bits on the CPU, token after token, with
the bounds that the kernels' roundings have against it.

A token's places, positions and visible keys are worked out here from the batch's description alone; keys are gathered one by one,
so that what a token does not see takes no part in its result.
"""
import math

import torch

HALF = {torch.bfloat16: 2.0 ** -8, torch.float32: 2.0 ** -24}      # half a step of the type
F = 2.0 ** -24


def make(B, queries, lengths, heads, page, prefix=0, dtype=torch.bfloat16, order="head", seed=0, spare=3, device="cuda:0", peak=2.0):
    """A batch on the device: q, k, v of the new tokens, and a cache filled throughout (unwritten places too)."""
    g = torch.Generator().manual_seed(seed)
    Hq, Hkv, D = heads
    own = [-(-n // page) for n in lengths]
    front = -(-prefix // page)
    total = sum(own) + front + spare
    perm = torch.randperm(total, generator=g).to(torch.int32)
    table = torch.full((B, max([1, *own])), -1, dtype=torch.int32)
    at = front
    for b, n in enumerate(own):
        table[b, :n] = perm[at:at + n]
        at += n
    shape = (total, Hkv, page, D) if order == "head" else (total, page, Hkv, D) if order == "token" else (Hkv, total, page, D)
    back = {"head": lambda t: t, "token": lambda t: t.transpose(1, 2), "outer": lambda t: t.transpose(0, 1)}[order]
    T = sum(queries)
    c = {"q": (peak * torch.randn(T, Hq, D, generator=g)).to(dtype), "k": torch.randn(T, Hkv, D, generator=g).to(dtype),
         "v": torch.randn(T, Hkv, D, generator=g).to(dtype), "table": table, "lengths": torch.tensor(lengths, dtype=torch.int32),
         "starts": torch.tensor([0] + queries).cumsum(0).to(torch.int32), "prefix_table": perm[:front].clone()}
    c = {n: t.to(device) for n, t in c.items()}
    for n in ("k_pages", "v_pages"):
        c[n] = back(torch.randn(shape, generator=g).to(dtype).to(device))
    return {**c, "prefix": prefix, "page": page, "max_q": max([1, *queries]), "max_length": max([0, *lengths])}


def places(c):
    """[(token, sequence, place among its own tokens)] of every row that belongs to a sequence."""
    starts, lengths = c["starts"].tolist(), c["lengths"].tolist()
    return [(t, b, lengths[b] - (starts[b + 1] - starts[b]) + t - starts[b]) for b in range(len(lengths)) for t in range(starts[b], starts[b + 1])]


def attend(c, scale=None, limit=None):
    """(out, lse, out's bound, lse's bound), float64 on the CPU.  The bound of a kernel's element, counting roundings:
        a score           a sum of D products in float32, and its scaling:                      D + 8 roundings of sum |q| |k| scale
        a weight          exp of that (2 more), in the bfloat16 product rounded to bfloat16:     half a step of it
        the sums          one rounding for each of the n keys and as many again where pieces join
        out               one rounding to its type
    """
    q, kp, vp = (c[n].detach().cpu() for n in ("q", "k_pages", "v_pages"))
    T, Hq, D = q.shape
    pages, Hkv, page, _ = kp.shape
    G = Hq // Hkv
    scale = 1.0 / math.sqrt(D) if scale is None else scale
    out = torch.zeros(T, Hq, D, dtype=torch.float64)
    lse = torch.full((T, Hq), -math.inf, dtype=torch.float64)
    tol, tol_lse = torch.zeros_like(out), torch.zeros_like(lse)
    table, front = c["table"].tolist(), c["prefix_table"].tolist()
    dtype = q.dtype
    for t, b, p in places(c):
        if limit is not None and t - int(c["starts"][b]) >= limit:
            out[t], lse[t] = math.nan, math.nan
            continue
        seen = [(front[i // page], i % page) for i in range(c["prefix"])]
        seen += [(table[b][i // page], i % page) for i in range(min(p + 1, len(table[b]) * page))]
        seen = [(g, s) for g, s in seen if 0 <= g < pages]
        if not seen:
            continue
        g, s = torch.tensor(seen).T
        k, v = kp[g, :, s].double(), vp[g, :, s].double()                        # [n, Hkv, D]
        x = q[t].double().view(Hkv, G, D)
        scores = torch.einsum("hgd,nhd->hgn", x, k) * scale
        size = torch.einsum("hgd,nhd->hgn", x.abs(), k.abs()).amax(-1, keepdim=True) * scale
        w = torch.softmax(scores, dim=-1)
        n = len(seen)
        out[t] = torch.einsum("hgn,nhd->hgd", w, v).reshape(Hq, D)
        lse[t] = torch.logsumexp(scores, dim=-1).reshape(Hq)
        spread = torch.einsum("hgn,nhd->hgd", w, v.abs())
        weight = (D + 8) * F * size + 4 * F
        rounded = HALF[dtype] if dtype == torch.bfloat16 else 0.0
        tol[t] = (spread * (2 * weight + rounded + (2 * n + 64) * F)).reshape(Hq, D) + HALF[dtype] * out[t].abs() * 1.01 + 1e-30
        tol_lse[t] = (weight + (2 * n + 64) * F).reshape(Hq) + 4 * F * lse[t].abs()
    return out, lse, tol, tol_lse


def same(got, want, tol, what=""):
    got = got.detach().cpu().double()
    fine = torch.isfinite(want)
    assert torch.equal(torch.isnan(got), torch.isnan(want)), what
    assert torch.equal(got[~fine & ~torch.isnan(want)], want[~fine & ~torch.isnan(want)]), what
    off = ((got - want).abs() / tol.clamp(min=1e-38))[fine]
    assert off.numel() == 0 or float(off.max()) <= 1.0, f"{what}: {float(off.max()):.3g} times the bound"


def append(c, rope, interleaved, position):
    """(q_out, k_pages, v_pages, bounds of the first two), float64 on the CPU."""
    q, k, v, kp, vp = (c[n].detach().cpu().double() for n in ("q", "k", "v", "k_pages", "v_pages"))
    pages, page = kp.shape[0], kp.shape[2]
    half = HALF[c["q"].dtype]
    q_out, tq, tk = torch.zeros_like(q), torch.zeros_like(q), torch.zeros_like(kp)
    table = c["table"].tolist()

    def turn(x, row):
        y, size = x.clone(), torch.zeros_like(x)
        for i in range(rope.shape[1]):
            a, b = (2 * i, 2 * i + 1) if interleaved else (i, i + rope.shape[1])
            co, si = float(rope[row, i, 0]), float(rope[row, i, 1])
            y[..., a], y[..., b] = x[..., a] * co - x[..., b] * si, x[..., b] * co + x[..., a] * si
            size[..., a] = size[..., b] = x[..., a].abs() + x[..., b].abs()
        return y, half * y.abs() * 1.01 + 3 * F * size

    for t, b, p in places(c):
        row = position + p
        if rope is not None and not 0 <= row < rope.shape[0]:
            q_out[t] = math.nan
            continue
        q_out[t], tq[t] = turn(q[t], row) if rope is not None else (q[t], tq[t])
        if 0 <= p < len(table[b]) * page and 0 <= table[b][p // page] < pages:
            g, s = table[b][p // page], p % page
            kp[g, :, s], tk[g, :, s] = turn(k[t], row) if rope is not None else (k[t], 0.0)
            vp[g, :, s] = v[t]
    return q_out, kp, vp, tq, tk
