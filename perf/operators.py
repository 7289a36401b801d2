"""The attention in front of the Walsh-Hadamard output layer, over a paged cache, as measurable cases.

    op = "append"   new keys and values go into the cache's pages, the position rotation applied on the way, and the
                    queries are rotated                                                    wht_attention_append
         "attend"   softmax attention of the new tokens over the pages: a prefix that every sequence of the batch
                    shares, then the sequence's own pages, causal among the new tokens     wht_attention_paged

B sequences; sequence b has queries[b] new tokens (1 when decoding) and lengths[b] tokens of its own in the cache, the
new ones included and last; every one of them comes after `prefix` shared tokens.  Head counts and widths are those of
the layer's workloads (4 x 64, 12 x 64, 16 x 64, 16 x 96, 16 x 128, 32 x 128, 64 x 128), with fewer key heads beside.
"""
import math
import random

import torch

own = False

_DEV = "cuda:0"
_DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32}
_HEADS = [(4, 4, 64), (12, 12, 64), (16, 16, 64), (16, 4, 64), (6, 2, 64), (16, 16, 96), (12, 4, 96), (16, 16, 128), (16, 1, 128),
          (32, 8, 128), (32, 32, 128), (40, 8, 128), (64, 8, 128)]
_SCORES = 1.1e9                         # elements of the padded score matrix of the plain form: the largest listed case's
_KEYS = 6.0e8                           # elements of the padded own keys


def _append(name, B, queries, lengths, heads, dtype="bf16", page=64, layout="head", prefix=0, rotary=None, interleaved=False, ragged=1):
    return {"name": name, "op": "append", "B": B, "q_min": queries[0], "q_max": queries[1], "len_min": lengths[0], "len_max": lengths[1],
            "Hq": heads[0], "Hkv": heads[1], "D": heads[2], "dtype": dtype, "page": page, "layout": layout, "prefix": prefix,
            "rotary": heads[2] if rotary is None else rotary, "interleaved": interleaved, "ragged": ragged}


def _attend(name, B, queries, lengths, heads, dtype="bf16", page=64, layout="head", prefix=0, lse=False, ragged=1):
    return {"name": name, "op": "attend", "B": B, "q_min": queries[0], "q_max": queries[1], "len_min": lengths[0], "len_max": lengths[1],
            "Hq": heads[0], "Hkv": heads[1], "D": heads[2], "dtype": dtype, "page": page, "layout": layout, "prefix": prefix, "lse": lse,
            "ragged": ragged}


def listed():
    return [
        # one sequence being decoded, a token far into a long text: the call is all latency
        _append("append_decode_1", 1, (1, 1), (7001, 7001), (32, 8, 128), prefix=120000),
        # a decoding batch of sequences of all lengths behind a common prompt
        _append("append_decode_256", 256, (1, 1), (1, 2048), (32, 8, 128), prefix=8192, page=16),
        # one prompt of odd length at the Base width (16 x 96), neighbours rotated, half of the head
        _append("append_prompt_4099", 1, (4099, 4099), (4099, 4099), (16, 16, 96), rotary=48, interleaved=True, layout="token"),
        # a packed batch of prompts at the widest layer (64 x 128)
        _append("append_prompts_32k", 11, (2000, 4000), (4000, 6000), (64, 8, 128), prefix=1024),
        # one sequence, no prefix: a single user's decoding over a long text
        _attend("decode_1x32k", 1, (1, 1), (32001, 32001), (32, 8, 128)),
        # the smallest configuration, float32 (4 x 64), a few sequences behind a short system prompt
        _attend("decode_f32_16", 16, (1, 1), (1, 300), (4, 4, 64), dtype="f32", prefix=515, page=16, lse=True),
        # serving at 32 x 128: 64 conversations behind a long system prompt
        _attend("decode_64", 64, (1, 1), (1, 2048), (32, 8, 128), prefix=8192),
        # the Base width (16 x 96), every head with keys of its own, many short answers
        _attend("decode_200x96", 200, (1, 1), (1, 700), (16, 16, 96), prefix=1001, page=16, layout="token"),
        # many samples from one very long document at 64 x 128
        _attend("decode_256", 256, (1, 1), (1, 2048), (64, 8, 128), prefix=32768),
        # drafted tokens being verified: a few queries of every sequence at once
        _attend("verify_32x5", 32, (2, 5), (5, 3000), (32, 8, 128), prefix=4096, lse=True),
        # questions to a common document: ragged prompts behind a prefix
        _attend("prompts_behind_prefix", 4, (301, 1003), (301, 1003), (16, 16, 128), prefix=2048),
        # prompts from their first token on
        _attend("prompts_2x4096", 2, (4095, 4096), (4096, 4096), (32, 8, 128)),
    ]


def draw(rng):
    """Either operator, all head layouts, types, page sizes and layouts; batches, lengths and prefixes spread over their
    logarithm, sequences without a token of their own among them."""
    def spread(lo, hi):
        return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(max(lo, 1)), math.log(hi)))))))

    heads = rng.choice(_HEADS)
    dtype = "f32" if rng.random() < 0.2 else "bf16"
    page, layout = rng.choice([16, 32, 64, 128]), rng.choice(["head", "token"])
    ragged = rng.randrange(1, 1 << 20)
    prefix = 0 if rng.random() < 0.25 else spread(1, 32768)
    B = spread(1, 256)
    if rng.random() < 0.5:
        top = min(8192, 32768 * 80 * 128 // (B * (heads[0] + 2 * heads[1]) * heads[2]))
        q = 1 if rng.random() < 0.4 else spread(1, max(2, top))
        most = q + spread(1, 2048)
        rotary = rng.choice([heads[2], heads[2], heads[2] // 2])
        return _strip(_append("", B, (max(1, q // 2), q), (q, most), heads, dtype, page, layout, prefix, rotary, rng.random() < 0.3, ragged))
    kind = rng.choice(["decode", "decode", "few", "prompt"])
    if kind == "prompt":
        B = spread(1, 8)
    q = 1 if kind == "decode" else spread(2, 8) if kind == "few" else spread(16, 4096)
    most = q + (0 if kind == "prompt" and rng.random() < 0.5 else spread(1, 4096))
    while B * heads[0] * q * (prefix + most) > _SCORES or B * most * heads[1] * heads[2] > _KEYS:
        if kind == "prompt" and q > 64:
            q, most = q // 2 + 1, most // 2 + 1
        else:
            B, prefix = max(1, B // 2), prefix * 3 // 4
    least = 0 if kind == "decode" else max(1, q // 2)
    return _strip(_attend("", B, (max(1, q // 2), q), (least, most), heads, dtype, page, layout, prefix, rng.random() < 0.4, ragged))


def _strip(case):
    del case["name"]
    return case


# ------------------------------------------------------------------------------------------------
# inputs

def _counts(case):
    """New tokens and own lengths of every sequence: by the case alone, so that its work is known without its inputs."""
    r = random.Random(case["ragged"])
    queries = [r.randint(case["q_min"], case["q_max"]) for _ in range(case["B"])]
    lengths = [r.randint(case["len_min"], case["len_max"]) for _ in range(case["B"])]
    if case["q_max"] > 1 or case["op"] == "append":
        lengths = [max(n, q) for n, q in zip(lengths, queries)]
    return queries, lengths


def prepare(case, seed):
    """A serving program's state: the fused projection's output [T, (Hq + 2 Hkv) D] that q, k and v are slices of, a
    cache whose pages lie in any order, the page tables and lengths, and the table of cos and sin."""
    gen = torch.Generator(device=_DEV)
    gen.manual_seed(int(seed))
    B, Hq, Hkv, D, page = case["B"], case["Hq"], case["Hkv"], case["D"], case["page"]
    dt = _DTYPES[case["dtype"]]
    queries, lengths = _counts(case)
    T, decode = sum(queries), case["q_max"] == 1
    own_pages = [-(-n // page) for n in lengths]
    prefix_pages = -(-case["prefix"] // page) if case["op"] == "attend" else 0
    width, total = max(1, max(own_pages)), sum(own_pages) + prefix_pages + 3
    order = torch.randperm(total, device=_DEV, generator=gen).to(torch.int32)
    table = torch.full((B, width), -1, dtype=torch.int32, device=_DEV)
    have = torch.tensor(own_pages, device=_DEV)
    table[torch.arange(width, device=_DEV)[None, :] < have[:, None]] = order[prefix_pages:prefix_pages + sum(own_pages)]

    def pages():
        shape = (total, Hkv, page, D) if case["layout"] == "head" else (total, page, Hkv, D)
        p = torch.empty(shape, dtype=dt, device=_DEV).normal_(generator=gen)
        return p if case["layout"] == "head" else p.transpose(1, 2)

    s = {"op": case["op"], "k_pages": pages(), "v_pages": pages(), "table": table, "prefix": case["prefix"],
         "lengths": torch.tensor(lengths, dtype=torch.int32, device=_DEV), "max_q": case["q_max"], "max_length": max(lengths),
         "starts": None if decode else torch.tensor([0] + queries, device=_DEV).cumsum(0).to(torch.int32)}
    if case["op"] == "append":
        fused = torch.empty(T, (Hq + 2 * Hkv) * D, dtype=dt, device=_DEV).normal_(generator=gen).view(T, Hq + 2 * Hkv, D)
        s["q"], s["k"], s["v"] = fused[:, :Hq], fused[:, Hq:Hq + Hkv], fused[:, Hq + Hkv:]
        angles = torch.arange(case["prefix"] + max(lengths), dtype=torch.float64, device=_DEV)[:, None] \
            * 10000.0 ** (-torch.arange(0, case["rotary"], 2, dtype=torch.float64, device=_DEV) / case["rotary"])
        s["rope"] = torch.stack((angles.cos(), angles.sin()), dim=2).float()        # [positions, rotary / 2, 2]
        s["interleaved"] = case["interleaved"]
    else:
        s["q"] = 2.0 * torch.empty(T, Hq, D, dtype=dt, device=_DEV).normal_(generator=gen)
        s["prefix_table"] = order[:prefix_pages].contiguous()
        s["lse"] = case["lse"]
    return s


# ------------------------------------------------------------------------------------------------
# one pass

def run(state):
    s = state
    if own:
        import paper_2603_08343_amd as wht
        if s["op"] == "append":
            q = wht.wht_attention_append(s["q"], s["k"], s["v"], s["k_pages"], s["v_pages"], s["table"], s["lengths"], s["rope"],
                                         q_starts=s["starts"], position=s["prefix"], interleaved=s["interleaved"])
            return q, s["k_pages"], s["v_pages"]
        return wht.wht_attention_paged(s["q"], s["k_pages"], s["v_pages"], s["table"], s["lengths"], q_starts=s["starts"],
                                       prefix_table=s["prefix_table"], prefix_length=s["prefix"], max_q=s["max_q"],
                                       max_length=s["max_length"], want_lse=s["lse"])
    return _plain_append(s) if s["op"] == "append" else _plain_attend(s)


def _sequence_of(s, T):
    """For every token: its sequence, its place among the sequence's new tokens, and its place among its own tokens."""
    B = s["lengths"].numel()
    token = torch.arange(T, device=_DEV)
    starts = torch.arange(B + 1, device=_DEV) if s["starts"] is None else s["starts"].long()
    seq = torch.searchsorted(starts[1:], token, right=True)
    j = token - starts[seq]
    return starts, seq, j, s["lengths"].long()[seq] - (starts[1:] - starts[:-1])[seq] + j


def _rotate(x, cs, interleaved):
    """x [T, H, D] in 32 bits; cs [T, r, 2]: the pairs of the first 2 r elements turned by their angles."""
    x = x.float()
    r = cs.shape[1]
    c, sn = cs[:, None, :, 0], cs[:, None, :, 1]
    a, b = (x[..., 0:2 * r:2], x[..., 1:2 * r:2]) if interleaved else (x[..., :r], x[..., r:2 * r])
    u, v = a * c - b * sn, b * c + a * sn
    turned = torch.stack((u, v), dim=-1).flatten(-2) if interleaved else torch.cat((u, v), dim=-1)
    return torch.cat((turned, x[..., 2 * r:]), dim=-1)


def _plain_append(s):
    T, page = s["q"].shape[0], s["k_pages"].shape[2]
    _, seq, _, place = _sequence_of(s, T)
    cs = s["rope"][place + s["prefix"]]
    where = s["table"].long()[seq, place // page]
    s["k_pages"][where, :, place % page] = _rotate(s["k"], cs, s["interleaved"]).to(s["k"].dtype)
    s["v_pages"][where, :, place % page] = s["v"]
    return _rotate(s["q"], cs, s["interleaved"]).to(s["q"].dtype), s["k_pages"], s["v_pages"]


def _plain_attend(s):
    q, table, P = s["q"], s["table"].long().clamp(min=0), s["prefix"]
    (T, Hq, D), (_, Hkv, page, _) = q.shape, s["k_pages"].shape
    B, G, Q = table.shape[0], Hq // Hkv, s["max_q"]
    starts, seq, j, _ = _sequence_of(s, T)
    # queries padded to [B, Hkv, Q G, D], scaled
    rows = (starts[:-1, None] + torch.arange(Q, device=_DEV)).clamp(max=T - 1)
    x = (q[rows].float() / math.sqrt(D)).view(B, Q, Hkv, G, D).permute(0, 2, 1, 3, 4).reshape(B, Hkv, Q * G, D)
    # own keys and values padded to [B, Hkv, L, D]; what no token has written is left out
    L = table.shape[1] * page
    there = torch.arange(L, device=_DEV) < s["lengths"][:, None]
    k, v = (torch.where(there[:, None, :, None], p[table].permute(0, 2, 1, 3, 4).reshape(B, Hkv, L, D).float(), 0.0)
            for p in (s["k_pages"], s["v_pages"]))
    sees = s["lengths"][:, None] - (starts[1:] - starts[:-1])[:, None] + torch.arange(1, Q + 1, device=_DEV)
    hidden = torch.arange(L, device=_DEV) >= sees[:, :, None]                                    # [B, Q, L]
    scores = torch.matmul(x, k.transpose(-1, -2).contiguous()).view(B, Hkv, Q, G, L)
    scores = scores.masked_fill_(hidden[:, None, :, None, :], -math.inf).view(B, Hkv, Q * G, L)
    most = scores.amax(dim=-1, keepdim=True)
    if P > 0:
        kp, vp = (p[s["prefix_table"].long()].permute(1, 0, 2, 3).reshape(Hkv, -1, D)[:, :P].float()
                  for p in (s["k_pages"], s["v_pages"]))
        front = torch.matmul(x.permute(1, 0, 2, 3).reshape(Hkv, B * Q * G, D), kp.transpose(-1, -2).contiguous())
        most = torch.maximum(most, front.amax(dim=-1).view(Hkv, B, Q * G, 1).transpose(0, 1))
    most = torch.where(most == -math.inf, 0.0, most)
    weights = torch.exp(scores.sub_(most))
    total, y = weights.sum(dim=-1, keepdim=True), torch.matmul(weights, v)
    if P > 0:
        weights = torch.exp(front.sub_(most.transpose(0, 1).reshape(Hkv, B * Q * G, 1)))
        total = total + weights.sum(dim=-1).view(Hkv, B, Q * G, 1).transpose(0, 1)
        y = y + torch.matmul(weights, vp).view(Hkv, B, Q * G, D).transpose(0, 1)
    y = y / torch.where(total == 0, 1.0, total)
    out = y.view(B, Hkv, Q, G, D).permute(0, 2, 1, 3, 4)[seq, j].reshape(T, Hq, D).to(q.dtype)
    if not s["lse"]:
        return out
    return out, (most + torch.log(total)).view(B, Hkv, Q, G).permute(0, 2, 1, 3)[seq, j].reshape(T, Hq)


# ------------------------------------------------------------------------------------------------
# what a pass cannot do without

def work(case):
    queries, lengths = _counts(case)
    T, Hq, Hkv, D = sum(queries), case["Hq"], case["Hkv"], case["D"]
    size = 4 if case["dtype"] == "f32" else 2
    if case["op"] == "append":
        positions = max(lengths) - min(n - q for n, q in zip(lengths, queries)) if T > case["B"] else len(set(lengths))
        return {"bytes": 2 * T * (Hq + 2 * Hkv) * D * size + min(T, positions) * case["rotary"] * 4 + 8 * case["B"] + 4 * T,
                "flops": 3 * T * (Hq + Hkv) * case["rotary"]}
    # pairs of a query and a key that it sees; a decoded sequence without a token of its own sees the prefix
    pairs = sum(q * case["prefix"] + q * n - q * (q - 1) // 2 for q, n in zip(queries, lengths))
    keys = case["prefix"] + sum(lengths)
    return {"bytes": 2 * T * Hq * D * size + 2 * keys * Hkv * D * size + (4 * T * Hq if case["lse"] else 0) + 4 * keys // case["page"],
            "flops": 4 * pairs * Hq * D}


# ------------------------------------------------------------------------------------------------
# the same in 64 bits, from the definition, one sequence after the other

def exact(case, seed):
    s = prepare(case, seed)
    queries, lengths = _counts(case)
    page, P, at = case["page"], case["prefix"], 0
    if case["op"] == "append":
        q, kc, vc = s["q"].double(), s["k_pages"].double(), s["v_pages"].double()
        for b, (nq, n) in enumerate(zip(queries, lengths)):
            tokens = slice(at, at + nq)
            place = torch.arange(n - nq, n, device=_DEV)
            angle = torch.view_as_complex(s["rope"][P + n - nq:P + n].double().contiguous())[:, None]

            def turn(x):
                x, r = x.double().clone(), angle.shape[-1]
                first, second = (slice(0, 2 * r, 2), slice(1, 2 * r, 2)) if case["interleaved"] else (slice(0, r), slice(r, 2 * r))
                z = torch.complex(x[..., first], x[..., second]) * angle
                x[..., first], x[..., second] = z.real, z.imag
                return x

            q[tokens] = turn(s["q"][tokens])
            at_pages = s["table"][b].long()[place // page]
            kc[at_pages, :, place % page] = turn(s["k"][tokens])
            vc[at_pages, :, place % page] = s["v"][tokens].double()
            at += nq
        return q, kc, vc
    Hq, Hkv, D = case["Hq"], case["Hkv"], case["D"]
    G = Hq // Hkv
    out = torch.zeros(sum(queries), Hq, D, dtype=torch.float64, device=_DEV)
    lse = torch.full((sum(queries), Hq), -math.inf, dtype=torch.float64, device=_DEV)

    def tokens_of(pages, table, n):
        return pages[table.long()[:-(-n // page)]].transpose(0, 1).reshape(Hkv, -1, D)[:, :n].double()

    front = [tokens_of(p, s["prefix_table"], P) for p in (s["k_pages"], s["v_pages"])]
    block = max(1, (1 << 27) // (Hq * (P + max(lengths) + 1)))                   # queries of one product
    for b, (nq, n) in enumerate(zip(queries, lengths)):
        k, v = (torch.cat((f, tokens_of(p, s["table"][b], n)), dim=1) for f, p in zip(front, (s["k_pages"], s["v_pages"])))
        for lo in range(0, nq if P + n > 0 else 0, block):
            hi = min(nq, lo + block)
            x = s["q"][at + lo:at + hi].double().view(hi - lo, Hkv, G, D).permute(1, 2, 0, 3).reshape(Hkv, -1, D)
            logits = (x @ k.transpose(1, 2).contiguous() / math.sqrt(D)).view(Hkv, G, hi - lo, P + n)
            last = torch.arange(P + n - nq + lo, P + n - nq + hi, device=_DEV)
            logits.masked_fill_(torch.arange(P + n, device=_DEV) > last[:, None], -math.inf)
            norm = torch.logsumexp(logits, dim=-1)                               # [Hkv, G, queries]
            weights = torch.nan_to_num(torch.exp(logits - norm[..., None]), nan=0.0).view(Hkv, -1, P + n)
            out[at + lo:at + hi] = (weights @ v).view(Hkv, G, hi - lo, D).permute(2, 0, 1, 3).reshape(hi - lo, Hq, D)
            lse[at + lo:at + hi] = norm.permute(2, 0, 1).reshape(hi - lo, Hq)
        at += nq
    return (out, lse) if case["lse"] else out
