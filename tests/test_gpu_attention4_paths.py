"""Attention over the cache in 4 bits on each of the ways that a call can take (attention4_plan.h), at sizes where a worker has many blocks: codes on their way two blocks
ahead, shares that go on to the next head and sequence, lists of pages that are read more than once.  What a case is there for is asked of the library's own rules.
Results against the definition in 64 bits (attention4_check); places that no token has written hold bytes of 255: NaN."""
import math
import random
import zlib

import pytest
import torch

import attention4_check as check
import attention4_routes as routes
import attention_check

B16, F32 = torch.bfloat16, torch.float32


def _ragged(B, most, seed):
    r = random.Random(seed)
    return [0, 1, most] + [r.randint(0, most) for _ in range(B - 3)]


def _queries(B, most, seed):
    r = random.Random(seed)
    return [0, most] + [r.randint(1, most) for _ in range(B - 2)]


# name: (queries, lengths, heads, page, prefix, order, table's width or None, what the call has to take; numbers but 0 and 1: at least)
CASES = {
    # the line: through a sequence, to the next head, the next sequence; more than 64 sequences; a wave a joined row
    "line_64": ([1] * 100, _ragged(100, 1300, 5), (32, 16, 64), 16, 0, "head", None, {"front": 0, "whole": 0, "gang": 0, "tiles": 1, "share": 8, "join_waves": 1}),
    "line_96": ([1] * 90, _ragged(90, 1300, 6), (12, 12, 96), 32, 0, "head", None, {"front": 0, "gang": 0, "tiles": 1, "share": 5, "join_waves": 4}),
    "line_128": ([1] * 64, _ragged(64, 2200, 7), (32, 8, 128), 64, 0, "head", None, {"front": 0, "gang": 0, "tiles": 1, "share": 8}),
    "line_gang_96": ([1] * 80, _ragged(80, 1700, 8), (12, 12, 96), 16, 0, "token", None, {"gang": 1, "tiles": 1, "share": 8}),
    "line_gang_128": ([1] * 70, _ragged(70, 2000, 9), (16, 8, 128), 128, 0, "token", None, {"gang": 1, "tiles": 1, "share": 8}),
    "line_behind_prefix": ([1] * 100, _ragged(100, 1100, 10), (16, 8, 64), 16, 100, "head", None, {"front": 0, "own_few": 1, "gang": 0, "share": 5}),
    "line_pages_of_8": ([1] * 100, _ragged(100, 2500, 11), (16, 16, 64), 8, 0, "head", None, {"tiles": 2, "share": 17}),           # 64 pages are 16 blocks
    "line_gang_pages_of_8": ([1] * 70, _ragged(70, 1700, 12), (12, 12, 96), 8, 0, "token", None, {"gang": 1, "tiles": 2, "share": 8}),
    "line_pages_of_16_long": ([1] * 50, _ragged(50, 10500, 13), (16, 16, 64), 16, 0, "head", None, {"tiles": 1, "share": 33}),     # 64 pages are 32 blocks
    "line_drafts": (_queries(70, 4, 14), _ragged(70, 1800, 14), (32, 8, 128), 16, 0, "head", None, {"tiles": 1, "own_cap": 16, "share": 5}),
    "line_drafts_two_tiles": (_queries(120, 4, 15), _ragged(120, 1800, 15), (20, 4, 64), 16, 0, "head", None, {"tiles": 2, "own_cap": 20, "share": 5}),
    "line_drafts_96": (_queries(60, 5, 16), _ragged(60, 1600, 16), (16, 16, 96), 32, 0, "head", None, {"tiles": 1, "share": 5}),
    "line_drafts_gang": (_queries(60, 3, 17), _ragged(60, 1600, 17), (16, 16, 96), 16, 0, "token", None, {"gang": 1, "share": 5}),
    "line_drafts_pages_of_8": (_queries(70, 4, 18), _ragged(70, 1900, 18), (16, 8, 64), 8, 0, "head", None, {"tiles": 2, "share": 5}),
    # a sequence's rows of a key head by a workgroup
    "whole_128": ([1] * 32, _ragged(32, 2500, 19), (32, 8, 128), 16, 0, "head", None, {"whole": 1, "tiles": 1, "share": 8}),
    "whole_pages_of_8": ([1] * 16, _ragged(16, 2560, 20), (16, 16, 64), 8, 0, "token", None, {"whole": 1, "tiles": 2, "share": 10}),
    "whole_drafts": (_queries(40, 5, 21), _ragged(40, 1700, 21), (20, 4, 64), 16, 0, "head", None, {"whole": 1, "tiles": 2, "share": 5}),
    "whole_behind_prefix": (_queries(16, 3, 22), _ragged(16, 800, 22), (16, 8, 96), 16, 700, "token", None, {"whole": 1, "front": 0, "share": 5}),
    # the prefix apart: the rows of all sequences are one more item on the line
    "front_few": ([1] * 4, [0, 1, 33, 300], (8, 8, 64), 16, 30011, "head", None, {"front": 1, "front_few": 1, "share": 3}),
    "front_few_drafts": ([2, 1, 3, 1], [2, 9, 65, 300], (16, 8, 128), 16, 20203, "head", None, {"front": 1, "front_few": 1, "share": 3}),
    "front_few_gang": ([1] * 4, [0, 1, 33, 300], (12, 12, 96), 8, 14003, "token", None, {"front": 1, "front_few": 1, "gang": 1, "share": 3}),
    # ... tiles of the many-rows kernel, beside the line
    "front_tiles": ([1] * 40, _ragged(40, 2500, 23), (32, 8, 128), 16, 1703, "head", None, {"front": 1, "front_few": 0, "share": 5, "front_splits": 2}),
    "front_tiles_drafts": (_queries(44, 3, 24), _ragged(44, 4000, 24), (8, 2, 128), 32, 1703, "head", None, {"front": 1, "front_few": 0, "share": 3, "front_splits": 2}),
    "front_tiles_gang": ([1] * 50, _ragged(50, 1300, 25), (12, 12, 96), 16, 300, "token", None, {"front": 1, "front_few": 0, "gang": 1, "share": 5}),
    "front_tiles_pages_of_8": ([1] * 70, _ragged(70, 1500, 26), (16, 8, 64), 8, 250, "head", None, {"front": 1, "front_few": 0, "front_splits": 1, "share": 5}),
    # codes past the caches, by what the table can hold
    "past_64": ([1] * 60, _ragged(60, 1500, 27), (16, 16, 64), 16, 0, "head", 512, {"past": 1, "tiles": 1, "share": 5}),
    "past_128": ([1] * 30, _ragged(30, 3500, 28), (8, 8, 128), 16, 40, "head", 1024, {"past": 1, "tiles": 1, "share": 5}),
    "past_drafts": (_queries(20, 4, 29), _ragged(20, 2600, 29), (16, 8, 128), 64, 0, "head", 128, {"past": 1, "tiles": 1, "share": 3}),
    "past_drafts_two_tiles": (_queries(40, 4, 30), _ragged(40, 1800, 30), (40, 8, 64), 32, 0, "head", 512, {"past": 1, "tiles": 2, "share": 3}),
    "past_beside_tiles": ([1] * 40, _ragged(40, 3000, 31), (16, 4, 128), 16, 1100, "head", 1024, {"past": 1, "front": 1, "front_few": 0, "share": 3}),
    # a share of more pages than the many-rows kernel lists at a time: of the prefix, of a prefix and the sequence's own
    "pages_listed_twice": ([5], [5], (512, 64, 64), 8, 17003, "head", None, {"own_few": 0, "own_splits": 4}),
    "pages_listed_twice_own": ([7], [4500], (1000, 200, 64), 8, 701, "head", None, {"own_few": 0, "own_splits": 1}),
}
OLD = 120                                                            # pages that any sequence may have tokens in


def _seed(name):
    return zlib.crc32(name.encode()) % 1000


def make(name, dtype, device):
    """Sequences share their older pages; the last page of each, and all of the third one's, are its own."""
    queries, lengths, heads, page, prefix, order, width, _ = CASES[name]
    lengths = [max(n, q) for n, q in zip(lengths, queries)]
    Hq, Hkv, D = heads
    g = torch.Generator().manual_seed(_seed(name))
    own, front = [-(-n // page) for n in lengths], -(-prefix // page)
    alone = [n if b == 2 else min(n, 1) for b, n in enumerate(own)]
    total = front + sum(alone) + OLD + 3
    perm = torch.randperm(total, generator=g).to(torch.int32)
    table = torch.full((len(queries), width or max([1, *own])), -1, dtype=torch.int32)
    at, old = front, perm[front + sum(alone):front + sum(alone) + OLD]
    for b, n in enumerate(own):
        table[b, :n - alone[b]] = old[torch.randint(0, OLD, (n - alone[b],), generator=g)]
        table[b, n - alone[b]:n] = perm[at:at + alone[b]]
        at += alone[b]
    T = sum(queries)
    c = {"q": torch.randn(T, Hq, D, generator=g).to(dtype), "table": table, "lengths": torch.tensor(lengths, dtype=torch.int32),
         "starts": torch.tensor([0] + queries).cumsum(0).to(torch.int32), "prefix_table": perm[:front].clone()}
    used = torch.zeros(total, page, dtype=torch.bool)
    for row, n, q in [(c["prefix_table"], prefix, 1), *zip(table, lengths, queries)]:
        i = torch.arange(n if q else 0)
        used[row.long()[i // page], i % page] = True
    back = {"head": lambda t: t, "token": lambda t: t.transpose(1, 2).contiguous().transpose(1, 2)}[order]
    for n in ("k", "v"):
        codes = torch.randint(0, 256, (total, Hkv, page, D // 2), generator=g, dtype=torch.uint8)
        scales = torch.randint(122, 128, (total, Hkv, page, D // 32), generator=g, dtype=torch.uint8)
        for t in (codes, scales):
            t[(~used)[:, None].expand(-1, Hkv, -1)] = 255
        c[n + "_pages"], c[n + "_scales"] = back(codes), back(scales)
    c = {n: t.to(device) for n, t in c.items()}
    for n in ("k_pages", "v_pages", "k_scales", "v_scales"):         # a copy to the GPU keeps the order in memory only of dense tensors
        assert order == "head" or c[n].transpose(1, 2).is_contiguous()
    return {**c, "prefix": prefix, "page": page, "max_q": max([1, *queries]), "max_length": None if width else max([0, *lengths])}


def takes(name, c, **more):
    r, want = routes.route(c, max_length=c["max_length"], **more), CASES[name][-1]
    f32 = c["q"].dtype == F32
    for key, value in want.items():
        if key == "gang":
            assert (r["gang_log2"] > 0) == bool(value), (key, r)
        elif key == "past":
            assert r["past"] == (0 if f32 else 1) and not r["gang_log2"], (key, r)
        elif value > 1 and key in ("share", "front_splits"):
            assert r[key] >= value, (key, r)
        else:
            assert r[key] == value, (key, r)
    if name.startswith("pages_listed_twice"):
        steps = -(-(-(-c["prefix"] // 64) - (-int(c["lengths"][0]) // 64)) // r["own_splits"])
        assert steps * 64 // c["page"] > 508, steps
    if r["own_few"]:
        blocks = {"line_pages_of_8": 16, "line_pages_of_16_long": 32, "whole_pages_of_8": 16 if f32 else 0}.get(name, 0)
        assert r["share"] > blocks, r                                # a list of 64 pages and more


@pytest.mark.parametrize("dtype", [B16, F32], ids=str)
@pytest.mark.parametrize("name", CASES)
def test_cases_take_the_ways_that_they_name(name, dtype):
    c = make(name, dtype, "cpu")
    takes(name, c)
    takes(name, c, rows=c["q"].shape[0] + 3)


def _paged(c, transformed, **more):
    import paper_2603_08343_amd as wht
    return wht.wht_attention_paged4(c["q"], c["k_pages"], c["v_pages"], c["k_scales"], c["v_scales"], c["table"], c["lengths"], transform=transformed,
                                    want_lse=True, **{"q_starts": c["starts"], "prefix_table": c["prefix_table"], "prefix_length": c["prefix"], "max_q": c["max_q"],
                                                      "max_length": c["max_length"], **more})


def _transformed(name, dtype):
    return (_seed(name) % 2 == 0) == (dtype == B16)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [B16, F32], ids=str)
@pytest.mark.parametrize("name", CASES)
def test_every_way(name, dtype):
    c = make(name, dtype, "cuda:0")
    takes(name, c)
    transformed = _transformed(name, dtype)
    single = c["max_q"] == 1 and c["q"].shape[0] == c["lengths"].shape[0]
    out, lse = _paged(c, transformed, **({"q_starts": None} if single else {}))
    want, want_lse, tol, tol_lse = check.attend4(c, transformed)
    attention_check.same(out, want, tol, "out")
    attention_check.same(lse, want_lse, tol_lse, "lse")
    again = _paged(c, transformed)
    assert torch.equal(out, again[0]) and torch.equal(lse, again[1])

    # into the middle of larger buffers, by a workspace of no numbers: nothing in front of them, between or behind
    import paper_2603_08343_amd as wht
    (T, Hq, D), (Hkv, page) = c["q"].shape, c["k_pages"].shape[1:3]
    most = c["table"].shape[1] * page if c["max_length"] is None else c["max_length"]
    need = wht.wht_attention4_workspace_bytes(T, c["lengths"].shape[0], Hq, Hkv, D, c["max_q"], most, c["prefix"], 0 if dtype == F32 else 1)
    workspace, outs, lses = (torch.full(n, x, dtype=t, device="cuda:0") for n, x, t in (((need + 1024,), 255, torch.uint8), ((T + 2, Hq + 1, D + 16), 7.0, dtype), ((T + 2, Hq), 7.0, F32)))
    at = outs[1:-1, :Hq, 8:D + 8]
    _paged(c, transformed, out=at, lse=lses[1:-1], workspace=workspace[512:512 + need])
    assert torch.equal(at, out) and torch.equal(lses[1:-1], lse)
    at.fill_(7.0)
    lses[1:-1].fill_(7.0)
    assert (outs == 7.0).all() and (lses == 7.0).all() and (workspace[:512] == 255).all() and (workspace[512 + need:] == 255).all()


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [B16, F32], ids=str)
@pytest.mark.parametrize("name", CASES)
def test_every_way_around_bad_pages_and_blocks_that_are_no_numbers(name, dtype):
    """Numbers that name no page, in the prefix (its last one, in part, as well) and in the sequences' own; blocks of NaN that all rows of a sequence see, and ones
    that only some do; rows of NaN behind the sequences' own."""
    c = make(name, dtype, "cuda:0")
    r, pages, page, Hkv = random.Random(_seed(name)), c["k_pages"].shape[0], c["page"], c["k_pages"].shape[1]
    lengths, starts, table, front = c["lengths"].tolist(), c["starts"].tolist(), c["table"].cpu(), c["prefix_table"]
    for b, n in enumerate(lengths):
        if b == 2 and n:                                             # its pages are its own: in the middle of a share
            for side, p in (("v", n // 2), ("k", n // 3)):
                c[side + "_scales"][int(table[b, p // page]), r.randrange(Hkv), p % page, r.randrange(2)] = 253
        elif n > 2 and starts[b + 1] - starts[b] > 1 and (n - 2) // page == (n - 1) // page:
            for side, byte in (("v", 253), ("k", 254)):              # the newest but one
                c[side + "_scales"][int(table[b, (n - 2) // page]), r.randrange(Hkv), (n - 2) % page, r.randrange(2)] = byte
    for i in {0, len(front) // 3, len(front) - 1} if len(front) else ():
        front[i] = r.choice([-1, pages, 1 << 30, -(1 << 31)])
    for b, n in enumerate(lengths):
        if n and b % 3 == 0:
            c["table"][b, r.randrange(-(-n // page))] = r.choice([-7, pages, (1 << 31) - 1])
    transformed, T = not _transformed(name, dtype), c["q"].shape[0]
    want, want_lse, tol, tol_lse = check.attend4(c, transformed)
    takes(name, c, rows=T + 3)
    q = torch.cat((c["q"], torch.full_like(c["q"][:1], math.nan).expand(3, -1, -1)))
    out, lse = _paged({**c, "q": q}, transformed)
    attention_check.same(out[:T], want, tol, "out")
    attention_check.same(lse[:T], want_lse, tol_lse, "lse")
    assert (out[T:] == 0).all() and (lse[T:] == -math.inf).all()


@pytest.mark.gpu
@pytest.mark.parametrize("name", [n for n, c in CASES.items() if max(c[0]) > 2])
@pytest.mark.parametrize("dtype", [B16, F32], ids=str)
def test_every_way_with_a_max_q_that_is_too_small(name, dtype):
    c = make(name, dtype, "cuda:0")
    limit, transformed = c["max_q"] - 1, _transformed(name, dtype)
    out, lse = _paged(c, transformed, max_q=limit)
    want, want_lse, tol, tol_lse = check.attend4(c, transformed, limit=limit)
    attention_check.same(out, want, tol, "out")
    attention_check.same(lse, want_lse, tol_lse, "lse")



@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [B16, F32], ids=str)
@pytest.mark.parametrize("transformed", [False, True])
@pytest.mark.parametrize("byte", [251, 252, 253])
@pytest.mark.parametrize("queries,lengths,heads", [([1, 1], [1, 1], (4, 2, 64)), ([1, 1], [90, 33], (4, 2, 96)), ([3, 2], [40, 2], (20, 4, 128)), ([40, 9], [40, 100], (4, 2, 96)),
                                                   ([35, 1], [300, 1], (8, 2, 128))], ids=str)
def test_the_largest_scales(queries, lengths, heads, byte, transformed, dtype):
    """2^125 is a scale as any other, 253 is no number, of codes of zero as well.  Only the first key has codes other than zero -- with the transform one in 32, so that
    its block's sums are its own size -- and the base of a row's weights is no less than its score: sums stay below 6 * 2^125, and every result is finite."""
    c = check.make4(2, queries, lengths, heads, 16, dtype=dtype)
    D = heads[2]
    first = [(int(c["table"][b, 0]), h) for b in range(2) for h in range(heads[1])]
    c["v_pages"].zero_()
    c["v_scales"].fill_(byte)
    for i, (g, h) in enumerate(first):
        codes = torch.zeros(D, dtype=torch.uint8)
        if transformed:
            codes[torch.arange(0, D, 32) + (5 * i + 3) % 32] = torch.tensor([7, 15, 13, 1], dtype=torch.uint8)[:D // 32]
        else:
            codes[:] = (torch.arange(D) * 7 + i) % 16
        c["v_pages"][g, h, 0] = (codes[0::2] | codes[1::2] << 4).to(c["v_pages"].device)
    out, lse, tol, tol_lse = check.attend4(c, transformed)
    assert torch.isnan(out).all() if byte == 253 else torch.isfinite(out).all() and float(out.abs().max()) >= 2.0 ** (byte - 127 - 40)       # the first key has some weight
    for max_length in (max(lengths), 1 << 20):
        got, got_lse = _paged(c, transformed, max_length=max_length)
        attention_check.same(got, out, tol, "out")
        attention_check.same(got_lse, lse, tol_lse, "lse")


@pytest.mark.gpu
@pytest.mark.parametrize("queries,max_length", [([3], 100), ([3], 1 << 20), ([60], 100)], ids=str)
def test_heads_far_apart(queries, max_length):
    """Heads outside pages, more than 4 GiB apart: offsets in 64 bits, of the append as well."""
    pages, page, D, device = 70000, 1024, 128, "cuda:0"
    small = check.make4(1, queries, [100], (4, 2, D), page)
    wide = dict(small)
    for n in ("k_pages", "v_pages", "k_scales", "v_scales"):         # 9.2 GB of codes a side
        t = torch.zeros(2, pages, page, small[n].shape[3], dtype=torch.uint8, device=device).transpose(0, 1)
        t[pages - 1] = small[n][int(small["table"][0, 0])]
        wide[n] = t
    wide["table"] = torch.full_like(small["table"], pages - 1)
    assert wide["k_pages"].stride(1) > 1 << 32
    got = _paged(wide, True, max_length=max_length)
    want, want_lse, tol, tol_lse = check.attend4(small, True)
    attention_check.same(got[0], want, tol, "out")
    attention_check.same(got[1], want_lse, tol_lse, "lse")
    import paper_2603_08343_amd as wht
    rope = wht.wht_attention_rope_table(100, D)
    for c in (small, wide):
        c["q_out"] = wht.wht_attention_append4(c["q"], c["k"], c["v"], c["k_pages"], c["v_pages"], c["k_scales"], c["v_scales"], c["table"], c["lengths"], rope,
                                               q_starts=c["starts"])
    assert torch.equal(small["q_out"], wide["q_out"])
    for n in ("k_pages", "v_pages", "k_scales", "v_scales"):
        assert torch.equal(small[n][int(small["table"][0, 0])], wide[n][pages - 1]), n
