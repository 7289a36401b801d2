"""Attention over the paged cache on each of the ways that a call can take (attention_plan.h), at sizes that reach them: what a case is there for is asked of the
library's own rules.  Results against the definition in 64 bits (attention_check); places that no token has written hold NaN and infinities."""
import math
import random

import pytest
import torch

import attention_check as check
import attention_routes as routes

BF16, F32 = torch.bfloat16, torch.float32


def _ragged(B, most, seed):
    r = random.Random(seed)
    return [0, 1, most] + [r.randint(0, most) for _ in range(B - 3)]


def _queries(B, most, seed):
    r = random.Random(seed)
    return [0, most] + [r.randint(1, most) for _ in range(B - 2)]


# name: (queries, lengths, heads, page, prefix, order, table's width or None, what the call has to take)
CASES = {
    # the prefix apart: the rows of all sequences are one more item on the few-rows kernel's line
    "front_few": ([1] * 4, [0, 1, 33, 300], (8, 8, 64), 16, 20011, "head", None, {"front": 1, "front_few": 1, "share": 3}),
    "front_few_drafts": ([2, 1, 3, 1], [2, 9, 65, 300], (16, 8, 128), 16, 4203, "token", None, {"front": 1, "front_few": 1, "own_cap": 14}),
    "front_few_gang": ([1] * 4, [0, 1, 33, 300], (12, 12, 96), 8, 3003, "token", None, {"front": 1, "front_few": 1, "gang": 1}),
    # ... tiles of the many-rows kernel, beside the few-rows kernel's line
    "front_tiles": ([1] * 40, _ragged(40, 1500, 1), (32, 8, 128), 16, 1703, "head", None, {"front": 1, "front_few": 0, "share": 2, "front_splits": 2}),
    "front_tiles_drafts": (_queries(44, 3, 2), _ragged(44, 300, 2), (8, 2, 128), 32, 1703, "token", None, {"front": 1, "front_few": 0, "front_splits": 2}),
    "front_tiles_whole": ([1] * 70, _ragged(70, 100, 3), (8, 8, 64), 16, 250, "head", None, {"front": 1, "front_few": 0, "front_splits": -1}),
    "front_tiles_gang": ([1] * 50, _ragged(50, 100, 4), (12, 12, 96), 16, 300, "token", None, {"front": 1, "front_few": 0, "gang": 1}),
    # many blocks a worker: it goes on through a sequence, to the next head, the next sequence; a wave a joined row
    "line": ([1] * 100, _ragged(100, 2000, 5), (32, 8, 64), 16, 0, "head", None, {"front": 0, "share": 8, "join_waves": 1}),
    "line_behind_prefix": ([1] * 100, _ragged(100, 1000, 6), (16, 8, 64), 16, 100, "token", None, {"front": 0, "share": 6, "join_waves": 4}),
    "line_of_small_pages": ([1] * 100, _ragged(100, 2500, 7), (16, 16, 64), 8, 0, "head", None, {"front": 0, "share": 17}),
    "line_gang": ([1] * 80, _ragged(80, 1500, 8), (12, 12, 96), 16, 0, "token", None, {"front": 0, "share": 8, "gang": 1}),
    "line_drafts": (_queries(70, 4, 9), _ragged(70, 1200, 9), (32, 8, 128), 16, 0, "head", None, {"front": 0, "share": 3}),
    # keys past the caches, by what the table can hold
    "streams": ([1] * 3, [0, 1, 700], (8, 8, 128), 16, 0, "head", 1024, {"streams": 1, "share": 1}),
    "streams_line": ([1] * 30, _ragged(30, 1500, 10), (8, 8, 128), 16, 40, "token", 128, {"streams": 1, "share": 3}),
    "streams_drafts": (_queries(20, 4, 11), _ragged(20, 900, 11), (16, 8, 128), 64, 0, "head", 64, {"streams": 1, "share": 2}),
    "streams_beside_tiles": ([1] * 40, _ragged(40, 300, 12), (16, 4, 128), 16, 1100, "head", 256, {"streams": 1, "front": 1, "front_few": 0}),
    # a share of more pages than the many-rows kernel lists at a time
    "pages_listed_twice": ([5], [5], (512, 64, 64), 8, 17003, "head", None, {"own_few": 0, "own_splits": 4}),
}


def make(name, dtype, device):
    queries, lengths, heads, page, prefix, order, width, _ = CASES[name]
    lengths = [max(n, q) for n, q in zip(lengths, queries)]
    c = check.make(len(queries), queries, lengths, heads, page, prefix, dtype, order, seed=len(name), device=device)
    if width:
        table = torch.full((len(queries), width), -1, dtype=torch.int32, device=device)
        table[:, :c["table"].shape[1]] = c["table"]
        c["table"], c["max_length"] = table, None
    used = torch.zeros(c["k_pages"].shape[0], page, dtype=torch.bool)
    for row, n in [(c["prefix_table"], prefix), *zip(c["table"], lengths)]:
        at = torch.arange(n)
        used[row.cpu().long()[at // page], at % page] = True
    unused = (~used).to(device)[:, None, :, None].expand_as(c["k_pages"])
    c["k_pages"][unused], c["v_pages"][unused] = math.nan, math.inf
    return c


def takes(name, c, **more):
    r, want = routes.route(c, max_length=c["max_length"], **more), CASES[name][-1]
    for key, value in want.items():
        if key == "gang":
            assert r["gang_log2"] > 0 or c["q"].dtype == F32, r      # rows of 384 bytes are whole lines
        elif key == "streams":
            assert r["streams"] and not r["gang_log2"], r
        elif key in ("share", "front_splits") and value > 0:
            assert r[key] >= value, r
        else:
            assert r[key] == abs(value), (key, r)
    if name == "pages_listed_twice":
        steps = -(-(-(-c["prefix"] // 64) + 1) // r["own_splits"])
        assert steps * 64 // c["page"] > 508, steps


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("name", CASES)
def test_cases_take_the_ways_that_they_name(name, dtype):
    takes(name, make(name, dtype, "cpu"))


def _paged(c, **more):
    import paper_2603_08343_amd as wht
    return wht.wht_attention_paged(c["q"], c["k_pages"], c["v_pages"], c["table"], c["lengths"], c["starts"], c["prefix_table"], c["prefix"],
                                   want_lse=True, **{"max_q": c["max_q"], "max_length": c["max_length"], **more})


def _compare(c, limit=None, padding=0):
    """padding: rows of NaN behind the sequences' own."""
    T = c["q"].shape[0]
    q = torch.cat((c["q"], torch.full_like(c["q"][:1], math.nan).expand(padding, -1, -1)))
    out, lse = _paged({**c, "q": q}, **({} if limit is None else {"max_q": limit}))
    want, want_lse, tol, tol_lse = check.attend(c, limit=limit)
    check.same(out[:T], want, tol, "out")
    check.same(lse[:T], want_lse, tol_lse, "lse")
    assert (out[T:] == 0).all() and (lse[T:] == -math.inf).all()


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("name", CASES)
def test_every_way(name, dtype):
    c = make(name, dtype, "cuda:0")
    takes(name, c)
    _compare(c)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("name", CASES)
def test_every_way_around_bad_pages(name, dtype):
    """Numbers that name no page: in the prefix (its last one, in part, as well) and in the sequences' own."""
    c = make(name, dtype, "cuda:0")
    r, pages = random.Random(13), c["k_pages"].shape[0]
    front = c["prefix_table"]
    for i in {0, len(front) // 3, len(front) - 1} if len(front) else ():
        front[i] = r.choice([-1, pages, 1 << 30, -(1 << 31)])
    for b, n in enumerate(c["lengths"].tolist()):
        if n and b % 3 == 0:
            c["table"][b, r.randrange(-(-n // c["page"]))] = r.choice([-7, pages, (1 << 31) - 1])
    takes(name, c)
    _compare(c)


@pytest.mark.gpu
@pytest.mark.parametrize("name", [n for n, c in CASES.items() if max(c[0]) > 2])
@pytest.mark.parametrize("dtype", [BF16, F32])
def test_every_way_with_padding_and_a_max_q_that_is_too_small(name, dtype):
    c = make(name, dtype, "cuda:0")
    limit = c["max_q"] - 1
    _compare(c, padding=3)
    if name != "pages_listed_twice":                                 # four rows of eight: the few-rows kernel's then
        assert routes.route(c, max_q=limit, max_length=c["max_length"])["front"] == CASES[name][-1].get("front", 0)
    _compare(c, limit=limit, padding=3)


@pytest.mark.gpu
@pytest.mark.parametrize("name", ["front_few", "front_tiles", "front_tiles_whole", "line", "streams"])
def test_padding_behind_single_tokens(name):
    _compare(make(name, BF16, "cuda:0"), padding=5)


@pytest.mark.gpu
@pytest.mark.parametrize("name", ["front_few", "front_tiles", "line", "line_drafts", "streams_line", "pages_listed_twice"])
def test_every_way_bit_for_bit(name):
    c = make(name, BF16, "cuda:0")
    first = _paged(c)
    for _ in range(3):
        again = _paged(c)
        assert torch.equal(first[0], again[0]) and torch.equal(first[1], again[1])
