"""GPU: the paged cache in 4 bits and its attention (include/wht_attention4.h) against the definition in 64 bits, with bounds that
count the kernels' roundings.  Codes and scales are compared bit by bit."""
import math

import pytest
import torch

import attention_check
import attention4_check as check
import paper_2603_08343_amd as wht
from paper_2603_08343_amd import attention4

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
B16, F32 = torch.bfloat16, torch.float32


def call_append(c, rope, **kw):
    return wht.wht_attention_append4(c["q"], c["k"], c["v"], c["k_pages"], c["v_pages"], c["k_scales"], c["v_scales"], c["table"], c["lengths"], rope,
                                     q_starts=c["starts"], **kw)


def call_paged(c, **kw):
    kw = {"q_starts": c["starts"], "prefix_table": c["prefix_table"], "prefix_length": c["prefix"], "max_q": c["max_q"], "max_length": c["max_length"], **kw}
    return wht.wht_attention_paged4(c["q"], c["k_pages"], c["v_pages"], c["k_scales"], c["v_scales"], c["table"], c["lengths"], **kw)


def after_append(c, rope, place, interleaved, transformed, before):
    """What the pages have to hold, and the rows that want_values gives."""
    q, tol, k, v = check.append4(c, rope, place, interleaved, transformed)
    want = {n: t.clone() for n, t in before.items()}
    values = [torch.zeros_like(k), torch.zeros_like(v)]
    pages, page = c["k_pages"].shape[0], c["k_pages"].shape[2]
    table = c["table"].tolist()
    sides = [check.encode(k), check.encode(v)]
    q_want = torch.zeros_like(q)
    ok = torch.ones(q.shape[0], dtype=torch.bool) if rope is None else ((place >= 0) & (place < rope.shape[0])).all(-1)
    for t, b, p in attention_check.places(c):
        q_want[t] = q[t]
        for x in values:
            x[t] = math.nan
        if ok[t] and 0 <= p < len(table[b]) * page and 0 <= table[b][p // page] < pages:
            g, s = table[b][p // page], p % page
            for n, (codes, scales), x in zip(("k", "v"), sides, values):
                want[n + "_pages"][g, :, s], want[n + "_scales"][g, :, s] = codes[t], scales[t]
                x[t] = check.decode(codes[t], scales[t])
    return q_want, tol, want, values


def own_places(c, pairs, position):
    place = torch.zeros(c["q"].shape[0], pairs, dtype=torch.long)
    for t, _, p in attention_check.places(c):
        place[t] = position + p
    return place


def check_append(c, rope, position=0, positions=None, axes=None, interleaved=False, transformed=True, **kw):
    before = {n: c[n].cpu() for n in ("k_pages", "v_pages", "k_scales", "v_scales")}
    pairs = 0 if rope is None else rope.shape[1]
    place = own_places(c, pairs, position) if positions is None else positions.cpu().long()[:, list(axes)]
    want_q, tol, want, values = after_append(c, rope, place, interleaved, transformed, before)
    got_q, got_k, got_v = call_append(c, rope, position=position, positions=positions, axes=axes, interleaved=interleaved, transform=transformed, want_values=True, **kw)
    torch.cuda.synchronize()
    attention_check.same(got_q, want_q, tol, "q")
    for n in want:
        assert torch.equal(c[n].cpu(), want[n]), n
    for got, x in ((got_k, values[0]), (got_v, values[1])):
        assert torch.equal(torch.nan_to_num(got.cpu().double(), nan=-7.0), torch.nan_to_num(x, nan=-7.0))


APPENDS = [  # B, queries, lengths, heads, page, order, rotary, interleaved, transformed, dtype, position
    (1, [1], [1], (4, 4, 64), 16, "head", 64, False, True, B16, 0),
    (3, [1, 1, 1], [70, 1, 33], (8, 2, 128), 16, "token", 128, False, True, B16, 5),
    (2, [5, 37], [40, 37], (3, 3, 96), 8, "head", 96, False, True, B16, 1),
    (2, [4, 0], [9, 3], (12, 4, 96), 32, "outer", 48, True, False, F32, 7),
    (2, [9, 17], [9, 50], (16, 1, 128), 64, "head", 64, True, True, F32, 0),
    (1, [130], [200], (5, 5, 64), 128, "token", 16, False, False, B16, 3),
    (2, [3, 4], [3, 4], (40, 8, 128), 16, "head", 0, False, True, B16, 0),
    (2, [20, 3], [21, 3], (64, 8, 128), 16, "head", 128, False, True, B16, 0),
    (1, [3], [3], (1, 1, 96), 16, "head", 80, False, True, F32, 0),
    (2, [7, 2], [7, 2], (16, 16, 96), 16, "token", 96, True, True, F32, 0),
]


@pytest.mark.parametrize("case", APPENDS, ids=str)
def test_append(case):
    B, queries, lengths, heads, page, order, rotary, interleaved, transformed, dtype, position = case
    c = check.make4(B, queries, lengths, heads, page, dtype=dtype, order=order)
    rope = wht.wht_attention_rope_table(position + max(lengths), rotary, device=DEV) if rotary else None
    check_append(c, rope, position, interleaved=interleaved, transformed=transformed)


@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("cyclic", [False, True])
@pytest.mark.parametrize("heads,rotary,sections", [((4, 2, 64), 64, (8, 12, 12)), ((6, 2, 96), 96, (24, 24)), ((8, 8, 128), 64, (5, 9, 11, 7))], ids=str)
def test_append_with_several_axes(heads, rotary, sections, cyclic, interleaved):
    c = check.make4(3, [11, 1, 6], [11, 30, 9], heads, 16)
    g = torch.Generator().manual_seed(1)
    positions = torch.randint(0, 50, (18, len(sections)), generator=g).to(torch.int32).to(DEV)
    rope = wht.wht_attention_rope_table(50, rotary, device=DEV)
    check_append(c, rope, positions=positions, axes=wht.wht_rotary_axes(sections, cyclic), interleaved=interleaved)


def test_append_positions_outside_the_table():
    """On any axis that a pair is on: a row of NaN, and nothing stored; an axis without a pair may be anything."""
    c = check.make4(2, [4, 3], [4, 8], (4, 2, 64), 16)
    rope = wht.wht_attention_rope_table(20, 64, device=DEV)
    positions = torch.tensor([[0, 0, 19], [20, 0, 0], [0, -1, 0], [0, 0, 20], [2 ** 31 - 1, 1, 1], [-2 ** 31, 1, 1], [3, 4, 5]], dtype=torch.int32, device=DEV)
    check_append(c, rope, positions=positions, axes=wht.wht_rotary_axes((10, 10, 12)))


def test_append_places_that_are_not_there():
    """Bad pages, places past the table, padding rows, more new tokens than own ones."""
    c = check.make4(3, [4, 3, 2], [4, 40, 1], (4, 2, 64), 16)
    c["table"][0, 0] = c["k_pages"].shape[0]
    c["table"][1, 2] = -5
    c["lengths"][1] = 49                                             # past the table's three pages
    for n in ("q", "k", "v"):
        c[n] = torch.cat((c[n], torch.full_like(c[n][:2], 3.0)))     # padding
    check_append(c, wht.wht_attention_rope_table(100, 64, device=DEV), 1)


@pytest.mark.parametrize("dtype", [B16, F32], ids=str)
@pytest.mark.parametrize("transformed", [False, True])
def test_append_large_small_and_odd_numbers(dtype, transformed):
    """Zero blocks, signed zeros, the type's largest and smallest numbers, halfway cases, NaN and infinities."""
    c = check.make4(1, [12], [12], (2, 2, 64), 16, dtype=dtype)
    big = torch.finfo(dtype).max
    for x in (c["k"], c["v"]):
        x[0], x[1] = 0.0, -0.0
        x[2, 0], x[2, 1] = big, -big
        x[3] = big
        x[4], x[5] = 2.0 ** -126, 2.0 ** -133
        x[6, :, 5], x[6, :, 40] = math.nan, math.inf
        x[7, 0, 3], x[7, 1, 63] = -math.inf, math.nan
        x[8] = torch.tensor([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, 6.0]).repeat(8)
        x[9] = -x[8]
        x[10], x[10, :, 31], x[10, :, 32] = 2.0 ** -40, 6.0, 6.5
        x[11, :, ::3] = 0.0
    check_append(c, None, transformed=transformed)


def test_append_only_keys_in_place_and_strided():
    c = check.make4(2, [5, 1], [20, 1], (4, 2, 64), 16)
    fused = torch.randn(6, 9, 64, device=DEV).to(B16)                # a slice each, and a head between
    c["q"], c["k"], c["v"] = fused[:, :4], fused[:, 5:7], fused[:, 7:]
    rope = wht.wht_attention_rope_table(30, 64, device=DEV)
    twin = {n: t.clone() if torch.is_tensor(t) else t for n, t in c.items()}
    got = call_append(c, rope, q_out=c["q"])
    assert got is c["q"]
    q = wht.wht_attention_append4(None, twin["k"], twin["v"], *(twin[n] for n in ("k_pages", "v_pages", "k_scales", "v_scales")), twin["table"], twin["lengths"], rope,
                                  q_starts=twin["starts"])
    assert q is None
    out = call_append(twin, rope)
    torch.cuda.synchronize()
    assert torch.equal(out, c["q"]) and all(torch.equal(c[n], twin[n]) for n in ("k_pages", "v_pages", "k_scales", "v_scales"))


ATTENDS = [  # B, queries, lengths, heads, page, prefix, order, transformed, dtype
    (1, [1], [1], (4, 4, 64), 16, 0, "head", True, B16),
    (1, [1], [0], (8, 2, 128), 16, 0, "head", True, B16),                         # nothing to see
    (3, [1, 1, 1], [1, 77, 200], (8, 2, 128), 16, 0, "token", True, B16),
    (3, [1, 1, 1], [0, 31, 64], (6, 2, 96), 8, 45, "head", True, F32),
    (2, [3, 1], [3, 40], (12, 4, 96), 32, 0, "outer", False, B16),
    (2, [5, 2], [50, 300], (20, 4, 64), 64, 70, "head", True, B16),               # two tiles of rows
    (2, [4, 4], [9, 4], (32, 4, 128), 16, 33, "token", True, F32),
    (2, [1, 1], [700, 3], (32, 1, 128), 16, 0, "head", False, B16),
    (1, [40], [40], (4, 4, 64), 16, 0, "head", True, B16),                        # many rows
    (2, [70, 33], [70, 95], (8, 2, 128), 16, 50, "head", True, B16),
    (2, [100, 0], [130, 7], (4, 2, 96), 8, 0, "token", False, B16),
    (2, [35, 64], [80, 64], (4, 4, 64), 128, 100, "outer", True, F32),
    (1, [129], [200], (3, 1, 128), 16, 0, "head", True, F32),
    (1, [50], [50], (4, 1, 96), 16, 77, "head", True, F32),
    (40, [1] * 40, list(range(0, 120, 3)), (16, 8, 128), 16, 900, "head", True, B16),      # the prefix apart: rows of all sequences
    (36, [1] * 36, [20] * 36, (16, 16, 64), 16, 600, "head", False, F32),
    (9, [2] * 9, [30] * 9, (24, 12, 96), 16, 2000, "head", True, B16),
    (8, [1] * 8, [50] * 8, (32, 32, 64), 16, 700, "head", True, B16),             # a front of few rows
    (20, [1] * 20, [300] * 20, (16, 16, 96), 16, 0, "token", True, B16),          # heads side by side
    (2, [5, 1], [2, 7], (8, 2, 128), 16, 0, "head", True, B16),                   # more new tokens than the sequence has
    (2, [50, 3], [20, 9], (4, 2, 64), 16, 0, "head", True, F32),
    (1, [40], [700], (4, 1, 96), 16, 300, "head", True, B16),                     # a tile's keys in shares
    (2, [45, 20], [900, 20], (4, 2, 128), 32, 0, "token", False, F32),
    (3, [2, 4, 1], [60, 40, 90], (20, 4, 64), 8, 0, "head", True, B16),           # pages of 8
    (2, [33, 40], [70, 41], (4, 2, 128), 8, 21, "head", True, B16),
]


# Few rows are taken item by item where the longest that lengths can be is short, and on a line of all items' blocks else: the caller's max_length decides.
LONG = 1 << 20


@pytest.mark.parametrize("case", ATTENDS, ids=str)
def test_attend(case):
    B, queries, lengths, heads, page, prefix, order, transformed, dtype = case
    c = check.make4(B, queries, lengths, heads, page, prefix, dtype, order)
    out, lse, tol, tol_lse = check.attend4(c, transformed)
    for max_length in (c["max_length"], LONG):
        got, got_lse = call_paged(c, transform=transformed, want_lse=True, max_length=max_length)
        attention_check.same(got, out, tol, "out")
        attention_check.same(got_lse, lse, tol_lse, "lse")
        assert torch.equal(call_paged(c, transform=transformed, max_length=max_length), got)


@pytest.mark.parametrize("case", [c for c in ATTENDS if sum(c[1]) > 1][::2], ids=str)
def test_what_a_row_does_not_see_takes_no_part(case):
    """Every byte that no row sees is 0xff: NaN, with codes of -6; values that some rows of a sequence see and others do not are NaN too."""
    B, queries, lengths, heads, page, prefix, order, transformed, dtype = case
    c = check.make4(B, queries, lengths, heads, page, prefix, dtype, order)
    seen = torch.zeros(c["k_pages"].shape[0], page, dtype=torch.bool)
    for i in range(prefix):
        seen[int(c["prefix_table"][i // page]), i % page] = True
    table = c["table"].cpu()
    for b, n in enumerate(lengths):
        for i in range(n if queries[b] else 0):
            seen[int(table[b, i // page]), i % page] = True
    for n in ("k_pages", "v_pages", "k_scales", "v_scales"):
        c[n][~seen.to(DEV)[:, None].expand(-1, heads[1], -1)] = 255
    for b, n in enumerate(lengths):
        if queries[b] > 1 and n > 1:                                 # its newest but one, of one head, in one block
            p = n - 2
            c["v_scales"][int(table[b, p // page]), 0, p % page, 1] = 253
            c["k_scales"][int(table[b, p // page]), heads[1] - 1, p % page, 0] = 254
    out, lse, tol, tol_lse = check.attend4(c, transformed)
    for max_length in (c["max_length"], LONG):
        got, got_lse = call_paged(c, transform=transformed, want_lse=True, max_length=max_length)
        attention_check.same(got, out, tol, "out")
        attention_check.same(got_lse, lse, tol_lse, "lse")


@pytest.mark.parametrize("queries,heads", [([1, 1, 1], (8, 2, 128)), ([3, 1, 2], (12, 4, 96)), ([5, 2, 1], (20, 4, 64))], ids=str)
def test_codes_past_the_caches(queries, heads):
    """A table that can hold enough for the rule that reads codes past the caches."""
    c = check.make4(3, queries, [300, 77, 150], heads, 16, 40)
    wide = torch.full((3, LONG // 16), -1, dtype=torch.int32, device=DEV)
    wide[:, :c["table"].shape[1]] = c["table"]
    out, lse, tol, tol_lse = check.attend4(c, True)
    got, got_lse = call_paged({**c, "table": wide}, want_lse=True, max_length=LONG)
    attention_check.same(got, out, tol, "out")
    attention_check.same(got_lse, lse, tol_lse, "lse")
    assert torch.equal(got, call_paged(c, max_length=LONG))


@pytest.mark.parametrize("queries,heads", [([1, 1], (4, 2, 64)), ([6, 3], (8, 2, 128)), ([60, 40], (4, 2, 96))], ids=str)
@pytest.mark.parametrize("page", [8, 16])
@pytest.mark.parametrize("dtype", [B16, F32], ids=str)
def test_bad_pages_lengths_and_rows(queries, heads, dtype, page):
    """Page numbers outside the cache count as not there, on both sides; too small a max_q gives rows of NaN, padding rows zeros."""
    c = check.make4(2, queries, [90, 70], heads, page, 60, dtype)
    c["table"][0, 1], c["table"][1, 2] = -1, 2 ** 31 - 1
    c["prefix_table"][1] = c["k_pages"].shape[0]
    c["q"] = torch.cat((c["q"], torch.full_like(c["q"][:3], math.nan)))
    limit = max(queries) - 1 if max(queries) > 1 else None
    out, lse, tol, tol_lse = check.attend4(c, True, limit=limit)
    for max_length in (c["max_length"], LONG):
        got, got_lse = call_paged(c, max_q=limit or 1, want_lse=True, max_length=max_length)
        attention_check.same(got, out, tol, "out")
        attention_check.same(got_lse, lse, tol_lse, "lse")


@pytest.mark.parametrize("queries,heads", [([1, 1], (4, 2, 64)), ([3, 2], (8, 2, 128)), ([40, 9], (4, 2, 96))], ids=str)
@pytest.mark.parametrize("byte", [0, 1, 2, 207, 252])
def test_scales_of_any_size(byte, queries, heads):
    """The least and the largest scale bytes, of values: results are the sums of the numbers that they stand for.  The sums in front of the division
    by the weights' are of up to 2^30 keys, with weights up to 2^8: from numbers of 6 * 2^80 on (scale byte 207), times 2^38 below 2^122, they may pass
    float32's largest.  With 252 here, 40 keys of up to 2^127.6, they do where half of the weight is on values of one sign; such results are not finite."""
    c = check.make4(2, queries, [40, 33], heads, 16, dtype=F32)
    c["v_scales"].fill_(byte)
    out, _, tol, _ = check.attend4(c, False)
    got = call_paged(c, transform=False).cpu().double()
    if byte < 3:                                                     # some are below 2^-126, where a float32 sum keeps fewer bits
        tol = tol + 300 * 2.0 ** -149
    if byte > 207:
        out[~torch.isfinite(got)] = got[~torch.isfinite(got)]
    attention_check.same(got, out, tol, "out")


@pytest.mark.parametrize("max_length", [200, LONG])
@pytest.mark.parametrize("peak", [60.0, 4e4])
@pytest.mark.parametrize("queries", [[1, 1], [40, 33]], ids=str)
def test_large_scores(peak, queries, max_length):
    """Scores of hundreds and of 2^20: one key takes all the weight, or a few; the row's maximum is taken off exactly."""
    c = check.make4(2, queries, [200, 60], (4, 2, 64), 16, 40, F32)
    c["q"] *= peak
    out, lse, tol, tol_lse = check.attend4(c, True)
    got, got_lse = call_paged(c, want_lse=True, max_length=max_length)
    attention_check.same(got, out, tol, "out")
    attention_check.same(got_lse, lse, tol_lse, "lse")


@pytest.mark.parametrize("queries", [[1, 1], [40, 33]], ids=str)
def test_queries_that_are_not_finite_or_hardly(queries):
    """A float32 query past bfloat16's largest number is finite, and its scores with small keys are; NaN and infinity stay in their own rows."""
    c = check.make4(2, queries, [200, 60], (4, 2, 64), 16, 0, F32)
    c["k_scales"].sub_(110)
    c["q"][:] = c["q"] * 1e20
    c["q"][0, 0, 0] = torch.finfo(F32).max
    out, lse, tol, tol_lse = check.attend4(c, True)
    got, got_lse = call_paged(c, want_lse=True, scale=0.125)
    attention_check.same(got, out, tol, "out")
    attention_check.same(got_lse, lse, tol_lse, "lse")
    c["q"][0, 1, 5], c["q"][0, 2, 7] = math.nan, math.inf
    bad = call_paged(c, scale=0.125)
    same = torch.ones(bad.shape[:2], dtype=torch.bool)
    same[0, 1:3] = False
    assert torch.equal(bad[same.to(DEV)], got[same.to(DEV)]) and torch.isnan(bad[0, 1:3]).all()


def test_a_long_cache_past_32_bits():
    """Pages more than 4 GiB apart: offsets in 64 bits, codes and scales."""
    heads, page = (2, 1, 128), 1024
    pages = 70000
    codes = torch.zeros(2, pages, 1, page, 64, dtype=torch.uint8, device=DEV)      # 4.6 GB a side
    scales = torch.full((2, pages, 1, page, 4), 127, dtype=torch.uint8, device=DEV)
    c = check.make4(1, [3], [100], heads, page, 0)
    for i, n in enumerate("kv"):
        codes[i, pages - 1], scales[i, pages - 1] = c[n + "_pages"][int(c["table"][0, 0])], c[n + "_scales"][int(c["table"][0, 0])]
        c[n + "_pages"], c[n + "_scales"] = codes[i], scales[i]
    c["table"].fill_(pages - 1)
    small = {**c, "table": torch.zeros_like(c["table"]), **{n: c[n][pages - 1:] for n in ("k_pages", "v_pages", "k_scales", "v_scales")}}
    out, _, tol, _ = check.attend4(small, True)
    attention_check.same(call_paged(c), out, tol)
    rope = wht.wht_attention_rope_table(200, 128, device=DEV)
    check_append(small, rope)                                        # the same memory
    twin = {n: small[n].clone() for n in ("k_pages", "v_pages", "k_scales", "v_scales")}
    call_append(c, rope)
    assert all(torch.equal(twin[n], small[n]) for n in twin)


@pytest.mark.parametrize("max_length", [100, LONG])
def test_other_streams_and_a_workspace_of_the_callers(max_length):
    c = check.make4(3, [1, 1, 1], [100, 20, 60], (8, 2, 128), 16, 30)
    want = call_paged(c, max_length=max_length)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    out, lse = torch.empty_like(c["q"]), torch.empty(3, 8, device=DEV)
    need = wht.wht_attention4_workspace_bytes(3, 3, 8, 2, 128, 1, max_length, 30, 1)
    assert (need > 0) == (max_length == LONG)
    workspace = torch.full((max(need, 16),), 255, dtype=torch.uint8, device=DEV)
    got = call_paged(c, out=out, lse=lse, workspace=workspace, stream=side, max_length=max_length)
    side.synchronize()
    assert got[0] is out and got[1] is lse and torch.equal(out, want)
    with torch.cuda.stream(side):
        again = call_paged(c, max_length=max_length)
    side.synchronize()
    assert torch.equal(again, want)
    if need:
        with pytest.raises(attention4.WhtAttention4Error):
            call_paged(c, workspace=workspace[:need - 16], max_length=max_length)


@pytest.mark.parametrize("queries,max_length", [([1, 1, 1], 80), ([1, 1, 1], LONG), ([40, 2, 5], 80)], ids=str)
def test_captured_steps_follow_the_arrays(queries, max_length):
    """Append and attention in one graph, replayed with new inputs, lengths and eager work between; two graphs of one workspace in turn."""
    lengths = [50 + q for q in queries]
    c = check.make4(3, queries, lengths, (8, 2, 128), 16, 30)
    c["table"] = torch.arange(15, dtype=torch.int32, device=DEV).view(3, 5)
    rope = wht.wht_attention_rope_table(200, 128, device=DEV)
    q0, need = c["q"].clone(), wht.wht_attention4_workspace_bytes(sum(queries), 3, 8, 2, 128, max(queries), max_length, 30, 1)
    workspace = torch.empty(max(need, 16), dtype=torch.uint8, device=DEV)
    out = [torch.empty_like(q0) for _ in range(2)]

    def step(i, ws):
        q = call_append(c, rope, position=30)
        return wht.wht_attention_paged4(q, c["k_pages"], c["v_pages"], c["k_scales"], c["v_scales"], c["table"], c["lengths"], q_starts=c["starts"],
                                        prefix_table=c["prefix_table"], prefix_length=30, max_q=max(queries), max_length=max_length, out=out[i], workspace=ws)

    step(0, workspace)
    torch.cuda.synchronize()
    graphs = []
    for i in range(2):
        graphs.append(torch.cuda.CUDAGraph())
        with torch.cuda.graph(graphs[i]):
            step(i, workspace)
    for turn in range(4):
        c["q"].copy_(torch.randn_like(q0))
        c["k"].normal_()
        c["lengths"] += 1
        eager = step(0, None).clone()
        out[0].fill_(-1)
        for i in range(2):
            graphs[i].replay()
        torch.cuda.synchronize()
        assert torch.equal(out[0], eager) and torch.equal(out[1], eager), turn


@pytest.mark.parametrize("dtype", [B16, F32], ids=str)
def test_a_blocks_steps_together(dtype):
    """A prompt, then steps of one token, through append, attention and the output layer: against the same in 64 bits over the stored numbers."""
    heads, D = 4, 64
    pages = [torch.zeros(8, heads, 16, D // 2, dtype=torch.uint8, device=DEV) for _ in range(2)] + [torch.zeros(8, heads, 16, D // 32, dtype=torch.uint8, device=DEV) for _ in range(2)]
    table = torch.tensor([[3, 1, 6], [0, 2, 5]], dtype=torch.int32, device=DEV)
    rope = wht.wht_attention_rope_table(48, D, device=DEV)
    alpha, beta = torch.randn(heads * D, device=DEV), torch.randn(heads * D, device=DEV)
    g = torch.Generator().manual_seed(3)
    length = 0
    for new in (17, 1, 1):
        length += new
        q, k, v = (torch.randn(2 * new, heads, D, generator=g).to(dtype).to(DEV) for _ in range(3))
        lengths = torch.full((2,), length, dtype=torch.int32, device=DEV)
        starts = torch.tensor([0, new, 2 * new], dtype=torch.int32, device=DEV)
        q4 = wht.wht_attention_append4(q, k, v, *pages, table, lengths, rope, q_starts=starts)
        a = wht.wht_attention_paged4(q4, *pages, table, lengths, q_starts=starts, max_q=new)
        y = wht.wht_affine_forward(a.view(2 * new, -1), alpha, beta)
        c = {"q": q4, "k_pages": pages[0], "v_pages": pages[1], "k_scales": pages[2], "v_scales": pages[3], "table": table, "lengths": lengths, "starts": starts,
             "prefix": 0, "prefix_table": table[0, :0]}
        out, _, tol, _ = check.attend4(c, True)
        attention_check.same(a, out, tol)
        z = a.double().cpu().view(2 * new, -1) @ check.sylvester(heads * D) / math.sqrt(heads * D)
        want = alpha.cpu().double() * z + beta.cpu().double()
        assert float((y.cpu().double() - want).abs().max()) <= float(want.abs().max()) * 2 * attention_check.HALF[dtype] + 1e-3
    # what four bits leave of the sequence: keys turned, transformed and stored are within a quarter of their block's largest
    stored = check.transform(check.decode(pages[1], pages[3]), 8)
    last = stored[int(table[0, (length - 1) // 16]), :, (length - 1) % 16]
    assert float((last - v[new - 1].cpu().double()).norm() / v[new - 1].cpu().double().norm()) < 0.25


def test_rows_without_a_sequence_and_batches_without_one():
    """More rows than sequences (padding), no sequence at all, sequences without new tokens: zeros, on either way of few rows."""
    c = check.make4(2, [1, 1], [30, 20], (4, 2, 64), 16)
    for max_length in (30, LONG):
        for starts, live in (([0, 1, 2], [0, 1]), ([0, 0, 1], [0]), ([0, 0, 0], [])):
            q = torch.cat((c["q"], torch.full_like(c["q"], 3.0)))
            d = {**c, "q": q, "starts": torch.tensor(starts, dtype=torch.int32, device=DEV)}
            out, lse, tol, tol_lse = check.attend4(d, True)
            got, got_lse = call_paged(d, want_lse=True, max_length=max_length)
            attention_check.same(got, out, tol)
            attention_check.same(got_lse, lse, tol_lse)
            assert not got[len(live):].any() and torch.isneginf(got_lse[len(live):]).all()
        none = {**c, "table": c["table"][:0], "lengths": c["lengths"][:0], "starts": torch.zeros(1, dtype=torch.int32, device=DEV)}
        got = call_paged(none, max_length=max_length)
        assert got.shape == c["q"].shape and not got.any()


def test_results_do_not_depend_on_the_way_the_call_is_marshalled(monkeypatch):
    c = check.make4(3, [2, 1, 3], [100, 20, 60], (8, 2, 128), 16, 30)
    rope = wht.wht_attention_rope_table(200, 128, device=DEV)
    axes, positions = wht.wht_rotary_axes((32, 32)), torch.randint(0, 200, (6, 2), device=DEV, dtype=torch.int32)
    def all_calls():
        d = {n: t.clone() if torch.is_tensor(t) else t for n, t in c.items()}
        r = list(call_append(d, rope, positions=positions, axes=axes, want_values=True)) + [d[n] for n in ("k_pages", "v_pages", "k_scales", "v_scales")]
        r.append(call_append(d, rope, position=4, transform=False, interleaved=True))
        assert wht.wht_attention_append4(None, d["k"], d["v"], *(d[n] for n in ("k_pages", "v_pages", "k_scales", "v_scales")), d["table"], d["lengths"], rope, q_starts=d["starts"]) is None
        r += list(call_paged(c, want_lse=True)) + [call_paged(c, transform=False, scale=0.3)]
        return r
    native = all_calls()
    monkeypatch.setattr(attention4, "_native_module", attention4._NoNative)
    assert all(torch.equal(torch.nan_to_num(a), torch.nan_to_num(b)) for a, b in zip(native, all_calls()))


def test_plain_calls_are_marshalled_natively():
    c = check.make4(2, [1, 2], [20, 5], (4, 2, 64), 16)
    native, rope = attention4._native(), wht.wht_attention_rope_table(30, 64, device=DEV)
    pages = [c[n] for n in ("k_pages", "v_pages", "k_scales", "v_scales")]
    rest = [c["table"], c["lengths"]]
    for q, want, kind in ((c["q"], False, torch.Tensor), (c["q"], True, tuple), (None, False, tuple), (None, True, tuple)):
        got = native.append4(q, c["k"], c["v"], *pages, *rest, rope, c["starts"], 0, None, None, False, True, None, None, None, want)
        assert isinstance(got, kind)
        again = wht.wht_attention_append4(q, c["k"], c["v"], *pages, *rest, rope, q_starts=c["starts"], want_values=want)
        assert (again is None) if q is None and not want else isinstance(again, kind)
    assert native.paged4(c["q"], *pages, *rest, c["starts"], None, 0, 2, 20, None, True, None, None, False, None).shape == c["q"].shape
    assert native.rotate(c["q"], rope, None, None, False, False, None).shape == c["q"].shape
    assert native.append4(c["q"].half(), c["k"], c["v"], *pages, *rest, rope, c["starts"], 0, None, None, False, True, None, None, None, False) is None


def test_refusals_name_the_argument():
    c = check.make4(2, [1, 1], [20, 5], (4, 2, 64), 16)
    args = [c[n] for n in ("q", "k", "v", "k_pages", "v_pages", "k_scales", "v_scales", "table", "lengths")]
    rope = wht.wht_attention_rope_table(30, 64, device=DEV)
    ok = dict(zip(("q", "k", "v", "k_pages", "v_pages", "k_scales", "v_scales", "table", "lengths"), args))

    def refuse(error, match, keywords=None, **change):
        with pytest.raises(error, match=match):
            wht.wht_attention_append4(**{**ok, **change}, rope=change.get("rope", rope), **(keywords or {})) if "rope" not in change else \
                wht.wht_attention_append4(**{**ok, **change}, **(keywords or {}))

    refuse(ValueError, "k_pages must be a uint8", k_pages=c["k_pages"].to(torch.int8))
    refuse(ValueError, "v_pages must match", v_pages=c["v_pages"][:1])
    refuse(ValueError, "k_scales must be", k_scales=c["k_scales"][..., :1])
    refuse(ValueError, "v_scales must match", v_scales=c["v_scales"].transpose(1, 2).contiguous().transpose(1, 2))
    refuse(ValueError, "k must be a", k=c["k"][:, :, :32])
    refuse(ValueError, "v must have the other tensors' dtype", v=c["v"].float())
    refuse(TypeError, "float32 or bfloat16", q=c["q"].half(), k=c["k"].half(), v=c["v"].half())
    refuse(ValueError, "k must have 2 heads", k=c["q"])
    refuse(ValueError, "positions must be", {"positions": torch.zeros(3, 2, dtype=torch.int32, device=DEV)})
    refuse(ValueError, "axes must be below 1", {"axes": bytes([1] * 32)})
    refuse(ValueError, "one number for each", {"axes": bytes(31), "positions": torch.zeros(2, 2, dtype=torch.int32, device=DEV)})
    refuse(TypeError, "axes must be the axis", {"axes": "tt"})
    refuse(ValueError, "come together", {"k_out": torch.empty_like(c["k"])})
    refuse(ValueError, "rope must be", rope=rope.double())
    refuse(wht.WhtAttention4Error, "misaligned|16-byte", q=c["q"].new_empty(2, 4, 65)[:, :, 1:])
    refuse(wht.WhtAttention4Error, "status", rope=wht.wht_attention_rope_table(30, 24, device=DEV))
    same = c["k_pages"][:1].expand(c["k_pages"].shape)
    refuse(wht.WhtAttention4Error, "overlap", k_pages=same, v_pages=same)
    one = c["k_scales"][:1].expand(c["k_scales"].shape)
    refuse(wht.WhtAttention4Error, "overlap", k_scales=one, v_scales=one)
    with pytest.raises(wht.WhtAttention4Error, match="scale"):
        call_paged(c, scale=-1.0)
    with pytest.raises(ValueError, match="prefix_table must name"):
        call_paged(c, prefix_length=40)
    with pytest.raises(ValueError, match="one row"):
        wht.wht_attention_paged4(c["q"][:1], *args[3:7], c["table"], c["lengths"])
    assert call_append({**c, **{n: c[n][:0] for n in ("q", "k", "v")}}, rope).shape == (0, 4, 64)
