"""The paged cache's append and its attention on the GPU, against the definition in 64 bits (attention_check)."""
import math

import numpy as np
import pytest
import torch

import attention_check as check

pytestmark = pytest.mark.gpu
BF16, F32 = torch.bfloat16, torch.float32


def _wht():
    import paper_2603_08343_amd as wht
    return wht


def _paged(c, lse=True, starts=True, **more):
    return _wht().wht_attention_paged(c["q"], c["k_pages"], c["v_pages"], c["table"], c["lengths"], q_starts=c["starts"] if starts else None,
                                      prefix_table=c["prefix_table"], prefix_length=c["prefix"], want_lse=lse,
                                      **{"max_q": c["max_q"], "max_length": c["max_length"], **more})


def _compare(c, what="", **more):
    out, lse = _paged(c, **more)
    limit = more.get("max_q")
    want, want_lse, tol, tol_lse = check.attend(c, more.get("scale"), limit if limit and limit < c["max_q"] else None)
    check.same(out, want, tol, f"{what} out")
    check.same(lse, want_lse, tol_lse, f"{what} lse")


# heads x types; lengths of nothing, one, around the kernels' steps (32, 64, 128 keys), and some that several workgroups share
HEADS = [(4, 4, 64), (6, 2, 64), (3, 3, 96), (10, 2, 96), (4, 4, 128), (8, 2, 128), (20, 4, 128), (16, 1, 128)]
LENGTHS = [0, 1, 2, 31, 32, 33, 63, 64, 65, 127, 128, 129, 300, 1000]


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("heads", HEADS)
@pytest.mark.parametrize("prefix,page,order", [(0, 16, "head"), (37, 8, "token"), (128, 64, "outer"), (515, 32, "head")])
def test_decode(dtype, heads, prefix, page, order):
    n = len(LENGTHS)
    c = check.make(n, [1] * n, LENGTHS, heads, page, prefix, dtype, order, seed=1)
    out, lse = _paged(c, starts=False)
    want, want_lse, tol, tol_lse = check.attend({**c, "starts": torch.arange(n + 1)})
    check.same(out, want, tol, "out")
    check.same(lse, want_lse, tol_lse, "lse")
    assert torch.equal(out, _paged(c, lse=False)), "without the statistic, with q_starts"


@pytest.mark.parametrize("heads", [(12, 4, 96), (8, 8, 96), (16, 16, 96)])
@pytest.mark.parametrize("queries,prefix", [([1] * 9, 0), ([1] * 9, 200), ([1, 1, 2, 1, 1, 1, 1, 1, 1], 200)])
def test_heads_whose_rows_share_lines(heads, queries, prefix):
    """Rows of 192 bytes one after the other: four heads side by side; the rows of all sequences few, and many, against the prefix."""
    lengths = [0, 1, 2, 33, 64, 300, 31, 1000, 128]
    c = check.make(9, queries, [max(n, q) for n, q in zip(lengths, queries)], heads, 16, prefix, BF16, "token", seed=30)
    _compare(c)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("heads", [(4, 4, 64), (3, 3, 96), (8, 2, 128), (64, 1, 64), (12, 1, 128)])
@pytest.mark.parametrize("length,prefix,page", [(1, 0, 8), (1, 1, 16), (0, 5, 16), (5000, 0, 16), (700, 4000, 64), (130, 0, 1024)])
def test_one_sequence(dtype, heads, length, prefix, page):
    _compare(check.make(1, [1], [length], heads, page, prefix, dtype, seed=2))


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("heads", [(4, 4, 64), (6, 2, 96), (8, 2, 128), (20, 4, 128)])
@pytest.mark.parametrize("prefix", [0, 200])
def test_a_few_queries_each(dtype, heads, prefix):
    c = check.make(7, [1, 3, 0, 5, 2, 4, 6], [1, 3, 40, 200, 2, 131, 6], heads, 16, prefix, dtype, "token", seed=3)
    _compare(c)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("heads", [(2, 2, 64), (6, 2, 96), (4, 1, 128), (5, 1, 128)])
@pytest.mark.parametrize("queries,lengths,prefix,page", [
    ([129], [129], 0, 16), ([64, 1, 0, 200], [64, 100, 7, 333], 0, 64), ([33, 127, 40], [50, 127, 40], 77, 8), ([300], [300], 1, 32)])
def test_prompts(dtype, heads, queries, lengths, prefix, page):
    _compare(check.make(len(queries), queries, lengths, heads, page, prefix, dtype, seed=4))


@pytest.mark.parametrize("B,heads", [(70, (2, 1, 64)), (200, (4, 4, 64)), (130, (6, 2, 128))])
def test_a_prompt_among_many_short_ones(B, heads):
    """More sequences than a wave has lanes, one of them long, some without a token."""
    queries = [(i * 7) % 4 for i in range(B)]
    queries[B // 2] = 300
    c = check.make(B, queries, [n + (i * 5) % 40 for i, n in enumerate(queries)], heads, 16, 20, seed=31)
    _compare(c)


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_prompts_in_more_tiles_than_workgroups(dtype):
    """No partial results: the kernel writes the outputs itself, and the rows that no tile covers."""
    c = check.make(9, [40] * 9, [40, 41, 60, 40, 45, 40, 40, 100, 40], (64, 64, 64), 16, 10, dtype, seed=5)
    q = torch.cat((c["q"], torch.full_like(c["q"][:5], math.nan)))                # five rows of padding
    out, lse = _paged({**c, "q": q})
    want, want_lse, tol, tol_lse = check.attend(c)
    check.same(out[:360], want, tol)
    check.same(lse[:360], want_lse, tol_lse)
    assert (out[360:] == 0).all() and (lse[360:] == -math.inf).all()
    out, lse = _paged({**c, "q": q}, max_q=33)                                    # too small: loud
    check.same(out[:360], *check.attend(c, limit=33)[::2])
    assert (out[360:] == 0).all()


@pytest.mark.parametrize("queries,max_q", [([1, 3, 2], 2), ([1, 40, 2], 30), ([1, 1, 1], 1)])
def test_padding_and_a_max_q_that_is_too_small(queries, max_q):
    c = check.make(3, queries, [9, 50, 2], (4, 2, 64), 16, 20, seed=6)
    T = sum(queries)
    q = torch.cat((c["q"], torch.full_like(c["q"][:3], math.nan)))
    out, lse = _paged({**c, "q": q}, max_q=max_q)
    want, want_lse, tol, tol_lse = check.attend(c, limit=max_q if max_q < max(queries) else None)
    check.same(out[:T], want, tol)
    check.same(lse[:T], want_lse, tol_lse)
    assert (out[T:] == 0).all() and (lse[T:] == -math.inf).all()


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("queries,lengths", [([1, 1, 1], [5, 70, 130]), ([3, 2, 5], [5, 70, 130]), ([40, 64, 100], [45, 70, 130])])
def test_what_is_not_seen_has_no_influence(dtype, queries, lengths):
    """Infinities and NaN in unwritten places, in pages of nobody, and in later tokens' keys and values."""
    c = check.make(3, queries, lengths, (4, 2, 64), 16, 21, dtype, seed=7)
    want, want_lse, tol, tol_lse = check.attend(c)
    used = torch.zeros(c["k_pages"].shape[0], 16, dtype=torch.bool)
    for row, n in [(c["prefix_table"], 21), *zip(c["table"], lengths)]:
        for i in range(n):
            used[int(row[i // 16]), i % 16] = True
    for name, value in (("k_pages", math.nan), ("v_pages", math.inf)):
        c[name][(~used).to(c[name].device)[:, None, :, None].expand_as(c[name])] = value
    out, lse = _paged(c)
    check.same(out, want, tol, "unwritten places")
    check.same(lse, want_lse, tol_lse, "unwritten places")
    # the last token's own key and value: no other token sees them
    last = []
    for b, (nq, n) in enumerate(zip(queries, lengths)):
        page, slot = int(c["table"][b][(n - 1) // 16]), (n - 1) % 16
        c["k_pages"][page, 0, slot] = math.nan
        c["v_pages"][page, 1, slot, 3] = -math.inf
        c["v_pages"][page, 1, slot, 40] = math.inf
        c["v_pages"][page, 1, slot, 41] = math.nan
        last.append(int(c["starts"][b + 1]) - 1)
    out, lse = _paged(c)
    others = torch.ones(sum(queries), dtype=torch.bool)
    others[last] = False
    check.same(out[others.to(out.device)], want[others], tol[others], "earlier tokens")
    check.same(lse[others.to(out.device)], want_lse[others], tol_lse[others], "earlier tokens")
    got = out[last].cpu().float()
    assert torch.isnan(got[:, :2]).all() and torch.isnan(lse[last][:, :2]).all()
    assert (got[:, 2:, 3] == -math.inf).all() and (got[:, 2:, 40] == math.inf).all() and torch.isnan(got[:, 2:, 41]).all()
    rest = [i for i in range(64) if i not in (3, 40, 41)]
    check.same(out[last][:, 2:, rest], want[last][:, 2:, rest], tol[last][:, 2:, rest], "the last tokens' other elements")


@pytest.mark.parametrize("queries", [[1, 1, 1], [2, 4, 3], [50, 60, 40]])
def test_bad_pages_are_not_read(queries):
    """A page number that names no page: its tokens are not there."""
    c = check.make(3, queries, [60, 300, 41], (4, 2, 128), 16, 50, seed=8)
    c["table"][0, 0], c["table"][1, 5], c["table"][2, 2], c["prefix_table"][1] = -1, 1 << 30, c["k_pages"].shape[0], -(1 << 31)
    _compare(c)
    c["prefix_table"][:], c["table"][2, :] = -1, -7                               # nothing is left for sequence 2
    _compare(c)
    out, lse = _paged(c)
    s = c["starts"].tolist()
    assert (out[s[2]:] == 0).all() and (lse[s[2]:] == -math.inf).all()


def test_lengths_out_of_range_are_cut():
    c = check.make(4, [1, 1, 2, 1], [20, 30, 2, 1], (4, 2, 64), 16, 9, seed=9)
    bad = c["lengths"].clone()
    bad[0], bad[1], bad[2] = 1 << 30, -5, 1                                       # past the table; negative; fewer than its new tokens
    out, lse = _paged({**c, "lengths": bad}, max_length=1 << 20)
    cut = bad.clamp(min=0, max=c["table"].shape[1] * 16)
    want, want_lse, tol, tol_lse = check.attend({**c, "lengths": cut})
    check.same(out, want, tol)
    check.same(lse, want_lse, tol_lse)
    c["starts"][:] = torch.tensor([3, -9, 1 << 30, 2, 70])                        # no ascending starts: in bounds, whatever comes out
    _paged(c)
    torch.cuda.synchronize()


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("kind", ["large", "tiny", "equal"])
def test_scores_of_all_sizes(dtype, kind):
    """One key takes all the weight; all weights alike; scores so large that exp of them overflows."""
    for queries, lengths in (([1, 1], [500, 64]), ([3, 2], [500, 64]), ([130, 64], [500, 64])):
        c = check.make(2, queries, lengths, (4, 2, 64), 16, 100, dtype, seed=10, peak={"large": 100.0, "tiny": 1e-20, "equal": 0.0}[kind])
        _compare(c, kind)


def test_scale():
    c = check.make(2, [1, 2], [100, 64], (4, 2, 64), 16, 10, seed=11)
    _compare(c, scale=0.5)
    _compare(c, scale=1e-3)


def test_strides():
    """Slices of wider tensors; a table that is a slice; outputs into one."""
    wht = _wht()
    c = check.make(3, [1, 2, 3], [100, 64, 7], (4, 2, 96), 32, 40, seed=12)
    want, want_lse, tol, tol_lse = check.attend(c)
    wide = torch.full((6, 9, 112), math.nan, dtype=BF16, device="cuda:0")
    wide[:, 2:6, 8:104] = c["q"]
    table = torch.full((3, 20), -1, dtype=torch.int32, device="cuda:0")
    table[:, 5:5 + c["table"].shape[1]] = c["table"]
    store = torch.full((6, 5, 4, 104), 7.0, dtype=BF16, device="cuda:0")
    lse = torch.empty(6, 4, device="cuda:0")
    out, _ = wht.wht_attention_paged(wide[:, 2:6, 8:104], c["k_pages"], c["v_pages"], table[:, 5:5 + c["table"].shape[1]], c["lengths"], c["starts"],
                                     c["prefix_table"], c["prefix"], 3, out=store[:, 1, :, :96], lse=lse)
    check.same(out, want, tol)
    check.same(lse, want_lse, tol_lse)
    store[:, 1, :, :96] = 7.0
    assert (store == 7.0).all()


def test_no_rows_and_no_sequences():
    wht = _wht()
    c = check.make(2, [0, 0], [5, 9], (4, 2, 64), 16, 10, seed=13)
    out, lse = _paged(c)
    assert out.shape == (0, 4, 64) and lse.shape == (0, 4)
    none = {**c, "table": c["table"][:0], "lengths": c["lengths"][:0], "starts": torch.zeros(1, dtype=torch.int32, device="cuda:0")}
    for rows in (0, 3):
        q = torch.ones(rows, 4, 64, dtype=BF16, device="cuda:0")
        for max_q in (1, 100):
            out, lse = _paged({**none, "q": q}, max_q=max_q)
            assert out.shape == q.shape and (out == 0).all() and (lse == -math.inf).all()
        q_out = wht.wht_attention_append(q, q[:, :2], q[:, :2], none["k_pages"], none["v_pages"], none["table"], none["lengths"], None, none["starts"])
        assert (q_out == 0).all()


def test_a_given_workspace_and_bit_for_bit():
    wht = _wht()
    for queries in ([1, 1, 1], [4, 3, 2], [100, 64, 9]):
        c = check.make(3, queries, [700, 64, 2000], (8, 2, 128), 16, 300, seed=14)
        need = wht.wht_attention_workspace_bytes(sum(queries), 3, 8, 2, 128, c["max_q"], c["max_length"], 300, 1)
        ws = torch.full((need + 16,), 255, dtype=torch.uint8, device="cuda:0")          # NaN throughout
        first = _paged(c, workspace=ws)
        for _ in range(3):
            again = _paged(c, workspace=ws)
            assert torch.equal(first[0], again[0]) and torch.equal(first[1], again[1])
        assert (ws[need:] == 255).all()
        with pytest.raises(wht.WhtAttentionError, match="workspace"):
            _paged(c, workspace=ws[:need - 1])


def test_another_stream():
    c = check.make(5, [1] * 5, [700, 64, 2000, 1, 0], (8, 2, 128), 16, 300, seed=15)
    want = _paged(c)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    got = _paged(c, stream=side)
    side.synchronize()
    assert torch.equal(want[0], got[0]) and torch.equal(want[1], got[1])
    with torch.cuda.stream(side):
        got = _paged(c)
    side.synchronize()
    assert torch.equal(want[0], got[0])


# ------------------------------------------------------------------------------------------------ append

@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("heads", [(4, 4, 64), (5, 3, 96), (8, 2, 128), (64, 1, 64)])
@pytest.mark.parametrize("rotary", [0, 32, 1])
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("queries,lengths,page,order", [([1] * 6, [1, 0, 16, 17, 64, 100], 16, "head"), ([3, 0, 40, 1], [3, 5, 90, 65], 64, "token"),
                                                        ([9], [70], 8, "outer")])
def test_append(dtype, heads, rotary, interleaved, queries, lengths, page, order):
    wht = _wht()
    rotary = heads[2] if rotary == 1 else rotary
    c = check.make(len(queries), queries, lengths, heads, page, 0, dtype, order, seed=21)
    rope = wht.wht_attention_rope_table(200, rotary, device="cuda:0") if rotary else None
    want = check.append(c, None if rope is None else rope.cpu().double(), interleaved, 77)
    before = [c["q"].clone(), c["k"].clone(), c["v"].clone()]
    starts = c["starts"] if max(queries) > 1 or len(queries) == 1 else None
    q = wht.wht_attention_append(c["q"], c["k"], c["v"], c["k_pages"], c["v_pages"], c["table"], c["lengths"], rope, starts, 77, interleaved)
    check.same(q, want[0], want[3], "q")
    check.same(c["k_pages"], want[1], want[4], "k")
    assert torch.equal(c["v_pages"].cpu().double(), want[2]), "v"
    assert all(torch.equal(a, c[n]) for a, n in zip(before, "qkv"))


def test_append_slices_without_queries_and_in_place():
    wht = _wht()
    c = check.make(4, [2, 1, 3, 0], [40, 1, 35, 9], (4, 2, 128), 16, 0, seed=22)
    rope = wht.wht_attention_rope_table(64, 128, device="cuda:0")
    want = check.append(c, rope.cpu().double(), False, 0)
    fused = torch.cat((c["q"], c["k"], c["v"]), dim=1)                            # [T, 8, 128]
    q, k, v = fused[:, :4], fused[:, 4:6], fused[:, 6:]
    kp, vp = c["k_pages"].clone(), c["v_pages"].clone()
    assert wht.wht_attention_append(None, k, v, kp, vp, c["table"], c["lengths"], rope, c["starts"]) is None
    check.same(kp, want[1], want[4])
    assert torch.equal(vp.cpu().double(), want[2])
    back = wht.wht_attention_append(q, k, v, c["k_pages"], c["v_pages"], c["table"], c["lengths"], rope, c["starts"], q_out=q)
    assert back.data_ptr() == fused.data_ptr()
    check.same(fused[:, :4], want[0], want[3])
    assert torch.equal(fused[:, 4:], torch.cat((c["k"], c["v"]), dim=1))


def test_append_where_there_is_no_place():
    """Padding rows, pages that are none, positions without a row in the table, more new tokens than the sequence has."""
    wht = _wht()
    c = check.make(5, [1, 2, 1, 3, 1], [20, 30, 5, 1, 40], (4, 2, 64), 16, 0, seed=23)
    c["table"][0, 1], c["table"][1, 1] = -1, 1 << 29
    rope = wht.wht_attention_rope_table(35, 64, device="cuda:0")
    want = check.append(c, rope.cpu().double(), True, 0)
    pad = torch.ones(2, 4, 64, dtype=BF16, device="cuda:0")
    q, k, v = torch.cat((c["q"], pad)), torch.cat((c["k"], pad[:, :2])), torch.cat((c["v"], pad[:, :2]))
    out = wht.wht_attention_append(q, k, v, c["k_pages"], c["v_pages"], c["table"], c["lengths"], rope, c["starts"], 0, True)
    assert (out[8:] == 0).all()
    check.same(out[:8], want[0], want[3])
    check.same(c["k_pages"], want[1], want[4])
    assert torch.equal(c["v_pages"].cpu().double(), want[2])


def test_append_past_the_table():
    """A sequence that has outgrown its row of the table: its tokens are not stored, and nothing else is written over."""
    wht = _wht()
    for lengths in ([48, 49, 60, 1 << 30], [47, 50, -3, (1 << 31) - 1]):
        c = check.make(4, [1, 3, 2, 1], [48, 48, 48, 48], (4, 2, 64), 16, 0, seed=29)
        c["lengths"] = torch.tensor(lengths, dtype=torch.int32, device="cuda:0")
        want = check.append(c, None, False, 0)
        out = wht.wht_attention_append(c["q"], c["k"], c["v"], c["k_pages"], c["v_pages"], c["table"], c["lengths"], None, c["starts"])
        assert torch.equal(out, c["q"])
        assert torch.equal(c["k_pages"].cpu().double(), want[1]) and torch.equal(c["v_pages"].cpu().double(), want[2])


def test_offsets_past_32_bits():
    """A cache of more than 4 GiB: its last pages."""
    wht = _wht()
    pages = (9 << 30) // (64 * 128 * 2)
    free, _ = torch.cuda.mem_get_info()
    if free < 2.2 * (9 << 30):
        pytest.skip("not enough memory")
    c = check.make(2, [1, 1], [200, 70], (4, 1, 128), 64, 100, seed=24)
    big = [torch.zeros(pages, 1, 64, 128, dtype=BF16, device="cuda:0") for _ in range(2)]
    n = c["k_pages"].shape[0]
    for t, name in zip(big, ("k_pages", "v_pages")):
        t[pages - n:] = c[name]
    moved = {**c, "k_pages": big[0], "v_pages": big[1], "table": torch.where(c["table"] >= 0, c["table"] + (pages - n), -1),
             "prefix_table": c["prefix_table"] + (pages - n)}
    want, got = _paged(c), _paged(moved)
    assert torch.equal(want[0], got[0]) and torch.equal(want[1], got[1])
    for x in (c, moved):
        wht.wht_attention_append(None, x["k"], x["v"], x["k_pages"], x["v_pages"], x["table"], x["lengths"], None)
    assert torch.equal(big[0][pages - n:], c["k_pages"]) and torch.equal(big[1][pages - n:], c["v_pages"])


# ------------------------------------------------------------------------------------------------ together

@pytest.mark.parametrize("prefix", [0, 90])
def test_a_captured_step_replays(prefix):
    """Append and attention of a decoding step in a graph: every replay, with lengths that grow, against the eager calls."""
    wht = _wht()
    c = check.make(4, [1] * 4, [50, 64, 1, 130], (8, 2, 128), 16, prefix, seed=25)
    c["lengths"] -= 1
    width = torch.full((4, 14), -1, dtype=torch.int32, device="cuda:0")
    width[:, :c["table"].shape[1]] = c["table"]
    spare = torch.arange(c["k_pages"].shape[0], c["k_pages"].shape[0] + 20, dtype=torch.int32, device="cuda:0").view(4, 5)
    for b, n in enumerate([50, 64, 1, 130]):
        have = -(-n // 16)
        width[b, have:have + 5] = spare[b]
    kp, vp = (torch.cat((c[n], torch.full((20, *c[n].shape[1:]), math.nan, dtype=BF16, device="cuda:0"))) for n in ("k_pages", "v_pages"))
    rope = wht.wht_attention_rope_table(400, 128, device="cuda:0")
    inputs = torch.empty(4, 12, 128, dtype=BF16, device="cuda:0").normal_()

    def step(k_pages, v_pages, lengths):
        lengths.add_(1)
        q = wht.wht_attention_append(inputs[:, :8], inputs[:, 8:10], inputs[:, 10:], k_pages, v_pages, width, lengths, rope, position=prefix)
        return wht.wht_attention_paged(q, k_pages, v_pages, width, lengths, prefix_table=c["prefix_table"], prefix_length=prefix, want_lse=True)

    eager = [kp.clone(), vp.clone(), c["lengths"].clone()]
    graphed = [kp, vp, c["lengths"].clone()]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step(*[t.clone() for t in graphed])
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = step(*graphed)
    for i in range(6):
        inputs.normal_()
        want = step(*eager)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.isfinite(out[0]).all(), i
        assert torch.equal(out[0], want[0]) and torch.equal(out[1], want[1]), i
        assert torch.equal(graphed[2], eager[2])
    assert torch.equal(graphed[0].nan_to_num(7.0), eager[0].nan_to_num(7.0)) and torch.equal(graphed[1].nan_to_num(7.0), eager[1].nan_to_num(7.0))


def test_refusals():
    wht = _wht()
    c = check.make(2, [1, 1], [20, 30], (4, 2, 64), 16, 10, seed=26)

    def paged(error, match, q_starts=None, prefix=10, **change):
        x = {**c, **change}
        with pytest.raises(error, match=match):
            wht.wht_attention_paged(x["q"], x["k_pages"], x["v_pages"], x["table"], x["lengths"], q_starts, x["prefix_table"], prefix,
                                    **{n: x[n] for n in ("out", "lse", "scale", "max_q", "max_length") if n in change})

    q, p = c["q"], c["k_pages"]
    paged(ValueError, "q must be", q=q[:, :, :32])
    paged(ValueError, "q must be", q=q.cpu())
    paged(ValueError, "q must have the cache's dtype", q=q.float())
    paged(TypeError, "float32 or bfloat16", q=q.half(), k_pages=p.half(), v_pages=p.half())
    paged(wht.WhtAttentionError, "status 2", q=q[:, :3])
    paged(ValueError, "v_pages must match", v_pages=p.float())
    paged(ValueError, "v_pages must match", v_pages=p.transpose(1, 2).contiguous().transpose(1, 2))
    paged(ValueError, "k_pages must be", k_pages=p[0])
    paged(wht.WhtAttentionError, "status 2", k_pages=p[:, :, :12], v_pages=c["v_pages"][:, :, :12])
    paged(ValueError, "table must be", table=c["table"].long())
    paged(ValueError, "lengths must be", lengths=c["lengths"][:1])
    paged(ValueError, "q_starts must be", q_starts=c["starts"][:2])
    paged(ValueError, "without q_starts", q=torch.cat((q, q)))
    paged(ValueError, "prefix_table must name", prefix=17)
    paged(ValueError, "out must have", out=torch.empty(2, 5, 64, dtype=BF16, device="cuda:0"))
    paged(ValueError, "lse must be", lse=torch.empty(2, 4, dtype=BF16, device="cuda:0"))
    for scale in (0.0, -1.0, math.nan, math.inf):
        paged(wht.WhtAttentionError, "status 2", scale=scale)
    paged(wht.WhtAttentionError, "status 2", max_q=0)
    odd = torch.empty(2 * 4 * 64 + 4, dtype=BF16, device="cuda:0")[4:].view(2, 4, 64)
    paged(wht.WhtAttentionError, "status 4", q=odd)

    def append(error, match, rope=None, **change):
        x = {**c, **change}
        with pytest.raises(error, match=match):
            wht.wht_attention_append(x["q"], x["k"], x["v"], x["k_pages"], x["v_pages"], x["table"], x["lengths"], rope, **{n: x[n] for n in ("position",) if n in change})

    append(ValueError, "k must have 2 heads", k=c["q"])
    append(ValueError, "same number of rows", v=c["v"][:1])
    append(ValueError, "same number of rows", q=c["q"][:1])
    append(ValueError, "rope must be", rope=torch.zeros(10, 32, 2, dtype=torch.float64, device="cuda:0"))
    append(wht.WhtAttentionError, "status 2", rope=torch.zeros(10, 40, 2, device="cuda:0"))
    append(wht.WhtAttentionError, "status 2", position=-1)
    kept = c["k_pages"].clone()
    append(ValueError, "without q_starts", k=torch.cat((c["k"], c["k"])), v=torch.cat((c["v"], c["v"])), q=None)
    assert torch.equal(kept, c["k_pages"])


@pytest.mark.parametrize("interleaved", [False, True])
def test_native_marshalling_and_python_give_the_same(monkeypatch, interleaved):
    """The extension module takes the plain calls, and without it attention.py's own code does the same."""
    wht = _wht()
    from paper_2603_08343_amd import attention
    c = check.make(3, [2, 1, 3], [40, 1, 35], (4, 2, 128), 16, 20, seed=27)
    d = check.make(3, [1, 1, 1], [40, 1, 0], (4, 2, 64), 16, 20, F32, "token", seed=28)
    rope = [wht.wht_attention_rope_table(64, n, device="cuda:0") for n in (128, 32)]

    def calls():
        got = []
        for x, r, starts in ((c, rope[0], c["starts"]), (d, rope[1], None)):
            kp, vp = x["k_pages"].clone(), x["v_pages"].clone()
            got.append(wht.wht_attention_append(x["q"], x["k"], x["v"], kp, vp, x["table"], x["lengths"], r, starts, 20, interleaved))
            assert wht.wht_attention_append(None, x["k"], x["v"], kp, vp, x["table"], x["lengths"], None, starts) is None
            got += [kp, vp, _paged(x, lse=False), *_paged(x), *_paged(x, scale=0.25, max_length=None, out=torch.empty_like(x["q"]))]
            got.append(_paged({**x, "prefix": 0, "prefix_table": None}, lse=False, starts=starts is not None, max_q=None))
        return got

    native = attention._native()
    assert native is not attention._NoNative
    taken = []

    class Counting:
        @staticmethod
        def append(*args):
            taken.append(native.append(*args))
            return taken[-1]

        @staticmethod
        def paged(*args):
            taken.append(native.paged(*args))
            return taken[-1]

    monkeypatch.setattr(attention, "_native_module", Counting)
    ours = calls()
    assert len(taken) == 12 and all(x is not None for x in taken)
    monkeypatch.setattr(attention, "_native_module", attention._NoNative)
    assert all(torch.equal(a, b) for a, b in zip(ours, calls()))
    monkeypatch.setattr(attention, "_native_module", native)
    with pytest.raises(wht.WhtAttentionError, match="status 2"):
        _paged(c, scale=-1.0)


@pytest.mark.parametrize("native", [True, False])
@pytest.mark.parametrize("want_lse", [True, 1, np.True_, False, 0, None])
def test_want_lse_is_a_truth_value(monkeypatch, native, want_lse):
    from paper_2603_08343_amd import attention
    if not native:
        monkeypatch.setattr(attention, "_native_module", attention._NoNative)
    c = check.make(2, [1, 1], [20, 30], (4, 2, 64), 16, 10, seed=32)
    got = _paged(c, lse=want_lse)
    if want_lse:
        assert type(got) is tuple and got[0].shape == (2, 4, 64) and got[1].shape == (2, 4)
    else:
        assert got.shape == (2, 4, 64)


@pytest.mark.parametrize("native", [True, False])
@pytest.mark.parametrize("shape", [(0, 2, 16, 64), (5, 0, 16, 64), (5, 2, 0, 64), (5, 2, 16, 0)])
def test_empty_pages_are_refused(monkeypatch, native, shape):
    """Behind a prefix too, whose pages are counted by the page's size."""
    wht = _wht()
    from paper_2603_08343_amd import attention
    if not native:
        monkeypatch.setattr(attention, "_native_module", attention._NoNative)
    c = check.make(2, [1, 1], [20, 30], (4, 2, 64), 16, 10, seed=33)
    pages = torch.empty(shape, dtype=BF16, device="cuda:0")
    rows = torch.empty(2, shape[1], shape[3], dtype=BF16, device="cuda:0")
    for prefix in (0, 10):
        with pytest.raises(ValueError, match="k_pages must not be empty"):
            wht.wht_attention_paged(c["q"], pages, pages, c["table"], c["lengths"], None, c["prefix_table"], prefix)
    with pytest.raises(ValueError, match="k_pages must not be empty"):
        wht.wht_attention_append(None, rows, rows, pages, pages, c["table"], c["lengths"], None)


@pytest.mark.parametrize("native", [True, False])
@pytest.mark.parametrize("T", [0, 2])
def test_append_without_queries_returns_none(monkeypatch, native, T):
    """Whether a q_out is given or not, which stays as it was."""
    wht = _wht()
    from paper_2603_08343_amd import attention
    if not native:
        monkeypatch.setattr(attention, "_native_module", attention._NoNative)
    c = check.make(2, [1, 1], [20, 30], (4, 2, 64), 16, 0, seed=34)
    if T == 0:
        c = {**c, "k": c["k"][:0], "v": c["v"][:0], "table": c["table"][:0], "lengths": c["lengths"][:0]}
    q_out = torch.full((T, 4, 64), 7.0, dtype=BF16, device="cuda:0")
    for given in (None, q_out):
        assert wht.wht_attention_append(None, c["k"], c["v"], c["k_pages"], c["v_pages"], c["table"], c["lengths"], None, q_out=given) is None
    assert (q_out == 7.0).all()


def test_numbers_that_do_not_fit_are_refused():
    wht = _wht()
    c = check.make(2, [1, 1], [20, 30], (4, 2, 64), 16, 10, seed=35)
    for name, x in (("max_q", (1 << 32) + 1), ("max_q", 1.5), ("max_length", 1 << 64), ("prefix", 1 << 64), ("prefix", 9.5)):
        with pytest.raises(ValueError, match="must be a whole number"):
            _paged({**c, **({"prefix": x} if name == "prefix" else {})}, **({name: x} if name != "prefix" else {}))
    with pytest.raises(ValueError, match="position must be a whole number"):
        wht.wht_attention_append(None, c["k"], c["v"], c["k_pages"], c["v_pages"], c["table"], c["lengths"], None, position=1 << 64)
    # as many pages as 32 bits do not count
    wide = c["k_pages"][:1].expand(1 << 32, 2, 16, 64)
    with pytest.raises(ValueError, match="number of pages must be"):
        wht.wht_attention_paged(c["q"], wide, wide, c["table"], c["lengths"])
    want = _paged(c)
    got = _paged(c, max_q=np.int64(c["max_q"]), max_length=np.int32(c["max_length"]))
    assert torch.equal(want[0], got[0]) and torch.equal(want[1], got[1])


@pytest.mark.parametrize("dtype,heads,T", [(F32, (16, 128), (1 << 24) + 5), (BF16, (4, 64), (1 << 26) + 5)])
def test_append_of_more_tokens_than_one_row_of_a_grid_has(dtype, heads, T):
    """2^32 threads, a workgroup a token and a wave a token; all but the last five tokens are in pages that are none."""
    wht = _wht()
    H, D = heads
    g = torch.Generator(device="cuda:0").manual_seed(36)
    k, v = (torch.randn(1, H, D, generator=g, device="cuda:0").to(dtype) for _ in range(2))
    pages = [torch.zeros(1, H, 1024, D, dtype=dtype, device="cuda:0") for _ in range(2)]
    table = torch.full((1, T // 1024 + 1), -1, dtype=torch.int32, device="cuda:0")
    table[0, -1] = 0
    numbers = torch.tensor([T, 0, T], dtype=torch.int32, device="cuda:0")
    wht.wht_attention_append(None, k.expand(T, H, D), v.expand(T, H, D), *pages, table, numbers[:1], None, numbers[1:])
    for page, row in zip(pages, (k, v)):
        assert (page[0, :, :5] == row[0][:, None]).all() and (page[0, :, 5:] == 0).all()


def test_attention_of_more_rows_than_one_row_of_a_grid_has():
    """2^26 rows to join: a wave each, 2^32 threads."""
    B, H, D = 1 << 20, 64, 64
    if torch.cuda.mem_get_info()[0] < 60 << 30:
        pytest.skip("not enough memory")
    g = torch.Generator(device="cuda:0").manual_seed(37)
    q = torch.randn(1, H, D, generator=g, device="cuda:0").to(BF16).expand(B, H, D)
    k_pages, v_pages = (torch.randn(2, H, 8, D, generator=g, device="cuda:0").to(BF16) for _ in range(2))
    table = (torch.arange(B, dtype=torch.int32, device="cuda:0") & 1)[:, None]
    out = _wht().wht_attention_paged(q, k_pages, v_pages, table, torch.ones(B, dtype=torch.int32, device="cuda:0"))
    assert all((out[i::2] == v_pages[i, :, 0]).all() for i in range(2))             # one key each: its value


def far_scores(c, seed):
    """Queries and keys whose scores are exact and so far apart that the greatest takes all the weight: q's first element is 181 times a power of two of either sign, the
    keys' one of five, three of them common; beside them rows of ordinary size.  Returns where the exact rows are."""
    g = torch.Generator().manual_seed(seed)
    T, Hq, _ = c["q"].shape
    sizes = torch.tensor([4.0] + [181 * 2.0 ** e for e in (11, 12, 14, 27, 28, 31, 53, 93)])
    pick = torch.randint(0, len(sizes), (T, Hq), generator=g)
    q, sign = torch.zeros(c["q"].shape), torch.randint(0, 2, (T, Hq), generator=g) * 2 - 1
    q[:, :, 0] = sizes[pick] * sign
    k = torch.zeros(c["k_pages"].shape)
    levels = torch.tensor([0.5, 0.25, 0.125])[torch.randint(0, 3, k.shape[:3], generator=g)]
    rare = torch.rand(k.shape[:3], generator=g)
    levels[rare < 0.02], levels[rare > 0.98] = 1.0, 0.0625
    k[..., 0] = levels
    c["q"].copy_(q)
    c["k_pages"].copy_(k)
    return pick > 0


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("heads", [(4, 4, 64), (6, 2, 96), (8, 2, 128)])
@pytest.mark.parametrize("queries,lengths,prefix", [([1] * 6, [0, 1, 33, 300, 64, 700], 0), ([1] * 6, [0, 1, 33, 300, 64, 700], 515), ([3, 1, 2], [40, 1, 700], 77),
                                                    ([130, 33, 64], [500, 33, 64], 0), ([200], [1300], 70), ([64] * 3, [64, 90, 200], 10)])
def test_scores_so_large_that_a_rounding_of_them_is_large(dtype, heads, queries, lengths, prefix):
    """From 2^31 on a rounding of a score may be 128, and exp2 of that infinite or zero."""
    c = check.make(len(queries), queries, lengths, heads, 16, prefix, dtype, seed=38)
    exact = far_scores(c, 39)
    out, lse = _paged(c)
    want, want_lse, tol, tol_lse = check.attend(c)
    n = prefix + max(lengths)
    sums = (2 * n + 64) * check.F                                   # weights are exactly one and zero: additions, and the output's own rounding
    tol[exact] = (sums * float(c["v_pages"].float().abs().max()) + check.HALF[dtype] * want.abs() * 1.01)[exact]
    tol_lse[exact] = (sums + 4 * check.F * want_lse.abs())[exact]
    check.same(lse, want_lse, tol_lse, "lse")
    check.same(out, want, tol, "out")


def test_outputs_over_themselves_are_refused():
    wht = _wht()
    c = check.make(2, [1, 1], [20, 30], (4, 2, 64), 16, 10, seed=40)
    for over in (torch.empty(1, 4, 64, dtype=BF16, device="cuda:0").expand(2, 4, 64), torch.empty(2, 1, 64, dtype=BF16, device="cuda:0").expand(2, 4, 64)):
        with pytest.raises(wht.WhtAttentionError, match="overlap itself"):
            _paged(c, out=over)
        with pytest.raises(wht.WhtAttentionError, match="overlap itself"):
            wht.wht_attention_append(c["q"], c["k"], c["v"], c["k_pages"], c["v_pages"], c["table"], c["lengths"], None, q_out=over)
    n = c["k_pages"].shape[0]
    shared = [c[t][:1].expand(n, -1, -1, -1) for t in ("k_pages", "v_pages")]
    with pytest.raises(wht.WhtAttentionError, match="overlap itself"):
        wht.wht_attention_append(None, c["k"], c["v"], *shared, c["table"], c["lengths"], None)
    _paged({**c, "k_pages": shared[0], "v_pages": shared[1]})        # reading them is as good as ever
