"""The append to the cache in 4 bits on each of the ways that a call can take: a wave a token where there are many of them, a workgroup where there are few and wide
ones, and more heads than either takes at once.  Codes and scales against the definition bit by bit, queries within the bounds that count their roundings."""
import pytest
import torch

import attention4_check as check
import paper_2603_08343_amd as wht
from test_gpu_attention4 import check_append

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
B16, F32 = torch.bfloat16, torch.float32

# From 2048 tokens on, and where a token has fewer than 256 vectors of 8 elements of its queries, keys and values, a wave takes a token, 4 heads of 128 (5 of 96, 8 of 64) at a
# time, else a workgroup, four times as many; four such rounds of bfloat16 queries, two of float32, are read together.
CASES = [  # queries, lengths, heads, page, order, rotary, interleaved, transformed, dtype
    ([1000, 1051], [1000, 1200], (32, 8, 128), 16, "head", 128, False, True, B16),       # a wave a token: 8 rounds of queries, 4 of keys and values
    ([2048], [2100], (32, 8, 128), 64, "token", 64, True, False, B16),
    ([1025, 3, 1025], [1030, 3, 1500], (16, 16, 96), 16, "head", 96, False, True, B16),
    ([2047], [2047], (16, 16, 96), 32, "token", 48, False, True, B16),                   # one fewer: a workgroup
    ([2049], [2049], (12, 4, 64), 16, "outer", 64, False, True, B16),
    ([700, 1350], [700, 1400], (16, 4, 128), 16, "head", 128, False, True, F32),
    ([2050], [2050], (12, 12, 96), 8, "token", 96, True, False, F32),
    ([20, 3], [40, 3], (80, 8, 128), 16, "head", 128, False, True, B16),                 # a workgroup: 5 rounds of queries, the fifth in part
    ([13], [13], (136, 2, 128), 16, "head", 128, True, True, B16),                       # 9
    ([9, 8], [9, 30], (105, 5, 96), 16, "head", 96, False, False, B16),                  # 20 heads at a time
    ([17], [17], (257, 1, 64), 16, "token", 32, False, True, B16),                       # 32 heads at a time
    ([11], [11], (48, 48, 128), 32, "head", 0, False, True, F32),
    ([5], [5], (90, 18, 96), 16, "token", 96, False, True, F32),
]


@pytest.mark.parametrize("case", CASES, ids=str)
def test_append(case):
    queries, lengths, heads, page, order, rotary, interleaved, transformed, dtype = case
    c = check.make4(len(queries), queries, lengths, heads, page, dtype=dtype, order=order)
    rope = wht.wht_attention_rope_table(3 + max(lengths), rotary, device=DEV) if rotary else None
    twin = {n: t.clone() if torch.is_tensor(t) else t for n, t in c.items()}
    check_append(c, rope, 3, interleaved=interleaved, transformed=transformed)
    check_append(twin, rope, 3, interleaved=interleaved, transformed=transformed, q_out=twin["q"])           # in place
    alone = {n: t.clone() if torch.is_tensor(t) else t for n, t in c.items()}
    for n in ("k_pages", "v_pages", "k_scales", "v_scales"):
        alone[n].zero_()
        c[n].zero_()
    pages = [alone[n] for n in ("k_pages", "v_pages", "k_scales", "v_scales")]
    kw = {"q_starts": c["starts"], "position": 3, "interleaved": interleaved, "transform": transformed}
    wht.wht_attention_append4(c["q"], c["k"], c["v"], *(c[n] for n in ("k_pages", "v_pages", "k_scales", "v_scales")), c["table"], c["lengths"], rope, **kw)
    wht.wht_attention_append4(None, c["k"], c["v"], *pages, c["table"], c["lengths"], rope, **kw)           # without queries: the other number of vectors
    assert all(torch.equal(c[n], alone[n]) for n in ("k_pages", "v_pages", "k_scales", "v_scales"))


@pytest.mark.parametrize("cyclic", [False, True])
@pytest.mark.parametrize("heads,T", [((32, 8, 128), 2051), ((80, 8, 128), 30)], ids=str)
def test_several_axes(heads, T, cyclic):
    c = check.make4(1, [T], [T], heads, 16)
    positions = torch.randint(0, 50, (T, 3), generator=torch.Generator().manual_seed(2)).to(torch.int32)
    positions[7, 1] = 50                                             # outside the table: a row of NaN, not stored
    rope = wht.wht_attention_rope_table(50, heads[2], device=DEV)
    check_append(c, rope, positions=positions.to(DEV), axes=wht.wht_rotary_axes((16, 24, 24), cyclic))


@pytest.mark.parametrize("T", [2050, 60])
def test_places_that_are_not_there(T):
    """Bad pages, places past the table and padding rows among many tokens."""
    c = check.make4(2, [T - 20, 20], [T - 20, 40], (32, 8, 128), 16)
    c["table"][0, 1], c["table"][1, 1] = c["k_pages"].shape[0], -1
    c["lengths"][0] += 16 * c["table"].shape[1] - (T - 20) + 5       # five past the table
    for n in ("q", "k", "v"):
        c[n] = torch.cat((c[n], torch.full_like(c[n][:3], 3.0)))
    check_append(c, wht.wht_attention_rope_table(5000, 128, device=DEV), 1)
