"""What a call of the attention over 4 bits launches, by the library's own rules (csrc/attention4_plan.h, built for the host as csrc/attention_query.cpp), so
that a test of a kernel's path says that its call takes it."""
import ctypes
import functools

from paper_2603_08343_amd import build

NAMES = ("front", "front_few", "own_few", "whole", "front_splits", "own_splits", "own_cap", "join_waves", "gang_log2", "past", "tiles", "workers")
BLOCK = 32                                                           # kBlockKeys


@functools.lru_cache(maxsize=None)
def _lib():
    lib = ctypes.CDLL(build.ATTENTION_QUERY_LIB)
    i32, i64 = ctypes.c_int32, ctypes.c_int64
    lib.wht_query_attention4.argtypes = [i64, i32, i32, i32, i32, i32, i64, i64, i64, i32, i32, i64, ctypes.POINTER(i64)]
    lib.wht_query_attention4.restype = None
    lib.wht_query_line_share4.argtypes = [i32, i32, i32, i32]
    return lib


def route(c, max_q=None, max_length=None, rows=None):
    """Of a batch as attention4_check.make4 describes it: the plan, and `share`, the blocks of a worker on the few-rows kernel's line, or of a wave of an item
    that is taken whole (the longest's)."""
    T, q_heads, dim = c["q"].shape
    heads, page = c["k_pages"].shape[1:3]
    B, width = c["table"].shape
    capacity = width * page
    max_length = capacity if max_length is None else max_length
    f32 = c["q"].element_size() == 4
    out = (ctypes.c_int64 * len(NAMES))()
    _lib().wht_query_attention4(T if rows is None else rows, B, q_heads, heads, dim, c["max_q"] if max_q is None else max_q, max_length, min(capacity, max_length),
                                c["prefix"], 0 if f32 else 1, page, c["k_pages"].stride(1), out)
    r = dict(zip(NAMES, out))
    if r["own_few"]:
        starts, front = c["starts"].tolist(), -(-c["prefix"] // BLOCK)
        each = [-(-n // BLOCK) + (0 if r["front"] else front) for b, n in enumerate(c["lengths"].tolist()) if starts[b + 1] > starts[b]]
        total = (sum(each) + (front if r["front_few"] and r["front"] else 0)) * (heads >> r["gang_log2"])
        r["share"] = -(-max(each) // (4 if f32 and r["tiles"] == 2 else 8)) if r["whole"] else _lib().wht_query_line_share4(total, r["own_cap"], r["gang_log2"], r["workers"])
    return r
