"""What an attention call launches, by the library's own rules (csrc/attention_plan.h, built for the host as csrc/attention_query.cpp), so that
a test of a kernel's path says that its call takes it."""
import ctypes
import functools

from paper_2603_08343_amd import build

NAMES = ("front", "front_few", "own_few", "front_splits", "own_splits", "own_cap", "join_waves", "gang_log2", "streams")
BLOCK, WORKERS_LOG2 = 32, 11                                         # kBlockKeys, kWorkersLog2


@functools.lru_cache(maxsize=None)
def _lib():
    lib = ctypes.CDLL(build.ATTENTION_QUERY_LIB)
    i32, i64 = ctypes.c_int32, ctypes.c_int64
    lib.wht_query_attention.argtypes = [i64, i32, i32, i32, i32, i32, i64, i64, i64, i32, i64, ctypes.POINTER(i64)]
    lib.wht_query_attention.restype = None
    lib.wht_query_line_share.argtypes = [i32, i32, i32]
    return lib


def route(c, max_q=None, max_length=None, rows=None):
    """Of a batch that attention_check.make describes: the plan, and `share`, the few-rows kernel's blocks a worker."""
    T, q_heads, dim = c["q"].shape
    heads, page = c["k_pages"].shape[1:3]
    B, width = c["table"].shape
    capacity = width * page
    max_length = capacity if max_length is None else max_length
    out = (ctypes.c_int64 * len(NAMES))()
    _lib().wht_query_attention(T if rows is None else rows, B, q_heads, heads, dim, c["max_q"] if max_q is None else max_q, max_length, min(capacity, max_length),
                               c["prefix"], {2: 1, 4: 0}[c["q"].element_size()], c["k_pages"].stride(1), out)
    r = dict(zip(NAMES, out))
    if r["own_few"]:
        starts, front = c["starts"].tolist(), -(-c["prefix"] // BLOCK)
        each = [-(-n // BLOCK) + (0 if r["front"] else front) for b, n in enumerate(c["lengths"].tolist()) if starts[b + 1] > starts[b]]
        total = (sum(each) + (front if r["front_few"] and r["front"] else 0)) * (heads >> r["gang_log2"])
        r["share"] = _lib().wht_query_line_share(total, r["own_cap"], r["gang_log2"])
    return r
