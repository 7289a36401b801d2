// How an attention call's work is cut and where its partial results lie (include/wht_attention.h): plain arithmetic on sizes, which
// the host decides a call by and the kernels look their share up with.  Compiles without HIP.
#pragma once
#include <stddef.h>
#include <stdint.h>

#include <initializer_list>

#include "../../include/wht_attention.h"

#if defined(__HIPCC__)
#define WHT_HD __host__ __device__ __forceinline__
#else
#define WHT_HD inline
#endif

namespace wht {

WHT_HD int64_t ceil_div64(int64_t a, int64_t b) { return (a + b - 1) / b; }
WHT_HD int ceil_div(int a, int b) { return (a + b - 1) / b; }

// A row is one query of one head.  Rows that read the same keys -- G = q_heads / heads query heads, all new tokens of the
// sequence -- are taken together as the columns of one matrix product with the keys.
constexpr int kFewRows = 32;        // few-rows kernel: one tile of rows, every wave takes keys of its own
constexpr int kTileRows = 128;      // many-rows kernel: 32 rows per wave, all waves take the same keys
constexpr int kBlockKeys = 32;      // keys of one step of a wave in the few-rows kernel
constexpr int kStepKeys = 64;       // keys of one step of a workgroup in the many-rows kernel
constexpr int kWorkgroups = 512;    // two per compute unit; of float32 heads 96 and 128 wide, which take more than half of its LDS (103 and 137 KB), it holds one at a time
constexpr int kWorkers = 4 * kWorkgroups;       // waves of the few-rows kernel's grid

// A launch has below 2^32 threads along x.  Kernels that take a token or row each have this many workgroups there, and as many rows of them as it takes.
constexpr int kGridLog2 = 22;
constexpr int64_t kMostWorkgroups = ((int64_t)1 << 32) / 256 - 1;       // of 256 threads, along x

// What one call launches.  `front`: the rows of all sequences against the prefix; `own`: each sequence's rows against its own
// keys -- or, where there is no front, against prefix and own keys as one range.  A front of few rows is one more sequence on the
// few-rows kernel's line; one of many rows shares the launch with it.  Its workgroups come first in the grid: where they are one a compute unit or fewer, the line
// runs beside them; where splits_for makes them two (4 shares of 128 tiles and the like), they fill every place and the line begins as they end.  256 sequences at
// 64 and 8 x 128 behind 32768 tokens, two / one a compute unit: with 1024 to 2048 tokens of their own 529 / 474 us, with 32 to 64 293 / 343.
struct AttentionPlan {
    bool front, front_few, own_few;
    int front_splits, own_splits;           // many-rows kernel: workgroups that share a tile's keys
    bool combine;
    int32_t own_cap;                        // rows of one slot of the few-rows kernel's partial results
    size_t front_rows, own_rows;            // rows of partial results
    size_t front_at, own_at, front_sums_at, own_sums_at, cum_at, bytes;     // byte offsets in the workspace
};

// Workgroups that share a tile's keys: so that every compute unit has one, and at most one for every 256 keys begun (a tile's own keys are cut evenly in steps of 64,
// so that shares may be shorter: 257 keys of 8 tiles 192 and 65).  A second one there is worth 8 % (8 sequences of 128 new
// tokens behind 16256, 32 heads of 128: 351 us with one, 325 with two), less than partial results of short ranges cost (1000 new tokens at
// 32 x 128: 29 and 45 us), so that tiles are split for it where the shares are long.  It goes by the longest that lengths can be, and is blind to the type, though a step
// costs float32 16 times the matrix cycles.  With a table 32 times as wide as the sequences are long: 1000 new tokens at 32 x 128 30.3 -> 38.0 us, 4 x 200 at 16 x 64
// 12.1 -> 16.0, two of 4096 at 32 and 8 x 128 296 -> 290.
inline int splits_for(int64_t tiles, int64_t keys) {
    if (tiles <= 0) return 1;
    int64_t s = kWorkgroups / tiles;
    if (s > 1 && keys / s < 4096) s = kWorkgroups / 2 / tiles;
    const int64_t most = ceil_div64(keys, 256);
    if (s > most) s = most;
    return s < 1 ? 1 : (int)s;
}

// Tiles of all sequences' rows, at most: every sequence may leave one in part.
inline int64_t most_tiles(int64_t T, int64_t B, int64_t G, int64_t max_q) {
    const int64_t packed = T * G / kTileRows + B, each = B * ceil_div64((max_q < T ? max_q : T) * G, kTileRows);
    return packed < each ? packed : each;
}

// The many-rows kernel's workgroups go to the 8 dies in turn.  Groups (a sequence's head and share of its keys, `per` of them a sequence) are dealt to the
// dies, the tiles of a group one after the other, so that its keys are in one L2 once.  A workgroup looks its tile up, so that sequences of few new tokens among longer ones launch no tiles without rows:
// one prompt of 2000 tokens and 63 of one, each with 500 before, 32 and 8 heads of 128, 133 -> 87 us; 512 among 199 of one 275 -> 97; where all are alike
// the look-up adds 0.5 us.  Of sequence b's groups those of die x: how many, and the k-th.
constexpr int kDies = 8;
WHT_HD int die_groups(int b, int per, int x) { return ((b + 1) * per - x + kDies - 1) / kDies - (b * per - x + kDies - 1) / kDies; }
WHT_HD int die_group(int b, int per, int x, int k) { return ((x - b * per) & (kDies - 1)) + kDies * k; }
// The line of a die's tiles, counted up to more than a grid has, so that the sum of any numbers that q_starts may hold fits 32 bits (64 lanes' sums too): one
// sequence has 2^23 rows of tiles at most.
constexpr int kMostTiles = 1 << 24;
static_assert(kMostTiles > kMostWorkgroups / kDies, "counts are cut off where no workgroup looks");
WHT_HD int add_tiles(int sum, int tiles) { return sum + tiles < kMostTiles ? sum + tiles : kMostTiles; }
// Workgroups that a die needs at most.
inline int64_t die_blocks(int64_t T, int64_t B, int64_t G, int64_t max_q, int64_t per) {
    const int64_t packed = ceil_div64(per, kDies) * (T * G / kTileRows + B), each = ceil_div64(B * per, kDies) * ceil_div64((max_q < T ? max_q : T) * G, kTileRows);
    return packed < each ? packed : each;
}

inline AttentionPlan plan_attention(int64_t T, int32_t B, int32_t q_heads, int32_t heads, int32_t head_dim, int32_t max_q,
                                    int64_t max_length, int64_t prefix, int workers = kWorkers) {
    AttentionPlan p{};
    const int64_t G = q_heads / heads;
    p.own_few = max_q * G <= kFewRows;
    // Several sequences of few rows each: their rows together read the prefix once.  Where a sequence's own rows fill tiles by themselves nothing is saved
    // by that, and prefix and own keys are one range; as where the prefix, read by every sequence, is two blocks for each worker or fewer:
    // apart / as one range, in us: 15 sequences behind 1 token, 16 heads of 128, 28.4 / 11.9; 8 behind 2048, 8 key heads, 22.1 / 20.1;
    // 32 behind 1024 (four blocks) 18.2 / 29.2.  Counting the prefix's blocks alone, it is wrong where the own keys are many and the prefix short beside them:
    // 200 behind 64, 16 of 64 (three blocks) 60.5 / 50.8, which are taken apart.
    p.front = prefix > 0 && B > 1 && p.own_few && (int64_t)B * heads * ceil_div64(prefix, kBlockKeys) > 2 * kWorkers;
    p.front_few = T * G <= kFewRows;
    p.front_splits = p.own_splits = 1;
    if (p.front) {
        if (!p.front_few) {
            p.front_splits = splits_for(ceil_div64(T * G, kTileRows) * heads, prefix);
            p.front_rows = (size_t)p.front_splits * (size_t)(T * q_heads);
        }
    }
    p.own_cap = p.front && p.front_few ? (int32_t)(T * G) : max_q * (int32_t)G;
    if (p.own_few) p.own_rows = (((size_t)B + 1) * heads + (size_t)workers) * (size_t)p.own_cap;
    else {
        p.own_splits = splits_for(most_tiles(T, B, G, max_q) * heads, max_length + prefix);
        if (p.own_splits > 1) p.own_rows = (size_t)p.own_splits * (size_t)(T * q_heads);
    }
    p.combine = p.front || p.own_few || p.own_splits > 1;
    size_t at = 0;
    auto take = [&](size_t bytes) { const size_t here = at; at += (bytes + 255) & ~(size_t)255; return here; };
    p.front_at = take(p.front_rows * head_dim * 4);
    p.own_at = take(p.own_rows * head_dim * 4);
    p.front_sums_at = take(p.front_rows * 8);
    p.own_sums_at = take(p.own_rows * 8);
    p.cum_at = take(p.own_few ? ((size_t)B + 2) * 4 : 0);
    p.bytes = at;
    return p;
}

// The few-rows kernel's line: the blocks of all items one after the other, an equal share of them to a worker (a wave).  The pieces of an item
// of n blocks from u0 on lie in the slots item + w of the workers w that it meets: first .. first + count - 1.  A piece writes `rows`
// rows of results, 4 bytes an element, for the keys and values it reads: where there is more than a block for every worker, a share is a
// block for every eight rows at least.  For every four / eight / sixteen rows, in us, 32 and 8 x 128: 8 sequences of 8 new tokens and 750 to 1500 of their own
// 28.3 / 23.6 / 24.9, 4 of 8 and 2000 to 4000 27.0 / 23.8 / 26.8, 32 of 8 and 750 to 1500 52.4 / 50.0 / 49.9, 8 of 4 and 750 to 1500 19.8 / 20.3 / 20.3.
// With a gang of heads a worker is a workgroup, an item a group of heads, and every slot holds one piece for each of them.
struct Slots { int64_t first; int count; };
template <int WORKERS = kWorkers>
WHT_HD int line_share(int total, int rows, int gang_log2) {
    int even;
    if constexpr ((WORKERS & (WORKERS - 1)) == 0) {
        const int workers_log2 = __builtin_ctz(WORKERS) - gang_log2;
        even = (total + (1 << workers_log2) - 1) >> workers_log2;
    } else even = (int)((((uint64_t)(unsigned)total << gang_log2) + WORKERS - 1) / WORKERS);
    const int least = even > 1 ? (rows + 7) >> 3 : 1;
    return even > least ? even : least;
}
template <int WORKERS = kWorkers>
WHT_HD Slots item_slots(int item, int u0, int n, int total, int rows, int gang_log2) {
    if (n == 0) return {0, 0};
    const int per = line_share<WORKERS>(total, rows, gang_log2), w0 = u0 / per, w1 = (u0 + n - 1) / per;
    return {(int64_t)item + w0, w1 - w0 + 1};
}
// Four heads side by side: where a row is no whole number of 128-byte lines, and the next head's row follows it in memory.
constexpr int kGangLog2 = 2;
inline int gang_log2_of(int32_t heads, int64_t row_bytes, int64_t head_stride_bytes) {
    return row_bytes % 128 != 0 && head_stride_bytes == row_bytes && heads % (1 << kGangLog2) == 0 ? kGangLog2 : 0;
}

// Whether the few-rows kernel reads a call's own keys and values past the caches (a prefix that several sequences share is not): where they are more than the share
// of the 256 MB Infinity Cache that a step of a few layers leaves each of them.  Lengths are on the GPU: it goes by what they can be, and counts a prefix once.  Three caches
// read in turn, kept / past, us: 1 sequence at 32 and 8 x 128, 80 MB 23.4 / 23.8, 96 MB 26.3 / 26.2, 112 MB 31.3 / 28.6, 256 MB 55.4 / 49.0; 16 of them 21.7 / 22.2,
// 25.6 / 25.3, 31.2 / 28.1, 55.6 / 48.9; 128 at 16 x 64 23.8 / 23.2, 26.5 / 25.6, 30.3 / 27.9, 55.0 / 49.3; 16 float32 ones at 12 x 64 28.0 / 28.5, 29.3 / 29.3,
// 33.8 / 32.5, 58.3 / 53.6.  Not with four heads side by side, whose lines are shared by two loads: 200 sequences at 16 x 96 96.8 / 100.3.
inline bool streams(int32_t B, int32_t heads, int32_t head_dim, int64_t size, int64_t max_length, int64_t prefix, int32_t gang_log2) {
    return gang_log2 == 0 && ((double)B * max_length + prefix) * heads * head_dim * 2 * size >= 96e6;
}

// Waves that share a row's pieces where the few-rows kernel left them: more where few rows have to fill the chip.  Both kernels with 16 / 4 / 1 of them, in us, 128 wide:
// 32 rows of 256 pieces 30.6 / 32.3 / 45.7, 16 of 1000 22.0 / 33.5 / 91.3, 256 of 256 24.4 / 24.6 / 30.5, but of 32 pieces 19.0 / 18.3 / 18.9 and 32 of 4 10.3 / 10.1 / 9.7;
// 512 of 64 25.2 / 23.9 / 26.1, 1024 of 64 31.3 / 26.1 / 26.7, but of 8 47.0 / 42.1 / 41.6; 2048 of 4 83.6 / 74.9 / 72.4; 4096 of 2 157.2 / 140.1 / 134.3.  How many
// pieces a row has is not asked for, which costs up to 1.3 us where they are few and up to a tenth between 1024 and 2048 rows.
inline int join_waves(int64_t rows) { return rows <= 256 ? 16 : rows <= 2048 ? 4 : 1; }

// Argument checks, in the order of the status codes.
inline bool good_rows(const wht_attention_rows_t* r, int heads, int head_dim, int size) {
    return ((uintptr_t)r->data & 15u) == 0 && r->token_stride * size % 16 == 0 && r->head_stride * size % 16 == 0 && r->token_stride >= 0 &&
           (r->head_stride >= head_dim || heads == 1) && r->head_stride >= 0 && r->head_stride * size < (int64_t)1 << 31;
}

// What is written has a place of its own for every vector: of its dimensions, from the shortest stride on, each passes all of those before.
struct Dimension { int64_t count, stride; };
inline bool apart(Dimension a, Dimension b, Dimension c, int head_dim) {
    auto swap_longer = [](Dimension& x, Dimension& y) { if (x.count > 1 && (y.count <= 1 || x.stride > y.stride)) { const Dimension t = x; x = y; y = t; } };
    swap_longer(a, b);
    swap_longer(b, c);
    swap_longer(a, b);
    double extent = head_dim;                                       // the products may pass 64 bits
    for (const Dimension& d : {a, b, c}) {
        if (d.count <= 1) continue;
        if ((double)d.stride < extent) return false;
        extent += (double)(d.count - 1) * (double)d.stride;
    }
    return true;
}

inline int check_cache(const wht_attention_cache_t* c, const wht_attention_batch_t* b, int32_t dtype) {
    if (!c || !b || !c->k || !c->v || !b->table || !b->lengths) return WHT_ERR_NULL_PTR;
    if (dtype != WHT_DTYPE_F32 && dtype != WHT_DTYPE_BF16) return WHT_ERR_BAD_DTYPE;
    const int size = dtype == WHT_DTYPE_F32 ? 4 : 2;
    if (c->head_dim != 64 && c->head_dim != 96 && c->head_dim != 128) return WHT_ERR_BAD_DIM;
    if (c->page_size < WHT_ATTENTION_MIN_PAGE || c->page_size > WHT_ATTENTION_MAX_PAGE || (c->page_size & (c->page_size - 1)) != 0) return WHT_ERR_BAD_DIM;
    if (c->heads < 1 || c->heads > 1024 || c->pages < 1 || b->B < 0 || b->B > 1 << 30 || b->width < 1 || b->table_stride < 0) return WHT_ERR_BAD_DIM;
    if ((int64_t)b->width * c->page_size > (int64_t)1 << 30) return WHT_ERR_BAD_DIM;
    // the kernels multiply a page's number by its stride in bytes (both 32 bits) and keep a row's place in its page in 31
    if (c->page_stride < 0 || c->page_stride * size >= (int64_t)1 << 32 || c->token_stride < c->head_dim ||
        (c->page_size - 1) * c->token_stride * size >= (int64_t)1 << 31 || c->head_stride < 0) return WHT_ERR_BAD_DIM;
    if (((uintptr_t)c->k & 15u) != 0 || ((uintptr_t)c->v & 15u) != 0 || c->page_stride * size % 16 != 0 || c->head_stride * size % 16 != 0 ||
        c->token_stride * size % 16 != 0) return WHT_ERR_MISALIGNED;
    if (((uintptr_t)b->table & 3u) != 0 || ((uintptr_t)b->lengths & 3u) != 0 || ((uintptr_t)b->q_starts & 3u) != 0) return WHT_ERR_MISALIGNED;
    return WHT_OK;
}

inline int check_append(const wht_attention_rows_t* q, const wht_attention_rows_t* k, const wht_attention_rows_t* v,
                        const wht_attention_rows_t* q_out, int64_t T, int32_t q_heads, const wht_attention_cache_t* c,
                        const wht_attention_batch_t* b, const float* rope, int64_t rope_rows, int32_t rotary, int64_t position,
                        int32_t dtype) {
    if (!q || !k || !v || !q_out || !k->data || !v->data || (q->data && !q_out->data) || (rotary != 0 && !rope)) return WHT_ERR_NULL_PTR;
    if (int rc = check_cache(c, b, dtype)) return rc;
    const int size = dtype == WHT_DTYPE_F32 ? 4 : 2;
    if (T < 0 || T > (int64_t)1 << 30 || (q->data && (q_heads < 1 || q_heads > 1024))) return WHT_ERR_BAD_DIM;
    if (rotary < 0 || rotary % 16 != 0 || rotary > c->head_dim || rope_rows < 0 || rope_rows > (int64_t)1 << 30) return WHT_ERR_BAD_DIM;
    if (position < 0 || position > (int64_t)1 << 30) return WHT_ERR_BAD_DIM;
    if (!good_rows(k, c->heads, c->head_dim, size) || !good_rows(v, c->heads, c->head_dim, size) || ((uintptr_t)rope & 15u) != 0) return WHT_ERR_MISALIGNED;
    if (q->data && (!good_rows(q, q_heads, c->head_dim, size) || !good_rows(q_out, q_heads, c->head_dim, size))) return WHT_ERR_MISALIGNED;
    if (q->data && !apart({T, q_out->token_stride}, {q_heads, q_out->head_stride}, {1, 0}, c->head_dim)) return WHT_ERR_MISALIGNED;
    if (!apart({c->pages, c->page_stride}, {c->heads, c->head_stride}, {c->page_size, c->token_stride}, c->head_dim)) return WHT_ERR_MISALIGNED;
    return WHT_OK;
}

inline int check_sizes(int64_t T, int32_t B, int32_t q_heads, int32_t heads, int32_t head_dim, int32_t max_q, int64_t max_length,
                       int64_t prefix, int32_t dtype) {
    if (dtype != WHT_DTYPE_F32 && dtype != WHT_DTYPE_BF16) return WHT_ERR_BAD_DTYPE;
    if (head_dim != 64 && head_dim != 96 && head_dim != 128) return WHT_ERR_BAD_DIM;
    if (T < 0 || B < 0 || B > 1 << 20 || heads < 1 || heads > 1024 || q_heads < 1 || q_heads > 1024 || q_heads % heads != 0) return WHT_ERR_BAD_DIM;
    if (T * q_heads > (int64_t)1 << 30 || max_q < 1 || (int64_t)max_q * (q_heads / heads) > (int64_t)1 << 30) return WHT_ERR_BAD_DIM;
    if (prefix < 0 || prefix > (int64_t)1 << 30 || max_length < 0 || max_length > (int64_t)1 << 30) return WHT_ERR_BAD_DIM;
    return WHT_OK;
}

// The kernels' exponentials are of base 2.
inline float base2_scale(float scale) {
    const double s = (double)scale * 1.4426950408889634074;
    return s <= 3.4028234663852886e38 ? (float)s : __builtin_inff();        // past the largest float; what rounds to it is taken
}

inline int check_paged(const wht_attention_rows_t* q, const wht_attention_rows_t* out, const float* lse, int64_t T, int32_t q_heads,
                       const wht_attention_cache_t* c, const wht_attention_batch_t* b, const int32_t* prefix_table, int64_t prefix,
                       int32_t max_q, int64_t max_length, float scale, int32_t dtype) {
    if (!q || !out || !q->data || !out->data || (prefix > 0 && !prefix_table)) return WHT_ERR_NULL_PTR;
    if (int rc = check_cache(c, b, dtype)) return rc;
    if (int rc = check_sizes(T, b->B, q_heads, c->heads, c->head_dim, max_q, max_length, prefix, dtype)) return rc;
    if (!(scale > 0.0f) || !(base2_scale(scale) < __builtin_inff())) return WHT_ERR_BAD_DIM;
    // the few-rows kernel counts the blocks of its line in 31 bits
    const int64_t own = (int64_t)b->width * c->page_size < max_length ? (int64_t)b->width * c->page_size : max_length;
    if (((int64_t)b->B + 1) * (own / kBlockKeys + prefix / kBlockKeys + 2) > INT32_MAX / c->heads) return WHT_ERR_BAD_DIM;
    const int size = dtype == WHT_DTYPE_F32 ? 4 : 2;
    if (!good_rows(q, q_heads, c->head_dim, size) || !good_rows(out, q_heads, c->head_dim, size)) return WHT_ERR_MISALIGNED;
    if (!apart({T, out->token_stride}, {q_heads, out->head_stride}, {1, 0}, c->head_dim)) return WHT_ERR_MISALIGNED;
    if (((uintptr_t)lse & 3u) != 0 || ((uintptr_t)prefix_table & 3u) != 0) return WHT_ERR_MISALIGNED;
    return WHT_OK;
}

}  // namespace wht
