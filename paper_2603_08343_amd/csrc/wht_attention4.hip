// Dispatch and C ABI of the paged cache in 4 bits, its attention (include/wht_attention4.h) and rotary positions of several axes
// (include/wht_rotary.h).
#include "attention4_device.h"

namespace wht {

template <class F>
static int with_type(int dtype, int head_dim, F&& f) {
    auto width = [&](auto t) {
        switch (head_dim) {
        case 64: return f(t, std::integral_constant<int, 64>{});
        case 96: return f(t, std::integral_constant<int, 96>{});
        default: return f(t, std::integral_constant<int, 128>{});
        }
    };
    return dtype == WHT_DTYPE_F32 ? width(float{}) : width(bf16{});
}

// f with a std::bool_constant for each flag.
template <class F> static void with_flags(F&& f) { f(); }
template <class F, class... Rest>
static void with_flags(F&& f, bool first, Rest... rest) {
    if (first) with_flags([&](auto... x) { f(std::true_type{}, x...); }, rest...);
    else with_flags([&](auto... x) { f(std::false_type{}, x...); }, rest...);
}

static int launched() { return hipGetLastError() == hipSuccess ? WHT_OK : WHT_ERR_LAUNCH; }

static dim3 grid_of(int64_t blocks) {
    const int64_t x = (int64_t)1 << kGridLog2;
    return blocks <= x ? dim3((unsigned)blocks) : dim3((unsigned)x, (unsigned)ceil_div64(blocks, x));
}

static Batch batch_of(const wht_attention_batch_t* b, int64_t T, int64_t most) {
    return {b->table, b->lengths, b->q_starts, b->table_stride, b->B, (int)T, (int)most};
}

static Turning turning(const float* rope, int64_t rope_rows, int32_t rotary, int32_t interleaved, const int32_t* positions, int32_t axes,
                       const uint8_t* pair_axes, int32_t inverse) {
    Turning t{};
    t.rope = rope; t.positions = positions; t.rope_rows = rope_rows; t.rotary = rotary; t.axes = axes;
    t.interleaved = interleaved != 0; t.inverse = inverse != 0;
    for (int i = 0; i < rotary / 2; ++i) {
        if (pair_axes) t.pair_axes[i] = pair_axes[i];
        t.used |= 1 << t.pair_axes[i];
    }
    return t;
}

// A wave takes a token where there are enough of them to fill the chip, or where it has few vectors of 8 elements of its queries, keys and values; a workgroup
// where few tokens have many, which is sooner done.  Workgroup / wave, in us: 32 and 8 x 128 (768 vectors) 256 tokens 7.1 / 12.3, 1024 11.7 / 16.4, 4096 27.7 / 26.9,
// 16384 118 / 103; 16 x 96 (576) 256 7.4 / 13.2, 1024 13.0 / 16.5, 4096 31.9 / 29.7; 12 x 64 (288) 256 7.0 / 8.5, 1024 9.1 / 9.3, 4096 23.2 / 16.6;
// 16 and 4 x 64 (192) 256 7.1 / 6.9, 1024 8.7 / 7.2.
constexpr int kManyTokens4 = 2048, kWideToken4 = 256;

static int append4(const wht_attention_rows_t* q, const wht_attention_rows_t* k, const wht_attention_rows_t* v, const wht_attention_rows_t* q_out,
                   const wht_attention_rows_t* k_out, const wht_attention_rows_t* v_out, int64_t T, int32_t q_heads, const wht_attention_cache4_t* c,
                   const wht_attention_batch_t* b, const Turning& turn, int64_t position, int32_t transform, int32_t dtype, hipStream_t stream) {
    const int64_t size = dtype == WHT_DTYPE_F32 ? 4 : 2;
    Append4Args a{};
    a.batch = batch_of(b, T, INT32_MAX);
    a.places = b->width * c->page_size;
    a.q = static_cast<const unsigned char*>(q->data);
    a.kn = static_cast<const unsigned char*>(k->data);
    a.vn = static_cast<const unsigned char*>(v->data);
    a.q_out = static_cast<unsigned char*>(q_out->data);
    a.k_out = static_cast<unsigned char*>(k_out->data);
    a.v_out = static_cast<unsigned char*>(v_out->data);
    a.k = static_cast<unsigned char*>(c->k);
    a.v = static_cast<unsigned char*>(c->v);
    a.ks = c->k_scales;
    a.vs = c->v_scales;
    a.q_ts = q->token_stride * size; a.q_hs = q->head_stride * size;
    a.k_ts = k->token_stride * size; a.k_hs = k->head_stride * size;
    a.v_ts = v->token_stride * size; a.v_hs = v->head_stride * size;
    a.qo_ts = q_out->token_stride * size; a.qo_hs = q_out->head_stride * size;
    a.ko_ts = k_out->token_stride * size; a.ko_hs = k_out->head_stride * size;
    a.vo_ts = v_out->token_stride * size; a.vo_hs = v_out->head_stride * size;
    a.page_stride = c->page_stride; a.head_stride = c->head_stride; a.token_stride = c->token_stride;
    a.s_page_stride = c->scale_page_stride; a.s_head_stride = c->scale_head_stride; a.s_token_stride = c->scale_token_stride;
    a.q_heads = q_heads; a.heads = c->heads; a.pages = c->pages; a.page_shift = __builtin_ctz((unsigned)c->page_size); a.position = (int)position;
    a.transform = transform != 0;
    a.turn = turn;
    return with_type(dtype, c->head_dim, [&](auto t, auto d) {
        using E = decltype(t);
        constexpr int D = decltype(d)::value;
        const int vectors = (int)((a.q ? q_heads : 0) + 2 * c->heads) * (D / 8);
        if (T >= kManyTokens4 || vectors < kWideToken4) hipLaunchKernelGGL((append4_kernel<E, D, 64>), grid_of(ceil_div64(T, 4)), dim3(256), 0, stream, a);
        else hipLaunchKernelGGL((append4_kernel<E, D, 256>), dim3((unsigned)T, 1, a.q ? 2 : 1), dim3(256), 0, stream, a);
        return launched();
    });
}

static int rotate(const wht_attention_rows_t* x, const wht_attention_rows_t* out, int64_t T, int32_t heads, int32_t head_dim, const Turning& turn,
                  int32_t dtype, hipStream_t stream) {
    const int64_t size = dtype == WHT_DTYPE_F32 ? 4 : 2;
    RotaryArgs a{};
    a.x = static_cast<const unsigned char*>(x->data);
    a.out = static_cast<unsigned char*>(out->data);
    a.x_ts = x->token_stride * size; a.x_hs = x->head_stride * size;
    a.o_ts = out->token_stride * size; a.o_hs = out->head_stride * size;
    a.T = (int)T; a.heads = heads; a.pairs = (int)(head_dim * size / 32);
    a.turn = turn;
    with_flags([&](auto f32, auto interleaved) {
        using E = std::conditional_t<decltype(f32)::value, float, bf16>;
        hipLaunchKernelGGL((rotary_kernel<E, decltype(interleaved)::value>), grid_of(ceil_div64(T, 4)), dim3(256), 0, stream, a);
    }, dtype == WHT_DTYPE_F32, turn.interleaved);
    return launched();
}

static int paged4(const wht_attention_rows_t* q, const wht_attention_rows_t* out, float* lse, int64_t T, int32_t q_heads,
                  const wht_attention_cache4_t* c, const wht_attention_batch_t* b, const int32_t* prefix_table, int64_t prefix, int32_t max_q,
                  int64_t max_length, float scale, int32_t transform, int32_t dtype, const AttentionPlan4& p, unsigned char* ws, hipStream_t stream) {
    const int64_t size = dtype == WHT_DTYPE_F32 ? 4 : 2;
    const int64_t table_keys = (int64_t)b->width * c->page_size;
    Attention4Args args{};
    AttentionArgs& a = args.base;
    a.batch = batch_of(b, T, table_keys < max_length ? table_keys : max_length);
    a.q = static_cast<const unsigned char*>(q->data);
    a.k = static_cast<const unsigned char*>(c->k);
    a.v = static_cast<const unsigned char*>(c->v);
    a.out = static_cast<unsigned char*>(out->data);
    a.lse = lse;
    a.q_ts = q->token_stride * size; a.q_hs = q->head_stride * size;
    a.out_ts = out->token_stride * size; a.out_hs = out->head_stride * size;
    a.head_stride = c->head_stride;
    a.page_stride = (unsigned)c->page_stride; a.token_stride = (unsigned)c->token_stride;
    args.ks = c->k_scales; args.vs = c->v_scales;
    args.s_head_stride = c->scale_head_stride;
    args.s_page_stride = (unsigned)c->scale_page_stride; args.s_token_stride = (unsigned)c->scale_token_stride;
    args.transform = transform != 0;
    a.prefix_table = prefix_table;
    a.q_heads = q_heads; a.heads = c->heads; a.G = q_heads / c->heads; a.pages = c->pages; a.page_shift = __builtin_ctz((unsigned)c->page_size);
    a.prefix = (int)prefix; a.max_q = max_q;
    a.scale = base2_scale(scale);
    Attention4Args f = args;
    int64_t front_blocks = 0;
    if (p.front && !p.front_few) {
        f.base.use_prefix = 1; f.base.splits = p.front_splits;
        f.base.part = reinterpret_cast<float*>(ws + p.front_at); f.base.sums = reinterpret_cast<float*>(ws + p.front_sums_at);
        front_blocks = kDies * die_blocks(T, 1, a.G, T, (int64_t)c->heads * f.base.splits);
    }
    a.use_prefix = !p.front && prefix > 0;
    a.front_item = p.front && p.front_few;
    a.gang_log2 = gang_log2_of(c->heads, c->head_dim / 2, a.head_stride);
    const bool past = streams4(b->B, c->heads, c->head_dim, a.batch.most, a.use_prefix ? prefix : 0, a.gang_log2);
    a.splits = p.own_splits; a.rows_cap = p.own_cap;
    a.part = reinterpret_cast<float*>(ws + p.own_at); a.sums = reinterpret_cast<float*>(ws + p.own_sums_at);
    a.cum = reinterpret_cast<int*>(ws + p.cum_at);
    const bool two_tiles = tiles4(c->page_size, p.own_cap) == 2;
    const int workgroups = workgroups4(dtype == WHT_DTYPE_F32, c->head_dim, two_tiles ? 2 : 1, front_blocks > 0);
    const int64_t each = die_blocks(T, b->B, a.G, max_q, (int64_t)c->heads * a.splits), own_blocks = p.own_few ? workgroups : (each + 1) * kDies;
    if (front_blocks + own_blocks > kMostWorkgroups) return WHT_ERR_BAD_DIM;
    a.fill = (int)each;
    const int rc = with_type(dtype, c->head_dim, [&](auto t, auto d) {
        using E = decltype(t);
        constexpr int D = decltype(d)::value;
        const dim3 grid((unsigned)(front_blocks + own_blocks)), block(256);
        if (p.whole) {
            with_flags([&](auto two, auto multi) {
                constexpr int kTiles = decltype(two)::value ? 2 : 1;
                constexpr bool kMulti = decltype(multi)::value;
                const dim3 items((unsigned)(b->B * c->heads)), threads(64 * kWholeWaves<E, kTiles>);
                if constexpr (kTiles == 2 && kMulti) {
                    if (a.page_shift < 4) {
                        hipLaunchKernelGGL((whole_rows4_kernel<E, D, kTiles, kMulti, true>), items, threads, 0, stream, args);
                        return;
                    }
                }
                hipLaunchKernelGGL((whole_rows4_kernel<E, D, kTiles, kMulti, false>), items, threads, 0, stream, args);
            }, two_tiles, a.page_shift < 4 || max_q > 1);
            return launched();
        }
        if (!p.own_few) hipLaunchKernelGGL((many_rows4_kernel<E, D>), grid, block, 0, stream, args);
        else
            with_flags([&](auto two, auto multi, auto front, auto past) {
                constexpr int kTiles = decltype(two)::value ? 2 : 1;
                constexpr bool kMulti = decltype(multi)::value, kFront = decltype(front)::value, kPast = decltype(past)::value && sizeof(E) == 2;
                if constexpr (kTiles == 2 && kMulti) {
                    if (a.page_shift < 4) {                         // the one kernel for pages of 8 tokens
                        hipLaunchKernelGGL((few_rows4_kernel<E, D, kTiles, kMulti, kFront, true, false>), grid, block, 0, stream, args, f, (int)front_blocks);
                        return;
                    }
                }
                hipLaunchKernelGGL((few_rows4_kernel<E, D, kTiles, kMulti, kFront, false, kPast>), grid, block, 0, stream, args, f, (int)front_blocks);
            }, two_tiles, a.page_shift < 4 || max_q > 1, front_blocks > 0, past);  // max_q = 1: a sequence's rows all see the same keys
        return launched();
    });
    if (rc) return rc;
    if (!p.combine) return WHT_OK;

    JoinArgs j{};
    j.batch = a.batch; j.out = a.out; j.lse = lse; j.out_ts = a.out_ts; j.out_hs = a.out_hs;
    j.front_part = reinterpret_cast<float*>(ws + p.front_at); j.front_sums = reinterpret_cast<float*>(ws + p.front_sums_at);
    j.own_part = a.part; j.own_sums = a.sums; j.cum = a.cum;
    j.q_heads = q_heads; j.heads = a.heads; j.G = a.G; j.max_q = max_q; j.prefix = a.prefix; j.gang_log2 = a.gang_log2;
    j.front = p.front; j.front_few = p.front_few; j.front_splits = p.front_splits;
    j.own_few = p.own_few; j.own_splits = p.own_splits; j.own_cap = a.rows_cap; j.own_prefix = a.use_prefix;
    return with_type(dtype, c->head_dim, [&](auto t, auto d) {
        using E = decltype(t);
        constexpr int D = decltype(d)::value;
        const int64_t rows = T * q_heads;
        with_flags([&](auto turn, auto more) {
            constexpr bool kTurn = decltype(turn)::value;
            constexpr int kWorkersOf = decltype(more)::value && D != 128 && sizeof(E) == 2 ? kMostWorkers4 : kWorkers;
            if (!p.own_few) hipLaunchKernelGGL((join_splits_kernel<E, D, kTurn>), dim3((unsigned)ceil_div64(rows, 256 / (D / 4))), dim3(256), 0, stream, j);
            else if (join_waves(rows) == 16) hipLaunchKernelGGL((join_kernel<E, D, 16, kTurn, kWorkersOf>), dim3((unsigned)rows), dim3(1024), 0, stream, j);
            else if (join_waves(rows) == 4) hipLaunchKernelGGL((join_kernel<E, D, 4, kTurn, kWorkersOf>), dim3((unsigned)rows), dim3(256), 0, stream, j);
            else hipLaunchKernelGGL((join_kernel<E, D, 1, kTurn, kWorkersOf>), grid_of(ceil_div64(rows, 4)), dim3(256), 0, stream, j);
        }, transform != 0, workgroups > kWorkgroups);
        return launched();
    });
}

}  // namespace wht

extern "C" {

int wht_rotary_rotate(const wht_attention_rows_t* x, const wht_attention_rows_t* out, int64_t T, int32_t heads, int32_t head_dim, const float* rope,
                      int64_t rope_rows, int32_t rotary, int32_t interleaved, const int32_t* positions, int32_t axes, const uint8_t* pair_axes,
                      int32_t inverse, int32_t dtype, void* stream) {
    using namespace wht;
    if (int rc = check_rotary(x, out, T, heads, head_dim, rope, rope_rows, rotary, positions, axes, pair_axes, dtype)) return rc;
    if (T == 0) return WHT_OK;
    return rotate(x, out, T, heads, head_dim, turning(rope, rope_rows, rotary, interleaved, positions, axes, pair_axes, inverse), dtype, static_cast<hipStream_t>(stream));
}

const char* wht_rotary_status_string(int status) {
    switch (status) {
    case WHT_OK:             return "ok";
    case WHT_ERR_NULL_PTR:   return "a required pointer is NULL";
    case WHT_ERR_BAD_DIM:    return "a size is not taken: head_dim a multiple of 16 up to 256; rotary a multiple of 16 from 16 to head_dim; heads up to 1024; up to 4 axes, and every pair's among them; counts not negative and up to 2^30";
    case WHT_ERR_BAD_DTYPE:  return "dtype must be WHT_DTYPE_F32 or WHT_DTYPE_BF16";
    case WHT_ERR_MISALIGNED: return "tensors must be 16-byte aligned and their strides 16-byte steps of at least a row (heads: below 2 GiB); what is written must not overlap itself";
    case WHT_ERR_LAUNCH:     return "the HIP runtime refused a kernel launch";
    default:                 return "unknown status";
    }
}

int wht_attention_append4(const wht_attention_rows_t* q, const wht_attention_rows_t* k, const wht_attention_rows_t* v, const wht_attention_rows_t* q_out,
                          const wht_attention_rows_t* k_out, const wht_attention_rows_t* v_out, int64_t T, int32_t q_heads,
                          const wht_attention_cache4_t* cache, const wht_attention_batch_t* batch, const float* rope, int64_t rope_rows, int32_t rotary,
                          int32_t interleaved, int64_t position, const int32_t* positions, int32_t axes, const uint8_t* pair_axes, int32_t transform,
                          int32_t dtype, void* stream) {
    using namespace wht;
    if (int rc = check_append4(q, k, v, q_out, k_out, v_out, T, q_heads, cache, batch, rope, rope_rows, rotary, position, positions, axes, pair_axes, dtype)) return rc;
    if (T == 0) return WHT_OK;
    return append4(q, k, v, q_out, k_out, v_out, T, q_heads, cache, batch, turning(rope, rope_rows, rotary, interleaved, positions, axes, pair_axes, 0), position,
                   transform, dtype, static_cast<hipStream_t>(stream));
}

size_t wht_attention4_workspace_bytes(int64_t T, int32_t B, int32_t q_heads, int32_t heads, int32_t head_dim, int32_t max_q, int64_t max_length,
                                      int64_t prefix_length, int32_t dtype) {
    using namespace wht;
    if (check_sizes(T, B, q_heads, heads, head_dim, max_q, max_length, prefix_length, dtype) != WHT_OK || T == 0) return 0;
    return plan_attention4(T, B, q_heads, heads, head_dim, max_q, max_length, prefix_length).bytes;
}

int wht_attention_paged4(const wht_attention_rows_t* q, const wht_attention_rows_t* out, float* lse, int64_t T, int32_t q_heads,
                         const wht_attention_cache4_t* cache, const wht_attention_batch_t* batch, const int32_t* prefix_table, int64_t prefix_length,
                         int32_t max_q, int64_t max_length, float scale, int32_t transform, int32_t dtype, void* workspace, size_t workspace_bytes,
                         void* stream) {
    using namespace wht;
    if (int rc = check_paged4(q, out, lse, T, q_heads, cache, batch, prefix_table, prefix_length, max_q, max_length, scale, dtype)) return rc;
    if (T == 0) return WHT_OK;
    const AttentionPlan4 p = plan_attention4(T, batch->B, q_heads, cache->heads, cache->head_dim, max_q, max_length, prefix_length);
    if (p.bytes > 0 && (!workspace || workspace_bytes < p.bytes)) return WHT_ERR_WORKSPACE;
    if (((uintptr_t)workspace & 15u) != 0) return WHT_ERR_MISALIGNED;
    return paged4(q, out, lse, T, q_heads, cache, batch, prefix_table, prefix_length, max_q, max_length, scale, transform, dtype, p,
                  static_cast<unsigned char*>(workspace), static_cast<hipStream_t>(stream));
}

const char* wht_attention4_status_string(int status) {
    switch (status) {
    case WHT_OK:             return "ok";
    case WHT_ERR_NULL_PTR:   return "a required pointer is NULL";
    case WHT_ERR_BAD_DIM:    return "a size is not taken: head_dim 64, 96 or 128; page_size a power of two, 8 to 1024; q_heads a multiple of heads, at most 1024; rotary a multiple of 16 up to head_dim; up to 4 axes, and every pair's among them; counts not negative and below 2^30; strides of at least a row, a page below 4 GiB; scale > 0 and at most 2.3e38";
    case WHT_ERR_BAD_DTYPE:  return "dtype must be WHT_DTYPE_F32 or WHT_DTYPE_BF16";
    case WHT_ERR_MISALIGNED: return "tensors and codes must be 16-byte aligned and their strides 16-byte steps of at least a row (heads: below 2 GiB); what is written must not overlap itself";
    case WHT_ERR_WORKSPACE:  return "workspace is NULL or smaller than wht_attention4_workspace_bytes";
    case WHT_ERR_LAUNCH:     return "the HIP runtime refused a kernel launch";
    default:                 return "unknown status";
    }
}

}  // extern "C"
