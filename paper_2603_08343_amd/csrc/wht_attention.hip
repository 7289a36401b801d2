// Dispatch and C ABI of the paged cache and its attention (include/wht_attention.h).
#include "attention_device.h"

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

// f with a std::bool_constant for each of three flags.
template <class F>
static void with_flags(F&& f, bool a, bool b, bool c) {
    auto third = [&](auto x, auto y) { if (c) f(x, y, std::true_type{}); else f(x, y, std::false_type{}); };
    auto second = [&](auto x) { if (b) third(x, std::true_type{}); else third(x, std::false_type{}); };
    if (a) second(std::true_type{}); else second(std::false_type{});
}

static int launched() { return hipGetLastError() == hipSuccess ? WHT_OK : WHT_ERR_LAUNCH; }

// Vector pairs of a token's queries and keys from which on a workgroup takes it, not a wave.  Workgroup / wave, in us: 4 x 64 (32 pairs), 64000 tokens
// 104 / 50; 16 and 1 x 128 (136), 32000 tokens 66 / 50; 16 and 4 x 64 float32 (160), 67966 tokens 163 / 158; 16 x 128 (256), 8326 tokens 36.5 / 39.6;
// 32 and 8 x 128 (320), 16000 tokens 73 / 78.
constexpr int kWideToken = 256;

static dim3 grid_of(int64_t blocks) {
    const int64_t x = (int64_t)1 << kGridLog2;
    return blocks <= x ? dim3((unsigned)blocks) : dim3((unsigned)x, (unsigned)ceil_div64(blocks, x));
}

static int page_shift(const wht_attention_cache_t* c) { return __builtin_ctz((unsigned)c->page_size); }

static Batch batch_of(const wht_attention_batch_t* b, int64_t T, int64_t most) {
    return {b->table, b->lengths, b->q_starts, b->table_stride, b->B, (int)T, (int)most};
}

static int append(const wht_attention_rows_t* q, const wht_attention_rows_t* k, const wht_attention_rows_t* v, const wht_attention_rows_t* q_out,
                  int64_t T, int32_t q_heads, const wht_attention_cache_t* c, const wht_attention_batch_t* b, const float* rope,
                  int64_t rope_rows, int32_t rotary, int32_t interleaved, int64_t position, int32_t dtype, hipStream_t stream) {
    const int64_t size = dtype == WHT_DTYPE_F32 ? 4 : 2;
    AppendArgs a{};
    a.batch = batch_of(b, T, INT32_MAX);
    a.places = b->width * c->page_size;
    a.q = static_cast<const unsigned char*>(q->data);
    a.kn = static_cast<const unsigned char*>(k->data);
    a.vn = static_cast<const unsigned char*>(v->data);
    a.q_out = static_cast<unsigned char*>(q_out->data);
    a.k = static_cast<unsigned char*>(c->k);
    a.v = static_cast<unsigned char*>(c->v);
    a.q_ts = q->token_stride * size; a.q_hs = q->head_stride * size;
    a.k_ts = k->token_stride * size; a.k_hs = k->head_stride * size;
    a.v_ts = v->token_stride * size; a.v_hs = v->head_stride * size;
    a.qo_ts = q_out->token_stride * size; a.qo_hs = q_out->head_stride * size;
    a.page_stride = c->page_stride * size; a.head_stride = c->head_stride * size; a.token_stride = c->token_stride * size;
    a.rope = rope; a.rope_rows = rope_rows; a.rotary = rotary; a.interleaved = interleaved != 0; a.position = (int)position;
    a.q_heads = q_heads; a.heads = c->heads; a.pages = c->pages; a.page_shift = page_shift(c);
    return with_type(dtype, c->head_dim, [&](auto t, auto d) {
        using E = decltype(t);
        constexpr int D = decltype(d)::value;
        const int pairs = (int)((a.q ? q_heads : 0) + c->heads) * (int)(D * sizeof(E) / 32);
        if (pairs < kWideToken) hipLaunchKernelGGL((append_kernel<E, D, 64>), grid_of(ceil_div64(T, 4)), dim3(256), 0, stream, a);
        else hipLaunchKernelGGL((append_kernel<E, D, 256>), grid_of(T), dim3(256), 0, stream, a);
        return launched();
    });
}

static int paged(const wht_attention_rows_t* q, const wht_attention_rows_t* out, float* lse, int64_t T, int32_t q_heads,
                 const wht_attention_cache_t* c, const wht_attention_batch_t* b, const int32_t* prefix_table, int64_t prefix, int32_t max_q,
                 int64_t max_length, float scale, int32_t dtype, const AttentionPlan& p, unsigned char* ws, hipStream_t stream) {
    const int64_t size = dtype == WHT_DTYPE_F32 ? 4 : 2;
    const int64_t table_keys = (int64_t)b->width * c->page_size;
    AttentionArgs a{};
    a.batch = batch_of(b, T, table_keys < max_length ? table_keys : max_length);
    a.q = static_cast<const unsigned char*>(q->data);
    a.k = static_cast<const unsigned char*>(c->k);
    a.v = static_cast<const unsigned char*>(c->v);
    a.out = static_cast<unsigned char*>(out->data);
    a.lse = lse;
    a.q_ts = q->token_stride * size; a.q_hs = q->head_stride * size;
    a.out_ts = out->token_stride * size; a.out_hs = out->head_stride * size;
    a.head_stride = c->head_stride * size;
    a.page_stride = (unsigned)(c->page_stride * size); a.token_stride = (unsigned)(c->token_stride * size);
    a.prefix_table = prefix_table;
    a.q_heads = q_heads; a.heads = c->heads; a.G = q_heads / c->heads; a.pages = c->pages; a.page_shift = page_shift(c);
    a.prefix = (int)prefix; a.max_q = max_q;
    a.scale = base2_scale(scale);
    AttentionArgs f = a;
    int64_t front_blocks = 0;
    if (p.front && !p.front_few) {
        f.use_prefix = 1; f.splits = p.front_splits;
        f.part = reinterpret_cast<float*>(ws + p.front_at); f.sums = reinterpret_cast<float*>(ws + p.front_sums_at);
        front_blocks = kDies * die_blocks(T, 1, a.G, T, (int64_t)c->heads * f.splits);
    }
    a.use_prefix = !p.front && prefix > 0;
    a.front_item = p.front && p.front_few;
    a.gang_log2 = gang_log2_of(c->heads, c->head_dim * size, a.head_stride);
    const bool stream_keys = streams(b->B, c->heads, c->head_dim, size, a.batch.most, a.use_prefix ? prefix : 0, a.gang_log2);
    a.splits = p.own_splits; a.rows_cap = p.own_cap;
    a.part = reinterpret_cast<float*>(ws + p.own_at); a.sums = reinterpret_cast<float*>(ws + p.own_sums_at);
    a.cum = reinterpret_cast<int*>(ws + p.cum_at);
    const int64_t each = die_blocks(T, b->B, a.G, max_q, (int64_t)c->heads * a.splits), own_blocks = p.own_few ? kWorkgroups : (each + 1) * kDies;
    if (front_blocks + own_blocks > kMostWorkgroups) return WHT_ERR_BAD_DIM;
    a.fill = (int)each;
    const int rc = with_type(dtype, c->head_dim, [&](auto t, auto d) {
        using E = decltype(t);
        constexpr int D = decltype(d)::value;
        const dim3 grid((unsigned)(front_blocks + own_blocks)), block(256);
        if (!p.own_few) hipLaunchKernelGGL((many_rows_kernel<E, D>), grid, block, 0, stream, a);
        else
            with_flags([&](auto multi, auto front, auto past) {
                hipLaunchKernelGGL((few_rows_kernel<E, D, decltype(multi)::value, decltype(front)::value, decltype(past)::value>), grid, block, 0, stream, a, f, (int)front_blocks);
            }, max_q > 1, front_blocks > 0, stream_keys);           // max_q = 1: a sequence's rows all see the same keys
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
        const int64_t rows = T * q_heads;
        if (!p.own_few) hipLaunchKernelGGL((join_splits_kernel<decltype(t), decltype(d)::value>), dim3((unsigned)ceil_div64(rows, 256 / (decltype(d)::value / 4))), dim3(256), 0, stream, j);
        else if (join_waves(rows) == 16) hipLaunchKernelGGL((join_kernel<decltype(t), decltype(d)::value, 16>), dim3((unsigned)rows), dim3(1024), 0, stream, j);
        else if (join_waves(rows) == 4) hipLaunchKernelGGL((join_kernel<decltype(t), decltype(d)::value, 4>), dim3((unsigned)rows), dim3(256), 0, stream, j);
        else hipLaunchKernelGGL((join_kernel<decltype(t), decltype(d)::value, 1>), grid_of(ceil_div64(rows, 4)), dim3(256), 0, stream, j);
        return launched();
    });
}

}  // namespace wht

extern "C" {

int wht_attention_append(const wht_attention_rows_t* q, const wht_attention_rows_t* k, const wht_attention_rows_t* v,
                         const wht_attention_rows_t* q_out, int64_t T, int32_t q_heads, const wht_attention_cache_t* cache,
                         const wht_attention_batch_t* batch, const float* rope, int64_t rope_rows, int32_t rotary, int32_t interleaved,
                         int64_t position, int32_t dtype, void* stream) {
    using namespace wht;
    if (int rc = check_append(q, k, v, q_out, T, q_heads, cache, batch, rope, rope_rows, rotary, position, dtype)) return rc;
    if (T == 0) return WHT_OK;
    return append(q, k, v, q_out, T, q_heads, cache, batch, rope, rope_rows, rotary, interleaved, position, dtype, static_cast<hipStream_t>(stream));
}

size_t wht_attention_workspace_bytes(int64_t T, int32_t B, int32_t q_heads, int32_t heads, int32_t head_dim, int32_t max_q,
                                     int64_t max_length, int64_t prefix_length, int32_t dtype) {
    using namespace wht;
    if (check_sizes(T, B, q_heads, heads, head_dim, max_q, max_length, prefix_length, dtype) != WHT_OK || T == 0) return 0;
    return plan_attention(T, B, q_heads, heads, head_dim, max_q, max_length, prefix_length).bytes;
}

int wht_attention_paged(const wht_attention_rows_t* q, const wht_attention_rows_t* out, float* lse, int64_t T, int32_t q_heads,
                        const wht_attention_cache_t* cache, const wht_attention_batch_t* batch, const int32_t* prefix_table,
                        int64_t prefix_length, int32_t max_q, int64_t max_length, float scale, int32_t dtype, void* workspace,
                        size_t workspace_bytes, void* stream) {
    using namespace wht;
    if (int rc = check_paged(q, out, lse, T, q_heads, cache, batch, prefix_table, prefix_length, max_q, max_length, scale, dtype)) return rc;
    if (T == 0) return WHT_OK;
    const AttentionPlan p = plan_attention(T, batch->B, q_heads, cache->heads, cache->head_dim, max_q, max_length, prefix_length);
    if (p.bytes > 0 && (!workspace || workspace_bytes < p.bytes)) return WHT_ERR_WORKSPACE;
    if (((uintptr_t)workspace & 15u) != 0) return WHT_ERR_MISALIGNED;
    return paged(q, out, lse, T, q_heads, cache, batch, prefix_table, prefix_length, max_q, max_length, scale, dtype, p,
                 static_cast<unsigned char*>(workspace), static_cast<hipStream_t>(stream));
}

const char* wht_attention_status_string(int status) {
    switch (status) {
    case WHT_OK:             return "ok";
    case WHT_ERR_NULL_PTR:   return "a required pointer is NULL";
    case WHT_ERR_BAD_DIM:    return "a size is not taken: head_dim 64, 96 or 128; page_size a power of two, 8 to 1024; q_heads a multiple of heads, at most 1024; rotary a multiple of 16 up to head_dim; counts not negative and below 2^30; a page below 4 GiB; scale > 0 and at most 2.3e38";
    case WHT_ERR_BAD_DTYPE:  return "dtype must be WHT_DTYPE_F32 or WHT_DTYPE_BF16";
    case WHT_ERR_MISALIGNED: return "tensors must be 16-byte aligned and their strides 16-byte steps of at least a row (heads: below 2 GiB); what is written must not overlap itself";
    case WHT_ERR_WORKSPACE:  return "workspace is NULL or smaller than wht_attention_workspace_bytes";
    case WHT_ERR_LAUNCH:     return "the HIP runtime refused a kernel launch";
    default:                 return "unknown status";
    }
}

}  // extern "C"
