// Attention over the cache in 4 bits (include/wht_attention4.h) for gfx950.
//
// A code times its scale has three significant bits, which bfloat16 holds exactly: keys and values become bfloat16 on their way to the matrix
// cores, one instruction for two of them, scale included, and the products are those of attention_device.h.  Float32 queries and weights enter the same
// products as the sum of three bfloat16 terms (24 bits), three products each, where products in float32 would take sixteen times the cycles.  The weights of bfloat16
// queries are rounded to bfloat16, as with the 16-bit cache: a second term would double the products with the values.  Their sum is not rounded.  Results of 65001 keys are
// off by 0.0017 of their norm then, of prompts and behind a long prefix by 0.0022, where the rounding of the results alone is 0.0016 to 0.0017.
#pragma once
#include "append4_device.h"

namespace wht {

struct Attention4Args {
    AttentionArgs base;                                             // page_stride, head_stride, token_stride: of codes
    const unsigned char *ks, *vs;
    int64_t s_head_stride;
    unsigned s_page_stride, s_token_stride;
    int transform;
};

template <class T> constexpr int kTerms = sizeof(T) == 4 ? 3 : 1;

// x as a sum of bfloat16 terms.
template <int TERMS>
__device__ __forceinline__ void split(float x, bf16 (&t)[TERMS]) {
#pragma unroll
    for (int i = 0; i < TERMS; ++i) {
        t[i] = (bf16)x;
        x -= (float)t[i];
    }
}
// Eight elements of a row, as terms; zeros where there is no row.
template <class T, int TERMS>
__device__ __forceinline__ void load_terms(const unsigned char* p, bool there, bf16x8 (&q)[TERMS]) {
    if constexpr (TERMS == 1) q[0] = __builtin_bit_cast(bf16x8, there ? *reinterpret_cast<const u32x4*>(p) : u32x4{0, 0, 0, 0});
    else {
        float x[8] = {};
        if (there) load8<T>(x, p);
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            // an infinity or NaN is its first term, a finite number's is finite: what bfloat16's largest leaves of it is the second's
            const bool finite = fabsf(x[i]) < __builtin_inff();
            const float most = __uint_as_float(0x7f7f0000u);
            bf16 t[TERMS];
            t[0] = (bf16)(finite ? fminf(fmaxf(x[i], -most), most) : x[i]);
            float rest = finite ? x[i] - (float)t[0] : 0.0f;
#pragma unroll
            for (int k = 1; k < TERMS; ++k) {
                t[k] = (bf16)rest;
                rest -= (float)t[k];
            }
#pragma unroll
            for (int k = 0; k < TERMS; ++k) q[k][i] = t[k];
        }
    }
}

// ------------------------------------------------------------------------------------------------
// Few rows (decoding).  As in attention_device.h every wave works by itself on its share of the line of 32-key blocks, without a barrier.  Rows are the
// columns of 16 x 16 products, TILES times 16 of them:
//
//     S^T = K Q^T     a lane holds a quarter of key lane % 16's elements, as it loaded them: keys go from memory to the product in registers
//     O^T += V^T P^T  values pass LDS, where transposing reads turn a lane's row into columns
//
// A lane's scores are of row lane % 16, keys 4 (lane / 16) + i of either half of the block, and its weights the second product's operand as they stand.

template <class T, int D, int TILES>
struct Few4 {
    static constexpr int kElements = D / 4;                         // of a row, that a lane holds
    static constexpr int kWords = kElements / 8;                    // of codes
    static constexpr int kScales = D == 96 ? 2 : 1;                 // blocks that a lane's elements are of
    static constexpr int kBlocks = D / 16, kTermsOf = kTerms<T>;
    using L = Head<bf16, D>;
    static constexpr int kWaveBytes = 32 * L::kRowBytes;
    static constexpr int kAhead = 2;                                // blocks whose codes are in registers or on their way

    // Where 16-byte chunk `chunk` of row `row` of the values stands in its row in LDS.  A write takes eight rows' chunks at a time, which have to fill 128
    // bytes, a transposing read 32 bytes of eight rows, which have to fill 256: no bank conflicts.
    static __device__ __forceinline__ int place(int row, int chunk) {
        if constexpr (D == 128) return chunk ^ ((row & 3) << 1 | ((row >> 2) & 1) * 9);
        else if constexpr (D == 64) return chunk ^ (row & 7);
        else return chunk ^ (((row >> 2) & 1) << 1 | ((row >> 1) & 1));
    }

    // Codes and scale bytes of a lane's part of two keys or values.
    struct Part { unsigned code[2][kWords]; unsigned scale[2][kScales]; };
    struct State {
        float top, most, base, l;                                   // as RowState's
        f32x4 o[kBlocks];
    };
    struct Odd { int first[D / 8]; };                               // by eight elements: the first key whose value is not a number

    static __device__ __forceinline__ int scale_index(int i) { return ((int)(threadIdx.x >> 4 & 3) * kElements + i * 8) / 32; }

    // A word of codes; PAST: read once, not kept in the caches.
    template <class V, bool PAST>
    static __device__ __forceinline__ V words(const unsigned char* from) {
        if constexpr (PAST) return __builtin_nontemporal_load(reinterpret_cast<const V*>(from));
        else return *reinterpret_cast<const V*>(from);
    }
    // Of key or value k of the two: `codes` and `scales` on from places that all lanes share, by what is the lane's own.
    template <bool PAST>
    static __device__ __forceinline__ void load(Part& p, int k, const unsigned char* codes, const unsigned char* scales, unsigned code_off, unsigned scale_off) {
        const unsigned char* from = codes + code_off;
        if constexpr (D == 128) {
            const u32x4 x = words<u32x4, PAST>(from);
#pragma unroll
            for (int i = 0; i < 4; ++i) p.code[k][i] = x[i];
        } else {
#pragma unroll
            for (int i = 0; i < kWords; ++i) p.code[k][i] = words<unsigned, PAST>(from + i * 4);
        }
        p.scale[k][0] = scales[scale_off];
        if constexpr (kScales == 2) p.scale[k][1] = scales[scale_off + (unsigned)(scale_index(kWords - 1) - scale_index(0))];
    }
    static __device__ __forceinline__ float scale_at(const unsigned (&scale)[kScales], int i) {
        if constexpr (kScales == 1) return scale_of(scale[0]);
        else return scale_of(scale_index(i) == scale_index(0) ? scale[0] : scale[1]);
    }

    // Rows' maxima over the four lanes that hold a row.
    static __device__ __forceinline__ float over_lanes(float x) {
        unsigned u = __float_as_uint(x);
        auto both = __builtin_amdgcn_permlane32_swap(u, u, false, false);
        u = __float_as_uint(fmaxf(__uint_as_float(both[0]), __uint_as_float(both[1])));
        both = __builtin_amdgcn_permlane16_swap(u, u, false, false);
        return fmaxf(__uint_as_float(both[0]), __uint_as_float(both[1]));
    }

    // As rebase() of attention_device.h without slack, for a tile of 16 rows; the factor is that between the bases as they were used.
    static __device__ __forceinline__ void rebase(float scale, f32x4 (&s)[2], State& st) {
        float mx = WHT_NEG_INF;
#pragma unroll
        for (int k = 0; k < 2; ++k)
#pragma unroll
            for (int i = 0; i < 4; ++i) mx = fmaxf(mx, s[k][i]);
        mx = over_lanes(mx);
        if (__any(mx > st.most)) {
            const bool was_far = st.most != st.top;
            const float now = fmaxf(st.top, mx), m = now == WHT_NEG_INF ? 0.0f : now * scale;
            const bool far = fabsf(m) >= kFar;
            const float to = far ? (was_far ? (st.top - now) * scale : __builtin_fmaf(-now, scale, st.base)) : was_far ? __builtin_fmaf(st.top, scale, -m) : st.base - m;
            const float f = st.top == WHT_NEG_INF ? 0.0f : __builtin_amdgcn_exp2f(to);
            st.l *= f;
#pragma unroll
            for (int d = 0; d < kBlocks; ++d) st.o[d] *= f;
            st.top = now;
            st.base = far ? 0.0f : m;
            st.most = far ? WHT_NEG_INF : now;
            if (__any(far)) {
                const float off = far ? now : 0.0f;
#pragma unroll
                for (int k = 0; k < 2; ++k) s[k] -= off;
            }
        }
    }

    // 8 keys by 16 columns of the values in LDS, transposed, from column 16 d on.
    static __device__ __forceinline__ bf16x8 values(unsigned buf, int d) {
        const int lane = threadIdx.x & 63, g = lane >> 4, in = lane & 15, row = g * 4 + (in >> 2), c = d * 2 + ((in & 3) >> 1);
        const unsigned at = buf + row * L::kRowBytes + place(row, c) * 16 + (in & 1) * 8;
        bf16x8 v;
#pragma unroll
        for (int e = 0; e < 2; ++e) {
            const short4v x = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) short4v*)(uintptr_t)(at + e * 16 * L::kRowBytes));
            const bf16x4 y = __builtin_bit_cast(bf16x4, x);
#pragma unroll
            for (int i = 0; i < 4; ++i) v[e * 4 + i] = y[i];
        }
        return v;
    }

    // Blocks [n0, n1) of `table`'s tokens, of which there are `keys`; limit: how many of them this lane's rows see, all_see: how many every row sees.
    // Codes of two blocks are on their way while a third is worked on.
    // NARROW: pages of 8 tokens; STREAM: codes are read past the caches.
    template <bool MULTI, bool NARROW, bool STREAM>
    static __device__ __forceinline__ void run(const Attention4Args& args, const int* table, int n0, int n1, int keys, const int (&limit)[TILES], int all_see,
                                               int head, unsigned buf, const bf16x8 (&q)[TILES][kTermsOf][kWords], Odd& odd, State (&st)[TILES]) {
        const AttentionArgs& a = args.base;
        const int lane = threadIdx.x & 63, c = lane & 15, g = lane >> 4, shift = a.page_shift;
        const unsigned char *kc = a.k + head * a.head_stride, *vc = a.v + head * a.head_stride, *ks = args.ks + head * args.s_head_stride, *vs = args.vs + head * args.s_head_stride;
        const unsigned slot0 = NARROW ? c & 7 : c, code_off = slot0 * a.token_stride + g * (kElements / 2), scale_off = slot0 * args.s_token_stride + scale_index(0);
        const int last = min(n1 * kBlockKeys, keys);
        int key0 = n0 * kBlockKeys;
        while (key0 < last) {
            // 64 pages at a time, one per lane
            const int first = key0 >> shift, end = min((int64_t)last, (int64_t)(first + 64) << shift);
            int page = -1;
            const bool listed = ((int64_t)(first + lane) << shift) < end;
            if (listed) page = table[first + lane];
            if (page >= a.pages) page = -1;
            const bool bad = __any(listed && page < 0);
            const int named = max(page, 0);                         // keys that are not there are read from a page that is, and not used
            // of 16 (pages of 8 tokens: 8) keys the page, and where its rows are, are the same for all lanes
            auto row_of = [&](int key, uint64_t& codes, uint64_t& scales) {
                const unsigned at = __builtin_amdgcn_readlane(named, min((key >> shift) - first, 63)), slot = key & ((1 << shift) - 1);
                codes = (uint64_t)at * a.page_stride + slot * a.token_stride;
                scales = (uint64_t)at * args.s_page_stride + slot * args.s_token_stride;
            };
            auto fetch = [&](int from, Part& k, Part& v) {
                uint64_t codes[2], scales[2];
                row_of(from, codes[0], scales[0]);
                row_of(from + 16, codes[1], scales[1]);
                if constexpr (!NARROW) {
#pragma unroll
                    for (int i = 0; i < 2; ++i) {
                        load<STREAM>(k, i, kc + codes[i], ks + scales[i], code_off, scale_off);
                        load<STREAM>(v, i, vc + codes[i], vs + scales[i], code_off, scale_off);
                    }
                } else {
#pragma unroll
                    for (int i = 0; i < 2; ++i) {
                        uint64_t more_codes, more_scales;
                        row_of(from + 16 * i + 8, more_codes, more_scales);
                        const uint64_t at = c < 8 ? codes[i] : more_codes, scale = c < 8 ? scales[i] : more_scales;
                        load<STREAM>(k, i, kc + at, ks + scale, code_off, scale_off);
                        load<STREAM>(v, i, vc + at, vs + scale, code_off, scale_off);
                    }
                }
            };
            auto there = [&](int key) {                             // by all lanes
                const int at = __shfl(page, min((key >> shift) - first, 63));
                return key < end && at >= 0;
            };

            // 32 keys from `from` on; what is two blocks further on is fetched as soon as this one's codes are used
            auto block = [&](int from, Part& kp, Part& vp) {
                f32x4 s[TILES][2];
#pragma unroll
                for (int n = 0; n < TILES; ++n)
#pragma unroll
                    for (int k = 0; k < 2; ++k) s[n][k] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
                for (int k = 0; k < 2; ++k)
#pragma unroll
                    for (int i = 0; i < kWords; ++i) {
                        const bf16x8 x = decode(kp.code[k][i], scale_at(kp.scale[k], i));
#pragma unroll
                        for (int n = 0; n < TILES; ++n)
#pragma unroll
                            for (int e = kTermsOf - 1; e >= 0; --e) s[n][k] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(x, q[n][e][i], s[n][k], 0, 0, 0);
                    }
                const int next = from + kBlockKeys;
                if (bad || next > end) {                            // values of keys that are not there: zeros
#pragma unroll
                    for (int k = 0; k < 2; ++k) {
                        const bool known = there(from + 16 * k + c);
#pragma unroll
                        for (int i = 0; i < kWords; ++i) vp.code[k][i] = known ? vp.code[k][i] : 0;
#pragma unroll
                        for (int i = 0; i < kScales; ++i) vp.scale[k][i] = known ? vp.scale[k][i] : 127;
                    }
                }
                // A value that is not a number is in all 32 of its block; a key that a row does not see has a weight of zero, and zero times NaN is NaN: where
                // rows see different keys such blocks stay out of the product, and rows that see one get it by itself.
                bool any_odd = false;
                if constexpr (MULTI) {
                    if (all_see < min(next, keys)) {
                        bool mine = false;
#pragma unroll
                        for (int k = 0; k < 2; ++k)
#pragma unroll
                            for (int i = 0; i < kScales; ++i) mine |= vp.scale[k][i] >= 253;
                        any_odd = __any(mine);
                        if (any_odd) {
                            if (lane < D / 8) odd.first[lane] = INT_MAX;
                            reads_done();
#pragma unroll
                            for (int k = 0; k < 2; ++k) {
#pragma unroll
                                for (int i = 0; i < kWords; ++i)
                                    if (!(fabsf(scale_at(vp.scale[k], i)) < __builtin_inff())) {
                                        atomicMin(&odd.first[g * kWords + i], from + 16 * k + c);
                                        vp.code[k][i] = 0;
                                    }
#pragma unroll
                                for (int i = 0; i < kScales; ++i)
                                    if (vp.scale[k][i] >= 253) vp.scale[k][i] = 127;
                            }
                            reads_done();
                        }
                    }
                }
                // a wave's reads and writes of LDS happen in their order: no waits
#pragma unroll
                for (int k = 0; k < 2; ++k)
#pragma unroll
                    for (int i = 0; i < kWords; ++i) {
                        const int row = 16 * k + c;
                        *(__attribute__((address_space(3))) u32x4*)(uintptr_t)(buf + row * L::kRowBytes + place(row, g * kWords + i) * 16) =
                            __builtin_bit_cast(u32x4, decode(vp.code[k][i], scale_at(vp.scale[k], i)));
                    }
                if (from + kAhead * kBlockKeys < end) fetch(from + kAhead * kBlockKeys, kp, vp);

                bf16x8 w[TILES][kTermsOf];
#pragma unroll
                for (int n = 0; n < TILES; ++n) {
                    if (bad) {
#pragma unroll
                        for (int k = 0; k < 2; ++k)
#pragma unroll
                            for (int i = 0; i < 4; ++i) s[n][k][i] = there(from + 16 * k + 4 * g + i) ? s[n][k][i] : WHT_NEG_INF;
                    }
                    if (next > all_see) {
#pragma unroll
                        for (int k = 0; k < 2; ++k)
#pragma unroll
                            for (int i = 0; i < 4; ++i) s[n][k][i] = from + 16 * k + 4 * g + i < limit[n] ? s[n][k][i] : WHT_NEG_INF;
                    }
                    rebase(a.scale, s[n], st[n]);
                    float sum = 0.0f;
#pragma unroll
                    for (int k = 0; k < 2; ++k)
#pragma unroll
                        for (int i = 0; i < 4; ++i) {
                            const float p = __builtin_amdgcn_exp2f(__builtin_fmaf(s[n][k][i], a.scale, -st[n].base));
                            sum += p;
                            bf16 t[kTermsOf];
                            split<kTermsOf>(p, t);
#pragma unroll
                            for (int e = 0; e < kTermsOf; ++e) w[n][e][k * 4 + i] = t[e];
                        }
                    st[n].l += sum;
                }
                asm volatile("" ::: "memory");
#pragma unroll
                for (int d = 0; d < kBlocks; ++d) {
                    const bf16x8 v = values(buf, d);
#pragma unroll
                    for (int n = 0; n < TILES; ++n)
#pragma unroll
                        for (int e = kTermsOf - 1; e >= 0; --e) st[n].o[d] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(v, w[n][e], st[n].o[d], 0, 0, 0);
                }
                if (MULTI && any_odd) {
#pragma unroll
                    for (int d = 0; d < kBlocks; ++d) {
                        const int seen = odd.first[d * 2 + (g >> 1)];
#pragma unroll
                        for (int n = 0; n < TILES; ++n)
                            if (seen < limit[n]) st[n].o[d] += __builtin_nanf("");
                    }
                    reads_done();
                }
                asm volatile("" ::: "memory");
            };

            Part k[kAhead], v[kAhead];
#pragma unroll
            for (int i = 0; i < kAhead; ++i)
                if (i == 0 || key0 + i * kBlockKeys < end) fetch(key0 + i * kBlockKeys, k[i], v[i]);
            while (key0 < end) {
#pragma unroll
                for (int i = 0; i < kAhead; ++i) {
                    if (key0 >= end) break;
                    block(key0, k[i], v[i]);
                    key0 += kBlockKeys;
                }
            }
        }
    }
    // Queries, what they see, and empty sums of the rows of a sequence and a key head.
    static __device__ __forceinline__ void begin(const AttentionArgs& a, const Sequence& s, int head, int rows, bf16x8 (&q)[TILES][kTermsOf][kWords], int (&limit)[TILES],
                                                 int (&whole)[TILES], State (&st)[TILES]) {
        const int c = threadIdx.x & 15, g = threadIdx.x >> 4 & 3;
#pragma unroll
        for (int i = 0; i < TILES; ++i) {
            const int row = i * kSmallTile + c, token = row / a.G, qh = head * a.G + row % a.G;
            limit[i] = min(max(s.length - s.queries + token + 1, 0), s.length);
            whole[i] = a.prefix;
            const unsigned char* at = a.q + (s.first + token) * a.q_ts + qh * a.q_hs + g * kElements * sizeof(T);
#pragma unroll
            for (int e = 0; e < kWords; ++e) {
                bf16x8 x[kTermsOf];
                load_terms<T, kTermsOf>(at + e * 8 * sizeof(T), row < rows, x);
#pragma unroll
                for (int k = 0; k < kTermsOf; ++k) q[i][k][e] = x[k];
            }
            st[i].top = st[i].most = WHT_NEG_INF;
            st[i].base = st[i].l = 0.0f;
#pragma unroll
            for (int d = 0; d < kBlocks; ++d) st[i].o[d] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
        }
    }
};

template <class T, int D, int TILES>
struct FewShared {
    __align__(16) unsigned char buf[4 * Few4<T, D, TILES>::kWaveBytes];
    typename Few4<T, D, TILES>::Odd odd[4];
};

// The line is that of few_rows() in attention_device.h.  FRONT: the prefix is the launch's other workgroups' work.
template <class T, int D, int TILES, bool MULTI, bool FRONT, bool NARROW, bool STREAM>
__device__ __forceinline__ void few_rows4(const Attention4Args& args, int block, FewShared<T, D, TILES>& shared) {
    using F = Few4<T, D, TILES>;
    const AttentionArgs& a = args.base;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), c = lane & 15, g = lane >> 4;
    const int B = a.batch.B + a.front_item;

    // each lane's run of sequences and the runs' prefix sums
    const int run = max(ceil_div(B, 64), 1), b0 = min(B, lane * run), b1 = min(B, b0 + run);
    Sequence held{0, 0, 0};
    int mine = 0;
    for (int b = b0; b < b1; ++b) {
        held = line_sequence(a, b);
        mine += line_blocks(a, b, held);
    }
    int upto = mine;
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
        const int x = __shfl_up(upto, o);
        if (lane >= o) upto += x;
    }
    const int all = __builtin_amdgcn_readlane(upto, 63), groups = a.heads >> a.gang_log2, worker = a.gang_log2 == 0 ? block * 4 + wave : block;
    if (block == 0 && wave == 0) {
        int n = upto - mine;
        for (int b = b0; b < b1; ++b) { a.cum[b] = n; n += line_blocks(a, b, line_sequence(a, b)); }
        if (lane == 0) a.cum[B] = all;
    }
    const int total = all * groups, per = line_share<4 * workgroups4(sizeof(T) == 4, D, TILES, FRONT)>(total, a.rows_cap, a.gang_log2);
    int u = min((int64_t)total, (int64_t)worker * per);
    const int end = min(total, u + per);
    if (u >= end) return;
    const int from = __popcll(__ballot(upto * groups <= u));       // the lane whose run has block u
    int b = from * run, cum = __builtin_amdgcn_readlane(upto - mine, from);
    const unsigned buf = __builtin_amdgcn_readfirstlane(lds_address(shared.buf)) + wave * F::kWaveBytes;

    while (u < end) {
        Sequence s;
        if (run == 1) s = {__builtin_amdgcn_readlane(held.first, b), __builtin_amdgcn_readlane(held.queries, b), __builtin_amdgcn_readlane(held.length, b)};
        else s = line_sequence(a, b);
        const int n = line_blocks(a, b, s);
        if (u >= (cum + n) * groups) { cum += n; ++b; continue; }
        const int within = u - cum * groups, group = within / n, n0 = within - group * n, n1 = min(n, n0 + (end - u));
        const int in_gang = a.gang_log2 == 0 ? 0 : wave, head = (group << a.gang_log2) + in_gang;
        const bool stacked = b >= a.batch.B;
        const int rows = min(s.queries * a.G, a.rows_cap);
        const int front = a.use_prefix || stacked ? ceil_div(a.prefix, kBlockKeys) : 0;
        const int all_see = min(max(s.length - s.queries + 1, 0), s.length);
        const int keys = min(max(s.length - s.queries + min(s.queries, a.max_q), 0), s.length);           // what the last of the rows sees
        bf16x8 q[TILES][F::kTermsOf][F::kWords];
        typename F::State st[TILES];
        int limit[TILES], whole[TILES];
        F::begin(a, s, head, rows, q, limit, whole, st);
#pragma unroll 1
        for (int part = FRONT ? 1 : 0; part < 2; ++part) {          // the prefix, the sequence
            const int lo = part ? max(n0 - front, 0) : n0, hi = part ? n1 - front : min(n1, front);
            if (lo >= hi) continue;
            const int* table = part ? a.batch.table + b * a.batch.table_stride : a.prefix_table;
            F::template run<MULTI, NARROW, STREAM>(args, table, lo, hi, part ? keys : a.prefix, part ? limit : whole, part ? all_see : a.prefix, head, buf, q, shared.odd[wave], st);
        }
#pragma unroll
        for (int i = 0; i < TILES; ++i) {
            st[i].l += __shfl_xor(st[i].l, 16);
            st[i].l += __shfl_xor(st[i].l, 32);
            const int row = i * kSmallTile + c;
            if (row >= rows) continue;
            const int64_t at = (((int64_t)(b * groups + group + worker) << a.gang_log2) + in_gang) * a.rows_cap + row;
            if (g == 0) *reinterpret_cast<f32x2*>(a.sums + at * 2) = f32x2{st[i].top * a.scale, st[i].l};
#pragma unroll
            for (int d = 0; d < F::kBlocks; ++d) *reinterpret_cast<f32x4*>(a.part + at * D + d * 16 + g * 4) = st[i].o[d];
        }
        u += n1 - n0;
    }
}

// ------------------------------------------------------------------------------------------------
// A sequence's rows of a key head whole, by a workgroup, whose waves join their shares in LDS: one launch where the line and its join are two, for calls so
// small that those are most of their time.  The waves of the line would be no more, or hardly.

template <class T, int TILES> constexpr int kWholeWaves = sizeof(T) == 4 && TILES == 2 ? 4 : 8;

template <class T, int D, int TILES>
struct WholeShared {
    static constexpr int kRows = TILES * kSmallTile, kWaves = kWholeWaves<T, TILES>;
    union {
        __align__(256) unsigned char buf[kWaves * Few4<T, D, TILES>::kWaveBytes];
        float o[kWaves][kRows][D];
    };
    typename Few4<T, D, TILES>::Odd odd[kWaves];
    float top[kWaves][kRows], l[kWaves][kRows];
};

template <class T, int D, int TILES, bool MULTI, bool NARROW>
__global__ __launch_bounds__((64 * kWholeWaves<T, TILES>)) void whole_rows4_kernel(Attention4Args args) {
    using F = Few4<T, D, TILES>;
    using S = WholeShared<T, D, TILES>;
    __shared__ S shared;
    const AttentionArgs& a = args.base;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), c = lane & 15, g = lane >> 4;
    const int b = blockIdx.x / a.heads, head = blockIdx.x - b * a.heads;
    if ((a.batch.q_starts || a.batch.T > a.batch.B) && threadIdx.x < 256)         // rows of no sequence, and past max_q
        for (int die = blockIdx.x; die < kDies; die += gridDim.x) fill_rows<T, D>(a, die);
    const Sequence s = sequence(a.batch, b);
    if (s.queries == 0) return;
    const int rows = min(min(s.queries, a.max_q) * a.G, S::kRows);
    const int front = a.use_prefix ? ceil_div(a.prefix, kBlockKeys) : 0;
    const int all_see = min(max(s.length - s.queries + 1, 0), s.length);
    const int keys = min(max(s.length - s.queries + min(s.queries, a.max_q), 0), s.length);
    const int n = front + ceil_div(keys, kBlockKeys), per = ceil_div(n, S::kWaves), n0 = min(n, wave * per), n1 = min(n, n0 + per);
    bf16x8 q[TILES][F::kTermsOf][F::kWords];
    typename F::State st[TILES];
    int limit[TILES], whole[TILES];
    F::begin(a, s, head, rows, q, limit, whole, st);
    const unsigned buf = __builtin_amdgcn_readfirstlane(lds_address(shared.buf)) + wave * F::kWaveBytes;
#pragma unroll 1
    for (int part = 0; part < 2; ++part) {                          // the prefix, the sequence
        const int lo = part ? max(n0 - front, 0) : n0, hi = part ? n1 - front : min(n1, front);
        if (lo >= hi) continue;
        const int* table = part ? a.batch.table + b * a.batch.table_stride : a.prefix_table;
        F::template run<MULTI, NARROW, false>(args, table, lo, hi, part ? keys : a.prefix, part ? limit : whole, part ? all_see : a.prefix, head, buf, q, shared.odd[wave], st);
    }
    workgroup_barrier();                                            // the shares lie where values did
#pragma unroll
    for (int i = 0; i < TILES; ++i) {
        const int row = i * kSmallTile + c;
        st[i].l += __shfl_xor(st[i].l, 16);
        st[i].l += __shfl_xor(st[i].l, 32);
        if (g == 0) { shared.top[wave][row] = st[i].top * a.scale; shared.l[wave][row] = st[i].l; }
#pragma unroll
        for (int d = 0; d < F::kBlocks; ++d) *reinterpret_cast<f32x4*>(&shared.o[wave][row][d * 16 + g * 4]) = st[i].o[d];
    }
    __syncthreads();
    // four outputs to a thread; a wave's rows are whole, and so are the eight threads of 32 outputs
    constexpr int kLanes = D / 4, kRowsOfWave = 64 / kLanes;
    for (int row0 = wave * kRowsOfWave; row0 < rows; row0 += S::kWaves * kRowsOfWave) {
        const int row = min(row0 + lane / kLanes, S::kRows - 1), col = lane % kLanes * 4;
        float m = WHT_NEG_INF, l = 0.0f;
#pragma unroll
        for (int w = 0; w < S::kWaves; ++w) m = fmaxf(m, shared.top[w][row]);
        const float base = m == WHT_NEG_INF ? 0.0f : m;
        f32x4 o = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
        for (int w = 0; w < S::kWaves; ++w) {
            const float f = __builtin_amdgcn_exp2f(shared.top[w][row] - base);
            l += shared.l[w][row] * f;
            o += f * *reinterpret_cast<const f32x4*>(&shared.o[w][row][col]);
        }
        o *= l == 0.0f ? 0.0f : 1.0f / l;
        if (args.transform) o = transform_outputs(o);
        if (row0 + lane / kLanes >= rows || lane >= kRowsOfWave * kLanes) continue;
        const int token = row / a.G, qh = head * a.G + row % a.G;
        const int64_t t = s.first + token;
        store4<T>(a.out + t * a.out_ts + qh * a.out_hs + col * sizeof(T), o);
        if (a.lse && col == 0) a.lse[t * a.q_heads + qh] = l == 0.0f ? WHT_NEG_INF : (m + __builtin_amdgcn_logf(l)) * kLn2;
    }
}

// ------------------------------------------------------------------------------------------------
// Many rows: the pipeline of attention_device.h -- 128 rows a workgroup, 64 keys a step, keys and values in LDS twice over -- behind registers: a thread holds
// the codes of the steps after those in LDS, and makes bfloat16 rows of them as a step begins.

// Where chunks stand in LDS, as in Head, but for rows that are written from registers: a write takes eight rows' chunks at a time, which have to fill 128 bytes
// (r0, r1, ...: the bits of a row's number).  Reads are as there: K's 16 rows at a time fill 256 bytes, V's 64 bytes of four rows.
template <int D>
struct Written : Head<bf16, D> {
    static __device__ __forceinline__ int k_place(int r, int c) {
        if constexpr (D == 128) return c ^ (r & 15);
        else if constexpr (D == 64) return c ^ ((r >> 1 & 3) | ((r ^ r >> 3) & 1) << 2);
        else { const int p = c + (r >> 2 & 1) + 2 * ((r >> 1 ^ r >> 3) & 1); return p >= 12 ? p - 12 : p; }
    }
    static __device__ __forceinline__ int v_place(int r, int c) {
        if constexpr (D == 128) return c ^ ((r & 3) << 2 | (r >> 2 & 1) << 1 | (r >> 1 & 1));
        else if constexpr (D == 64) return c ^ ((r >> 1 & 1) << 2 | (r >> 2 & 1) << 1 | (r & 1));
        else return c ^ ((r >> 2 & 1) << 1 | (r >> 1 & 1));
    }
};

template <class T, int D>
struct Many4 {
    using L = Head<bf16, D>;
    using W = Written<D>;
    static constexpr int kTermsOf = kTerms<T>;
    static constexpr int kBytes = D == 64 ? 8 : 16;                 // of codes, that a lane takes of a step: a wave 16 rows
    static constexpr int kPieces = D / 2 / kBytes;                  // of a row: 4, 3, 4
    static constexpr int kWords = kBytes / 4;
    static constexpr int kTileBytes = kStepKeys * L::kRowBytes;

    struct Raw { unsigned code[kWords]; unsigned scale; };

    // See ManyRange::stream.
    static __device__ __forceinline__ void stream(const Attention4Args& args, const Keys& k, PageList& list, int lo, int hi, int limit, int all_see, int any_sees, int level,
                                                  int head, unsigned buf, const u32x4 (&q)[kTermsOf][L::kSteps], FirstOdd<D>& odd, RowState<L>& st) {
        const AttentionArgs& a = args.base;
        const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), shift = a.page_shift;
        const int pre0 = min(lo, k.front) * kStepKeys, pre1 = min(min(hi, k.front) * kStepKeys, k.prefix);
        const int own0 = max(lo - k.front, 0) * kStepKeys, own1 = min(max(hi - k.front, 0) * kStepKeys, k.own);
        const int pre_pages = pre1 > pre0 ? ((pre1 - 1) >> shift) - (pre0 >> shift) + 1 : 0, own_pages = own1 > own0 ? ((own1 - 1) >> shift) - (own0 >> shift) + 1 : 0;
        const int pre_at = -(pre0 >> shift), own_at = pre_pages - (own0 >> shift);
        bool wrong = false;
        for (int i = threadIdx.x; i < pre_pages + own_pages; i += 256) {
            const int page = i < pre_pages ? k.prefix_table[i - pre_at] : k.own_table[i - own_at];
            const bool good = page >= 0 && page < a.pages;
            list.page[i] = good ? page : -1;
            wrong |= !good;
        }
        wrong = __any(wrong);
        if (lane == 0) list.bad[wave] = wrong;
        __syncthreads();
        const bool bad = __builtin_amdgcn_readfirstlane(list.bad[0] | list.bad[1] | list.bad[2] | list.bad[3]) != 0;

        // the thread's piece of a step's rows
        const int r = wave * 16 + (lane & 15), piece = lane >> 4;
        const bool loads = piece < kPieces;
        const unsigned char *kc = a.k + head * a.head_stride, *vc = a.v + head * a.head_stride, *ks = args.ks + head * args.s_head_stride, *vs = args.vs + head * args.s_head_stride;
        const unsigned code_off = (lane & 15) * a.token_stride + min(piece, kPieces - 1) * kBytes, scale_off = (lane & 15) * args.s_token_stride + min(piece, kPieces - 1) * kBytes / 16;
        auto take = [&](const unsigned char* from, const unsigned char* scale, Raw& x) {
            if constexpr (kWords == 4) {
                const u32x4 w = *reinterpret_cast<const u32x4*>(from);
#pragma unroll
                for (int i = 0; i < 4; ++i) x.code[i] = w[i];
            } else {
                const uint64_t w = *reinterpret_cast<const uint64_t*>(from);
                x.code[0] = (unsigned)w;
                x.code[1] = (unsigned)(w >> 32);
            }
            x.scale = *scale;
        };
        // Where a step's keys are all there, in pages of 16 tokens at least, a wave's 16 are in one page, and a lane's place in it is the same every step.
        auto fetch = [&](int t, const unsigned char* codes, const unsigned char* scales, Raw& x) {
            const bool own = t >= k.front;
            const int key0 = (own ? t - k.front : t) * kStepKeys, keys = own ? k.own : k.prefix, list_at = own ? own_at : pre_at;
            if (!bad && shift >= 4 && key0 + kStepKeys <= keys) {
                const int key = key0 + wave * 16;
                const unsigned page = __builtin_amdgcn_readfirstlane(list.page[(key >> shift) + list_at]), slot = key & ((1 << shift) - 1);
                take(codes + ((uint64_t)page * a.page_stride + slot * a.token_stride) + code_off, scales + ((uint64_t)page * args.s_page_stride + slot * args.s_token_stride) + scale_off, x);
            } else {
                const int key = key0 + r, page = loads && key < keys ? list.page[(key >> shift) + list_at] : -1;
                const unsigned slot = (unsigned)(key & ((1 << shift) - 1));
                const unsigned char *from = zero_chunk, *scale = zero_chunk;
                if (page >= 0) {
                    from = codes + ((uint64_t)(unsigned)page * a.page_stride + slot * a.token_stride + piece * kBytes);
                    scale = scales + ((uint64_t)(unsigned)page * args.s_page_stride + slot * args.s_token_stride + piece * kBytes / 16);
                }
                take(from, scale, x);
            }
        };
        auto put_k = [&](int t, const Raw& x) {
            if (!loads) return;
            const float f = scale_of(x.scale);
            const unsigned at = buf + (t & 1) * kTileBytes + r * L::kRowBytes;
#pragma unroll
            for (int i = 0; i < kWords; ++i)
                *(__attribute__((address_space(3))) u32x4*)(uintptr_t)(at + W::k_place(r, piece * kWords + i) * 16) = __builtin_bit_cast(u32x4, decode(x.code[i], f));
        };
        // From this step on rows of the workgroup see different keys: blocks that are no numbers stay out of the product, and rows that see one get it at the end.
        const int uneven = k.front + level / kStepKeys;
        auto put_v = [&](int t, Raw& x) {
            if (!loads) return;
            if (t >= uneven && x.scale >= 253) {
                list.odd[wave] = 1;
#pragma unroll 1
                for (int i = 0; i < kBytes * 2; ++i) {
                    const int col = piece * kBytes * 2 + i, key = (t - k.front) * kStepKeys + r;
                    atomicMin(&odd.above[col], key);
                    atomicMin(&odd.below[col], key);
                }
                x.scale = 127;
#pragma unroll
                for (int i = 0; i < kWords; ++i) x.code[i] = 0;
            }
            const float f = scale_of(x.scale);
            const unsigned at = buf + (2 + (t & 1)) * kTileBytes + r * L::kRowBytes;
#pragma unroll
            for (int i = 0; i < kWords; ++i)
                *(__attribute__((address_space(3))) u32x4*)(uintptr_t)(at + W::v_place(r, piece * kWords + i) * 16) = __builtin_bit_cast(u32x4, decode(x.code[i], f));
        };
        // the first or second 32 keys or values of step t
        auto keys_at = [&](int t, int half) { return fresh(buf + (t & 1) * kTileBytes + half * 32 * L::kRowBytes); };
        auto values_at = [&](int t, int half) { return fresh(buf + (2 + (t & 1)) * kTileBytes + half * 32 * L::kRowBytes); };

        // Blocks of 32 keys count as steps do.
        const int front = 2 * k.front, pre_full = any_sees < 0 ? 0 : k.prefix / 32, own_full = any_sees < 0 ? 0 : all_see / 32;
        auto full = [&](int j) { return j < front ? j < pre_full : j - front < own_full; };
        auto hide = [&](f32x16& s, int j) {
            const bool own = j >= front;
            const int key0 = (own ? j - front : j) * 32, sees = own ? limit : k.prefix, list_at = own ? own_at : pre_at;
#pragma unroll
            for (int i = 0; i < 16; ++i) {
                const int key = key0 + key_of(i);
                bool seen = key < sees;
                if (bad && seen) seen = list.page[(key >> shift) + list_at] >= 0;
                s[i] = seen ? s[i] : WHT_NEG_INF;
            }
        };
        auto in_sight = [&](int j) { return j < front ? any_sees >= 0 : (j - front) * 32 < any_sees; };

        u32x4 frag[L::kSteps];                                      // keys of the block after the one whose scores are at hand
        auto read_keys = [&](unsigned at) {
            const unsigned first_chunk = KeyReads<bf16, D, W>::first(at);
#pragma unroll
            for (int i = 0; i < L::kSteps; ++i) frag[i] = lds_read<u32x4>(KeyReads<bf16, D, W>::chunk(first_chunk, i));
        };
        auto product = [&](f32x16& s) {
            s = f32x16{};
#pragma unroll
            for (int i = 0; i < L::kSteps; ++i)
#pragma unroll
                for (int e = kTermsOf - 1; e >= 0; --e) s = score_step<bf16>(frag[i], q[e][i], s);
        };
        // the weights of `s`, and their products with the values at `vat`
        auto accumulate4 = [&](f32x16& s, unsigned vat) {
            weigh(s, a.scale, st);
            bf16x8 w[kTermsOf][2];
#pragma unroll
            for (int i = 0; i < 16; ++i) {
                bf16 t[kTermsOf];
                split<kTermsOf>(s[i], t);
#pragma unroll
                for (int e = 0; e < kTermsOf; ++e) w[e][i >> 3][i & 7] = t[e];
            }
#pragma unroll
            for (int d = 0; d < L::kBlocks; ++d) {
#pragma unroll
                for (int half = 0; half < 2; ++half) {
                    const bf16x8 v = values<D, W>(vat, half, d);
#pragma unroll
                    for (int e = kTermsOf - 1; e >= 0; --e) st.o[d] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(v, w[e][half], st.o[d], 0, 0, 0);
                }
                asm volatile("" ::: "memory");                      // one block's values in registers at a time
            }
        };

        // See full_block of ManyRange::stream.
        auto full_block = [&](f32x16& s, f32x16& ahead, unsigned vat, unsigned kat, bool more) {
            if constexpr (kTermsOf == 1) {
                const unsigned first_chunk = KeyReads<bf16, D, W>::first(kat);
                bf16x8 w[2];
                float sum[2] = {0.0f, 0.0f};
                ahead = f32x16{};
#pragma unroll
                for (int i = 0; i < L::kSteps; ++i) {
                    ahead = score_step<bf16>(frag[i], q[0][i], ahead);
                    frag[i] = __builtin_bit_cast(u32x4, values<D, W>(vat, i / L::kBlocks, i % L::kBlocks));
#pragma unroll
                    for (int e = 16 * i / L::kSteps; e < 16 * (i + 1) / L::kSteps; ++e) {
                        const float p = __builtin_amdgcn_exp2f(__builtin_fmaf(s[e], a.scale, -st.base));
                        sum[e & 1] += p;
                        w[e >> 3][e & 7] = (bf16)p;
                    }
                    __builtin_amdgcn_sched_barrier(0);
                }
                float mx = WHT_NEG_INF;
#pragma unroll
                for (int i = 0; i < L::kSteps; ++i) {
                    st.o[i % L::kBlocks] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, frag[i]), w[i / L::kBlocks], st.o[i % L::kBlocks], 0, 0, 0);
                    frag[i] = lds_read<u32x4>(KeyReads<bf16, D, W>::chunk(first_chunk, i));
                    // the last of `ahead` is a few instructions old
                    if (i >= L::kSteps / 2)
#pragma unroll
                        for (int e = 16 * (2 * i - L::kSteps) / L::kSteps; e < 16 * (2 * i - L::kSteps + 2) / L::kSteps; ++e) mx = fmaxf(mx, ahead[e]);
                    __builtin_amdgcn_sched_barrier(0);
                }
                st.l += sum[0] + sum[1];
                if (more) ::wht::rebase<L, 8>(mx, a.scale, ahead, st);
            } else {
                product(ahead);
                accumulate4(s, vat);
                read_keys(kat);
                if (more) ::wht::rebase<L, 8>(largest(ahead), a.scale, ahead, st);
            }
        };

        Raw rk, rv;
        fetch(lo, kc, ks, rk);
        fetch(lo, vc, vs, rv);
        put_k(lo, rk);
        put_v(lo, rv);
        if (lo + 1 < hi) {
            fetch(lo + 1, kc, ks, rk);
            fetch(lo + 1, vc, vs, rv);
            put_k(lo + 1, rk);
        }
        if (lo + 2 < hi) fetch(lo + 2, kc, ks, rk);
        workgroup_barrier();
        read_keys(keys_at(lo, 0));
        f32x16 s, other;
        product(s);
        if (bad || !full(2 * lo)) hide(s, 2 * lo);
        ::wht::rebase<L, 8>(largest(s), a.scale, s, st);
        read_keys(keys_at(lo, 1));
        auto refill = [&](int t) {
            if (t + 1 < hi) put_v(t + 1, rv);
            if (t + 2 < hi) {
                put_k(t + 2, rk);
                fetch(t + 2, vc, vs, rv);
            }
            if (t + 3 < hi) fetch(t + 3, kc, ks, rk);
        };
        // A step's barrier stands in both loops below: a wave takes a step in either, whatever the others do.
        for (int t = lo; t < hi; ++t) {
            // steps whose blocks, and the first of the next one, are seen by all rows of the wave
            const int blocks = 2 * t >= front || pre_full == front ? front + own_full : pre_full;
            for (const int end = bad ? t : min(uneven, blocks >= 2 * hi ? hi : min(hi - 1, (blocks - 1) / 2)); t < end; ++t) {
                workgroup_barrier();                                // V of this step and K of the next are in LDS; what is replaced next has been read
                refill(t);
                full_block(s, other, values_at(t, 0), keys_at(t + 1, 0), true);
                full_block(other, s, values_at(t, 1), keys_at(t + 1, 1), t + 1 < hi);
            }
            if (t == hi) break;
            workgroup_barrier();
            refill(t);
#pragma unroll 1
            for (int half = 0; half < 2; ++half) {
                const int j = 2 * t + half;
                if (!in_sight(j)) break;                            // nor is any that follows
                const bool more = j + 1 < 2 * hi && in_sight(j + 1);
                if (more) product(other);
                accumulate4(s, values_at(t, half));
                if (more) {
                    if (t + 1 < hi) read_keys(keys_at(t + 1, half));
                    if (bad || !full(j + 1)) hide(other, j + 1);
                    ::wht::rebase<L, 8>(largest(other), a.scale, other, st);
                    s = other;
                }
            }
        }
    }

    static __device__ __forceinline__ void run(const Attention4Args& args, const Keys& k, PageList& list, int t0, int t1, int limit, int all_see, int any_sees, int level,
                                               int head, unsigned buf, const u32x4 (&q)[kTermsOf][L::kSteps], FirstOdd<D>& odd, RowState<L>& st) {
        for (int c = threadIdx.x; c < D; c += 256) odd.above[c] = odd.below[c] = INT_MAX;
        if (threadIdx.x < 4) list.odd[threadIdx.x] = 0;
        const int per_list = max(((kListed - 4) << args.base.page_shift) / kStepKeys, 1);           // each part may begin and end within a page
        for (int lo = t0; lo < t1; lo += per_list) {
            if (lo > t0) workgroup_barrier();                       // the last steps' reads are done
            stream(args, k, list, lo, min(t1, lo + per_list), limit, all_see, any_sees, level, head, buf, q, odd, st);
        }
        workgroup_barrier();
        if ((list.odd[0] | list.odd[1] | list.odd[2] | list.odd[3]) != 0) add_odd<bf16, D>(limit, odd, st);
    }
};

template <int D>
struct ManyShared {
    __align__(16) unsigned char buf[256 * Head<bf16, D>::kRowBytes];
    FirstOdd<D> odd;
    PageList list;
};

// H (of 32) / 8 of a row's outputs, whose block d a lane and the one 32 away hold as RowState does.
template <int D>
__device__ __forceinline__ void transform_row(RowState<Head<bf16, D>>& st) {
#pragma unroll
    for (int d = 0; d < D / 32; ++d) {
        f32x16& x = st.o[d];
#pragma unroll
        for (int h = 1; h < 16; h *= 2)
#pragma unroll
            for (int i = 0; i < 16; ++i)
                if (!(i & h)) {
                    const float a = x[i], b = x[i + h];
                    x[i] = a + b;
                    x[i + h] = a - b;
                }
#pragma unroll
        for (int i = 0; i < 16; ++i) {
            const float other = other_half(x[i]);
            x[i] = (threadIdx.x & 32 ? other - x[i] : x[i] + other) * 0.125f;
        }
    }
}

// The line of tiles is that of many_rows() in attention_device.h.  STACKED: the rows of all sequences, against the prefix alone.
template <class T, int D, bool STACKED>
__device__ __forceinline__ void many_rows4(const Attention4Args& args, int block, ManyShared<D>& shared) {
    using L = Head<bf16, D>;
    using R = Many4<T, D>;
    const AttentionArgs& a = args.base;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int x = block % kDies, y = block / kDies, groups = a.heads * a.splits;
    auto tiles_of = [&](int queries) { return (int)(((int64_t)queries * a.G + kTileRows - 1) / kTileRows); };
    int b = 0, cum = 0;
    Sequence s{0, a.batch.T, 0};
    if constexpr (STACKED) {
        if (y >= die_groups(0, groups, x) * tiles_of(s.queries)) return;
    } else {
        if (y == a.fill) {                                          // the grid's last workgroups, one per die
            if (a.splits == 1) fill_rows<T, D>(a, x);
            return;
        }
        const int B = a.batch.B, run = max(ceil_div(B, 64), 1), b0 = min(B, lane * run), b1 = min(B, b0 + run);
        auto tiles_at = [&](int i) { return die_groups(i, groups, x) * tiles_of(min(s.queries, a.max_q)); };
        int mine = 0;
        for (int i = b0; i < b1; ++i) {
            s = sequence(a.batch, i);
            mine = add_tiles(mine, tiles_at(i));
        }
        int upto = mine;
#pragma unroll
        for (int o = 1; o < 64; o <<= 1) {
            const int v = __shfl_up(upto, o);
            if (lane >= o) upto += v;
        }
        if (y >= __builtin_amdgcn_readlane(upto, 63)) return;
        const int from = __popcll(__ballot(upto <= y));             // the lane whose run has it
        b = from * run;
        cum = __builtin_amdgcn_readlane(upto - mine, from);
        if (run == 1) s = {__builtin_amdgcn_readlane(s.first, b), __builtin_amdgcn_readlane(s.queries, b), __builtin_amdgcn_readlane(s.length, b)};
        else
            for (s = sequence(a.batch, b); y >= cum + tiles_at(b); s = sequence(a.batch, ++b)) cum += tiles_at(b);
    }
    const int queries = STACKED ? s.queries : min(s.queries, a.max_q);
    // of a group the tiles that see most come first
    const int tiles = tiles_of(queries), k = (y - cum) / tiles, tile = tiles - 1 - (y - cum - k * tiles);
    const int group = die_group(b, groups, x, k), part = group % a.splits, head = group / a.splits;
    const int64_t rows = (int64_t)queries * a.G;
    const int row0 = tile * kTileRows + wave * 32, row = row0 + (lane & 31);
    const int token = row / a.G, qh = head * a.G + row % a.G;
    const bool there = row < rows;
    u32x4 q[R::kTermsOf][L::kSteps];
    const unsigned char* q_at = a.q + (s.first + (there ? token : 0)) * a.q_ts + qh * a.q_hs;
#pragma unroll
    for (int c = 0; c < L::kSteps; ++c) {
        bf16x8 t[R::kTermsOf];
        load_terms<T, R::kTermsOf>(q_at + (2 * c + (lane >> 5)) * 8 * sizeof(T), there, t);
#pragma unroll
        for (int e = 0; e < R::kTermsOf; ++e) q[e][c] = __builtin_bit_cast(u32x4, t[e]);
    }
    // own tokens that row r of the tile sees: length - queries + its token + 1
    auto sees = [&](int64_t r) { return STACKED ? 0 : min(max(s.length - s.queries + (int)(min(r, rows - 1) / a.G) + 1, 0), s.length); };
    const int keys = sees(tile * kTileRows + kTileRows - 1);
    const int limit = sees(row), all_see = sees(row0), any_sees = row0 < rows ? sees(row0 + 31) : -1;
    const int front = a.use_prefix ? ceil_div(a.prefix, kStepKeys) : 0;
    const int total = front + ceil_div(keys, kStepKeys), per = ceil_div(total, a.splits);
    const int t0 = min(total, part * per), t1 = min(total, t0 + per);
    RowState<L> st;
    st.clear();
    const Keys keys_of{a.prefix_table, a.batch.table + b * a.batch.table_stride, front, a.use_prefix ? a.prefix : 0, keys};
    R::run(args, keys_of, shared.list, t0, t1, limit, all_see, any_sees, sees((int64_t)tile * kTileRows), head, __builtin_amdgcn_readfirstlane(lds_address(shared.buf)), q,
           shared.odd, st);
    st.l += other_half(st.l);
    const int64_t t = s.first + token;
    if (a.splits > 1 || STACKED) {
        if (!there) return;
        const int64_t at = ((int64_t)part * a.batch.T + t) * a.q_heads + qh;
        if (lane < 32) { a.sums[at * 2] = st.top * a.scale; a.sums[at * 2 + 1] = st.l; }
#pragma unroll
        for (int d = 0; d < L::kBlocks; ++d)
#pragma unroll
            for (int i = 0; i < 4; ++i)
                *reinterpret_cast<f32x4*>(a.part + at * D + d * 32 + i * 8 + (lane >> 5) * 4) = f32x4{st.o[d][4 * i], st.o[d][4 * i + 1], st.o[d][4 * i + 2], st.o[d][4 * i + 3]};
    } else {
        const float inv = st.l == 0.0f ? 0.0f : 1.0f / st.l;
#pragma unroll
        for (int d = 0; d < L::kBlocks; ++d)
#pragma unroll
            for (int i = 0; i < 16; ++i) st.o[d][i] *= inv;
        if (args.transform) transform_row<D>(st);
        if (!there) return;
        if (a.lse && lane < 32) a.lse[t * a.q_heads + qh] = st.l == 0.0f ? WHT_NEG_INF : (st.top * a.scale + __builtin_amdgcn_logf(st.l)) * kLn2;
#pragma unroll
        for (int d = 0; d < L::kBlocks; ++d)
#pragma unroll
            for (int i = 0; i < 4; ++i)
                store4<T>(a.out + t * a.out_ts + qh * a.out_hs + (d * 32 + i * 8 + (lane >> 5) * 4) * sizeof(T),
                          f32x4{st.o[d][4 * i], st.o[d][4 * i + 1], st.o[d][4 * i + 2], st.o[d][4 * i + 3]});
    }
}

// ------------------------------------------------------------------------------------------------

template <class T, int D>
__global__ __launch_bounds__(256, (sizeof(T) == 2 ? 2 : 1)) void many_rows4_kernel(Attention4Args a) {
    __shared__ ManyShared<D> shared;
    many_rows4<T, D, false>(a, blockIdx.x, shared);
}

template <class T, int D, int TILES, bool MULTI, bool FRONT, bool NARROW, bool STREAM>
__global__ __launch_bounds__(256, (sizeof(T) == 4 ? 1 : workgroups4(false, D, TILES, FRONT) / 256)) void few_rows4_kernel(Attention4Args a, Attention4Args front, int front_blocks) {
    if constexpr (FRONT) {
        __shared__ union Both {
            FewShared<T, D, TILES> few;
            ManyShared<D> many;
        } shared;
        const int block = blockIdx.x;
        if (block < front_blocks) many_rows4<T, D, true>(front, block, shared.many);
        else few_rows4<T, D, TILES, MULTI, true, NARROW, STREAM>(a, block - front_blocks, shared.few);
    } else {
        __shared__ FewShared<T, D, TILES> shared;
        few_rows4<T, D, TILES, MULTI, false, NARROW, STREAM>(a, blockIdx.x, shared);
    }
}

}  // namespace wht
