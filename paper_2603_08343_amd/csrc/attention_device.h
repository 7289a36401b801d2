// Kernels of the paged cache and its attention (include/wht_attention.h) for gfx950.
#pragma once
#include <hip/hip_runtime.h>
#include <limits.h>

#include "attention_plan.h"

namespace wht {

typedef __bf16 bf16;
typedef bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef bf16 bf16x4 __attribute__((ext_vector_type(4)));
typedef bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef short short4v __attribute__((ext_vector_type(4)));
typedef unsigned short ushort2v __attribute__((ext_vector_type(2)));
typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef unsigned u32x4 __attribute__((ext_vector_type(4)));
typedef __attribute__((address_space(3))) unsigned char lds_byte;

constexpr float kLn2 = 0.693147180559945309f;
#define WHT_NEG_INF (-__builtin_inff())

// ------------------------------------------------------------------------------------------------
// The batch

struct Batch {
    const int *table, *lengths, *q_starts;
    int64_t table_stride;
    int B, T, most;                     // most: lengths are cut to it
};

struct Sequence { int first, queries, length; };     // first row, new tokens, own tokens

__device__ __forceinline__ Sequence sequence(const Batch& bt, int b) {
    int lo = b, hi = b + 1;
    if (bt.q_starts) { lo = bt.q_starts[b]; hi = bt.q_starts[b + 1]; }
    lo = min(max(lo, 0), bt.T);
    hi = min(max(hi, lo), bt.T);
    return {lo, hi - lo, min(max(bt.lengths[b], 0), bt.most)};
}

// The sequence that row t belongs to, -1 for none: the number of sequences that end at or before t.  A wave looks at 64 evenly
// spaced ends at a time, so that two dependent loads serve 4096 sequences.
__device__ __forceinline__ int sequence_of(const Batch& bt, int t) {
    if (!bt.q_starts) return t < bt.B ? t : -1;
    int lo = 0, n = bt.B;               // the answer is in [lo, lo + n]
    while (n > 0) {
        const int step = (n + 63) >> 6, lane = threadIdx.x & 63, at = (lane + 1) * step - 1;
        const bool ended = at < n && bt.q_starts[1 + lo + at] <= t;
        const int whole = __popcll(__ballot(ended));
        lo += whole * step;
        n = min(n - whole * step, step - 1);
    }
    return lo < bt.B ? lo : -1;
}

// Which of a grid's workgroups (grid_of) this is.
__device__ __forceinline__ int block_of() { return (int)((blockIdx.y << kGridLog2) + blockIdx.x); }

// ------------------------------------------------------------------------------------------------
// Append: bound by memory, and one token by the latency of its chain (length -> table entry -> store).  A workgroup, or a wave of it (THREADS), takes one
// token, so that what is looked up for it -- sequence, page, angles -- is looked up once; a thread takes the same 16-byte vector pair
// of every (THREADS / pairs)-th head, with that pair's cosines and sines in registers over the heads.  32766 tokens at 64 and 8 heads of 128 in
// bfloat16 (1.34 GB): 244 us, 5.5 TB/s; one token at 32 and 8 heads: 2.6 us.

struct AppendArgs {
    Batch batch;
    const unsigned char *q, *kn, *vn;
    unsigned char *q_out, *k, *v;
    int64_t q_ts, q_hs, k_ts, k_hs, v_ts, v_hs, qo_ts, qo_hs;       // bytes
    int64_t page_stride, head_stride, token_stride;                 // bytes
    const float* rope;
    int64_t rope_rows;
    int q_heads, heads, pages, page_shift, rotary, interleaved, position, places;         // places: that a row of the table has
};

template <class T> struct Vec16 { static constexpr int n = 16 / sizeof(T); T e[n]; };

template <class T>
__device__ __forceinline__ void load16(float (&f)[16 / sizeof(T)], const unsigned char* p) {
    const u32x4 raw = *reinterpret_cast<const u32x4*>(p);
    const Vec16<T> v = __builtin_bit_cast(Vec16<T>, raw);
#pragma unroll
    for (int i = 0; i < Vec16<T>::n; ++i) f[i] = (float)v.e[i];
}
template <class T>
__device__ __forceinline__ void store16(unsigned char* p, const float (&f)[16 / sizeof(T)]) {
    Vec16<T> v;
#pragma unroll
    for (int i = 0; i < Vec16<T>::n; ++i) v.e[i] = (T)f[i];
    *reinterpret_cast<u32x4*>(p) = __builtin_bit_cast(u32x4, v);
}

template <class T, int D, int THREADS>
__global__ __launch_bounds__(256) void append_kernel(AppendArgs a) {
    constexpr int N = 16 / sizeof(T), kPairs = D / (2 * N), kHeads = THREADS / kPairs;
    const int thread = threadIdx.x % THREADS, pair = thread % kPairs, first = thread / kPairs;
    const int t = THREADS == 256 ? block_of() : __builtin_amdgcn_readfirstlane(block_of() * (256 / THREADS) + threadIdx.x / THREADS);
    if (t >= a.batch.T) return;
    const int b = sequence_of(a.batch, t);
    int64_t place = -1, position = -1;
    if (b >= 0) {
        const Sequence s = sequence(a.batch, b);
        const int p = s.length - s.queries + (t - s.first);
        if (t >= s.first && t < s.first + s.queries) {
            position = (int64_t)a.position + p;
            if (p >= 0 && p < a.places) {
                const int page = a.batch.table[b * a.batch.table_stride + (p >> a.page_shift)];
                if (page >= 0 && page < a.pages) place = page * a.page_stride + (p & ((1 << a.page_shift) - 1)) * a.token_stride;
            }
        }
    }
    const bool turns = a.rotary > 0, known = !turns || (position >= 0 && position < a.rope_rows);
    if (!known) place = -1;
    // where the pair's two vectors stand in a head, and its angles
    const int half = a.rotary / 2, turned = a.rotary / (2 * N);     // vector pairs that turn
    const bool turn = known && pair < turned;
    int e0 = pair * 2 * N, e1 = e0 + N;
    if (pair < turned && !a.interleaved) { e0 = pair * N; e1 = half + pair * N; }
    float c[N], s[N];
#pragma unroll
    for (int i = 0; i < N; ++i) { c[i] = 1.0f; s[i] = 0.0f; }
    if (turn) {
        const f32x4* cs = reinterpret_cast<const f32x4*>(a.rope + position * a.rotary + pair * 2 * N);
#pragma unroll
        for (int i = 0; i < N / 2; ++i) {
            const f32x4 w = cs[i];
            c[2 * i] = w[0]; s[2 * i] = w[1]; c[2 * i + 1] = w[2]; s[2 * i + 1] = w[3];
        }
    }
    auto rotate = [&](float (&x)[N], float (&y)[N]) {
        if (!turn) return;
        if (a.interleaved) {
#pragma unroll
            for (int i = 0; i < N / 2; ++i) {
                const float u = x[2 * i], w = x[2 * i + 1], g = y[2 * i], h = y[2 * i + 1];
                x[2 * i] = u * c[i] - w * s[i];
                x[2 * i + 1] = w * c[i] + u * s[i];
                y[2 * i] = g * c[N / 2 + i] - h * s[N / 2 + i];
                y[2 * i + 1] = h * c[N / 2 + i] + g * s[N / 2 + i];
            }
        } else {
#pragma unroll
            for (int i = 0; i < N; ++i) {
                const float u = x[i], w = y[i];
                x[i] = u * c[i] - w * s[i];
                y[i] = w * c[i] + u * s[i];
            }
        }
    };
    if (first >= kHeads) return;                                    // 96 wide: the threads are no multiple of the pairs
    constexpr int kSize = sizeof(T);
    if (a.q) {
        for (int h = first; h < a.q_heads; h += kHeads) {
            unsigned char* to = a.q_out + t * a.qo_ts + h * a.qo_hs;
            float x[N], y[N];
            if (b >= 0 && known) {
                const unsigned char* from = a.q + t * a.q_ts + h * a.q_hs;
                load16<T>(x, from + e0 * kSize);
                load16<T>(y, from + e1 * kSize);
                rotate(x, y);
            } else {
#pragma unroll
                for (int i = 0; i < N; ++i) x[i] = y[i] = b >= 0 ? __builtin_nanf("") : 0.0f;
            }
            store16<T>(to + e0 * kSize, x);
            store16<T>(to + e1 * kSize, y);
        }
    }
    if (place < 0) return;
    for (int h = first; h < a.heads; h += kHeads) {
        const unsigned char* from = a.kn + t * a.k_ts + h * a.k_hs;
        const int64_t to = place + h * a.head_stride;
        float x[N], y[N];
        load16<T>(x, from + e0 * kSize);
        load16<T>(y, from + e1 * kSize);
        const unsigned char* vf = a.vn + t * a.v_ts + h * a.v_hs;
        const u32x4 v0 = *reinterpret_cast<const u32x4*>(vf + e0 * kSize), v1 = *reinterpret_cast<const u32x4*>(vf + e1 * kSize);
        rotate(x, y);
        store16<T>(a.k + to + e0 * kSize, x);
        store16<T>(a.k + to + e1 * kSize, y);
        *reinterpret_cast<u32x4*>(a.v + to + e0 * kSize) = v0;
        *reinterpret_cast<u32x4*>(a.v + to + e1 * kSize) = v1;
    }
}

// ------------------------------------------------------------------------------------------------
// Attention.  For one key head, R = up to 32 rows (queries) are the columns of
//
//     S^T = K Q^T   [keys x rows]        O^T += V^T P^T   [head_dim x rows],     P = exp2(S scale log2(e) - m)
//
// on the 32 x 32 matrix instructions.  The scores of a column then lie in the two lanes r and r + 32, 16 keys each, so that the softmax's
// maximum is 16 register operations and one exchange, a column's factor is one register, and -- the order of the keys within a
// product being free -- the weights are the second product's B operand where they stand: no value of S or P changes lanes.

struct AttentionArgs {
    Batch batch;
    const unsigned char *q, *k, *v;
    unsigned char* out;
    float *lse, *part, *sums;
    int* cum;
    const int* prefix_table;
    int64_t q_ts, q_hs, out_ts, out_hs;             // bytes
    int64_t head_stride;                            // bytes
    unsigned page_stride, token_stride;             // bytes
    int q_heads, heads, G, pages, page_shift, prefix, max_q;
    int splits, fill, rows_cap;                     // fill: the workgroups (of each die) that take the rows no tile covers; rows_cap: rows of one slot of partial results
    int use_prefix;                                 // the range begins with the prefix
    int gang_log2;                                  // few rows: heads that a worker takes side by side
    int front_item;                                 // few rows: the rows of all sequences against the prefix are one more sequence on the line
    float scale;                                    // scale * log2(e)
};

template <class T, int D>
struct Head {
    static constexpr int kChunks = D * sizeof(T) / 16;              // 16-byte chunks of a row
    static constexpr int kRowBytes = kChunks * 16;
    static constexpr int kSteps = kChunks / 2;                      // chunk pairs: lanes below 32 take the even one, the others the odd one
    static constexpr int kBlocks = D / 32;
    static constexpr bool kF32 = sizeof(T) == 4;

    // Where chunk c of row r stands in LDS.  K is read a chunk per row over 32 rows: 16 rows' reads have to reach all 16 groups of
    // four banks.  V is read 64 (bf16: transposing reads, four rows each) or 128 bytes of a row at a time.
    static __device__ __forceinline__ int k_place(int r, int c) {
        if constexpr (kChunks == 8) return c ^ ((r >> 1) & 7);
        else if constexpr (kChunks == 16 || kChunks == 32) return c ^ (r & 15);
        else { const int p = c + ((r >> (kChunks == 12 ? 2 : 1)) & (kChunks == 12 ? 3 : 7)); return p >= kChunks ? p - kChunks : p; }
    }
    static __device__ __forceinline__ int k_chunk(int r, int p) {
        if constexpr (kChunks == 12 || kChunks == 24) { const int c = p - ((r >> (kChunks == 12 ? 2 : 1)) & (kChunks == 12 ? 3 : 7)); return c < 0 ? c + kChunks : c; }
        else return k_place(r, p);
    }
    static __device__ __forceinline__ int v_place(int r, int c) {
        if constexpr (!kF32) {
            if constexpr (kChunks == 16) return c ^ ((r & 3) << 2);
            else if constexpr (kChunks == 8) return c ^ (((r >> 1) & 1) << 2);
            else return c;
        } else {
            if constexpr (kChunks == 24) { const int p = c + 8 * ((r >> 2) & 1); return p >= 24 ? p - 24 : p; }
            else return c ^ (((r >> 2) & 1) << 3);
        }
    }
    static __device__ __forceinline__ int v_chunk(int r, int p) {
        if constexpr (kF32 && kChunks == 24) { const int c = p - 8 * ((r >> 2) & 1); return c < 0 ? c + 24 : c; }
        else return v_place(r, p);
    }
};

// What a lane of a row (column of the products) keeps: the score that the row's weights are relative to (its maximum, or a little less: rebase), how far scores may
// pass it, what is taken off a scaled score in front of the exponential, this lane's share of the sum, and its half of the row's outputs.
template <class H>
struct RowState {
    float top, most, base, l;
    f32x16 o[H::kBlocks];
    __device__ __forceinline__ void clear() {
        top = most = WHT_NEG_INF;                                   // nothing seen yet: weights of zero
        base = l = 0.0f;
#pragma unroll
        for (int d = 0; d < H::kBlocks; ++d)
#pragma unroll
            for (int i = 0; i < 16; ++i) o[d][i] = 0.0f;
    }
};

// The value that the lane 32 away holds.
__device__ __forceinline__ float other_half(float x) {
    const unsigned u = __float_as_uint(x);
    const auto both = __builtin_amdgcn_permlane32_swap(u, u, false, false);
    return __uint_as_float((threadIdx.x & 32) ? both[0] : both[1]);
}

__device__ __forceinline__ unsigned lds_address(const void* p) { return (unsigned)(uintptr_t)(__attribute__((address_space(3))) const void*)p; }

// 16 bytes per lane from memory to LDS at base + 16 * lane, past the registers.  Assembly, because the compiler would otherwise wait for
// every such load in flight before any read of LDS; which have landed is known where wait_loads stands.  Reads of what is overwritten
// have returned (lgkmcnt).
// m0 is named as overwritten: the compiler, which never holds a value there for long, puts none across the statement then (that it cannot keep a reserved
// register's value over it is what the warning says, and what is meant).
// STREAM: read once, not kept in the caches.
#pragma clang diagnostic push
#pragma clang diagnostic ignored "-Winline-asm"
template <bool STREAM>
__device__ __forceinline__ void load_to_lds(const unsigned char* from, unsigned to) {
    if constexpr (STREAM) asm volatile("s_mov_b32 m0, %1\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %0, off nt" : : "v"(from), "s"(to) : "memory", "m0");
    else asm volatile("s_mov_b32 m0, %1\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %0, off" : : "v"(from), "s"(to) : "memory", "m0");
}
// The same from a place that all lanes share, `off` bytes on.
__device__ __forceinline__ void load_to_lds(const unsigned char* from, unsigned off, unsigned to) {
    asm volatile("s_mov_b32 m0, %2\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %0, %1" : : "v"(off), "s"(from), "s"(to) : "memory", "m0");
}
#pragma clang diagnostic pop
template <int PENDING> __device__ __forceinline__ void wait_loads() { asm volatile("s_waitcnt vmcnt(%0)" ::"n"(PENDING) : "memory"); }
__device__ __forceinline__ void reads_done() { asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory"); }
__device__ __forceinline__ void workgroup_barrier() {
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
}

// Loaded in place of keys that are not there.
static __device__ __align__(16) unsigned char zero_chunk[16];

// LDS addresses.  Where a row's chunks are a power of two, a place is the row's first one with the chunk's bits flipped in: one register and an
// exclusive or for each, which is less than the registers that all of them would take (fresh() keeps the compiler from doing that).
__device__ __forceinline__ unsigned fresh(unsigned x) {
    asm volatile("" : "+v"(x));
    return x;
}
template <class V>
__device__ __forceinline__ V lds_read(unsigned at) { return *(const __attribute__((address_space(3))) V*)(uintptr_t)at; }

template <class T, int D, class HEAD = Head<T, D>>
struct KeyReads {                                                   // a lane reads chunks h, 2 + h, 4 + h, ... of row lane % 32
    using H = HEAD;
    static constexpr bool kFlip = (H::kChunks & (H::kChunks - 1)) == 0;
    static __device__ __forceinline__ unsigned first(unsigned buf) {
        const int lane = threadIdx.x & 63, row = lane & 31, h = lane >> 5;
        return kFlip ? buf + row * H::kRowBytes + H::k_place(row, h) * 16 : buf + row * H::kRowBytes;
    }
    static __device__ __forceinline__ unsigned chunk(unsigned first, int c) {
        const int lane = threadIdx.x & 63, row = lane & 31, h = lane >> 5;
        return kFlip ? first ^ (c * 32) : first + H::k_place(row, 2 * c + h) * 16;
    }
};

template <class T>
__device__ __forceinline__ f32x16 score_step(u32x4 k, u32x4 q, f32x16 s) {
    if constexpr (sizeof(T) == 2) return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, k), __builtin_bit_cast(bf16x8, q), s, 0, 0, 0);
    const f32x4 kf = __builtin_bit_cast(f32x4, k), qf = __builtin_bit_cast(f32x4, q);
#pragma unroll
    for (int i = 0; i < 4; ++i) s = __builtin_amdgcn_mfma_f32_32x32x2f32(kf[i], qf[i], s, 0, 0, 0);
    return s;
}

// S^T of 32 keys in LDS at `buf` (16-byte aligned rows) and the wave's rows.
template <class T, int D>
__device__ __forceinline__ f32x16 scores(unsigned buf, const u32x4 (&q)[Head<T, D>::kSteps]) {
    const unsigned first = KeyReads<T, D>::first(buf);
    f32x16 s{};
#pragma unroll
    for (int c = 0; c < Head<T, D>::kSteps; ++c) s = score_step<T>(lds_read<u32x4>(KeyReads<T, D>::chunk(first, c)), q[c], s);
    return s;
}

// Key, of 32, whose score a lane's register i holds.
__device__ __forceinline__ int key_of(int i) { return (i >> 2) * 8 + ((threadIdx.x >> 5) & 1) * 4 + (i & 3); }

// The base of a row's weights follows its maximum; SLACK: not step by step, but when the maximum has grown by more than a factor of 2^SLACK.  With
// many rows, where the vector units' time counts, that is 8: one of a wave's 32 rows has a new maximum in most steps, and each
// one multiplies all the sums over.  Weights are up to 256 then, which float32 sums hold as exactly; but the largest of a row is no longer
// 1, which bfloat16 holds exactly: the error of the outputs, with that of their own rounding, goes from 1.9e-3 to 2.3e-3 of their norm.
// Float32 products hold a weight of 256 as exactly as one of 1 (two prompts of 4096 at 32 and 8 x 128: 1.07e-6; with the base at the maximum itself, in elementary
// operations, 1.04e-6).  With few rows, bound by memory, it is 0.
//
// A weight is exp2(s scale - base), one rounding, with base = top scale rounded: what that rounding is off by is a factor that all weights share, but for those that bfloat16
// rounds and their sum, which is not rounded.  Of a maximum of 2^31 it may be 2^128 or 2^-128, and the weights infinite or zero.  From kFar on, where the factor may be 1 + 2e-5,
// the maximum is taken off the scores themselves (exactly where it matters), in every step, and the base is zero.
constexpr float kFar = 1024.0f;

template <class H, int SLACK>
__device__ __forceinline__ void rebase(float mx, float scale, f32x16& s, RowState<H>& st) {
    mx = fmaxf(mx, other_half(mx));
    if (__any(mx > st.most)) {
        const float now = fmaxf(st.top, mx), m = now == WHT_NEG_INF ? 0.0f : now * scale;
        const bool far = fabsf(m) >= kFar;
        const float f = __builtin_amdgcn_exp2f(far ? (st.top - now) * scale : st.top * scale - m);
        st.l *= f;
#pragma unroll
        for (int d = 0; d < H::kBlocks; ++d)
#pragma unroll
            for (int i = 0; i < 16; ++i) st.o[d][i] *= f;
        st.top = now;
        st.base = far ? 0.0f : m;
        st.most = far ? WHT_NEG_INF : SLACK == 0 ? now : now + fminf(SLACK / scale, 3e38f);
        if (__any(far)) {
#pragma unroll
            for (int i = 0; i < 16; ++i) s[i] -= far ? now : 0.0f;
        }
    }
}
__device__ __forceinline__ float largest(const f32x16& s) {
    float mx = s[0];
#pragma unroll
    for (int i = 1; i < 16; ++i) mx = fmaxf(mx, s[i]);
    return mx;
}

// Scores become weights, and their sum.
template <class H>
__device__ __forceinline__ void weigh(f32x16& s, float scale, RowState<H>& st) {
    float sum[2] = {0.0f, 0.0f};
#pragma unroll
    for (int i = 0; i < 16; ++i) {
        s[i] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[i], scale, -st.base));
        sum[i & 1] += s[i];
    }
    st.l += sum[0] + sum[1];
}

// The A operand of the second product in bfloat16: 16 of 32 values in LDS at `buf` (ks: which), 32 columns from 32 d on.  A transposing read gives
// lane i of 16 the i-th of 16 columns, four rows of it, that the 16 lanes address as 4 x 4 pieces of 8 bytes.
template <int D, class H = Head<bf16, D>>
__device__ __forceinline__ bf16x8 values(unsigned buf, int ks, int d) {
    const int lane = threadIdx.x & 63, g = lane >> 4, in = lane & 15, row = (g >> 1) * 4 + (in >> 2), c = (g & 1) * 2 + ((in & 3) >> 1);
    const unsigned at = (H::kChunks & (H::kChunks - 1)) == 0 ? (buf + row * H::kRowBytes + H::v_place(row, c) * 16 + (in & 1) * 8) ^ (d * 64)
                                                             : buf + row * H::kRowBytes + H::v_place(row, d * 4 + c) * 16 + (in & 1) * 8;
    bf16x8 v;
#pragma unroll
    for (int e = 0; e < 2; ++e) {
        const short4v x = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) short4v*)(uintptr_t)(at + (ks * 16 + e * 8) * H::kRowBytes));
        const bf16x4 y = __builtin_bit_cast(bf16x4, x);
#pragma unroll
        for (int i = 0; i < 4; ++i) v[e * 4 + i] = y[i];
    }
    return v;
}

// o += (V^T P^T) over 32 keys in LDS at `buf`, for the 32 columns of V from 32 d on.
template <class T, int D>
__device__ __forceinline__ void block_product(unsigned buf, int d, const f32x16& p, f32x16& o) {
    using H = Head<T, D>;
    if constexpr (!H::kF32) {
#pragma unroll
        for (int ks = 0; ks < 2; ++ks) {
            bf16x8 w;
#pragma unroll
            for (int i = 0; i < 8; ++i) w[i] = (bf16)p[ks * 8 + i];
            o = __builtin_amdgcn_mfma_f32_32x32x16_bf16(values<D>(buf, ks, d), w, o, 0, 0, 0);
        }
    } else {
        constexpr bool kFlip = (H::kChunks & (H::kChunks - 1)) == 0;
        const int lane = threadIdx.x & 63, col = lane & 31, h4 = (lane >> 5) * 4;
        const unsigned at = kFlip ? (buf + h4 * H::kRowBytes + H::v_place(h4, col >> 2) * 16 + (col & 3) * 4) ^ (d * 128)
                                  : buf + h4 * H::kRowBytes + H::v_place(h4, d * 8 + (col >> 2)) * 16 + (col & 3) * 4;
#pragma unroll
        for (int i = 0; i < 16; ++i) {
            const float v = lds_read<float>(at + ((i >> 2) * 8 + (i & 3)) * H::kRowBytes);
            o = __builtin_amdgcn_mfma_f32_32x32x2f32(v, p[i], o, 0, 0, 0);
        }
    }
}

// Whether LOADS KiB in LDS hold anything that is not finite.
template <class T, int LOADS>
__device__ __forceinline__ bool any_odd(unsigned buf) {
    constexpr unsigned kMagnitude = sizeof(T) == 4 ? 0x7fffffffu : 0x7fff7fffu;
    unsigned most = 0;
    ushort2v most2 = {0, 0};
#pragma unroll
    for (int i = 0; i < LOADS; ++i) {
        const u32x4 x = lds_read<u32x4>(buf + (threadIdx.x & 63) * 16 + i * 1024);
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            if constexpr (sizeof(T) == 4) most = max(most, x[e] & kMagnitude);
            else most2 = __builtin_elementwise_max(most2, __builtin_bit_cast(ushort2v, x[e] & kMagnitude));
        }
    }
    return __any(sizeof(T) == 4 ? most >= 0x7f800000u : most2[0] >= 0x7f80 || most2[1] >= 0x7f80);
}

// The first of a block's keys whose value in a column is +infinity or NaN (above), -infinity or NaN (below); their number where there is none.
template <int D> struct FirstOdd { int above[D], below[D]; };

// To the outputs of a row that sees `seen` keys of them.
template <class T, int D>
__device__ __forceinline__ void add_odd(int seen, const FirstOdd<D>& first, RowState<Head<T, D>>& st) {
#pragma unroll
    for (int d = 0; d < Head<T, D>::kBlocks; ++d)
#pragma unroll
        for (int i = 0; i < 16; ++i) {
            const int c = d * 32 + key_of(i);
            st.o[d][i] += (first.above[c] < seen ? -WHT_NEG_INF : 0.0f) + (first.below[c] < seen ? WHT_NEG_INF : 0.0f);
            if ((i & 3) == 3) asm volatile("" ::: "memory");        // rare: its registers count, its time does not
        }
}

// Of 32 rows in LDS, by one wave, which makes zeros of them.
template <class T, int D>
__device__ __forceinline__ void take_odd(unsigned buf, FirstOdd<D>& first) {
    using H = Head<T, D>;
    for (int c = threadIdx.x & 63; c < D; c += 64) {
        int above = 32, below = 32;
#pragma unroll 1
        for (int k = 31; k >= 0; --k) {
            auto* p = (__attribute__((address_space(3))) T*)(uintptr_t)(buf + k * H::kRowBytes + H::v_place(k, c * (int)sizeof(T) / 16) * 16 + c * (int)sizeof(T) % 16);
            const float v = (float)*p;
            if (!(fabsf(v) < __builtin_inff())) {
                if (v != WHT_NEG_INF) above = k;
                if (v != -WHT_NEG_INF) below = k;
                *p = (T)0.0f;
            }
        }
        first.above[c] = above;
        first.below[c] = below;
    }
    reads_done();                                                   // the wave's own writes: no other wave looks at `first` or the rows
}

// O^T += V^T P^T over 32 keys in LDS at `buf`, which are this wave's.  A key that a row does not see has a weight of zero, and zero times infinity would still
// be NaN: where rows see different ones of the keys (GUARD, `uneven`; a row sees the first `seen` of the 32), values that are not finite
// stay out of the product, and the rows that see one get it by itself.
template <class T, int D, bool GUARD>
__device__ __forceinline__ void accumulate(unsigned buf, const f32x16& p, int seen, bool uneven, FirstOdd<D>& first, RowState<Head<T, D>>& st) {
    bool odd = false;
    if constexpr (GUARD) {
        odd = uneven && any_odd<T, Head<T, D>::kChunks / 2>(buf);
        if (odd) take_odd<T, D>(buf, first);
    }
#pragma unroll
    for (int d = 0; d < Head<T, D>::kBlocks; ++d) block_product<T, D>(buf, d, p, st.o[d]);
    if (odd) {
        add_odd<T, D>(seen, first, st);
        reads_done();
    }
}

// A row of q, as the B operand of the first product; zeros where there is no row.
template <class T, int D>
__device__ __forceinline__ void load_row(const unsigned char* p, bool there, u32x4 (&q)[Head<T, D>::kSteps]) {
    const int h = (threadIdx.x >> 5) & 1;
#pragma unroll
    for (int c = 0; c < Head<T, D>::kSteps; ++c) {
        if (there) q[c] = *reinterpret_cast<const u32x4*>(p + (2 * c + h) * 16);
        else q[c] = u32x4{0, 0, 0, 0};
    }
}

// ------------------------------------------------------------------------------------------------
// Few rows (decoding): memory-bound.  128 sequences of up to 4096 tokens, 32 and 8 heads of 128 in bfloat16 (1 GB): 169 us with the join, 5.9 TB/s; one block for
// one worker, all latency (length, table, keys, results): 5.4 us.  Every wave works by itself, through LDS slots of its own, without a barrier: V of a block of 32 keys is in flight
// while its scores are formed, K of the next one while V is used.  All (sequence, head) items' blocks form one line that the grid's
// waves share evenly, whatever the sequences' lengths: a wave's share begins and ends anywhere in an item.  Every piece of an item leaves a
// slot of partial results, numbered item + worker (each step along the line raises one of the two), which join_kernel puts together.
// Gang: where a token's rows of neighbouring heads share 128-byte lines, the four waves of a workgroup are one worker that takes four heads' rows, whole lines
// together, at the same time (200 sequences at 16 x 96, rows of 192 bytes one after the other: 537 MB fetched without it, 416 with it, of 406 that there are).

template <class T, int D, bool MULTI, bool STREAM>
struct FewRange {
    using H = Head<T, D>;
    static constexpr int kLoads = H::kChunks / 2;                   // of one wave for 32 rows

    // Where a lane's 16 bytes of each load come from, relative to the cache's start; -1 where there is no key.  `page`: lane i holds the number of the
    // page first + i of the table (-1: none).
    static __device__ __forceinline__ void addresses(int64_t (&off)[kLoads], const AttentionArgs& a, int page, int first, int key0, int end) {
        const int lane = threadIdx.x & 63;
        if (a.page_shift >= 5) {                                    // the 32 keys are in one page
            const int at = __builtin_amdgcn_readlane(page, (key0 >> a.page_shift) - first);
            const uint64_t base = (uint64_t)(unsigned)at * a.page_stride + (unsigned)(key0 & ((1 << a.page_shift) - 1)) * a.token_stride;
#pragma unroll
            for (int i = 0; i < kLoads; ++i) {
                const int r = (i * 64 + lane) / H::kChunks;
                off[i] = at >= 0 && key0 + r < end ? (int64_t)(base + (unsigned)r * a.token_stride) : -1;
            }
        } else {
#pragma unroll
            for (int i = 0; i < kLoads; ++i) {
                const int key = key0 + (i * 64 + lane) / H::kChunks, at = __shfl(page, (key >> a.page_shift) - first);
                off[i] = at >= 0 && key < end ? (int64_t)((uint64_t)(unsigned)at * a.page_stride + (unsigned)(key & ((1 << a.page_shift) - 1)) * a.token_stride) : -1;
            }
        }
    }
    template <bool V, bool PAST>
    static __device__ __forceinline__ void issue(const int64_t (&off)[kLoads], const unsigned char* base, unsigned to) {
        const int lane = threadIdx.x & 63;
#pragma unroll
        for (int i = 0; i < kLoads; ++i) {
            const int r = (i * 64 + lane) / H::kChunks, p = (i * 64 + lane) % H::kChunks;
            const int c = V ? H::v_chunk(r, p) : H::k_chunk(r, p);
            const unsigned char* from = off[i] >= 0 ? base + off[i] + c * 16 : zero_chunk;
            load_to_lds<PAST>(from, to + i * 1024);
        }
    }
    // past: they are read once
    template <bool V>
    static __device__ __forceinline__ void issue(const int64_t (&off)[kLoads], const unsigned char* base, unsigned to, bool past) {
        reads_done();
        if (STREAM && past) issue<V, true>(off, base, to);
        else issue<V, false>(off, base, to);
    }

    // blocks [n0, n1) of `table`'s tokens, of which there are `keys`; limit: how many of them this lane's row sees, all_see: how many every row sees
    static __device__ __forceinline__ void run(const AttentionArgs& a, const int* table, int n0, int n1, int keys, int limit, int all_see, bool past,
                                               const unsigned char* kbase, const unsigned char* vbase, unsigned kbuf,
                                               const u32x4 (&q)[H::kSteps], FirstOdd<D>& odd, RowState<H>& st) {
        const int lane = threadIdx.x & 63;
        const unsigned vbuf = kbuf + 32 * H::kRowBytes;
        const int last = min(n1 * kBlockKeys, keys);
        int key0 = n0 * kBlockKeys;
        while (key0 < last) {
            // 64 pages at a time, one per lane
            const int first = key0 >> a.page_shift, end = min((int64_t)last, (int64_t)(first + 64) << a.page_shift);
            int page = -1;
            const bool listed = ((int64_t)(first + lane) << a.page_shift) < end;
            if (listed) page = table[first + lane];
            if (page >= a.pages) page = -1;
            const bool bad = __any(listed && page < 0);
            int64_t off[kLoads];
            addresses(off, a, page, first, key0, end);
            issue<false>(off, kbase, kbuf, past);
            issue<true>(off, vbase, vbuf, past);
            while (true) {
                const int next = key0 + kBlockKeys;
                const bool more = next < end;
                wait_loads<kLoads>();
                f32x16 s[1] = {scores<T, D>(kbuf, q)};
                if (more) {
                    addresses(off, a, page, first, next, end);
                    issue<false>(off, kbase, kbuf, past);
                }
                if (bad || key0 + kBlockKeys > all_see) {
#pragma unroll
                    for (int i = 0; i < 16; ++i) {
                        const int key = key0 + key_of(i), at = bad ? __shfl(page, (key >> a.page_shift) - first) : 0;
                        s[0][i] = key < limit && at >= 0 ? s[0][i] : WHT_NEG_INF;
                    }
                }
                rebase<H, 0>(largest(s[0]), a.scale, s[0], st);
                weigh(s[0], a.scale, st);
                if (more) wait_loads<kLoads>();
                else wait_loads<0>();
                accumulate<T, D, MULTI>(vbuf, s[0], limit - key0, all_see < min(key0 + kBlockKeys, keys), odd, st);
                key0 = next;
                if (!more) break;
                issue<true>(off, vbase, vbuf, past);
            }
            reads_done();
        }
    }
};

__device__ __forceinline__ int blocks_of(const AttentionArgs& a, const Sequence& s) {
    return s.queries > 0 ? (a.use_prefix ? ceil_div(a.prefix, kBlockKeys) : 0) + ceil_div(s.length, kBlockKeys) : 0;
}
// The line's b-th sequence; the one past the last stands for the front, the rows of all of them.
__device__ __forceinline__ Sequence line_sequence(const AttentionArgs& a, int b) { return b < a.batch.B ? sequence(a.batch, b) : Sequence{0, a.batch.T, 0}; }
__device__ __forceinline__ int line_blocks(const AttentionArgs& a, int b, const Sequence& s) { return b < a.batch.B ? blocks_of(a, s) : ceil_div(a.prefix, kBlockKeys); }

constexpr int kListed = 512;        // pages that a workgroup of the many-rows kernel has in LDS at a time; -1 where a number names none
struct PageList { int page[kListed]; int bad[4], odd[4]; };         // by wave: whether a page was bad, a value not finite

// What a workgroup of either kernel has in LDS.
template <class T, int D>
struct Shared {
    __align__(16) unsigned char buf[256 * Head<T, D>::kRowBytes];   // few rows: 32 keys and values of each wave; many: two steps' 64
    FirstOdd<D> odd[4];             // few rows: of each wave's block; many: of all keys (the first of the four)
    PageList list;
};

// FRONT: the prefix is the launch's other workgroups' work.
template <class T, int D, bool MULTI, bool STREAM, bool FRONT>
__device__ __forceinline__ void few_rows(const AttentionArgs& a, int block, Shared<T, D>& shared) {
    using H = Head<T, D>;
    constexpr int kWaveBytes = 2 * 32 * H::kRowBytes;
    auto& buf = shared.buf;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int B = a.batch.B + a.front_item;

    // Each lane's run of sequences and the runs' prefix sums; every wave does this by itself, so that the chain of loads before the first keys is the
    // shortest there is.  Up to 64 sequences a lane holds one, and they are not looked up again.
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
    // a worker: a wave, or (gang) a workgroup whose waves take four heads side by side
    const int all = __builtin_amdgcn_readlane(upto, 63), groups = a.heads >> a.gang_log2, worker = a.gang_log2 == 0 ? block * 4 + wave : block;
    if (block == 0 && wave == 0) {
        int c = upto - mine;
        for (int b = b0; b < b1; ++b) { a.cum[b] = c; c += line_blocks(a, b, line_sequence(a, b)); }
        if (lane == 0) a.cum[B] = all;
    }
    const int total = all * groups, per = line_share(total, a.rows_cap, a.gang_log2);
    int u = min((int64_t)total, (int64_t)worker * per);
    const int end = min(total, u + per);
    if (u >= end) return;
    const int from = __popcll(__ballot(upto * groups <= u));       // the lane whose run has block u
    int b = from * run, cum = __builtin_amdgcn_readlane(upto - mine, from);

    while (u < end) {
        Sequence s;
        if (run == 1) s = {__builtin_amdgcn_readlane(held.first, b), __builtin_amdgcn_readlane(held.queries, b), __builtin_amdgcn_readlane(held.length, b)};
        else s = line_sequence(a, b);
        const int n = line_blocks(a, b, s);
        if (u >= (cum + n) * groups) { cum += n; ++b; continue; }
        const int within = u - cum * groups, group = within / n, n0 = within - group * n, n1 = min(n, n0 + (end - u));
        const int in_gang = a.gang_log2 == 0 ? 0 : wave, head = (group << a.gang_log2) + in_gang;
        const bool stacked = b >= a.batch.B;
        const int rows = min(s.queries * a.G, a.rows_cap), row = lane & 31;
        const int token = row / a.G, qh = head * a.G + row % a.G;
        u32x4 q[H::kSteps];
        load_row<T, D>(a.q + (s.first + token) * a.q_ts + qh * a.q_hs, row < rows, q);
        RowState<H> st;
        st.clear();
        const unsigned char *kbase = a.k + head * a.head_stride, *vbase = a.v + head * a.head_stride;
        const unsigned own = __builtin_amdgcn_readfirstlane(lds_address(buf)) + wave * kWaveBytes;
        FirstOdd<D>& first = shared.odd[wave];
        const int front = a.use_prefix || stacked ? ceil_div(a.prefix, kBlockKeys) : 0;
        const int limit = min(max(s.length - s.queries + token + 1, 0), s.length), all_see = min(max(s.length - s.queries + 1, 0), s.length);
        const int keys = min(max(s.length - s.queries + min(s.queries, a.max_q), 0), s.length);           // what the last of the rows sees
#pragma unroll 1
        for (int part = FRONT ? 1 : 0; part < 2; ++part) {          // the prefix, the sequence
            const int lo = part ? max(n0 - front, 0) : n0, hi = part ? n1 - front : min(n1, front);
            if (lo >= hi) continue;
            FewRange<T, D, MULTI, STREAM>::run(a, part ? a.batch.table + b * a.batch.table_stride : a.prefix_table, lo, hi, part ? keys : a.prefix, part ? limit : a.prefix,
                                       part ? all_see : a.prefix, FRONT || part || a.batch.B == 1, kbase, vbase, own, q, first, st);
        }
        st.l += other_half(st.l);
        if (row < rows) {
            const int64_t at = (((int64_t)(b * groups + group + worker) << a.gang_log2) + in_gang) * a.rows_cap + row;
            if (lane < 32) *reinterpret_cast<f32x2*>(a.sums + at * 2) = f32x2{st.top * a.scale, st.l};
#pragma unroll
            for (int d = 0; d < H::kBlocks; ++d)
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    *reinterpret_cast<f32x4*>(a.part + at * D + d * 32 + i * 8 + (lane >> 5) * 4) = f32x4{st.o[d][4 * i], st.o[d][4 * i + 1], st.o[d][4 * i + 2], st.o[d][4 * i + 3]};
        }
        u += n1 - n0;
    }
}

// ------------------------------------------------------------------------------------------------
// Many rows: a workgroup takes 128 rows, 32 per wave, and all its waves the same 64 keys a step; keys and values lie in LDS twice over, the
// next steps' in flight.  A wave takes 32 keys at a time, as a pipeline: the products with the next 32 keys stand beside the exponentials of
// these, those with their values beside the next ones' maximum, and every fragment is read from LDS as many products ahead as there are in one of the two,
// into the registers of the one just used.  Per 32 keys 128 wide: 16 matrix instructions of 32 cycles, 60 vector instructions of 4 and 16 exponentials of 16.
// Two prompts of 4096 tokens, 32 and 8 heads of 128: 300 us, 916 TFLOP/s (a library product of 8192 x 8192 x 8192 here: 1215).  What bounds it is no one
// of its parts: 8 x 128 tokens behind 16256 keys, 32 heads, take 327 us; without the loads into LDS 258, without the reads from it 237, without either
// 185, without the products 209, without the exponentials 294.  A second workgroup on a compute unit gains 8 %.

// The keys of one item: the prefix's first, then the sequence's.  Steps of 64 keys count through both (front: the first of the sequence's), so that a step's
// keys are of one of them.
struct Keys {
    const int *prefix_table, *own_table;
    int front, prefix, own;             // own: of the sequence, those that any row of the workgroup sees
};

template <class T, int D>
struct ManyRange {
    using H = Head<T, D>;
    static constexpr int kLoads = H::kChunks / 4;                   // of one wave for a quarter of 64 rows
    static constexpr int kTileBytes = kStepKeys * H::kRowBytes;

    // steps [lo, hi), whose pages fit the list; limit: how many of the sequence's keys this lane's row sees, all_see, any_sees: every, any row of the wave
    // (-1: it has none), level: how many every row of the workgroup sees.  LDS: keys of even, of odd steps, values of even, of odd steps.
    static __device__ __forceinline__ void stream(const AttentionArgs& a, const Keys& k, PageList& list, int lo, int hi, int limit, int all_see, int any_sees, int level,
                                                  const unsigned char* kbase, const unsigned char* vbase, unsigned buf, const u32x4 (&q)[H::kSteps], FirstOdd<D>& odd,
                                                  RowState<H>& st) {
        const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), shift = a.page_shift;
        // the list: pages of the prefix's keys in these steps, then of the sequence's; a key's page is at (key >> shift) + the part's offset
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
        const unsigned to = buf + wave * kLoads * 1024;
        unsigned koff[kLoads], voff[kLoads];
#pragma unroll
        for (int i = 0; i < kLoads; ++i) {
            const int n = (wave * kLoads + i) * 64 + lane, r = n / H::kChunks, p = n % H::kChunks;
            koff[i] = (unsigned)(r - wave * 16) * a.token_stride + H::k_chunk(r, p) * 16;
            voff[i] = (unsigned)(r - wave * 16) * a.token_stride + H::v_chunk(r, p) * 16;
        }
        __syncthreads();
        const bool bad = __builtin_amdgcn_readfirstlane(list.bad[0] | list.bad[1] | list.bad[2] | list.bad[3]) != 0;

        // Loads of a step.  Where its keys are all there, in pages of 16 tokens at least, a wave's 16 of the 64 are in one page, and a lane's place in
        // it is the same every step.
        auto load = [&](int t, const unsigned char* base, const unsigned (&off)[kLoads], unsigned at) {
            const bool own = t >= k.front;
            const int key0 = (own ? t - k.front : t) * kStepKeys, keys = own ? k.own : k.prefix, list_at = own ? own_at : pre_at;
            if (!bad && shift >= 4 && key0 + kStepKeys <= keys) {
                const int key = key0 + wave * 16, page = __builtin_amdgcn_readfirstlane(list.page[(key >> shift) + list_at]);
                const unsigned char* from = base + ((uint64_t)(unsigned)page * a.page_stride + (unsigned)(key & ((1 << shift) - 1)) * a.token_stride);
#pragma unroll
                for (int i = 0; i < kLoads; ++i) load_to_lds(from, off[i], at + i * 1024);
            } else {
#pragma unroll
                for (int i = 0; i < kLoads; ++i) {
                    const int r = ((wave * kLoads + i) * 64 + lane) / H::kChunks, key = key0 + r;
                    const int page = key < keys ? list.page[(key >> shift) + list_at] : -1;
                    const uint64_t from = (uint64_t)(unsigned)page * a.page_stride + (unsigned)(key & ((1 << shift) - 1)) * a.token_stride;
                    load_to_lds<false>(page >= 0 ? base + from + (off[i] - (unsigned)(r - wave * 16) * a.token_stride) : zero_chunk, at + i * 1024);
                }
            }
        };
        auto load_k = [&](int t) { load(t, kbase, koff, to + (t & 1) * kTileBytes); };
        auto load_v = [&](int t) { load(t, vbase, voff, to + (2 + (t & 1)) * kTileBytes); };
        // the first or second 32 keys or values of step t
        auto keys_at = [&](int t, int half) { return fresh(buf + (t & 1) * kTileBytes + half * 32 * H::kRowBytes); };
        auto values_at = [&](int t, int half) { return fresh(buf + (2 + (t & 1)) * kTileBytes + half * 32 * H::kRowBytes); };

        // Blocks of 32 keys count as steps do.  What all rows of the wave see all of; the scores of what they do not, hidden.
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

        // From this step on rows of the workgroup see different keys, and a key that a row does not see has a weight of zero, but zero times infinity is NaN: values
        // that are not finite are taken out of LDS by the wave that loaded them, and given to the rows that see them at the end.
        const int uneven = k.front + level / kStepKeys;
        auto clean_values = [&](int t) {
            const unsigned at = to + (2 + (t & 1)) * kTileBytes;
            if (!any_odd<T, kLoads>(at)) return;
            list.odd[wave] = 1;
#pragma unroll 1
            for (int n = lane; n < kLoads * 64; n += 64) {
                const int r = (wave * kLoads * 64 + n) / H::kChunks, c = H::v_chunk(r, (wave * kLoads * 64 + n) % H::kChunks);
#pragma unroll 1
                for (int e = 0; e < 16 / (int)sizeof(T); ++e) {
                    auto* p = (__attribute__((address_space(3))) T*)(uintptr_t)(at + n * 16 + e * sizeof(T));
                    const float v = (float)*p;
                    if (fabsf(v) < __builtin_inff()) continue;
                    const int col = c * (16 / (int)sizeof(T)) + e, key = (t - k.front) * kStepKeys + r;
                    if (v != WHT_NEG_INF) atomicMin(&odd.above[col], key);
                    if (v != -WHT_NEG_INF) atomicMin(&odd.below[col], key);
                    *p = (T)0.0f;
                }
            }
        };

        u32x4 frag[H::kSteps];                                      // keys of the block after the one whose scores are at hand
        auto read_keys = [&](unsigned at) {
            const unsigned first_chunk = KeyReads<T, D>::first(at);
#pragma unroll
            for (int i = 0; i < H::kSteps; ++i) frag[i] = lds_read<u32x4>(KeyReads<T, D>::chunk(first_chunk, i));
        };
        // The weights of `s` and their products with the values at `vat`; the scores `ahead` of the keys in `frag`, which becomes those at `kat`.  Where there are no
        // more keys, these are what lies there, and not used.
        auto full_block = [&](f32x16& s, f32x16& ahead, unsigned vat, unsigned kat, bool more) {
            if constexpr (!H::kF32) {
                const unsigned first_chunk = KeyReads<T, D>::first(kat);
                bf16x8 w[2];
                float sum[2] = {0.0f, 0.0f};
                ahead = f32x16{};
#pragma unroll
                for (int i = 0; i < H::kSteps; ++i) {
                    ahead = score_step<T>(frag[i], q[i], ahead);
                    frag[i] = __builtin_bit_cast(u32x4, values<D>(vat, i / H::kBlocks, i % H::kBlocks));
#pragma unroll
                    for (int e = 16 * i / H::kSteps; e < 16 * (i + 1) / H::kSteps; ++e) {
                        const float p = __builtin_amdgcn_exp2f(__builtin_fmaf(s[e], a.scale, -st.base));
                        sum[e & 1] += p;
                        w[e >> 3][e & 7] = (bf16)p;
                    }
                    __builtin_amdgcn_sched_barrier(0);
                }
                float mx = WHT_NEG_INF;
#pragma unroll
                for (int i = 0; i < H::kSteps; ++i) {
                    st.o[i % H::kBlocks] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, frag[i]), w[i / H::kBlocks], st.o[i % H::kBlocks], 0, 0, 0);
                    frag[i] = lds_read<u32x4>(KeyReads<T, D>::chunk(first_chunk, i));
                    // the last of `ahead` is a few instructions old
                    if (i >= H::kSteps / 2)
#pragma unroll
                        for (int e = 16 * (2 * i - H::kSteps) / H::kSteps; e < 16 * (2 * i - H::kSteps + 2) / H::kSteps; ++e) mx = fmaxf(mx, ahead[e]);
                    __builtin_amdgcn_sched_barrier(0);
                }
                st.l += sum[0] + sum[1];
                if (more) rebase<H, 8>(mx, a.scale, ahead, st);
            } else {
                ahead = f32x16{};
#pragma unroll
                for (int i = 0; i < H::kSteps; ++i) ahead = score_step<T>(frag[i], q[i], ahead);
                weigh(s, a.scale, st);
                accumulate<T, D, false>(vat, s, 0, false, odd, st);
                read_keys(kat);
                if (more) rebase<H, 8>(largest(ahead), a.scale, ahead, st);
            }
        };
        load_k(lo);
        load_v(lo);
        if (lo + 1 < hi) load_k(lo + 1);
        wait_loads<0>();
        workgroup_barrier();
        f32x16 s = scores<T, D>(keys_at(lo, 0), q), other;
        if (bad || !full(2 * lo)) hide(s, 2 * lo);
        rebase<H, 8>(largest(s), a.scale, s, st);
        read_keys(keys_at(lo, 1));
        // A step's barrier stands in both loops below: a wave takes a step in either, whatever the others do.
        for (int t = lo; t < hi; ++t) {
            // steps whose blocks, and the first of the next one, are seen by all rows of the wave
            const int blocks = 2 * t >= front || pre_full == front ? front + own_full : pre_full;
            for (const int end = bad ? t : min(uneven, blocks >= 2 * hi ? hi : min(hi - 1, (blocks - 1) / 2)); t < end; ++t) {
                wait_loads<0>();
                workgroup_barrier();                                // V of this step and K of the next have landed; what they replace next has been read
                if (t + 1 < hi) load_v(t + 1);
                if (t + 2 < hi) load_k(t + 2);
                full_block(s, other, values_at(t, 0), keys_at(t + 1, 0), true);
                full_block(other, s, values_at(t, 1), keys_at(t + 1, 1), t + 1 < hi);
            }
            if (t == hi) break;
            wait_loads<0>();
            if (t >= uneven) clean_values(t);
            workgroup_barrier();
            if (t + 1 < hi) load_v(t + 1);
            if (t + 2 < hi) load_k(t + 2);
#pragma unroll 1
            for (int half = 0; half < 2; ++half) {
                const int j = 2 * t + half;
                if (!in_sight(j)) break;                            // nor is any that follows
                const bool more = j + 1 < 2 * hi && in_sight(j + 1);
                if (more) {
                    other = f32x16{};
#pragma unroll
                    for (int i = 0; i < H::kSteps; ++i) other = score_step<T>(frag[i], q[i], other);
                }
                weigh(s, a.scale, st);
                const unsigned values = values_at(t, half);
#pragma unroll
                for (int d = 0; d < H::kBlocks; ++d) {
                    block_product<T, D>(values, d, s, st.o[d]);
                    asm volatile("" ::: "memory");                  // one block's values in registers at a time
                }
                if (more) {
                    if (t + 1 < hi) read_keys(keys_at(t + 1, half));
                    if (bad || !full(j + 1)) hide(other, j + 1);
                    rebase<H, 8>(largest(other), a.scale, other, st);
                    s = other;
                }
            }
        }
    }

    static __device__ __forceinline__ void run(const AttentionArgs& a, const Keys& k, PageList& list, int t0, int t1, int limit, int all_see, int any_sees, int level,
                                               const unsigned char* kbase, const unsigned char* vbase, unsigned buf, const u32x4 (&q)[H::kSteps], FirstOdd<D>& odd,
                                               RowState<H>& st) {
        for (int c = threadIdx.x; c < D; c += 256) odd.above[c] = odd.below[c] = INT_MAX;
        if (threadIdx.x < 4) list.odd[threadIdx.x] = 0;
        const int per_list = max(((kListed - 4) << a.page_shift) / kStepKeys, 1);           // each part may begin and end within a page
        for (int lo = t0; lo < t1; lo += per_list) {
            if (lo > t0) workgroup_barrier();                       // the last steps' reads are done
            stream(a, k, list, lo, min(t1, lo + per_list), limit, all_see, any_sees, level, kbase, vbase, buf, q, odd, st);
        }
        workgroup_barrier();
        if ((list.odd[0] | list.odd[1] | list.odd[2] | list.odd[3]) != 0) add_odd<T, D>(limit, odd, st);
    }
};

template <class T>
__device__ __forceinline__ void store4(unsigned char* p, f32x4 x) {
    if constexpr (sizeof(T) == 4) *reinterpret_cast<f32x4*>(p) = x;
    else {
        bf16x4 y;
#pragma unroll
        for (int i = 0; i < 4; ++i) y[i] = (bf16)x[i];
        *reinterpret_cast<bf16x4*>(p) = y;
    }
}

// Rows that no tile covers: padding (zeros) and tokens from the max_q-th of their sequence on (NaN).  A workgroup of each die takes a share.
template <class T, int D>
__device__ __forceinline__ void fill_rows(const AttentionArgs& a, int die) {
    auto fill = [&](int lo, int hi, float value, float lse) {
        const int64_t n = (int64_t)(hi - lo) * a.q_heads * (D / 4);
        for (int64_t i = threadIdx.x; i < n; i += 256) {
            const int64_t row = i / (D / 4);
            const int64_t t = lo + row / a.q_heads, h = row % a.q_heads;
            store4<T>(a.out + t * a.out_ts + h * a.out_hs + (i % (D / 4)) * 4 * sizeof(T), f32x4{value, value, value, value});
            if (a.lse && i % (D / 4) == 0) a.lse[t * a.q_heads + h] = lse;
        }
    };
    for (int b = die; b < a.batch.B; b += kDies) {
        const Sequence s = sequence(a.batch, b);
        if (s.queries > a.max_q) fill(s.first + a.max_q, s.first + s.queries, __builtin_nanf(""), __builtin_nanf(""));
    }
    const int last = min(max(a.batch.q_starts ? a.batch.q_starts[a.batch.B] : a.batch.B, 0), a.batch.T);
    const int left = a.batch.T - last;
    fill(last + (int)((int64_t)left * die / kDies), last + (int)((int64_t)left * (die + 1) / kDies), 0.0f, WHT_NEG_INF);
}

// STACKED: the rows of all sequences, against the prefix alone.
template <class T, int D, bool STACKED>
__device__ __forceinline__ void many_rows(const AttentionArgs& a, int block, Shared<T, D>& shared) {
    using H = Head<T, D>;
    using R = ManyRange<T, D>;
    auto& buf = shared.buf;
    auto& list = shared.list;
    auto& odd = shared.odd;
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
        // Which tile: the line of the die's groups' tiles, looked up as the few-rows kernel looks up its own line.
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
    const int group = die_group(b, groups, x, k), split = group % a.splits, head = group / a.splits;
    const int64_t rows = (int64_t)queries * a.G;
    const int row0 = tile * kTileRows + wave * 32, row = row0 + (lane & 31);
    const int token = row / a.G, qh = head * a.G + row % a.G;
    const bool there = row < rows;
    u32x4 q[H::kSteps];
    load_row<T, D>(a.q + (s.first + (there ? token : 0)) * a.q_ts + qh * a.q_hs, there, q);
    // own tokens that row r of the tile sees: length - queries + its token + 1
    auto sees = [&](int64_t r) { return STACKED ? 0 : min(max(s.length - s.queries + (int)(min(r, rows - 1) / a.G) + 1, 0), s.length); };
    const int keys = sees(tile * kTileRows + kTileRows - 1);
    const int limit = sees(row), all_see = sees(row0), any_sees = row0 < rows ? sees(row0 + 31) : -1;
    const int front = a.use_prefix ? ceil_div(a.prefix, kStepKeys) : 0;
    const int total = front + ceil_div(keys, kStepKeys), per = ceil_div(total, a.splits);
    const int t0 = min(total, split * per), t1 = min(total, t0 + per);
    RowState<H> st;
    st.clear();
    const unsigned char *kbase = a.k + head * a.head_stride, *vbase = a.v + head * a.head_stride;
    const Keys keys_of{a.prefix_table, a.batch.table + b * a.batch.table_stride, front, a.use_prefix ? a.prefix : 0, keys};
    R::run(a, keys_of, list, t0, t1, limit, all_see, any_sees, sees((int64_t)tile * kTileRows), kbase, vbase, __builtin_amdgcn_readfirstlane(lds_address(buf)), q, odd[0], st);
    if (!there) return;
    st.l += other_half(st.l);
    const int64_t t = s.first + token;
    if (a.splits > 1 || STACKED) {
        const int64_t at = ((int64_t)split * a.batch.T + t) * a.q_heads + qh;
        if (lane < 32) { a.sums[at * 2] = st.top * a.scale; a.sums[at * 2 + 1] = st.l; }
#pragma unroll
        for (int d = 0; d < H::kBlocks; ++d)
#pragma unroll
            for (int i = 0; i < 4; ++i)
                *reinterpret_cast<f32x4*>(a.part + at * D + d * 32 + i * 8 + (lane >> 5) * 4) = f32x4{st.o[d][4 * i], st.o[d][4 * i + 1], st.o[d][4 * i + 2], st.o[d][4 * i + 3]};
    } else {
        const float inv = st.l == 0.0f ? 0.0f : 1.0f / st.l;
        if (a.lse && lane < 32) a.lse[t * a.q_heads + qh] = st.l == 0.0f ? WHT_NEG_INF : (st.top * a.scale + __builtin_amdgcn_logf(st.l)) * kLn2;
#pragma unroll
        for (int d = 0; d < H::kBlocks; ++d)
#pragma unroll
            for (int i = 0; i < 4; ++i)
                store4<T>(a.out + t * a.out_ts + qh * a.out_hs + (d * 32 + i * 8 + (lane >> 5) * 4) * sizeof(T),
                          f32x4{st.o[d][4 * i] * inv, st.o[d][4 * i + 1] * inv, st.o[d][4 * i + 2] * inv, st.o[d][4 * i + 3] * inv});
    }
}

// ------------------------------------------------------------------------------------------------
// The kernels.  Where rows of all sequences meet the prefix (compute-bound) and each sequence's few rows its own keys (memory-bound), one launch does
// both, so that a compute unit may hold a workgroup of each (where the first kind's leave room: AttentionPlan).

template <class T, int D>
__global__ __launch_bounds__(256, (sizeof(T) == 2 ? 2 : 1)) void many_rows_kernel(AttentionArgs a) {
    __shared__ Shared<T, D> shared;
    many_rows<T, D, false>(a, blockIdx.x, shared);
}

template <class T, int D, bool MULTI, bool FRONT, bool STREAM>
__global__ __launch_bounds__(256, (sizeof(T) == 2 ? 2 : 1)) void few_rows_kernel(AttentionArgs a, AttentionArgs front, int front_blocks) {
    __shared__ Shared<T, D> shared;
    if constexpr (FRONT) {
        const int block = blockIdx.x;
        if (block < front_blocks) many_rows<T, D, true>(front, block, shared);
        else few_rows<T, D, MULTI, STREAM, true>(a, block - front_blocks, shared);
    } else few_rows<T, D, MULTI, STREAM, false>(a, blockIdx.x, shared);
}

// ------------------------------------------------------------------------------------------------
// Joins the partial results of a row, in a chain of dependent loads (where its pieces are, the pieces): 4 us where there are few, 8 us for 3584 rows of 15 pieces.
// out = sum_p 2^(m_p - M) o_p / sum_p 2^(m_p - M) l_p.  WAVES waves share a row's pieces; D / 4 lanes take a
// piece's outputs, 16 bytes each, so that a wave reads two pieces (four of 64 wide) at a time.

struct JoinArgs {
    Batch batch;
    unsigned char* out;
    float* lse;
    const float *front_part, *front_sums, *own_part, *own_sums;
    const int* cum;
    int64_t out_ts, out_hs;
    int q_heads, heads, G, max_q, prefix, gang_log2;
    int front, front_few, front_splits;                 // front: there is one
    int own_few, own_splits, own_cap, own_prefix;       // own_prefix: the own range begins with the prefix
};

struct Parts { const float *part, *sums; int64_t at, step; int n; };        // rows at, at + step, ...

// The pieces that the few-rows kernel left of the line's b-th sequence, n blocks long, and a head; total: blocks of all sequences.
template <int WORKERS>
__device__ __forceinline__ Parts slots(const JoinArgs& a, int b, int head, int n, int total, int row) {
    const int groups = a.heads >> a.gang_log2, group = head >> a.gang_log2;
    const Slots p = item_slots<WORKERS>(b * groups + group, a.cum[b] * groups + group * n, n, total * groups, a.own_cap, a.gang_log2);
    return {a.own_part, a.own_sums, ((p.first << a.gang_log2) + (head - (group << a.gang_log2))) * a.own_cap + row, (int64_t)a.own_cap << a.gang_log2, p.count};
}

// H (of 32) / 8 of a row's outputs, four to a lane.
__device__ __forceinline__ f32x4 transform_outputs(f32x4 x) {
    x = f32x4{x[0] + x[1], x[0] - x[1], x[2] + x[3], x[2] - x[3]};
    x = f32x4{x[0] + x[2], x[1] + x[3], x[0] - x[2], x[1] - x[3]};
#pragma unroll
    for (int h = 1; h < 8; h <<= 1)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const float other = __shfl_xor(x[i], h);
            x[i] = threadIdx.x & h ? other - x[i] : x[i] + other;
        }
    return x * 0.125f;
}

// TRANSFORM: of the cache in 4 bits, whose values may be transformed.
template <class T, int D, int WAVES, bool TRANSFORM = false, int WORKERS = kWorkers>
__global__ __launch_bounds__(WAVES == 1 ? 256 : 64 * WAVES) void join_kernel(JoinArgs a) {
    constexpr int kLanes = D / 4, kAtOnce = 64 / kLanes, kUnroll = 4;
    struct Share { float m, l; f32x4 o[kLanes]; };
    __shared__ Share shares[WAVES];
    const int lane = threadIdx.x & 63, wave = WAVES == 1 ? 0 : __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int64_t r = WAVES == 1 ? (int64_t)block_of() * 4 + (threadIdx.x >> 6) : blockIdx.x;
    if (r >= (int64_t)a.batch.T * a.q_heads) return;
    const int t = (int)(r / a.q_heads), qh = (int)(r % a.q_heads), head = qh / a.G, g = qh % a.G;
    const int b = __builtin_amdgcn_readfirstlane(sequence_of(a.batch, t));
    float value = 0.0f, m = WHT_NEG_INF, l = 0.0f;
    f32x4 o = {0.0f, 0.0f, 0.0f, 0.0f};
    const int group = lane / kLanes, col = (lane % kLanes) * 4;
    auto add = [&](const Parts& p) {
        // the wave takes every WAVES-th run of 64 pieces, or an even share where there are fewer
        const int run = min(64, ceil_div(p.n, WAVES));
        for (int lo = wave * run; lo < p.n; lo += WAVES * run) {
            const int n = min(run, p.n - lo);
            f32x4 x[kUnroll];
            auto fetch = [&](int i) {
#pragma unroll
                for (int e = 0; e < kUnroll; ++e) {
                    const int at = i + e * kAtOnce + group;
                    const bool there = group < kAtOnce && at < n;
                    x[e] = there ? *reinterpret_cast<const f32x4*>(p.part + (p.at + (lo + at) * p.step) * D + col) : f32x4{0.0f, 0.0f, 0.0f, 0.0f};
                }
            };
            fetch(0);                                               // with the sums: what they weigh is known when both are there
            float pm = WHT_NEG_INF, pl = 0.0f;
            if (lane < n) {
                const f32x2 y = *reinterpret_cast<const f32x2*>(p.sums + (p.at + (lo + lane) * p.step) * 2);
                pm = y[0];
                pl = y[1];
            }
            float most = pm;
#pragma unroll
            for (int d = 1; d < 64; d <<= 1) most = fmaxf(most, __shfl_xor(most, d));
            const float now = fmaxf(m, most), base = now == WHT_NEG_INF ? 0.0f : now;
            const float f = __builtin_amdgcn_exp2f(m - base), w = __builtin_amdgcn_exp2f(pm - base);
            float sum = pl * w;
#pragma unroll
            for (int d = 1; d < 64; d <<= 1) sum += __shfl_xor(sum, d);
            l = l * f + sum;
            o *= f;
            m = now;
            for (int i = 0; i < n; i += kAtOnce * kUnroll) {
                if (i > 0) fetch(i);
#pragma unroll
                for (int e = 0; e < kUnroll; ++e) {
                    const int at = i + e * kAtOnce + group;
                    o += __shfl(w, min(at, n - 1)) * x[e];
                }
            }
        }
    };
    // shares of the prefix stand in the same places for every row: they are on their way while the row's sequence is looked up
    if (a.front && !a.front_few) add({a.front_part, a.front_sums, r, (int64_t)a.batch.T * a.q_heads, a.front_splits});
    const bool empty = b < 0;
    if (b >= 0) {
        const Sequence s = sequence(a.batch, b);
        const int j = t - s.first;
        if (j < 0 || j >= s.queries || j >= a.max_q) value = __builtin_nanf("");
        else {
            const int total = a.cum[a.batch.B + (a.front && a.front_few)];
            if (a.front && a.front_few) add(slots<WORKERS>(a, a.batch.B, head, ceil_div(a.prefix, kBlockKeys), total, t * a.G + g));
            add(slots<WORKERS>(a, b, head, (a.own_prefix ? ceil_div(a.prefix, kBlockKeys) : 0) + ceil_div(s.length, kBlockKeys), total, j * a.G + g));
        }
    }
    const f32x4 mine = o;
#pragma unroll
    for (int e = 1; e < kAtOnce; ++e)
#pragma unroll
        for (int i = 0; i < 4; ++i) o[i] += __shfl(mine[i], lane + e * kLanes);              // the first group's lanes hold the sum
    if constexpr (WAVES > 1) {
        if (lane < kLanes) shares[wave].o[lane] = o;
        if (lane == 0) { shares[wave].m = m; shares[wave].l = l; }
        __syncthreads();
        if (wave > 0) return;
        m = WHT_NEG_INF;
        for (int w = 0; w < WAVES; ++w) m = fmaxf(m, shares[w].m);
        const float base = m == WHT_NEG_INF ? 0.0f : m;
        l = 0.0f;
        o = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
        for (int w = 0; w < WAVES; ++w) {
            const float f = __builtin_amdgcn_exp2f(shares[w].m - base);
            l += shares[w].l * f;
            o += f * shares[w].o[lane % kLanes];
        }
    }
    if (empty) { l = 0.0f; m = WHT_NEG_INF; o = f32x4{0.0f, 0.0f, 0.0f, 0.0f}; }              // padding
    if (value != 0.0f) l = value;
    const float inv = l == 0.0f ? 0.0f : 1.0f / l;
    if constexpr (TRANSFORM) o = transform_outputs(o);
    if (lane < kLanes) store4<T>(a.out + t * a.out_ts + qh * a.out_hs + lane * 4 * sizeof(T), value != 0.0f ? f32x4{value, value, value, value} : o * inv);
    if (a.lse && lane == 0) a.lse[r] = l == 0.0f ? WHT_NEG_INF : (m + __builtin_amdgcn_logf(l)) * kLn2;
}

// The same where every row has its pieces at the same places: the shares that a tile's keys were split into.  D / 4 lanes take a row, so that a wave has two
// or more; which row it is matters only for what is written, and is looked up beside the loads.
template <class T, int D, bool TRANSFORM = false>
__global__ __launch_bounds__(256) void join_splits_kernel(JoinArgs a) {
    constexpr int kLanes = D / 4, kRows = 256 / kLanes, kUnroll = 4;
    const int64_t rows = (int64_t)a.batch.T * a.q_heads, r = (int64_t)blockIdx.x * kRows + threadIdx.x / kLanes;
    const int t0 = (int)min((int64_t)blockIdx.x * kRows / a.q_heads, (int64_t)a.batch.T - 1);       // sequence_of takes a whole wave
    const bool there = threadIdx.x < kRows * kLanes && r < rows;
    const int64_t at = there ? r : 0;
    const int col = threadIdx.x % kLanes * 4, t = (int)(at / a.q_heads);
    float m = WHT_NEG_INF, l = 0.0f;
    f32x4 o = {0.0f, 0.0f, 0.0f, 0.0f};
    for (int lo = 0; lo < a.own_splits; lo += kUnroll) {
        f32x2 ml[kUnroll];
        f32x4 x[kUnroll];
#pragma unroll
        for (int e = 0; e < kUnroll; ++e) {
            const int64_t p = at + min(lo + e, a.own_splits - 1) * rows;
            ml[e] = *reinterpret_cast<const f32x2*>(a.own_sums + p * 2);
            x[e] = *reinterpret_cast<const f32x4*>(a.own_part + p * D + col);
            if (lo + e >= a.own_splits) ml[e] = f32x2{WHT_NEG_INF, 0.0f};
        }
        float now = m;
#pragma unroll
        for (int e = 0; e < kUnroll; ++e) now = fmaxf(now, ml[e][0]);
        const float base = now == WHT_NEG_INF ? 0.0f : now, f = __builtin_amdgcn_exp2f(m - base);
        l *= f;
        o *= f;
        m = now;
#pragma unroll
        for (int e = 0; e < kUnroll; ++e) {
            const float w = __builtin_amdgcn_exp2f(ml[e][0] - base);
            l += ml[e][1] * w;
            if (lo + e < a.own_splits) o += w * x[e];
        }
    }
    int b = sequence_of(a.batch, t0);                               // of the block's first row; the others' is that or one soon after
    if constexpr (TRANSFORM) o = transform_outputs(o);
    if (!there) return;
    float value = 0.0f;
    while (b >= 0 && b < a.batch.B) {
        const Sequence s = sequence(a.batch, b);
        if (t < s.first + s.queries) {
            if (t < s.first || t - s.first >= a.max_q) value = l = __builtin_nanf("");
            break;
        }
        ++b;
    }
    if (b < 0 || b >= a.batch.B) { l = 0.0f; o = f32x4{0.0f, 0.0f, 0.0f, 0.0f}; m = WHT_NEG_INF; }      // padding: no workgroup wrote its pieces
    const float inv = l == 0.0f ? 0.0f : 1.0f / l;
    store4<T>(a.out + t * a.out_ts + (r % a.q_heads) * a.out_hs + col * sizeof(T), value == 0.0f ? o * inv : f32x4{value, value, value, value});
    if (a.lse && col == 0) a.lse[r] = l == 0.0f ? WHT_NEG_INF : (m + __builtin_amdgcn_logf(l)) * kLn2;
}

}  // namespace wht
