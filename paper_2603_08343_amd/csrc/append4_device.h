// Append to the cache in 4 bits (include/wht_attention4.h) for gfx950.
#pragma once
#include "rotary_device.h"

namespace wht {


// A scale byte as the number that the conversions take: they look at its exponent, and a NaN makes NaN of every code.
__device__ __forceinline__ float scale_of(unsigned byte) { return __uint_as_float(byte >= 253 ? 0x7fc00000u : byte << 23); }

// The eight numbers of a word of codes; exact in bfloat16.
__device__ __forceinline__ bf16x8 decode(unsigned codes, float scale) {
    const bf16x2 a = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, 0), b = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, 1);
    const bf16x2 c = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, 2), d = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, 3);
    return bf16x8{a[0], a[1], b[0], b[1], c[0], c[1], d[0], d[1]};
}

// The value that the lane 1 (2) away holds, of four.
template <int X>
__device__ __forceinline__ unsigned near_lane(unsigned x) {
    constexpr int kPermutation = X == 1 ? 0xB1 : 0x4E;              // quad_perm 1 0 3 2, 2 3 0 1
    return (unsigned)__builtin_amdgcn_update_dpp(0, (int)x, kPermutation, 0xF, 0xF, true);
}
template <int X> __device__ __forceinline__ float near_lane(float x) { return __uint_as_float(near_lane<X>(__float_as_uint(x))); }
template <int X>
__device__ __forceinline__ uint64_t near_lane(uint64_t x) {
    return (uint64_t)near_lane<X>((unsigned)(x >> 32)) << 32 | near_lane<X>((unsigned)x);
}
template <int X> __device__ __forceinline__ double near_lane(double x) { return __builtin_bit_cast(double, near_lane<X>(__builtin_bit_cast(uint64_t, x))); }

__device__ __forceinline__ float flip(float x, unsigned sign) { return __uint_as_float(__float_as_uint(x) ^ sign); }
__device__ __forceinline__ double flip(double x, unsigned sign) { return __builtin_bit_cast(double, __builtin_bit_cast(uint64_t, x) ^ (uint64_t)sign << 32); }

// Walsh-Hadamard transform of the 32 numbers that four lanes hold, eight each: three steps in registers, two between lanes (the neighbour's number and
// one's own, with the sign that the lane's place gives it).
template <class F>
__device__ __forceinline__ void transform32(F (&x)[8]) {
#pragma unroll
    for (int h = 1; h < 8; h *= 2)
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (!(i & h)) {
                const F a = x[i], b = x[i + h];
                x[i] = a + b;
                x[i + h] = a - b;
            }
    const unsigned odd1 = threadIdx.x << 31, odd2 = (threadIdx.x & 2) << 30;
#pragma unroll
    for (int i = 0; i < 8; ++i) x[i] = near_lane<1>(x[i]) + flip(x[i], odd1);
#pragma unroll
    for (int i = 0; i < 8; ++i) x[i] = near_lane<2>(x[i]) + flip(x[i], odd2);
}

// Codes of eight of a block's 32 numbers times 2^power, and the block's scale byte.  The numbers are in 64 bits: a code is decided by which side of a border a
// number is on, and what a sum in 32 bits is off by would now and then decide it.  Their upper 20 bits, with one more that stands for any lower ones, leave
// every border where it is; as float32 numbers, in units of the scale, they go to the nearest code as the hardware does it.
__device__ __forceinline__ unsigned encode(const double (&x)[8], int power, unsigned& scale) {
    constexpr unsigned kMagnitude = 0x7fffffffu;
    double most = __builtin_fabs(x[0]);
    unsigned top = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        most = __builtin_fmax(most, __builtin_fabs(x[i]));
        top = max(top, (unsigned)(__builtin_bit_cast(uint64_t, x[i]) >> 32) & kMagnitude);          // a NaN, which the maximum passes over
    }
    most = __builtin_fmax(most, near_lane<1>(most));
    most = __builtin_fmax(most, near_lane<2>(most));
    top = max(top, near_lane<1>(top));
    top = max(top, near_lane<2>(top));
    if (top >= 0x7ff00000u) { scale = 255; return 0; }
    const uint64_t bits = __builtin_bit_cast(uint64_t, most);
    const int exponent = (int)(bits >> 52);                         // of the largest magnitude, + 1023
    // the least e with most * 2^power <= 1.5 * 2^(e + 2)
    int e = exponent + power - 1023 - ((bits & 0xfffffffffffffull) <= 0x8000000000000ull ? 2 : 1);
    e = exponent == 0 ? -124 : min(max(e, -124), 125);
    scale = (unsigned)(e + 127);
    const int shift = (e - power) << 20;
    float y[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const uint64_t u = __builtin_bit_cast(uint64_t, x[i]);
        // the exponent in units of the scale, not below 2^-23, which is a zero; then float32's bias
        const int hi = max((int)((unsigned)(u >> 32) & kMagnitude) - shift, 1000 << 20);
        const unsigned near = ((unsigned)hi << 3) - (896u << 23);
        y[i] = __uint_as_float((near | min((unsigned)u, 1u)) | ((unsigned)(u >> 32) & ~kMagnitude));
    }
    unsigned w = 0;
    w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, y[0], y[1], 1.0f, 0);
    w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, y[2], y[3], 1.0f, 1);
    w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, y[4], y[5], 1.0f, 2);
    w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, y[6], y[7], 1.0f, 3);
    // a zero without a sign: a magnitude and 7 carry into the sign's place unless it is zero
    const unsigned magnitude = w & 0x77777777u;
    return magnitude | (w & (magnitude + 0x77777777u) & 0x88888888u);
}

// ------------------------------------------------------------------------------------------------
// Many tokens are bound by what a lane computes beside its loads: of 30000 at 64 and 8 heads of 128 with the transform (1.26 GB: 280 us, 4.5 TB/s) the vector units are
// busy most of the time, a key's or value's block in 64 bits with some 330 instructions a wave, a query's with 100.  One token is bound by the latency of its
// chain (length -> table entry -> store) and of its instructions (4.2 us; 5.0 with queries, keys and values by the same workgroup).  A workgroup, or a wave of it
// (THREADS), takes a token.  A lane takes 8 elements, so that four lanes hold a block and a scale is two exchanges between neighbours; the elements that
// turn with them are another lane's, and are read a second time, from the nearest cache.  Of the same place in every kHeads-th head, with that place's cosines
// and sines in registers.

struct Append4Args {
    Batch batch;
    const unsigned char *q, *kn, *vn;
    unsigned char *q_out, *k_out, *v_out, *k, *v, *ks, *vs;
    int64_t q_ts, q_hs, k_ts, k_hs, v_ts, v_hs, qo_ts, qo_hs, ko_ts, ko_hs, vo_ts, vo_hs;       // bytes
    int64_t page_stride, head_stride, token_stride, s_page_stride, s_head_stride, s_token_stride;
    int q_heads, heads, pages, page_shift, position, places;        // places: that a row of the table has
    int transform;
    Turning turn;
};

// Eight elements as they stand in memory.
template <class T> struct Eight { u32x4 w[sizeof(T) / 2]; };
template <class T>
__device__ __forceinline__ Eight<T> read8(const unsigned char* p) {
    Eight<T> x;
#pragma unroll
    for (int i = 0; i < (int)sizeof(T) / 2; ++i) x.w[i] = reinterpret_cast<const u32x4*>(p)[i];
    return x;
}
template <class T>
__device__ __forceinline__ void widen(const Eight<T>& x, float (&f)[8]) {
#pragma unroll
    for (int i = 0; i < (int)sizeof(T) / 2; ++i) {
        const Vec16<T> v = __builtin_bit_cast(Vec16<T>, x.w[i]);
#pragma unroll
        for (int e = 0; e < Vec16<T>::n; ++e) f[i * Vec16<T>::n + e] = (float)v.e[e];
    }
}
template <class T>
__device__ __forceinline__ void load8(float (&f)[8], const unsigned char* p) { widen<T>(read8<T>(p), f); }
template <class T>
__device__ __forceinline__ void store8(unsigned char* p, const float (&f)[8]) {
    if constexpr (sizeof(T) == 2) store16<T>(p, f);
    else {
        *reinterpret_cast<f32x4*>(p) = f32x4{f[0], f[1], f[2], f[3]};
        *reinterpret_cast<f32x4*>(p + 16) = f32x4{f[4], f[5], f[6], f[7]};
    }
}

template <class T, int D, int THREADS>
__global__ __launch_bounds__(256) void append4_kernel(Append4Args a) {
    constexpr int kVectors = D / 8, kOfWave = 64 / kVectors, kHeads = kOfWave * (THREADS / 64), kSize = sizeof(T), kUnroll = sizeof(T) == 2 ? 4 : 2;
    const int lane = threadIdx.x & 63, vector = lane % kVectors, first = (threadIdx.x % THREADS >> 6) * kOfWave + lane / kVectors;
    const int t = THREADS == 256 ? block_of() : __builtin_amdgcn_readfirstlane(block_of() * (256 / THREADS) + threadIdx.x / THREADS);
    if (t >= a.batch.T) return;
    // This lane's eight elements, and the eight that turn with them.  A workgroup's first rounds are on their way before it is known where they go.
    const int half = a.turn.rotary / 2, e0 = vector * 8;
    const bool turns = e0 < a.turn.rotary, low = a.turn.interleaved || e0 < half, across = turns && !a.turn.interleaved;
    const int partner = low ? e0 + half : e0 - half;
    struct Both { Eight<T> x, y; };
    auto read = [&](const unsigned char* from) {
        Both r;
        r.x = r.y = read8<T>(from + e0 * kSize);
        if (across) r.y = read8<T>(from + partner * kSize);
        return r;
    };
    const unsigned char* q_from = a.q + t * a.q_ts;
    // where there are few tokens, queries are one workgroup's and keys and values another's
    const bool apart = THREADS == 256 && gridDim.z == 2, does_q = a.q && (!apart || blockIdx.z == 0), does_kv = !apart || blockIdx.z == 1;
    const int q_rounds = does_q ? ceil_div(a.q_heads, kHeads) : 0, rounds = ceil_div(2 * a.heads, kHeads);
    auto read_q = [&](int round) { return read(q_from + min(first + round * kHeads, a.q_heads - 1) * a.q_hs); };
    auto read_kv = [&](int round) {                                 // keys, then values
        const int n = min(first + round * kHeads, 2 * a.heads - 1);
        return read(n < a.heads ? a.kn + t * a.k_ts + n * a.k_hs : a.vn + t * a.v_ts + (n - a.heads) * a.v_hs);
    };
    Both raw[kUnroll], raw_kv;
    if constexpr (THREADS == 256) {
        if (does_kv) raw_kv = read_kv(0);
#pragma unroll
        for (int i = 0; i < kUnroll; ++i)
            if (i < q_rounds) raw[i] = read_q(i);
    }

    const int b = sequence_of(a.batch, t);                          // by whole waves
    if (lane >= kOfWave * kVectors) return;                         // 96 wide: the lanes are no multiple of the vectors
    bool there = false, known = true;
    int64_t codes_at = 0, scales_at = 0;
    Places p{};
    if (b >= 0) {
        const Sequence s = sequence(a.batch, b);
        const int n = s.length - s.queries + (t - s.first);
        if (a.turn.rotary > 0) {
            p = places_of(a.turn, t, (int64_t)a.position + n);
            known = p.known;
        }
        if (known && t >= s.first && t < s.first + s.queries && n >= 0 && n < a.places) {
            const int page = a.batch.table[b * a.batch.table_stride + (n >> a.page_shift)], slot = n & ((1 << a.page_shift) - 1);
            there = page >= 0 && page < a.pages;
            codes_at = page * a.page_stride + slot * a.token_stride;
            scales_at = page * a.s_page_stride + slot * a.s_token_stride;
        }
    }

    // the angles; an element's own turns it by +, its partner's way by -
    const bool turn = known && b >= 0 && turns;
    float c[8], s[8];
    if (turn) {
        if (a.turn.interleaved) {
            float c4[4], s4[4];
            angles<4>(a.turn, p, e0 / 2, c4, s4);
#pragma unroll
            for (int i = 0; i < 8; ++i) { c[i] = c4[i / 2]; s[i] = i & 1 ? s4[i / 2] : -s4[i / 2]; }
        } else {
            angles<8>(a.turn, p, low ? e0 : partner, c, s);
#pragma unroll
            for (int i = 0; i < 8; ++i) s[i] = low ? -s[i] : s[i];
        }
    }
    auto widen_both = [&](const Both& r, float (&x)[8], float (&y)[8]) {
        widen<T>(r.x, x);
        widen<T>(r.y, y);
        if (turn && a.turn.interleaved)
#pragma unroll
            for (int i = 0; i < 8; i += 2) { const float u = y[i]; y[i] = y[i + 1]; y[i + 1] = u; }
    };

    if (does_q) {
        unsigned char* to = a.q_out + t * a.qo_ts + e0 * kSize;
        if (b >= 0 && known) {
            if (a.transform && turn)
#pragma unroll
                for (int i = 0; i < 8; ++i) { c[i] *= 0.125f; s[i] *= 0.125f; }
            for (int r0 = 0; r0 < q_rounds; r0 += kUnroll) {
                if (THREADS != 256 || r0 > 0)
#pragma unroll
                    for (int i = 0; i < kUnroll; ++i)
                        if (r0 + i < q_rounds) raw[i] = read_q(r0 + i);
#pragma unroll
                for (int i = 0; i < kUnroll; ++i) {
                    if (r0 + i >= q_rounds) break;
                    float x[8], y[8];
                    widen_both(raw[i], x, y);
                    if (turn) {
#pragma unroll
                        for (int e = 0; e < 8; ++e) x[e] = x[e] * c[e] + y[e] * s[e];
                    } else if (a.transform) {
#pragma unroll
                        for (int e = 0; e < 8; ++e) x[e] *= 0.125f;
                    }
                    if (a.transform) transform32(x);
                    const int h = first + (r0 + i) * kHeads;
                    if (h < a.q_heads) store8<T>(to + h * a.qo_hs, x);
                }
            }
            if (a.transform && turn)
#pragma unroll
                for (int i = 0; i < 8; ++i) { c[i] *= 8.0f; s[i] *= 8.0f; }
        } else {
            float x[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) x[i] = b >= 0 ? __builtin_nanf("") : 0.0f;
            for (int h = first; h < a.q_heads; h += kHeads) store8<T>(to + h * a.qo_hs, x);
        }
    }
    if (!does_kv || (!there && !a.k_out)) return;
    for (int r = 0; r < rounds; ++r) {
        const int n = first + r * kHeads, at = min(n, 2 * a.heads - 1);
        const bool key = at < a.heads;
        const int h = key ? at : at - a.heads;
        unsigned codes = 0, scale = b >= 0 ? 255 : 127;             // of a token that is not stored: NaN; of padding: zero
        if (there) {
            float x[8], y[8];
            double z[8];
            if (THREADS != 256 || r > 0) raw_kv = read_kv(r);
            widen_both(raw_kv, x, y);
            if (turn && key) {
#pragma unroll
                for (int i = 0; i < 8; ++i) z[i] = (double)x[i] * c[i] + (double)y[i] * s[i];
            } else {
#pragma unroll
                for (int i = 0; i < 8; ++i) z[i] = (double)x[i];
            }
            if (a.transform) transform32(z);
            codes = encode(z, a.transform ? -2 : 0, scale);
            if (n < 2 * a.heads) {
                *reinterpret_cast<unsigned*>((key ? a.k : a.v) + codes_at + h * a.head_stride + vector * 4) = codes;
                if ((vector & 3) == 0) (key ? a.ks : a.vs)[scales_at + h * a.s_head_stride + vector / 4] = (unsigned char)scale;
            }
        }
        if (a.k_out && n < 2 * a.heads) {
            const bf16x8 v = decode(codes, scale_of(scale));
            float x[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) x[i] = (float)v[i];
            store8<T>(key ? a.k_out + t * a.ko_ts + h * a.ko_hs + e0 * kSize : a.v_out + t * a.vo_ts + h * a.vo_hs + e0 * kSize, x);
        }
    }
}

}  // namespace wht
