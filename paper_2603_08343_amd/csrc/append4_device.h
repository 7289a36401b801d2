// Append to the cache in 4 bits (include/wht_attention4.h) for gfx950.
#pragma once
#include "rotary_device.h"

namespace wht {

typedef float f32x8 __attribute__((ext_vector_type(8)));

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

// Walsh-Hadamard transform of the 32 numbers that four lanes hold, eight each: three steps in registers, two between lanes.
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
#pragma unroll
    for (int i = 0; i < 8; ++i) { const F other = near_lane<1>(x[i]); x[i] = threadIdx.x & 1 ? other - x[i] : x[i] + other; }
#pragma unroll
    for (int i = 0; i < 8; ++i) { const F other = near_lane<2>(x[i]); x[i] = threadIdx.x & 2 ? other - x[i] : x[i] + other; }
}

// Codes of eight of a block's 32 numbers, and the block's scale byte.  The numbers are in 64 bits: a code is decided by which side of a border a
// number is on, and what a sum in 32 bits is off by would now and then decide it.  They are made 32 bits wide with the last bit standing for whatever
// was cut off, which leaves every border where it is, and go to the nearest code as the hardware does it.
__device__ __forceinline__ unsigned encode(const double (&x)[8], unsigned& scale) {
    constexpr uint64_t kMagnitude = ~(uint64_t)0 >> 1;
    uint64_t most = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) { const uint64_t m = __builtin_bit_cast(uint64_t, x[i]) & kMagnitude; most = m > most ? m : most; }
    uint64_t other = near_lane<1>(most);
    most = other > most ? other : most;
    other = near_lane<2>(most);
    most = other > most ? other : most;
    const int exponent = (int)(most >> 52);                         // of the largest magnitude, + 1023
    // the least e with most <= 1.5 * 2^(e + 2)
    int e = exponent - 1023 - ((most & 0xfffffffffffffull) <= 0x8000000000000ull ? 2 : 1);
    e = exponent == 0 ? -124 : min(max(e, -124), 125);
    if (exponent == 0x7ff) { scale = 255; return 0; }
    scale = (unsigned)(e + 127);
    const double by = __builtin_bit_cast(double, (uint64_t)(1023 - e) << 52);
    float y[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const double exact = x[i] * by;                             // a power of two
        const float near = (float)exact;
        const unsigned u = __float_as_uint(near);
        const double back = (double)near;
        // towards zero, then odd
        const unsigned odd = (__builtin_fabs(back) > __builtin_fabs(exact) ? u - 1 : u) | 1;
        y[i] = __uint_as_float(back == exact ? u : odd);
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
// Bound by memory where there are many tokens, and one token by the latency of its chain (length -> table entry -> store).  A workgroup, or a wave of
// it (THREADS), takes a token.  A lane takes 8 elements, so that four lanes hold a block and a scale is two exchanges between neighbours; the elements that
// turn with them are another lane's, and are read a second time, from the nearest cache.  Of the same place in every kHeads-th head, with that
// place's cosines and sines in registers.

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

template <class T>
__device__ __forceinline__ void load8(float (&f)[8], const unsigned char* p) {
    if constexpr (sizeof(T) == 2) load16<T>(f, p);
    else {
        const f32x4 lo = *reinterpret_cast<const f32x4*>(p), hi = *reinterpret_cast<const f32x4*>(p + 16);
#pragma unroll
        for (int i = 0; i < 4; ++i) { f[i] = lo[i]; f[4 + i] = hi[i]; }
    }
}
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
    constexpr int kVectors = D / 8, kOfWave = 64 / kVectors, kHeads = kOfWave * (THREADS / 64), kSize = sizeof(T);
    const int lane = threadIdx.x & 63, vector = lane % kVectors, first = (threadIdx.x % THREADS >> 6) * kOfWave + lane / kVectors;
    const int t = THREADS == 256 ? block_of() : __builtin_amdgcn_readfirstlane(block_of() * (256 / THREADS) + threadIdx.x / THREADS);
    if (t >= a.batch.T) return;
    const int b = sequence_of(a.batch, t);
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
    if (lane >= kOfWave * kVectors) return;                         // 96 wide: the lanes are no multiple of the vectors

    // this lane's elements' partners, and the angles; an element's own angle turns it by +, its partner's way by -
    const int half = a.turn.rotary / 2, e0 = vector * 8;
    const bool turn = known && b >= 0 && e0 < a.turn.rotary, low = a.turn.interleaved || e0 < half;
    const int partner = low ? e0 + half : e0 - half;
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
    // the eight elements and their partners
    auto load = [&](const unsigned char* from, float (&x)[8], float (&y)[8]) {
        load8<T>(x, from + e0 * kSize);
        if (!turn) return;
        if (a.turn.interleaved) {
#pragma unroll
            for (int i = 0; i < 8; ++i) y[i] = x[i ^ 1];
        } else load8<T>(y, from + partner * kSize);
    };

    if (a.q) {
        for (int h = first; h < a.q_heads; h += kHeads) {
            float x[8], y[8];
            if (b >= 0 && known) {
                load(a.q + t * a.q_ts + h * a.q_hs, x, y);
                if (turn)
#pragma unroll
                    for (int i = 0; i < 8; ++i) x[i] = x[i] * c[i] + y[i] * s[i];
                if (a.transform) {
                    transform32(x);
#pragma unroll
                    for (int i = 0; i < 8; ++i) x[i] *= 0.125f;
                }
            } else {
#pragma unroll
                for (int i = 0; i < 8; ++i) x[i] = b >= 0 ? __builtin_nanf("") : 0.0f;
            }
            store8<T>(a.q_out + t * a.qo_ts + h * a.qo_hs + e0 * kSize, x);
        }
    }
    if (!there && !a.k_out) return;
    for (int n = first; n < 2 * a.heads; n += kHeads) {             // keys, then values
        const bool key = n < a.heads;
        const int h = key ? n : n - a.heads;
        unsigned codes = 0, scale = b >= 0 ? 255 : 127;             // of a token that is not stored: NaN; of padding: zero
        if (there) {
            float x[8], y[8];
            double z[8];
            if (key) load(a.kn + t * a.k_ts + h * a.k_hs, x, y);
            else load8<T>(x, a.vn + t * a.v_ts + h * a.v_hs + e0 * kSize);
#pragma unroll
            for (int i = 0; i < 8; ++i) z[i] = key && turn ? (double)x[i] * c[i] + (double)y[i] * s[i] : (double)x[i];
            if (a.transform) {
                transform32(z);
#pragma unroll
                for (int i = 0; i < 8; ++i) z[i] *= 0.25;
            }
            codes = encode(z, scale);
            *reinterpret_cast<unsigned*>((key ? a.k : a.v) + codes_at + h * a.head_stride + vector * 4) = codes;
            if ((vector & 3) == 0) (key ? a.ks : a.vs)[scales_at + h * a.s_head_stride + vector / 4] = (unsigned char)scale;
        }
        if (a.k_out) {
            const bf16x8 v = decode(codes, scale_of(scale));
            float x[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) x[i] = (float)v[i];
            store8<T>(key ? a.k_out + t * a.ko_ts + h * a.ko_hs + e0 * kSize : a.v_out + t * a.vo_ts + h * a.vo_hs + e0 * kSize, x);
        }
    }
}

}  // namespace wht
