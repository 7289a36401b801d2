// Rotary positions of several axes (include/wht_rotary.h) for gfx950.
#pragma once
#include "attention_device.h"
#include "attention4_plan.h"

namespace wht {

// What a call turns heads by.  positions == nullptr: one axis, and a token's position is known otherwise.
struct Turning {
    const float* rope;
    const int* positions;
    int64_t rope_rows;
    int rotary, axes, used;                                         // used: the axes that pairs are on, as bits
    bool interleaved, inverse;
    uint8_t pair_axes[kMaxPairs];
};

// A token's row of `rope` on each axis; `known`: those of all axes that pairs are on are in the table.
struct Places { int at[WHT_ROTARY_MAX_AXES]; bool known; };

__device__ __forceinline__ Places places_of(const Turning& t, int token, int64_t position) {
    Places p;
    p.known = true;
#pragma unroll
    for (int a = 0; a < WHT_ROTARY_MAX_AXES; ++a) {
        const int64_t x = !t.positions ? position : t.positions[(int64_t)token * t.axes + (a < t.axes ? a : 0)];
        p.known &= (x >= 0 && x < t.rope_rows) || !(t.used >> a & 1);
        p.at[a] = (int)x;
    }
    return p;
}
__device__ __forceinline__ int place_on(const Places& p, int axis) {
    const int lo = axis & 1 ? p.at[1] : p.at[0], hi = axis & 1 ? p.at[3] : p.at[2];
    return axis & 2 ? hi : lo;
}

// Cosines and sines of N pairs from pair `first` on.  Pairs that are on one axis stand side by side.
template <int N>
__device__ __forceinline__ void angles(const Turning& t, const Places& p, int first, float (&c)[N], float (&s)[N]) {
    bool one = true;
    const int axis = t.axes > 1 ? t.pair_axes[first] : 0;
    if (t.axes > 1)
#pragma unroll
        for (int i = 1; i < N; ++i) one &= t.pair_axes[first + i] == axis;
    if (one) {
        const f32x4* from = reinterpret_cast<const f32x4*>(t.rope + (int64_t)place_on(p, axis) * t.rotary + first * 2);
#pragma unroll
        for (int i = 0; i < N / 2; ++i) {
            const f32x4 w = from[i];
            c[2 * i] = w[0]; s[2 * i] = w[1]; c[2 * i + 1] = w[2]; s[2 * i + 1] = w[3];
        }
    } else {
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const f32x2 w = *reinterpret_cast<const f32x2*>(t.rope + (int64_t)place_on(p, t.pair_axes[first + i]) * t.rotary + (first + i) * 2);
            c[i] = w[0]; s[i] = w[1];
        }
    }
    if (t.inverse)
#pragma unroll
        for (int i = 0; i < N; ++i) s[i] = -s[i];
}

// ------------------------------------------------------------------------------------------------
// Every element is read and written once: memory.  32760 tokens of 40 heads of 128 in bfloat16 (671 MB): 127 us, 5.3 TB/s; 773 tokens of 20 heads of 64: 4.1 us,
// most of it the chain position -> angle (4.8 with the elements read behind it).  A wave takes a token, so that positions and angles are looked up once; a
// lane takes the same pair of 16-byte vectors, which hold each other's partners, of every heads_at_once-th head.

struct RotaryArgs {
    const unsigned char* x;
    unsigned char* out;
    int64_t x_ts, x_hs, o_ts, o_hs;                                 // bytes
    int T, heads, pairs;                                            // pairs of vectors in a head
    Turning turn;
};

template <class T, bool INTERLEAVED>
__global__ __launch_bounds__(256) void rotary_kernel(RotaryArgs a) {
    constexpr int N = 16 / sizeof(T), kSize = sizeof(T), kUnroll = 4;
    const int lane = threadIdx.x & 63, t = __builtin_amdgcn_readfirstlane(block_of() * 4 + (threadIdx.x >> 6));
    if (t >= a.T) return;
    const int heads_at_once = 64 / a.pairs, pair = lane % a.pairs, first = lane / a.pairs;
    if (first >= heads_at_once) return;                             // a head's pairs do not divide the wave
    const int turned = a.turn.rotary / (2 * N);
    const bool turn = pair < turned;
    int e0 = pair * 2 * N, e1 = e0 + N;
    if (turn && !INTERLEAVED) { e0 = pair * N; e1 = a.turn.rotary / 2 + pair * N; }
    const unsigned char* from = a.x + t * a.x_ts;
    unsigned char* to = a.out + t * a.o_ts;
    u32x4 raw[kUnroll][2];
    auto read = [&](int h0) {
#pragma unroll
        for (int i = 0; i < kUnroll; ++i) {
            const int h = min(h0 + i * heads_at_once, a.heads - 1);
            raw[i][0] = *reinterpret_cast<const u32x4*>(from + h * a.x_hs + e0 * kSize);
            raw[i][1] = *reinterpret_cast<const u32x4*>(from + h * a.x_hs + e1 * kSize);
        }
    };
    read(first);                                                    // on their way before the positions are
    const Places p = places_of(a.turn, t, t);
    float c[N], s[N];
#pragma unroll
    for (int i = 0; i < N; ++i) { c[i] = 1.0f; s[i] = 0.0f; }
    if (turn && p.known) angles<N>(a.turn, p, pair * N, c, s);
    for (int h0 = first; h0 < a.heads; h0 += heads_at_once * kUnroll) {
        if (h0 > first) read(h0);
#pragma unroll
        for (int i = 0; i < kUnroll; ++i) {
            const int h = h0 + i * heads_at_once;
            if (h >= a.heads) break;
            if (turn || !p.known) {
                const Vec16<T> v = __builtin_bit_cast(Vec16<T>, raw[i][0]), w = __builtin_bit_cast(Vec16<T>, raw[i][1]);
                float x[N], y[N], fx[N], fy[N];
#pragma unroll
                for (int e = 0; e < N; ++e) { x[e] = (float)v.e[e]; y[e] = (float)w.e[e]; }
                if constexpr (INTERLEAVED) {
#pragma unroll
                    for (int e = 0; e < N / 2; ++e) {
                        fx[2 * e] = x[2 * e] * c[e] - x[2 * e + 1] * s[e];
                        fx[2 * e + 1] = x[2 * e + 1] * c[e] + x[2 * e] * s[e];
                        fy[2 * e] = y[2 * e] * c[N / 2 + e] - y[2 * e + 1] * s[N / 2 + e];
                        fy[2 * e + 1] = y[2 * e + 1] * c[N / 2 + e] + y[2 * e] * s[N / 2 + e];
                    }
                } else {
#pragma unroll
                    for (int e = 0; e < N; ++e) {
                        fx[e] = x[e] * c[e] - y[e] * s[e];
                        fy[e] = y[e] * c[e] + x[e] * s[e];
                    }
                }
                if (!p.known)
#pragma unroll
                    for (int e = 0; e < N; ++e) fx[e] = fy[e] = __builtin_nanf("");
                store16<T>(to + h * a.o_hs + e0 * kSize, fx);
                store16<T>(to + h * a.o_hs + e1 * kSize, fy);
            } else {
                *reinterpret_cast<u32x4*>(to + h * a.o_hs + e0 * kSize) = raw[i][0];
                *reinterpret_cast<u32x4*>(to + h * a.o_hs + e1 * kSize) = raw[i][1];
            }
        }
    }
}

}  // namespace wht
