// Rotary positions: the pairs of the first R values of every head turned by the angle position * frequency, for queries and keys in one launch.
//
//   (u, v) -> c (u cos a - v sin a, u sin a + v cos a),   a = position_t * frequency_i;   the gradient is turned back (sin a changes its sign).
//
// Pairs are (i, i + R/2) ("half") or (2i, 2i + 1) ("interleaved"); values R.. of a head pass through.  Angles of far positions need more than float32
// (position 2^20 at frequency 1: half an ulp is 0.03), so they are kept as turns in 64-bit fixed point: frequency / 2 pi as a fraction of 2^64, from float64, times
// the position modulo 2^64, is the angle modulo a turn without a rounding of its own; its distance from the nearest quarter of a turn as float32 is within 2^-28 of a
// turn, below the rounding of the sine itself.  A token's sines and cosines are formed once per CTA, in shared memory, for all heads.
//
// Bound by HBM: every value read once and written once.  A thread moves V values at a time, 16 bytes of bfloat16 where widths and addresses allow (half: V of the first half and
// the V that belong to them), of the same place in ROT_HEADS heads, whose loads are under way together and which share the sines and cosines that it reads.
#pragma once
#include <type_traits>

#include "psgd_values.cuh"

namespace psgd {

constexpr int ROT_THREADS = 256;
constexpr int ROT_HEADS = 4;                       // heads of an item
constexpr int ROT_PAIRS = 2048;                    // angles of a CTA in shared memory

struct RotaryTensor { const void* in; void* out; long long in_token, in_head, out_token, out_head; };     // strides in elements
struct RotaryArgs {
    long long T;
    int heads_q, heads, rotated, head;             // heads: of both tensors
    int per_head, turned;                          // places of V values in a head, and how many of them hold (first values of) pairs
    int groups;                                    // of ROT_HEADS heads
    int tokens;                                    // per CTA at a time
    FastDiv by_head, by_groups;                    // per_head, groups
    FastDiv by_pairs;                              // rotated / 2
    RotaryTensor q, k;
    const long long* positions;
    const double* frequencies;                     // radians per position, [rotated / 2]
    float scale, sign;
};

// Cosine and sine of position * frequency; NaN where the frequency is not finite (as an integer that would be some angle).  The angle's upper two bits, rounded, are whole quarters
// of a turn; what is left, at most an eighth, keeps 24 bits of its own in float32.
__device__ __forceinline__ float2 turn_of(long long position, double frequency) {
    const double t = frequency * 0.15915494309189533577;                     // 1 / 2 pi
    const unsigned long long step = (unsigned long long)__double2ll_rn((t - rint(t)) * 18446744073709551616.0);
    const unsigned long long angle = step * (unsigned long long)position, quarters = (angle + (1ull << 61)) >> 62;
    float s, c;
    sincospif((float)(long long)(angle - (quarters << 62)) * 1.0842021724855044e-19f + (float)(t - t), &s, &c);      // 2^-63: half turns
    if (quarters & 1) { const float u = c; c = -s; s = u; }
    return quarters & 2 ? make_float2(-c, -s) : make_float2(c, s);
}

// V values side by side: 2 to 32 bytes
template <typename X, int V> struct Some {
    static constexpr int BYTES = V * (int)sizeof(X);
    typedef typename std::conditional<BYTES == 2, unsigned short, typename std::conditional<BYTES == 4, unsigned, typename std::conditional<BYTES == 8, uint2, uint4>::type>::type>::type Word;
    Word w[BYTES == 32 ? 2 : 1];
    __device__ __forceinline__ void load(const X* p) {
        w[0] = reinterpret_cast<const Word*>(p)[0];
        if constexpr (BYTES == 32) w[1] = reinterpret_cast<const Word*>(p)[1];
    }
    __device__ __forceinline__ void store(X* p) const {
        reinterpret_cast<Word*>(p)[0] = w[0];
        if constexpr (BYTES == 32) reinterpret_cast<Word*>(p)[1] = w[1];
    }
    __device__ __forceinline__ void get(float (&x)[V]) const {
        const X* v = reinterpret_cast<const X*>(w);
#pragma unroll
        for (int j = 0; j < V; ++j) x[j] = (float)v[j];
    }
    __device__ __forceinline__ void set(const float (&x)[V]) {
        if constexpr (sizeof(X) == 2 && V > 1) {
#pragma unroll
            for (int j = 0; j < V; j += 2) reinterpret_cast<unsigned*>(w)[j / 2] = pack_bf16(x[j], x[j + 1]);
        } else {
#pragma unroll
            for (int j = 0; j < V; ++j) reinterpret_cast<X*>(w)[j] = (X)x[j];
        }
    }
};

template <typename X, int V, bool HALF>
__global__ void __launch_bounds__(ROT_THREADS) k_rotary(const __grid_constant__ RotaryArgs a) {
    constexpr int PAIRS = HALF ? V : (V == 1 ? 1 : V / 2);                   // of a place
    constexpr bool SPLIT = HALF || V == 1;                                   // a pair's values lie in two places
    __shared__ __align__(16) float2 turn[ROT_PAIRS];                         // cosine, sine; two pairs of a place side by side, then those of the next place: no bank twice
    grid_trigger();
    grid_wait();
    const int pairs = a.rotated / 2, places = pairs / PAIRS, second = HALF ? pairs : 1;
    for (long long t0 = (long long)blockIdx.x * a.tokens; t0 < a.T; t0 += (long long)gridDim.x * a.tokens) {
        const int tokens = (int)min((long long)a.tokens, a.T - t0);
        __syncthreads();
        for (int i = threadIdx.x; i < tokens * pairs; i += ROT_THREADS) {
            const int t = i / a.by_pairs, p = i - t * pairs;
            const float2 cs = turn_of(a.positions[t0 + t], a.frequencies[p]);
            const int at = PAIRS == 1 ? p : ((p % PAIRS / 2) * places + p / PAIRS) * 2 + (p & 1);
            turn[t * pairs + at] = make_float2(cs.x * a.scale, cs.y * a.scale * a.sign);
        }
        __syncthreads();
        const int items = tokens * a.groups * a.per_head;
        for (int i = threadIdx.x; i < items; i += ROT_THREADS) {
            const int tg = i / a.by_head, place = i - tg * a.per_head;
            const int t = tg / a.by_groups, h0 = (tg - t * a.groups) * ROT_HEADS;
            const bool turned = place < a.turned;
            const int col = turned ? place * (SPLIT && !HALF ? 2 : V) : a.rotated + (place - a.turned) * V;
            Some<X, V> u[ROT_HEADS], v[SPLIT ? ROT_HEADS : 1];
            const auto at = [&](int h, bool out) -> X* {
                const RotaryTensor& x = h >= a.heads_q ? a.k : a.q;
                const long long head = h >= a.heads_q ? h - a.heads_q : h;
                return out ? (X*)x.out + (t0 + t) * x.out_token + head * x.out_head + col : (X*)x.in + (t0 + t) * x.in_token + head * x.in_head + col;
            };
#pragma unroll
            for (int j = 0; j < ROT_HEADS; ++j) {
                if (h0 + j >= a.heads) break;
                const X* from = at(h0 + j, false);
                u[j].load(from);
                if constexpr (SPLIT) {
                    if (turned) v[j].load(from + second);
                }
            }
            float c[PAIRS], s[PAIRS];
            if (turned) {
                const float2* cs = turn + t * pairs;
                if constexpr (PAIRS == 1) {
                    c[0] = cs[place].x;
                    s[0] = cs[place].y;
                } else {
#pragma unroll
                    for (int k = 0; k < PAIRS; k += 2) {
                        const float4 two = *reinterpret_cast<const float4*>(cs + (k / 2 * places + place) * 2);
                        c[k] = two.x; s[k] = two.y; c[k + 1] = two.z; s[k + 1] = two.w;
                    }
                }
            }
#pragma unroll
            for (int j = 0; j < ROT_HEADS; ++j) {
                if (h0 + j >= a.heads) break;
                X* to = at(h0 + j, true);
                if (turned) {
                    float p[V];
                    u[j].get(p);
                    if constexpr (SPLIT) {
                        float q[V];
                        v[j].get(q);
#pragma unroll
                        for (int e = 0; e < V; ++e) {
                            const float x = p[e], y = q[e];
                            p[e] = x * c[e] - y * s[e];
                            q[e] = x * s[e] + y * c[e];
                        }
                        v[j].set(q);
                        v[j].store(to + second);
                    } else {
#pragma unroll
                        for (int e = 0; e < PAIRS; ++e) {
                            const float x = p[2 * e], y = p[2 * e + 1];
                            p[2 * e] = x * c[e] - y * s[e];
                            p[2 * e + 1] = x * s[e] + y * c[e];
                        }
                    }
                    u[j].set(p);
                }
                u[j].store(to);
            }
        }
    }
}

}  // namespace psgd
