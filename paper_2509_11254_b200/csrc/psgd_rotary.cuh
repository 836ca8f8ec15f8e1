// Rotary positions: the pairs of the first R values of every head turned by the angle position * frequency, for queries and keys in one launch.
//
//   (u, v) -> c (u cos a - v sin a, u sin a + v cos a),   a = position_t * frequency_i;   the gradient is turned back (sin a changes its sign).
//
// Pairs are (i, i + R/2) ("half") or (2i, 2i + 1) ("interleaved"); values R.. of a head pass through.  Angles of far positions need more than float32
// (position 2^20 at frequency 1: half an ulp is 0.03), so they are kept as turns in 64-bit fixed point: frequency / 2 pi as a fraction of 2^64, from float64, times
// the position modulo 2^64, is the angle modulo a turn without a rounding of its own; its upper 32 bits as float32 are within 2^-25 of a turn.  A token's sines and
// cosines are formed once per CTA, in shared memory, for all heads.
//
// Bound by HBM: every value read once and written once.  A thread moves 16 bytes at a time (half: 16 of the first half and the 16 that belong to them).
#pragma once
#include <type_traits>

#include "psgd_values.cuh"

namespace psgd {

constexpr int ROT_THREADS = 256;
constexpr int ROT_ITEMS = 4;                       // items of a thread under way at a time
constexpr int ROT_PAIRS = 2048;                    // angles of a CTA in shared memory

struct RotaryTensor { const void* in; void* out; long long in_token, in_head, out_token, out_head; };     // strides in elements
struct RotaryArgs {
    long long T;
    int heads_q, heads, rotated, head;             // heads: of both tensors
    int per_head, turned;                          // items per head, and how many of them hold pairs
    int tokens;                                    // per CTA at a time
    FastDiv by_head, by_heads;                     // per_head, heads
    FastDiv by_pairs;                              // rotated / 2
    RotaryTensor q, k;
    const long long* positions;
    const double* frequencies;                     // radians per position, [rotated / 2]
    float scale, sign;
};

// the angle position * frequency in turns, within -1/2..1/2
__device__ __forceinline__ float turns_of(long long position, double frequency) {
    const double t = frequency * 0.15915494309189533577;                     // 1 / 2 pi
    const unsigned long long step = (unsigned long long)__double2ll_rn((t - rint(t)) * 18446744073709551616.0);
    return (float)(int)((step * (unsigned long long)position) >> 32) * 2.3283064365386963e-10f;          // 2^-32
}

// V: values of a thread's item side by side (half: twice), 8 or 1
template <typename X, int V, bool HALF>
__global__ void __launch_bounds__(ROT_THREADS) k_rotary(const __grid_constant__ RotaryArgs a) {
    typedef typename std::conditional<V == 1, X, typename std::conditional<sizeof(X) == 2, Raw16, Raw32>::type>::type Raw;
    __shared__ float2 turn[ROT_PAIRS];                                       // cosine, sine
    grid_trigger();
    grid_wait();
    const int pairs = a.rotated / 2;
    for (long long t0 = (long long)blockIdx.x * a.tokens; t0 < a.T; t0 += (long long)gridDim.x * a.tokens) {
        const int tokens = (int)min((long long)a.tokens, a.T - t0);
        __syncthreads();
        for (int i = threadIdx.x; i < tokens * pairs; i += ROT_THREADS) {
            const int t = i / a.by_pairs, p = i - t * pairs;
            float s, c;
            sincospif(2.f * turns_of(a.positions[t0 + t], a.frequencies[p]), &s, &c);
            turn[i] = make_float2(c * a.scale, s * a.scale * a.sign);
        }
        __syncthreads();
        const int items = tokens * a.heads * a.per_head;
        for (int i0 = threadIdx.x; i0 < items; i0 += ROT_THREADS * ROT_ITEMS) {
            Raw u[ROT_ITEMS], v[ROT_ITEMS];
            X* to[ROT_ITEMS];
            int at[ROT_ITEMS];                                               // first angle; -1: values that pass through
#pragma unroll
            for (int j = 0; j < ROT_ITEMS; ++j) {
                const int i = i0 + j * ROT_THREADS;
                if (i >= items) break;
                const int hh = i / a.by_head, unit = i - hh * a.per_head;
                const int t = hh / a.by_heads, h = hh - t * a.heads;
                const bool key = h >= a.heads_q;
                const RotaryTensor& x = key ? a.k : a.q;
                const int head = key ? h - a.heads_q : h;
                const bool turned = unit < a.turned;
                int col;
                if (turned) col = HALF ? unit * V : unit * (V == 1 ? 2 : V);
                else col = a.rotated + (unit - a.turned) * V;
                const X* from = (const X*)x.in + (t0 + t) * x.in_token + head * x.in_head + col;
                to[j] = (X*)x.out + (t0 + t) * x.out_token + head * x.out_head + col;
                at[j] = turned ? t * pairs + (HALF ? col : col / 2) : -1;
                if constexpr (V == 8) {
                    load8(u[j], from);
                    if (HALF && turned) load8(v[j], from + pairs);
                } else {
                    u[j] = from[0];
                    if (turned) v[j] = from[HALF ? pairs : 1];
                }
            }
#pragma unroll
            for (int j = 0; j < ROT_ITEMS; ++j) {
                if (i0 + j * ROT_THREADS >= items) break;
                const float2* cs = turn + at[j];
                if constexpr (V == 1) {
                    if (at[j] < 0) {
                        to[j][0] = u[j];
                    } else {
                        const float p = (float)u[j], q = (float)v[j];
                        to[j][0] = (X)(p * cs[0].x - q * cs[0].y);
                        to[j][HALF ? pairs : 1] = (X)(p * cs[0].y + q * cs[0].x);
                    }
                } else {
                    float p[8];
                    widen(u[j], p);
                    if (at[j] >= 0 && HALF) {
                        float q[8];
                        widen(v[j], q);
#pragma unroll
                        for (int e = 0; e < 8; ++e) {
                            const float x = p[e], y = q[e];
                            p[e] = x * cs[e].x - y * cs[e].y;
                            q[e] = x * cs[e].y + y * cs[e].x;
                        }
                        store8(to[j] + pairs, q);
                    } else if (at[j] >= 0) {
#pragma unroll
                        for (int e = 0; e < 4; ++e) {
                            const float x = p[2 * e], y = p[2 * e + 1];
                            p[2 * e] = x * cs[e].x - y * cs[e].y;
                            p[2 * e + 1] = x * cs[e].y + y * cs[e].x;
                        }
                    }
                    store8(to[j], p);
                }
            }
        }
    }
}

}  // namespace psgd
