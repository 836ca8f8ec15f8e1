// Activation checkpoints in 8 bits, and the gated unit of the feed-forward block with its two inputs kept that way.
//
// A checkpoint of a matrix [T][F] holds, per row and group of 32 values, one scale 2^e (e the smallest integer with
// max|x| <= 127 * 2^e, kept within -126..121, stored as the byte e + 127; 255 marks a group with an infinity or a NaN, which
// stands for NaN) and the whole numbers rint(x / 2^e) within -127..127 as int8, rows padded with zeros to whole groups:
// 1 + 1/32 bytes per value.  With a power of two as scale every stored value is exact in bfloat16, so that
// products of checkpoints run on the tensor cores without another rounding.
//
// All kernels here are one pass over their operands and bound by HBM: a thread moves 8 values (16 bytes of bfloat16, 8 of
// int8), four neighbouring threads share a group, and the group's maximum is two shuffles.
#pragma once
#include <cuda_bf16.h>
#include <stdint.h>

#include "psgd_tile.cuh"

namespace psgd {

constexpr int ACT_GROUP = 32;
constexpr int ACT_NAN = 255;

struct ActShape { long long T; int F, G; };      // G = groups per row; the int8 rows hold 32 G bytes

// Eight values as they lie in memory, and as float32.  VEC: the address is 16-byte aligned and all eight exist; else element by
// element, zeros beyond the row's end.  Loading and converting are apart so that a thread can ask for several rows before it
// waits for the first.
struct Raw16 { uint4 a; };
struct Raw32 { float4 a, b; };
template <bool VEC>
__device__ __forceinline__ void load8(Raw16& r, const __nv_bfloat16* row, int col, int F) {
    if (VEC) {
        r.a = __ldg(reinterpret_cast<const uint4*>(row + col));
    } else {
        unsigned w[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const unsigned lo = col + 2 * j < F ? __ldg(reinterpret_cast<const unsigned short*>(row) + col + 2 * j) : 0u;
            const unsigned hi = col + 2 * j + 1 < F ? __ldg(reinterpret_cast<const unsigned short*>(row) + col + 2 * j + 1) : 0u;
            w[j] = lo | hi << 16;
        }
        r.a = make_uint4(w[0], w[1], w[2], w[3]);
    }
}
template <bool VEC>
__device__ __forceinline__ void load8(Raw32& r, const float* row, int col, int F) {
    if (VEC) {
        r.a = __ldg(reinterpret_cast<const float4*>(row + col));
        r.b = __ldg(reinterpret_cast<const float4*>(row + col) + 1);
    } else {
        float w[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) w[j] = col + j < F ? __ldg(row + col + j) : 0.f;
        r.a = make_float4(w[0], w[1], w[2], w[3]);
        r.b = make_float4(w[4], w[5], w[6], w[7]);
    }
}
__device__ __forceinline__ void widen(const Raw16& r, float (&x)[8]) {
    const unsigned w[4] = {r.a.x, r.a.y, r.a.z, r.a.w};
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        x[2 * j] = __uint_as_float(w[j] << 16);
        x[2 * j + 1] = __uint_as_float(w[j] & 0xffff0000u);
    }
}
__device__ __forceinline__ void widen(const Raw32& r, float (&x)[8]) {
    x[0] = r.a.x; x[1] = r.a.y; x[2] = r.a.z; x[3] = r.a.w;
    x[4] = r.b.x; x[5] = r.b.y; x[6] = r.b.z; x[7] = r.b.w;
}
template <typename X> struct RawOf { typedef Raw32 type; };
template <> struct RawOf<__nv_bfloat16> { typedef Raw16 type; };

template <bool VEC>
__device__ __forceinline__ void store8(__nv_bfloat16* row, int col, int F, const float (&x)[8]) {
    if (VEC) {
        *reinterpret_cast<uint4*>(row + col) = make_uint4(pack_bf16(x[0], x[1]), pack_bf16(x[2], x[3]), pack_bf16(x[4], x[5]), pack_bf16(x[6], x[7]));
    } else {
#pragma unroll
        for (int j = 0; j < 8; ++j) if (col + j < F) row[col + j] = __float2bfloat16_rn(x[j]);
    }
}
template <bool VEC>
__device__ __forceinline__ void store8(float* row, int col, int F, const float (&x)[8]) {
    if (VEC) {
        reinterpret_cast<float4*>(row + col)[0] = make_float4(x[0], x[1], x[2], x[3]);
        reinterpret_cast<float4*>(row + col)[1] = make_float4(x[4], x[5], x[6], x[7]);
    } else {
#pragma unroll
        for (int j = 0; j < 8; ++j) if (col + j < F) row[col + j] = x[j];
    }
}

// Eight values of a group whose other 24 belong to the three neighbouring lanes (all four call) -> int8 and the scale byte.
__device__ __forceinline__ void pack8(const float (&x)[8], uint2& q, int& scale_byte) {
    unsigned top = 0;
#pragma unroll
    for (int j = 0; j < 8; ++j) top = max(top, __float_as_uint(x[j]) & 0x7fffffffu);
    const unsigned quad = 0xfu << ((threadIdx.y * blockDim.x + threadIdx.x) & 28);   // blockDim.x is a multiple of 4
    top = max(top, __shfl_xor_sync(quad, top, 1));
    top = max(top, __shfl_xor_sync(quad, top, 2));
    // max|x| = f 2^k with f in [1, 2):  f <= 127/64 asks for e = k - 6, a larger f for k - 5
    int e = (int)(top >> 23) - 127 - 6 + ((top & 0x7fffffu) > 0x7e0000u ? 1 : 0);
    e = min(max(e, -126), 121);
    const bool fine = top < 0x7f800000u;
    scale_byte = fine ? e + 127 : ACT_NAN;
    const float inv = __uint_as_float((unsigned)(127 - e) << 23);
    unsigned b[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        const float y = fminf(fmaxf(x[j] * inv, -127.f), 127.f);           // beyond 127 only where e met its upper end
        b[j] = __float_as_uint(y + 12582912.f);                            // 1.5 * 2^23: the whole number in the low byte, ties to even
    }
    q.x = __byte_perm(__byte_perm(b[0], b[1], 0x0040), __byte_perm(b[2], b[3], 0x0040), 0x5410);
    q.y = __byte_perm(__byte_perm(b[4], b[5], 0x0040), __byte_perm(b[6], b[7], 0x0040), 0x5410);
    if (!fine) q = make_uint2(0u, 0u);
}
__device__ __forceinline__ float scale_of(int byte) { return byte == ACT_NAN ? NAN : __uint_as_float((unsigned)byte << 23); }
__device__ __forceinline__ void unpack8(uint2 q, float scale, float (&x)[8]) {
    const unsigned w[2] = {q.x ^ 0x80808080u, q.y ^ 0x80808080u};          // q + 128 in every byte
#pragma unroll
    for (int j = 0; j < 8; ++j) x[j] = (__uint_as_float(__byte_perm(w[j / 4], 0x4B000000u, 0x7440 + (j & 3))) - (XE_MAGIC + 128.f)) * scale;
}

// Thread layout of all kernels: threadIdx.x (and blockIdx.x) runs over the 4 G units of 8 values of a row, the rest over rows.  A
// thread asks for ACT_ROWS rows before it works on any, so that enough bytes are under way for HBM's latency.
// VEC: F is a multiple of 8 and every operand 16-byte aligned in every row.
constexpr int ACT_ROWS = 2, ACT_ROWS_PACK = 4;
struct ActCursor { int col; long long row, step; };
__device__ __forceinline__ ActCursor act_cursor() {
    ActCursor c;
    c.col = (blockIdx.x * blockDim.x + threadIdx.x) * 8;
    c.row = (long long)blockIdx.y * blockDim.y + threadIdx.y;
    c.step = (long long)gridDim.y * blockDim.y;
    return c;
}

template <typename X, bool VEC>
__global__ void __launch_bounds__(256) k_act_pack(ActShape s, const X* __restrict__ x, long long ldx, int8_t* __restrict__ q, uint8_t* __restrict__ scales) {
    const ActCursor c = act_cursor();
    if (c.col >= s.G * ACT_GROUP) return;             // whole groups of four lanes leave together
    constexpr int R = ACT_ROWS_PACK;
    const bool real = !VEC || c.col < s.F;            // (a unit behind the row's end belongs to the padding of its last group)
    for (long long r0 = c.row; r0 < s.T; r0 += R * c.step) {
        typename RawOf<X>::type raw[R] = {};
        if (real) {
#pragma unroll
            for (int i = 0; i < R; ++i) load8<VEC>(raw[i], x + min(r0 + i * c.step, s.T - 1) * ldx, c.col, s.F);
        }
#pragma unroll
        for (int i = 0; i < R; ++i) {
            const long long r = r0 + i * c.step;
            if (r >= s.T) break;
            float v[8];
            widen(raw[i], v);
            uint2 b;
            int sb;
            pack8(v, b, sb);
            *reinterpret_cast<uint2*>(q + r * s.G * ACT_GROUP + c.col) = b;
            if ((c.col & 31) == 0) scales[r * s.G + c.col / ACT_GROUP] = (uint8_t)sb;
        }
    }
}

template <typename X, bool VEC>
__global__ void __launch_bounds__(256) k_act_unpack(ActShape s, const int8_t* __restrict__ q, const uint8_t* __restrict__ scales, X* __restrict__ x, long long ldx) {
    const ActCursor c = act_cursor();
    if (c.col >= s.F) return;
    constexpr int R = ACT_ROWS_PACK;
    for (long long r0 = c.row; r0 < s.T; r0 += R * c.step) {
        uint2 b[R];
        int sb[R];
#pragma unroll
        for (int i = 0; i < R; ++i) {
            const long long r = min(r0 + i * c.step, s.T - 1);
            b[i] = __ldg(reinterpret_cast<const uint2*>(q + r * s.G * ACT_GROUP + c.col));
            sb[i] = __ldg(scales + r * s.G + c.col / ACT_GROUP);
        }
#pragma unroll
        for (int i = 0; i < R; ++i) {
            const long long r = r0 + i * c.step;
            if (r >= s.T) break;
            float v[8];
            unpack8(b[i], scale_of(sb[i]), v);
            store8<VEC>(x + r * ldx, c.col, s.F, v);
        }
    }
}

__device__ __forceinline__ float rcp(float x) {
    float y;
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
__device__ __forceinline__ float sigmoid(float g) { return rcp(1.f + ex2(-g * LOG2E)); }

// h = gate sigmoid(gate) up from the unrounded inputs, both inputs packed in the same pass
template <bool VEC>
__global__ void __launch_bounds__(256) k_swiglu_forward(ActShape s, const __nv_bfloat16* __restrict__ gate, long long ldg, const __nv_bfloat16* __restrict__ up, long long ldu,
                                                        __nv_bfloat16* __restrict__ h, long long ldh, int8_t* __restrict__ qg, uint8_t* __restrict__ sg,
                                                        int8_t* __restrict__ qu, uint8_t* __restrict__ su) {
    const ActCursor c = act_cursor();
    if (c.col >= s.G * ACT_GROUP) return;
    constexpr int R = ACT_ROWS;
    const bool real = !VEC || c.col < s.F;
    for (long long r0 = c.row; r0 < s.T; r0 += R * c.step) {
        Raw16 rg[R] = {}, ru[R] = {};
        if (real) {
#pragma unroll
            for (int i = 0; i < R; ++i) {
                const long long r = min(r0 + i * c.step, s.T - 1);
                load8<VEC>(rg[i], gate + r * ldg, c.col, s.F);
                load8<VEC>(ru[i], up + r * ldu, c.col, s.F);
            }
        }
#pragma unroll
        for (int i = 0; i < R; ++i) {
            const long long r = r0 + i * c.step;
            if (r >= s.T) break;
            float g[8], u[8], y[8];
            widen(rg[i], g);
            widen(ru[i], u);
#pragma unroll
            for (int j = 0; j < 8; ++j) y[j] = g[j] * sigmoid(g[j]) * u[j];
            if (real) store8<VEC>(h + r * ldh, c.col, s.F, y);
            uint2 b;
            int sb;
            pack8(g, b, sb);
            const long long at = r * s.G * ACT_GROUP + c.col, sat = r * s.G + c.col / ACT_GROUP;
            *reinterpret_cast<uint2*>(qg + at) = b;
            if ((c.col & 31) == 0) sg[sat] = (uint8_t)sb;
            pack8(u, b, sb);
            *reinterpret_cast<uint2*>(qu + at) = b;
            if ((c.col & 31) == 0) su[sat] = (uint8_t)sb;
        }
    }
}

// d_gate = dh up s (1 + gate (1 - s)),  d_up = dh gate s,  h = gate s up  (s = sigmoid(gate)), gate and up from their checkpoints
template <bool H, bool VEC>
__global__ void __launch_bounds__(256) k_swiglu_backward(ActShape s, const __nv_bfloat16* __restrict__ dh, long long lddh, const int8_t* __restrict__ qg,
                                                         const uint8_t* __restrict__ sg, const int8_t* __restrict__ qu, const uint8_t* __restrict__ su,
                                                         __nv_bfloat16* __restrict__ dg, long long lddg, __nv_bfloat16* __restrict__ du, long long lddu,
                                                         __nv_bfloat16* __restrict__ h, long long ldh) {
    const ActCursor c = act_cursor();
    if (c.col >= s.F) return;
    constexpr int R = ACT_ROWS;
    for (long long r0 = c.row; r0 < s.T; r0 += R * c.step) {
        Raw16 rd[R];
        uint2 bg[R], bu[R];
        int eg[R], eu[R];
#pragma unroll
        for (int i = 0; i < R; ++i) {
            const long long r = min(r0 + i * c.step, s.T - 1);
            const long long at = r * s.G * ACT_GROUP + c.col, sat = r * s.G + c.col / ACT_GROUP;
            load8<VEC>(rd[i], dh + r * lddh, c.col, s.F);
            bg[i] = __ldg(reinterpret_cast<const uint2*>(qg + at));
            bu[i] = __ldg(reinterpret_cast<const uint2*>(qu + at));
            eg[i] = __ldg(sg + sat);
            eu[i] = __ldg(su + sat);
        }
#pragma unroll
        for (int i = 0; i < R; ++i) {
            const long long r = r0 + i * c.step;
            if (r >= s.T) break;
            float d[8], g[8], u[8], a[8], b[8], y[8];
            widen(rd[i], d);
            unpack8(bg[i], scale_of(eg[i]), g);
            unpack8(bu[i], scale_of(eu[i]), u);
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const float sig = sigmoid(g[j]), act = g[j] * sig;
                a[j] = d[j] * u[j] * (sig + act * (1.f - sig));
                b[j] = d[j] * act;
                y[j] = act * u[j];
            }
            store8<VEC>(dg + r * lddg, c.col, s.F, a);
            store8<VEC>(du + r * lddu, c.col, s.F, b);
            if (H) store8<VEC>(h + r * ldh, c.col, s.F, y);
        }
    }
}

}  // namespace psgd
