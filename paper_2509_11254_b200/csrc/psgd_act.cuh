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

__device__ __forceinline__ void load8(const __nv_bfloat16* row, int col, int F, bool vec, float (&x)[8]) {
    if (vec && col + 8 <= F) {
        const uint4 v = __ldg(reinterpret_cast<const uint4*>(row + col));
        const unsigned w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            x[2 * j] = __uint_as_float(w[j] << 16);
            x[2 * j + 1] = __uint_as_float(w[j] & 0xffff0000u);
        }
    } else {
#pragma unroll
        for (int j = 0; j < 8; ++j) x[j] = col + j < F ? __bfloat162float(row[col + j]) : 0.f;
    }
}
__device__ __forceinline__ void load8(const float* row, int col, int F, bool vec, float (&x)[8]) {
    if (vec && col + 8 <= F) {
        const float4 a = __ldg(reinterpret_cast<const float4*>(row + col)), b = __ldg(reinterpret_cast<const float4*>(row + col) + 1);
        x[0] = a.x; x[1] = a.y; x[2] = a.z; x[3] = a.w;
        x[4] = b.x; x[5] = b.y; x[6] = b.z; x[7] = b.w;
    } else {
#pragma unroll
        for (int j = 0; j < 8; ++j) x[j] = col + j < F ? row[col + j] : 0.f;
    }
}
__device__ __forceinline__ void store8(__nv_bfloat16* row, int col, int F, bool vec, const float (&x)[8]) {
    if (vec && col + 8 <= F) {
        *reinterpret_cast<uint4*>(row + col) = make_uint4(pack_bf16(x[0], x[1]), pack_bf16(x[2], x[3]), pack_bf16(x[4], x[5]), pack_bf16(x[6], x[7]));
    } else {
#pragma unroll
        for (int j = 0; j < 8; ++j) if (col + j < F) row[col + j] = __float2bfloat16_rn(x[j]);
    }
}
__device__ __forceinline__ void store8(float* row, int col, int F, bool vec, const float (&x)[8]) {
    if (vec && col + 8 <= F) {
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

// Thread layout of all kernels: threadIdx.x (and blockIdx.x) runs over the 4 G units of 8 values of a row, the rest over rows.
struct ActCursor { int col; long long row, step; };
__device__ __forceinline__ ActCursor act_cursor() {
    ActCursor c;
    c.col = (blockIdx.x * blockDim.x + threadIdx.x) * 8;
    c.row = (long long)blockIdx.y * blockDim.y + threadIdx.y;
    c.step = (long long)gridDim.y * blockDim.y;
    return c;
}

template <typename X>
__global__ void __launch_bounds__(256) k_act_pack(ActShape s, const X* x, long long ldx, bool vec, int8_t* q, uint8_t* scales) {
    const ActCursor c = act_cursor();
    if (c.col >= s.G * ACT_GROUP) return;             // whole groups of four lanes leave together
#pragma unroll 2
    for (long long r = c.row; r < s.T; r += c.step) {
        float v[8];
        load8(x + r * ldx, c.col, s.F, vec, v);
        uint2 b;
        int sb;
        pack8(v, b, sb);
        *reinterpret_cast<uint2*>(q + r * s.G * ACT_GROUP + c.col) = b;
        if ((c.col & 31) == 0) scales[r * s.G + c.col / ACT_GROUP] = (uint8_t)sb;
    }
}

template <typename X>
__global__ void __launch_bounds__(256) k_act_unpack(ActShape s, const int8_t* q, const uint8_t* scales, X* x, long long ldx, bool vec) {
    const ActCursor c = act_cursor();
    if (c.col >= s.F) return;
#pragma unroll 2
    for (long long r = c.row; r < s.T; r += c.step) {
        float v[8];
        unpack8(__ldg(reinterpret_cast<const uint2*>(q + r * s.G * ACT_GROUP + c.col)), scale_of(scales[r * s.G + c.col / ACT_GROUP]), v);
        store8(x + r * ldx, c.col, s.F, vec, v);
    }
}

__device__ __forceinline__ float rcp(float x) {
    float y;
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
__device__ __forceinline__ float sigmoid(float g) { return rcp(1.f + ex2(-g * LOG2E)); }

// h = gate sigmoid(gate) up from the unrounded inputs, both inputs packed in the same pass
__global__ void __launch_bounds__(256) k_swiglu_forward(ActShape s, const __nv_bfloat16* gate, long long ldg, const __nv_bfloat16* up, long long ldu, __nv_bfloat16* h,
                                                        long long ldh, int vec /* bit 0 gate, 1 up, 2 h */, int8_t* qg, uint8_t* sg, int8_t* qu, uint8_t* su) {
    const ActCursor c = act_cursor();
    if (c.col >= s.G * ACT_GROUP) return;
#pragma unroll 2
    for (long long r = c.row; r < s.T; r += c.step) {
        float g[8], u[8], y[8];
        load8(gate + r * ldg, c.col, s.F, vec & 1, g);
        load8(up + r * ldu, c.col, s.F, vec & 2, u);
#pragma unroll
        for (int j = 0; j < 8; ++j) y[j] = g[j] * sigmoid(g[j]) * u[j];
        store8(h + r * ldh, c.col, s.F, vec & 4, y);
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

// d_gate = dh up s (1 + gate (1 - s)),  d_up = dh gate s,  h = gate s up  (s = sigmoid(gate)), gate and up from their checkpoints
template <bool H>
__global__ void __launch_bounds__(256) k_swiglu_backward(ActShape s, const __nv_bfloat16* dh, long long lddh, const int8_t* qg, const uint8_t* sg, const int8_t* qu,
                                                         const uint8_t* su, __nv_bfloat16* dg, long long lddg, __nv_bfloat16* du, long long lddu, __nv_bfloat16* h,
                                                         long long ldh, int vec /* bit 0 dh, 1 dg, 2 du, 3 h */) {
    const ActCursor c = act_cursor();
    if (c.col >= s.F) return;
#pragma unroll 2
    for (long long r = c.row; r < s.T; r += c.step) {
        const long long at = r * s.G * ACT_GROUP + c.col, sat = r * s.G + c.col / ACT_GROUP;
        float d[8], g[8], u[8], a[8], b[8], y[8];
        load8(dh + r * lddh, c.col, s.F, vec & 1, d);
        unpack8(__ldg(reinterpret_cast<const uint2*>(qg + at)), scale_of(sg[sat]), g);
        unpack8(__ldg(reinterpret_cast<const uint2*>(qu + at)), scale_of(su[sat]), u);
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const float sig = sigmoid(g[j]), act = g[j] * sig;
            a[j] = d[j] * u[j] * (sig + act * (1.f - sig));
            b[j] = d[j] * act;
            y[j] = act * u[j];
        }
        store8(dg + r * lddg, c.col, s.F, vec & 2, a);
        store8(du + r * lddu, c.col, s.F, vec & 4, b);
        if (H) store8(h + r * ldh, c.col, s.F, vec & 8, y);
    }
}

}  // namespace psgd
