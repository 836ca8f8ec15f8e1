// Activation checkpoints in 8 bits, and the gated unit of the feed-forward block with its two inputs kept that way.
//
// A checkpoint of a matrix [T][F] holds, per row and group of 32 values, one scale 2^e (e the smallest integer with
// max|x| <= 127 * 2^e, kept within -126..121, stored as the byte e + 127; 255 marks a group with an infinity or a NaN, which
// stands for NaN) and the whole numbers rint(x / 2^e) within -127..127 as int8, rows padded with zeros to whole groups:
// 1 + 1/32 bytes per value.  With a power of two as scale every stored value is exact in bfloat16, so that
// products of checkpoints run on the tensor cores without another rounding.
//
// All kernels here are one pass over their operands and bound by HBM.  Aligned operands: a thread moves 8 values (16 bytes of
// bfloat16, 8 of int8), four neighbouring threads share a group, and the group's maximum is two shuffles.  Rows of any
// other length or alignment: a lane per value and a warp per group, whose 2-byte accesses still come as whole sectors (with
// 8 values per thread there, stores of 2 bytes 16 bytes apart made the backward pass of 4096 x 2051 72 us, against 18 of 4096 x 2048).
//
// Measured (8.06, 10.06, 3.03 and 3.03 bytes per value; of the 6533 GB/s of a copy), 16384 x 5504: gated unit forward 128 us (87 %), backward with h
// 157 us (88 %), pack 52 us (80 %), unpack 50 us (84 %).
#pragma once
#include <cuda_bf16.h>
#include <stdint.h>

#include "psgd_tile.cuh"

namespace psgd {

constexpr int ACT_GROUP = 32;
constexpr int ACT_NAN = 255;

struct ActShape { long long T; int F, G; };      // G = groups per row; the int8 rows hold 32 G bytes

// Eight values as they lie in memory, and as float32.
struct Raw16 { uint4 a; };
struct Raw32 { float4 a, b; };
__device__ __forceinline__ void load8(Raw16& r, const __nv_bfloat16* p) { r.a = __ldg(reinterpret_cast<const uint4*>(p)); }
__device__ __forceinline__ void load8(Raw32& r, const float* p) {
    r.a = __ldg(reinterpret_cast<const float4*>(p));
    r.b = __ldg(reinterpret_cast<const float4*>(p) + 1);
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
__device__ __forceinline__ void store8(__nv_bfloat16* p, const float (&x)[8]) {
    *reinterpret_cast<uint4*>(p) = make_uint4(pack_bf16(x[0], x[1]), pack_bf16(x[2], x[3]), pack_bf16(x[4], x[5]), pack_bf16(x[6], x[7]));
}
__device__ __forceinline__ void store8(float* p, const float (&x)[8]) {
    reinterpret_cast<float4*>(p)[0] = make_float4(x[0], x[1], x[2], x[3]);
    reinterpret_cast<float4*>(p)[1] = make_float4(x[4], x[5], x[6], x[7]);
}
__device__ __forceinline__ float load1(const float* p) { return __ldg(p); }
__device__ __forceinline__ float load1(const __nv_bfloat16* p) { return __uint_as_float((unsigned)__ldg(reinterpret_cast<const unsigned short*>(p)) << 16); }
__device__ __forceinline__ void store1(float* p, float x) { *p = x; }
__device__ __forceinline__ void store1(__nv_bfloat16* p, float x) { *p = __float2bfloat16_rn(x); }

// The largest magnitude of eight raw values as float32 bits; a NaN wins over everything.
__device__ __forceinline__ unsigned top_of(const Raw16& r) {
    const auto two = [](unsigned w) { return *reinterpret_cast<const __nv_bfloat162*>(&w); };
    const __nv_bfloat162 m = __hmax2_nan(__hmax2_nan(__habs2(two(r.a.x)), __habs2(two(r.a.y))), __hmax2_nan(__habs2(two(r.a.z)), __habs2(two(r.a.w))));
    const unsigned w = *reinterpret_cast<const unsigned*>(&m);
    return max(w << 16, w & 0xffff0000u);             // bits of non-negative numbers compare like the numbers, NaN above infinity
}
__device__ __forceinline__ unsigned top_of(const Raw32& r) {
    const float x[8] = {r.a.x, r.a.y, r.a.z, r.a.w, r.b.x, r.b.y, r.b.z, r.b.w};
    unsigned top = 0;
#pragma unroll
    for (int j = 0; j < 8; ++j) top = max(top, __float_as_uint(x[j]) & 0x7fffffffu);
    return top;
}
// The scale of a group from its largest magnitude's bits:  max|x| = f 2^k with f in [1, 2), f <= 127/64 asks for e = k - 6, a larger f for k - 5.
struct GroupScale { int byte; float inv; bool fine, over; };
__device__ __forceinline__ GroupScale group_scale(unsigned top) {
    const int want = (int)((top + 0x1ffffu) >> 23) - 127 - 6;      // (the carry out of the mantissa when it is above 0x7e0000)
    const int e = min(max(want, -126), 121);
    GroupScale g;
    g.fine = top < 0x7f800000u;
    g.over = want > 121;                                           // only here |x| / 2^e can exceed 127
    g.byte = g.fine ? e + 127 : ACT_NAN;
    g.inv = __uint_as_float((unsigned)(127 - e) << 23);
    return g;
}
// rint(x inv) in the low byte, ties to even (the addend is 1.5 * 2^23)
__device__ __forceinline__ unsigned quantize(float x, const GroupScale& g) { return __float_as_uint(fmaf(x, g.inv, 12582912.f)); }
__device__ __forceinline__ unsigned quantize_clamped(float x, const GroupScale& g) { return __float_as_uint(fminf(fmaxf(x * g.inv, -127.f), 127.f) + 12582912.f); }

// Eight values (and `top`, their largest magnitude's bits) of a group whose other 24 belong to the three neighbouring lanes (all four
// call) -> int8 and the scale byte.
__device__ __forceinline__ void pack8(const float (&x)[8], unsigned top, uint2& q, int& scale_byte) {
    const unsigned quad = 0xfu << ((threadIdx.y * blockDim.x + threadIdx.x) & 28);   // blockDim.x is a multiple of 4
    top = max(top, __shfl_xor_sync(quad, top, 1));
    top = max(top, __shfl_xor_sync(quad, top, 2));
    const GroupScale g = group_scale(top);
    scale_byte = g.byte;
    unsigned b[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) b[j] = quantize(x[j], g);
    if (g.over) {
#pragma unroll
        for (int j = 0; j < 8; ++j) b[j] = quantize_clamped(x[j], g);
    }
    q.x = __byte_perm(__byte_perm(b[0], b[1], 0x0040), __byte_perm(b[2], b[3], 0x0040), 0x5410);
    q.y = __byte_perm(__byte_perm(b[4], b[5], 0x0040), __byte_perm(b[6], b[7], 0x0040), 0x5410);
    if (!g.fine) q = make_uint2(0u, 0u);
}
__device__ __forceinline__ float scale_of(int byte) { return byte == ACT_NAN ? NAN : __uint_as_float((unsigned)byte << 23); }
__device__ __forceinline__ void unpack8(uint2 q, int scale_byte, float (&x)[8]) {
    const float scale = scale_of(scale_byte);
    const unsigned w[2] = {q.x ^ 0x80808080u, q.y ^ 0x80808080u};          // q + 128 in every byte
    unsigned f[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) f[j] = __byte_perm(w[j / 4], 0x4B000000u, 0x7440 + (j & 3));   // 2^23 + 128 + q
    if (scale_byte < 127 + 100) {                                          // one fma, exact; beyond, 2^23 times the scale would overflow
        const float bias = -(XE_MAGIC + 128.f) * scale;
#pragma unroll
        for (int j = 0; j < 8; ++j) x[j] = fmaf(__uint_as_float(f[j]), scale, bias);
    } else {
#pragma unroll
        for (int j = 0; j < 8; ++j) x[j] = (__uint_as_float(f[j]) - (XE_MAGIC + 128.f)) * scale;
    }
}

__device__ __forceinline__ float rcp(float x) {
    float y;
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
__device__ __forceinline__ float sigmoid(float g) { return rcp(1.f + ex2(-g * LOG2E)); }
// d_gate, d_up and h of one value
__device__ __forceinline__ void gated_backward(float d, float g, float u, float& dg, float& du, float& h) {
    const float sig = sigmoid(g), act = g * sig;
    dg = d * u * fmaf(act, 1.f - sig, sig);
    du = d * act;
    h = act * u;
}

// ---- aligned operands: F a multiple of 8, every operand 16-byte aligned in every row ----
// threadIdx.x (and blockIdx.x) runs over the 4 G units of 8 values of a row, the rest over rows, as many CTAs as are resident at
// once.  A thread keeps D of its rows on their way: it asks for row i + D before it works on row i, so that bytes are
// under way all the time and not only between two bursts of work.  Rows in flight times CTAs per multiprocessor is held
// by registers; the pairs below were the best of six each (forward 156 us with bursts of two rows, 128 us so).
constexpr int PACK_DEPTH = 4, PACK_CTAS = 4, FORWARD_DEPTH = 3, FORWARD_CTAS = 3, BACKWARD_DEPTH = 2, BACKWARD_CTAS = 3;
struct ActCursor { int col; long long row, step; };
__device__ __forceinline__ ActCursor act_cursor() {
    ActCursor c;
    c.col = (blockIdx.x * blockDim.x + threadIdx.x) * 8;
    c.row = (long long)blockIdx.y * blockDim.y + threadIdx.y;
    c.step = (long long)gridDim.y * blockDim.y;
    return c;
}
// Work: a type In with what a thread has of a row, load(In&, row) and work(const In&, row)
template <int D, typename Work>
__device__ __forceinline__ void act_rows(long long T, const ActCursor& c, Work& k) {
    typename Work::In in[D] = {};
#pragma unroll
    for (int i = 0; i < D; ++i) if (c.row + i * c.step < T) k.load(in[i], c.row + i * c.step);
    for (long long r0 = c.row; r0 < T; r0 += D * c.step) {
#pragma unroll
        for (int i = 0; i < D; ++i) {
            const long long r = r0 + i * c.step;
            if (r >= T) return;
            const typename Work::In now = in[i];
            if (r + D * c.step < T) k.load(in[i], r + D * c.step);
            k.work(now, r);
        }
    }
}

template <typename X>
struct PackWork {
    typedef typename RawOf<X>::type In;
    int col, F, G;
    const X* x;
    long long ldx;
    int8_t* q;
    uint8_t* scales;
    __device__ __forceinline__ void load(In& in, long long r) const {
        if (col < F) load8(in, x + r * ldx + col);    // (a unit behind the row's end belongs to the padding of its last group)
    }
    __device__ __forceinline__ void work(const In& in, long long r) const {
        float v[8];
        widen(in, v);
        uint2 b;
        int sb;
        pack8(v, top_of(in), b, sb);
        const long long g = r * G + (col >> 5);
        *reinterpret_cast<uint2*>(q + g * ACT_GROUP + (col & 31)) = b;
        if ((col & 31) == 0) scales[g] = (uint8_t)sb;
    }
};
template <typename X>
__global__ void __launch_bounds__(256, PACK_CTAS) k_act_pack(ActShape s, const X* __restrict__ x, long long ldx, int8_t* __restrict__ q, uint8_t* __restrict__ scales) {
    const ActCursor c = act_cursor();
    if (c.col >= s.G * ACT_GROUP) return;             // whole groups of four lanes leave together
    PackWork<X> k{c.col, s.F, s.G, x, ldx, q, scales};
    act_rows<PACK_DEPTH>(s.T, c, k);
}

struct Kept8 { uint2 b; int scale; };
template <typename X>
struct UnpackWork {
    typedef Kept8 In;
    int col, G;
    const int8_t* q;
    const uint8_t* scales;
    X* x;
    long long ldx;
    __device__ __forceinline__ void load(In& in, long long r) const {
        const long long g = r * G + (col >> 5);
        in.b = __ldg(reinterpret_cast<const uint2*>(q + g * ACT_GROUP + (col & 31)));
        in.scale = __ldg(scales + g);
    }
    __device__ __forceinline__ void work(const In& in, long long r) const {
        float v[8];
        unpack8(in.b, in.scale, v);
        store8(x + r * ldx + col, v);
    }
};
template <typename X>
__global__ void __launch_bounds__(256, PACK_CTAS) k_act_unpack(ActShape s, const int8_t* __restrict__ q, const uint8_t* __restrict__ scales, X* __restrict__ x, long long ldx) {
    grid_trigger();                                   // (before a product in the same call)
    const ActCursor c = act_cursor();
    if (c.col >= s.F) return;
    UnpackWork<X> k{c.col, s.G, q, scales, x, ldx};
    act_rows<PACK_DEPTH>(s.T, c, k);
}

// h = gate sigmoid(gate) up from the unrounded inputs, both inputs packed in the same pass
struct GatedForward {
    const __nv_bfloat16 *gate, *up;
    __nv_bfloat16* h;
    long long ldg, ldu, ldh;
    int8_t *qg, *qu;
    uint8_t *sg, *su;
};
struct ForwardWork {
    struct In { Raw16 g, u; };
    int col, F, G;
    const GatedForward& a;
    __device__ __forceinline__ void load(In& in, long long r) const {
        if (col >= F) return;
        load8(in.g, a.gate + r * a.ldg + col);
        load8(in.u, a.up + r * a.ldu + col);
    }
    __device__ __forceinline__ void work(const In& in, long long r) const {
        float x[8], u[8], y[8];
        widen(in.g, x);
        widen(in.u, u);
#pragma unroll
        for (int j = 0; j < 8; ++j) y[j] = x[j] * sigmoid(x[j]) * u[j];
        if (col < F) store8(a.h + r * a.ldh + col, y);
        const long long g = r * G + (col >> 5), at = g * ACT_GROUP + (col & 31);
        uint2 b;
        int sb;
        pack8(x, top_of(in.g), b, sb);
        *reinterpret_cast<uint2*>(a.qg + at) = b;
        if ((col & 31) == 0) a.sg[g] = (uint8_t)sb;
        pack8(u, top_of(in.u), b, sb);
        *reinterpret_cast<uint2*>(a.qu + at) = b;
        if ((col & 31) == 0) a.su[g] = (uint8_t)sb;
    }
};
__global__ void __launch_bounds__(256, FORWARD_CTAS) k_swiglu_forward(ActShape s, const __grid_constant__ GatedForward a) {
    const ActCursor c = act_cursor();
    if (c.col >= s.G * ACT_GROUP) return;
    ForwardWork k{c.col, s.F, s.G, a};
    act_rows<FORWARD_DEPTH>(s.T, c, k);
}

// d_gate = dh up s (1 + gate (1 - s)),  d_up = dh gate s,  h = gate s up  (s = sigmoid(gate)), gate and up from their checkpoints
struct GatedBackward {
    const __nv_bfloat16* dh;
    const int8_t *qg, *qu;
    const uint8_t *sg, *su;
    __nv_bfloat16 *dg, *du, *h;
    long long lddh, lddg, lddu, ldh;
};
template <bool H>
struct BackwardWork {
    struct In { Raw16 d; Kept8 g, u; };
    int col, G;
    const GatedBackward& a;
    __device__ __forceinline__ void load(In& in, long long r) const {
        const long long g = r * G + (col >> 5), at = g * ACT_GROUP + (col & 31);
        load8(in.d, a.dh + r * a.lddh + col);
        in.g.b = __ldg(reinterpret_cast<const uint2*>(a.qg + at));
        in.u.b = __ldg(reinterpret_cast<const uint2*>(a.qu + at));
        in.g.scale = __ldg(a.sg + g);
        in.u.scale = __ldg(a.su + g);
    }
    __device__ __forceinline__ void work(const In& in, long long r) const {
        float d[8], x[8], u[8], o[8], p[8], y[8];
        widen(in.d, d);
        unpack8(in.g.b, in.g.scale, x);
        unpack8(in.u.b, in.u.scale, u);
#pragma unroll
        for (int j = 0; j < 8; ++j) gated_backward(d[j], x[j], u[j], o[j], p[j], y[j]);
        store8(a.dg + r * a.lddg + col, o);
        store8(a.du + r * a.lddu + col, p);
        if (H) store8(a.h + r * a.ldh + col, y);
    }
};
template <bool H>
__global__ void __launch_bounds__(256, BACKWARD_CTAS) k_swiglu_backward(ActShape s, const __grid_constant__ GatedBackward a) {
    const ActCursor c = act_cursor();
    if (c.col >= s.F) return;
    BackwardWork<H> k{c.col, s.G, a};
    act_rows<BACKWARD_DEPTH>(s.T, c, k);
}

// ---- any length and alignment: a lane per value, a warp per group, LANE_GROUPS groups of a row at a time ----
// blockDim = (32, 8); blockIdx.x, threadIdx.y: groups of a row, blockIdx.y: rows
constexpr int LANE_GROUPS = 4;
template <typename Body>
__device__ __forceinline__ void lane_groups(const ActShape& s, Body&& body) {
    const int g0 = (blockIdx.x * 8 + threadIdx.y) * LANE_GROUPS;
    if (g0 >= s.G) return;
    for (long long r = blockIdx.y; r < s.T; r += gridDim.y) body(r, g0);
}
// the checkpoint of LANE_GROUPS groups whose values the lanes hold (zeros behind the row's end)
__device__ __forceinline__ void pack_lanes(const float (&x)[LANE_GROUPS], long long row_group, int g0, int G, int8_t* q, uint8_t* scales) {
#pragma unroll
    for (int i = 0; i < LANE_GROUPS; ++i) {
        if (g0 + i >= G) break;
        const GroupScale s = group_scale(__reduce_max_sync(0xffffffffu, __float_as_uint(x[i]) & 0x7fffffffu));
        const unsigned b = s.over ? quantize_clamped(x[i], s) : quantize(x[i], s);
        q[(row_group + i) * ACT_GROUP + threadIdx.x] = (int8_t)(s.fine ? b & 0xffu : 0u);
        if (threadIdx.x == 0) scales[row_group + i] = (uint8_t)s.byte;
    }
}
template <typename X>
__global__ void __launch_bounds__(256) k_act_pack_any(ActShape s, const X* __restrict__ x, long long ldx, int8_t* __restrict__ q, uint8_t* __restrict__ scales) {
    lane_groups(s, [&](long long r, int g0) {
        float v[LANE_GROUPS];
#pragma unroll
        for (int i = 0; i < LANE_GROUPS; ++i) {
            const int col = (g0 + i) * ACT_GROUP + threadIdx.x;
            v[i] = col < s.F ? load1(x + r * ldx + col) : 0.f;
        }
        pack_lanes(v, r * s.G + g0, g0, s.G, q, scales);
    });
}
template <typename X>
__global__ void __launch_bounds__(256) k_act_unpack_any(ActShape s, const int8_t* __restrict__ q, const uint8_t* __restrict__ scales, X* __restrict__ x, long long ldx) {
    lane_groups(s, [&](long long r, int g0) {
        float v[LANE_GROUPS];
#pragma unroll
        for (int i = 0; i < LANE_GROUPS; ++i) {
            const long long g = r * s.G + min(g0 + i, s.G - 1);
            v[i] = (float)__ldg(q + g * ACT_GROUP + threadIdx.x) * scale_of(__ldg(scales + g));
        }
#pragma unroll
        for (int i = 0; i < LANE_GROUPS; ++i) {
            const int col = (g0 + i) * ACT_GROUP + threadIdx.x;
            if (col < s.F) store1(x + r * ldx + col, v[i]);
        }
    });
}
__global__ void __launch_bounds__(256) k_swiglu_forward_any(ActShape s, const __grid_constant__ GatedForward a) {
    lane_groups(s, [&](long long r, int g0) {
        float x[LANE_GROUPS], u[LANE_GROUPS];
#pragma unroll
        for (int i = 0; i < LANE_GROUPS; ++i) {
            const int col = (g0 + i) * ACT_GROUP + threadIdx.x;
            x[i] = col < s.F ? load1(a.gate + r * a.ldg + col) : 0.f;
            u[i] = col < s.F ? load1(a.up + r * a.ldu + col) : 0.f;
        }
#pragma unroll
        for (int i = 0; i < LANE_GROUPS; ++i) {
            const int col = (g0 + i) * ACT_GROUP + threadIdx.x;
            if (col < s.F) store1(a.h + r * a.ldh + col, x[i] * sigmoid(x[i]) * u[i]);
        }
        pack_lanes(x, r * s.G + g0, g0, s.G, a.qg, a.sg);
        pack_lanes(u, r * s.G + g0, g0, s.G, a.qu, a.su);
    });
}
template <bool H>
__global__ void __launch_bounds__(256) k_swiglu_backward_any(ActShape s, const __grid_constant__ GatedBackward a) {
    lane_groups(s, [&](long long r, int g0) {
        float d[LANE_GROUPS], x[LANE_GROUPS], u[LANE_GROUPS];
#pragma unroll
        for (int i = 0; i < LANE_GROUPS; ++i) {
            const int col = (g0 + i) * ACT_GROUP + threadIdx.x;
            const long long g = r * s.G + min(g0 + i, s.G - 1);
            d[i] = col < s.F ? load1(a.dh + r * a.lddh + col) : 0.f;
            x[i] = (float)__ldg(a.qg + g * ACT_GROUP + threadIdx.x) * scale_of(__ldg(a.sg + g));
            u[i] = (float)__ldg(a.qu + g * ACT_GROUP + threadIdx.x) * scale_of(__ldg(a.su + g));
        }
#pragma unroll
        for (int i = 0; i < LANE_GROUPS; ++i) {
            const int col = (g0 + i) * ACT_GROUP + threadIdx.x;
            float o, p, y;
            gated_backward(d[i], x[i], u[i], o, p, y);
            if (col < s.F) {
                store1(a.dg + r * a.lddg + col, o);
                store1(a.du + r * a.lddu + col, p);
                if (H) store1(a.h + r * a.ldh + col, y);
            }
        }
    });
}

// rows of 16-bit values to another alignment and row stride
__global__ void __launch_bounds__(256) k_copy_rows(ActShape s, const unsigned short* __restrict__ src, long long lds, unsigned short* __restrict__ dst, long long ldd) {
    lane_groups(s, [&](long long r, int g0) {
        unsigned short v[LANE_GROUPS];
#pragma unroll
        for (int i = 0; i < LANE_GROUPS; ++i) {
            const int col = (g0 + i) * ACT_GROUP + threadIdx.x;
            v[i] = col < s.F ? __ldg(src + r * lds + col) : (unsigned short)0;
        }
#pragma unroll
        for (int i = 0; i < LANE_GROUPS; ++i) {
            const int col = (g0 + i) * ACT_GROUP + threadIdx.x;
            if (col < s.F) dst[r * ldd + col] = v[i];
        }
    });
}

}  // namespace psgd
