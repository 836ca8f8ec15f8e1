// Activation checkpoints in 8 bits, and the gated unit of the feed-forward block with its two inputs kept that way.
//
// A checkpoint of a matrix [T][F] holds, per row and group of 32 values, one scale 2^e (e the smallest integer with
// max|x| <= 127 * 2^e, kept within -126..121, stored as the byte e + 127; 255 marks a group with an infinity or a NaN, which
// stands for NaN) and the whole numbers rint(x / 2^e) within -127..127 as int8, rows padded with zeros to whole groups:
// 1 + 1/32 bytes per value.  With a power of two as scale every stored value is exact in bfloat16, so that
// products of checkpoints run on the tensor cores without another rounding.
//
// All kernels here are one pass over their operands and bound by HBM.  A thread moves 8 values (16 bytes of bfloat16, 8 of int8), four
// neighbouring threads share a group, and the group's maximum is two shuffles.  Rows of bfloat16 of any other length or alignment (ANY): a warp
// takes 256 values of a row, loads and stores the aligned 16-byte units that they lie in, and shifts between those and
// its lanes' values with shuffles (in) and through shared memory (out).  Float32 rows without alignment: a lane per value.
//
// Measured (8.06, 10.06, 3.03 and 3.03 bytes per value; of the 6533 GB/s of a copy), 16384 x 5504: gated unit forward 128 us (87 %), backward with h
// 151 us (91 %), pack 54 us (77 %; float32, 5.03 bytes: 70 us, 99 %), unpack 47 us (89 %).  16384 x 5461: 201, 213, 74 and 61 us, bound by instructions (a lane per value
// there: 313, 320, 112 and 147 us; value-by-value stores at the ends of each warp's part instead of shared memory: 333 and 343 us).
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
__device__ __forceinline__ void load8(Raw16& r, const __nv_bfloat16* p) { r.a = *reinterpret_cast<const uint4*>(p); }
__device__ __forceinline__ void load8(Raw32& r, const float* p) {
    r.a = *reinterpret_cast<const float4*>(p);
    r.b = reinterpret_cast<const float4*>(p)[1];
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
__device__ __forceinline__ uint4 pack_bf16x8(const float (&x)[8]) {
    return make_uint4(pack_bf16(x[0], x[1]), pack_bf16(x[2], x[3]), pack_bf16(x[4], x[5]), pack_bf16(x[6], x[7]));
}
__device__ __forceinline__ void store8(__nv_bfloat16* p, const float (&x)[8]) {
    *reinterpret_cast<uint4*>(p) = pack_bf16x8(x);
}
__device__ __forceinline__ void store8(float* p, const float (&x)[8]) {
    reinterpret_cast<float4*>(p)[0] = make_float4(x[0], x[1], x[2], x[3]);
    reinterpret_cast<float4*>(p)[1] = make_float4(x[4], x[5], x[6], x[7]);
}

// Rows of bfloat16 that start at any even address.  The lanes of a warp (256 values of a row) load the aligned 16-byte units that its values lie
// in, lane 31 also the 33rd; a lane's eight values are cut out of its own and the next lane's unit when they are used.
struct RawAny { uint4 a, b; };
__device__ __forceinline__ unsigned shift_of(const __nv_bfloat16* p) { return (unsigned)reinterpret_cast<uintptr_t>(p) & 15u; }
// The unit at halfword `at` of a row (from 1 - 8 on), `len` halfwords long.  `inner`: seven halfwords on either side of the row belong to the matrix
// too and may come along; else only the row's own values are read, the others are zeros.
__device__ __forceinline__ void load_unit(uint4& u, const __nv_bfloat16* row, int at, int len, bool inner) {
    if (at >= len) return;
    if (inner) {
        u = *reinterpret_cast<const uint4*>(row + at);
        return;
    }
    const unsigned short* h = reinterpret_cast<const unsigned short*>(row);
    unsigned w[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int j = at + 2 * i;
        const unsigned x = j >= 0 && j < len ? h[j] : 0u, y = j + 1 >= 0 && j + 1 < len ? h[j + 1] : 0u;
        w[i] = x | y << 16;
    }
    u = make_uint4(w[0], w[1], w[2], w[3]);
}
// 16 bytes of a and b from byte `sh` (even, below 16) on
__device__ __forceinline__ uint4 cut_out(const uint4& a, const uint4& b, unsigned sh) {
    const unsigned w[8] = {a.x, a.y, a.z, a.w, b.x, b.y, b.z, b.w};
    unsigned t[6], u[5];
#pragma unroll
    for (int i = 0; i < 6; ++i) t[i] = sh & 8 ? w[i + 2] : w[i];
#pragma unroll
    for (int i = 0; i < 5; ++i) u[i] = sh & 4 ? t[i + 1] : t[i];
    const unsigned bits = (sh & 2) * 8;
    return make_uint4(__funnelshift_r(u[0], u[1], bits), __funnelshift_r(u[1], u[2], bits), __funnelshift_r(u[2], u[3], bits), __funnelshift_r(u[3], u[4], bits));
}
// A lane's eight values to p; the lanes of a warp hold a row's values one after the other, `valid` of which exist from lane 0 on (all lanes call).
// The warp's bytes go through shared memory, laid out there as they fall on 16-byte units in memory: whole units are written as such, the
// one or two that belong to the warp in part value by value.
constexpr int ANY_UNITS = 34;
__device__ __forceinline__ void store_any(__nv_bfloat16* p, const uint4& v, int valid, uint4* image) {
    const int lane = threadIdx.x & 31;                // blockDim.x is a multiple of 32
    const unsigned sh = shift_of(p);                  // the same in all lanes
    unsigned* word = reinterpret_cast<unsigned*>(image) + sh / 4 + 4 * lane;
    if (sh & 2) {                                     // halves of words: the lane before has the first one
        const unsigned before = __shfl_up_sync(0xffffffffu, v.w, 1);
        word[0] = __funnelshift_r(before, v.x, 16);
        word[1] = __funnelshift_r(v.x, v.y, 16);
        word[2] = __funnelshift_r(v.y, v.z, 16);
        word[3] = __funnelshift_r(v.z, v.w, 16);
        if (lane == 31) word[4] = v.w >> 16;
    } else {
        word[0] = v.x;
        word[1] = v.y;
        word[2] = v.z;
        word[3] = v.w;
    }
    __syncwarp();
    const int from = (int)sh, to = from + 2 * valid;  // bytes of the image that exist
    unsigned char* out = reinterpret_cast<unsigned char*>(p) - sh - 16 * lane;
    if (16 * lane >= from && 16 * lane + 16 <= to) *reinterpret_cast<uint4*>(out + 16 * lane) = image[lane];
    const int last = to / 16;                         // lanes 0-7: the first unit, where it begins before the warp; 8-15: the last, where it ends behind it
    const int at = (lane < 8 ? 0 : 16 * last) + 2 * (lane & 7);
    if (lane < 16 && (lane < 8 ? from > 0 : last > 0 || from == 0) && at >= from && at < to)
        *reinterpret_cast<unsigned short*>(out + at) = reinterpret_cast<const unsigned short*>(image)[at / 2];
    __syncwarp();
}

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
// 0 for g below -87.3, where it is less than 2^-126 (in float32 arithmetic 1 + exp(-g) is infinite from -88.7 on): g sigmoid(g) is off by less than 1.1e-36 there.
__device__ __forceinline__ float sigmoid(float g) { return rcp(1.f + ex2(-g * LOG2E)); }
// d_gate, d_up and h of one value
__device__ __forceinline__ void gated_backward(float d, float g, float u, float& dg, float& du, float& h) {
    const float sig = sigmoid(g), act = g * sig;
    dg = d * u * fmaf(act, 1.f - sig, sig);
    du = d * act;
    h = act * u;
}

// ---- eight values per thread ----
// threadIdx.x (and blockIdx.x) runs over the 4 G units of 8 values of a row, the rest over rows, as many CTAs as are resident at
// once.  A thread keeps D of its rows on their way: it asks for row i + D before it works on row i, so that bytes are
// under way all the time and not only between two bursts of work.  Rows in flight times CTAs per multiprocessor is held
// by registers; the pairs below were the best of six each (forward 156 us with bursts of two rows, 128 us so).  Rows of any alignment need
// their registers for the cutting: one row on its way (16384 x 5461, forward and backward: 201 and 213 us, with two 298 and 241).
constexpr int PACK_DEPTH = 4, PACK32_DEPTH = 2, PACK_CTAS = 4, FORWARD_DEPTH = 3, FORWARD_CTAS = 3, BACKWARD_DEPTH = 2, BACKWARD_CTAS = 3;
struct ActCursor { int col; long long row, step; };
__device__ __forceinline__ ActCursor act_cursor() {
    grid_trigger();
    grid_wait();
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

// What a thread has of a row of bfloat16, and where its values go: aligned rows (ANY false), or rows of any length and alignment, whose warps stay
// within a row (blockDim.x a multiple of 32) and keep all their lanes.
template <bool ANY> struct Row16 {
    typedef Raw16 Raw;
    const __nv_bfloat16* p;
    long long ld;
    int F;
    __device__ __forceinline__ Row16(const __nv_bfloat16* p, long long ld, long long, int F) : p(p), ld(ld), F(F) {}
    __device__ __forceinline__ void load(Raw& r, long long row, int col) const {
        if (col < F) load8(r, p + row * ld + col);    // (a unit behind the row's end belongs to the padding of its last group)
    }
    __device__ __forceinline__ Raw16 values(const Raw& r, long long, int) const { return r; }
};
template <> struct Row16<true> {
    typedef RawAny Raw;
    const __nv_bfloat16* p;
    long long ld, rows;
    int F, edge;                                      // edge: rows at either end of the matrix that are not inner ones
    __device__ __forceinline__ Row16(const __nv_bfloat16* p, long long ld, long long rows, int F) : p(p), ld(ld), rows(rows), F(F), edge(ld >= 7 ? 1 : 7) {}
    __device__ __forceinline__ void load(Raw& r, long long row, int col) const {
        const __nv_bfloat16* x = p + row * ld;
        const int at = col - (int)shift_of(x) / 2;
        const bool inner = row >= edge && row + edge < rows;
        load_unit(r.a, x, at, F, inner);
        if ((threadIdx.x & 31) == 31) load_unit(r.b, x, at + 8, F, inner);
    }
    __device__ __forceinline__ Raw16 values(const Raw& r, long long row, int col) const {
        uint4 next = make_uint4(__shfl_down_sync(0xffffffffu, r.a.x, 1), __shfl_down_sync(0xffffffffu, r.a.y, 1), __shfl_down_sync(0xffffffffu, r.a.z, 1),
                                __shfl_down_sync(0xffffffffu, r.a.w, 1));
        if ((threadIdx.x & 31) == 31) next = r.b;
        uint4 v = cut_out(r.a, next, shift_of(p + row * ld));
        const int n = F - col;
        if (n < 8) {                                  // zeros behind the row's end
            unsigned w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
            for (int i = 0; i < 4; ++i) w[i] = n > 2 * i + 1 ? w[i] : n > 2 * i ? w[i] & 0xffffu : 0u;
            v = make_uint4(w[0], w[1], w[2], w[3]);
        }
        return {v};
    }
};
// n: how many of the thread's eight values exist; of its warp's, if ANY
template <bool ANY>
__device__ __forceinline__ void store16(__nv_bfloat16* p, const float (&x)[8], int n, uint4* image) {
    if (ANY) store_any(p, pack_bf16x8(x), n, image);
    else if (n > 0) store8(p, x);
}
__device__ __forceinline__ int valid_of(int F, int col, int of) { return min(max(F - col, 0), of); }
template <bool ANY>
__device__ __forceinline__ int valid_out(int F, int col) { return ANY ? valid_of(F, col & ~255, 256) : valid_of(F, col, 8); }
template <bool ANY>
__device__ __forceinline__ uint4* warp_image() {
    __shared__ uint4 image[ANY ? 8 * ANY_UNITS : 1];
    return ANY ? image + ((threadIdx.y * blockDim.x + threadIdx.x) >> 5) * ANY_UNITS : nullptr;
}
// the checkpoint of a thread's eight values, row group g
__device__ __forceinline__ void keep8(const float (&x)[8], unsigned top, long long g, int col, bool live, int8_t* q, uint8_t* scales) {
    uint2 b;
    int sb;
    pack8(x, top, b, sb);
    if (!live) return;
    *reinterpret_cast<uint2*>(q + g * ACT_GROUP + (col & 31)) = b;
    if ((col & 31) == 0) scales[g] = (uint8_t)sb;
}

template <bool ANY>
struct PackWork16 {
    typedef typename Row16<ANY>::Raw In;
    int col, G;
    Row16<ANY> x;
    int8_t* q;
    uint8_t* scales;
    __device__ __forceinline__ void load(In& in, long long r) const {
        x.load(in, r, col);
    }
    __device__ __forceinline__ void work(const In& in, long long r) const {
        const Raw16 raw = x.values(in, r, col);
        float v[8];
        widen(raw, v);
        keep8(v, top_of(raw), r * G + (col >> 5), col, col < G * ACT_GROUP, q, scales);
    }
};
struct PackWork32 {
    typedef Raw32 In;
    int col, F, G;
    const float* x;
    long long ldx;
    int8_t* q;
    uint8_t* scales;
    __device__ __forceinline__ void load(In& in, long long r) const {
        if (col < F) load8(in, x + r * ldx + col);
    }
    __device__ __forceinline__ void work(const In& in, long long r) const {
        float v[8];
        widen(in, v);
        keep8(v, top_of(in), r * G + (col >> 5), col, true, q, scales);
    }
};
template <bool ANY>
__global__ void __launch_bounds__(256, PACK_CTAS) k_act_pack(ActShape s, const __nv_bfloat16* x, long long ldx, int8_t* q, uint8_t* scales) {
    const ActCursor c = act_cursor();
    if (!ANY && c.col >= s.G * ACT_GROUP) return;     // whole groups of four lanes leave together
    PackWork16<ANY> k{c.col, s.G, Row16<ANY>(x, ldx, s.T, s.F), q, scales};
    act_rows<ANY ? 1 : PACK_DEPTH>(s.T, c, k);
}
__global__ void __launch_bounds__(256, PACK_CTAS) k_act_pack32(ActShape s, const float* x, long long ldx, int8_t* q, uint8_t* scales) {
    const ActCursor c = act_cursor();
    if (c.col >= s.G * ACT_GROUP) return;
    PackWork32 k{c.col, s.F, s.G, x, ldx, q, scales};
    act_rows<PACK32_DEPTH>(s.T, c, k);
}

struct Kept8 { uint2 b; int scale; };
__device__ __forceinline__ void load_kept(Kept8& k, const int8_t* q, const uint8_t* scales, long long g, int col) {
    k.b = *reinterpret_cast<const uint2*>(q + g * ACT_GROUP + (col & 31));
    k.scale = scales[g];
}
template <typename X, bool ANY>
struct UnpackWork {
    typedef Kept8 In;
    int col, out, G;
    const int8_t* q;
    const uint8_t* scales;
    X* x;
    long long ldx;
    uint4* image;
    __device__ __forceinline__ void load(In& in, long long r) const {
        if (col < G * ACT_GROUP) load_kept(in, q, scales, r * G + (col >> 5), col);
    }
    __device__ __forceinline__ void work(const In& in, long long r) const {
        float v[8];
        unpack8(in.b, in.scale, v);
        if constexpr (sizeof(X) == 2) store16<ANY>(x + r * ldx + col, v, out, image);
        else store8(x + r * ldx + col, v);
    }
};
template <typename X, bool ANY>
__global__ void __launch_bounds__(256, PACK_CTAS) k_act_unpack(ActShape s, const int8_t* q, const uint8_t* scales, X* x, long long ldx) {
    const ActCursor c = act_cursor();
    if (!ANY && c.col >= s.F) return;
    UnpackWork<X, ANY> k{c.col, valid_out<ANY>(s.F, c.col), s.G, q, scales, x, ldx, warp_image<ANY>()};
    act_rows<ANY ? 1 : PACK_DEPTH>(s.T, c, k);
}

// h = gate sigmoid(gate) up from the unrounded inputs, both inputs packed in the same pass
struct GatedForward {
    const __nv_bfloat16 *gate, *up;
    __nv_bfloat16* h;
    long long ldg, ldu, ldh;
    int8_t *qg, *qu;
    uint8_t *sg, *su;
};
template <bool ANY>
struct ForwardWork {
    struct In { typename Row16<ANY>::Raw g, u; };
    int col, out, G;
    Row16<ANY> gate, up;
    const GatedForward& a;
    uint4* image;
    __device__ __forceinline__ void load(In& in, long long r) const {
        gate.load(in.g, r, col);
        up.load(in.u, r, col);
    }
    __device__ __forceinline__ void work(const In& in, long long r) const {
        const Raw16 rg = gate.values(in.g, r, col), ru = up.values(in.u, r, col);
        float x[8], u[8], y[8];
        widen(rg, x);
        widen(ru, u);
#pragma unroll
        for (int j = 0; j < 8; ++j) y[j] = x[j] * sigmoid(x[j]) * u[j];
        store16<ANY>(a.h + r * a.ldh + col, y, out, image);
        const long long g = r * G + (col >> 5);
        const bool live = !ANY || col < G * ACT_GROUP;
        keep8(x, top_of(rg), g, col, live, a.qg, a.sg);
        keep8(u, top_of(ru), g, col, live, a.qu, a.su);
    }
};
template <bool ANY>
__global__ void __launch_bounds__(256, FORWARD_CTAS) k_swiglu_forward(ActShape s, const __grid_constant__ GatedForward a) {
    const ActCursor c = act_cursor();
    if (!ANY && c.col >= s.G * ACT_GROUP) return;
    ForwardWork<ANY> k{c.col, valid_out<ANY>(s.F, c.col), s.G, Row16<ANY>(a.gate, a.ldg, s.T, s.F), Row16<ANY>(a.up, a.ldu, s.T, s.F), a, warp_image<ANY>()};
    act_rows<ANY ? 1 : FORWARD_DEPTH>(s.T, c, k);
}

// d_gate = dh up s (1 + gate (1 - s)),  d_up = dh gate s,  h = gate s up  (s = sigmoid(gate)), gate and up from their checkpoints
struct GatedBackward {
    const __nv_bfloat16* dh;
    const int8_t *qg, *qu;
    const uint8_t *sg, *su;
    __nv_bfloat16 *dg, *du, *h;
    long long lddh, lddg, lddu, ldh;
};
template <bool H, bool ANY>
struct BackwardWork {
    struct In { typename Row16<ANY>::Raw d; Kept8 g, u; };
    int col, out, G;
    Row16<ANY> dh;
    const GatedBackward& a;
    uint4* image;
    __device__ __forceinline__ void load(In& in, long long r) const {
        dh.load(in.d, r, col);
        if (col >= G * ACT_GROUP) return;
        const long long g = r * G + (col >> 5);
        load_kept(in.g, a.qg, a.sg, g, col);
        load_kept(in.u, a.qu, a.su, g, col);
    }
    __device__ __forceinline__ void work(const In& in, long long r) const {
        float d[8], x[8], u[8], o[8], p[8], y[8];
        widen(dh.values(in.d, r, col), d);
        unpack8(in.g.b, in.g.scale, x);
        unpack8(in.u.b, in.u.scale, u);
#pragma unroll
        for (int j = 0; j < 8; ++j) gated_backward(d[j], x[j], u[j], o[j], p[j], y[j]);
        store16<ANY>(a.dg + r * a.lddg + col, o, out, image);
        store16<ANY>(a.du + r * a.lddu + col, p, out, image);
        if (H) store16<ANY>(a.h + r * a.ldh + col, y, out, image);
    }
};
template <bool H, bool ANY>
__global__ void __launch_bounds__(256, BACKWARD_CTAS) k_swiglu_backward(ActShape s, const __grid_constant__ GatedBackward a) {
    const ActCursor c = act_cursor();
    if (!ANY && c.col >= s.F) return;
    BackwardWork<H, ANY> k{c.col, valid_out<ANY>(s.F, c.col), s.G, Row16<ANY>(a.dh, a.lddh, s.T, s.F), a, warp_image<ANY>()};
    act_rows<ANY ? 1 : BACKWARD_DEPTH>(s.T, c, k);
}

// rows of 16-bit values to another alignment and row stride
struct CopyWork {
    typedef RawAny In;
    int col, out;
    Row16<true> src;
    __nv_bfloat16* dst;
    long long ldd;
    uint4* image;
    __device__ __forceinline__ void load(In& in, long long r) const { src.load(in, r, col); }
    __device__ __forceinline__ void work(const In& in, long long r) const { store_any(dst + r * ldd + col, src.values(in, r, col).a, out, image); }
};
__global__ void __launch_bounds__(256, PACK_CTAS) k_copy_rows(ActShape s, const __nv_bfloat16* src, long long lds, __nv_bfloat16* dst, long long ldd) {
    const ActCursor c = act_cursor();
    CopyWork k{c.col, valid_out<true>(s.F, c.col), Row16<true>(src, lds, s.T, s.F), dst, ldd, warp_image<true>()};
    act_rows<1>(s.T, c, k);
}

// ---- float32 rows of any length and alignment: a lane per value, a warp per group, LANE_GROUPS groups of a row at a time ----
// blockDim = (32, 8); blockIdx.x, threadIdx.y: groups of a row, blockIdx.y: rows
constexpr int LANE_GROUPS = 4;
template <typename Body>
__device__ __forceinline__ void lane_groups(const ActShape& s, Body&& body) {
    grid_trigger();
    grid_wait();
    const int g0 = (blockIdx.x * 8 + threadIdx.y) * LANE_GROUPS;
    if (g0 >= s.G) return;
    for (long long r = blockIdx.y; r < s.T; r += gridDim.y) body(r, g0);
}
__global__ void __launch_bounds__(256) k_act_pack32_any(ActShape s, const float* x, long long ldx, int8_t* q, uint8_t* scales) {
    lane_groups(s, [&](long long r, int g0) {
        float v[LANE_GROUPS];
#pragma unroll
        for (int i = 0; i < LANE_GROUPS; ++i) {
            const int col = (g0 + i) * ACT_GROUP + threadIdx.x;
            v[i] = col < s.F ? x[r * ldx + col] : 0.f;             // zeros behind the row's end
        }
#pragma unroll
        for (int i = 0; i < LANE_GROUPS; ++i) {
            if (g0 + i >= s.G) break;
            const long long g = r * s.G + g0 + i;
            const GroupScale gs = group_scale(__reduce_max_sync(0xffffffffu, __float_as_uint(v[i]) & 0x7fffffffu));
            const unsigned b = gs.over ? quantize_clamped(v[i], gs) : quantize(v[i], gs);
            q[g * ACT_GROUP + threadIdx.x] = (int8_t)(gs.fine ? b & 0xffu : 0u);
            if (threadIdx.x == 0) scales[g] = (uint8_t)gs.byte;
        }
    });
}
__global__ void __launch_bounds__(256) k_act_unpack32_any(ActShape s, const int8_t* q, const uint8_t* scales, float* x, long long ldx) {
    lane_groups(s, [&](long long r, int g0) {
        float v[LANE_GROUPS];
#pragma unroll
        for (int i = 0; i < LANE_GROUPS; ++i) {
            const long long g = r * s.G + min(g0 + i, s.G - 1);
            v[i] = (float)q[g * ACT_GROUP + threadIdx.x] * scale_of(scales[g]);
        }
#pragma unroll
        for (int i = 0; i < LANE_GROUPS; ++i) {
            const int col = (g0 + i) * ACT_GROUP + threadIdx.x;
            if (col < s.F) x[r * ldx + col] = v[i];
        }
    });
}

}  // namespace psgd
