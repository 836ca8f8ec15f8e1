// What the kernels of the training operators do with single values: loads and stores of eight at a time, rows of any alignment, the 8-bit form of a group of
// 32, dependent launches.  No kernels here: several translation units include it.
#pragma once
#include <cuda_bf16.h>
#include <cuda_runtime.h>
#include <stdint.h>

namespace psgd {

// Dependent launches: a kernel may start while the one before it on the stream still runs (its set-up and its CTAs' start then cost nothing); `grid_wait`
// returns when that one has finished and its writes are visible, so everything that touches global memory comes after it, and nothing
// is loaded through the read-only path, which expects memory that no one writes while the kernel lives.  `grid_trigger` lets the next start.
__device__ __forceinline__ void grid_wait() { asm volatile("griddepcontrol.wait;\n" ::: "memory"); }
__device__ __forceinline__ void grid_trigger() { asm volatile("griddepcontrol.launch_dependents;\n" ::: "memory"); }

// Division by a launch constant: q = n * mul >> shift for 0 <= n < 2^31 (mul = floor(2^shift / d) + 1, shift = 31 + ceil(log2 d)).
struct FastDiv { unsigned mul, shift; };
inline FastDiv fast_div(unsigned d) {
    unsigned l = 0;
    while ((1ull << l) < d) ++l;
    return {(unsigned)(((unsigned long long)1 << (31 + l)) / d + 1), 31 + l};
}
__device__ __forceinline__ int operator/(int n, FastDiv d) { return (int)(((unsigned long long)(unsigned)n * d.mul) >> d.shift); }

constexpr float LOG2E = 1.4426950408889634f;
constexpr float XE_MAGIC = 8388608.f;         // 2^23: adding it leaves the rounded whole number in the low mantissa bits

__device__ __forceinline__ float ex2(float x) {
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
__device__ __forceinline__ unsigned pack_bf16(float lo, float hi) {
    __nv_bfloat162 h = __floats2bfloat162_rn(lo, hi);
    return *reinterpret_cast<unsigned*>(&h);
}

constexpr int ACT_GROUP = 32;
constexpr int ACT_NAN = 255;

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

// the checkpoint of a thread's eight values, row group g
__device__ __forceinline__ void keep8(const float (&x)[8], unsigned top, long long g, int col, bool live, int8_t* q, uint8_t* scales) {
    uint2 b;
    int sb;
    pack8(x, top, b, sb);
    if (!live) return;
    *reinterpret_cast<uint2*>(q + g * ACT_GROUP + (col & 31)) = b;
    if ((col & 31) == 0) scales[g] = (uint8_t)sb;
}

}  // namespace psgd
