// Layer norm of rows (also without centring), forward and backward.
//
//   s = x + r (rounded to x's type; s = x without r),  m = mean(s) (0 without centring),  f = 1 / sqrt(mean((s - m)^2) + eps),
//   y = (s - m) f w + b;
//   g = dy w,  xh = (s - m) f,  ds = f (g - mean(g) - xh mean(g xh)) + what reaches s from elsewhere  (mean(g) only with centring),
//   dw = sum over rows of dy xh,  db = sum over rows of dy.
//
// One pass over the operands, bound by HBM.  A warp, or as many warps as a row needs (blockDim.x threads, blockDim.y rows side by side), hold a row in registers, VPT units
// of eight values per thread.  The sum of squares is taken about the warp's own mean and the warps' results are joined exactly (squares about the joint mean =
// sum of the warps' squares + n_w (mean_w - mean)^2), so that a large mean costs no bits and a row takes one exchange between its warps, none where a warp
// has it alone.  The CTAs stay and walk over the rows: weights are read once into shared memory, and in the backward pass every thread sums dw and db of its
// columns over its rows; the CTA adds its rows' sums, k_norm_join those of the CTAs, in a fixed order.
//
// Rows of whole 16-byte units come through a ring in shared memory: every thread copies its own units of the rows to come asynchronously (cp.async) and reads back only
// what it copied itself, so that there is nothing to wait for but its own copies, rows are under way whatever the registers hold, and the backward pass
// reads a row a second time from there.  Rows of bfloat16 of any other width or alignment go the same way where all operands lie alike (PHASE: matrices of one odd width, for
// instance): the units are then those of memory, and a CTA takes rows that begin at the same place in them.  Anything else (.._any): a value per lane, the next row's values in
// registers.  16384 x 2051 with a residual: 61 us forward and 74 backward (with a second gradient) by units, 103 and 115 by lanes.
// Sums and statistics are float32.  Rounded once: s to x's type, y, ds; the 8-bit form is that of the rounded y.
#pragma once
#include "psgd_values.cuh"

namespace psgd {

constexpr int NORM_THREADS = 512;                  // most threads of a CTA
constexpr int NORM_WARPS = NORM_THREADS / 32;

// Pairs of float32: one instruction for two additions, products or fused ones.
typedef unsigned long long F2;
__device__ __forceinline__ F2 pair(float lo, float hi) {
    F2 r;
    asm("mov.b64 %0, {%1, %2};\n" : "=l"(r) : "f"(lo), "f"(hi));
    return r;
}
__device__ __forceinline__ void unpair(F2 v, float& lo, float& hi) { asm("mov.b64 {%0, %1}, %2;\n" : "=f"(lo), "=f"(hi) : "l"(v)); }
__device__ __forceinline__ F2 add2(F2 a, F2 b) {
    F2 r;
    asm("add.rn.f32x2 %0, %1, %2;\n" : "=l"(r) : "l"(a), "l"(b));
    return r;
}
__device__ __forceinline__ F2 mul2(F2 a, F2 b) {
    F2 r;
    asm("mul.rn.f32x2 %0, %1, %2;\n" : "=l"(r) : "l"(a), "l"(b));
    return r;
}
__device__ __forceinline__ F2 fma2(F2 a, F2 b, F2 c) {
    F2 r;
    asm("fma.rn.f32x2 %0, %1, %2, %3;\n" : "=l"(r) : "l"(a), "l"(b), "l"(c));
    return r;
}
// eight values
struct Eight { F2 p[4]; };
__device__ __forceinline__ Eight eight(const float (&x)[8]) { return {{pair(x[0], x[1]), pair(x[2], x[3]), pair(x[4], x[5]), pair(x[6], x[7])}}; }
__device__ __forceinline__ void singles(const Eight& v, float (&x)[8]) {
#pragma unroll
    for (int j = 0; j < 4; ++j) unpair(v.p[j], x[2 * j], x[2 * j + 1]);
}
// Where the values of a thread's unit u lie in a row.  VEC: eight side by side (rows and widths of whole 16-byte units).  Else a value per lane: 32
// columns apart, the warp's lanes side by side, any width and alignment.  `n`: how many of the eight exist (from the first on).
template <bool VEC>
__device__ __forceinline__ int cell_col(int u) { return VEC ? u * 8 : (u & ~31) * 8 + (u & 31); }
// In the ring kernels a unit is two pieces of four values: side by side where x is bfloat16 (16 bytes), 128 columns apart where it is float32, so that every access of a
// warp is to whole lines (a unit of 32 bytes per lane: 16384 x 1024 forward with a residual 62 us, backward 80).
template <typename X>
__device__ __forceinline__ int piece_col(int u, int h) { return sizeof(X) == 2 ? u * 8 + 4 * h : (u & ~31) * 8 + 128 * h + (u & 31) * 4; }
// The i-th unit of a thread: a warp's VPT * 32 units lie one after the other, so that a thread's are a constant apart.
template <int VPT>
__device__ __forceinline__ int unit_of(int i) { return ((int)(threadIdx.x >> 5) * VPT + i) * 32 + (int)(threadIdx.x & 31); }
template <bool VEC>
__device__ __forceinline__ int cell_count(int col, int F) { return VEC ? (col < F ? 8 : 0) : min(max((F - col + 31) >> 5, 0), 8); }

template <typename X, bool VEC> struct Cell;
template <> struct Cell<__nv_bfloat16, true> { typedef Raw16 Raw; };
template <> struct Cell<float, true> { typedef Raw32 Raw; };
struct RawLanes16 { unsigned short h[8]; };
struct RawLanes32 { float f[8]; };
template <> struct Cell<__nv_bfloat16, false> { typedef RawLanes16 Raw; };
template <> struct Cell<float, false> { typedef RawLanes32 Raw; };

// values that do not exist read as zeros
template <typename X> __device__ __forceinline__ void cell_load(Raw16& r, const X* p, int n) {
    r.a = make_uint4(0u, 0u, 0u, 0u);
    if (n) load8(r, p);
}
template <typename X> __device__ __forceinline__ void cell_load(Raw32& r, const X* p, int n) {
    r.a = r.b = make_float4(0.f, 0.f, 0.f, 0.f);
    if (n) load8(r, p);
}
template <typename X> __device__ __forceinline__ void cell_load(RawLanes16& r, const X* p, int n) {
#pragma unroll
    for (int j = 0; j < 8; ++j) r.h[j] = j < n ? reinterpret_cast<const unsigned short*>(p)[32 * j] : (unsigned short)0;
}
template <typename X> __device__ __forceinline__ void cell_load(RawLanes32& r, const X* p, int n) {
#pragma unroll
    for (int j = 0; j < 8; ++j) r.f[j] = j < n ? p[32 * j] : 0.f;
}
__device__ __forceinline__ void widen(const RawLanes16& r, float (&x)[8]) {
#pragma unroll
    for (int j = 0; j < 8; ++j) x[j] = __uint_as_float((unsigned)r.h[j] << 16);
}
__device__ __forceinline__ void widen(const RawLanes32& r, float (&x)[8]) {
#pragma unroll
    for (int j = 0; j < 8; ++j) x[j] = r.f[j];
}
template <bool VEC, typename X> __device__ __forceinline__ void cell_store(X* p, const float (&x)[8], int n) {
    if (VEC) {
        if (n) store8(p, x);
    } else {
#pragma unroll
        for (int j = 0; j < 8; ++j)
            if (j < n) p[32 * j] = (X)x[j];            // round to nearest even where X is bfloat16
    }
}
template <typename X> __device__ __forceinline__ void round_to(float (&x)[8]) {
    if (sizeof(X) == 2) {
#pragma unroll
        for (int j = 0; j < 8; j += 2) {
            const unsigned w = pack_bf16(x[j], x[j + 1]);
            x[j] = __uint_as_float(w << 16);
            x[j + 1] = __uint_as_float(w & 0xffff0000u);
        }
    }
}
// The 8-bit form of a thread's eight values (zeros where they do not exist) of a row whose first group is `g0` and that has G groups; all lanes call.
template <bool VEC>
__device__ __forceinline__ void cell_keep(const float (&x)[8], int col, long long g0, int G, int8_t* q, uint8_t* scales) {
    if (VEC) {
        unsigned top = 0;
#pragma unroll
        for (int j = 0; j < 8; ++j) top = max(top, __float_as_uint(x[j]) & 0x7fffffffu);
        keep8(x, top, g0 + (col >> 5), col, col < G * ACT_GROUP, q, scales);
    } else {
        const int g = col >> 5, lane = col & 31;       // (the same group in all lanes)
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            if (g + j >= G) break;
            const GroupScale s = group_scale(__reduce_max_sync(0xffffffffu, __float_as_uint(x[j]) & 0x7fffffffu));
            const unsigned b = s.over ? quantize_clamped(x[j], s) : quantize(x[j], s);
            q[(g0 + g + j) * ACT_GROUP + lane] = (int8_t)(s.fine ? b & 0xffu : 0u);
            if (lane == 0) scales[g0 + g + j] = (uint8_t)s.byte;
        }
    }
}

__device__ __forceinline__ unsigned smem_addr(const void* p) { return (unsigned)__cvta_generic_to_shared(p); }
// Waits for the threads that share a row (threadIdx.y); a warp alone needs no barrier.
__device__ __forceinline__ void row_sync() {
    if (blockDim.x == 32) __syncwarp();
    else asm volatile("bar.sync %0, %1;\n" ::"r"((int)threadIdx.y + 1), "r"((int)blockDim.x) : "memory");
}
__device__ __forceinline__ float warp_sum(float x) {
#pragma unroll
    for (int o = 16; o; o >>= 1) x += __shfl_xor_sync(0xffffffffu, x, o);
    return x;
}

struct NormParam { const void* p; int bf16; };         // a vector over the columns, or nullptr
__device__ __forceinline__ float param_at(const NormParam& v, int col, float none) {
    if (!v.p) return none;
    return v.bf16 ? __bfloat162float(reinterpret_cast<const __nv_bfloat16*>(v.p)[col]) : reinterpret_cast<const float*>(v.p)[col];
}
template <bool VEC>
__device__ __forceinline__ void param_cell(float (&w)[8], const NormParam& v, int col, int n, float none) {
#pragma unroll
    for (int j = 0; j < 8; ++j) w[j] = j < n ? param_at(v, col + (VEC ? j : 32 * j), none) : 0.f;
}

struct NormForward {
    long long T;
    int F, center;
    float eps;
    const void *x, *r;                                 // r: added to x, or nullptr
    void *s, *y;                                       // s: the sum, or nullptr
    long long ldx, ldr, lds, ldy;
    NormParam w, b;
    float *mean, *rstd;                                // mean: or nullptr
    int stages;                                        // rows of a ring
    int8_t* q;                                         // the 8-bit form of y, or nullptr
    uint8_t* scales;
};

// Of a row that several warps share: the joint mean and sum of squared deviations from each warp's own.  `mine`: places of the row's warps, `have`: how many values
// warp (lane & 15) has.
struct RowStats { float mean, m2; };
__device__ __forceinline__ float sum16(float x) {
#pragma unroll
    for (int o = 8; o; o >>= 1) x += __shfl_xor_sync(0xffffffffu, x, o);
    return x;
}
__device__ __forceinline__ RowStats join_warps(float m, float sq, float2* mine, float have, float per, bool center) {
    const int warps = blockDim.x >> 5, lane = threadIdx.x & 31;
    if (lane == 0) mine[threadIdx.x >> 5] = make_float2(m, sq);
    row_sync();
    const float2 t = (lane & 15) < warps ? mine[lane & 15] : make_float2(0.f, 0.f);
    RowStats s;
    s.mean = center ? sum16(have * t.x) * per : 0.f;
    const float d = t.x - s.mean;
    s.m2 = sum16(fmaf(have * d, d, t.y));
    return s;
}

// A thread's share of a ring: `stages` (1 or 2) rows of its group, of each up to three operands of type T beside an x of type X.  The first (float32: each) pieces of the
// row's units lie in a plane one after the other, so that a warp's accesses are side by side.
__device__ __forceinline__ void copy16(unsigned to, const void* from) { asm volatile("cp.async.cg.shared.global [%0], [%1], 16;\n" ::"r"(to), "l"(from) : "memory"); }
__device__ __forceinline__ void copy8(unsigned to, const void* from) { asm volatile("cp.async.ca.shared.global [%0], [%1], 8;\n" ::"r"(to), "l"(from) : "memory"); }
__device__ __forceinline__ uint4 shared16(unsigned at) {
    uint4 v;
    asm volatile("ld.shared.v4.u32 {%0, %1, %2, %3}, [%4];\n" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "r"(at) : "memory");
    return v;
}
__device__ __forceinline__ uint2 shared8(unsigned at) {
    uint2 v;
    asm volatile("ld.shared.v2.u32 {%0, %1}, [%2];\n" : "=r"(v.x), "=r"(v.y) : "r"(at) : "memory");
    return v;
}
// the first `bytes` of 16, zeros behind them
__device__ __forceinline__ void copy16_of(unsigned to, const void* from, int bytes) {
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;\n" ::"r"(to), "l"(from), "r"(bytes) : "memory");
}
__device__ __forceinline__ F2 pair_of(unsigned x, unsigned y) { return pair(__uint_as_float(x), __uint_as_float(y)); }
// bytes of a unit in one plane, and of all planes of an operand
template <typename T, typename X> __device__ __forceinline__ constexpr int unit_bytes() { return sizeof(X) == 2 ? 16 : 4 * (int)sizeof(T); }
template <typename T, int VPT> __device__ __forceinline__ int operand_bytes() { return VPT * (int)blockDim.x * 8 * (int)sizeof(T); }
// Columns of a thread's pieces, and how many of a unit's values exist.  Aligned rows: pieces that do not exist fetch the row's last one: no branches.
// PHASE: rows of bfloat16 of any width and alignment that all operands share (the same place within 16 bytes in every row).  The units are those of memory: the first one begins
// `phase` values before the row.  A CTA takes rows whose phase is the same (every gridDim.x-th, a multiple of eight), so that its columns stay its own.
template <typename X, int VPT, bool PHASE>
struct Place {
    int at[VPT][sizeof(X) == 2 ? 1 : 2], n[VPT], phase;
    __device__ __forceinline__ Place(int F, int phase) : phase(phase) {
#pragma unroll
        for (int i = 0; i < VPT; ++i) {
            const int u = unit_of<VPT>(i), c0 = piece_col<X>(u, 0), c1 = piece_col<X>(u, 1);
            if constexpr (PHASE) {
                at[i][0] = c0 - phase;
                n[i] = min(max(F + phase - c0, 0), 8);             // (from the unit's beginning on, the values before the row included)
                continue;
            }
            at[i][0] = min(c0, F - (sizeof(X) == 2 ? 8 : 4));
            if constexpr (sizeof(X) == 4) at[i][1] = min(c1, F - 4);
            n[i] = (c0 < F ? 4 : 0) + (c1 < F ? 4 : 0);
        }
    }
    __device__ __forceinline__ int low(int i) const { return PHASE && unit_of<VPT>(i) == 0 ? phase : 0; }      // values of the unit that lie before the row
    __device__ __forceinline__ bool whole(int i) const { return n[i] - low(i) == 8; }
    // PHASE: zeros where a value is not the row's
    __device__ __forceinline__ void clear(int i, Eight& v) const {
        if (!PHASE || whole(i)) return;
        float x[8];
        singles(v, x);
#pragma unroll
        for (int j = 0; j < 8; ++j) x[j] = j >= low(i) && j < n[i] ? x[j] : 0.f;
        v = eight(x);
    }
};
// PHASE: how many values before row `row` of matrix `p` its first unit of 16 bytes begins
__device__ __forceinline__ int phase_of(const void* p, long long row, long long ld) { return (int)((reinterpret_cast<uintptr_t>(p) / 2 + (unsigned long long)(row * ld)) & 7); }
// PHASE: a unit, up to the row's end (zeros behind it).  What lies before the row in its first unit is the row before it, or, before the matrix, not read.
__device__ __forceinline__ void phase_ask(unsigned to, const __nv_bfloat16* from, int n, const __nv_bfloat16* matrix) {
    if (n > 0 && from < matrix) {
        for (int j = 0; j < 8; ++j) {
            const unsigned short h = from + j >= matrix && j < n ? reinterpret_cast<const unsigned short*>(from)[j] : (unsigned short)0;
            asm volatile("st.shared.u16 [%0], %1;\n" ::"r"(to + 2 * j), "h"(h) : "memory");
        }
        return;
    }
    copy16_of(to, n > 0 ? from : matrix + (8 - phase_of(matrix, 0, 0)) % 8, 2 * n);
}
// `operand`: where the operand's planes begin
template <typename T, typename X, int VPT, bool PHASE>
__device__ __forceinline__ void ring_ask(unsigned operand, const T* row, const Place<X, VPT, PHASE>& p, const T* matrix) {
    if constexpr (PHASE) {
#pragma unroll
        for (int i = 0; i < VPT; ++i) phase_ask(operand + unit_of<VPT>(i) * 16, row + p.at[i][0], p.n[i], matrix);
        return;
    }
    constexpr int B = unit_bytes<T, X>();
    const unsigned to = operand + unit_of<VPT>(0) * B;
#pragma unroll
    for (int i = 0; i < VPT; ++i) {
        if constexpr (B == 16) copy16(to + i * 32 * B, row + p.at[i][0]);
        else copy8(to + i * 32 * B, row + p.at[i][0]);
        if constexpr (sizeof(X) == 4) {
            const unsigned second = to + VPT * blockDim.x * B + i * 32 * B;
            if constexpr (B == 16) copy16(second, row + p.at[i][1]);
            else copy8(second, row + p.at[i][1]);
        }
    }
}
template <typename T, typename X, int VPT>
__device__ __forceinline__ Eight ring_read(unsigned operand, int i) {
    constexpr int B = unit_bytes<T, X>();
    const unsigned at = operand + unit_of<VPT>(i) * B;
    if constexpr (sizeof(T) == 4) {
        const uint4 a = shared16(at), b = shared16(at + VPT * blockDim.x * B);
        return {{pair_of(a.x, a.y), pair_of(a.z, a.w), pair_of(b.x, b.y), pair_of(b.z, b.w)}};
    } else {
        uint4 a;
        if constexpr (B == 16) {
            a = shared16(at);
        } else {
            const uint2 lo = shared8(at), hi = shared8(at + VPT * blockDim.x * B);
            a = make_uint4(lo.x, lo.y, hi.x, hi.y);
        }
        float v[8];
        widen(Raw16{a}, v);
        return eight(v);
    }
}
// A unit's values to a row of T beside an x of type X.
template <typename T, typename X, int VPT, bool PHASE>
__device__ __forceinline__ void unit_store(T* row, const Place<X, VPT, PHASE>& p, int i, const Eight& v) {
    float x[8];
    singles(v, x);
    if constexpr (sizeof(T) == 4) {
        if (p.n[i] > 0) *reinterpret_cast<float4*>(row + p.at[i][0]) = make_float4(x[0], x[1], x[2], x[3]);
        if (p.n[i] > 4) *reinterpret_cast<float4*>(row + p.at[i][1]) = make_float4(x[4], x[5], x[6], x[7]);
    } else {
        const uint4 b = pack_bf16x8(x);
        if constexpr (PHASE) {
            if (p.whole(i)) {
                *reinterpret_cast<uint4*>(row + p.at[i][0]) = b;
            } else {                                   // the row's beginning or its end
                const unsigned w[4] = {b.x, b.y, b.z, b.w};
#pragma unroll
                for (int j = 0; j < 8; ++j)
                    if (j >= p.low(i) && j < p.n[i]) reinterpret_cast<unsigned short*>(row + p.at[i][0])[j] = (unsigned short)(w[j / 2] >> (j & 1) * 16);
            }
        } else if constexpr (sizeof(X) == 2) {
            if (p.n[i] > 0) *reinterpret_cast<uint4*>(row + p.at[i][0]) = b;
        } else {
            if (p.n[i] > 0) *reinterpret_cast<uint2*>(row + p.at[i][0]) = make_uint2(b.x, b.y);
            if (p.n[i] > 4) *reinterpret_cast<uint2*>(row + p.at[i][1]) = make_uint2(b.z, b.w);
        }
    }
}
// the sum of a unit's values that exist
__device__ __forceinline__ float sum_of(const Eight& v, int n) {
    float a, b, c, d;
    unpair(add2(v.p[0], v.p[1]), a, b);
    unpair(add2(v.p[2], v.p[3]), c, d);
    return (n > 0 ? a + b : 0.f) + (n > 4 ? c + d : 0.f);
}
// A unit of x + r, rounded to their type, written to row s.  Sums of bfloat16 are rounded once by the packed addition itself.
template <typename X, int VPT, bool PHASE>
__device__ __forceinline__ Eight ring_sum(unsigned x_at, unsigned r_at, int i, X* s, const Place<X, VPT, PHASE>& p) {
    Eight v;
    if constexpr (sizeof(X) == 2) {
        const uint4 x = shared16(x_at + unit_of<VPT>(i) * 16), r = shared16(r_at + unit_of<VPT>(i) * 16);
        const auto sum = [](unsigned u, unsigned v) {
            const __nv_bfloat162 t = __hadd2(*reinterpret_cast<const __nv_bfloat162*>(&u), *reinterpret_cast<const __nv_bfloat162*>(&v));
            return *reinterpret_cast<const unsigned*>(&t);
        };
        const uint4 t = make_uint4(sum(x.x, r.x), sum(x.y, r.y), sum(x.z, r.z), sum(x.w, r.w));
        float f[8];
        widen(Raw16{t}, f);
        v = eight(f);
        if constexpr (PHASE) {
            unit_store<X, X, VPT, PHASE>(s, p, i, v);  // (rounded already: the same bits)
            p.clear(i, v);
        } else if (p.n[i]) {
            *reinterpret_cast<uint4*>(s + p.at[i][0]) = t;
        }
    } else {
        v = ring_read<X, X, VPT>(x_at, i);
        const Eight r = ring_read<X, X, VPT>(r_at, i);
#pragma unroll
        for (int j = 0; j < 4; ++j) v.p[j] = add2(v.p[j], r.p[j]);
        unit_store<X, X, VPT, PHASE>(s, p, i, v);
    }
    return v;
}
// The 8-bit form of a unit's values of a row of T (see cell_keep); all lanes call.
template <typename T, typename X>
__device__ __forceinline__ void unit_keep(const Eight& v, int u, int n, long long g0, int G, int8_t* q, uint8_t* scales) {
    float x[8];
    singles(v, x);
#pragma unroll
    for (int j = 0; j < 8; ++j) x[j] = j < n ? x[j] : 0.f;
    round_to<T>(x);
    if constexpr (sizeof(X) == 2) {
        cell_keep<true>(x, u * 8, g0, G, q, scales);
    } else {
#pragma unroll
        for (int h = 0; h < 2; ++h) {                  // eight lanes share a group
            const int col = piece_col<X>(u, h);
            unsigned top = 0;
#pragma unroll
            for (int j = 0; j < 4; ++j) top = max(top, __float_as_uint(x[4 * h + j]) & 0x7fffffffu);
#pragma unroll
            for (int o = 1; o < 8; o <<= 1) top = max(top, __shfl_xor_sync(0xffffffffu, top, o));
            const GroupScale s = group_scale(top);
            unsigned b[4];
#pragma unroll
            for (int j = 0; j < 4; ++j) b[j] = s.over ? quantize_clamped(x[4 * h + j], s) : quantize(x[4 * h + j], s);
            const unsigned w = __byte_perm(__byte_perm(b[0], b[1], 0x0040), __byte_perm(b[2], b[3], 0x0040), 0x5410);
            if ((col >> 5) >= G) continue;
            *reinterpret_cast<unsigned*>(q + (g0 + (col >> 5)) * ACT_GROUP + (col & 31)) = s.fine ? w : 0u;
            if ((col & 31) == 0) scales[g0 + (col >> 5)] = (uint8_t)s.byte;
        }
    }
}
// One group of copies per row, empty ones behind the last row included: a row's have landed when at most stages - 1 younger groups are under way.
__device__ __forceinline__ void ring_commit() { asm volatile("cp.async.commit_group;\n" ::: "memory"); }
__device__ __forceinline__ void ring_wait(int stages) {
    if (stages == 1) asm volatile("cp.async.wait_group 0;\n" ::: "memory");
    else asm volatile("cp.async.wait_group 1;\n" ::: "memory");
}
// A vector over the columns as float32 in shared memory: a plane of first pieces, a plane of second ones (zeros where there is none), by the whole CTA.
template <typename X>
__device__ __forceinline__ void param_planes(unsigned char* to, const NormParam& v, int units, int F, int phase, float none) {
    for (int k = threadIdx.y * blockDim.x + threadIdx.x; k < 2 * units; k += blockDim.x * blockDim.y) {
        const int c = piece_col<X>(k >> 1, k & 1) - phase;
        float x[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) x[j] = c + j >= 0 && c + j < F ? param_at(v, c + j, none) : 0.f;
        reinterpret_cast<float4*>(to)[(k & 1) * units + (k >> 1)] = make_float4(x[0], x[1], x[2], x[3]);
    }
}
// a unit of it; `units`: of a plane
template <int VPT>
__device__ __forceinline__ Eight param_read(unsigned planes, int units, int i) {
    const unsigned at = planes + unit_of<VPT>(i) * 16;
    const uint4 a = shared16(at), b = shared16(at + units * 16);
    return {{pair_of(a.x, a.y), pair_of(a.z, a.w), pair_of(b.x, b.y), pair_of(b.z, b.w)}};
}

template <typename X, typename Y, int VPT, bool PHASE>
__global__ void __launch_bounds__(NORM_THREADS) k_norm_forward(const __grid_constant__ NormForward a) {
    extern __shared__ __align__(16) unsigned char ring_raw[];          // w, b, then the rings; PHASE with an 8-bit form: a row of each group at last
    __shared__ float2 stat[2][NORM_WARPS];             // by rows taken in turn: a row's exchange is over when the next but one writes
    __shared__ float counts[NORM_WARPS];
    grid_trigger();
    const int F = a.F, tid = threadIdx.x, warps = blockDim.x >> 5, units = VPT * blockDim.x;
    const int phase = PHASE ? phase_of(a.x, blockIdx.x, a.ldx) : 0;
    const Place<X, VPT, PHASE> p(F, phase);
    int have = 0;
#pragma unroll
    for (int i = 0; i < VPT; ++i) have += max(p.n[i] - p.low(i), 0);
    const float in_warp = (float)__reduce_add_sync(0xffffffffu, have), per = 1.f / (float)F, per_warp = 1.f / fmaxf(in_warp, 1.f);
    if (threadIdx.y == 0 && (tid & 31) == 0) counts[tid >> 5] = in_warp;
    grid_wait();
    const long long step = (long long)gridDim.x * blockDim.y;
    long long row = PHASE ? blockIdx.x + (long long)gridDim.x * threadIdx.y : (long long)blockIdx.x * blockDim.y + threadIdx.y, asked = row;
    // rows: the one that is asked for next (x, r) and the one at work (s, y)
    const X *x = (const X*)a.x + row * a.ldx, *r = a.r ? (const X*)a.r + row * a.ldr : nullptr;
    X* s = a.s ? (X*)a.s + row * a.lds : nullptr;
    Y* y = (Y*)a.y + row * a.ldy;
    const int operand = operand_bytes<X, VPT>(), stage = r ? 2 * operand : operand, stages = a.stages;
    const unsigned params = smem_addr(ring_raw), ring = params + units * 64 + threadIdx.y * stages * stage;
    const auto ask = [&](unsigned to) {
        if (asked < a.T) {
            ring_ask<X, X, VPT, PHASE>(to, x, p, (const X*)a.x);
            if (r) ring_ask<X, X, VPT, PHASE>(to + operand, r, p, (const X*)a.r);
        }
        ring_commit();
        asked += step;
        x += step * a.ldx;
        if (r) r += step * a.ldr;
    };
    for (int k = 0; k < stages; ++k) ask(ring + k * stage);
    param_planes<X>(ring_raw, a.w, units, F, phase, 1.f);
    param_planes<X>(ring_raw + units * 32, a.b, units, F, phase, 0.f);
    __syncthreads();
    const float in_lane = (tid & 15) < warps ? counts[tid & 15] : 0.f;
    const int G = (F + ACT_GROUP - 1) / ACT_GROUP;
    // PHASE: the row's rounded result as it lies in memory, for the groups of its 8-bit form, which begin with the row
    const unsigned image = params + units * 64 + blockDim.y * stages * stage + threadIdx.y * (units * 16 + 16);
    unsigned from = ring;
    for (int turn = 0; row < a.T; row += step, turn ^= 1) {
        Eight v[VPT];
        ring_wait(stages);
        if (r) {
#pragma unroll
            for (int i = 0; i < VPT; ++i) v[i] = ring_sum<X, VPT, PHASE>(from, from + operand, i, s, p);
        } else {
#pragma unroll
            for (int i = 0; i < VPT; ++i) {
                v[i] = ring_read<X, X, VPT>(from, i);
                p.clear(i, v[i]);
            }
            if (s) {
#pragma unroll
                for (int i = 0; i < VPT; ++i) unit_store<X, X, VPT, PHASE>(s, p, i, v[i]);
            }
        }
        float m = 0.f;
        if (a.center) {
#pragma unroll
            for (int i = 0; i < VPT; ++i) m += sum_of(v[i], p.n[i]);
            m = warp_sum(m) * per_warp;
            const F2 off = pair(-m, -m);
#pragma unroll
            for (int i = 0; i < VPT; ++i)
#pragma unroll
                for (int j = 0; j < 4; ++j) v[i].p[j] = add2(v[i].p[j], off);
            if constexpr (PHASE) {
#pragma unroll
                for (int i = 0; i < VPT; ++i) p.clear(i, v[i]);
            }
        }
        float sq = 0.f;
#pragma unroll
        for (int i = 0; i < VPT; ++i) {
            const F2 first = fma2(v[i].p[1], v[i].p[1], mul2(v[i].p[0], v[i].p[0])), second = fma2(v[i].p[3], v[i].p[3], mul2(v[i].p[2], v[i].p[2]));
            float t[4];
            unpair(first, t[0], t[1]);
            unpair(second, t[2], t[3]);
            sq += (p.n[i] > 0 ? t[0] + t[1] : 0.f) + (p.n[i] > 4 ? t[2] + t[3] : 0.f);
        }
        RowStats st{m, warp_sum(sq)};
        ask(from);                                     // (every value has been used)
        from = stages == 1 || from != ring ? ring : ring + stage;
        if (warps > 1) st = join_warps(st.mean, st.m2, stat[turn] + threadIdx.y * warps, in_lane, per, a.center);
        const float f = rsqrtf(fmaf(st.m2, per, a.eps));
        if (tid == 0) {
            a.rstd[row] = f;
            if (a.mean) a.mean[row] = st.mean;
        }
        const F2 off = pair(m - st.mean, m - st.mean), ff = pair(f, f);
#pragma unroll
        for (int i = 0; i < VPT; ++i) {
            const Eight w = param_read<VPT>(params, units, i), b = param_read<VPT>(params + units * 32, units, i);
            Eight o;
#pragma unroll
            for (int j = 0; j < 4; ++j) o.p[j] = fma2(mul2(add2(v[i].p[j], off), ff), w.p[j], b.p[j]);
            unit_store<Y, X, VPT, PHASE>(y, p, i, o);
            if constexpr (PHASE) {
                if (a.q) {
                    float t[8];
                    singles(o, t);
                    const uint4 b = pack_bf16x8(t);
                    asm volatile("st.shared.v4.u32 [%0], {%1, %2, %3, %4};\n" ::"r"(image + unit_of<VPT>(i) * 16), "r"(b.x), "r"(b.y), "r"(b.z), "r"(b.w) : "memory");
                }
            } else if (a.q) {
                unit_keep<Y, X>(o, unit_of<VPT>(i), p.n[i], row * G, G, a.q, a.scales);
            }
        }
        if constexpr (PHASE) {
            if (a.q) {
                row_sync();
#pragma unroll
                for (int i = 0; i < VPT; ++i) {
                    const int u = unit_of<VPT>(i);
                    const unsigned at = image + u * 16;
                    float t[8];
                    widen(Raw16{cut_out(shared16(at), shared16(at + 16), 2 * phase)}, t);
                    unit_keep<Y, X>(eight(t), u, min(max(F - u * 8, 0), 8), row * G, G, a.q, a.scales);
                }
                if (warps == 1) __syncwarp();          // (several: the next row's exchange comes before its values)
            }
        }
        if (s) s += step * a.lds;
        y += step * a.ldy;
    }
}

// Rows of any width up to NORM_THREADS units and any alignment: one unit per thread, a value per lane.
template <typename X, typename Y>
__global__ void __launch_bounds__(NORM_THREADS) k_norm_forward_any(const __grid_constant__ NormForward a) {
    typedef typename Cell<X, false>::Raw Raw;
    __shared__ float2 stat[2][NORM_WARPS];
    __shared__ float counts[NORM_WARPS];
    grid_trigger();
    const int F = a.F, tid = threadIdx.x, warps = blockDim.x >> 5, col = cell_col<false>(tid), n = cell_count<false>(col, F);
    const float in_warp = (float)__reduce_add_sync(0xffffffffu, n), per = 1.f / (float)F, per_warp = 1.f / fmaxf(in_warp, 1.f);
    if (threadIdx.y == 0 && (tid & 31) == 0) counts[tid >> 5] = in_warp;
    __syncthreads();
    const float in_lane = (tid & 15) < warps ? counts[tid & 15] : 0.f;
    grid_wait();
    float w[8], b[8];
    param_cell<false>(w, a.w, col, n, 1.f);
    param_cell<false>(b, a.b, col, n, 0.f);
    const int G = (F + ACT_GROUP - 1) / ACT_GROUP;
    const long long step = (long long)gridDim.x * blockDim.y;
    long long row = (long long)blockIdx.x * blockDim.y + threadIdx.y;
    Raw next, add;
    const auto ask = [&](long long at) {
        if (at >= a.T) return;
        cell_load(next, (const X*)a.x + at * a.ldx + col, n);
        if (a.r) cell_load(add, (const X*)a.r + at * a.ldr + col, n);
    };
    ask(row);
    for (int turn = 0; row < a.T; row += step, turn ^= 1) {
        float v[8];
        widen(next, v);
        if (a.r) {
            float u[8];
            widen(add, u);
#pragma unroll
            for (int j = 0; j < 8; ++j) v[j] += u[j];
            round_to<X>(v);
        }
        ask(row + step);
        if (a.s) cell_store<false>((X*)a.s + row * a.lds + col, v, n);
        float m = 0.f, sq = 0.f;
        if (a.center) m = warp_sum(((v[0] + v[1]) + (v[2] + v[3])) + ((v[4] + v[5]) + (v[6] + v[7]))) * per_warp;
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            v[j] = j < n ? v[j] - m : 0.f;
            sq = fmaf(v[j], v[j], sq);
        }
        RowStats st{m, warp_sum(sq)};
        if (warps > 1) st = join_warps(st.mean, st.m2, stat[turn] + threadIdx.y * warps, in_lane, per, a.center);
        const float f = rsqrtf(fmaf(st.m2, per, a.eps)), off = m - st.mean;
        if (tid == 0) {
            a.rstd[row] = f;
            if (a.mean) a.mean[row] = st.mean;
        }
#pragma unroll
        for (int j = 0; j < 8; ++j) v[j] = j < n ? fmaf((v[j] + off) * f, w[j], b[j]) : 0.f;
        cell_store<false>((Y*)a.y + row * a.ldy + col, v, n);
        if (a.q) {
            round_to<Y>(v);
            cell_keep<false>(v, col, row * G, G, a.q, a.scales);
        }
    }
}

// Rows that are too wide for registers: a CTA per row, three passes over it (the second and third find it in L1 and L2).
template <typename X, typename Y, bool VEC>
__global__ void __launch_bounds__(NORM_THREADS) k_norm_forward_wide(const __grid_constant__ NormForward a) {
    typedef typename Cell<X, VEC>::Raw Raw;
    __shared__ float part[2][NORM_WARPS];
    grid_trigger();
    grid_wait();
    const int F = a.F, tid = threadIdx.x, G = (F + ACT_GROUP - 1) / ACT_GROUP;
    const int units = (F + 255) / 256 * 32;            // whole warps of units
    const auto total = [&](float v, float* to) {
        v = warp_sum(v);
        if ((tid & 31) == 0) to[tid >> 5] = v;
        __syncthreads();
        float sum = 0.f;
        for (int w = 0; w < (int)blockDim.x >> 5; ++w) sum += to[w];
        return sum;
    };
    for (long long row = blockIdx.x; row < a.T; row += gridDim.x) {
        const X *x = (const X*)a.x + row * a.ldx, *r = a.r ? (const X*)a.r + row * a.ldr : nullptr;
        X* s = a.s ? (X*)a.s + row * a.lds : nullptr;
        Y* y = (Y*)a.y + row * a.ldy;
        const auto values = [&](int u, float (&v)[8], int& col, int& n) {
            col = cell_col<VEC>(u);
            n = cell_count<VEC>(col, F);
            Raw raw;
            cell_load(raw, x + col, n);
            widen(raw, v);
            if (r) {
                float w[8];
                cell_load(raw, r + col, n);
                widen(raw, w);
#pragma unroll
                for (int j = 0; j < 8; ++j) v[j] += w[j];
                round_to<X>(v);
            }
        };
        float sum = 0.f, sq = 0.f;
        for (int u = tid; u < units; u += blockDim.x) {
            float v[8];
            int col, n;
            values(u, v, col, n);
            if (s) cell_store<VEC>(s + col, v, n);
            sum += ((v[0] + v[1]) + (v[2] + v[3])) + ((v[4] + v[5]) + (v[6] + v[7]));
        }
        const float mean = a.center ? total(sum, part[0]) / (float)F : 0.f;
        for (int u = tid; u < units; u += blockDim.x) {
            float v[8];
            int col, n;
            values(u, v, col, n);
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const float d = j < n ? v[j] - mean : 0.f;
                sq = fmaf(d, d, sq);
            }
        }
        const float f = rsqrtf(total(sq, part[1]) / (float)F + a.eps);
        if (tid == 0) {
            a.rstd[row] = f;
            if (a.mean) a.mean[row] = mean;
        }
        for (int u = tid; u < units; u += blockDim.x) {
            float v[8];
            int col, n;
            values(u, v, col, n);
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const int c = col + (VEC ? j : 32 * j);
                v[j] = j < n ? fmaf((v[j] - mean) * f, param_at(a.w, c, 1.f), param_at(a.b, c, 0.f)) : 0.f;
            }
            cell_store<VEC>(y + col, v, n);
            if (a.q) {
                round_to<Y>(v);
                cell_keep<VEC>(v, col, row * G, G, a.q, a.scales);
            }
        }
        __syncthreads();                               // (the sums' places are free again)
    }
}

struct NormBackward {
    long long T;
    int F, center;
    const void *dy, *x, *add;                          // add: what reaches x from elsewhere, or nullptr
    void* dx;
    long long lddy, ldx, ldadd, lddx;
    NormParam w;
    const float *mean, *rstd;                          // mean: nullptr without centring
    int stages;                                        // rows of a ring
    float* part;                                       // [CTAs][2][F]: dw, db
    float *dw, *db;                                    // db: or nullptr
    float2* sums;                                      // wide rows: [T] mean(g), mean(g xh)
};
struct NormJoin { int F, parts; const float* part; float *dw, *db; };      // db: or nullptr

// The sums s1 and s2 of a row over its warps.
__device__ __forceinline__ void sum_warps(float& s1, float& s2, float2* mine) {
    const int warps = blockDim.x >> 5;
    if ((threadIdx.x & 31) == 0) mine[threadIdx.x >> 5] = make_float2(s1, s2);
    row_sync();
    s1 = s2 = 0.f;
#pragma unroll 4
    for (int k = 0; k < warps; ++k) {
        const float2 t = mine[k];
        s1 += t.x;
        s2 += t.y;
    }
}
// At the end: the CTA's sums of dw and db, its rows side by side (threadIdx.y) through `sums` [blockDim.y][2][pitch]; a CTA alone writes the results.  `column(i, j)`: of value j
// of the thread's unit i (FOUR: four of them side by side at a multiple of four), `n`: how many of its values exist.  The first `phase` columns are not the row's (PHASE, where
// the pitch is a row's units and a row alone goes that way too: 16 bytes at a time into shared memory, a line at a time out of it).
template <int VPT, bool FOUR, typename Column>
__device__ __forceinline__ void write_columns(const NormBackward& a, float* sums, int pitch, int phase, const Eight (&dw)[VPT], const Eight (&db)[VPT], const int (&n)[VPT], Column&& column) {
    const int F = a.F;
    float* pw = gridDim.x == 1 ? a.dw : a.part + (size_t)blockIdx.x * 2 * F;
    float* pb = gridDim.x == 1 ? a.db : pw + F;
    const bool alone = blockDim.y == 1 && pitch == F;
    if (!alone) __syncthreads();                       // (nobody reads what lay there)
    float *to_w = alone ? pw : sums + (size_t)threadIdx.y * 2 * pitch, *to_b = alone ? pb : to_w + pitch;
    const bool whole = (((uintptr_t)to_w | (uintptr_t)to_b) & 15) == 0;
#pragma unroll
    for (int i = 0; i < VPT; ++i) {
        float p[8], q[8];
        singles(dw[i], p);
        singles(db[i], q);
        if (FOUR && whole) {
#pragma unroll
            for (int j = 0; j < 8; j += 4)
                if (j < n[i]) {
                    const int c = column(i, j);
                    *reinterpret_cast<float4*>(to_w + c) = make_float4(p[j], p[j + 1], p[j + 2], p[j + 3]);
                    if (to_b) *reinterpret_cast<float4*>(to_b + c) = make_float4(q[j], q[j + 1], q[j + 2], q[j + 3]);
                }
            continue;
        }
#pragma unroll
        for (int j = 0; j < 8; ++j)
            if (j < n[i]) {
                const int c = column(i, j);
                to_w[c] = p[j];
                if (to_b) to_b[c] = q[j];
            }
    }
    if (alone) return;
    __syncthreads();
    for (int c = threadIdx.y * blockDim.x + threadIdx.x; c < F; c += blockDim.x * blockDim.y) {
        float w = 0.f, b = 0.f;
        for (int k = 0; k < (int)blockDim.y; ++k) {
            w += sums[(size_t)k * 2 * pitch + phase + c];
            b += sums[(size_t)k * 2 * pitch + pitch + phase + c];
        }
        pw[c] = w;
        if (pb) pb[c] = b;
    }
}

template <typename X, typename Y, int VPT, bool PHASE>
__global__ void __launch_bounds__(NORM_THREADS) k_norm_backward(const __grid_constant__ NormBackward a) {
    extern __shared__ __align__(16) unsigned char ring_raw[];          // w, then the rings; at the end the sums of the rows side by side
    __shared__ float2 stat[2][NORM_WARPS];
    grid_trigger();
    const int F = a.F, warps = blockDim.x >> 5, units = VPT * blockDim.x;
    const int phase = PHASE ? phase_of(a.x, blockIdx.x, a.ldx) : 0;
    const Place<X, VPT, PHASE> p(F, phase);
    grid_wait();
    const long long step = (long long)gridDim.x * blockDim.y;
    long long row = PHASE ? blockIdx.x + (long long)gridDim.x * threadIdx.y : (long long)blockIdx.x * blockDim.y + threadIdx.y, asked = row;
    // rows: the one that is asked for next (dy, x, add) and the one at work (dx)
    const Y* dy = (const Y*)a.dy + row * a.lddy;
    const X *x = (const X*)a.x + row * a.ldx, *add = a.add ? (const X*)a.add + row * a.ldadd : nullptr;
    X* dx = (X*)a.dx + row * a.lddx;
    const int at_x = operand_bytes<Y, VPT>(), at_add = at_x + operand_bytes<X, VPT>(), stage = add ? at_add + operand_bytes<X, VPT>() : at_add, stages = a.stages;
    const unsigned params = smem_addr(ring_raw), ring = params + units * 32 + threadIdx.y * stages * stage;
    float nm = 0.f, nf = 0.f;                          // the next row's mean and rstd
    const auto ask_stats = [&](long long i) {
        if (i >= a.T) return;
        nf = a.rstd[i];
        if (a.mean) nm = a.mean[i];
    };
    const auto ask = [&](unsigned to) {
        if (asked < a.T) {
            ring_ask<Y, X, VPT, PHASE>(to, dy, p, (const Y*)a.dy);
            ring_ask<X, X, VPT, PHASE>(to + at_x, x, p, (const X*)a.x);
            if (add) ring_ask<X, X, VPT, PHASE>(to + at_add, add, p, (const X*)a.add);
        }
        ring_commit();
        asked += step;
        dy += step * a.lddy;
        x += step * a.ldx;
        if (add) add += step * a.ldadd;
    };
    for (int k = 0; k < stages; ++k) ask(ring + k * stage);
    ask_stats(row);
    param_planes<X>(ring_raw, a.w, units, F, phase, 1.f);
    __syncthreads();
    Eight dw[VPT], db[VPT];
#pragma unroll
    for (int i = 0; i < VPT; ++i)
#pragma unroll
        for (int j = 0; j < 4; ++j) dw[i].p[j] = db[i].p[j] = 0ull;
    const float per = 1.f / (float)F;
    unsigned from = ring;
    for (int turn = 0; row < a.T; row += step, turn ^= 1) {
        const float f = nf, m = nm;
        ask_stats(row + step);
        const F2 off = pair(-m, -m), ff = pair(f, f);
        ring_wait(stages);
        F2 t1 = 0ull, t2 = 0ull;
#pragma unroll
        for (int i = 0; i < VPT; ++i) {
            Eight d = ring_read<Y, X, VPT>(from, i), v = ring_read<X, X, VPT>(from + at_x, i);
            p.clear(i, d);
            p.clear(i, v);
            const Eight w = param_read<VPT>(params, units, i);
#pragma unroll
            for (int j = 0; j < 4; ++j) {              // (w is 0 where there is no value, and its dw and db go nowhere)
                const F2 xh = mul2(add2(v.p[j], off), ff), g = mul2(d.p[j], w.p[j]);
                t1 = add2(t1, g);
                t2 = fma2(g, xh, t2);
                dw[i].p[j] = fma2(d.p[j], xh, dw[i].p[j]);
                db[i].p[j] = add2(db[i].p[j], d.p[j]);
            }
        }
        float s1, s2, hi;
        unpair(t1, s1, hi);
        s1 = warp_sum(s1 + hi);
        unpair(t2, s2, hi);
        s2 = warp_sum(s2 + hi);
        if (warps > 1) sum_warps(s1, s2, stat[turn] + threadIdx.y * warps);
        s1 = a.center ? s1 * per * -f : 0.f;
        s2 *= -per * f * f;
        const F2 c1 = pair(s1, s1), c2 = pair(s2, s2);
#pragma unroll
        for (int i = 0; i < VPT; ++i) {
            const Eight v = ring_read<X, X, VPT>(from + at_x, i), w = param_read<VPT>(params, units, i);
            Eight d = ring_read<Y, X, VPT>(from, i);
#pragma unroll
            for (int j = 0; j < 4; ++j) d.p[j] = fma2(mul2(d.p[j], w.p[j]), ff, fma2(add2(v.p[j], off), c2, c1));
            if (add) {
                const Eight u = ring_read<X, X, VPT>(from + at_add, i);
#pragma unroll
                for (int j = 0; j < 4; ++j) d.p[j] = add2(d.p[j], u.p[j]);
            }
            unit_store<X, X, VPT, PHASE>(dx, p, i, d);
        }
        dx += step * a.lddx;
        ask(from);
        from = stages == 1 || from != ring ? ring : ring + stage;
    }
    asm volatile("cp.async.wait_all;\n" ::: "memory");
    write_columns<VPT, true>(a, reinterpret_cast<float*>(ring_raw), PHASE ? units * 8 : F, phase, dw, db, p.n, [](int i, int j) { return piece_col<X>(unit_of<VPT>(i), j >> 2) + (j & 3); });
}

template <typename X, typename Y>
__global__ void __launch_bounds__(NORM_THREADS) k_norm_backward_any(const __grid_constant__ NormBackward a) {
    typedef typename Cell<X, false>::Raw RawX;
    typedef typename Cell<Y, false>::Raw RawY;
    extern __shared__ __align__(16) unsigned char ring_raw[];          // at the end the sums of the rows side by side
    __shared__ float2 stat[2][NORM_WARPS];
    grid_trigger();
    const int F = a.F, tid = threadIdx.x, warps = blockDim.x >> 5, col = cell_col<false>(tid), n = cell_count<false>(col, F);
    grid_wait();
    float w[8], dw[8], db[8];
    param_cell<false>(w, a.w, col, n, 1.f);
#pragma unroll
    for (int j = 0; j < 8; ++j) dw[j] = db[j] = 0.f;
    const long long step = (long long)gridDim.x * blockDim.y;
    long long row = (long long)blockIdx.x * blockDim.y + threadIdx.y;
    RawX nx, na;
    RawY ny;
    float nm = 0.f, nf = 0.f;
    const auto ask = [&](long long at) {
        if (at >= a.T) return;
        nf = a.rstd[at];
        if (a.mean) nm = a.mean[at];
        cell_load(nx, (const X*)a.x + at * a.ldx + col, n);
        cell_load(ny, (const Y*)a.dy + at * a.lddy + col, n);
        if (a.add) cell_load(na, (const X*)a.add + at * a.ldadd + col, n);
    };
    ask(row);
    const float per = 1.f / (float)F;
    for (int turn = 0; row < a.T; row += step, turn ^= 1) {
        const float f = nf, m = nm;
        float v[8], d[8], u[8];
        widen(nx, v);
        widen(ny, d);
        if (a.add) widen(na, u);
        ask(row + step);
        float s1 = 0.f, s2 = 0.f;
#pragma unroll
        for (int j = 0; j < 8; ++j) {                  // (dy is 0 where there is no value)
            v[j] = (v[j] - m) * f;
            dw[j] = fmaf(d[j], v[j], dw[j]);
            db[j] += d[j];
            d[j] *= w[j];
            s1 += d[j];
            s2 = fmaf(d[j], v[j], s2);
        }
        s1 = warp_sum(s1);
        s2 = warp_sum(s2);
        if (warps > 1) sum_warps(s1, s2, stat[turn] + threadIdx.y * warps);
        s1 = a.center ? s1 * per * -f : 0.f;
        s2 *= -per;
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            d[j] = fmaf(fmaf(v[j], s2, d[j]), f, s1);
            if (a.add) d[j] += u[j];
        }
        cell_store<false>((X*)a.dx + row * a.lddx + col, d, n);
    }
    const Eight sums_w[1] = {eight(dw)}, sums_b[1] = {eight(db)};
    const int many[1] = {n};
    write_columns<1, false>(a, reinterpret_cast<float*>(ring_raw), F, 0, sums_w, sums_b, many, [=](int, int j) { return col + 32 * j; });
}

// Wide rows: first the two sums of every row (a CTA per row), then dx and the sums over rows (256 units of the columns per CTA, gridDim.y CTAs share the rows).
template <typename X, typename Y, bool VEC>
__global__ void __launch_bounds__(NORM_THREADS) k_norm_sums_wide(const __grid_constant__ NormBackward a) {
    __shared__ float2 part[NORM_WARPS];
    grid_trigger();
    grid_wait();
    const int F = a.F, tid = threadIdx.x, units = (F + 255) / 256 * 32;
    for (long long row = blockIdx.x; row < a.T; row += gridDim.x) {
        const X* x = (const X*)a.x + row * a.ldx;
        const Y* dy = (const Y*)a.dy + row * a.lddy;
        const float f = a.rstd[row], m = a.mean ? a.mean[row] : 0.f;
        float s1 = 0.f, s2 = 0.f;
        for (int u = tid; u < units; u += blockDim.x) {
            const int col = cell_col<VEC>(u), n = cell_count<VEC>(col, F);
            typename Cell<X, VEC>::Raw rx;
            typename Cell<Y, VEC>::Raw ry;
            cell_load(rx, x + col, n);
            cell_load(ry, dy + col, n);
            float v[8], d[8];
            widen(rx, v);
            widen(ry, d);
#pragma unroll
            for (int j = 0; j < 8; ++j)
                if (j < n) {
                    const float g = d[j] * param_at(a.w, col + (VEC ? j : 32 * j), 1.f);
                    s1 += g;
                    s2 = fmaf(g, (v[j] - m) * f, s2);
                }
        }
        s1 = warp_sum(s1);
        s2 = warp_sum(s2);
        if ((tid & 31) == 0) part[tid >> 5] = make_float2(s1, s2);
        __syncthreads();
        if (tid == 0) {
            s1 = s2 = 0.f;
            for (int k = 0; k < (int)blockDim.x >> 5; ++k) { s1 += part[k].x; s2 += part[k].y; }
            a.sums[row] = make_float2(a.center ? s1 / (float)F : 0.f, s2 / (float)F);
        }
        __syncthreads();
    }
}
template <typename X, typename Y, bool VEC>
__global__ void __launch_bounds__(256) k_norm_apply_wide(const __grid_constant__ NormBackward a) {
    grid_trigger();
    grid_wait();
    const int F = a.F, col = cell_col<VEC>(blockIdx.x * 256 + threadIdx.x), n = cell_count<VEC>(col, F);
    float w[8], dw[8], db[8];
    param_cell<VEC>(w, a.w, col, n, 1.f);
#pragma unroll
    for (int j = 0; j < 8; ++j) dw[j] = db[j] = 0.f;
    for (long long row = blockIdx.y; row < a.T; row += gridDim.y) {
        typename Cell<X, VEC>::Raw rx, ra;
        typename Cell<Y, VEC>::Raw ry;
        cell_load(rx, (const X*)a.x + row * a.ldx + col, n);
        cell_load(ry, (const Y*)a.dy + row * a.lddy + col, n);
        if (a.add) cell_load(ra, (const X*)a.add + row * a.ldadd + col, n);
        const float f = a.rstd[row], m = a.mean ? a.mean[row] : 0.f;
        const float2 s = a.sums[row];
        float v[8], d[8], o[8];
        widen(rx, v);
        widen(ry, d);
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const float xh = (v[j] - m) * f;
            dw[j] = fmaf(d[j], xh, dw[j]);
            db[j] += d[j];
            o[j] = f * (fmaf(-xh, s.y, d[j] * w[j]) - s.x);
        }
        if (a.add) {
            widen(ra, v);
#pragma unroll
            for (int j = 0; j < 8; ++j) o[j] += v[j];
        }
        cell_store<VEC>((X*)a.dx + row * a.lddx + col, o, n);
    }
    float* pw = gridDim.y == 1 ? a.dw : a.part + (size_t)blockIdx.y * 2 * F;
    float* pb = gridDim.y == 1 ? a.db : pw + F;
#pragma unroll
    for (int j = 0; j < 8; ++j)
        if (j < n) {
            const int c = col + (VEC ? j : 32 * j);
            pw[c] = dw[j];
            if (pb) pb[c] = db[j];
        }
}

// Adds the CTAs' sums: blockIdx.x = 32 columns, blockIdx.y = dw or db; every 32nd part per warp, then the warps, in a fixed order.
__global__ void __launch_bounds__(1024) k_norm_join(const __grid_constant__ NormJoin a) {
    __shared__ float xs[32][33];
    grid_trigger();
    grid_wait();
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, col = blockIdx.x * 32 + lane;
    float sum = 0.f;
    if (col < a.F) {
        const float* p = a.part + (size_t)blockIdx.y * a.F + col;
#pragma unroll 8
        for (int k = warp; k < a.parts; k += 32) sum += p[(size_t)k * 2 * a.F];
    }
    xs[warp][lane] = sum;
    __syncthreads();
    sum = warp_sum(xs[lane][warp]);                    // warp: a column, lane: a warp's share
    const int c = blockIdx.x * 32 + warp;
    if (lane == 0 && c < a.F) (blockIdx.y ? a.db : a.dw)[c] = sum;
}

}  // namespace psgd
