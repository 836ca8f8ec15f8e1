// Layer norm of rows (also without centring), forward and backward.
//
//   s = x + r (rounded to x's type; s = x without r),  m = mean(s) (0 without centring),  f = 1 / sqrt(mean((s - m)^2) + eps),
//   y = (s - m) f w + b;
//   g = dy w,  xh = (s - m) f,  ds = f (g - mean(g) - xh mean(g xh)) + what reaches s from elsewhere  (mean(g) only with centring),
//   dw = sum over rows of dy xh,  db = sum over rows of dy.
//
// One pass over the operands, bound by HBM.  blockDim.x threads share a row (blockDim.y rows per CTA side by side), each works on VPT units of eight
// values of it.  The sum of squares is taken about the warp's own mean and the warps' results are joined exactly (squares about the joint mean = sum of the
// warps' squares + n_w (mean_w - mean)^2), so that a large mean costs no bits and a row takes one exchange between its warps, none where a warp has it alone.
// The CTAs stay and walk over the rows: weights are loaded once, and in the backward pass every thread sums dw and db of its columns over its
// rows; the CTA adds its rows' sums, k_norm_join those of the CTAs, in a fixed order.
//
// Rows of whole 16-byte units go through a ring in shared memory (RING): every thread copies its own units of the rows to come asynchronously (cp.async) and reads back only
// what it copied itself, so that there is nothing to wait for but its own copies, several rows per group are under way whatever the registers hold, and the
// backward pass reads a row a second time from there.  Rows of any other width or alignment: a value per lane, the next row's values in registers.
// Sums and statistics are float32.  Rounded once: s to x's type, y, ds; the 8-bit form is that of the rounded y.
#pragma once
#include "psgd_values.cuh"

namespace psgd {

constexpr int NORM_UNIT = 8;
constexpr int NORM_THREADS = 512;                  // most threads of a CTA
constexpr int NORM_WARPS = NORM_THREADS / 32;

// Where the values of a thread's unit u lie in a row.  VEC: eight side by side (rows and widths of whole 16-byte units).  Else a value per lane: 32
// columns apart, the warp's lanes side by side, any width and alignment.  `n`: how many of the eight exist (from the first on).
template <bool VEC>
__device__ __forceinline__ int cell_col(int u) { return VEC ? u * 8 : (u & ~31) * 8 + (u & 31); }
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

// Mean and sum of squared deviations of a row from each thread's values.  `n`: how many a thread's units have, `have`: how many the warp has.
struct RowStats { float mean, m2; };
template <int VPT>
__device__ __forceinline__ RowStats row_stats(const float (&v)[VPT][8], const int (&n)[VPT], float have, int F, bool center, float2* mine, const float* counts) {
    const int warps = blockDim.x >> 5, lane = threadIdx.x & 31;
    float m = 0.f;
    if (center) {
        float sum = 0.f;
#pragma unroll
        for (int i = 0; i < VPT; ++i) sum += ((v[i][0] + v[i][1]) + (v[i][2] + v[i][3])) + ((v[i][4] + v[i][5]) + (v[i][6] + v[i][7]));
        m = warp_sum(sum) / fmaxf(have, 1.f);
    }
    float sq = 0.f;
#pragma unroll
    for (int i = 0; i < VPT; ++i)
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const float d = j < n[i] ? v[i][j] - m : 0.f;
            sq = fmaf(d, d, sq);
        }
    sq = warp_sum(sq);
    RowStats s{m, sq};
    if (warps > 1) {
        if (lane == 0) mine[threadIdx.x >> 5] = make_float2(m, sq);
        row_sync();
        if (center) {
            s.mean = 0.f;
            for (int w = 0; w < warps; ++w) s.mean = fmaf(counts[w], mine[w].x, s.mean);
            s.mean /= (float)F;
        }
        s.m2 = 0.f;
        for (int w = 0; w < warps; ++w) {
            const float d = mine[w].x - s.mean;
            s.m2 += fmaf(counts[w] * d, d, mine[w].y);
        }
    }
    return s;
}

// A thread's share of a ring: `stages` rows of its group, of each up to three operands.  Unit i of an operand lies at its plane + (i * blockDim.x + threadIdx.x) * 16; the second
// halves of float32 units follow in a plane of their own, so that a warp's accesses are side by side.
template <typename X> __device__ __forceinline__ int plane_bytes(int vpt) { return vpt * (int)blockDim.x * 8 * (int)sizeof(X); }
__device__ __forceinline__ void copy16(unsigned to, const void* from) { asm volatile("cp.async.cg.shared.global [%0], [%1], 16;\n" ::"r"(to), "l"(from) : "memory"); }
__device__ __forceinline__ uint4 shared16(unsigned at) {
    uint4 v;
    asm volatile("ld.shared.v4.u32 {%0, %1, %2, %3}, [%4];\n" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "r"(at) : "memory");
    return v;
}
template <typename X, int VPT>
__device__ __forceinline__ void ring_ask(unsigned plane, const X* row, const int (&col)[VPT], const int (&n)[VPT]) {
#pragma unroll
    for (int i = 0; i < VPT; ++i) {
        if (!n[i]) continue;
        const unsigned to = plane + (i * blockDim.x + threadIdx.x) * 16;
        copy16(to, row + col[i]);
        if (sizeof(X) == 4) copy16(to + VPT * blockDim.x * 16, row + col[i] + 4);
    }
}
template <typename X, int VPT>
__device__ __forceinline__ void ring_read(unsigned plane, int i, int n, float (&v)[8]) {
    const unsigned at = plane + (i * blockDim.x + threadIdx.x) * 16;
    uint4 a = make_uint4(0u, 0u, 0u, 0u), b = a;
    if (n) a = shared16(at);
    if (sizeof(X) == 4) {
        if (n) b = shared16(at + VPT * blockDim.x * 16);
        const unsigned w[8] = {a.x, a.y, a.z, a.w, b.x, b.y, b.z, b.w};
#pragma unroll
        for (int j = 0; j < 8; ++j) v[j] = __uint_as_float(w[j]);
    } else {
        widen(Raw16{a}, v);
    }
}
// One group of copies per row, empty ones behind the last row included: a row's have landed when at most stages - 1 younger groups are under way.
__device__ __forceinline__ void ring_commit() { asm volatile("cp.async.commit_group;\n" ::: "memory"); }
__device__ __forceinline__ void ring_wait(int stages) {
    if (stages == 4) asm volatile("cp.async.wait_group 3;\n" ::: "memory");
    else if (stages == 3) asm volatile("cp.async.wait_group 2;\n" ::: "memory");
    else asm volatile("cp.async.wait_group 1;\n" ::: "memory");
}

template <typename X, typename Y, bool RING, int VPT>
__global__ void __launch_bounds__(NORM_THREADS) k_norm_forward(const __grid_constant__ NormForward a) {
    typedef typename Cell<X, RING>::Raw Raw;
    extern __shared__ __align__(16) unsigned char ring_raw[];
    __shared__ float2 stat[2][NORM_WARPS];             // by rows taken in turn: a row's exchange is over when the next but one writes
    __shared__ float counts[NORM_WARPS];
    grid_trigger();
    const int F = a.F, tid = threadIdx.x, warps = blockDim.x >> 5;
    int col[VPT], n[VPT];
    int have = 0;
#pragma unroll
    for (int i = 0; i < VPT; ++i) {
        col[i] = cell_col<RING>(tid + i * (int)blockDim.x);
        n[i] = cell_count<RING>(col[i], F);
        have += n[i];
    }
    const float in_warp = (float)__reduce_add_sync(0xffffffffu, have);
    if (threadIdx.y == 0 && (tid & 31) == 0) counts[tid >> 5] = in_warp;
    __syncthreads();
    grid_wait();
    const X *x = (const X*)a.x, *r = (const X*)a.r;
    X* s = (X*)a.s;
    Y* y = (Y*)a.y;
    const long long step = (long long)gridDim.x * blockDim.y;
    long long row = (long long)blockIdx.x * blockDim.y + threadIdx.y;
    const int plane = plane_bytes<X>(VPT), stage = r ? 2 * plane : plane;
    const unsigned ring = RING ? smem_addr(ring_raw) + threadIdx.y * a.stages * stage : 0u;
    Raw next[VPT], add[VPT];
    const auto ask = [&](long long at, unsigned to) {
        if constexpr (RING) {
            if (at < a.T) {
                ring_ask<X, VPT>(to, x + at * a.ldx, col, n);
                if (r) ring_ask<X, VPT>(to + plane, r + at * a.ldr, col, n);
            }
            ring_commit();
        } else if (at < a.T) {
#pragma unroll
            for (int i = 0; i < VPT; ++i) {
                cell_load(next[i], x + at * a.ldx + col[i], n[i]);
                if (r) cell_load(add[i], r + at * a.ldr + col[i], n[i]);
            }
        }
    };
    if constexpr (RING) {
        for (int k = 0; k < a.stages; ++k) ask(row + k * step, ring + k * stage);
    } else {
        ask(row, 0u);
    }
    float w[VPT][8], b[VPT][8];
#pragma unroll
    for (int i = 0; i < VPT; ++i) {
        param_cell<RING>(w[i], a.w, col[i], n[i], 1.f);
        param_cell<RING>(b[i], a.b, col[i], n[i], 0.f);
    }
    const int G = (F + ACT_GROUP - 1) / ACT_GROUP;
    unsigned from = ring;
    for (int turn = 0; row < a.T; row += step, turn ^= 1) {
        float v[VPT][8];
        if constexpr (RING) ring_wait(a.stages);
#pragma unroll
        for (int i = 0; i < VPT; ++i) {
            float u[8];
            if constexpr (RING) {
                ring_read<X, VPT>(from, i, n[i], v[i]);
                if (r) ring_read<X, VPT>(from + plane, i, n[i], u);
            } else {
                widen(next[i], v[i]);
                if (r) widen(add[i], u);
            }
            if (r) {
#pragma unroll
                for (int j = 0; j < 8; ++j) v[i][j] += u[j];
                round_to<X>(v[i]);
            }
        }
        if constexpr (!RING) ask(row + step, 0u);
        if (s) {
#pragma unroll
            for (int i = 0; i < VPT; ++i) cell_store<RING>(s + row * a.lds + col[i], v[i], n[i]);
        }
        const RowStats st = row_stats<VPT>(v, n, in_warp, F, a.center, stat[turn] + threadIdx.y * warps, counts);
        if constexpr (RING) {                          // (every value has been used)
            ask(row + a.stages * step, from);
            from = from + stage == ring + a.stages * stage ? ring : from + stage;
        }
        const float f = rsqrtf(st.m2 / (float)F + a.eps);
        if (tid == 0) {
            a.rstd[row] = f;
            if (a.mean) a.mean[row] = st.mean;
        }
#pragma unroll
        for (int i = 0; i < VPT; ++i) {
            float o[8];
#pragma unroll
            for (int j = 0; j < 8; ++j) o[j] = fmaf((v[i][j] - st.mean) * f, w[i][j], b[i][j]);
            cell_store<RING>(y + row * a.ldy + col[i], o, n[i]);
            if (a.q) {
#pragma unroll
                for (int j = 0; j < 8; ++j) o[j] = j < n[i] ? o[j] : 0.f;
                round_to<Y>(o);
                cell_keep<RING>(o, col[i], row * G, G, a.q, a.scales);
            }
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

template <typename X, typename Y, bool RING, int VPT>
__global__ void __launch_bounds__(NORM_THREADS) k_norm_backward(const __grid_constant__ NormBackward a) {
    typedef typename Cell<X, RING>::Raw RawX;
    typedef typename Cell<Y, RING>::Raw RawY;
    extern __shared__ __align__(16) unsigned char ring_raw[];      // the ring; at the end the sums of the rows side by side, [blockDim.y][2][F]
    __shared__ float2 stat[2][NORM_WARPS];
    grid_trigger();
    const int F = a.F, tid = threadIdx.x, warps = blockDim.x >> 5;
    int col[VPT], n[VPT];
#pragma unroll
    for (int i = 0; i < VPT; ++i) {
        col[i] = cell_col<RING>(tid + i * (int)blockDim.x);
        n[i] = cell_count<RING>(col[i], F);
    }
    grid_wait();
    const Y* dy = (const Y*)a.dy;
    const X *x = (const X*)a.x, *add = (const X*)a.add;
    X* dx = (X*)a.dx;
    const long long step = (long long)gridDim.x * blockDim.y;
    long long row = (long long)blockIdx.x * blockDim.y + threadIdx.y;
    const int plane = plane_bytes<X>(VPT), plane_dy = plane_bytes<Y>(VPT), stage = plane_dy + (add ? 2 : 1) * plane;
    const unsigned ring = RING ? smem_addr(ring_raw) + threadIdx.y * a.stages * stage : 0u;
    RawX nx[VPT], na[VPT];
    RawY ny[VPT];
    float nm = 0.f, nf = 0.f;                          // the next row's mean and rstd
    const auto ask_stats = [&](long long at) {
        if (at >= a.T) return;
        nf = a.rstd[at];
        if (a.mean) nm = a.mean[at];
    };
    const auto ask = [&](long long at, unsigned to) {
        if constexpr (RING) {
            if (at < a.T) {
                ring_ask<Y, VPT>(to, dy + at * a.lddy, col, n);
                ring_ask<X, VPT>(to + plane_dy, x + at * a.ldx, col, n);
                if (add) ring_ask<X, VPT>(to + plane_dy + plane, add + at * a.ldadd, col, n);
            }
            ring_commit();
        } else if (at < a.T) {
#pragma unroll
            for (int i = 0; i < VPT; ++i) {
                cell_load(nx[i], x + at * a.ldx + col[i], n[i]);
                cell_load(ny[i], dy + at * a.lddy + col[i], n[i]);
                if (add) cell_load(na[i], add + at * a.ldadd + col[i], n[i]);
            }
        }
    };
    if constexpr (RING) {
        for (int k = 0; k < a.stages; ++k) ask(row + k * step, ring + k * stage);
    } else {
        ask(row, 0u);
    }
    ask_stats(row);
    float w[VPT][8], dw[VPT][8], db[VPT][8];
#pragma unroll
    for (int i = 0; i < VPT; ++i) {
        param_cell<RING>(w[i], a.w, col[i], n[i], 1.f);
#pragma unroll
        for (int j = 0; j < 8; ++j) dw[i][j] = db[i][j] = 0.f;
    }
    const float per = 1.f / (float)F;
    unsigned from = ring;
    for (int turn = 0; row < a.T; row += step, turn ^= 1) {
        RawX cx[VPT], ca[VPT];
        RawY cy[VPT];
        if constexpr (!RING) {
#pragma unroll
            for (int i = 0; i < VPT; ++i) { cx[i] = nx[i]; cy[i] = ny[i]; ca[i] = na[i]; }
            ask(row + step, 0u);
        }
        const float f = nf, m = nm;
        ask_stats(row + step);
        if constexpr (RING) ring_wait(a.stages);
        // a unit's x and dy, both times they are needed
        const auto values = [&](int i, float (&v)[8], float (&d)[8]) {
            if constexpr (RING) {
                ring_read<Y, VPT>(from, i, n[i], d);
                ring_read<X, VPT>(from + plane_dy, i, n[i], v);
            } else {
                widen(cx[i], v);
                widen(cy[i], d);
            }
        };
        float s1 = 0.f, s2 = 0.f;
#pragma unroll
        for (int i = 0; i < VPT; ++i) {
            float v[8], d[8];
            values(i, v, d);
#pragma unroll
            for (int j = 0; j < 8; ++j) {              // (dy and w are zeros where there is no value)
                const float xh = (v[j] - m) * f, g = d[j] * w[i][j];
                s1 += g;
                s2 = fmaf(g, xh, s2);
                dw[i][j] = fmaf(d[j], xh, dw[i][j]);
                db[i][j] += d[j];
            }
        }
        s1 = warp_sum(s1);
        s2 = warp_sum(s2);
        if (warps > 1) {
            float2* mine = stat[turn] + threadIdx.y * warps;
            if ((tid & 31) == 0) mine[tid >> 5] = make_float2(s1, s2);
            row_sync();
            s1 = s2 = 0.f;
            for (int k = 0; k < warps; ++k) { s1 += mine[k].x; s2 += mine[k].y; }
        }
        s1 = a.center ? s1 * per : 0.f;
        s2 *= per;
#pragma unroll
        for (int i = 0; i < VPT; ++i) {
            float v[8], d[8];
            values(i, v, d);
#pragma unroll
            for (int j = 0; j < 8; ++j) d[j] = f * (fmaf(-((v[j] - m) * f), s2, d[j] * w[i][j]) - s1);
            if (add) {
                if constexpr (RING) ring_read<X, VPT>(from + plane_dy + plane, i, n[i], v);
                else widen(ca[i], v);
#pragma unroll
                for (int j = 0; j < 8; ++j) d[j] += v[j];
            }
            cell_store<RING>(dx + row * a.lddx + col[i], d, n[i]);
        }
        if constexpr (RING) {
            ask(row + a.stages * step, from);
            from = from + stage == ring + a.stages * stage ? ring : from + stage;
        }
    }
    // the CTA's sums: its rows side by side (threadIdx.y) through shared memory; a CTA alone writes the results
    float* pw = gridDim.x == 1 ? a.dw : a.part + (size_t)blockIdx.x * 2 * F;
    float* pb = gridDim.x == 1 ? a.db : pw + F;
    const bool alone = blockDim.y == 1;
    float* sums = reinterpret_cast<float*>(ring_raw) + (size_t)threadIdx.y * 2 * F;
    if (RING) asm volatile("cp.async.wait_all;\n" ::: "memory");
    if (!alone) __syncthreads();
    float *to_w = alone ? pw : sums, *to_b = alone ? pb : sums + F;
#pragma unroll
    for (int i = 0; i < VPT; ++i)
#pragma unroll
        for (int j = 0; j < 8; ++j)
            if (j < n[i]) {
                const int c = col[i] + (RING ? j : 32 * j);
                to_w[c] = dw[i][j];
                if (to_b) to_b[c] = db[i][j];
            }
    if (alone) return;
    __syncthreads();
    for (int c = threadIdx.y * blockDim.x + tid; c < 2 * F; c += blockDim.x * blockDim.y) {
        float sum = 0.f;
        for (int k = 0; k < (int)blockDim.y; ++k) sum += reinterpret_cast<float*>(ring_raw)[(size_t)k * 2 * F + c];
        if (c < F) pw[c] = sum;
        else if (pb) pb[c - F] = sum;
    }
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
