// Layer norm of rows (also without centring), forward and backward.
//
//   s = x + r (rounded to x's type; s = x without r),  m = mean(s) (0 without centring),  f = 1 / sqrt(mean((s - m)^2) + eps),
//   y = (s - m) f w + b;
//   g = dy w,  xh = (s - m) f,  ds = f (g - mean(g) - xh mean(g xh)) + what reaches s from elsewhere  (mean(g) only with centring),
//   dw = sum over rows of dy xh,  db = sum over rows of dy.
//
// One pass over the operands, bound by HBM.  blockDim.x threads share a row (blockDim.y rows per CTA), each holds VPT units of eight values of it in
// registers between the statistics and the result.  The sum of squares is taken about the warp's own mean and the warps' results are
// joined exactly (squares about the joint mean = sum of the warps' squares + n_w (mean_w - mean)^2), so that a large mean costs no bits and
// a row takes one exchange between its warps.  The CTAs stay and walk over the rows: weights are loaded once, and in the backward pass every
// thread sums dw and db of its columns over the CTA's rows; those partial sums are added by k_norm_join in a fixed order.
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

template <typename X, typename Y, bool VEC, int VPT>
__global__ void __launch_bounds__(NORM_THREADS) k_norm_forward(const __grid_constant__ NormForward a) {
    typedef typename Cell<X, VEC>::Raw Raw;
    __shared__ float2 stat[2][NORM_WARPS];             // by rows taken in turn: a row's exchange is over when the next but one writes
    __shared__ float counts[NORM_WARPS];
    grid_trigger();
    const int F = a.F, tid = threadIdx.x, warps = blockDim.x >> 5;
    int col[VPT], n[VPT];
    int have = 0;
#pragma unroll
    for (int i = 0; i < VPT; ++i) {
        col[i] = cell_col<VEC>(tid + i * (int)blockDim.x);
        n[i] = cell_count<VEC>(col[i], F);
        have += n[i];
    }
    const float in_warp = (float)__reduce_add_sync(0xffffffffu, have);
    if (threadIdx.y == 0 && (tid & 31) == 0) counts[tid >> 5] = in_warp;
    __syncthreads();
    grid_wait();
    float w[VPT][8], b[VPT][8];
#pragma unroll
    for (int i = 0; i < VPT; ++i) {
        param_cell<VEC>(w[i], a.w, col[i], n[i], 1.f);
        param_cell<VEC>(b[i], a.b, col[i], n[i], 0.f);
    }
    const int G = (F + ACT_GROUP - 1) / ACT_GROUP;
    const X *x = (const X*)a.x, *r = (const X*)a.r;
    X* s = (X*)a.s;
    Y* y = (Y*)a.y;
    const long long step = (long long)gridDim.x * blockDim.y;
    long long row = (long long)blockIdx.x * blockDim.y + threadIdx.y;
    Raw next[VPT], add[VPT];
    const auto ask = [&](long long at) {
#pragma unroll
        for (int i = 0; i < VPT; ++i) {
            cell_load(next[i], x + at * a.ldx + col[i], n[i]);
            if (r) cell_load(add[i], r + at * a.ldr + col[i], n[i]);
        }
    };
    if (row < a.T) ask(row);
    for (int turn = 0; row < a.T; row += step, turn ^= 1) {
        float v[VPT][8];
#pragma unroll
        for (int i = 0; i < VPT; ++i) {
            widen(next[i], v[i]);
            if (r) {
                float u[8];
                widen(add[i], u);
#pragma unroll
                for (int j = 0; j < 8; ++j) v[i][j] += u[j];
                round_to<X>(v[i]);
            }
        }
        if (row + step < a.T) ask(row + step);
        if (s) {
#pragma unroll
            for (int i = 0; i < VPT; ++i) cell_store<VEC>(s + row * a.lds + col[i], v[i], n[i]);
        }
        const RowStats st = row_stats<VPT>(v, n, in_warp, F, a.center, stat[turn] + threadIdx.y * warps, counts);
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
            cell_store<VEC>(y + row * a.ldy + col[i], o, n[i]);
            if (a.q) {
#pragma unroll
                for (int j = 0; j < 8; ++j) o[j] = j < n[i] ? o[j] : 0.f;
                round_to<Y>(o);
                cell_keep<VEC>(o, col[i], row * G, G, a.q, a.scales);
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
    float* part;                                       // [CTAs][2][F]: dw, db
    float2* sums;                                      // wide rows: [T] mean(g), mean(g xh)
    int chunks;                                        // wide rows: CTAs that share a column
};
struct NormJoin { int F, parts; const float* part; float *dw, *db; };      // db: or nullptr

template <typename X, typename Y, bool VEC, int VPT>
__global__ void __launch_bounds__(NORM_THREADS) k_norm_backward(const __grid_constant__ NormBackward a) {
    typedef typename Cell<X, VEC>::Raw RawX;
    typedef typename Cell<Y, VEC>::Raw RawY;
    extern __shared__ float columns[];                 // [2][F] where a CTA takes several rows at a time
    __shared__ float2 stat[2][NORM_WARPS];
    grid_trigger();
    const int F = a.F, tid = threadIdx.x, warps = blockDim.x >> 5;
    int col[VPT], n[VPT];
#pragma unroll
    for (int i = 0; i < VPT; ++i) {
        col[i] = cell_col<VEC>(tid + i * (int)blockDim.x);
        n[i] = cell_count<VEC>(col[i], F);
    }
    grid_wait();
    float w[VPT][8], dw[VPT][8], db[VPT][8];
#pragma unroll
    for (int i = 0; i < VPT; ++i) {
        param_cell<VEC>(w[i], a.w, col[i], n[i], 1.f);
#pragma unroll
        for (int j = 0; j < 8; ++j) dw[i][j] = db[i][j] = 0.f;
    }
    const Y* dy = (const Y*)a.dy;
    const X *x = (const X*)a.x, *add = (const X*)a.add;
    X* dx = (X*)a.dx;
    const long long step = (long long)gridDim.x * blockDim.y;
    long long row = (long long)blockIdx.x * blockDim.y + threadIdx.y;
    RawX nx[VPT], na[VPT];
    RawY ny[VPT];
    float nm = 0.f, nf = 0.f;
    const auto ask = [&](long long at) {
        nf = a.rstd[at];
        if (a.mean) nm = a.mean[at];
#pragma unroll
        for (int i = 0; i < VPT; ++i) {
            cell_load(nx[i], x + at * a.ldx + col[i], n[i]);
            cell_load(ny[i], dy + at * a.lddy + col[i], n[i]);
            if (add) cell_load(na[i], add + at * a.ldadd + col[i], n[i]);
        }
    };
    if (row < a.T) ask(row);
    const float per = 1.f / (float)F;
    for (int turn = 0; row < a.T; row += step, turn ^= 1) {
        RawX cx[VPT], ca[VPT];
        RawY cy[VPT];
#pragma unroll
        for (int i = 0; i < VPT; ++i) { cx[i] = nx[i]; cy[i] = ny[i]; ca[i] = na[i]; }
        const float f = nf, m = nm;
        if (row + step < a.T) ask(row + step);
        float s1 = 0.f, s2 = 0.f;
#pragma unroll
        for (int i = 0; i < VPT; ++i) {
            float v[8], d[8];
            widen(cx[i], v);
            widen(cy[i], d);
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
            widen(cx[i], v);
            widen(cy[i], d);
#pragma unroll
            for (int j = 0; j < 8; ++j) d[j] = f * (fmaf(-((v[j] - m) * f), s2, d[j] * w[i][j]) - s1);
            if (add) {
                widen(ca[i], v);
#pragma unroll
                for (int j = 0; j < 8; ++j) d[j] += v[j];
            }
            cell_store<VEC>(dx + row * a.lddx + col[i], d, n[i]);
        }
    }
    // the CTA's sums: its rows side by side (threadIdx.y) one after the other
    float* part = a.part + (size_t)blockIdx.x * 2 * F;
    for (int k = 0; k < (int)blockDim.y; ++k) {
        const bool first = k == 0, last = k + 1 == (int)blockDim.y;
        if ((int)threadIdx.y == k) {
#pragma unroll
            for (int i = 0; i < VPT; ++i)
#pragma unroll
                for (int j = 0; j < 8; ++j)
                    if (j < n[i]) {
                        const int c = col[i] + (VEC ? j : 32 * j);
                        const float p = (first ? 0.f : columns[c]) + dw[i][j], q = (first ? 0.f : columns[F + c]) + db[i][j];
                        float* to = last ? part : columns;
                        to[c] = p;
                        to[F + c] = q;
                    }
        }
        if (!last) __syncthreads();
    }
}

// Wide rows: first the two sums of every row (a CTA per row), then dx and the sums over rows (256 units of the columns per CTA, `chunks` CTAs share the rows).
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
    float* part = a.part + (size_t)blockIdx.y * 2 * F;
#pragma unroll
    for (int j = 0; j < 8; ++j)
        if (j < n) {
            const int c = col + (VEC ? j : 32 * j);
            part[c] = dw[j];
            part[F + c] = db[j];
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
