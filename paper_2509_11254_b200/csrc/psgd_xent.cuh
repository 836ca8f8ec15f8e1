// Row kernels of the last layer's softmax cross entropy.
//
//   lse_t = log sum_v exp(l_tv),   loss_t = lse_t - l_{t, y_t}   (0 where y_t is the ignored label),
//   loss = sum_t w_t loss_t / Z,   Z = sum of w_t over the rows that count   (0 where Z = 0),
//   d loss / d l_tv = w_t (exp(l_tv - lse_t) - [v = y_t]) / Z.
//
// The product kernel leaves, per row and segment of 64 columns (128 without gradients), the maximum and the sum of exp(l - maximum), and per logit the
// distance from its segment's maximum in steps of 2^-10 in the base-two exponent (16 bits, at most 3.4e-4 of relative error in p,
// a sixth of the rounding of a bfloat16; the sums come from the unrounded logits).  k_xent_rows joins the segments of a row and
// rewrites the 16 bits of every logit as the bfloat16 gradient w_t (p - [v = y_t]), rounded once more so.  The label's own gradient comes from its unrounded
// logit.  1 / Z is left to the epilogues of the products that follow: it would put the same rounding error on every row.
// The losses and the label's p - 1 are formed from the maximum and the logarithm of the sum apart: their sum, the log-sum-exp, is rounded at
// the size of the logits, which for a token with 1 - p of 1e-5 was up to a fifth of its loss and gradient (now 7 roundings of 2^-24).
// Sums over rows and segments are formed in a fixed order; the last CTA to finish adds up the loss.
//
// Bound by HBM: k_xent_rows reads and writes 2 bytes per logit, a CTA per row (or part of one where rows are few), whose statistics it joins
// first.  Measured: 4096 x 32000 in 95 us, 5.5 TB/s, 84 % of a copy; forming the logits a second time instead would take
// 123 us of tensor-core time at a width of 768 and more at larger ones.  k_xent_loss reads 8 bytes per 128 logits: 16384 x 32000 in 15 us, 1 % of the product.
#pragma once
#include "psgd_tile.cuh"

namespace psgd {

constexpr int XE_THREADS = 256;
constexpr int XE_ROW_CTAS = 5;     // of k_xent_rows per multiprocessor: 48 registers (with 128, two CTAs, the kernel took 139 instead of 92 us on 4096 x 32000)
constexpr int XE_W_LABEL = 8;      // == PSGD_W_LABEL

struct RowsArgs {
    int rows, V, nseg;
    const float2* stats;
    const float* label_logit;
    const long long* labels;       // of these rows
    long long ignore;
    const float* weight;           // of these rows, or nullptr
    float* loss;                   // of these rows
    float* lse;
    unsigned short* q;             // k_xent_rows: exponents in, gradients out
    long long ldq;
    int* status;
    // the mean over all rows, by the last CTA
    double2* sums;                 // weighted loss and weight of one row (k_xent_rows) or of one CTA's rows (k_xent_loss), over all launches of this call
    int n_sums, first_sum;
    int* done;
    int done_at;                   // CTAs that report, over all launches of this call
    float* mean;
};

// weight of a row in the loss; `bad` rows have a label that is neither ignored nor a column
__device__ __forceinline__ float row_weight(const float* weight, long long i, long long label, long long ignore, int V, bool& bad) {
    const bool in = label >= 0 && label < V;
    bad = !in && label != ignore;
    return in && label != ignore ? (weight ? weight[i] : 1.f) : 0.f;
}

// Sums over the block of two values (fixed order); the result is valid in thread 0.
template <int N>
__device__ __forceinline__ double2 block_sum2(double x, double y) {
    __shared__ double sx[N / 32], sy[N / 32];
#pragma unroll
    for (int o = 16; o; o >>= 1) { x += __shfl_xor_sync(0xffffffffu, x, o); y += __shfl_xor_sync(0xffffffffu, y, o); }
    if ((threadIdx.x & 31) == 0) { sx[threadIdx.x >> 5] = x; sy[threadIdx.x >> 5] = y; }
    __syncthreads();
    if (threadIdx.x == 0)
        for (int i = 1; i < N / 32; ++i) { x += sx[i]; y += sy[i]; }
    return make_double2(x, y);
}

// the last CTA to get here adds up the loss of all rows
__device__ __forceinline__ void report_rows(const RowsArgs& a) {
    __shared__ int last;
    __syncthreads();
    if (threadIdx.x == 0) {
        __threadfence();
        last = atomicAdd(a.done, 1) == a.done_at - 1;
    }
    __syncthreads();
    if (!last) return;
    __threadfence();
    double num = 0.0, z = 0.0;
    constexpr int UN = 4;                                      // under way per thread; more registers would cost the kernel occupancy
    for (int b = threadIdx.x; b < a.n_sums; b += UN * XE_THREADS) {
        double2 s[UN];
#pragma unroll
        for (int j = 0; j < UN; ++j) s[j] = __ldcg(a.sums + min(b + j * XE_THREADS, a.n_sums - 1));
#pragma unroll
        for (int j = 0; j < UN; ++j)
            if (b + j * XE_THREADS < a.n_sums) { num += s[j].x; z += s[j].y; }
    }
    const double2 s = block_sum2<XE_THREADS>(num, z);
    if (threadIdx.x == 0) *a.mean = (s.y != 0.0 || s.x != s.x) ? (float)(s.x / s.y) : 0.f;
}

// Statistics of a row: its maximum `top` and `rest`, the sum of exp(l - top) less the 1 of the maximum itself (-1 where there is nothing). Where
// one logit stands far above the others, rest is 1 - p of it and keeps all its bits, which a sum next to 1 would lose.
__device__ __forceinline__ void merge_stat(float& top, float& rest, float t, float r, float log2e = LOG2E) {
    const bool first = top >= t;
    const float high = first ? top : t, low = first ? t : top, from = high == -INFINITY ? 0.f : high;
    rest = fmaf(1.f + (first ? r : rest), ex2((low - from) * log2e), first ? rest : r);
    top = high;
}
__device__ __forceinline__ void warp_stat(float& top, float& rest, float log2e = LOG2E) {
#pragma unroll
    for (int o = 16; o; o >>= 1) {
        const float t = __shfl_xor_sync(0xffffffffu, top, o), r = __shfl_xor_sync(0xffffffffu, rest, o);
        merge_stat(top, rest, t, r, log2e);
    }
}
// the row's outputs (the loss not from lse, whose rounding is one of the size of the logits); returns its share of the loss and of the weight
__device__ __forceinline__ double2 write_loss(const RowsArgs& a, int row, float top, float log_sum) {
    const long long label = a.labels[row];
    bool bad;
    const float w = row_weight(a.weight, row, label, a.ignore, a.V, bad);
    float loss = 0.f;
    if (bad) { loss = NAN; atomicOr(a.status, XE_W_LABEL); }
    else if (label != a.ignore) loss = (top - a.label_logit[row]) + log_sum;
    a.lse[row] = top + log_sum;
    a.loss[row] = loss;
    return make_double2(bad ? (double)loss : label != a.ignore ? (double)w * (double)loss : 0.0, (double)w);     // a bad row's NaN reaches the mean
}

// Loss only: one warp per row.
__global__ void __launch_bounds__(XE_THREADS) k_xent_loss(const __grid_constant__ RowsArgs a) {
    __shared__ double2 mine[XE_THREADS / 32];
    grid_trigger();
    grid_wait();
    const int warp = threadIdx.x >> 5, row = blockIdx.x * (XE_THREADS / 32) + warp, lane = threadIdx.x & 31;
    double2 share = make_double2(0.0, 0.0);
    if (row < a.rows) {
        float top = -INFINITY, rest = -1.f;
        for (int j = lane; j < a.nseg; j += 8 * 32) {
            float2 s[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) s[i] = j + 32 * i < a.nseg ? a.stats[(size_t)row * a.nseg + j + 32 * i] : make_float2(-INFINITY, 0.f);
#pragma unroll
            for (int i = 0; i < 8; ++i) merge_stat(top, rest, s[i].x, s[i].y - 1.f);
        }
        warp_stat(top, rest);
        if (lane == 0) share = write_loss(a, row, top, log1pf(rest));
    }
    if (lane == 0) mine[warp] = share;
    __syncthreads();
    if (threadIdx.x == 0) {
        for (int i = 1; i < XE_THREADS / 32; ++i) { share.x += mine[i].x; share.y += mine[i].y; }
        a.sums[a.first_sum + blockIdx.x] = share;
    }
    report_rows(a);
}

// A row's stored exponents, units u0.. of eight, to w p in bfloat16 (zeros where the row does not count); `exponent`: of the largest p of a segment, from its maximum.
template <typename Exponent>
__device__ __forceinline__ void rewrite_exponents(uint4* q, const float2* st, int u0, int u1, float w, bool counts, float poison, Exponent&& exponent) {
    const int tid = threadIdx.x;
    constexpr int UN = 4;
    for (int b = u0 + tid; b < u1; b += XE_THREADS * UN) {
        uint4 v[UN];
        float ref[UN];
#pragma unroll
        for (int i = 0; i < UN; ++i) {
            const int u = b + i * XE_THREADS;
            if (u < u1) { v[i] = q[u]; ref[i] = st[u / (XE_SEG / 8)].x; }
        }
#pragma unroll
        for (int i = 0; i < UN; ++i) {
            const int u = b + i * XE_THREADS;
            if (u >= u1) break;
            const float off = exponent(ref[i]);
            const unsigned x[4] = {v[i].x, v[i].y, v[i].z, v[i].w};
            float d[8];
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const unsigned bits = (j & 1) ? x[j / 2] >> 16 : x[j / 2] & 0xffffu;
                const float steps = __uint_as_float(0x4B000000u | bits) - XE_MAGIC;
                const float p = ex2(fmaf(steps, -1.f / XE_STEPS, off));
                d[j] = (bits == XE_NONE ? poison : p) * w;
            }
            uint4 o = make_uint4(pack_bf16(d[0], d[1]), pack_bf16(d[2], d[3]), pack_bf16(d[4], d[5]), pack_bf16(d[6], d[7]));
            if (!counts) o = make_uint4(0u, 0u, 0u, 0u);
            q[u] = o;
        }
    }
}

// Loss and gradient of the logits: blockIdx.x = row, blockIdx.y = part of its columns.
__global__ void __launch_bounds__(XE_THREADS, XE_ROW_CTAS) k_xent_rows(const __grid_constant__ RowsArgs a) {
    grid_trigger();
    grid_wait();
    __shared__ float2 ws[XE_THREADS / 32];
    const int row = blockIdx.x, tid = threadIdx.x;
    const float2* st = a.stats + (size_t)row * a.nseg;
    float top = -INFINITY, rest = -1.f;
    for (int j = tid; j < a.nseg; j += XE_THREADS) merge_stat(top, rest, st[j].x, st[j].y - 1.f);
    warp_stat(top, rest);
    if ((tid & 31) == 0) ws[tid >> 5] = make_float2(top, rest);
    __syncthreads();
    top = ws[0].x;
    rest = ws[0].y;
#pragma unroll
    for (int i = 1; i < XE_THREADS / 32; ++i) merge_stat(top, rest, ws[i].x, ws[i].y);
    const float log_sum = log1pf(rest);
    if (blockIdx.y == 0 && tid == 0) a.sums[a.first_sum + row] = write_loss(a, row, top, log_sum);

    const long long label = a.labels[row];
    bool bad;
    const float w = row_weight(a.weight, row, label, a.ignore, a.V, bad);
    const bool counts = !bad && label != a.ignore;
    const float poison = (top + log_sum) - (top + log_sum);       // 0, or NaN where the row's logits were not finite
    uint4* q = reinterpret_cast<uint4*>(a.q + (size_t)row * a.ldq);
    const int units = (a.V + 7) / 8, per = (units + gridDim.y - 1) / gridDim.y;
    const int u0 = blockIdx.y * per, u1 = min(units, u0 + per);
    rewrite_exponents(q, st, u0, u1, w, counts, poison, [&](float ref) { return ((ref - top) - log_sum) * LOG2E + poison; });
    // the label's column again, by the thread that has just written it: p - 1 = (exp(l_y - top) - 1 - rest) / (1 + rest), without cancellation where
    // the label is the maximum
    const int lunit = counts ? (int)(label >> 3) : -1;
    if (lunit >= u0 && lunit < u1 && (lunit - u0) % XE_THREADS == tid) {
        const float d = ((ex2((a.label_logit[row] - top) * LOG2E) - 1.f) - rest) / (1.f + rest) + poison;
        reinterpret_cast<__nv_bfloat16*>(q)[label] = __float2bfloat16_rn(d * w);
    }
    report_rows(a);
}

}  // namespace psgd
