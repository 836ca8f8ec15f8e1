// Row kernels of the last layer's distance from a teacher of whom a few logits per row are known.
//
//   p_t = softmax(l_t / tau) over all V columns,   q_t = softmax(z_t / tau) over the row's list of entries (column i_k, teacher's logit z_k),
//   loss_t = tau^2 sum_k q_k (log q_k - log p_{i_k})   (0 for a row without an entry),
//   loss = sum_t w_t loss_t / Z,   Z = sum of w_t over the rows that have an entry   (0 where Z = 0),
//   d loss / d l_tv = w_t tau (p_tv - sum of q_k over the entries of column v) / Z.
//
// k_teach goes before the product: the teacher's probabilities, and the entries of every 32 rows ordered by segments of 128 columns, which is what a warp of
// the product's epilogue holds at a time, so that it finds the entries whose logits it has without a search.  It leaves the logits of all entries
// in float32; the other columns take the way of the cross entropy (psgd_xent.cuh): exponents in 16 bits, rewritten in place as bfloat16 gradients, here of
// l / tau.  At the entries' columns the gradient comes from the unrounded logit.  As there, sums of exponentials are kept without the 1 of their
// maximum: p - q of a column of which both are sure is ((e_p - e_q) + e_p rest_q - e_q rest_p) / ((1 + rest_p) (1 + rest_q)), e the exponential relative to the maximum.
// tau / Z is left to the epilogues of the products that follow.
//
// Bound as the cross entropy's kernels are (k_teach_rows: 2 bytes per logit read and written); k_teach reads 10 or 12 bytes per entry.
#pragma once
#include "psgd_xent.cuh"

namespace psgd {

constexpr int TEACH_ROWS = 32;     // rows of a block of entries
constexpr int TEACH_COLS = 128;    // columns of a segment
constexpr int TEACH_BINS = 2048;   // segments that k_teach counts at a time
constexpr int TEACH_MOST = 1024;   // entries of a row (k_teach_rows holds a row's in shared memory)

struct TeachArgs {
    long long T;
    int V, K;
    const void* logits;            // [T][K] float32 or bfloat16
    int bf16;
    long long ldl;
    const long long* index;        // [T][K]; negative: no entry
    long long ldi;
    float inv_tau;
    int nbins;
    float* z;                      // [T][K] (z - the row's maximum) / tau, -inf: no entry
    int* col;                      // [T][K] column, -1: no entry
    float* rest;                   // [T] sum of exp(z) without the maximum's 1
    long long* label;              // [T] 0: the row counts, -1: it has no entry, -2: an entry's column does not exist
    int* bins;                     // [blocks][nbins + 1]
    unsigned* entries;             // [blocks][32 K]
};

// One CTA per 32 rows.
__global__ void __launch_bounds__(256) k_teach(const __grid_constant__ TeachArgs a) {
    __shared__ int count[TEACH_BINS], warps[8];
    __shared__ int base, total;
    grid_trigger();
    grid_wait();
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, K = a.K;
    const long long row0 = (long long)blockIdx.x * TEACH_ROWS;
    const int rows = (int)min((long long)TEACH_ROWS, a.T - row0);
    const auto logit = [&](long long row, int k) {
        return a.bf16 ? __bfloat162float(((const __nv_bfloat16*)a.logits)[row * a.ldl + k]) : ((const float*)a.logits)[row * a.ldl + k];
    };
    for (int r = warp; r < rows; r += 8) {
        const long long row = row0 + r;
        float top = -INFINITY;
        int first = K;                                 // of the entries with the largest logit
        bool any = false, bad = false;
        for (int k = lane; k < K; k += 32) {
            const long long i = a.index[row * a.ldi + k];
            const float z = logit(row, k);
            if (i < 0 || z == -INFINITY) continue;
            any = true;
            bad = bad || i >= a.V;
            if (z > top) { top = z; first = k; }
        }
#pragma unroll
        for (int o = 16; o; o >>= 1) {
            const float t = __shfl_xor_sync(0xffffffffu, top, o);
            const int f = __shfl_xor_sync(0xffffffffu, first, o);
            if (t > top || (t == top && f < first)) { top = t; first = f; }
        }
        any = __any_sync(0xffffffffu, any);
        bad = __any_sync(0xffffffffu, bad);
        float rest = 0.f;
        for (int k = lane; k < K; k += 32) {
            const long long i = a.index[row * a.ldi + k];
            const float z = logit(row, k);
            const bool there = !bad && i >= 0 && z != -INFINITY;
            // (a maximum that is not finite leaves NaN behind; so does a NaN)
            const float x = there ? (z - top) * a.inv_tau : -INFINITY;
            if (there && (k != first || x != x)) rest += expf(x);
            a.z[row * K + k] = x;
            a.col[row * K + k] = there ? (int)i : -1;
        }
#pragma unroll
        for (int o = 16; o; o >>= 1) rest += __shfl_xor_sync(0xffffffffu, rest, o);
        if (lane == 0) {
            a.rest[row] = rest;
            a.label[row] = bad ? -2 : any ? 0 : -1;
        }
    }
    __syncthreads();
    // the block's entries by segment, TEACH_BINS segments at a time
    int* bins = a.bins + (size_t)blockIdx.x * (a.nbins + 1);
    unsigned* out = a.entries + (size_t)blockIdx.x * TEACH_ROWS * K;
    const int* col = a.col + row0 * K;
    const int n = rows * K;
    if (tid == 0) base = 0;
    for (int b0 = 0; b0 < a.nbins; b0 += TEACH_BINS) {
        const int here = min(TEACH_BINS, a.nbins - b0);
        for (int i = tid; i < TEACH_BINS; i += 256) count[i] = 0;
        __syncthreads();
        for (int e = tid; e < n; e += 256) {
            const int b = col[e] / TEACH_COLS - b0;
            if (col[e] >= 0 && b >= 0 && b < here) atomicAdd(count + b, 1);
        }
        __syncthreads();
        // where each begins: eight per thread, then the threads of a warp, then the warps
        int mine[TEACH_BINS / 256], sum = 0;
#pragma unroll
        for (int i = 0; i < TEACH_BINS / 256; ++i) { mine[i] = count[tid * (TEACH_BINS / 256) + i]; sum += mine[i]; }
        int upto = sum;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const int v = __shfl_up_sync(0xffffffffu, upto, o);
            if (lane >= o) upto += v;
        }
        if (lane == 31) warps[warp] = upto;
        __syncthreads();
        int at = base + upto - sum;
        for (int w = 0; w < warp; ++w) at += warps[w];
#pragma unroll
        for (int i = 0; i < TEACH_BINS / 256; ++i) {
            const int b = tid * (TEACH_BINS / 256) + i;
            count[b] = at;
            if (b < here) bins[b0 + b] = at;
            at += mine[i];
        }
        if (tid == 255) total = at;
        __syncthreads();
        for (int e = tid; e < n; e += 256) {
            const int c = col[e], b = c / TEACH_COLS - b0;
            if (c < 0 || b < 0 || b >= here) continue;
            const int r = e / K;
            out[atomicAdd(count + b, 1)] = (unsigned)(e - r * K) << 12 | (unsigned)r << 7 | (unsigned)(c % TEACH_COLS);       // (their order within a segment does not matter)
        }
        if (tid == 0) base = total;
        __syncthreads();
    }
    if (tid == 0) bins[a.nbins] = base;
}

struct TeachRows {
    int K;
    const float* z;                // of these rows, as all below
    const int* col;
    const float* rest;
    const float* logit;            // [rows][K], of the entries
    float tau, inv_tau;
};

// An entry's share of (1 + rest_q) sum q (log q - log p); nothing where q is 0, whatever p is.
__device__ __forceinline__ double teach_term(float z, float logit, float top, float inv_tau, float log_q, float log_p) {
    const float e = expf(z);
    return e == 0.f ? 0.0 : (double)e * (double)((z - log_q) - ((logit - top) * inv_tau - log_p));
}
// the row's outputs from the sum of its terms; returns its share of the loss and of the weight
__device__ __forceinline__ double2 write_distance(const RowsArgs& a, const TeachRows& t, int row, float top, float log_sum, double sum) {
    const long long label = a.labels[row];
    const float w = label == 0 ? (a.weight ? a.weight[row] : 1.f) : 0.f;
    float loss = 0.f;
    if (label == -2) { loss = NAN; atomicOr(a.status, XE_W_LABEL); }
    else if (label == 0) loss = (float)((double)t.tau * t.tau * sum / (1.0 + (double)t.rest[row]));
    const float lse = top * t.inv_tau + log_sum;
    a.lse[row] = lse;
    if (label == 0) loss += lse - lse == 0.f ? 0.f : NAN;          // a row whose logits are not finite
    a.loss[row] = loss;
    return make_double2(label == -2 ? (double)loss : label == 0 ? (double)w * (double)loss : 0.0, (double)w);
}

// Loss only: one warp per row.
__global__ void __launch_bounds__(XE_THREADS) k_teach_loss(const __grid_constant__ RowsArgs a, const __grid_constant__ TeachRows t) {
    __shared__ double2 mine[XE_THREADS / 32];
    grid_trigger();
    grid_wait();
    const int warp = threadIdx.x >> 5, row = blockIdx.x * (XE_THREADS / 32) + warp, lane = threadIdx.x & 31;
    const float log2e = LOG2E * t.inv_tau;
    double2 share = make_double2(0.0, 0.0);
    if (row < a.rows) {
        float top = -INFINITY, rest = -1.f;
        for (int j = lane; j < a.nseg; j += 8 * 32) {
            float2 s[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) s[i] = j + 32 * i < a.nseg ? a.stats[(size_t)row * a.nseg + j + 32 * i] : make_float2(-INFINITY, 0.f);
#pragma unroll
            for (int i = 0; i < 8; ++i) merge_stat(top, rest, s[i].x, s[i].y - 1.f, log2e);
        }
        warp_stat(top, rest, log2e);
        const float log_p = log1pf(rest), log_q = log1pf(t.rest[row]);
        double sum = 0.0;
        for (int k = lane; k < t.K; k += 32) {
            const size_t at = (size_t)row * t.K + k;
            if (t.col[at] >= 0) sum += teach_term(t.z[at], t.logit[at], top, t.inv_tau, log_q, log_p);
        }
#pragma unroll
        for (int o = 16; o; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
        if (lane == 0) share = write_distance(a, t, row, top, log_p, sum);
    }
    if (lane == 0) mine[warp] = share;
    __syncthreads();
    if (threadIdx.x == 0) {
        for (int i = 1; i < XE_THREADS / 32; ++i) { share.x += mine[i].x; share.y += mine[i].y; }
        a.sums[a.first_sum + blockIdx.x] = share;
    }
    report_rows(a);
}

// Loss and gradient of the logits: blockIdx.x = row, blockIdx.y = part of its columns.
__global__ void __launch_bounds__(XE_THREADS, XE_ROW_CTAS) k_teach_rows(const __grid_constant__ RowsArgs a, const __grid_constant__ TeachRows t) {
    grid_trigger();
    grid_wait();
    __shared__ float2 ws[XE_THREADS / 32];
    __shared__ int cols[TEACH_MOST];
    __shared__ float es[TEACH_MOST];                   // exp(z)
    const int row = blockIdx.x, tid = threadIdx.x;
    const float log2e = LOG2E * t.inv_tau;
    const float2* st = a.stats + (size_t)row * a.nseg;
    for (int k = tid; k < t.K; k += XE_THREADS) {
        cols[k] = t.col[(size_t)row * t.K + k];
        es[k] = expf(t.z[(size_t)row * t.K + k]);
    }
    float top = -INFINITY, rest = -1.f;
    for (int j = tid; j < a.nseg; j += XE_THREADS) merge_stat(top, rest, st[j].x, st[j].y - 1.f, log2e);
    warp_stat(top, rest, log2e);
    if ((tid & 31) == 0) ws[tid >> 5] = make_float2(top, rest);
    __syncthreads();
    top = ws[0].x;
    rest = ws[0].y;
#pragma unroll
    for (int i = 1; i < XE_THREADS / 32; ++i) merge_stat(top, rest, ws[i].x, ws[i].y, log2e);
    const float log_sum = log1pf(rest), rest_q = t.rest[row];
    const float* logit = t.logit + (size_t)row * t.K;
    if (blockIdx.y == 0) {
        const float log_q = log1pf(rest_q);
        double sum = 0.0;
        for (int k = tid; k < t.K; k += XE_THREADS)
            if (cols[k] >= 0) sum += teach_term(t.z[(size_t)row * t.K + k], logit[k], top, t.inv_tau, log_q, log_sum);
        const double2 s = block_sum2<XE_THREADS>(sum, 0.0);
        if (tid == 0) a.sums[a.first_sum + row] = write_distance(a, t, row, top, log_sum, s.x);
    }
    const bool counts = a.labels[row] == 0;
    const float w = counts ? (a.weight ? a.weight[row] : 1.f) : 0.f;
    const float lse = top * t.inv_tau + log_sum, poison = lse - lse;         // 0, or NaN where the row's logits were not finite
    uint4* q = reinterpret_cast<uint4*>(a.q + (size_t)row * a.ldq);
    const int units = (a.V + 7) / 8, per = (units + gridDim.y - 1) / gridDim.y;
    const int u0 = blockIdx.y * per, u1 = min(units, u0 + per);
    rewrite_exponents(q, st, u0, u1, w, counts, poison, [&](float ref) { return ((ref - top) * t.inv_tau - log_sum) * LOG2E + poison; });
    __syncthreads();
    // the entries' columns again; a column that is listed more than once by the first of its entries
    if (counts) {
        const float both = 1.f / ((1.f + rest) * (1.f + rest_q));
        for (int k = tid; k < t.K; k += XE_THREADS) {
            const int c = cols[k];
            if (c < 0 || (c >> 3) < u0 || (c >> 3) >= u1) continue;
            bool first = true;
            float e_q = 0.f;
            for (int j = 0; j < t.K; ++j)
                if (cols[j] == c) {
                    first = first && j >= k;
                    e_q += es[j];
                }
            if (!first) continue;
            const float e_p = ex2((logit[k] - top) * log2e);
            const float d = (((e_p - e_q) + e_p * rest_q) - e_q * rest) * both + poison;
            reinterpret_cast<__nv_bfloat16*>(q)[c] = __float2bfloat16_rn(d * w);
        }
    }
    report_rows(a);
}

}  // namespace psgd
