// Row kernels of the last layer's distance from a teacher of whom a few logits per row are known.
//
//   p_t = softmax(l_t / tau) over all V columns,   q_t = softmax(z_t / tau) over the row's list of entries (column i_k, teacher's logit z_k),
//   loss_t = tau^2 sum_k q_k (log q_k - log p_{i_k})   (0 for a row without an entry),
//   loss = sum_t w_t loss_t / Z,   Z = sum of w_t over the rows that have an entry   (0 where Z = 0),
//   d loss / d l_tv = w_t tau (p_tv - sum of q_k over the entries of column v) / Z.
//
// k_teach goes before the product: the teacher's probabilities, and the entries of every 32 rows ordered by blocks of 32 columns, which is what a warp of
// the product's epilogue turns into rows at a time, so that it finds the entries whose logits it has without a search.  It leaves the logits of all entries
// in float32; the other columns take the way of the cross entropy (psgd_xent.cuh): exponents in 16 bits, rewritten in place as bfloat16 gradients, here of
// l / tau.  At the entries' columns the gradient comes from the unrounded logit.  As there, sums of exponentials are kept without the 1 of their
// maximum: p - q of a column of which both are sure is ((e_p - e_q) + e_p rest_q - e_q rest_p) / ((1 + rest_p) (1 + rest_q)), e the exponential relative to the maximum.
// tau / Z is left to the epilogues of the products that follow.
//
// Bound as the cross entropy's kernels are (k_teach_rows: 2 bytes per logit read and written).
#pragma once
#include "psgd_xent.cuh"

namespace psgd {

constexpr int TEACH_ROWS = 32;     // rows of a block of entries
constexpr int TEACH_COLS = 32;     // columns of a block
constexpr int TEACH_BINS = 4096;   // blocks of columns that k_teach counts at a time
constexpr int TEACH_THREADS = 1024;
constexpr int TEACH_HELD = 4;      // entries per lane that k_teach keeps in registers
constexpr int TEACH_PAIRS = 128;   // entries of a row up to which k_teach_rows compares every pair
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
    int* bins;                     // [row blocks][nbins + 1]; nullptr: only `label` is written
    unsigned* entries;             // [row blocks][32 K]
};

// One CTA per 32 rows, a warp per row.  Bound by latency (10 or 12 bytes per entry are read and 12 written): a row's entries are all asked for at once and held in
// registers where there are up to 128 of them, longer lists are read again.  4096 rows of 64 entries: 12 us with four rows per warp one after the other, 6 us so.
__global__ void __launch_bounds__(TEACH_THREADS) k_teach(const __grid_constant__ TeachArgs a) {
    __shared__ int count[TEACH_BINS], warps[TEACH_THREADS / 32];
    __shared__ int base;
    constexpr int EACH = TEACH_BINS / TEACH_THREADS;
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, K = a.K;
    for (int i = tid; i < TEACH_BINS; i += TEACH_THREADS) count[i] = 0;
    if (tid == 0) base = 0;
    __syncthreads();
    grid_wait();
    grid_trigger();                                    // after the wait: the product's loads begin when this lets it start, and rely on all that came before being done
    const long long row = (long long)blockIdx.x * TEACH_ROWS + warp;
    const bool held = K <= 32 * TEACH_HELD, live = row < a.T;
    const long long* index = a.index + row * a.ldi;
    const auto logit = [&](int k) { return a.bf16 ? __bfloat162float(((const __nv_bfloat16*)a.logits)[row * a.ldl + k]) : ((const float*)a.logits)[row * a.ldl + k]; };
    long long mine[TEACH_HELD];
    float z[TEACH_HELD];
    int col[TEACH_HELD];
    if (live && held) {
#pragma unroll
        for (int j = 0; j < TEACH_HELD; ++j) {
            const int k = lane + 32 * j;
            mine[j] = k < K ? index[k] : -1;
            z[j] = k < K ? logit(k) : -INFINITY;
        }
    }
    // calls f(k, its index, its logit, place among the held ones)
    const auto entries = [&](auto&& f) {
        if (held) {
#pragma unroll
            for (int j = 0; j < TEACH_HELD; ++j)
                if (lane + 32 * j < K) f(lane + 32 * j, mine[j], z[j], j);
        } else {
            for (int k = lane; k < K; k += 32) f(k, index[k], logit(k), 0);
        }
    };
    if (live) {
        float top = -INFINITY;
        int first = K;                                 // of the entries with the largest logit
        bool any = false, bad = false;
        entries([&](int k, long long i, float v, int) {
            if (i < 0 || v == -INFINITY) return;
            any = true;
            bad = bad || i >= a.V;
            if (v > top) { top = v; first = k; }
        });
#pragma unroll
        for (int o = 16; o; o >>= 1) {
            const float t = __shfl_xor_sync(0xffffffffu, top, o);
            const int f = __shfl_xor_sync(0xffffffffu, first, o);
            if (t > top || (t == top && f < first)) { top = t; first = f; }
        }
        any = __any_sync(0xffffffffu, any);
        bad = __any_sync(0xffffffffu, bad);
        if (lane == 0) a.label[row] = bad ? -2 : any ? 0 : -1;
        if (!a.bins) return;
        float rest = 0.f;
        entries([&](int k, long long i, float v, int j) {
            const bool there = !bad && i >= 0 && v != -INFINITY;
            // (a maximum that is not finite leaves NaN behind; so does a NaN)
            const float x = there ? (v - top) * a.inv_tau : -INFINITY;
            if (there && (k != first || x != x)) rest += expf(x);
            const int c = there ? (int)i : -1;
            if (held) col[j] = c;
            a.z[row * K + k] = x;
            a.col[row * K + k] = c;
        });
#pragma unroll
        for (int o = 16; o; o >>= 1) rest += __shfl_xor_sync(0xffffffffu, rest, o);
        if (lane == 0) a.rest[row] = rest;
    }
    if (!a.bins) return;
    // the rows' entries by block of columns, TEACH_BINS blocks at a time
    int* bins = a.bins + (size_t)blockIdx.x * (a.nbins + 1);
    unsigned* out = a.entries + (size_t)blockIdx.x * TEACH_ROWS * K;
    const int* cols = a.col + row * K;
    // calls f(k, column) for the row's entries (a lane's own ones, which it has written itself)
    const auto columns = [&](auto&& f) {
        if (!live) return;
        if (held) {
#pragma unroll
            for (int j = 0; j < TEACH_HELD; ++j)
                if (lane + 32 * j < K && col[j] >= 0) f(lane + 32 * j, col[j]);
        } else {
            for (int k = lane; k < K; k += 32)
                if (cols[k] >= 0) f(k, cols[k]);
        }
    };
    for (int b0 = 0; b0 < a.nbins; b0 += TEACH_BINS) {
        const int here = min(TEACH_BINS, a.nbins - b0);
        columns([&](int, int c) {
            const int b = c / TEACH_COLS - b0;
            if (b >= 0 && b < here) atomicAdd(count + b, 1);
        });
        __syncthreads();
        // where each begins: a few per thread, then the threads of a warp, then the warps
        int mine_of[EACH], sum = 0;
#pragma unroll
        for (int i = 0; i < EACH; ++i) { mine_of[i] = count[tid * EACH + i]; sum += mine_of[i]; }
        int upto = sum;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const int v = __shfl_up_sync(0xffffffffu, upto, o);
            if (lane >= o) upto += v;
        }
        if (lane == 31) warps[warp] = upto;
        __syncthreads();
        int before = lane < warp ? warps[lane] : 0, all = warps[lane];
#pragma unroll
        for (int o = 16; o; o >>= 1) {
            before += __shfl_xor_sync(0xffffffffu, before, o);
            all += __shfl_xor_sync(0xffffffffu, all, o);
        }
        const int begin = base;
        int at = begin + before + upto - sum;
#pragma unroll
        for (int i = 0; i < EACH; ++i) {
            const int b = tid * EACH + i;
            count[b] = at;
            if (b < here) bins[b0 + b] = at;
            at += mine_of[i];
        }
        __syncthreads();
        columns([&](int k, int c) {
            const int b = c / TEACH_COLS - b0;
            if (b < 0 || b >= here) return;
            out[atomicAdd(count + b, 1)] = (unsigned)k << 10 | (unsigned)warp << 5 | (unsigned)(c % TEACH_COLS);       // (their order within a block does not matter)
        });
        if (tid == 0) {
            base = begin + all;
            if (b0 + TEACH_BINS >= a.nbins) bins[a.nbins] = begin + all;
        }
        if (b0 + TEACH_BINS >= a.nbins) break;
        __syncthreads();
        for (int i = tid; i < TEACH_BINS; i += TEACH_THREADS) count[i] = 0;
        __syncthreads();
    }
}

// The loss of one token: its logits without the tensor cores, whose tiles of 256 rows would work on one that exists.  A CTA forms those of 128 columns, a warp four of them at a
// time, every lane 16 bytes of their rows, ONE_UNITS times before it uses them; the hidden state lies in shared memory as float32.  Then the statistics and the listed
// entries' logits as the product's epilogue leaves them.  Bound by reading the vocabulary matrix once: 32000 x 768 in 12.8 us, of which the bytes take 7.5 (the tiles: 17.4 us);
// the whole call on 131072 x 2048 in 89 us (97), the bytes 82.  Two tokens at a time cost as much as the tiles.  As k_tile it starts beside k_teach, whose lists it needs at its end only.
constexpr int ONE_THREADS = 512, ONE_ROWS = 4, ONE_UNITS = 2;
constexpr int ONE_WIDTH = 16384;   // most columns of a hidden state
struct OneArgs {
    const __nv_bfloat16 *h, *w;
    long long ldw;
    int V, D, nbins;
    float log2e;
    float2* stats;                 // [segments of 128 columns]
    const int* bins;
    const unsigned* entries;
    float* entry_logit;
    int* done;                     // counter to clear for the next kernel
};
__global__ void __launch_bounds__(ONE_THREADS, 2) k_teach_one(const __grid_constant__ OneArgs a) {
    extern __shared__ __align__(16) float hidden[];                // D rounded up to 8, zeros behind D
    __shared__ float logit[XE_SEG_LOSS];
    grid_trigger();
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, units = (a.D + 7) / 8, whole = a.D / 8;
    // (the hidden state and the vocabulary matrix are older than the kernel before this one)
    for (int d = tid; d < units * 8; d += ONE_THREADS) hidden[d] = d < a.D ? __bfloat162float(a.h[d]) : 0.f;
    __syncthreads();
    const int col0 = blockIdx.x * XE_SEG_LOSS;
    for (int c = warp * ONE_ROWS; c < XE_SEG_LOSS && col0 + c < a.V; c += ONE_THREADS / 32 * ONE_ROWS) {
        float acc[ONE_ROWS] = {};
        const __nv_bfloat16* row[ONE_ROWS];
#pragma unroll
        for (int r = 0; r < ONE_ROWS; ++r) row[r] = a.w + (long long)min(col0 + c + r, a.V - 1) * a.ldw;
        const auto add = [&](const Raw16 (&raw)[ONE_ROWS], int u) {
            const float4 lo = *reinterpret_cast<const float4*>(hidden + u * 8), hi = *reinterpret_cast<const float4*>(hidden + u * 8 + 4);
            const float y[8] = {lo.x, lo.y, lo.z, lo.w, hi.x, hi.y, hi.z, hi.w};
#pragma unroll
            for (int r = 0; r < ONE_ROWS; ++r) {
                float x[8];
                widen(raw[r], x);
#pragma unroll
                for (int j = 0; j < 8; ++j) acc[r] = fmaf(x[j], y[j], acc[r]);
            }
        };
        for (int u0 = lane; u0 < whole; u0 += 32 * ONE_UNITS) {
            Raw16 raw[ONE_UNITS][ONE_ROWS];
#pragma unroll
            for (int i = 0; i < ONE_UNITS; ++i)
#pragma unroll
                for (int r = 0; r < ONE_ROWS; ++r) {
                    raw[i][r].a = make_uint4(0u, 0u, 0u, 0u);
                    if (u0 + 32 * i < whole) load8(raw[i][r], row[r] + (u0 + 32 * i) * 8);
                }
#pragma unroll
            for (int i = 0; i < ONE_UNITS; ++i)
                if (u0 + 32 * i < whole) add(raw[i], u0 + 32 * i);
        }
        if (whole < units && lane == 0) {              // the rows' ends: only their own values are read
            Raw16 raw[ONE_ROWS];
#pragma unroll
            for (int r = 0; r < ONE_ROWS; ++r) {
                unsigned h[4] = {};
#pragma unroll
                for (int j = 0; j < 8; ++j)
                    if (whole * 8 + j < a.D) h[j / 2] |= (unsigned)reinterpret_cast<const unsigned short*>(row[r])[whole * 8 + j] << (j & 1) * 16;
                raw[r].a = make_uint4(h[0], h[1], h[2], h[3]);
            }
            add(raw, whole);
        }
#pragma unroll
        for (int r = 0; r < ONE_ROWS; ++r) {
            float v = acc[r];
#pragma unroll
            for (int o = 16; o; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
            if (lane == 0) logit[c + r] = v;
        }
    }
    __syncthreads();
    grid_wait();
    if (blockIdx.x == 0 && tid == 0) *a.done = 0;
    if (warp == 0) {
        const int cols = min(XE_SEG_LOSS, a.V - col0);
        float v[XE_SEG_LOSS / 32], top = -INFINITY;
#pragma unroll
        for (int i = 0; i < XE_SEG_LOSS / 32; ++i) {
            v[i] = lane + 32 * i < cols ? logit[lane + 32 * i] : -INFINITY;
            top = fmaxf(top, v[i]);
        }
#pragma unroll
        for (int o = 16; o; o >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, o));
        const float ref = top == -INFINITY ? 0.f : top;
        float sum = 0.f;
#pragma unroll
        for (int i = 0; i < XE_SEG_LOSS / 32; ++i) sum += ex2((v[i] - ref) * a.log2e);
#pragma unroll
        for (int o = 16; o; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
        if (lane == 0) a.stats[blockIdx.x] = make_float2(top, sum);
    }
    // the segment's four blocks of columns, whose entries lie one after the other
    const int* at = a.bins + 4 * blockIdx.x;
    const int left = a.nbins - 4 * (int)blockIdx.x;
    const int begin[5] = {at[0], at[min(1, left)], at[min(2, left)], at[min(3, left)], at[min(4, left)]};
    for (int e = begin[0] + tid; e < begin[4]; e += ONE_THREADS) {
        const unsigned code = a.entries[e];
        const int block = (e >= begin[1]) + (e >= begin[2]) + (e >= begin[3]);
        a.entry_logit[code >> 10] = logit[32 * block + (int)(code & 31u)];
    }
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
__device__ __forceinline__ float teach_term(float z, float logit, float top, float inv_tau, float log_q, float log_p) {
    const float e = expf(z);
    return e == 0.f ? 0.f : e * ((z - log_q) - ((logit - top) * inv_tau - log_p));
}
// the row's outputs from the sum of its terms; returns its share of the loss and of the weight
__device__ __forceinline__ double2 write_distance(const RowsArgs& a, const TeachRows& t, int row, long long label, float w, float rest_q, float top, float log_sum, float sum) {
    float loss = 0.f;
    if (label == -2) { loss = NAN; atomicOr(a.status, XE_W_LABEL); }
    else if (label == 0) loss = t.tau * t.tau * (sum / (1.f + rest_q));
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
        constexpr int HELD = 2;                        // entries per lane that are asked for before the statistics
        const int* col = t.col + (size_t)row * t.K;
        const float *z = t.z + (size_t)row * t.K, *logit = t.logit + (size_t)row * t.K, rest_q = t.rest[row];
        const long long label = a.labels[row];
        const float weight = a.weight ? a.weight[row] : 1.f;
        int c[HELD];
        float zs[HELD], ls[HELD];
#pragma unroll
        for (int i = 0; i < HELD; ++i) {
            const int k = lane + 32 * i;
            c[i] = k < t.K ? col[k] : -1;
            zs[i] = k < t.K ? z[k] : 0.f;
            ls[i] = k < t.K ? logit[k] : 0.f;
        }
        float top = -INFINITY, rest = -1.f;
        for (int j = lane; j < a.nseg; j += 8 * 32) {
            float2 s[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) s[i] = j + 32 * i < a.nseg ? a.stats[(size_t)row * a.nseg + j + 32 * i] : make_float2(-INFINITY, 0.f);
#pragma unroll
            for (int i = 0; i < 8; ++i) merge_stat(top, rest, s[i].x, s[i].y - 1.f, log2e);
        }
        warp_stat(top, rest, log2e);
        const float log_p = log1pf(rest), log_q = log1pf(rest_q);
        float sum = 0.f;
#pragma unroll
        for (int i = 0; i < HELD; ++i)
            if (c[i] >= 0) sum += teach_term(zs[i], ls[i], top, t.inv_tau, log_q, log_p);
        for (int k = lane + 32 * HELD; k < t.K; k += 32)
            if (col[k] >= 0) sum += teach_term(z[k], logit[k], top, t.inv_tau, log_q, log_p);
#pragma unroll
        for (int o = 16; o; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
        if (lane == 0) share = write_distance(a, t, row, label, label == 0 ? weight : 0.f, rest_q, top, log_p, sum);
    }
    if (lane == 0) mine[warp] = share;
    __syncthreads();
    if (threadIdx.x == 0) {
        for (int i = 1; i < XE_THREADS / 32; ++i) { share.x += mine[i].x; share.y += mine[i].y; }
        a.sums[a.first_sum + blockIdx.x] = share;
    }
    report_rows(a);
}

__device__ __forceinline__ unsigned first_slot(int column) { return (unsigned)column * 2654435761u >> 16; }     // (multiplied by 2^32 / golden ratio: its upper bits spread)

// Loss and gradient of the logits: blockIdx.x = row, blockIdx.y = part of its columns.  Columns that a row lists more than once are found by comparing every pair of its
// entries where there are up to TEACH_PAIRS, else through a hash table (64 entries: 104 us on 4096 x 32000, 112 with the table; 1024 entries: a step of 4096 x 32000 x 768
// in 2060 us by pairs, 770 with the table).
__global__ void __launch_bounds__(XE_THREADS, XE_ROW_CTAS) k_teach_rows(const __grid_constant__ RowsArgs a, const __grid_constant__ TeachRows t) {
    grid_trigger();
    grid_wait();
    __shared__ float2 ws[XE_THREADS / 32];
    __shared__ __align__(16) int cols[TEACH_MOST];
    __shared__ float es[TEACH_MOST];                   // exp(z)
    __shared__ int seen[2 * TEACH_MOST];               // hash table of the listed columns, -1: free; bit 30: listed more than once
    constexpr int TWICE = 1 << 30;
    __shared__ float terms[XE_THREADS / 32];
    const int row = blockIdx.x, tid = threadIdx.x, K = t.K;
    const float log2e = LOG2E * t.inv_tau;
    const float2* st = a.stats + (size_t)row * a.nseg;
    const float *z = t.z + (size_t)row * K, *logit = t.logit + (size_t)row * K;
    // entry `tid` in registers, asked for before the statistics
    int c0 = -1;
    float z0 = -INFINITY, l0 = 0.f;
    if (tid < K) { c0 = t.col[(size_t)row * K + tid]; z0 = z[tid]; l0 = logit[tid]; }
    const float rest_q = t.rest[row], weight = a.weight ? a.weight[row] : 1.f;
    const long long label = a.labels[row];
    const bool counts = label == 0, hashed = K > TEACH_PAIRS;
    const float w = counts ? weight : 0.f;
    float top = -INFINITY, rest = -1.f;
    for (int j = tid; j < a.nseg; j += XE_THREADS) merge_stat(top, rest, st[j].x, st[j].y - 1.f, log2e);
    const unsigned slots = 2u << (32 - __clz(K - 1));  // the power of two from 2 K on
    for (int k = tid; hashed && k < (int)slots; k += XE_THREADS) seen[k] = -1;
    for (int k = tid; k < (K + 3) / 4 * 4; k += XE_THREADS) {
        cols[k] = k == tid ? c0 : k < K ? t.col[(size_t)row * K + k] : -1;
        es[k] = k == tid ? expf(z0) : k < K ? expf(z[k]) : 0.f;
    }
    warp_stat(top, rest, log2e);
    if ((tid & 31) == 0) ws[tid >> 5] = make_float2(top, rest);
    __syncthreads();
    top = ws[0].x;
    rest = ws[0].y;
#pragma unroll
    for (int i = 1; i < XE_THREADS / 32; ++i) merge_stat(top, rest, ws[i].x, ws[i].y, log2e);
    const float log_sum = log1pf(rest);
    if (blockIdx.y == 0 && (tid & ~31) < K) {          // warps with entries
        const float log_q = log1pf(rest_q);
        float sum = c0 >= 0 ? teach_term(z0, l0, top, t.inv_tau, log_q, log_sum) : 0.f;
        for (int k = tid + XE_THREADS; k < K; k += XE_THREADS)
            if (cols[k] >= 0) sum += teach_term(z[k], logit[k], top, t.inv_tau, log_q, log_sum);
#pragma unroll
        for (int o = 16; o; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
        if ((tid & 31) == 0) terms[tid >> 5] = sum;
    }
    const float lse = top * t.inv_tau + log_sum, poison = lse - lse;         // 0, or NaN where the row's logits were not finite
    uint4* q = reinterpret_cast<uint4*>(a.q + (size_t)row * a.ldq);
    const int units = (a.V + 7) / 8, per = (units + gridDim.y - 1) / gridDim.y;
    const int u0 = blockIdx.y * per, u1 = min(units, u0 + per);
    for (int k = tid; hashed && counts && k < K; k += XE_THREADS) {
        const int c = cols[k];
        if (c < 0 || (c >> 3) < u0 || (c >> 3) >= u1) continue;
        for (unsigned at = first_slot(c), n = 0; n < slots; ++at, ++n) {     // (half of the table stays free: it ends long before)
            const int old = atomicCAS(seen + (at & (slots - 1)), -1, c);
            if (old == -1) break;
            if ((old & ~TWICE) == c) { atomicOr(seen + (at & (slots - 1)), TWICE); break; }
        }
    }
    rewrite_exponents(q, st, u0, u1, w, counts, poison, [&](float ref) { return ((ref - top) * t.inv_tau - log_sum) * LOG2E + poison; });
    __syncthreads();
    if (blockIdx.y == 0 && tid == XE_THREADS - 1) {    // (a thread without an entry, mostly)
        float sum = 0.f;
        for (int i = 0; i < XE_THREADS / 32 && 32 * i < K; ++i) sum += terms[i];
        a.sums[a.first_sum + row] = write_distance(a, t, row, label, w, rest_q, top, log_sum, sum);
    }
    // the entries' columns again; a column that is listed more than once by the first of its entries
    if (counts) {
        const float both = 1.f / ((1.f + rest) * (1.f + rest_q));
        for (int k = tid; k < K; k += XE_THREADS) {
            const int c = cols[k];
            if (c < 0 || (c >> 3) < u0 || (c >> 3) >= u1) continue;
            bool many = false, first = true;           // whether its column is listed more than once, and not before
            if (hashed) {
                unsigned at = first_slot(c);
                for (unsigned n = 0; n < slots && (seen[at & (slots - 1)] & ~TWICE) != c; ++n) ++at;
                many = seen[at & (slots - 1)] & TWICE;
                for (int j = 0; many && j < k; ++j) first = first && cols[j] != c;
            } else {
                int same = 0, before = 0;
#pragma unroll 4
                for (int j = 0; j < K; j += 4) {
                    const int4 four = *reinterpret_cast<const int4*>(cols + j);
                    same += (four.x == c) + (four.y == c) + (four.z == c) + (four.w == c);
                    before += (four.x == c && j < k) + (four.y == c && j + 1 < k) + (four.z == c && j + 2 < k) + (four.w == c && j + 3 < k);
                }
                many = same > 1;
                first = before == 0;
            }
            if (!first) continue;
            float e_q = es[k];
            if (many)
                for (int j = k + 1; j < K; ++j) e_q += cols[j] == c ? es[j] : 0.f;
            const float e_p = ex2(((k == tid ? l0 : logit[k]) - top) * log2e);
            const float d = (((e_p - e_q) + e_p * rest_q) - e_q * rest) * both + poison;
            reinterpret_cast<__nv_bfloat16*>(q)[c] = __float2bfloat16_rn(d * w);
        }
    }
    report_rows(a);
}

}  // namespace psgd
