// Host side of the training operators declared in include/psgd.h: softmax cross entropy of the last layer with its
// gradients, 8-bit activation checkpoints, the weight gradient from them, and the gated unit.  Argument checks, workspace
// layout and the stream-ordered sequence of kernels; nothing here allocates, synchronises or keeps anything between calls.
#include "../../include/psgd.h"

#include <stdio.h>

#include <algorithm>

#include "psgd_act.cuh"
#include "psgd_host.cuh"
#include "psgd_tile.cuh"
#include "psgd_xent.cuh"

using namespace psgd;

namespace {

// What is behind the last PSGD_E_CUDA of this thread's calls (there is no handle to keep it in).
thread_local char call_error[160] = "no error";
psgd_status cuda_error(const char* what, const char* why) {
    snprintf(call_error, sizeof(call_error), "%s: %s", what, why);
    return PSGD_E_CUDA;
}
bool succeeded(const char* what, cudaError_t e) {
    if (e == cudaSuccess) return true;
    cuda_error(what, cudaGetErrorString(e));
    cudaGetLastError();                               // not left for whoever asks next
    return false;
}

constexpr int64_t MAX_EXTENT = (int64_t)1 << 30;
constexpr int KACC_F32 = 32;       // stages (2048 of k) per accumulator where the result is float32: the tensor cores' additions truncate, and the
                                   // error grows with the number of additions into one running sum (16384 of k: 1.3e-6 with 64, 0.6e-6 with 32).
                                   // A bfloat16 result keeps one sum over all of k: its rounding, 2e-3, is far above that.

constexpr int ROUND_COST = 6;      // of a unit beside its stages (epilogue not overlapped, refilling the ring), in stages

struct TilePlan { int64_t M, N, K; int mt, nt, kb, bn, full, S, kbps, tail, parts, units, gm; };

// Of a stage of 64 of k, in those of 256 columns.  A stage is bound by shared memory: 16 KB of A and bn / 16 KB of B per CTA are written by the copies
// and read by the MMAs (measured 0.31 us with 256 columns, 0.25 with 192, 0.23 with 128 on 48 pairs, 0.36, 0.26 and 0.24 on all of them).
double stage_cost(int bn) { return bn == 256 ? 1.0 : bn == 192 ? 0.80 : 0.70; }

void finish_plan(TilePlan& p, int pairs) {
    p.parts = p.parts || p.S > 1;
    p.units = p.full + p.tail * p.S;
    // raster: all row tiles next to each other while the row operand fits beside the rest in L2, else as many as make the
    // pairs at work cover all columns
    p.gm = (p.M * p.K * 2 <= (40 << 20)) ? p.mt : std::min(p.mt, std::max(8, std::min(32, pairs / p.nt)));
}

// Tiles of an M x N product over `pairs` CTA pairs.  The last, partly filled wave of R tiles may be cut into S pieces of k each, and
// the tiles may be 192 or 128 columns wide instead of 256; both are chosen for the least time in units of one 256-column stage:
// a round of units costs its stages and ROUND_COST, joining the pieces a launch and their way through memory.
TilePlan plan_tiles(int64_t M, int64_t N, int64_t K, int pairs, bool store) {
    TilePlan p{};
    p.M = M; p.N = N; p.K = K;
    p.mt = ceil_div(M, TG_BM);
    p.kb = ceil_div(K, TG_BK);
    double best = 1e300;
    for (int bn = TG_BN; bn >= (store ? 128 : TG_BN); bn -= 64) {
        const int nt = ceil_div(N, bn);
        const double stage = stage_cost(bn);
        const int64_t tiles = (int64_t)p.mt * nt;
        const int R = (int)(tiles % pairs);
        const double whole = (double)(tiles / pairs) * (p.kb + 1) * stage;
        for (int S = 1, most = store && R > 0 ? std::min(p.kb, 2 * pairs / R + 1) : 1; S <= most; ++S) {
            const int kbps = ceil_div(p.kb, S);
            if (ceil_div(p.kb, kbps) != S) continue;                           // no empty pieces
            double cost = whole + (R > 0 ? (double)ceil_div((int64_t)R * S, pairs) * (kbps + ROUND_COST) * stage : 0.0);
            if (S > 1) cost += 20 + 0.06 * R * S;         // 2048 x 768 x 4096 in three pieces of 256 columns: 25.6 us, whole with 128 columns: 23.2
            if (cost < best) { best = cost; p.bn = bn; p.nt = nt; p.S = S; p.kbps = kbps; p.tail = R; p.full = (int)(tiles - R); }
        }
    }
    finish_plan(p, pairs);
    return p;
}

// Two products that share one launch (launch_products): no waves to fill, only units that must not be longer than a pair's share of
// the whole work, so a product is cut along k, all its tiles alike, where its tiles would be.
void plan_two(TilePlan (&p)[2], const int64_t (&M)[2], int64_t N, const int64_t (&K)[2], int pairs) {
    double total = 0.0;
    for (int i = 0; i < 2; ++i) {
        TilePlan& q = p[i];
        q = TilePlan{};
        q.M = M[i]; q.N = N; q.K = K[i];
        q.mt = ceil_div(q.M, TG_BM);
        q.kb = ceil_div(q.K, TG_BK);
        double best = 1e300;
        for (int bn = TG_BN; bn >= 128; bn -= 64)
            if (ceil_div(N, bn) * stage_cost(bn) < best) { best = ceil_div(N, bn) * stage_cost(bn); q.bn = bn; q.nt = ceil_div(N, bn); }
        total += (double)q.mt * q.nt * (q.kb + ROUND_COST) * stage_cost(q.bn);
    }
    for (TilePlan& q : p) {
        const int tiles = q.mt * q.nt;
        const double most = 0.9 * total / pairs + 10;                          // cutting has a price: the pieces are added by another kernel
        for (int S = 1;; ++S) {
            const int kbps = ceil_div(q.kb, S);
            if (ceil_div(q.kb, kbps) != S) continue;
            q.S = S;
            q.kbps = kbps;
            if ((kbps + ROUND_COST) * stage_cost(q.bn) <= most || kbps == 1) break;
        }
        q.full = q.S > 1 ? 0 : tiles;
        q.tail = q.S > 1 ? tiles : 0;
        finish_plan(q, pairs);
    }
}
size_t part_bytes(const TilePlan& p) { return p.parts ? (size_t)(p.units - p.full) * TG_PART * 4 : 0; }

// bfloat16 matrix, `rows` rows of `cols` with row stride ld (elements): boxes of 64 columns and `box` rows, 128-byte swizzle
bool encode_operand(CUtensorMap* map, const void* p, int64_t rows, int64_t cols, int64_t ld, int box) {
    EncodeTiledFn fn = encode_tiled_fn();
    if (!fn) {
        cuda_error("cuTensorMapEncodeTiled", "not found in the driver");
        return false;
    }
    if (rows == 1) ld = align_up(cols, 8);                             // the stride of a single row is never used
    cuuint64_t dims[2] = {(cuuint64_t)cols, (cuuint64_t)rows};
    cuuint64_t strides[1] = {(cuuint64_t)ld * 2};
    cuuint32_t b[2] = {64, (cuuint32_t)box};
    cuuint32_t es[2] = {1, 1};
    if (fn(map, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 2, (void*)p, dims, strides, b, es, CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B,
           CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS) return true;
    cuda_error("cuTensorMapEncodeTiled", "operand refused");
    return false;
}

void set_problem(TileProblem& t, const TilePlan& p) {
    t.M = (int)p.M; t.N = (int)p.N;
    t.mt = p.mt; t.nt = p.nt; t.kb = p.kb; t.bn = p.bn; t.full = p.full; t.S = p.S; t.kbps = p.kbps; t.tail = p.tail; t.parts = p.parts; t.units = p.units; t.gm = p.gm;
    t.by_group = fast_div((unsigned)p.gm * p.nt); t.by_gm = fast_div(p.gm); t.by_rest = fast_div(std::max(1, p.mt % p.gm)); t.by_tail = fast_div(std::max(1, p.tail));
}

// Launch that may start before the kernel in front of it on the stream has finished (the kernels wait for that themselves).
template <typename... Params, typename... Args>
bool launch(void (*kernel)(Params...), dim3 grid, dim3 block, size_t smem, cudaStream_t st, const Args&... args) {
    cudaLaunchConfig_t c{};
    c.gridDim = grid; c.blockDim = block; c.dynamicSmemBytes = smem; c.stream = st;
    cudaLaunchAttribute at{};
    at.id = cudaLaunchAttributeProgrammaticStreamSerialization;
    at.val.programmaticStreamSerializationAllowed = 1;
    c.attrs = &at;
    c.numAttrs = 1;
    return succeeded("kernel launch", cudaLaunchKernelEx(&c, kernel, Params(args)...));
}

struct Operand { const void* p; int64_t ld; bool mn; };      // mn: stored [K][rows], else [rows][K]
bool encode(CUtensorMap* map, const Operand& o, int64_t rows, int64_t K, int box) {
    return o.mn ? encode_operand(map, o.p, K, rows, o.ld, TG_BK) : encode_operand(map, o.p, rows, K, o.ld, box);
}

// One product of K-major operands with a softmax epilogue.
template <int EPI>
psgd_status launch_softmax(const Operand& A, const Operand& B, const TilePlan& p, TileArgs& a, int pairs, cudaStream_t st) {
    CUtensorMap ma, mb;
    // Few tokens: only their rows are loaded, so that the TMA unit is left to the stream of B, of which each byte is used once (1 row against
    // 131072 x 2048: 137 -> 97 us, 5.5 TB/s; 64 rows against 32000 x 4096: 58.5 us with whole boxes, 60 without)
    const bool few = p.M <= 32;
    a.a_rows = few ? (int)align_up(p.M, 8) : 128;
    a.a_odd = !few;
    if (!encode(&ma, A, p.M, p.K, a.a_rows) || !encode(&mb, B, p.N, p.K, p.bn / 2)) return PSGD_E_CUDA;
    set_problem(a.p[0], p);
    const int n = std::min(p.units, pairs);
    a.first_q = p.units / n; a.first_r = p.units % n;
    allow_smem(k_tile<EPI>, tile_smem_bytes());
    return launch(k_tile<EPI>, dim3(2 * n), dim3(TG_THREADS), tile_smem_bytes(), st, ma, mb, ma, mb, a) ? PSGD_OK : PSGD_E_CUDA;
}

// One or two products (B MN-major) in one launch, then the pieces of their split tiles.  Two: the units of the first go round the pairs; the
// pairs that have one unit fewer of it do as many units of the second meanwhile as fit in that time.
psgd_status launch_products(int count, const Operand (&A)[2], const Operand (&B)[2], const TilePlan (&p)[2], TileArgs& a, int pairs, cudaStream_t st) {
    CUtensorMap m[4];
    for (int i = 0; i < count; ++i) {
        if (!encode(&m[2 * i], A[i], p[i].M, p[i].K, 128) || !encode(&m[2 * i + 1], B[i], p[i].N, p[i].K, p[i].bn / 2)) return PSGD_E_CUDA;
        set_problem(a.p[i], p[i]);
        a.p[i].a_mn = A[i].mn;
    }
    if (count == 1) { m[2] = m[0]; m[3] = m[1]; }
    const int second = count == 2 ? p[1].units : 0;
    const int n = std::min(p[0].units + second, pairs);
    a.first_q = p[0].units / n; a.first_r = p[0].units % n;
    a.extra = 0;
    if (second && a.first_r) {
        const int c0 = (p[0].S > 1 ? p[0].kbps : p[0].kb) + ROUND_COST, c1 = (p[1].full ? p[1].kb : p[1].kbps) + ROUND_COST;
        a.extra = std::min((c0 + c1 / 2) / c1, second / (n - a.first_r));
    }
    allow_smem(k_tile<EPI_STORE>, tile_smem_bytes());
    if (!launch(k_tile<EPI_STORE>, dim3(2 * n), dim3(TG_THREADS), tile_smem_bytes(), st, m[0], m[1], m[2], m[3], a)) return PSGD_E_CUDA;
    const int joins = (p[0].parts ? p[0].tail : 0) + (count == 2 && p[1].parts ? p[1].tail : 0);
    const int wide = std::max(p[0].bn, count == 2 ? p[1].bn : 0);
    if (joins && !launch(k_join, dim3(joins, wide / 32, TG_BM / 32), dim3(128), 0, st, a)) return PSGD_E_CUDA;
    return PSGD_OK;
}

bool operand_ok(const void* p, int64_t rows, int64_t cols, int64_t ld) { return aligned16(p) && ld >= cols && (rows == 1 || ld % 8 == 0); }
bool extent_ok(int64_t v) { return v >= 1 && v <= MAX_EXTENT; }
// Bytes of a matrix in memory: `rows` stretches of `width`, `step` apart (width <= step).
struct Stretch { const void* p; int64_t rows, width, step; };
bool overlap(const Stretch& a, const Stretch& b) {
    if (!a.p || !b.p || a.rows < 1 || b.rows < 1) return false;
    if (a.rows > b.rows) return overlap(b, a);
    const int64_t at = (int64_t)((uintptr_t)a.p - (uintptr_t)b.p);               // of a's first row, from b's
    const int64_t end_a = at + (a.rows - 1) * a.step + a.width, end_b = (b.rows - 1) * b.step + b.width;
    if (at >= end_b || end_a <= 0) return false;
    // rows that lie between one another (columns of one wider matrix): row by row; with equal steps the first rows that face each other speak for all but the ends
    const auto meets = [&](int64_t i) {
        const int64_t x = at + i * a.step;                                       // the first row of b that ends behind x
        const int64_t j = x < b.width ? 0 : (x - b.width) / b.step + 1;
        return j < b.rows && j * b.step < x + a.width;
    };
    const int64_t first = at >= 0 ? 0 : std::min(a.rows - 1, -at / a.step);
    for (int64_t i = first; i < (a.step == b.step ? std::min(a.rows, first + 2) : a.rows); ++i)
        if (meets(i)) return true;
    return a.step == b.step && meets(a.rows - 1);
}
Stretch stretch(const void* p, int64_t rows, int64_t cols, int64_t ld, int bytes) { return {p, rows, cols * bytes, (rows == 1 ? cols : ld) * bytes}; }
bool tiles_ok(int64_t M, int64_t N) { return ((M + 255) / 256) * ((N + 127) / 128) <= MAX_EXTENT; }     // units are counted in 32 bits

// ---- cross entropy ----
constexpr int64_t XENT_PIECE_LOGITS = (int64_t)1 << 29;   // logits whose 16-bit form the workspace holds at a time (1 GiB; half as many: 3 to 4 % slower)

constexpr int64_t XENT_PIECE_STATS = (int64_t)1 << 25;    // loss alone: statistics of 128 logits that it holds at a time (256 MiB)

struct XentPlan {
    int pairs, nseg;
    int64_t ldq, piece, pieces;
    TilePlan logits, two[2];          // of a whole piece; two: dH and dW
    size_t inv, done, sums, stats, label_logit, q, part, acc, total;
};
// Tokens are taken in pieces, all columns at a time, so that the stored exponents (loss alone: the statistics) stay within a fixed size however
// many tokens there are; a piece has at least 1024 tokens, below which the products with the vocabulary matrix would be bound by reading it.
void plan_gradients(TilePlan (&p)[2], int64_t rows, int64_t V, int64_t D, int pairs) {
    const int64_t M[2] = {rows, V}, K[2] = {V, rows};
    plan_two(p, M, D, K, pairs);
}
XentPlan plan_xent(int64_t T, int64_t V, int64_t D, bool grad) {
    XentPlan x{};
    x.pairs = std::max(1, device_sms() / 2);
    x.nseg = ceil_div(V, grad ? XE_SEG : XE_SEG_LOSS);
    x.ldq = (int64_t)align_up(V, XE_SEG);
    const int64_t fit = std::max<int64_t>(1024, (grad ? XENT_PIECE_LOGITS / x.ldq : XENT_PIECE_STATS / x.nseg) / TG_BM * TG_BM);
    x.pieces = ceil_div(T, fit);
    x.piece = std::min<int64_t>(T, align_up(ceil_div(T, x.pieces), TG_BM));
    x.pieces = ceil_div(T, x.piece);
    x.logits = plan_tiles(x.piece, V, D, x.pairs, false);
    size_t at = 256;                                  // the status word of calls that bring none
    auto take = [&](size_t bytes) { const size_t o = at; at = align_up(at + bytes, 256); return o; };
    x.inv = take(4);
    x.done = take(4);
    if (grad) {
        plan_gradients(x.two, x.piece, V, D, x.pairs);
    }
    x.sums = take((size_t)(grad ? T : ceil_div(T, XE_THREADS / 32)) * sizeof(double2));
    x.stats = take((size_t)x.piece * x.nseg * 8);
    x.label_logit = take((size_t)x.piece * 4);
    if (grad) {
        x.q = take((size_t)x.piece * x.ldq * 2);
        size_t part = part_bytes(x.two[0]) + part_bytes(x.two[1]);
        if (x.pieces > 1) {                           // the last piece may be shorter
            TilePlan last[2];
            plan_gradients(last, T - (x.pieces - 1) * x.piece, V, D, x.pairs);
            part = std::max(part, part_bytes(last[0]) + part_bytes(last[1]));
            x.acc = take((size_t)V * D * 4);
        }
        x.part = take(part);
    }
    x.total = at;
    return x;
}

psgd_status xent(const void* H, int64_t ldh, const void* W, int64_t ldw, const int64_t* labels, const float* weight, int64_t ignore, int64_t T, int64_t V, int64_t D,
                 float* loss, float* token_loss, float* lse, bool grad, void* dH, int64_t lddh, void* dW, int64_t lddw, int* status, void* ws, size_t ws_bytes, cudaStream_t st) {
    if (T < 0 || T > MAX_EXTENT || !extent_ok(V) || !extent_ok(D) || !tiles_ok(T, V) || !tiles_ok(V, D)) return PSGD_E_INVALID;
    if (!W || !loss || !ws || (T > 0 && (!H || !labels || !token_loss || !lse)) || (grad && (!dW || (T > 0 && !dH)))) return PSGD_E_NULL;
    if (!operand_ok(W, V, D, ldw) || (T > 0 && !operand_ok(H, T, D, ldh)) || (grad && ((T > 0 && lddh < D) || lddw < D))) return PSGD_E_INVALID;
    if ((uintptr_t)ws & 255) return PSGD_E_INVALID;
    if (grad) {                                       // both products run at once: one reads H and W while the other writes
        const Stretch h = stretch(H, T, D, ldh, 2), v = stretch(W, V, D, ldw, 2), dh = stretch(dH, T, D, lddh, 2), dw = stretch(dW, V, D, lddw, 2);
        if (overlap(dh, h) || overlap(dh, v) || overlap(dw, h) || overlap(dw, v) || overlap(dh, dw)) return PSGD_E_INVALID;
    }
    if (T == 0) {                                     // no token: loss 0, no gradient
        if (!succeeded("cudaMemsetAsync", cudaMemsetAsync(loss, 0, 4, st))) return PSGD_E_CUDA;
        if (grad && !succeeded("cudaMemset2DAsync", cudaMemset2DAsync(dW, (size_t)lddw * 2, 0, (size_t)D * 2, (size_t)V, st))) return PSGD_E_CUDA;
        return PSGD_OK;
    }
    const XentPlan x = plan_xent(T, V, D, grad);
    if (ws_bytes < x.total) return PSGD_E_WORKSPACE;
    char* w = (char*)ws;
    int* stat = status ? status : (int*)w;
    float* inv = (float*)(w + x.inv);
    int* done = (int*)(w + x.done);

    RowsArgs r{};
    r.V = (int)V; r.nseg = x.nseg;
    r.stats = (const float2*)(w + x.stats);
    r.label_logit = (const float*)(w + x.label_logit);
    r.ignore = ignore; r.ldq = x.ldq; r.status = stat; r.q = grad ? (unsigned short*)(w + x.q) : nullptr;
    r.done = done; r.sums = (double2*)(w + x.sums); r.n_sums = (int)(grad ? T : ceil_div(T, XE_THREADS / 32)); r.mean = loss;
    auto parts_of = [&](int64_t rows) {               // CTAs per row of k_xent_rows: two waves of eight per multiprocessor, at least 2048 columns each
        return (int)std::max<int64_t>(1, std::min<int64_t>({(2 * 8 * 2 * (int64_t)x.pairs + rows - 1) / rows, (V + 2047) / 2048, 1024}));
    };
    int64_t report = 0;
    for (int64_t t0 = 0; t0 < T; t0 += x.piece) {
        const int64_t rows = std::min<int64_t>(x.piece, T - t0);
        report += grad ? rows * parts_of(rows) : ceil_div(rows, XE_THREADS / 32);
    }
    if (report > INT32_MAX) return PSGD_E_INVALID;
    r.done_at = (int)report;

    for (int64_t t0 = 0; t0 < T; t0 += x.piece) {
        const int64_t rows = std::min<int64_t>(x.piece, T - t0);
        const bool first = t0 == 0, last = t0 + rows == T;
        const char* h = (const char*)H + (size_t)t0 * ldh * 2;
        TileArgs a{};
        a.status = stat;
        a.labels = (const long long*)labels + t0;
        a.stats = (float2*)(w + x.stats);
        a.label_logit = (float*)(w + x.label_logit);
        a.q = r.q; a.ldq = x.ldq; a.nseg = x.nseg;
        if (first) {
            a.done = done;
            a.norm = inv; a.norm_labels = (const long long*)labels; a.norm_weight = weight; a.norm_rows = T; a.ignore = ignore;
        }
        const bool whole = rows == x.piece;
        const TilePlan pl = whole ? x.logits : plan_tiles(rows, V, D, x.pairs, false);
        const Operand oh{h, ldh, false}, ow{W, ldw, false};
        psgd_status s = grad ? launch_softmax<EPI_SOFTMAX>(oh, ow, pl, a, x.pairs, st) : launch_softmax<EPI_LOSS>(oh, ow, pl, a, x.pairs, st);
        if (s != PSGD_OK) return s;
        r.rows = (int)rows;
        r.first_sum = (int)(grad ? t0 : t0 / (XE_THREADS / 32));      // (pieces are whole row tiles)
        r.labels = (const long long*)labels + t0;
        r.weight = weight ? weight + t0 : nullptr;
        r.loss = token_loss + t0;
        r.lse = lse + t0;
        if (!grad) {
            if (!launch(k_xent_loss, dim3(ceil_div(rows, XE_THREADS / 32)), dim3(XE_THREADS), 0, st, r)) return PSGD_E_CUDA;
            continue;
        }
        if (!launch(k_xent_rows, dim3((unsigned)rows, parts_of(rows)), dim3(XE_THREADS), 0, st, r)) return PSGD_E_CUDA;
        // dH = dL W: contraction over the vocabulary;  dW = dL^T H: over the tokens
        TilePlan p[2] = {x.two[0], x.two[1]};
        if (!whole) plan_gradients(p, rows, V, D, x.pairs);
        const Operand A[2] = {{r.q, x.ldq, false}, {r.q, x.ldq, true}}, B[2] = {{W, ldw, true}, {h, ldh, true}};
        TileArgs g{};
        g.status = stat;
        TileProblem &ph = g.p[0], &pw = g.p[1];
        ph.scale = pw.scale = inv;
        ph.part = (float*)(w + x.part);
        pw.part = ph.part + part_bytes(p[0]) / 4;
        ph.out = (char*)dH + (size_t)t0 * lddh * 2;
        ph.ldo = lddh;
        ph.vec = aligned16(ph.out) && lddh % 8 == 0;
        float* acc = (float*)(w + x.acc);
        pw.addend = first ? nullptr : acc;
        if (last) {
            pw.out = dW; pw.ldo = lddw;
            pw.vec = aligned16(dW) && lddw % 8 == 0 && (first || D % 4 == 0);
        } else {
            pw.out = acc; pw.ldo = D; pw.out_f32 = 1; pw.scale = nullptr;
            pw.vec = D % 4 == 0;
        }
        s = launch_products(2, A, B, p, g, x.pairs, st);
        if (s != PSGD_OK) return s;
    }
    return PSGD_OK;
}

// ---- 8-bit activations ----
struct ActGrid { dim3 grid, block; };
// 256 threads, CTAs for `resident` of them per multiprocessor: a row's units side by side, as many rows as fit.  `any`: a warp per 32 units of a row.
ActGrid act_grid(int64_t T, int G, int resident, bool any) {
    const int units = 4 * G, across = ceil_div(units, 256);
    const int bx = any ? 32 : (int)align_up(ceil_div(units, across), 4);
    const int by = std::max(1, 256 / bx);
    const int nx = ceil_div(units, bx);
    const int64_t y = std::min<int64_t>({ceil_div(T, by), 65535, std::max(1, device_sms() * resident / nx)});
    return {dim3(nx, (unsigned)y), dim3(bx, by)};
}
// a lane per value: eight warps with four groups of a row each, as many rows at a time as keep eight such CTAs per multiprocessor busy
ActGrid lane_grid(int64_t T, int G) {
    const int nx = ceil_div(G, 8 * LANE_GROUPS);
    const int64_t y = std::min<int64_t>({T, 65535, std::max(1, ceil_div((int64_t)device_sms() * 32, nx))});
    return {dim3(nx, (unsigned)y), dim3(32, 8)};
}
bool act_ok(int64_t T, int64_t F) { return T >= 0 && T <= MAX_EXTENT && extent_ok(F); }
bool vec8(const void* p, int64_t ld, int64_t F, int dtype) { return F % 8 == 0 && aligned16(p) && ld % (dtype == PSGD_DT_BF16 ? 8 : 4) == 0; }

bool launch_pack(const ActShape& s, const void* x, int64_t ldx, int dtype, int8_t* q, uint8_t* scales, cudaStream_t st) {
    const bool vec = vec8(x, ldx, s.F, dtype);
    const auto run = [&](auto kernel, const ActGrid& g, auto* p) { return launch(kernel, g.grid, g.block, 0, st, s, p, ldx, q, scales); };
    if (dtype == PSGD_DT_BF16) {
        const ActGrid g = act_grid(s.T, s.G, PACK_CTAS, !vec);
        return run(vec ? k_act_pack<false> : k_act_pack<true>, g, (const __nv_bfloat16*)x);
    }
    return vec ? run(k_act_pack32, act_grid(s.T, s.G, PACK_CTAS, false), (const float*)x) : run(k_act_pack32_any, lane_grid(s.T, s.G), (const float*)x);
}
bool launch_unpack(const ActShape& s, const int8_t* q, const uint8_t* scales, void* x, int64_t ldx, int dtype, cudaStream_t st) {
    const bool vec = vec8(x, ldx, s.F, dtype);
    const auto run = [&](auto kernel, const ActGrid& g, auto* p) { return launch(kernel, g.grid, g.block, 0, st, s, q, scales, p, ldx); };
    if (dtype == PSGD_DT_BF16) {
        const ActGrid g = act_grid(s.T, s.G, PACK_CTAS, !vec);
        return run(vec ? k_act_unpack<__nv_bfloat16, false> : k_act_unpack<__nv_bfloat16, true>, g, (__nv_bfloat16*)x);
    }
    return vec ? run(k_act_unpack<float, false>, act_grid(s.T, s.G, PACK_CTAS, false), (float*)x) : run(k_act_unpack32_any, lane_grid(s.T, s.G), (float*)x);
}
bool dtype_ok(int dtype) { return dtype == PSGD_DT_F32 || dtype == PSGD_DT_BF16; }
bool ckpt_ok(const void* q) { return ((uintptr_t)q & 15) == 0; }

struct WgradPlan { int pairs; int64_t ldx; TilePlan p; size_t x, part, total; };
// `by_parts`: a float32 result whose rows are not 16-byte aligned and whose tiles are summed in several steps: the steps add up in
// partial tiles (5284 x 3300 x 2789: the whole call 225 us with unaligned read-add-write, 135 us so)
WgradPlan plan_wgrad(int64_t T, int64_t O, int64_t F, bool by_parts) {
    WgradPlan g{};
    g.pairs = std::max(1, device_sms() / 2);
    g.ldx = (int64_t)align_up(F, ACT_GROUP);
    g.p = plan_tiles(O, F, T, g.pairs, true);
    if (by_parts && g.p.kb > KACC_F32) {
        if (g.p.S == 1) { g.p.tail = g.p.mt * g.p.nt; g.p.full = 0; }
        else if (g.p.full) { g.p.tail += g.p.full; g.p.full = 0; g.p.S = 1; g.p.kbps = g.p.kb; }
        g.p.parts = 1;
        finish_plan(g.p, g.pairs);
    }
    size_t at = 256;
    auto take = [&](size_t bytes) { const size_t o = at; at = align_up(at + bytes, 256); return o; };
    g.x = take((size_t)T * g.ldx * 2);
    g.part = take(part_bytes(g.p));
    g.total = at;
    return g;
}

}  // namespace

extern "C" {

const char* psgd_training_cuda_error(void) { return call_error; }

int psgd_overlap(const void* a, int64_t rows_a, int64_t width_a, int64_t step_a, const void* b, int64_t rows_b, int64_t width_b, int64_t step_b) {
    return overlap({a, rows_a, width_a, rows_a == 1 ? width_a : step_a}, {b, rows_b, width_b, rows_b == 1 ? width_b : step_b});
}

psgd_status psgd_xent_workspace(int64_t T, int64_t V, int64_t D, int grad, size_t* bytes) {
    if (!bytes) return PSGD_E_NULL;
    if (T < 0 || T > MAX_EXTENT || !extent_ok(V) || !extent_ok(D) || !tiles_ok(T, V) || !tiles_ok(V, D)) return PSGD_E_INVALID;
    *bytes = T == 0 ? 256 : plan_xent(T, V, D, grad != 0).total;
    return PSGD_OK;
}

psgd_status psgd_xent_loss(const void* H, int64_t ldh, const void* W, int64_t ldw, const int64_t* labels, const float* weight, int64_t ignore, int64_t T, int64_t V,
                           int64_t D, float* loss, float* token_loss, float* lse, int* status, void* ws, size_t ws_bytes, psgd_stream stream) try {
    return xent(H, ldh, W, ldw, labels, weight, ignore, T, V, D, loss, token_loss, lse, false, nullptr, 0, nullptr, 0, status, ws, ws_bytes, (cudaStream_t)stream);
} catch (...) {
    return cuda_error("host", "exception");
}

psgd_status psgd_xent_grad(const void* H, int64_t ldh, const void* W, int64_t ldw, const int64_t* labels, const float* weight, int64_t ignore, int64_t T, int64_t V,
                           int64_t D, float* loss, float* token_loss, float* lse, void* dH, int64_t lddh, void* dW, int64_t lddw, int* status, void* ws, size_t ws_bytes,
                           psgd_stream stream) try {
    return xent(H, ldh, W, ldw, labels, weight, ignore, T, V, D, loss, token_loss, lse, true, dH, lddh, dW, lddw, status, ws, ws_bytes, (cudaStream_t)stream);
} catch (...) {
    return cuda_error("host", "exception");
}

psgd_status psgd_act_pack(const void* x, int64_t ldx, int dtype, int64_t T, int64_t F, int8_t* q, uint8_t* scales, psgd_stream stream) {
    if (!act_ok(T, F) || !dtype_ok(dtype)) return PSGD_E_INVALID;
    if (T == 0) return PSGD_OK;
    if (!x || !q || !scales) return PSGD_E_NULL;
    if (ldx < F || !ckpt_ok(q)) return PSGD_E_INVALID;
    const ActShape s{T, (int)F, ceil_div(F, ACT_GROUP)};
    return launch_pack(s, x, ldx, dtype, q, scales, (cudaStream_t)stream) ? PSGD_OK : PSGD_E_CUDA;
}

psgd_status psgd_act_unpack(const int8_t* q, const uint8_t* scales, int64_t T, int64_t F, void* x, int64_t ldx, int dtype, psgd_stream stream) {
    if (!act_ok(T, F) || !dtype_ok(dtype)) return PSGD_E_INVALID;
    if (T == 0) return PSGD_OK;
    if (!x || !q || !scales) return PSGD_E_NULL;
    if (ldx < F || !ckpt_ok(q)) return PSGD_E_INVALID;
    const ActShape s{T, (int)F, ceil_div(F, ACT_GROUP)};
    return launch_unpack(s, q, scales, x, ldx, dtype, (cudaStream_t)stream) ? PSGD_OK : PSGD_E_CUDA;
}

psgd_status psgd_copy_rows(const void* src, int64_t lds, int64_t rows, int64_t cols, void* dst, int64_t ldd, psgd_stream stream) {
    if (rows < 0 || rows > MAX_EXTENT || !extent_ok(cols)) return PSGD_E_INVALID;
    if (rows == 0) return PSGD_OK;
    if (!src || !dst) return PSGD_E_NULL;
    if (lds < cols || ldd < cols) return PSGD_E_INVALID;
    const ActShape s{rows, (int)cols, ceil_div(cols, ACT_GROUP)};
    const ActGrid g = act_grid(rows, s.G, PACK_CTAS, true);
    return launch(k_copy_rows, g.grid, g.block, 0, (cudaStream_t)stream, s, (const __nv_bfloat16*)src, lds, (__nv_bfloat16*)dst, ldd) ? PSGD_OK : PSGD_E_CUDA;
}

psgd_status psgd_act_wgrad_workspace(int64_t T, int64_t O, int64_t F, size_t* bytes) {
    if (!bytes) return PSGD_E_NULL;
    if (!act_ok(T, F) || !extent_ok(O) || !tiles_ok(O, F)) return PSGD_E_INVALID;
    *bytes = T == 0 ? 256 : std::max(plan_wgrad(T, O, F, false).total, F % 4 ? plan_wgrad(T, O, F, true).total : 0);
    return PSGD_OK;
}

psgd_status psgd_act_wgrad(const void* dY, int64_t lddy, const int8_t* q, const uint8_t* scales, int64_t T, int64_t O, int64_t F, void* dW, int64_t lddw, int dtype,
                           int* status, void* ws, size_t ws_bytes, psgd_stream stream) try {
    cudaStream_t st = (cudaStream_t)stream;
    if (!act_ok(T, F) || !extent_ok(O) || !tiles_ok(O, F) || !dtype_ok(dtype)) return PSGD_E_INVALID;
    if (!dW || !ws || (T > 0 && (!dY || !q || !scales))) return PSGD_E_NULL;
    if (lddw < F || ((uintptr_t)ws & 255) || (T > 0 && (!operand_ok(dY, T, O, lddy) || !ckpt_ok(q)))) return PSGD_E_INVALID;
    if (T == 0) {
        const size_t es = dtype == PSGD_DT_F32 ? 4 : 2;
        return succeeded("cudaMemset2DAsync", cudaMemset2DAsync(dW, (size_t)lddw * es, 0, (size_t)F * es, (size_t)O, st)) ? PSGD_OK : PSGD_E_CUDA;
    }
    const bool vec = aligned16(dW) && lddw % (dtype == PSGD_DT_F32 ? 4 : 8) == 0;
    WgradPlan g = plan_wgrad(T, O, F, dtype == PSGD_DT_F32 && !vec);
    if (ws_bytes < g.total) g = plan_wgrad(T, O, F, false);       // (an aligned width whose result starts or steps unaligned)
    if (ws_bytes < g.total) return PSGD_E_WORKSPACE;
    if (overlap(stretch(dW, O, F, lddw, dtype == PSGD_DT_F32 ? 4 : 2), stretch(dY, T, O, lddy, 2))) return PSGD_E_INVALID;
    char* w = (char*)ws;
    const ActShape s{T, (int)F, ceil_div(F, ACT_GROUP)};
    if (!launch_unpack(ActShape{T, (int)g.ldx, s.G}, q, scales, w + g.x, g.ldx, PSGD_DT_BF16, st)) return PSGD_E_CUDA;     // the padding too: its values are zeros
    TileArgs a{};
    a.status = status ? status : (int*)w;
    TileProblem& t = a.p[0];
    t.out = dW; t.ldo = lddw; t.out_f32 = dtype == PSGD_DT_F32;
    t.vec = vec;
    t.kacc = t.out_f32 ? KACC_F32 : 0;
    t.part = (float*)(w + g.part);
    const Operand A[2] = {{dY, lddy, true}, {}}, B[2] = {{w + g.x, g.ldx, true}, {}};
    const TilePlan p[2] = {g.p, {}};
    return launch_products(1, A, B, p, a, g.pairs, st);
} catch (...) {
    return cuda_error("host", "exception");
}

psgd_status psgd_swiglu_forward(const void* gate, int64_t ldg, const void* up, int64_t ldu, int64_t T, int64_t F, void* h, int64_t ldh, int8_t* q_gate, uint8_t* s_gate,
                                int8_t* q_up, uint8_t* s_up, psgd_stream stream) {
    if (!act_ok(T, F)) return PSGD_E_INVALID;
    if (T == 0) return PSGD_OK;
    if (!gate || !up || !h || !q_gate || !s_gate || !q_up || !s_up) return PSGD_E_NULL;
    if (ldg < F || ldu < F || ldh < F || !ckpt_ok(q_gate) || !ckpt_ok(q_up)) return PSGD_E_INVALID;
    const ActShape s{T, (int)F, ceil_div(F, ACT_GROUP)};
    const GatedForward a{(const __nv_bfloat16*)gate, (const __nv_bfloat16*)up, (__nv_bfloat16*)h, ldg, ldu, ldh, q_gate, q_up, s_gate, s_up};
    const bool vec = vec8(gate, ldg, F, PSGD_DT_BF16) && vec8(up, ldu, F, PSGD_DT_BF16) && vec8(h, ldh, F, PSGD_DT_BF16);
    const ActGrid g = act_grid(T, s.G, FORWARD_CTAS, !vec);
    return launch(vec ? k_swiglu_forward<false> : k_swiglu_forward<true>, g.grid, g.block, 0, (cudaStream_t)stream, s, a) ? PSGD_OK : PSGD_E_CUDA;
}

psgd_status psgd_swiglu_backward(const void* dh, int64_t lddh, const int8_t* q_gate, const uint8_t* s_gate, const int8_t* q_up, const uint8_t* s_up, int64_t T, int64_t F,
                                 void* d_gate, int64_t ldg, void* d_up, int64_t ldu, void* h, int64_t ldh, psgd_stream stream) {
    if (!act_ok(T, F)) return PSGD_E_INVALID;
    if (T == 0) return PSGD_OK;
    if (!dh || !q_gate || !s_gate || !q_up || !s_up || !d_gate || !d_up) return PSGD_E_NULL;
    if (lddh < F || ldg < F || ldu < F || (h && ldh < F) || !ckpt_ok(q_gate) || !ckpt_ok(q_up)) return PSGD_E_INVALID;
    const ActShape s{T, (int)F, ceil_div(F, ACT_GROUP)};
    const GatedBackward a{(const __nv_bfloat16*)dh, q_gate, q_up, s_gate, s_up, (__nv_bfloat16*)d_gate, (__nv_bfloat16*)d_up, (__nv_bfloat16*)h, lddh, ldg, ldu, ldh};
    const bool vec = vec8(dh, lddh, F, PSGD_DT_BF16) && vec8(d_gate, ldg, F, PSGD_DT_BF16) && vec8(d_up, ldu, F, PSGD_DT_BF16) && (!h || vec8(h, ldh, F, PSGD_DT_BF16));
    const ActGrid g = act_grid(T, s.G, BACKWARD_CTAS, !vec);
    const auto run = [&](auto kernel) { return launch(kernel, g.grid, g.block, 0, (cudaStream_t)stream, s, a) ? PSGD_OK : PSGD_E_CUDA; };
    if (h) return run(vec ? k_swiglu_backward<true, false> : k_swiglu_backward<true, true>);
    return run(vec ? k_swiglu_backward<false, false> : k_swiglu_backward<false, true>);
}

}  // extern "C"
