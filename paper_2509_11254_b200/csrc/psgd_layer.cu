// Host side of the operators between a layer's matrix products, declared in include/psgd.h: layer norm and rotary positions, forward and backward.
// Argument checks, workspace layout and launches; nothing here allocates, synchronises or keeps anything between calls.
#include "psgd_norm.cuh"
#include "psgd_rotary.cuh"
#include "psgd_train.cuh"

using namespace psgd;

namespace {

typedef __nv_bfloat16 bf16;

// Rows of 16-byte units: the address, the stride and the width allow eight values at a time.
bool whole_units(const void* p, int64_t ld, int64_t F, int dtype) { return !p || (F % 8 == 0 && aligned16(p) && ld % (16 / size_of(dtype)) == 0); }
bool rows_ok(int64_t T, int64_t F) { return T >= 0 && T <= MAX_EXTENT && extent_ok(F); }

// ---- layer norm ----
// How the rows go: RING (16-byte units), PHASE (bfloat16 of any width and alignment, all operands alike), LANES (anything else, a value per lane)
enum NormRows { RING, PHASE, LANES };
// Whether two matrices of bfloat16 lie alike: the same place within 16 bytes in every row (one that is not there lies like any other)
bool alike(const void* p, int64_t ldp, const void* q, int64_t ldq, int64_t T) { return !q || ((((uintptr_t)p ^ (uintptr_t)q) & 15) == 0 && (T == 1 || (ldp - ldq) % 8 == 0)); }
// How a row's units are shared: `vpt` per thread, `threads` per row (whole warps), `rows` side by side per CTA, `stages` rows of a ring.
struct NormPlan { int vpt, threads, rows, stages; bool wide; int64_t ctas; size_t smem; };
constexpr int64_t NORM_SMEM = 200 << 10;            // of a multiprocessor's, for weights and rings

// `row_bytes`: of all operands of a row that are read.  The number of rows has no say in how a row is shared: the bits of aligned rows do not depend
// on their batch.
NormPlan plan_norm(int64_t T, int64_t F, NormRows rows, int64_t row_bytes, bool more, bool keep, bool backward) {
    NormPlan p{};
    const int64_t sms = device_sms();
    if (rows == LANES) {                                    // a value per lane: one unit per thread
        const int64_t units = (F + 255) / 256 * 32;
        p.wide = units > NORM_THREADS;
        p.vpt = 1;
        p.threads = p.wide ? NORM_THREADS : (int)units;
        p.rows = p.wide ? 1 : std::max(1, 256 / p.threads);
        p.smem = backward && p.rows > 1 ? (size_t)p.rows * 2 * F * 4 : 0;
        p.ctas = std::min<int64_t>((T + p.rows - 1) / p.rows, sms * std::max(1, (backward ? 512 : 1024) / (p.threads * p.rows)));
        return p;
    }
    // Units per thread: as many as registers hold, which is eight where the row has nothing to be added to (2048 columns: 24.8 us with eight, 29 with four; with
    // a residual 51 and 47) and four elsewhere, fewer where that leaves fewer places empty.
    const int64_t units = (F + 7 + (rows == PHASE ? 7 : 0)) / 8;
    double best = 1e300;
    for (int vpt : {8, 4, 3, 2, 1}) {
        if (vpt == 8 && (rows == PHASE || backward || more)) continue;
        const int64_t g = (int64_t)align_up((size_t)ceil_div(units, vpt), 32);
        if (g > NORM_THREADS || (vpt == 4 && rows == PHASE && backward && units <= 3 * NORM_THREADS)) continue;      // (four spill there: 8192 x 5003 119 us, three 89)
        const double cost = (double)g * (vpt + 1) + (g > 32 ? 16 : 0);       // a warp's part of a row costs about a unit beside its units, the exchange a little more
        if (cost < best) { best = cost; p.vpt = vpt; p.threads = (int)g; }
    }
    const int64_t slots = (int64_t)p.threads * p.vpt, params = slots * (backward ? 32 : 64);
    const int64_t row = row_bytes / F * slots * 8, image = rows == PHASE && keep ? slots * 16 + 16 : 0;
    p.wide = p.threads == 0 || params + row + image > NORM_SMEM;
    if (p.wide) {
        p.threads = NORM_THREADS;
        p.rows = 1;
        p.ctas = std::min<int64_t>(T, sms * 4);
        return p;
    }
    // Measured over widths of 256 to 8192: rows of several warps in CTAs of 512 threads (the ring of two rows then fits twice 8 rows of 12 KB), rows of one warp in CTAs of 256
    const int threads = p.threads > 32 ? NORM_THREADS : 256;
    p.rows = threads / p.threads;
    const int fit = std::max(1, (p.vpt == 1 ? (backward ? 768 : 1024) : p.vpt == 2 && !backward ? 768 : 512) / (p.threads * p.rows));       // CTAs per multiprocessor, by registers
    // Forward, a row is in registers while the next is on its way: a second row in the ring pays for short ones only (256 columns with a residual 23.7 us against
    // 26.8, 768: 17.4, 18.4; 2048: 49.0 with one, 51.7 with two).  Backward the row stays in the ring to the end.
    p.stages = (backward || row <= 4096) && params + (2 * row + image) * p.rows <= NORM_SMEM / fit ? 2 : 1;
    while (p.rows > 1 && params + (row + image) * p.rows > NORM_SMEM) --p.rows;
    p.smem = (size_t)(params + (row * p.stages + image) * p.rows);
    if (backward && (p.rows > 1 || rows == PHASE)) p.smem = std::max(p.smem, (size_t)p.rows * 2 * (rows == PHASE ? slots * 8 : F) * 4);
    // as many CTAs as fit, forward with long rows twice as many: who is done early takes another (2048 columns with a residual 49.0 -> 47.0 us)
    const int64_t resident = std::max<int64_t>(1, std::min<int64_t>(fit, NORM_SMEM / (int64_t)p.smem));
    const int64_t some = (T + p.rows - 1) / p.rows, most = sms * resident * (!backward && more && p.threads > 32 ? 2 : 1);
    // PHASE: rows eight apart begin alike whatever their stride
    p.ctas = rows == PHASE && T > 1 ? std::min((some + 7) / 8 * 8, std::max<int64_t>(8, most / 8 * 8)) : std::min(some, most);
    return p;
}

struct NormGrad { NormPlan p; int64_t parts; size_t part, sums, total; };
NormGrad plan_norm_grad(int64_t T, int64_t F, NormRows rows, int64_t row_bytes) {
    NormGrad g{};
    g.p = plan_norm(T, F, rows, row_bytes, false, false, true);
    // Wide rows: CTAs of 2048 columns that share the rows, four per multiprocessor; the wider the rows, the fewer for each stretch of columns, but never so few that a thread adds more
    // than T / 128 + 49 of them into one float32 sum (one round of CTAs alone: 1000 of
    // 4000 rows of 262144 columns); then several rounds of CTAs (1000 x 131072 bfloat16: 330 us with one, 356 with three).
    const int64_t tiles = (F + 2047) / 2048, round = std::max<int64_t>(1, device_sms() * 4 / tiles), needed = ceil_div(T, T / 128 + 48);
    g.parts = g.p.wide ? std::min<int64_t>(T, ceil_div(std::max(needed, round), round) * round) : g.p.ctas;
    g.part = 0;
    g.sums = align_up((size_t)g.parts * 2 * F * 4, 256);
    g.total = g.sums + (g.p.wide ? align_up((size_t)T * 8, 256) : 0);
    return g;
}

template <typename Args>
bool launch_norm(void (*kernel)(Args), const NormPlan& p, const Args& a, cudaStream_t st) {
    if (p.smem > 32 << 10) set_smem_attr((const void*)kernel, p.smem);      // (static shared memory comes on top)
    return launch(kernel, dim3((unsigned)p.ctas), dim3(p.threads, p.rows), p.smem, st, a);
}
template <typename X, typename Y, bool PHASED>
bool ring_forward(const NormForward& a, const NormPlan& p, cudaStream_t st) {
    switch (p.vpt) {
        case 1: return launch_norm(k_norm_forward<X, Y, 1, PHASED>, p, a, st);
        case 2: return launch_norm(k_norm_forward<X, Y, 2, PHASED>, p, a, st);
        case 3: return launch_norm(k_norm_forward<X, Y, 3, PHASED>, p, a, st);
        case 4: return launch_norm(k_norm_forward<X, Y, 4, PHASED>, p, a, st);
    }
    if constexpr (!PHASED) return launch_norm(k_norm_forward<X, Y, 8, false>, p, a, st);
    return false;
}
template <typename X, typename Y>
bool norm_forward(NormForward a, const NormPlan& p, NormRows rows, cudaStream_t st) {
    a.stages = p.stages;
    if (p.wide) return rows == RING ? launch_norm(k_norm_forward_wide<X, Y, true>, p, a, st) : launch_norm(k_norm_forward_wide<X, Y, false>, p, a, st);
    if (rows == RING) return ring_forward<X, Y, false>(a, p, st);
    if constexpr (sizeof(X) == 2)
        if (rows == PHASE) return ring_forward<X, Y, true>(a, p, st);
    return launch_norm(k_norm_forward_any<X, Y>, p, a, st);
}
template <typename X, typename Y, bool PHASED>
bool ring_backward(const NormBackward& a, const NormPlan& p, cudaStream_t st) {
    switch (p.vpt) {
        case 1: return launch_norm(k_norm_backward<X, Y, 1, PHASED>, p, a, st);
        case 2: return launch_norm(k_norm_backward<X, Y, 2, PHASED>, p, a, st);
        case 3: return launch_norm(k_norm_backward<X, Y, 3, PHASED>, p, a, st);
    }
    return launch_norm(k_norm_backward<X, Y, 4, PHASED>, p, a, st);
}
template <typename X, typename Y>
bool norm_backward(NormBackward a, const NormGrad& g, NormRows rows, cudaStream_t st) {
    const NormPlan& p = g.p;
    a.stages = p.stages;
    if (p.wide) {
        const dim3 grid(ceil_div(a.F, 2048), (unsigned)g.parts), block(256);
        if (rows == RING) return launch_norm(k_norm_sums_wide<X, Y, true>, p, a, st) && launch(k_norm_apply_wide<X, Y, true>, grid, block, 0, st, a);
        return launch_norm(k_norm_sums_wide<X, Y, false>, p, a, st) && launch(k_norm_apply_wide<X, Y, false>, grid, block, 0, st, a);
    }
    if (rows == RING) return ring_backward<X, Y, false>(a, p, st);
    if constexpr (sizeof(X) == 2)
        if (rows == PHASE) return ring_backward<X, Y, true>(a, p, st);
    return launch_norm(k_norm_backward_any<X, Y>, p, a, st);
}
// the pairs of types: x and y (dy) alike, or x float32 and y bfloat16
bool types_ok(int x, int y) { return dtype_ok(x) && dtype_ok(y) && (x == y || x == PSGD_DT_F32); }
template <typename Call>
bool by_type(int x, int y, Call&& call) { return x == PSGD_DT_BF16 ? call((bf16*)0, (bf16*)0) : y == PSGD_DT_BF16 ? call((float*)0, (bf16*)0) : call((float*)0, (float*)0); }

// ---- rotary positions ----
// A tensor [T][heads][head] as stretches of bytes: rows of tokens with their heads in them, or rows of heads with their tokens; else (values that are used
// several times, orders that mix) one stretch from its first byte to its last.  `once`: no value lies in two places.
Stretch extent_of(const void* p, int64_t T, int64_t heads, int64_t head, int64_t token, int64_t step, int bytes, bool& once) {
    if (heads <= 1) step = head;                       // (the stride of an extent of one is never used)
    const int64_t in_token = (heads - 1) * step + head;
    if (T <= 1) token = in_token;
    const int64_t in_head = (T - 1) * token + head;
    once = true;
    if (step >= head && token >= in_token) return {p, T, in_token * bytes, token * bytes};
    if (token >= head && step >= in_head) return {p, heads, in_head * bytes, step * bytes};
    once = false;
    const int64_t all = ((T - 1) * token + in_token) * bytes;
    return {p, 1, all, all};
}

}  // namespace

extern "C" {

psgd_status psgd_norm_forward(const void* x, int64_t ldx, int x_dtype, const void* r, int64_t ldr, const void* w, const void* b, int w_dtype, float eps, int center, int64_t T,
                              int64_t F, void* s, int64_t lds, void* y, int64_t ldy, int y_dtype, float* mean, float* rstd, int8_t* q, uint8_t* scales, psgd_stream stream) {
    if (!rows_ok(T, F) || !types_ok(x_dtype, y_dtype) || !dtype_ok(w_dtype) || !(eps >= 0.f)) return PSGD_E_INVALID;
    if (T == 0) return PSGD_OK;
    if (!x || !w || !y || !rstd || (r && !s) || (center && !mean) || (q && !scales)) return PSGD_E_NULL;
    if (ldx < F || ldy < F || (r && ldr < F) || (s && lds < F) || ((uintptr_t)q & 15)) return PSGD_E_INVALID;
    const int size = size_of(x_dtype);
    const int64_t params = F * size_of(w_dtype), groups = T * ((F + ACT_GROUP - 1) / ACT_GROUP);
    if (outputs_meet({stretch(s, T, F, lds, size), stretch(y, T, F, ldy, size_of(y_dtype)), stretch(center ? mean : nullptr, T * 4), stretch(rstd, T * 4), stretch(q, groups * ACT_GROUP),
                      stretch(q ? scales : nullptr, groups)},
                     {stretch(x, T, F, ldx, size), stretch(r, T, F, ldr, size), stretch(w, params), stretch(b, params)}))
        return PSGD_E_INVALID;
    const bool whole = whole_units(x, ldx, F, x_dtype) && whole_units(r, ldr, F, x_dtype) && whole_units(s, lds, F, x_dtype) && whole_units(y, ldy, F, y_dtype);
    const bool same = x_dtype == PSGD_DT_BF16 && alike(x, ldx, r, ldr, T) && alike(x, ldx, s, lds, T) && alike(x, ldx, y, ldy, T);
    const NormRows rows = whole ? RING : same ? PHASE : LANES;
    NormForward a{};
    a.T = T; a.F = (int)F; a.center = center != 0; a.eps = eps;
    a.x = x; a.r = r; a.s = s; a.y = y;
    a.ldx = ldx; a.ldr = ldr; a.lds = lds; a.ldy = ldy;
    a.w = {w, w_dtype == PSGD_DT_BF16}; a.b = {b, w_dtype == PSGD_DT_BF16};
    a.mean = center ? mean : nullptr; a.rstd = rstd; a.q = q; a.scales = scales;
    const NormPlan p = plan_norm(T, F, rows, F * size_of(x_dtype) * (r ? 2 : 1), r != nullptr, q != nullptr, false);
    const bool ok = by_type(x_dtype, y_dtype, [&](auto* tx, auto* ty) {
        return norm_forward<std::remove_pointer_t<decltype(tx)>, std::remove_pointer_t<decltype(ty)>>(a, p, rows, (cudaStream_t)stream);
    });
    return ok ? PSGD_OK : PSGD_E_CUDA;
}

psgd_status psgd_norm_workspace(int64_t T, int64_t F, size_t* bytes) {
    if (!bytes) return PSGD_E_NULL;
    if (!rows_ok(T, F)) return PSGD_E_INVALID;
    *bytes = 256;
    if (T > 0) {
        // whatever the types, the alignment and the operands (2 + 2, 4 + 2, 4 + 4 bytes per column, and x's again)
        *bytes = plan_norm_grad(T, F, LANES, 0).total;
        for (int each : {4, 6, 8, 10, 12}) *bytes = std::max({*bytes, plan_norm_grad(T, F, RING, F * each).total, plan_norm_grad(T, F, PHASE, F * each).total});
    }
    return PSGD_OK;
}

psgd_status psgd_norm_backward(const void* dy, int64_t lddy, int dy_dtype, const void* x, int64_t ldx, int x_dtype, const void* w, int w_dtype, const float* mean,
                               const float* rstd, const void* add, int64_t ldadd, int64_t T, int64_t F, void* dx, int64_t lddx, float* dw, float* db, void* ws,
                               size_t ws_bytes, psgd_stream stream) {
    cudaStream_t st = (cudaStream_t)stream;
    if (!rows_ok(T, F) || !types_ok(x_dtype, dy_dtype) || !dtype_ok(w_dtype)) return PSGD_E_INVALID;
    if (!dw || !ws || (T > 0 && (!dy || !x || !w || !rstd || !dx))) return PSGD_E_NULL;
    if (T == 0)
        return succeeded("cudaMemsetAsync", cudaMemsetAsync(dw, 0, (size_t)F * 4, st)) && (!db || succeeded("cudaMemsetAsync", cudaMemsetAsync(db, 0, (size_t)F * 4, st))) ? PSGD_OK
                                                                                                                                                          : PSGD_E_CUDA;
    if (lddy < F || ldx < F || (add && ldadd < F) || lddx < F || ((uintptr_t)ws & 255)) return PSGD_E_INVALID;
    const int size = size_of(x_dtype);
    const Stretch out = stretch(dx, T, F, lddx, size);
    if (overlap(out, stretch(dy, T, F, lddy, size_of(dy_dtype))) || overlap(out, stretch(x, T, F, ldx, size)) || overlap(out, stretch(add, T, F, ldadd, size))) return PSGD_E_INVALID;
    const bool whole = whole_units(dy, lddy, F, dy_dtype) && whole_units(x, ldx, F, x_dtype) && whole_units(add, ldadd, F, x_dtype) && whole_units(dx, lddx, F, x_dtype);
    const bool same = x_dtype == PSGD_DT_BF16 && alike(x, ldx, dy, lddy, T) && alike(x, ldx, add, ldadd, T) && alike(x, ldx, dx, lddx, T);
    // (16384 rows with a residual: 1801 columns 70 us by lanes, 75 by units; 2051: 113, 74; 4099, more than a CTA has lanes for: 591, 156.
    // 2051 columns of 512 rows: 8.1, 10.2; of 2048: 18.0, 16.3)
    const NormRows rows = whole ? RING : same && (F > 8 * NORM_THREADS || (F >= 2048 && T >= 2048)) ? PHASE : LANES;
    const NormGrad g = plan_norm_grad(T, F, rows, F * (size_of(dy_dtype) + size * (add ? 2 : 1)));
    if (ws_bytes < g.total) return PSGD_E_WORKSPACE;
    if (outputs_meet({out, stretch(dw, F * 4), stretch(db, F * 4), stretch(ws, (int64_t)g.total)},
                     {stretch(dy, T, F, lddy, size_of(dy_dtype)), stretch(x, T, F, ldx, size), stretch(add, T, F, ldadd, size), stretch(w, F * size_of(w_dtype)), stretch(mean, T * 4),
                      stretch(rstd, T * 4)}))
        return PSGD_E_INVALID;
    NormBackward a{};
    a.T = T; a.F = (int)F; a.center = mean != nullptr;
    a.dy = dy; a.x = x; a.add = add; a.dx = dx;
    a.lddy = lddy; a.ldx = ldx; a.ldadd = ldadd; a.lddx = lddx;
    a.w = {w, w_dtype == PSGD_DT_BF16};
    a.mean = mean; a.rstd = rstd;
    a.part = (float*)((char*)ws + g.part);
    a.dw = dw; a.db = db;
    a.sums = (float2*)((char*)ws + g.sums);
    const bool ok = by_type(x_dtype, dy_dtype, [&](auto* tx, auto* ty) {
        return norm_backward<std::remove_pointer_t<decltype(tx)>, std::remove_pointer_t<decltype(ty)>>(a, g, rows, st);
    });
    if (!ok) return PSGD_E_CUDA;
    if (g.parts == 1) return PSGD_OK;                  // (the one CTA has written the results)
    const NormJoin j{(int)F, (int)g.parts, a.part, dw, db};
    return launch(k_norm_join, dim3(ceil_div(F, 32), db ? 2 : 1), dim3(1024), 0, st, j) ? PSGD_OK : PSGD_E_CUDA;
}

psgd_status psgd_rotary(const void* q, int64_t q_token, int64_t q_head, int64_t heads_q, void* out_q, int64_t oq_token, int64_t oq_head, const void* k, int64_t k_token,
                        int64_t k_head, int64_t heads_k, void* out_k, int64_t ok_token, int64_t ok_head, const int64_t* positions, const double* frequencies, int64_t T,
                        int64_t head, int64_t rotated, int layout, int backward, float scale, int dtype, psgd_stream stream) {
    if (T < 0 || T > MAX_EXTENT || heads_q < 0 || heads_k < 0 || heads_q + heads_k > 65536 || head < 1 || (heads_q + heads_k) * head > MAX_EXTENT) return PSGD_E_INVALID;
    if (rotated < 2 || rotated % 2 || rotated > head || rotated > 2 * ROT_PAIRS || !dtype_ok(dtype)) return PSGD_E_INVALID;
    if (layout != PSGD_ROTARY_HALF && layout != PSGD_ROTARY_INTERLEAVED) return PSGD_E_INVALID;
    const int64_t strides[8] = {q_token, q_head, oq_token, oq_head, k_token, k_head, ok_token, ok_head};
    for (int64_t s : strides)
        if (s < 0) return PSGD_E_INVALID;
    const int64_t heads = heads_q + heads_k;
    if (T == 0 || heads == 0) return PSGD_OK;
    if (!positions || !frequencies || (heads_q && (!q || !out_q)) || (heads_k && (!k || !out_k))) return PSGD_E_NULL;
    const RotaryTensor t[2] = {{q, out_q, q_token, q_head, oq_token, oq_head}, {k, out_k, k_token, k_head, ok_token, ok_head}};
    const int64_t count[2] = {heads_q, heads_k};
    bool in_place = true;
    // the most values that a thread can move at a time: every address, stride and width is a multiple of it (of 16 bytes at most)
    const bool half = layout == PSGD_ROTARY_HALF;
    uint64_t all = (uint64_t)head | (uint64_t)rotated / (half ? 2 : 1);
    Stretch in[2] = {}, out[2] = {};
    for (int i = 0; i < 2; ++i) {
        if (!count[i]) continue;
        bool once;
        in[i] = extent_of(t[i].in, T, count[i], head, t[i].in_token, t[i].in_head, size_of(dtype), once);
        out[i] = extent_of(t[i].out, T, count[i], head, t[i].out_token, t[i].out_head, size_of(dtype), once);
        if (!once) return PSGD_E_INVALID;              // two values would be written to one place
        if (T > 1) all |= (uint64_t)(t[i].in_token | t[i].out_token);
        if (count[i] > 1) all |= (uint64_t)(t[i].in_head | t[i].out_head);
        const uint64_t at = (uint64_t)(uintptr_t)t[i].in | (uint64_t)(uintptr_t)t[i].out;
        all |= at % 16 ? at / size_of(dtype) : 0;
        in_place = in_place && t[i].in == t[i].out;
    }
    for (int i = 0; i < 2; ++i)
        for (int j = 0; j < 2; ++j) {
            // in place: the very tensor, so that every value is read and written by one thread
            const bool same = i == j && t[i].in == t[i].out && (T == 1 || t[i].in_token == t[i].out_token) && (count[i] <= 1 || t[i].in_head == t[i].out_head);
            if (count[i] && count[j] && !same && overlap(out[i], in[j])) return PSGD_E_INVALID;
        }
    if (heads_q && heads_k && overlap(out[0], out[1])) return PSGD_E_INVALID;
    const Stretch angles[2] = {stretch(positions, T * 8), stretch(frequencies, rotated / 2 * 8)};
    for (const Stretch& o : out)
        if (overlap(o, angles[0]) || overlap(o, angles[1])) return PSGD_E_INVALID;
    int V = 8;
    while (V > 1 && all % V) V /= 2;
    RotaryArgs a{};
    a.T = T; a.heads_q = (int)heads_q; a.heads = (int)heads; a.rotated = (int)rotated; a.head = (int)head;
    a.turned = (int)(half || V == 1 ? rotated / 2 / V : rotated / V);
    a.per_head = a.turned + (in_place ? 0 : (int)((head - rotated) / V));
    a.groups = ceil_div(heads, ROT_HEADS);
    const int64_t items = (int64_t)a.groups * a.per_head;         // per token
    const int sms = device_sms();
    // tokens of a CTA at a time: two rounds of items where there are enough tokens for every CTA, as many angles as shared memory is set aside for
    a.tokens = (int)std::max<int64_t>(1, std::min<int64_t>({2 * ROT_THREADS / items, T / (4 * sms), ROT_PAIRS / (rotated / 2)}));
    a.by_head = fast_div((unsigned)a.per_head); a.by_groups = fast_div((unsigned)a.groups); a.by_pairs = fast_div((unsigned)(rotated / 2));
    a.q = t[0]; a.k = t[1];
    a.positions = (const long long*)positions;
    a.frequencies = frequencies;
    a.scale = scale;
    a.sign = backward ? -1.f : 1.f;
    const dim3 grid((unsigned)std::min<int64_t>((T + a.tokens - 1) / a.tokens, (int64_t)sms * 8));
    const auto run = [&](auto kernel) { return launch(kernel, grid, dim3(ROT_THREADS), 0, (cudaStream_t)stream, a) ? PSGD_OK : PSGD_E_CUDA; };
    const auto by_width = [&](auto* x) {
        typedef std::remove_pointer_t<decltype(x)> X;
        if (V == 8) return half ? run(k_rotary<X, 8, true>) : run(k_rotary<X, 8, false>);
        if (V == 4) return half ? run(k_rotary<X, 4, true>) : run(k_rotary<X, 4, false>);
        if (V == 2) return half ? run(k_rotary<X, 2, true>) : run(k_rotary<X, 2, false>);
        return half ? run(k_rotary<X, 1, true>) : run(k_rotary<X, 1, false>);
    };
    return dtype == PSGD_DT_BF16 ? by_width((bf16*)0) : by_width((float*)0);
}

}  // extern "C"
