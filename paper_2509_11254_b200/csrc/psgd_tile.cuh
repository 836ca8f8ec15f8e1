// Tensor-core products of bfloat16 matrices for the training operators: the logits of the last layer (with the softmax
// statistics in the epilogue), the two gradients of that layer, and the weight gradient of a linear layer.
//
//     C [M][N] = sum_k A(m, k) B(n, k),     operands bfloat16, sums in float32 (tensor memory).
//
// Either operand lies in memory with k contiguous ("K-major", rows of the matrix) or with m (n) contiguous ("MN-major":
// the gradients contract over tokens, the slow index of every activation), which the shared-memory descriptors and
// the instruction descriptor express, so that no operand is ever transposed in memory.
//
// One unit of work is a 256 x 256 tile of C (or a range of k of one), computed by a PAIR of CTAs (tcgen05.mma cta_group::2):
// each CTA holds 128 rows of A, half of the columns' rows of B and 128 rows of the accumulator, so that per multiprocessor
// and 64 of k 32 KB are fetched for 128 x 256 x 64 products: half of what two separate 128 x 256 tiles would fetch.  The grid is
// persistent (one pair per two multiprocessors).  Roles: one thread issues the TMA loads into a six-stage ring, one
// thread of the even CTA issues the MMAs, eight warps of each CTA work on the accumulators, of which tensor memory
// holds two (512 columns), so that the epilogue of a unit runs beside the MMAs of the next.  (Sixteen warps leave 96 registers a
// thread: the softmax epilogue then spills, 127 -> 160 us on 4096 x 32000 x 768.)
//
// Whole waves of tiles run with all of k; the tiles of the last, partly filled wave are split over k so that every pair has
// work.  Their partial sums go to the workspace and k_join adds them in the order of k (a fixed order, no atomics; letting
// the last pair to arrive add them up alone cost 25 us of a 172 us product, one multiprocessor cannot read faster).
//
// Measured alone: logits with statistics 4096 x 32000 x 768 in 150 us (1.34 PFLOP/s; the epilogue's reads of tensor memory take the MMAs' bandwidth),
// 16384 x 32000 x 2048 in 1.33 ms (1.61), both gradients of the former in 265 us (1.52, tensor pipe 95 % active), weight gradient
// 16384 x 5504 x 2048 in 247 us (1.50).  Bound by the tensor cores at the clock that 1000 W allow (1450 MHz there); small products by
// 3300 cycles until the first boxes have landed and 3700 from the last MMA to the end.
// Every wait on an mbarrier is bounded: one that runs out sets PSGD_W_TIMEOUT in the status word and the kernel ends.  A warp of the epilogue whose wait
// for an accumulator has run out (because the warps before it gave up, or by itself) writes NaN from then on, so that no call's results look good by mistake.
#pragma once
#include <cuda_bf16.h>

#include "psgd_ptx.cuh"
#include "psgd_values.cuh"

namespace psgd {

constexpr int TG_BM = 256;                    // rows of C per unit (128 per CTA)
constexpr int TG_BN = 256;                    // columns of C per unit
constexpr int TG_BK = 64;                     // k per stage: 128 bytes of bfloat16, one swizzle row
constexpr int TG_STAGES = 6;
constexpr int TG_HALF_BYTES = 128 * TG_BK * 2;          // one operand of one stage in one CTA
constexpr int TG_STAGE_BYTES = 2 * TG_HALF_BYTES;
constexpr int TG_EPI_WARPS = 8;
constexpr int TG_THREADS = 64 + 32 * TG_EPI_WARPS;      // warp 0: TMA, warp 1: MMA and tensor-memory owner, warps 2-9: epilogue
constexpr int TG_STAGING = 4096;              // per epilogue warp: 32 rows of 128 bytes, turned from row-per-lane to row-contiguous
constexpr int TG_PART = TG_BM * TG_BN;        // floats of one partial tile
constexpr int XE_SEG = 64, XE_SEG_LOSS = 128; // columns per softmax statistic: where exponents are kept relative to its maximum, and loss only

inline size_t tile_smem_bytes() { return (size_t)TG_STAGES * TG_STAGE_BYTES + TG_EPI_WARPS * TG_STAGING + 1024 + 256; }

// EPI_LOSS, EPI_SOFTMAX: statistics of the logits without and with their stored exponents, the labels' logits on the way.  EPI_TEACH_LOSS, EPI_TEACH: the same of logits
// divided by a temperature, the logits of a list of columns per row on the way.  EPI_STORE: the product itself.
enum TileEpilogue { EPI_LOSS = 0, EPI_SOFTMAX = 1, EPI_STORE = 2, EPI_TEACH_LOSS = 3, EPI_TEACH = 4 };

// One product and how it is cut.
struct TileProblem {
    int M, N;
    int mt, nt, kb;            // tiles along M and N, stages along K
    int bn;                    // columns per tile
    int full;                  // tiles done in one piece (the first `full` in raster order)
    int S, kbps;               // pieces and stages per piece of every later tile
    int tail;                  // later tiles
    int parts;                 // later tiles go through memory as partial tiles and k_join: always where S > 1
    int units;
    int gm;                    // raster: groups of gm row tiles, column by column
    FastDiv by_group, by_gm, by_rest, by_tail;   // gm * nt, gm, rows of the last group, tail
    int kacc;                  // stages summed in one accumulator (0: all of them)
    int a_mn;                  // A is MN-major
    // EPI_STORE: out = scale * (sum + addend)
    void* out;
    long long ldo;             // elements
    int out_f32, vec;          // vec: every row of `out` (and of `addend`) 16-byte aligned
    const float* addend;       // [M][N] float32 or nullptr
    const float* scale;        // DEVICE scalar or nullptr
    float* part;               // partial tiles [S][tail][2][256 columns][128 rows]
};
struct TileArgs {
    TileProblem p[2];          // EPI_STORE: one or two products in one launch
    // Who does what: the units of p[0] go round the pairs, `first_q` each and one more for the first `first_r` pairs; meanwhile the other
    // pairs do `extra` units of p[1] each, and the rest of those go round all pairs.
    int first_q, first_r, extra;
    int* status;               // device status word
    // all but EPI_STORE
    int a_rows, a_odd;         // rows of A in a box, a multiple of 8, and whether the odd CTA has any: 128 and 1, less where all of M is one short
                               // tile.  The rows that no box brings are zeros for good (not garbage: that would cost the MMAs' power).
    const long long* labels;
    float2* stats;             // [M][nseg]: maximum and sum of exp(l - maximum) of each segment
    float* label_logit;        // [M]
    unsigned short* q;         // [M][ldq]: (maximum - l) log2(e) in steps of 2^-10, 65535 for "nothing left"
    long long ldq;
    int nseg;                  // statistics per row
    int* done;                 // counter to clear for the next kernel, or nullptr
    // EPI_TEACH_LOSS, EPI_TEACH: the listed entries by block of 32 rows and 32 columns (k_teach)
    const int* bins;           // [row blocks][nbins + 1]: where a block's entries begin among those of its rows
    const unsigned* entries;   // [row blocks][32 K]: place in the row's list << 10 | row of the block << 5 | column of the block
    float* entry_logit;        // [M][K]
    int nbins, K;
    float log2e;               // log2(e) / temperature
    float temperature;
    // EPI_SOFTMAX, EPI_TEACH: 1 (temperature) / (sum of the weights of the rows that count), formed by a warp that has nothing else to do
    float* norm;               // or nullptr
    const long long* norm_labels;
    const float* norm_weight;
    long long norm_rows, ignore;
};

// Shared-memory matrix descriptors, 128-byte swizzle.  K-major: rows of 128 bytes, groups of 8 rows 1024 bytes apart.
// MN-major: rows hold 64 consecutive m, groups of 8 k are 1024 bytes apart, blocks of 64 m TG_HALF_BYTES / 2 apart.
__device__ __forceinline__ unsigned long long tile_desc(unsigned addr, bool mn) {
    unsigned long long d = (unsigned long long)((addr >> 4) & 0x3FFF);
    d |= (unsigned long long)(mn ? (TG_HALF_BYTES / 2) >> 4 : 1) << 16;
    d |= (unsigned long long)(1024 >> 4) << 32;
    d |= (unsigned long long)1 << 46;
    d |= (unsigned long long)2 << 61;
    return d;
}
// D float32, A and B bfloat16, M = 256 over the pair
__device__ __forceinline__ unsigned tile_idesc(int n, bool amn, bool bmn) {
    return (1u << 4) | (1u << 7) | (1u << 10) | ((amn ? 1u : 0u) << 15) | ((bmn ? 1u : 0u) << 16) | ((unsigned)(n >> 3) << 17) | ((unsigned)(TG_BM >> 4) << 24);
}
__device__ __forceinline__ void pair_mma(unsigned d, unsigned long long da, unsigned long long db, unsigned idesc, unsigned acc) {
    asm volatile("{\n.reg .pred p;\nsetp.ne.b32 p, %4, 0;\ntcgen05.mma.cta_group::2.kind::f16 [%0], %1, %2, %3, p;\n}\n"
                 ::"r"(d), "l"(da), "l"(db), "r"(idesc), "r"(acc) : "memory");
}
// arrives on the barrier at this offset in both CTAs once every MMA issued so far has completed
__device__ __forceinline__ void pair_commit(unsigned bar) {
    asm volatile("tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.multicast::cluster.b64 [%0], %1;\n" ::"r"(bar), "h"((unsigned short)3) : "memory");
}
// box into this CTA's shared memory, bytes counted by a barrier of the pair's even CTA
__device__ __forceinline__ void pair_tma_2d(unsigned dst, const CUtensorMap* map, int x, int y, unsigned bar) {
    asm volatile("cp.async.bulk.tensor.2d.cta_group::2.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3}], [%4];\n"
                 ::"r"(dst), "l"(map), "r"(x), "r"(y), "r"(bar) : "memory");
}
__device__ __forceinline__ unsigned cluster_addr(unsigned local, unsigned rank) {
    unsigned r;
    asm volatile("mapa.shared::cluster.u32 %0, %1, %2;\n" : "=r"(r) : "r"(local), "r"(rank));
    return r;
}
// Arrival on a barrier of the pair's other CTA.  What it announces is that tensor memory has been read (tcgen05.wait::ld came
// before); no global write has to be visible for that, and a release at cluster scope would wait for all of them.
__device__ __forceinline__ void mbar_arrive_cluster(unsigned bar) {
    asm volatile("mbarrier.arrive.shared::cluster.b64 _, [%0];\n" ::"r"(bar) : "memory");
}
// 32 lanes x 32 consecutive columns of tensor memory -> 32 registers (lane = row of the accumulator); valid after tmem_wait
__device__ __forceinline__ void tmem_ld32(unsigned taddr, float (&v)[32]) {
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x32.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16, %17, %18, %19, %20, %21, %22, "
        "%23, %24, %25, %26, %27, %28, %29, %30, %31}, [%32];\n"
        : "=f"(v[0]), "=f"(v[1]), "=f"(v[2]), "=f"(v[3]), "=f"(v[4]), "=f"(v[5]), "=f"(v[6]), "=f"(v[7]), "=f"(v[8]), "=f"(v[9]), "=f"(v[10]), "=f"(v[11]),
          "=f"(v[12]), "=f"(v[13]), "=f"(v[14]), "=f"(v[15]), "=f"(v[16]), "=f"(v[17]), "=f"(v[18]), "=f"(v[19]), "=f"(v[20]), "=f"(v[21]), "=f"(v[22]),
          "=f"(v[23]), "=f"(v[24]), "=f"(v[25]), "=f"(v[26]), "=f"(v[27]), "=f"(v[28]), "=f"(v[29]), "=f"(v[30]), "=f"(v[31])
        : "r"(taddr) : "memory");
}
// the loaded registers pass through the wait, so that nothing that uses them can be scheduled before it
__device__ __forceinline__ void tmem_wait(float (&v)[32]) {
    asm volatile("tcgen05.wait::ld.sync.aligned;\n"
                 : "+f"(v[0]), "+f"(v[1]), "+f"(v[2]), "+f"(v[3]), "+f"(v[4]), "+f"(v[5]), "+f"(v[6]), "+f"(v[7]), "+f"(v[8]), "+f"(v[9]), "+f"(v[10]), "+f"(v[11]),
                   "+f"(v[12]), "+f"(v[13]), "+f"(v[14]), "+f"(v[15]), "+f"(v[16]), "+f"(v[17]), "+f"(v[18]), "+f"(v[19]), "+f"(v[20]), "+f"(v[21]), "+f"(v[22]),
                   "+f"(v[23]), "+f"(v[24]), "+f"(v[25]), "+f"(v[26]), "+f"(v[27]), "+f"(v[28]), "+f"(v[29]), "+f"(v[30]), "+f"(v[31])
                 :: "memory");
}
// One lane of a converged warp, the same one every time.  The warps that issue TMA loads and MMAs run their loops with all lanes and
// enter only the issue itself with one: descriptors and addresses then stay in uniform registers, which takes an MMA
// from 75 to 41 cycles of issue (a loop inside `if (lane == 0)` moves each operand to a uniform register every time).
__device__ __forceinline__ bool elect_one() {
    unsigned one;
    asm volatile("{\n.reg .pred p;\nelect.sync _|p, 0xffffffff;\nselp.u32 %0, 1, 0, p;\n}\n" : "=r"(one));
    return one != 0;
}
// Wait of such a warp: a test that has usually succeeded, else polling; all lanes agree on `dead`.
__device__ __forceinline__ void mbar_wait_all(unsigned bar, unsigned parity, int* flags, bool& dead) {
    if (!__all_sync(0xffffffffu, mbar_test(bar, parity))) {
        mbar_wait(bar, parity, flags, dead);
        dead = __any_sync(0xffffffffu, dead);
    }
}
__device__ __forceinline__ void tile_origin(const TileProblem& p, int tile, int& m0, int& n0) {
    const int g = tile / p.by_group, in = tile - g * (p.gm * p.nt);
    const bool rest = (g + 1) * p.gm > p.mt;
    const int rows = rest ? p.mt - g * p.gm : p.gm;
    const int n = in / (rest ? p.by_rest : p.by_gm);
    m0 = (g * p.gm + in - n * rows) * TG_BM;
    n0 = n * p.bn;
}
struct TileUnit { int which, m0, n0, kb0, kb1, piece; };   // which: product; piece: index of the partial tile, -1 for a whole tile
// The j-th unit of a pair; false: it has no more.
__device__ __forceinline__ bool tile_unit(const TileArgs& a, int j, TileUnit& w) {
    const int pair = blockIdx.x >> 1, pairs = gridDim.x >> 1;
    int u;
    const int mine = a.first_q + (pair < a.first_r ? 1 : 0);
    if (j < mine) {
        w.which = 0;
        u = pair + j * pairs;
    } else {
        j -= mine;
        w.which = 1;
        const int free_pairs = pairs - a.first_r;
        if (pair >= a.first_r && j < a.extra) u = j * free_pairs + pair - a.first_r;
        else u = a.extra * free_pairs + (j - (pair >= a.first_r ? a.extra : 0)) * pairs + pair;
        if (u >= a.p[1].units) return false;
    }
    const TileProblem& p = a.p[w.which];
    int tile = u;
    w.kb0 = 0;
    w.kb1 = p.kb;
    w.piece = -1;
    if (u >= p.full && p.parts) {
        // all tiles' first pieces, then all second pieces: pairs at work together read the same range of k and share operands in L2
        w.piece = u - p.full;
        const int s = w.piece / p.by_tail;
        tile = p.full + w.piece - s * p.tail;
        w.kb0 = s * p.kbps;
        w.kb1 = min(p.kb, w.kb0 + p.kbps);
    }
    tile_origin(p, tile, w.m0, w.n0);
    return true;
}

// Half a staging buffer holds 32 rows of four 16-byte units; unit j of row r lies where neither side meets a bank twice.
__device__ __forceinline__ int staged(int r, int j) { return r * 4 + (j ^ ((r >> 1) & 3)); }

// A 32 x 32 block of C, a row per lane -> rows through the warp's staging buffer -> out (+ addend, * scale).
// Row-per-lane stores would touch 32 lines per instruction.
__device__ __forceinline__ void emit_block(const TileProblem& a, uint4* xb, float (&v)[32], int row0, int col0, const float* addend, long long lda, float scale) {
    const int lane = threadIdx.x & 31, lrow = lane >> 2, lch = lane & 3;        // row-contiguous phase: row within a group of 8, unit
    const int rows = a.M - row0;
    // the last columns, or rows without alignment: a column per lane, a row per store (the block of 1001 x 771 float32: 7400 cycles with two half
    // rows per store and the row's address formed each time, 3000 so; an aligned one of bfloat16 1050)
    if (!a.vec || col0 + 32 > a.N) {
#pragma unroll
        for (int j = 0; j < 8; ++j)
            xb[lane * 8 + (j ^ (lane & 7))] = make_uint4(__float_as_uint(v[4 * j]), __float_as_uint(v[4 * j + 1]), __float_as_uint(v[4 * j + 2]), __float_as_uint(v[4 * j + 3]));
        __syncwarp();
        const float* xf = reinterpret_cast<const float*>(xb) + (lane & 3);
        const int top = min(rows, 32);
        const long long ldo = a.ldo;
        const size_t at = (size_t)row0 * ldo + col0 + lane;
        const float* y = addend ? addend + (size_t)row0 * lda + col0 + lane : nullptr;
        if (col0 + lane < a.N) {
            if (a.out_f32) {
                float* out = (float*)a.out + at;
#pragma unroll 8
                for (int r = 0; r < top; ++r) out[r * ldo] = (xf[(r * 8 + ((lane >> 2) ^ (r & 7))) * 4] + (y ? y[r * lda] : 0.f)) * scale;
            } else {
                __nv_bfloat16* out = (__nv_bfloat16*)a.out + at;
#pragma unroll 8
                for (int r = 0; r < top; ++r) out[r * ldo] = __float2bfloat16_rn((xf[(r * 8 + ((lane >> 2) ^ (r & 7))) * 4] + (y ? y[r * lda] : 0.f)) * scale);
            }
        }
        __syncwarp();
        return;
    }
    if (!a.out_f32 && !addend) {                                                // 32 columns of bfloat16
#pragma unroll
        for (int j = 0; j < 4; ++j)
            xb[staged(lane, j)] = make_uint4(pack_bf16(v[8 * j] * scale, v[8 * j + 1] * scale), pack_bf16(v[8 * j + 2] * scale, v[8 * j + 3] * scale),
                                             pack_bf16(v[8 * j + 4] * scale, v[8 * j + 5] * scale), pack_bf16(v[8 * j + 6] * scale, v[8 * j + 7] * scale));
        __syncwarp();
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int br = 8 * i + lrow;
            if (br < rows) *reinterpret_cast<uint4*>((__nv_bfloat16*)a.out + (size_t)(row0 + br) * a.ldo + col0 + 8 * lch) = xb[staged(br, lch)];
        }
        __syncwarp();
        return;
    }
#pragma unroll
    for (int h = 0; h < 2; ++h) {                                               // 16 columns of float32 at a time
        const int col1 = col0 + 16 * h;
        float4 y[4];
        if (addend) {
#pragma unroll
            for (int i = 0; i < 4; ++i)
                if (8 * i + lrow < rows) y[i] = *reinterpret_cast<const float4*>(addend + (size_t)(row0 + 8 * i + lrow) * lda + col1 + 4 * lch);
        }
#pragma unroll
        for (int j = 0; j < 4; ++j)
            xb[staged(lane, j)] = make_uint4(__float_as_uint(v[16 * h + 4 * j]), __float_as_uint(v[16 * h + 4 * j + 1]), __float_as_uint(v[16 * h + 4 * j + 2]),
                                             __float_as_uint(v[16 * h + 4 * j + 3]));
        __syncwarp();
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int br = 8 * i + lrow, row = row0 + br;
            const uint4 u = xb[staged(br, lch)];
            float4 x = make_float4(__uint_as_float(u.x), __uint_as_float(u.y), __uint_as_float(u.z), __uint_as_float(u.w));
            if (br < rows) {
                if (addend) { x.x += y[i].x; x.y += y[i].y; x.z += y[i].z; x.w += y[i].w; }
                x.x *= scale; x.y *= scale; x.z *= scale; x.w *= scale;
                if (a.out_f32) *reinterpret_cast<float4*>((float*)a.out + (size_t)row * a.ldo + col1 + 4 * lch) = x;
                else *reinterpret_cast<uint2*>((__nv_bfloat16*)a.out + (size_t)row * a.ldo + col1 + 4 * lch) = make_uint2(pack_bf16(x.x, x.y), pack_bf16(x.z, x.w));
            }
        }
        __syncwarp();
    }
}

constexpr float XE_STEPS = 1024.f;            // steps per factor of two in the stored exponents
constexpr unsigned XE_NONE = 65535u;

// EPI_STORE: one or two products whose B is MN-major, A either.  The others: one product of K-major operands.
template <int EPI>
__global__ void __cluster_dims__(2, 1, 1) __launch_bounds__(TG_THREADS, 1)
k_tile(const __grid_constant__ CUtensorMap tmA0, const __grid_constant__ CUtensorMap tmB0, const __grid_constant__ CUtensorMap tmA1, const __grid_constant__ CUtensorMap tmB1,
       const __grid_constant__ TileArgs a) {
    constexpr bool BMN = EPI == EPI_STORE, TEACH = EPI == EPI_TEACH_LOSS || EPI == EPI_TEACH, LOSS_ONLY = EPI == EPI_LOSS || EPI == EPI_TEACH_LOSS;
    extern __shared__ __align__(16) unsigned char tg_smem_raw[];
    // the offset of everything in shared memory is the same in both CTAs of the pair (descriptors and commits rely on it)
    unsigned char* base = reinterpret_cast<unsigned char*>((reinterpret_cast<uintptr_t>(tg_smem_raw) + 1023) & ~(uintptr_t)1023);
    unsigned char* staging = base + (size_t)TG_STAGES * TG_STAGE_BYTES;
    unsigned long long* bars = reinterpret_cast<unsigned long long*>(staging + TG_EPI_WARPS * TG_STAGING);
    const unsigned bar_full = smem_u32(bars), bar_empty = bar_full + 8 * TG_STAGES;
    const unsigned bar_accf = bar_empty + 8 * TG_STAGES, bar_acce = bar_accf + 16;
    unsigned* tmem_slot = reinterpret_cast<unsigned*>(bars + 2 * TG_STAGES + 4);
    const unsigned smem_base = smem_u32(base);

    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const int rank = blockIdx.x & 1;

    if (tid == 0) {
        for (int s = 0; s < TG_STAGES; ++s) { mbar_init(bar_full + 8 * s, 1); mbar_init(bar_empty + 8 * s, 1); }
        for (int b = 0; b < 2; ++b) { mbar_init(bar_accf + 8 * b, 1); mbar_init(bar_acce + 8 * b, 2 * TG_EPI_WARPS); }
        asm volatile("fence.mbarrier_init.release.cluster;\n" ::: "memory");
    }
    if (warp == 1) {
        asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], 512;\n" ::"r"(smem_u32(tmem_slot)) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;\n" ::: "memory");
    }
    const bool short_a = !BMN && (a.a_rows < 128 || !a.a_odd);
    if (short_a) {
        for (int i = tid; i < TG_STAGES * (TG_HALF_BYTES / 16); i += TG_THREADS)
            *reinterpret_cast<uint4*>(base + (size_t)(i / (TG_HALF_BYTES / 16)) * TG_STAGE_BYTES + (i % (TG_HALF_BYTES / 16)) * 16) = make_uint4(0u, 0u, 0u, 0u);
        asm volatile("fence.proxy.async.shared::cta;\n" ::: "memory");
    }
    asm volatile("tcgen05.fence::before_thread_sync;\n" ::: "memory");
    __syncthreads();
    cluster_arrive_release();
    cluster_wait_acquire();
    asm volatile("tcgen05.fence::after_thread_sync;\n" ::: "memory");
    const unsigned tmem = *tmem_slot;
    bool dead = false;
    grid_trigger();
    // TEACH: the kernel before this one orders a list that only the epilogue reads, and it lets this one start after its own wait, when everything before it is
    // done: the loads of the operands and the products need not wait for it (one token against 32000 x 768: 22.3 -> 20.7 us)
    if (!TEACH || warp >= 2) grid_wait();
    if (EPI != EPI_STORE && blockIdx.x == 0 && tid == 0 && a.done) *a.done = 0;

    if (warp == 0) {
        // ---- TMA producer of this CTA: its 128 rows of A and its half of B ----
        const unsigned full0 = cluster_addr(bar_full, 0);
        int s = 0, filled = 0;
        unsigned par = 1;                                      // a fresh barrier counts as released
        TileUnit w;
        for (int j = 0; !dead && tile_unit(a, j, w); ++j) {
            const TileProblem& p = a.p[w.which];
            const CUtensorMap* const ma = w.which ? &tmA1 : &tmA0;
            const CUtensorMap* const mb = w.which ? &tmB1 : &tmB0;
            const bool amn = BMN && p.a_mn, two = p.bn > 128;
            // bytes of B per stage: K-major boxes have bn / 2 rows, MN-major ones come in blocks of 64
            const unsigned a_bytes = BMN ? 2 * TG_HALF_BYTES : (unsigned)(a.a_rows * TG_BK * 2) << a.a_odd;       // of both CTAs
            const unsigned b_bytes = BMN ? (two ? TG_HALF_BYTES : TG_HALF_BYTES / 2) : (unsigned)p.bn / 2 * TG_BK * 2;
            const int nh = (min(p.bn, p.N - w.n0) + 31) / 32 * 16;
            const int m = w.m0 + rank * 128, n = w.n0 + rank * nh;
            for (int kb = w.kb0; kb < w.kb1; ++kb) {
                mbar_wait_all(bar_empty + 8 * s, par, a.status, dead);
                if (dead) break;
                if (elect_one()) {
                    const unsigned bar = full0 + 8 * s;
                    if (rank == 0) mbar_expect_tx(bar_full + 8 * s, a_bytes + 2 * b_bytes);
                    const unsigned da = smem_base + s * TG_STAGE_BYTES, db = da + TG_HALF_BYTES;
                    const int k = kb * TG_BK;
                    if (amn) {
                        pair_tma_2d(da, ma, m, k, bar);
                        pair_tma_2d(da + TG_HALF_BYTES / 2, ma, m + 64, k, bar);
                    } else if (BMN || rank == 0 || a.a_odd) {
                        pair_tma_2d(da, ma, k, m, bar);
                    }
                    if (BMN) {
                        pair_tma_2d(db, mb, n, k, bar);
                        if (two) pair_tma_2d(db + TG_HALF_BYTES / 2, mb, n + 64, k, bar);
                    } else {
                        pair_tma_2d(db, mb, k, n, bar);
                    }
                }
                __syncwarp();
                if (++s == TG_STAGES) { s = 0; par ^= 1; }
                if (filled < TG_STAGES) ++filled;
            }
        }
        // every copy has landed and every release has arrived here before the CTA may go
        if (filled < TG_STAGES) { s = 0; par = 0; }
        for (int i = 0; i < filled && !dead; ++i) {
            mbar_wait_all(bar_empty + 8 * s, par, a.status, dead);
            if (++s == TG_STAGES) { s = 0; par ^= 1; }
        }
        if (dead)
            for (int i = 0; i < 200; ++i) __nanosleep(1000);   // copies in flight land
    } else if (warp == 1) {
        // ---- MMA issuer (even CTA) ----
        if (rank == 0) {
            int s = 0, it = 0;
            unsigned par = 0;
            TileUnit w;
            for (int j = 0; !dead && tile_unit(a, j, w); ++j) {
                const TileProblem& p = a.p[w.which];
                const bool amn = BMN && p.a_mn;
                const unsigned idesc = tile_idesc((min(p.bn, p.N - w.n0) + 31) / 32 * 32, amn, BMN);
                const unsigned step_a = amn ? 2048 >> 4 : 32 >> 4, step_b = BMN ? 2048 >> 4 : 32 >> 4;   // 16 of k: two groups of 8 rows, or 32 bytes of a row
                for (int k0 = w.kb0; k0 < w.kb1 && !dead; ++it) {
                    const int k1 = p.kacc > 0 ? min(w.kb1, k0 + p.kacc) : w.kb1;
                    const unsigned d = tmem + (unsigned)((it & 1) * TG_BN);
                    if (it >= 2) {
                        mbar_wait_all(bar_acce + 8 * (it & 1), (unsigned)(((it >> 1) - 1) & 1), a.status, dead);
                        asm volatile("tcgen05.fence::after_thread_sync;\n" ::: "memory");
                    }
                    for (int kb = k0; kb < k1; ++kb) {
                        mbar_wait_all(bar_full + 8 * s, par, a.status, dead);
                        if (dead) break;
                        const unsigned sa = smem_base + s * TG_STAGE_BYTES;
                        const unsigned long long da = tile_desc(sa, amn), db = tile_desc(sa + TG_HALF_BYTES, BMN);
                        if (elect_one()) {
#pragma unroll
                            for (int k = 0; k < TG_BK / 16; ++k)
                                pair_mma(d, da + (unsigned long long)(k * step_a), db + (unsigned long long)(k * step_b), idesc, (kb > k0 || k > 0) ? 1u : 0u);
                            pair_commit(bar_empty + 8 * s);
                            if (kb == k1 - 1) pair_commit(bar_accf + 8 * (it & 1));
                        }
                        __syncwarp();
                        if (++s == TG_STAGES) { s = 0; par ^= 1; }
                    }
                    k0 = k1;
                }
            }
        } else if (!BMN && !LOSS_ONLY && blockIdx.x == 1 && a.norm) {
            if (TEACH) grid_wait();
            double z = 0.0;
            constexpr int UN = 8;
            for (long long i0 = lane; i0 < a.norm_rows; i0 += 32 * UN) {
                long long label[UN];
                float wt[UN];
#pragma unroll
                for (int j = 0; j < UN; ++j) {                 // no branch around the loads: all under way together
                    const long long i = min(i0 + 32 * j, a.norm_rows - 1);
                    label[j] = a.norm_labels[i];
                    wt[j] = a.norm_weight ? a.norm_weight[i] : 1.f;
                }
#pragma unroll
                for (int j = 0; j < UN; ++j) {
                    const bool counts = label[j] >= 0 && label[j] < a.p[0].N && label[j] != a.ignore && i0 + 32 * j < a.norm_rows;
                    z += counts ? (double)wt[j] : 0.0;
                }
            }
#pragma unroll
            for (int o = 16; o; o >>= 1) z += __shfl_xor_sync(0xffffffffu, z, o);
            if (lane == 0) *a.norm = z != 0.0 ? (float)((TEACH ? (double)a.temperature : 1.0) / z) : 0.f;
        }
    } else {
        // ---- epilogue: two warps per quarter of the rows, which share the columns ----
        const int quarter = warp & 3;                          // the tensor-memory lanes this warp may read
        const int share = (warp - 2) >> 2;
        const unsigned lane_base = tmem + ((unsigned)(quarter * 32) << 16);
        uint4* xb = reinterpret_cast<uint4*>(staging + (size_t)(warp - 2) * TG_STAGING);
        const unsigned acce0 = cluster_addr(bar_acce, 0);
        int it = 0;
        if (EPI == EPI_STORE) {
            TileUnit w;
            for (int j = 0; tile_unit(a, j, w); ++j) {
                const TileProblem& p = a.p[w.which];
                const float scale = p.scale ? *p.scale : 1.f;
                const int row0 = w.m0 + rank * 128 + quarter * 32;
                const int chunks = row0 < p.M ? (min(p.bn, p.N - w.n0) + 31) / 32 : 0;      // blocks of 32 columns that exist
                // partial tiles: lanes of a warp (rows) side by side
                float* part = w.piece >= 0 ? p.part + ((size_t)w.piece * 2 + rank) * (TG_PART / 2) + quarter * 32 + lane : nullptr;
                for (int k0 = w.kb0; k0 < w.kb1; ++it) {
                    const int k1 = p.kacc > 0 ? min(w.kb1, k0 + p.kacc) : w.kb1;
                    mbar_wait_warp(bar_accf + 8 * (it & 1), (unsigned)((it >> 1) & 1), a.status, dead);
                    asm volatile("tcgen05.fence::after_thread_sync;\n" ::: "memory");
                    if (share >= chunks && lane == 0) mbar_arrive_cluster(acce0 + 8 * (it & 1));
#pragma unroll 1
                    for (int c = share; c < chunks; c += TG_EPI_WARPS / 4) {
                        float v[32];
                        tmem_ld32(lane_base + (unsigned)((it & 1) * TG_BN + 32 * c), v);
                        tmem_wait(v);
                        if (c + TG_EPI_WARPS / 4 >= chunks) {  // this warp's last read: the accumulator is free
                            asm volatile("tcgen05.fence::before_thread_sync;\n" ::: "memory");
                            __syncwarp();
                            if (lane == 0) mbar_arrive_cluster(acce0 + 8 * (it & 1));
                        }
                        const bool more = k0 > w.kb0;          // the sum so far lies where this one goes
                        if (part) {
                            float* q = part + (size_t)(32 * c) * 128;
                            if (more) {
#pragma unroll
                                for (int i = 0; i < 32; ++i) v[i] += q[i * 128];
                            }
#pragma unroll
                            for (int i = 0; i < 32; ++i) q[i * 128] = dead ? NAN : v[i];
                        } else {
                            emit_block(p, xb, v, row0, w.n0 + 32 * c, more ? (const float*)p.out : p.addend, more ? p.ldo : (long long)p.N, dead ? NAN : scale);
                        }
                    }
                    k0 = k1;
                }
            }
        } else {
            // ---- softmax statistics of this warp's 128 columns, and the exponents in 16 bits ----
            // 64 columns at a time, each read from tensor memory once: those reads take the MMAs' bandwidth to it (two passes, maximum first,
            // cost 900 of the 9400 cycles of a 256 x 256 x 768 tile)
            const int lrow = lane >> 3, lch = lane & 7;        // row-contiguous phase: row within a group of 4, 16-byte unit
            const TileProblem& p = a.p[0];
            auto label_of = [&](const TileUnit& w) {           // the row's label, -1 where there is no row
                const int row = w.m0 + rank * 128 + quarter * 32 + lane;
                return row < p.M ? a.labels[row] : -1ll;
            };
            // where the entries of this warp's four blocks begin (lanes 0-3) and end (lane 4): asked for a tile ahead, the first 32 entries with the tile
            auto bin_of = [&](const TileUnit& w) {
                const int row = w.m0 + rank * 128 + quarter * 32, col = w.n0 + share * 128;
                return row < p.M && col < p.N && lane < 5 ? a.bins[(size_t)(row >> 5) * (a.nbins + 1) + min((col >> 5) + lane, a.nbins)] : 0;
            };
            const float log2e = TEACH ? a.log2e : LOG2E;
            TileUnit next;
            bool going = tile_unit(a, 0, next);
            long long next_label = !TEACH && going ? label_of(next) : -1ll;
            int next_bin = TEACH && going ? bin_of(next) : 0;
            for (; going; ++it) {
                const TileUnit w = next;
                const int row0 = w.m0 + rank * 128 + quarter * 32, col_base = w.n0 + share * 128, row = row0 + lane;
                const int b = it & 1;
                const int label_col = (int)min(max(next_label - (long long)col_base, -1ll), 128ll);   // among this warp's columns
                const int bin = next_bin;
                const unsigned* listed = a.entries + (size_t)(row0 >> 5) * 32 * a.K;
                int held = 0;                                  // the place of `entry` among its rows' entries
                unsigned entry = 0u;
                if constexpr (TEACH) {
                    held = __shfl_sync(0xffffffffu, bin, 0) + lane;
                    if (held < __shfl_sync(0xffffffffu, bin, 4)) entry = listed[held];
                }
                going = tile_unit(a, it + 1, next);
                if (!TEACH && going) next_label = label_of(next);        // asked for a tile ahead
                if (TEACH && going) next_bin = bin_of(next);
                mbar_wait_warp(bar_accf + 8 * b, (unsigned)((it >> 1) & 1), a.status, dead);
                asm volatile("tcgen05.fence::after_thread_sync;\n" ::: "memory");
                const unsigned taddr = lane_base + (unsigned)(b * TG_BN + share * 128);
                const int ncols = row0 < p.M ? min(128, p.N - col_base) : 0;       // (<= 0: none of these columns exists, or none of the rows)
                float last_top = -INFINITY, last_sum = 0.f;    // loss only: of the first 64 columns
#pragma unroll
                for (int c = 0; c < 128 / XE_SEG; ++c) {
                    const int left = ncols - XE_SEG * c;
                    if (left <= 0) break;
                    float v[2][32];
                    tmem_ld32(taddr + XE_SEG * c, v[0]);
                    tmem_ld32(taddr + XE_SEG * c + 32, v[1]);
                    tmem_wait(v[0]);
                    tmem_wait(v[1]);
                    if (left <= XE_SEG || c == 128 / XE_SEG - 1) {                 // the last read: the accumulator is free
                        asm volatile("tcgen05.fence::before_thread_sync;\n" ::: "memory");
                        __syncwarp();
                        if (lane == 0) mbar_arrive_cluster(acce0 + 8 * b);
                    }
                    if (left < XE_SEG) {
#pragma unroll
                        for (int j = 0; j < XE_SEG; ++j) if (j >= left) v[j >> 5][j & 31] = -INFINITY;
                    }
                    if constexpr (TEACH) {
                        // 32 columns at a time through shared memory, where any entry lies among them: a lane per entry fetches its row's
#pragma unroll
                        for (int h = 0; h < 2; ++h) {
                            const int lo = __shfl_sync(0xffffffffu, bin, 2 * c + h), hi = __shfl_sync(0xffffffffu, bin, 2 * c + h + 1);
                            if (lo == hi) continue;
#pragma unroll
                            for (int j = 0; j < 8; ++j)
                                xb[lane * 8 + (j ^ (lane & 7))] = make_uint4(__float_as_uint(v[h][4 * j]), __float_as_uint(v[h][4 * j + 1]), __float_as_uint(v[h][4 * j + 2]),
                                                                             __float_as_uint(v[h][4 * j + 3]));
                            __syncwarp();
                            const auto fetch = [&](unsigned e) {
                                const int r = e >> 5 & 31u, col = e & 31u;
                                a.entry_logit[(size_t)(row0 + r) * a.K + (e >> 10)] = reinterpret_cast<const float*>(xb)[(r * 8 + ((col >> 2) ^ (r & 7))) * 4 + (col & 3)];
                            };
                            if (held >= lo && held < hi) fetch(entry);
                            for (int e0 = max(lo + lane, held + 32); e0 < hi; e0 += 4 * 32) {      // (the places of a lane are 32 apart) more than a warp holds: four at a time
                                unsigned e[4];
#pragma unroll
                                for (int j = 0; j < 4; ++j) e[j] = e0 + 32 * j < hi ? listed[e0 + 32 * j] : 0u;
#pragma unroll
                                for (int j = 0; j < 4; ++j)
                                    if (e0 + 32 * j < hi) fetch(e[j]);
                            }
                            __syncwarp();
                        }
                    } else if (__any_sync(0xffffffffu, (label_col >> 6) == c)) {
#pragma unroll
                        for (int j = 0; j < XE_SEG; ++j) if (label_col == XE_SEG * c + j) a.label_logit[row] = v[j >> 5][j & 31];
                    }
                    float t[4] = {LOSS_ONLY ? last_top : -INFINITY, -INFINITY, -INFINITY, -INFINITY};
#pragma unroll
                    for (int j = 0; j < XE_SEG; ++j) t[j & 3] = fmaxf(t[j & 3], v[j >> 5][j & 31]);
                    const float top = fmaxf(fmaxf(t[0], t[1]), fmaxf(t[2], t[3]));
                    const float ref = top == -INFINITY ? 0.f : top;                // nothing but -inf: exp(-inf - 0) = 0
                    // eight at a time, so that the small terms meet before they meet the maximum's 1: it takes part in at most seven additions
                    float part[4];
                    unsigned pk[XE_SEG / 2];
#pragma unroll
                    for (int j = 0; j < XE_SEG; j += 8) {
                        float e[8];
#pragma unroll
                        for (int i = 0; i < 8; i += 2) {
                            const float t0 = (v[j >> 5][(j & 31) + i] - ref) * log2e, t1 = (v[j >> 5][(j & 31) + i + 1] - ref) * log2e;     // <= 0
                            e[i] = ex2(t0);
                            e[i + 1] = ex2(t1);
                            if (!LOSS_ONLY) {
                                const float q0 = fminf(fmaf(t0, -XE_STEPS, XE_MAGIC), XE_MAGIC + 65535.f);
                                const float q1 = fminf(fmaf(t1, -XE_STEPS, XE_MAGIC), XE_MAGIC + 65535.f);
                                pk[(j + i) / 2] = __byte_perm(__float_as_uint(q0), __float_as_uint(q1), 0x5410);
                            }
                        }
                        const float eight = ((e[0] + e[1]) + (e[2] + e[3])) + ((e[4] + e[5]) + (e[6] + e[7]));
                        part[j / 8 & 3] = j < 32 ? eight : part[j / 8 & 3] + eight;
                    }
                    float sum = (part[0] + part[1]) + (part[2] + part[3]);
                    if (LOSS_ONLY) sum = fmaf(last_sum, ex2((last_top - ref) * log2e), sum);
                    if (dead) sum = NAN;
                    if (LOSS_ONLY) {
                        last_top = top;
                        last_sum = sum;
                    } else {
                        if (row < p.M) a.stats[(size_t)row * a.nseg + (col_base + XE_SEG * c) / XE_SEG] = make_float2(top, sum);
#pragma unroll
                        for (int j = 0; j < 8; ++j) xb[lane * 8 + (j ^ (lane & 7))] = make_uint4(pk[4 * j], pk[4 * j + 1], pk[4 * j + 2], pk[4 * j + 3]);
                        __syncwarp();
#pragma unroll
                        for (int i = 0; i < 8; ++i) {
                            const int br = 4 * i + lrow;
                            if (row0 + br < p.M)               // rows of q are padded to whole segments
                                *reinterpret_cast<uint4*>(a.q + (size_t)(row0 + br) * a.ldq + col_base + XE_SEG * c + 8 * lch) = xb[br * 8 + (lch ^ (br & 7))];
                        }
                        __syncwarp();
                    }
                }
                if (LOSS_ONLY && ncols > 0 && row < p.M) a.stats[(size_t)row * a.nseg + col_base / XE_SEG_LOSS] = make_float2(last_top, last_sum);
                if (ncols <= 0 && lane == 0) mbar_arrive_cluster(acce0 + 8 * b);
            }
        }
    }
    asm volatile("tcgen05.fence::before_thread_sync;\n" ::: "memory");
    __syncthreads();
    cluster_arrive_release();
    cluster_wait_acquire();
    if (warp == 1) {
        asm volatile("tcgen05.fence::after_thread_sync;\n" ::: "memory");
        asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, 512;\n" ::"r"(tmem) : "memory");
    }
}

// Adds the pieces of the split tiles of both products: blockIdx.x = tail tile, .y = 32 columns of it, .z = 32 rows.  Each of four warps adds 8 of the
// columns, a row per lane, eight pieces under way at a time; each then writes 8 of the rows.
__global__ void __launch_bounds__(128) k_join(const __grid_constant__ TileArgs a) {
    __shared__ float xs[32][33];
    grid_trigger();
    grid_wait();
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int first = a.p[0].parts ? a.p[0].tail : 0;
    const int which = (int)blockIdx.x < first ? 0 : 1, tile = blockIdx.x - (which ? first : 0);
    const TileProblem& p = a.p[which];
    int m0, n0;
    tile_origin(p, p.full + tile, m0, n0);
    const int c0 = 32 * blockIdx.y, row0 = m0 + blockIdx.z * 32;
    if (c0 >= p.bn || n0 + c0 >= p.N || row0 >= p.M) return;
    const float* q = p.part + ((size_t)tile * 2 + (blockIdx.z >> 2)) * (TG_PART / 2) + (size_t)(c0 + 8 * warp) * 128 + (blockIdx.z & 3) * 32 + lane;
    const size_t step = (size_t)p.tail * TG_PART;
    float v[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
    if (n0 + c0 + 8 * warp < p.N) {
#pragma unroll 8
        for (int s = 0; s < p.S; ++s)
#pragma unroll
            for (int j = 0; j < 8; ++j) v[j] += q[(size_t)s * step + j * 128];
    }
#pragma unroll
    for (int j = 0; j < 8; ++j) xs[lane][8 * warp + j] = v[j];
    __syncthreads();
    const float scale = p.scale ? *p.scale : 1.f;
    const int col = n0 + c0 + lane;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const int row = row0 + 8 * warp + i;
        if (row < p.M && col < p.N) {
            const float x = (xs[8 * warp + i][lane] + (p.addend ? p.addend[(size_t)row * p.N + col] : 0.f)) * scale;
            if (p.out_f32) ((float*)p.out)[(size_t)row * p.ldo + col] = x;
            else ((__nv_bfloat16*)p.out)[(size_t)row * p.ldo + col] = __float2bfloat16_rn(x);
        }
    }
}

}  // namespace psgd
