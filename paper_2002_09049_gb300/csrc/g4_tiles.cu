// Linear layer of weights in 4-bit integers for more than a few tokens (mpq_g4_linear), on tcgen05 MMAs.
//
// 128 channels of weights, s (q - z) rounded to x's type, are the MMA's A (the accumulator's lanes), up to 256
// tokens its B (columns).  Packed weights come by TMA as they lie in memory (a ring of their own, tiles
// ahead), and groups of four warps turn them by turns into operands in tensor memory, a channel to a
// lane; x comes by TMA into 128-byte-swizzled shared memory.  (Operands in shared memory too, 141 us
// for 2,048 x 11,008 x 4,096: 64 KB in and out per 64 elements of K of a pair's CTA are 512 cycles at 128 bytes each,
// as many as the MMAs take.)  Eight warps write the outputs.  Roles run over their CTA's tiles without a pause.
//
// PAIRS: CTA pairs (cta_group::2) take 256 channels x 256 tokens, each CTA its own channels and half of the tokens'
// operand.  WIDE, NARROW: a CTA's 128 channels x up to 256 or 128 tokens; K may be split over the CTAs of a cluster,
// whose sums are joined in shared memory in the order of the ranks (equal inputs give equal bits).  NARROW: two
// warps issue the MMAs of every other stage, into accumulators of their own whose sums are added on the way out (one
// warp's waits and issue took 800 cycles a stage, 340 of them the MMAs').
//
// EXACT: no weight is rounded.  s (q - z) has 12 significant bits, so it is a term of bf16 and what that leaves, a second
// one: all of K goes by twice, once for either term, into the same sums.  fp16 holds 11 bits, all there are without
// zero points, but not every size: a channel's scales are taken times a power of two that brings the largest of them (of
// the CTA's share of K) to 2^11 or more, and its sums divided by it.  A scale of 2^-28 of that largest one or more is
// held as it is, a smaller one to 2^-36 of it.
//
// Measured, beside the rounded values': 2,048 x 11,008 x 4,096 bf16 191 us (102), fp16 without zero points 110 (104), with
// them 200 (105); 256 x 11,008 x 4,096 bf16 41.8 (24.4); 75 x 4,096 x 11,008 bf16 23.8 (14.3: its makers make both terms,
// 14.8 M warp instructions for 7.4).  fp16's powers spill 7 words in the pairs' form.
//
// Measured: 2,048 x 11,008 x 4,096 (T x C x d) 102 us, 1.81 PFLOP/s: a stage takes 1,024 cycles, its MMAs' own; 1,800 a
// tile between the last MMA and the next one's first; 344 tiles on 76 pairs are five rounds.  75 x 4,096 x 11,008 14.3
// us (weights from memory 15.0): 2 to the first MMA, 22 stages of 0.35 on 128 CTAs (1,700 warp instructions a stage to make its operands), 3 for
// the join of four ranks; without any of the work, roles waiting on each other alone, 10.3.
//
// Warps: 0 copies x, 1 issues MMAs (the even CTA's, of a pair; NARROW: 3 too), 2 copies weights, PAIRS: 3 tells the MMAs'
// warp that x has landed, 4 .. make operands, the last eight write outputs (these two by lane quarters, warp % 4).
// Every wait is bounded.
#include <cuda.h>
#include <math.h>
#include <string.h>

#include <algorithm>
#include <type_traits>

#include "g4.cuh"
#include "pair_common.cuh"
#include "sm100.cuh"
#include "token_tiles.cuh"
#include "waits.cuh"

MPQ_CHECKED_UNIT("g4_tiles.cu");

namespace mpq {
namespace {

using namespace sm100;

constexpr int H_M = TOKEN_M;             // channels of a CTA's tile
constexpr int H_K = 128;                 // elements of K in a stage: a packed tile's
constexpr int H_A_COLS = H_K / 2;        // TMEM columns of a stage's weights, two elements each
constexpr int H_MAX_STAGES = 8;
constexpr int H_MAX_PACKED = 8;
constexpr int H_COLS = TOKEN_COLS;       // of tensor memory, all
// PAIRS: CTA pairs, 256 tokens.  NARROW: up to 128 tokens, two warps that issue MMAs, each with an accumulator of its own.
// WIDE: up to 256, one.
enum Shape { PAIRS, WIDE, NARROW };
constexpr int H_MAKE0 = 4;               // first of the warps that make operands, in groups of four
constexpr int H_OUTS = 8;                // warps that write outputs, behind them
__host__ __device__ constexpr int makers(int shape) { return shape == PAIRS ? 2 : shape == WIDE ? 3 : 4; }
__host__ __device__ constexpr int first_out(int shape) { return H_MAKE0 + 4 * makers(shape); }
__host__ __device__ constexpr int tile_threads(int shape) { return (first_out(shape) + H_OUTS) * 32; }

struct TileCtrl {
    uint64_t x_full[H_MAX_STAGES];       // a stage's x has landed in this CTA
    uint64_t ready[H_MAX_STAGES];        // a stage's weights are operands (PAIR: in both CTAs, and its x has landed there)
    uint64_t empty[H_MAX_STAGES];        // the MMAs that read it completed
    uint64_t p_full[H_MAX_PACKED];       // packed weights have landed
    uint64_t p_empty[H_MAX_PACKED];      // and been read
    uint64_t d_full;                     // a tile's MMAs completed
    uint64_t d_empty;                    // its sums have been read
    uint64_t done;                       // every MMA completed
    uint32_t tmem_base;
    int abort;
};
constexpr int H_CTRL_BYTES = 1024;
static_assert(sizeof(TileCtrl) <= H_CTRL_BYTES, "control block");

struct TileArgs {
    mpq_g4_matrix L;
    const unsigned char *w;
    TokenRows rows;
    int y_type;
    int n_tile, held;                    // tokens of a tile; of them, in one CTA's shared memory
    int n_tiles, tiles;                  // tiles along the tokens; all (of a pair, or a cluster)
    int split;                           // CTAs that share a tile's K
    int terms;                           // of a weight's value: times that K goes by
    int stages, packed;                  // depths of the rings
    int acc_cols;                        // TMEM columns of an accumulator
};

__host__ __device__ inline int tile_stage_bytes(int held) { return held * H_K * 2; }
__host__ __device__ inline int packed_bytes(const mpq_g4_matrix &L) { return 8 * L.tile_bytes; }

// A place in a ring: the slot, and the parity of the phase in which it is filled (emptied: the other).
struct Place {
    int at = 0;
    uint32_t phase = 0;
    __device__ __forceinline__ void pass(int slots, int count = 1)   // count <= slots
    {
        at += count;
        if (at >= slots) {
            at -= slots;
            phase ^= 1u;
        }
    }
};

// D[tmem] (+)= A[tmem] B[smem]^T, kind::f16: A's rows on the lanes, two elements of K a column; PAIR: a CTA pair's,
// each CTA with its own rows of A (and D) and half of B's.
template <bool PAIR>
__device__ __forceinline__ void mma_f16_ts(uint32_t d, uint32_t a, uint64_t b, uint32_t idesc, uint32_t more)
{
    if constexpr (PAIR)
        asm volatile(
            "{\n\t.reg .pred p;\n\t"
            "setp.ne.b32 p, %4, 0;\n\t"
            "tcgen05.mma.cta_group::2.kind::f16 [%0], [%1], %2, %3, p;\n\t}" ::"r"(d), "r"(a), "l"(b), "r"(idesc),
            "r"(more)
            : "memory");
    else
        asm volatile(
            "{\n\t.reg .pred p;\n\t"
            "setp.ne.b32 p, %4, 0;\n\t"
            "tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n\t}" ::"r"(d), "r"(a), "l"(b), "r"(idesc),
            "r"(more)
            : "memory");
}

// True in one thread of a warp that is here as one.
__device__ __forceinline__ bool elected()
{
    uint32_t r;
    asm volatile("{\n\t.reg .pred p;\n\telect.sync _|p, 0xffffffff;\n\tselp.u32 %0, 1, 0, p;\n\t}" : "=r"(r));
    return r != 0;
}

// A wait that is not over at once: true if it or another role's gave up.  (Out of line: with this loop in its place a
// wait that is over at once costs its thread 190 cycles instead of 70, on the way of every stage.)
__device__ __noinline__ bool wait_failed(uint64_t *bar, uint32_t parity, bool other, long long budget, unsigned *status,
                                         volatile int *abort)
{
    const long long t0 = clock64();
    while (!(other ? mbar_try_wait_cluster(bar, parity) : mbar_try_wait(bar, parity))) {
        if (*abort) return true;
        if (clock64() - t0 <= budget) continue;
        *abort = 1;
        atomicOr(status, MPQ_TIMEOUT_G4);
        return true;
    }
    return false;
}

__device__ __forceinline__ void swap_if(bool c, uint4 &a, uint4 &b)
{
    const uint4 x = c ? b : a, y = c ? a : b;
    a = x;
    b = y;
}

// 32 columns of a warp's lane quarter, a lane per thread.
__device__ __forceinline__ void tmem_st_32(uint32_t taddr, const uint32_t (&v)[32])
{
    asm volatile(
        "tcgen05.st.sync.aligned.32x32b.x32.b32 [%0], "
        "{%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16,"
        "%17,%18,%19,%20,%21,%22,%23,%24,%25,%26,%27,%28,%29,%30,%31,%32};" ::"r"(taddr),
        "r"(v[0]), "r"(v[1]), "r"(v[2]), "r"(v[3]), "r"(v[4]), "r"(v[5]), "r"(v[6]), "r"(v[7]),
        "r"(v[8]), "r"(v[9]), "r"(v[10]), "r"(v[11]), "r"(v[12]), "r"(v[13]), "r"(v[14]),
        "r"(v[15]), "r"(v[16]), "r"(v[17]), "r"(v[18]), "r"(v[19]), "r"(v[20]), "r"(v[21]),
        "r"(v[22]), "r"(v[23]), "r"(v[24]), "r"(v[25]), "r"(v[26]), "r"(v[27]), "r"(v[28]),
        "r"(v[29]), "r"(v[30]), "r"(v[31])
        : "memory");
}

// Where a lane's channel's outputs go: tokens j0 .. of n_real, n0 the first of the tile.
struct Column {
    int i, lane;
    long long n0;
    int n_real;
};

// Two tokens' outputs in 16 bits.  Where rows take them by twos, neighbouring lanes exchange, and the even one stores
// two channels of token j, the odd one of j + 1 (a warp's store is whole sectors either way).
__device__ __forceinline__ void store_two(const TokenRows &r, uint16_t *Y, uint32_t own, const Column &at, int j)
{
    const size_t size = (r.tokens - 1) * r.ldy + r.channels;
    if (r.wide) {
        const int odd = at.lane & 1, c = at.i - odd;
        const uint32_t other = __shfl_xor_sync(0xffffffffu, own, 1);
        const uint32_t two = odd ? __byte_perm(other, own, 0x7632) : __byte_perm(own, other, 0x5410);
        if (j + odd < at.n_real && c < r.channels && MPQ_IN((at.n0 + j + odd) * r.ldy + c + 1, size))
            *reinterpret_cast<uint32_t *>(Y + (at.n0 + j + odd) * r.ldy + c) = two;
        return;
    }
    if (at.i >= r.channels) return;
    uint16_t *const y = Y + (at.n0 + j) * r.ldy + at.i;
    if (j < at.n_real && MPQ_IN((at.n0 + j) * r.ldy + at.i, size)) *y = (uint16_t)own;
    if (j + 1 < at.n_real && MPQ_IN((at.n0 + j + 1) * r.ldy + at.i, size)) y[r.ldy] = (uint16_t)(own >> 16);
}

__device__ __forceinline__ void store_one(const TokenRows &r, float *Y, float v, const Column &at, int j)
{
    if (at.i < r.channels && j < at.n_real &&
        MPQ_IN((at.n0 + j) * r.ldy + at.i, (r.tokens - 1) * r.ldy + r.channels))
        Y[(at.n0 + j) * r.ldy + at.i] = v;
}

__device__ __forceinline__ uint32_t pack16(int type, float a, float b)
{
    return type == MPQ_F16 ? pack2(a, b, __half()) : pack2(a, b, __nv_bfloat16());
}

// A channel's power of two (EXACT, fp16): its scales are taken times 2^n, n = a + b, and its sums 2^-n times.
struct Power {
    int a, b;
    __device__ __forceinline__ float scaled(float s) const { return s * pow2f(a) * pow2f(b); }
    __device__ __forceinline__ float back(float v) const { return v * pow2f(-a) * pow2f(-b); }
};
// Of channel `row` of a row tile, by the scales of its packed tiles k0 .. k1 - 1.  (Bits above the exponent's of infinity
// too: such a channel's outputs are no numbers anyway.)
__device__ __forceinline__ Power power_of(const TileArgs &a, int row_tile, int row, int k0, int k1)
{
    const int strip = row_tile * (H_M / 16) + (row >> 4), groups = 128 / a.L.group;
    uint32_t most = 0;
    if (strip < a.L.row_tiles) {
        const unsigned char *p = a.w + ((size_t)strip * a.L.k_tiles + k0) * a.L.tile_bytes + G4_CODES + (row & 15) * 2 * groups;
#pragma unroll 8
        for (int k = k0; k < k1; ++k, p += a.L.tile_bytes) {
            if (groups == 1) {
                most = __vmaxu2(most, *reinterpret_cast<const uint16_t *>(p) & 0x7fffu);
            } else if (groups == 2) {
                most = __vmaxu2(most, *reinterpret_cast<const uint32_t *>(p) & 0x7fff7fffu);
            } else {
                const uint2 s = *reinterpret_cast<const uint2 *>(p);
                most = __vmaxu2(most, __vmaxu2(s.x & 0x7fff7fffu, s.y & 0x7fff7fffu));
            }
        }
    }
    const int n = 127 + 11 - max((int)(max(most & 0xffffu, most >> 16) >> 7), 1);     // -117 .. 137
    return {n / 2, n - n / 2};
}

template <typename T, int SHAPE, bool EXACT>
__global__ void __launch_bounds__(tile_threads(SHAPE), 1)
g4_tiles_kernel(const TileArgs a, void *Y, WaitCtl wc, const __grid_constant__ CUtensorMap tmX,
                const __grid_constant__ CUtensorMap tmW)
{
    constexpr bool PAIR = SHAPE == PAIRS, POWERS = EXACT && !G4Pairs<T>::kBf16;
    extern __shared__ unsigned char raw[];
    unsigned char *const base = raw + ((1024u - (smem_u32(raw) & 1023u)) & 1023u);
    TileCtrl &ctl = *reinterpret_cast<TileCtrl *>(base);
    unsigned char *const ring = base + H_CTRL_BYTES;
    const uint32_t ring_u32 = smem_u32(ring);
    const int sb = tile_stage_bytes(a.held), pb = packed_bytes(a.L);
    unsigned char *const packed = ring + a.stages * sb;
    volatile int *const abort_flag = &ctl.abort;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const bool cluster = PAIR || a.split > 1;
    const int rank = cluster ? (int)cluster_ctarank() : 0, size = PAIR ? 2 : a.split;
    const int first = (int)blockIdx.x / size, step = (int)gridDim.x / size;
    const int k_tiles = a.L.k_tiles;
    // this CTA's share of the row
    const int k0 = PAIR ? 0 : (int)((long long)k_tiles * rank / a.split);
    const int k1 = PAIR ? k_tiles : (int)((long long)k_tiles * (rank + 1) / a.split);
    // stages of a tile: its packed tiles, for each term of the weights
    const int span = (k1 - k0) * (EXACT ? a.terms : 1);
    auto k_of = [&](int i) { return k0 + (EXACT && i >= k1 - k0 ? i - (k1 - k0) : i); };
    // halves of a stage (64 elements, a row of the swizzle) that the row reaches
    auto halves = [&](int k) { return k * H_K + 64 < a.L.d ? 2 : 1; };
    auto row_tile = [&](int tile) { return PAIR ? tile / a.n_tiles * 2 + rank : tile / a.n_tiles; };
    auto token0 = [&](int tile) { return (long long)(tile % a.n_tiles) * a.n_tile; };
    // A wait that gave up, or that another role has given up: true.  (Cluster-scope acquires only where one
    // thread takes arrivals of the other CTA's warps.)
    auto failed = [&](uint64_t *bar, uint32_t parity, bool other) {
        if (__builtin_expect(PAIR && other ? mbar_try_wait_cluster(bar, parity) : mbar_try_wait(bar, parity), 1))
            return false;
        return wait_failed(bar, parity, PAIR && other, wc.budget, wc.status, &ctl.abort);
    };
    auto warp_failed = [&](uint64_t *bar, uint32_t parity, bool other = false) {
        return __any_sync(0xffffffffu, failed(bar, parity, other)) != 0;
    };
    auto arrive = [&](uint64_t *bar) {   // at the CTA whose thread issues MMAs
        if (PAIR) mbar_arrive_cluster(bar, 0); else mbar_arrive(bar);
    };
    auto commit = [&](uint64_t *bar) {       // PAIR: in both CTAs
        if (PAIR) mma_commit_pair(bar, (uint16_t)3); else mma_commit(bar);
    };

    griddep_launch();
    if (threadIdx.x == 0) {
        for (int i = 0; i < a.stages; ++i) {
            mbar_init(&ctl.x_full[i], 1);
            mbar_init(&ctl.ready[i], PAIR ? 10 : 4);
            mbar_init(&ctl.empty[i], 1);
        }
        for (int i = 0; i < a.packed; ++i) {
            mbar_init(&ctl.p_full[i], 1);
            mbar_init(&ctl.p_empty[i], 4);
        }
        mbar_init(&ctl.d_full, SHAPE == NARROW ? 2 : 1);
        mbar_init(&ctl.d_empty, (PAIR ? 2 : 1) * H_OUTS);
        mbar_init(&ctl.done, SHAPE == NARROW ? 2 : 1);
        ctl.abort = 0;
        fence_barrier_init();
        if (!MPQ_CHECK_SMEM_END(packed - raw + (size_t)a.packed * pb)) ctl.abort = 1;
        prefetch_tensormap(&tmX);
        prefetch_tensormap(&tmW);
    }
    if (warp == 1) {
        if (PAIR)
            tmem_alloc_pair(&ctl.tmem_base, H_COLS);
        else
            tmem_alloc(&ctl.tmem_base, H_COLS);
    }
    tc_fence_before();
    __syncthreads();
    if (PAIR) cluster_sync();            // the barriers that the other CTA arrives on are ready
    tc_fence_after();
    const uint32_t tmem = ctl.tmem_base, operands = tmem + (uint32_t)((SHAPE == NARROW ? 2 : 1) * a.acc_cols);
    griddep_wait();

    if (warp == 0) {
        // -------------------------------------------------------------------- copies of x
        int n = 0;
        Place s;
        bool stop = wc.withhold == 1 || *abort_flag;
        for (int tile = first; tile < a.tiles && !stop; tile += step) {
            const int y0 = (int)token0(tile) + (PAIR ? rank * a.held : 0);
            for (int i = 0; i < span; ++i, ++n, s.pass(a.stages)) {
                const int k = k_of(i);
                const uint32_t at = ring_u32 + (uint32_t)(s.at * sb);
                if ((n >= a.stages && warp_failed(&ctl.empty[s.at], s.phase ^ 1u)) || !MPQ_CHECK((at & 1023u) == 0u)) {
                    stop = true;
                    break;
                }
                if (elected()) {
                    const int count = halves(k);
                    uint64_t *const bar = &ctl.x_full[s.at];
                    mbar_arrive_expect_tx(bar, (uint32_t)(count * a.held * 128));
                    for (int h = 0; h < count; ++h)
                        tma_load_2d(at + (uint32_t)(h * a.held * 128), &tmX, k * H_K + h * 64, y0, bar);
                }
                __syncwarp();
            }
        }
        // no copy may land after the CTA is gone (whatever became of the other roles: a barrier that these complete too
        // would never be full behind one that gave up)
        for (int i = max(0, n - a.stages); lane == 0 && i < n; ++i)
            drain_wait(&ctl.x_full[i % a.stages], (uint32_t)(i / a.stages) & 1u, wc, MPQ_TIMEOUT_G4);
        // ... nor an arrival for the pair's MMAs: their end comes in any case, the last stages' arrivals if no role gave up
        if (PAIR && lane == 0) {
            drain_wait_cluster(&ctl.done, 0, wc, MPQ_TIMEOUT_G4);
            for (int i = max(0, n - a.stages); i < n; ++i)
                if (*abort_flag || failed(&ctl.empty[i % a.stages], (uint32_t)(i / a.stages) & 1u, false)) break;
        }
        __syncwarp();
    } else if (warp == 2) {
        // -------------------------------------------------------------------- copies of weights
        int n = 0;
        Place p;
        bool stop = wc.withhold || *abort_flag;
        for (int tile = first; tile < a.tiles && !stop; tile += step) {
            const int r0 = row_tile(tile) * 8;
            for (int i = 0; i < span; ++i, ++n, p.pass(a.packed)) {
                if (n >= a.packed && warp_failed(&ctl.p_empty[p.at], p.phase ^ 1u)) {
                    stop = true;
                    break;
                }
                const uint32_t at = smem_u32(packed + p.at * pb);
                if (!MPQ_CHECK((at & 127u) == 0u)) {
                    stop = true;
                    break;
                }
                if (elected()) {         // (strips of 16 channels past the last are filled with zeros)
                    mbar_arrive_expect_tx(&ctl.p_full[p.at], (uint32_t)pb);
                    tma_load_3d(at, &tmW, 0, k_of(i), r0, &ctl.p_full[p.at]);
                }
                __syncwarp();
            }
        }
        for (int i = max(0, n - a.packed); lane == 0 && i < n; ++i)
            drain_wait(&ctl.p_full[i % a.packed], (uint32_t)(i / a.packed) & 1u, wc, MPQ_TIMEOUT_G4);
        __syncwarp();
    } else if (PAIR && warp == 3) {
        // -------------------------------------------------------------------- x has landed
        Place s;
        bool stop = false;
        for (int tile = first; tile < a.tiles && !stop; tile += step)
            for (int i = 0; i < span; ++i, s.pass(a.stages)) {
                stop = warp_failed(&ctl.x_full[s.at], s.phase);
                if (stop) break;
                if (elected()) arrive(&ctl.ready[s.at]);
                __syncwarp();
            }
    } else if (warp == 1 || (SHAPE == NARROW && warp == 3)) {
        // -------------------------------------------------------------------- MMAs
        // (the warp waits as one; a thread that waits alone keeps its warp's others at the next meeting point, which
        // costs it a hundred cycles a wait)
        if (!PAIR || rank == 0) {
            const int own = warp >> 1;   // NARROW: of two, which takes every other stage
            int t = 0, n = 0;            // tiles, stages so far
            Place s;
            bool stop = false;
            for (int tile = first; tile < a.tiles && !stop; tile += step, ++t) {
                const int real = (int)min((long long)a.n_tile, a.rows.tokens - token0(tile));
                const int m = PAIR ? 2 * H_M : H_M, cols = PAIR ? 256 : (real + 15) / 16 * 16;
                const uint32_t id = G4Pairs<T>::kBf16 ? idesc_bf16(m, cols) : idesc_f16(m, cols);
                const uint32_t d = tmem + (uint32_t)(SHAPE == NARROW ? own * a.acc_cols : 0);
                uint32_t more = 0;
                if (t > 0 && warp_failed(&ctl.d_empty, (uint32_t)(t - 1) & 1u, true)) break;
                for (int i = 0; i < span; ++i, ++n, s.pass(a.stages)) {
                    if (SHAPE == NARROW && (n & 1) != own) continue;
                    if ((!PAIR && warp_failed(&ctl.x_full[s.at], s.phase)) || warp_failed(&ctl.ready[s.at], s.phase, true)) {
                        stop = true;
                        break;
                    }
                    tc_fence_after();
                    const uint64_t bd = smem_desc_sw128(ring_u32 + (uint32_t)(s.at * sb));
                    const uint32_t at = operands + (uint32_t)(s.at * H_A_COLS);
                    if (elected()) {
                        const int count = halves(k_of(i));
                        for (int h = 0; h < count; ++h) {
                            const uint64_t bh = bd + (uint64_t)(h * a.held * 8);     // in 16 B units
#pragma unroll
                            for (int j = 0; j < 4; ++j)
                                mma_f16_ts<PAIR>(d, at + 32 * h + 8 * j, bh + 2 * j, id, more | (uint32_t)(h + j > 0));
                        }
                        commit(&ctl.empty[s.at]);
                    }
                    more = 1;
                    __syncwarp();
                }
                if (!stop && elected()) commit(&ctl.d_full);
                __syncwarp();
            }
            // every MMA issued above completes before tensor memory is released
            if (elected()) {
                commit(&ctl.done);
                drain_wait_cluster(&ctl.done, 0, wc, MPQ_TIMEOUT_G4);
            }
        }
        __syncwarp();
    } else if (warp < H_MAKE0) {
        // -------------------------------------------------------------------- (WIDE: no work for warp 3)
    } else if (warp < first_out(SHAPE)) {
        // -------------------------------------------------------------------- operands from packed weights
        // A thread has a channel: its 64 bytes of a packed tile, by quarters in an order in which eight lanes
        // (what shared memory serves at once) meet no bank twice, put right in registers.
        const int own = (warp - H_MAKE0) >> 2, q = warp & 3, row = q * 32 + lane, x = (lane >> 1) & 3;
        const int groups = 128 / a.L.group;
        const uint32_t to = operands + ((uint32_t)(q * 32) << 16);
        const unsigned char *const mine_at = packed + (row >> 4) * a.L.tile_bytes;
        // of all the stages of all the CTA's tiles, every makers(SHAPE)-th
        const long long stages = first < a.tiles ? (long long)((a.tiles - first - 1) / step + 1) * span : 0;
        Place p, s;
        p.pass(a.packed, own);
        s.pass(a.stages, own);
        int tile = first, at_stage = own;    // EXACT: of which tile this is which stage
        Power power = {0, 0};
        int power_tile = -1;                 // whose
        for (long long n = own; n < stages; n += makers(SHAPE), p.pass(a.packed, makers(SHAPE)), s.pass(a.stages, makers(SHAPE))) {
            bool second = false;             // the values' second term
            if constexpr (EXACT) {
                while (at_stage >= span) at_stage -= span, tile += step;
                second = at_stage >= k1 - k0;
                at_stage += makers(SHAPE);
                if (POWERS && power_tile != tile) {
                    power = power_of(a, row_tile(tile), row, k0, k1);
                    power_tile = tile;
                }
            }
            if (warp_failed(&ctl.p_full[p.at], p.phase)) break;
            const unsigned char *const t = mine_at + p.at * pb;
            uint4 w[4];
#pragma unroll
            for (int i = 0; i < 4; ++i)
                w[i] = *reinterpret_cast<const uint4 *>(t + (row & 15) * 64 + (i ^ x) * 16);
            uint2 sc;                // the row's scales of the tile's quarters, two a word
            uint32_t z = 0x08080808u;            // and zero points
            const unsigned char *const ss = t + G4_CODES + (row & 15) * 2 * groups;
            const unsigned char *const zs = t + G4_CODES + 32 * groups + (row & 15) * groups;
            if (groups == 1) {
                sc.x = sc.y = *reinterpret_cast<const uint16_t *>(ss) * 0x10001u;
                if (a.L.zeros) z = __byte_perm(*zs, 0, 0x0000);
            } else if (groups == 2) {
                const uint32_t two = *reinterpret_cast<const uint32_t *>(ss);
                sc = make_uint2(__byte_perm(two, 0, 0x1010), __byte_perm(two, 0, 0x3232));
                if (a.L.zeros) z = __byte_perm(*reinterpret_cast<const uint16_t *>(zs), 0, 0x1100);
            } else {
                sc = *reinterpret_cast<const uint2 *>(ss);
                if (a.L.zeros) z = *reinterpret_cast<const uint32_t *>(zs);
            }
            __syncwarp();
            if (elected()) mbar_arrive(&ctl.p_empty[p.at]);
            swap_if(x & 1, w[0], w[1]);
            swap_if(x & 1, w[2], w[3]);
            swap_if(x & 2, w[0], w[2]);
            swap_if(x & 2, w[1], w[3]);
            bool stop = false;
            const uint32_t scales[2] = {sc.x, sc.y};
            const bool far = !EXACT && g4_far<T>(scales);
#pragma unroll
            for (int h = 0; h < 2; ++h) {            // (behind the row's end: zeros, whose MMAs are left out)
                uint32_t v[32];
                auto convert = [&](auto f) {
#pragma unroll
                    for (int m = 0; m < 2; ++m) {
                        const uint32_t two = scales[h];
                        G4Scale g = g4_scale<T>(m ? two >> 16 : two & 0xffffu, z >> (8 * (2 * h + m)) & 255u);
                        if constexpr (POWERS) g.s = G4Pairs<T>::bits(__float2half2_rn(power.scaled(bf16_bits(g.bits))));
#pragma unroll
                        for (int i = 0; i < 4; ++i) {
                            const uint32_t word = h ? (m ? w[i].w : w[i].z) : (m ? w[i].y : w[i].x);
                            uint32_t p4[4];
                            if constexpr (decltype(f)::value == 2)
                                g4_rest<T>(word, g, p4);
                            else
                                g4_values<T, decltype(f)::value != 0>(word, g, p4);
#pragma unroll
                            for (int e = 0; e < 4; ++e) v[16 * m + 4 * i + e] = p4[e];
                        }
                    }
                };
                if (EXACT ? second : far)
                    convert(std::integral_constant<int, EXACT ? 2 : 1>());
                else
                    convert(std::integral_constant<int, 0>());
                if (h == 0) {
                    stop = n >= a.stages && warp_failed(&ctl.empty[s.at], s.phase ^ 1u);
                    if (stop) break;
                    tc_fence_after();
                }
                tmem_st_32(to + (uint32_t)(s.at * H_A_COLS + 32 * h), v);
            }
            if (stop) break;
            tmem_wait_st();
            tc_fence_before();
            __syncwarp();
            if (elected()) arrive(&ctl.ready[s.at]);
        }
    } else {
        // -------------------------------------------------------------------- outputs
        const int q = warp & 3, row = q * 32 + lane, half = (warp - first_out(SHAPE)) >> 2;
        int t = 0;
        for (int tile = first; tile < a.tiles; tile += step, ++t) {
            const long long n0 = token0(tile);
            const int real = (int)min((long long)a.n_tile, a.rows.tokens - n0);
            // NARROW: both accumulators have sums, but for a tile of one stage
            const int whose = span == 1 ? t & 1 : 0;
            const bool both = SHAPE == NARROW && span > 1;
            const int c = row_tile(tile) * H_M + row;
            const float bias = a.split == 1 && a.rows.bias && c < a.rows.channels ? a.rows.bias[c] : 0.0f;
            Power power = {0, 0};
            if (POWERS) power = power_of(a, row_tile(tile), row, k0, k1);
            auto value = [&](float v) { return POWERS ? power.back(v) : v; };
            if (warp_failed(&ctl.d_full, (uint32_t)t & 1u)) break;
            tc_fence_after();
            const uint32_t from = tmem + ((uint32_t)(q * 32) << 16) + (uint32_t)(SHAPE == NARROW ? whose * a.acc_cols : 0);
            const Column at{c, lane, n0, real};
            uint16_t *const y16 = static_cast<uint16_t *>(Y);
            if constexpr (PAIR) {
                // 16 bits: all of the sums to registers, so that the next tile's MMAs go on (8,300 cycles earlier)
                if (a.y_type != MPQ_F32) {
                    uint32_t two[64];
                    const int j0 = half * 128;
#pragma unroll
                    for (int u = 0; u < 4; ++u) {
                        float v[32];
                        tmem_ld_32x32b_x32(from + (uint32_t)(j0 + 32 * u), v);
#pragma unroll
                        for (int j = 0; j < 16; ++j)
                            two[16 * u + j] = pack16(a.y_type, value(v[2 * j]) + bias, value(v[2 * j + 1]) + bias);
                    }
                    tc_fence_before();
                    __syncwarp();
                    if (elected()) arrive(&ctl.d_empty);
#pragma unroll
                    for (int j = 0; j < 64; ++j)
                        if (j0 + 2 * j < real) store_two(a.rows, y16, two[j], at, j0 + 2 * j);
                    continue;
                }
            }
            for (int j0 = half * 16; j0 < real; j0 += H_OUTS / 4 * 16) {
                float v[16];
                __syncwarp();
                tmem_ld_32x32b_x16(from + (uint32_t)j0, v);
                if (both) {
                    float o[16];
                    tmem_ld_32x32b_x16(from + (uint32_t)(a.acc_cols + j0), o);
#pragma unroll
                    for (int j = 0; j < 16; ++j) v[j] += o[j];
                }
                if (POWERS) {
#pragma unroll
                    for (int j = 0; j < 16; ++j) v[j] = value(v[j]);
                }
                if (!PAIR && a.split > 1) {          // [token][128 channels]; the MMAs have read the ring
                    float *const part = reinterpret_cast<float *>(ring) + row;
#pragma unroll
                    for (int j = 0; j < 16; ++j) part[(j0 + j) * H_M] = v[j];
                    continue;
                }
#pragma unroll
                for (int j = 0; j < 16; ++j) v[j] += bias;
                if (a.y_type == MPQ_F32) {
#pragma unroll
                    for (int j = 0; j < 16; ++j) store_one(a.rows, static_cast<float *>(Y), v[j], at, j0 + j);
                } else {
#pragma unroll
                    for (int j = 0; j < 16; j += 2)
                        store_two(a.rows, y16, pack16(a.y_type, v[j], v[j + 1]), at, j0 + j);
                }
            }
            tc_fence_before();
            __syncwarp();
            if (elected()) arrive(&ctl.d_empty);
        }
    }

    if (!PAIR && a.split > 1) {
        cluster_sync();                  // every rank's sums are in its shared memory
        const long long n0 = token0(first);
        const JoinAt at{reinterpret_cast<const float *>(ring), n0,
                        (int)min((long long)a.n_tile, a.rows.tokens - n0), row_tile(first), rank};
        if (a.y_type == MPQ_F32)
            join_split<false>(a.rows, static_cast<float *>(Y), at, a.split);
        else if (a.y_type == MPQ_F16)
            join_split<false>(a.rows, static_cast<__half *>(Y), at, a.split);
        else
            join_split<false>(a.rows, static_cast<__nv_bfloat16 *>(Y), at, a.split);
    }
    if (cluster)
        cluster_sync();                  // no CTA leaves while its sums are read, or arrivals to it are on their way
    else
        __syncthreads();
    if (warp == 1) {
        tc_fence_after();
        if (PAIR)
            tmem_dealloc_pair(tmem, H_COLS);
        else
            tmem_dealloc(tmem, H_COLS);
    }
}

// Rows of x where a tile copy cannot read them, `to` elements apart and 16-byte aligned, the rest zeros.
__global__ void __launch_bounds__(256)
g4_rows_kernel(const uint16_t *X, long long ldx, int T, int d, uint16_t *to, int dp)
{
    griddep_launch();
    griddep_wait();
    const long long n = (long long)T * (dp / 8), step = (long long)gridDim.x * blockDim.x;
    for (long long i = (long long)blockIdx.x * blockDim.x + threadIdx.x; i < n; i += step) {
        const long long t = i / (dp / 8);
        const int j = (int)(i - t * (dp / 8)) * 8;
        const uint16_t *const x = X + t * ldx;
        uint32_t w[4];
#pragma unroll
        for (int e = 0; e < 4; ++e)
            w[e] = (j + 2 * e < d ? x[j + 2 * e] : 0u) | (j + 2 * e + 1 < d ? (uint32_t)x[j + 2 * e + 1] : 0u) << 16;
        if (MPQ_IN(t * dp + j + 7, (long long)T * dp))
            *reinterpret_cast<uint4 *>(to + t * dp + j) = make_uint4(w[0], w[1], w[2], w[3]);
    }
}

template <typename T, int SHAPE, bool EXACT>
mpq_status launch_tiles(const TileArgs &a, const CUtensorMap &tmX, const CUtensorMap &tmW, void *Y, int ctas, cudaStream_t stream)
{
    const size_t smem = token_smem(1024 + H_CTRL_BYTES + (size_t)a.stages * tile_stage_bytes(a.held) +
                                       (size_t)a.packed * packed_bytes(a.L), H_COLS);
    const mpq_status sm = token_check_sm();
    if (sm != MPQ_OK) return sm;
    static std::atomic<int> limit[kMaxDevices];
    cudaError_t e = allow_smem(reinterpret_cast<const void *>(g4_tiles_kernel<T, SHAPE, EXACT>), limit, smem);
    if (e != cudaSuccess) return cuda_status(e, "cudaFuncSetAttribute");
    WaitCtl wc;
    const mpq_status ws = wait_ctl(&wc);
    if (ws != MPQ_OK) return ws;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)ctas);
    cfg.blockDim = dim3(tile_threads(SHAPE));
    cfg.dynamicSmemBytes = smem;
    cfg.stream = stream;
    cudaLaunchAttribute attr[2];
    attr[0] = after_previous_kernel();
    attr[1].id = cudaLaunchAttributeClusterDimension;
    attr[1].val.clusterDim.x = SHAPE == PAIRS ? 2u : (unsigned)a.split;
    attr[1].val.clusterDim.y = 1;
    attr[1].val.clusterDim.z = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 2;
    e = cudaLaunchKernelEx(&cfg, g4_tiles_kernel<T, SHAPE, EXACT>, a, Y, wc, tmX, tmW);
    return cuda_status(e != cudaSuccess ? e : cudaGetLastError(), "g4 linear launch");
}

template <typename T, bool EXACT>
mpq_status launch_form(const TileArgs &a, int shape, const CUtensorMap &tmX, const CUtensorMap &tmW, void *Y, int ctas,
                       cudaStream_t stream)
{
    return shape == PAIRS  ? launch_tiles<T, PAIRS, EXACT>(a, tmX, tmW, Y, ctas, stream)
           : shape == WIDE ? launch_tiles<T, WIDE, EXACT>(a, tmX, tmW, Y, ctas, stream)
                           : launch_tiles<T, NARROW, EXACT>(a, tmX, tmW, Y, ctas, stream);
}

struct Form {
    int n;                               // tokens of a tile
    bool pair;
    int split;
};

// CTAs (clusters of `split`) that are resident at once: one CTA an SM; what whole clusters leave of the GPCs' SMs was
// measured (a cluster more than these takes a second round).
int resident(int split, int sms) { return split == 1 ? sms : split == 2 ? sms / 2 : split == 4 ? sms * 36 / 152 : sms * 14 / 152; }

// The form with the least modelled time (us): a start, and for each round of resident CTAs its stages, by their tokens
// (up to 128 the operands' making bounds them, 0.34 to 0.36 us; from 192 on the MMAs), the tile's way out, and the
// joining of a split; `terms`: K goes by so many times.  Fitted to 919 timings, weights in L2, of 91 sizes (16 <= T <= 2,048, 448 <= C <= 14,000, 500 <= d <= 11,008): the
// choice costs 1% on average against the best form, 15% at worst (16 x 1,024 x 1,024, where the few tokens' kernel is
// taken).  Some of them, us, with 32 / 64 / 128 / 256 tokens a tile, pairs: 32 x 4,096 x 4,096 (T x C x d; split by 4)
// 9.4, -, -, -, -; 256 x 11,008 x 4,096 -, -, 32.5, 25.4, 27.4; 2,048 x 11,008 x 4,096 -, 238, 148, 121, 105;
// 512 x 4,096 x 4,096 -, -, 18.8, 18.5 (split by 2), 26.7.
Form choose_form(int T, int C, int k_tiles, int terms, int sms, double &least)
{
    auto rounds = [](long long n, long long at_once) { return (double)((n + at_once - 1) / at_once); };
    Form best = {256, true, 1};
    least = 6.8 + rounds((C + 255LL) / 256 * ((T + 255LL) / 256), std::max(1, sms / 2)) * (0.512 * k_tiles * terms + 3.7);
    if (T <= 128) least = HUGE_VAL;
    for (int most = 32; most <= 256; most += most < 128 ? 32 : 64) {
        const int n = std::min(most, (T + 15) / 16 * 16);
        const long long tiles = (C + H_M - 1LL) / H_M * ((T + n - 1LL) / n);
        for (int split = 1; split <= TOKEN_MAX_SPLIT && split * 2 <= std::max(2, k_tiles); split *= 2) {
            const int stages = (k_tiles + split - 1) / split * terms;
            const double r = rounds(tiles, std::max(1, resident(split, sms)));
            const double t = 1.9 + r * (stages * std::max(0.3435 + 0.0001 * n, 0.0021 * n) + 0.46 +
                                        (n > 128 ? 0.0246 : 0.0283) * n + (split > 1 ? 2.9 - 0.0091 * n : 0.0));
            if (t < least) {
                best = {n, false, split};
                least = t;
            }
            if (split == 1 && tiles > 4LL * sms) break;
        }
    }
    return best;
}

}  // namespace

int g4_terms(int x_type, const mpq_g4_matrix *L) { return x_type == MPQ_BF16 || L->zeros ? 2 : 1; }

double g4_tiles_time(int T, int C, int d, int terms)
{
    double t;
    choose_form(T, C, (d + H_K - 1) / H_K, terms, sm_count(), t);
    return t;
}

mpq_status launch_g4_tiles(const void *X, int x_type, long long ldx, int T, const mpq_g4_matrix *L, const void *W,
                           const float *bias, void *Y, int y_type, long long ldy, int exact, cudaStream_t stream)
{
    TileArgs a = {};
    a.L = *L;
    a.w = static_cast<const unsigned char *>(W);
    a.y_type = y_type;
    const int C = L->rows, four = 4 * type_size(y_type), sms = sm_count();
    a.rows = {T, C, C % 4 == 0 && ldy % 4 == 0 && (uintptr_t)Y % four == 0, bias, ldy};
    double modelled;
    a.terms = exact ? g4_terms(x_type, L) : 1;
    Form f = choose_form(T, C, L->k_tiles, a.terms, sms, modelled);
    const G4Form asked = g4_test_form();
    if (asked.form == MPQ_G4_PAIRS) f = {256, true, 1};
    if (asked.form == MPQ_G4_TILES) {
        f = {std::min(asked.tokens, (T + 15) / 16 * 16), false, asked.split};
        if (f.split > 1 && f.split * 2 > L->k_tiles) {
            set_error("g4 linear: %d tiles of K are too few for %d CTAs", L->k_tiles, f.split);
            return MPQ_ERR_UNSUPPORTED;
        }
    }
    a.n_tile = f.n;
    a.held = f.pair ? f.n / 2 : f.n;
    a.split = f.pair ? 1 : f.split;
    a.acc_cols = 32;
    while (a.acc_cols < f.n) a.acc_cols *= 2;
    a.n_tiles = (T + f.n - 1) / f.n;
    const long long tiles = ((long long)C + (f.pair ? 2 : 1) * H_M - 1) / ((f.pair ? 2 : 1) * H_M) * a.n_tiles;
    if (tiles > (1 << 28)) {
        set_error("g4 linear: T = %d, C = %d are too large", T, C);
        return MPQ_ERR_UNSUPPORTED;
    }
    a.tiles = (int)tiles;
    const int ctas = f.pair      ? 2 * std::min(a.tiles, sms / 2)
                     : f.split > 1 ? a.tiles * f.split
                                   : std::min(a.tiles, sms);

    const int shape = f.pair ? PAIRS : f.n > 128 ? WIDE : NARROW;
    // as many packed tiles as groups or more, as many stages as fit beside them, then more packed tiles
    const int room = max_smem_optin() - 1024 - H_CTRL_BYTES, pb = packed_bytes(*L), sb = tile_stage_bytes(a.held);
    const int groups = makers(shape), accs = shape == NARROW ? 2 : 1;
    a.stages = std::min({H_MAX_STAGES, (room - groups * pb) / sb, (H_COLS - accs * a.acc_cols) / H_A_COLS});
    // A barrier's parity tells two phases apart, not more.  A group of makers that has made a stage knows that the MMAs
    // took the stage `stages` before it, and its next one is `groups` on: it meets a phase that is at most one behind if
    // there are as many stages as groups (NARROW: an even number of both, so that what one warp's MMAs took
    // says that it took the earlier ones; a stage's place is always the same warp's).  Packed tiles may land out of
    // order, so that a group knows only of its own: a slot is always the same group's.
    if (shape == NARROW) a.stages &= ~1;
    a.packed = std::min(H_MAX_PACKED, (room - a.stages * sb) / pb) / groups * groups;
    if (a.stages < groups || a.packed < groups) {
        set_error("g4 linear: shared memory has no room for %d stages", groups);
        return MPQ_ERR_UNSUPPORTED;
    }

    void *scratch = nullptr;
    int dp = L->d;
    if (!rows_aligned(X, x_type, T > 1 ? ldx : 0)) {
        dp = (L->d + 7) / 8 * 8;
        const mpq_status st = pool_scratch(&scratch, (size_t)T * dp * 2, stream);
        if (st != MPQ_OK) return st;
        const long long n = (long long)T * (dp / 8);
        const mpq_status ls = launch_waiting(g4_rows_kernel, dim3((unsigned)std::min((n + 255) / 256, 16LL * sms)),
                                             dim3(256), 0, stream, "g4 rows launch", static_cast<const uint16_t *>(X),
                                             ldx, T, L->d, static_cast<uint16_t *>(scratch), dp);
        if (ls != MPQ_OK) {
            cudaFreeAsync(scratch, stream);
            return ls;
        }
        X = scratch;
        ldx = dp;
    }
    CUtensorMap tmX, tmW;
    memset(&tmX, 0, sizeof(tmX));
    memset(&tmW, 0, sizeof(tmW));
    // packed weights by words of 8 bytes: [strips of 16 channels][tiles of 128][a tile]; a copy takes eight strips
    const cuuint64_t tile = (cuuint64_t)L->tile_bytes;
    const cuuint64_t w_dims[3] = {tile / 8, (cuuint64_t)L->k_tiles, (cuuint64_t)L->row_tiles};
    const cuuint64_t w_strides[2] = {tile, tile * (cuuint64_t)L->k_tiles};
    const cuuint32_t w_box[3] = {(cuuint32_t)L->tile_bytes / 8, 1, 8};
    const cuuint64_t dims[2] = {(cuuint64_t)dp, (cuuint64_t)T};
    const cuuint64_t strides[1] = {(cuuint64_t)(T > 1 ? ldx : (dp + 7) / 8 * 8) * 2};
    const cuuint32_t box[2] = {64, (cuuint32_t)a.held};
    mpq_status st = MPQ_OK;
    if (!encode_tile_map(&tmX, x_type == MPQ_BF16 ? CU_TENSOR_MAP_DATA_TYPE_BFLOAT16 : CU_TENSOR_MAP_DATA_TYPE_FLOAT16, 2,
                         X, dims, strides, box, CU_TENSOR_MAP_SWIZZLE_128B) ||
        !encode_tile_map(&tmW, CU_TENSOR_MAP_DATA_TYPE_FLOAT64, 3, W, w_dims, w_strides, w_box)) {
        set_error("g4 linear: tensor map encoding failed");
        st = MPQ_ERR_CUDA;
    } else if (x_type == MPQ_F16) {
        st = exact ? launch_form<__half, true>(a, shape, tmX, tmW, Y, ctas, stream)
                   : launch_form<__half, false>(a, shape, tmX, tmW, Y, ctas, stream);
    } else {
        st = exact ? launch_form<__nv_bfloat16, true>(a, shape, tmX, tmW, Y, ctas, stream)
                   : launch_form<__nv_bfloat16, false>(a, shape, tmX, tmW, Y, ctas, stream);
    }
    if (scratch) {
        const cudaError_t e = cudaFreeAsync(scratch, stream);
        if (st == MPQ_OK) st = cuda_status(e, "cudaFreeAsync");
    }
    return st;
}

}  // namespace mpq
