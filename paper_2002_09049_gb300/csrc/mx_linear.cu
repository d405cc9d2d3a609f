// Linear layer of microscaled 4-bit floats (mpq_mx_linear): Y[t][c] = sum_j x_tj w_cj + bias_c on the
// tensor cores' block-scaled MMAs (tcgen05.mma kind::mxf4).
//
// A K stage is 256 elements: 128-byte rows of codes, as they lie in memory, by TMA into 128-byte-
// swizzled K-major tiles, and the scales of both operands, 512 contiguous bytes per 128 rows x 128
// elements, by bulk copies.  Four warps move the scales from shared to tensor memory (each stage has
// columns of its own, written anew when its MMAs are done) a stage or more ahead of the thread that
// issues the MMAs: as tensor-core copies (tcgen05.cp) they would take 72 cycles each in line with the
// MMAs, 545 a stage beside the 513 of four 128 x 256 x 64 MMAs.  Accumulators are fp32 in tensor memory,
// one rounding (after the bias) on the way out.
//
// Few tokens (or few tiles): the weights' rows are the MMA's A (M = 128 channels on the accumulator's
// lanes), the tokens its B (N = 16 .. 256), so a handful of tokens costs no padding to 128.  The weights'
// bytes bound it (d / 2 + d / 32 a channel), and with few row tiles most SMs would idle: the K stages of a
// tile are split over the CTAs of a cluster, which leave their sums in shared memory and join them there
// in the order of the ranks (so equal inputs give equal bits).
//
// Many tokens: tokens on the lanes (a lane then writes runs of consecutive outputs), tiles of 256 tokens
// x 256 channels by CTA pairs (cta_group::2: each CTA holds 128 tokens and half of the channels).  One CTA
// alone with a 128 x 256 tile is bound by shared memory (52 KB a stage in and 48 KB read by the MMAs, 784
// cycles at 128 bytes each beside the MMAs' 513) and by what L2 delivers (43 bytes per SM and cycle measured:
// 1,200 cycles).  The pair halves B's share of both, 35 KB in and 32 KB read a stage: 0.5 us a stage, 0.25 of it
// the MMAs', and 5 us a tile for its start and its way out.  Each CTA loads all that it holds: a load for several
// CTAs at once would want its source in this GPU's own memory, which a pointer does not say.
//
// Measured: 1 x 4,096 x 4,096 (T x C x d) 5.0 us and 37 x 11,008 x 4,096 8.4 us (weights' bytes at 1.8 and 2.9
// TB/s; latency of one round of CTAs), 1,024 x 4,096 x 4,096 13.2 us, 2,048 x 4,096 x 11,008 51.7 us (3.6
// PFLOP/s; 128 tiles on 76 pairs are two rounds).
//
// Roles: warp 0 copies, warp 1 issues MMAs (the even CTA's, for a pair), warps 2..5 (TMEM lane quarter
// warp % 4) move scales, then write the outputs -- with warps 6..9 where there are such.  Every wait is
// bounded.
#include <cuda.h>
#include <math.h>
#include <string.h>

#include <algorithm>

#include "elements.cuh"
#include "mpq_internal.cuh"
#include "mx_ops.cuh"
#include "pair_common.cuh"
#include "sm100.cuh"
#include "waits.cuh"

MPQ_CHECKED_UNIT("mx_linear.cu");

namespace mpq {
namespace {

using namespace sm100;

constexpr int X_M = 128;                 // rows of A in a tile (accumulator lanes)
constexpr int X_N = 256;                 // most rows of B in a tile (accumulator columns)
constexpr int X_ROW = 128;               // bytes of a row's codes in a stage: 256 elements
constexpr int X_SF = 512;                // bytes of a scale tile (128 rows x 128 elements)
constexpr int X_A_BYTES = X_M * X_ROW;
constexpr int X_MAX_STAGES = 8;
constexpr int X_THREADS = 320;           // at most: warps 6..9 may be left out
constexpr int X_MAX_SPLIT = 8;           // CTAs of a cluster that splits K

struct MxCtrl {
    uint64_t full[X_MAX_STAGES];         // a stage's tiles and scales have landed
    uint64_t scaled[X_MAX_STAGES];       // its scales are in tensor memory
    uint64_t empty[X_MAX_STAGES];        // the MMAs that read what this CTA loads completed
    uint64_t done;                       // every MMA completed
    uint32_t tmem_base;
    int abort;
};
constexpr int X_CTRL_BYTES = 1024;
static_assert(sizeof(MxCtrl) <= X_CTRL_BYTES, "control block");

// The operands by their place in the MMA: A's rows on the accumulator's lanes, B's on its columns.
struct MxArgs {
    int a_rows, b_rows;
    int a_tiles;                         // row tiles of A (128 rows)
    int n_tile;                          // rows of B in a tile, a multiple of 16
    int b_held;                          // of them, in one CTA's shared memory
    int stages, k_stages, k_tiles;       // ring, K stages of a row, scale tiles of a row
    int split;                           // CTAs that share a tile's K stages
    int acc_cols, cols;                  // TMEM columns: the accumulator's (scales follow), all
    int n_tiles;                         // tiles along B (MANY)
    int wide;                            // output rows take 4 outputs at a time
    const unsigned char *a_scales, *b_scales;
    const float *bias;
    long long ldy;
};

__host__ __device__ inline int sf_b_bytes(int n_tile) { return n_tile > 128 ? 4 * X_SF : 2 * X_SF; }
__host__ __device__ inline int sf_b_cols(int n_tile) { return n_tile > 128 ? 8 : 4; }  // of a k tile
__host__ __device__ inline int sf_cols(int n_tile) { return 8 + 2 * sf_b_cols(n_tile); }
__host__ __device__ inline int stage_bytes(const MxArgs &a)
{
    return X_A_BYTES + a.b_held * X_ROW + 2 * X_SF + sf_b_bytes(a.n_tile);
}

// v[4 j + k] of the four lanes 4 q .. 4 q + 3 (lane l: channel l, k: token) to v[4 j + k] with lane l:
// token l, k: channel -- 4 x 4 transposes by two exchanges.
__device__ __forceinline__ void quad_transpose(float (&v)[16], int lane)
{
#pragma unroll
    for (int o = 1; o <= 2; o <<= 1) {
        const bool high = lane & o;
#pragma unroll
        for (int j = 0; j < 16; ++j) {
            if (j & o) continue;
            const float give = high ? v[j] : v[j + o];
            const float got = __shfl_xor_sync(0xffffffffu, give, o);
            if (high) v[j] = got; else v[j + o] = got;
        }
    }
}

__device__ __forceinline__ void store4(float *p, float a, float b, float c, float d)
{
    *reinterpret_cast<float4 *>(p) = make_float4(a, b, c, d);
}
template <typename T>
__device__ __forceinline__ void store4(T *p, float a, float b, float c, float d)
{
    *reinterpret_cast<uint2 *>(p) = make_uint2(pack2(a, b, T()), pack2(c, d, T()));
}

struct JoinAt {
    const float *part;                   // this rank's sums, [token][128 channels]
    long long n0;
    int n_real, tile, rank;
};

// The sums of a cluster's R ranks, in rank order; four channels to a thread, eight loads in flight.
template <typename T, int R>
__device__ __forceinline__ void join(const MxArgs &a, T *Y, const JoinAt &at)
{
    constexpr int U = 8 / R;
    static_assert(X_MAX_SPLIT == 8, "ranks to join");
    const int quads = at.n_real * (X_M / 4), step = R * (int)blockDim.x;
    const size_t size = (a.b_rows - 1) * a.ldy + a.a_rows;
    for (int i0 = (int)threadIdx.x + at.rank * (int)blockDim.x; i0 < quads; i0 += U * step) {
        float4 p[U][R];
#pragma unroll
        for (int u = 0; u < U; ++u)
#pragma unroll
            for (int r = 0; r < R; ++r)
                p[u][r] = ld_dsmem_f32x4(at.part + min(i0 + u * step, quads - 1) * 4, (uint32_t)r);
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int i = i0 + u * step;
            const int t = i / (X_M / 4), c = at.tile * X_M + (i % (X_M / 4)) * 4;
            if (i >= quads || c >= a.a_rows) continue;
            float v[4] = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
            for (int r = 0; r < R; ++r)
                v[0] += p[u][r].x, v[1] += p[u][r].y, v[2] += p[u][r].z, v[3] += p[u][r].w;
            if (a.bias) {
#pragma unroll
                for (int e = 0; e < 4; ++e) v[e] += c + e < a.a_rows ? a.bias[c + e] : 0.0f;
            }
            T *const y = Y + (at.n0 + t) * a.ldy + c;
            if (a.wide) {
                if (MPQ_IN((at.n0 + t) * a.ldy + c + 3, size)) store4(y, v[0], v[1], v[2], v[3]);
                continue;
            }
#pragma unroll
            for (int e = 0; e < 4; ++e)
                if (c + e < a.a_rows && MPQ_IN((at.n0 + t) * a.ldy + c + e, size)) y[e] = from_f32<T>(v[e]);
        }
    }
}

// MANY: A is the inputs, B the weights; a cluster is a CTA pair.  Else A is the weights, B the inputs, K split
// over clusters of a.split.
template <typename T, bool MANY>
__global__ void __launch_bounds__(MANY ? 192 : X_THREADS)
mx_linear_kernel(const MxArgs a, T *Y, WaitCtl wc, const __grid_constant__ CUtensorMap tmA,
                 const __grid_constant__ CUtensorMap tmB)
{
    extern __shared__ unsigned char raw[];
    const uint32_t raw_u32 = smem_u32(raw);
    unsigned char *const base = raw + ((1024u - (raw_u32 & 1023u)) & 1023u);
    MxCtrl &ctl = *reinterpret_cast<MxCtrl *>(base);
    unsigned char *const ring = base + X_CTRL_BYTES;
    const uint32_t ring_u32 = smem_u32(ring);
    volatile int *const abort_flag = &ctl.abort;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int sb = stage_bytes(a);
    const bool cluster = MANY || a.split > 1;
    const int rank = cluster ? (int)cluster_ctarank() : 0;
    // the tile: this CTA's row tile of A, the first row of B
    const int half = MANY ? rank : 0;    // of the pair: which half of B's rows it holds
    const int group = (int)blockIdx.x / (MANY ? 2 : a.split);
    const int tile = MANY ? (group / a.n_tiles) * 2 + rank : group;
    const long long n0 = MANY ? (long long)(group % a.n_tiles) * X_N : (long long)blockIdx.y * a.n_tile;
    const int n_real = (int)min((long long)a.n_tile, a.b_rows - n0);         // rows of B that there are
    const int a_sf = tile < a.a_tiles ? 1 : 0;                       // scale tiles (per k tile) of A, of B
    const int b_sf = (n_real + 127) / 128, b_skip = (int)(n0 % 128) / 32;
    const int k0 = MANY ? 0 : (int)((long long)a.k_stages * rank / a.split);
    const int k1 = MANY ? a.k_stages : (int)((long long)a.k_stages * (rank + 1) / a.split);

    griddep_launch();
    if (threadIdx.x == 0) {
        for (int i = 0; i < a.stages; ++i) {
            mbar_init(&ctl.full[i], 1);
            mbar_init(&ctl.scaled[i], MANY ? 8 : 4);         // warps of this CTA (even CTA: of the pair)
            mbar_init(&ctl.empty[i], 1);
        }
        mbar_init(&ctl.done, 1);
        ctl.abort = 0;
        fence_barrier_init();
        if (!MPQ_CHECK_SMEM_END(ring - raw + (size_t)a.stages * sb)) ctl.abort = 1;
        prefetch_tensormap(&tmA);
        prefetch_tensormap(&tmB);
    }
    if (warp == 1) {
        if (MANY)
            tmem_alloc_pair(&ctl.tmem_base, (uint32_t)a.cols);
        else
            tmem_alloc(&ctl.tmem_base, (uint32_t)a.cols);
    }
    tc_fence_before();
    __syncthreads();
    if (MANY) cluster_sync();            // the barriers that other CTAs arrive on are ready
    tc_fence_after();
    const uint32_t tmem = ctl.tmem_base;
    griddep_wait();

    if (warp == 0) {
        // ---------------------------------------------------------------- copies
        if (lane == 0) {
            const size_t sf_a = (size_t)tile * a.k_tiles * X_SF;
            const size_t sf_b = (size_t)(n0 / 128) * a.k_tiles * X_SF;
            int issued = k0;
            for (int k = k0; k < k1 && !wc.withhold; ++k) {
                const int i = k - k0, s = i % a.stages;
                if (i >= a.stages &&
                    !mbar_wait_cluster(&ctl.empty[s], (uint32_t)(i / a.stages - 1) & 1u, wc.budget)) {
                    *abort_flag = 1;
                    note_timeout(wc, MPQ_TIMEOUT_MX);
                }
                if (*abort_flag) break;
                const uint32_t at = ring_u32 + (uint32_t)(s * sb);
                const int kt = min(2, a.k_tiles - 2 * k);            // scale tiles (along K) of this stage
                if (!MPQ_CHECK(((k * X_ROW) & 15) == 0 && (at & 1023u) == 0u && kt > 0)) {
                    *abort_flag = 1;
                    break;
                }
                const uint32_t sfs = at + (uint32_t)(X_A_BYTES + a.b_held * X_ROW);
                uint64_t *const bar = &ctl.full[s];
                mbar_arrive_expect_tx(bar, (uint32_t)(X_A_BYTES + a.b_held * X_ROW +
                                                      (a_sf + b_sf) * kt * X_SF));
                tma_load_2d(at, &tmA, k * X_ROW, tile * X_M, bar);
                tma_load_2d(at + X_A_BYTES, &tmB, k * X_ROW, (int)n0 + half * (X_N / 2), bar);
                if (a_sf)
                    bulk_load(sfs, a.a_scales + sf_a + (size_t)(2 * k) * X_SF, (uint32_t)(kt * X_SF), bar);
                for (int r = 0; r < b_sf; ++r)
                    bulk_load(sfs + (uint32_t)((2 + 2 * r) * X_SF),
                              a.b_scales + sf_b + ((size_t)r * a.k_tiles + 2 * k) * X_SF,
                              (uint32_t)(kt * X_SF), bar);
                issued = k + 1;
            }
            // no copy may land after the CTA is gone
            for (int k = max(k0, issued - a.stages); k < issued; ++k)
                drain_wait(&ctl.full[(k - k0) % a.stages], (uint32_t)((k - k0) / a.stages) & 1u, wc,
                           MPQ_TIMEOUT_MX);
            // ... nor an arrival for the pair's MMAs
            for (int k = max(k0, issued - a.stages); MANY && k < issued && !*abort_flag; ++k)
                drain_wait_cluster(&ctl.empty[(k - k0) % a.stages], (uint32_t)((k - k0) / a.stages) & 1u,
                                   wc, MPQ_TIMEOUT_MX);
        }
        __syncwarp();
    } else if (warp == 1) {
        // ---------------------------------------------------------------- MMAs
        if (lane == 0 && half == 0) {
            const int n = MANY ? X_N : (n_real + 15) / 16 * 16, m = MANY ? 2 * X_M : X_M;
            const uint32_t id0 = idesc_mxf4(m, n, 0), id2 = idesc_mxf4(m, n, 2);
            const int bc = sf_b_cols(a.n_tile);
            int s = 0;
            uint32_t phase = 0;
            for (int k = k0; k < k1 && !*abort_flag; ++k) {
                // (moved by warps that saw the stage land: both CTAs' have, for a pair)
                if (!mbar_wait_cluster(&ctl.scaled[s], phase, wc.budget)) {
                    *abort_flag = 1;
                    note_timeout(wc, MPQ_TIMEOUT_MX);
                    break;
                }
                tc_fence_after();
                const uint32_t at = ring_u32 + (uint32_t)(s * sb);
                const uint32_t ta = tmem + (uint32_t)(a.acc_cols + s * sf_cols(a.n_tile)), tb = ta + 8;
                const uint64_t ad = smem_desc_sw128(at), bd = smem_desc_sw128(at + X_A_BYTES);
                const int steps = 2 * min(2, a.k_tiles - 2 * k);
                for (int j = 0; j < steps; ++j) {
                    const uint64_t o = (uint64_t)(j * 2);            // 32 bytes, in 16 B units
                    const uint32_t id = (j & 1) ? id2 : id0, more = k > k0 || j > 0 ? 1u : 0u;
                    const uint32_t sfa = ta + 4 * (j >> 1), sfb = tb + (uint32_t)(bc * (j >> 1));
                    if (MANY)
                        mma_mxf4_pair(tmem, ad + o, bd + o, id, sfa, sfb, more);
                    else
                        mma_mxf4(tmem, ad + o, bd + o, id, sfa, sfb, more);
                }
                if (MANY)                // both CTAs load for the pair
                    mma_commit_pair(&ctl.empty[s], (uint16_t)3);
                else
                    mma_commit(&ctl.empty[s]);
                if (++s == a.stages) {
                    s = 0;
                    phase ^= 1u;
                }
            }
            // every MMA issued above completes before its sums are read or tensor memory released
            if (MANY)
                mma_commit_pair(&ctl.done, (uint16_t)3);
            else
                mma_commit(&ctl.done);
            drain_wait_cluster(&ctl.done, 0, wc, MPQ_TIMEOUT_MX);
        }
        __syncwarp();
    } else {
        // ---------------------------------------------------------------- scales
        const int q = warp & 3;
        const uint32_t quarter = tmem + ((uint32_t)(q * 32) << 16);
        if (warp < 6) {
            const int bc = sf_b_cols(a.n_tile);
            int s = 0;
            uint32_t phase = 0;
            for (int k = k0; k < k1; ++k) {
                // (a slot lands anew only when the MMAs that read its columns are done)
                if (!mbar_wait(&ctl.full[s], phase, wc.budget)) {
                    *abort_flag = 1;
                    note_timeout(wc, MPQ_TIMEOUT_MX);
                }
                if (__any_sync(0xffffffffu, *abort_flag)) break;
                const uint32_t sfs = ring_u32 + (uint32_t)(s * sb + X_A_BYTES + a.b_held * X_ROW) +
                                     (uint32_t)(lane * 16);
                const uint32_t ta = quarter + (uint32_t)(a.acc_cols + s * sf_cols(a.n_tile));
                const int kt = min(2, a.k_tiles - 2 * k);
                // lane r of every quarter holds the words of rows r, 32 + r, 64 + r and 96 + r (of B, from
                // the tile's first row on: a tile of 32 or 64 rows may begin inside a scale tile)
                auto move = [&](uint32_t to, uint32_t from, int skip) {
                    const float4 w = ld_shared_v4(from);
                    const float v[4] = {skip == 0 ? w.x : skip == 1 ? w.y : skip == 2 ? w.z : w.w,
                                        skip == 2 ? w.w : skip == 1 ? w.z : w.y, skip == 1 ? w.w : w.z, w.w};
                    tmem_st_32x32b_x4(to, v);
                };
                for (int j = 0; j < kt; ++j) {
                    move(ta + 4 * j, sfs + (uint32_t)(j * X_SF), 0);
                    for (int r = 0; r < b_sf; ++r)
                        move(ta + 8 + (uint32_t)(bc * j + 4 * r), sfs + (uint32_t)((2 + 2 * r + j) * X_SF),
                             b_skip);
                }
                tmem_wait_st();
                tc_fence_before();
                __syncwarp();
                if (lane == 0) {
                    if (MANY)
                        mbar_arrive_cluster(&ctl.scaled[s], 0);
                    else
                        mbar_arrive(&ctl.scaled[s]);
                }
                if (++s == a.stages) {
                    s = 0;
                    phase ^= 1u;
                }
            }
        }
        // ---------------------------------------------------------------- outputs
        const int i = tile * X_M + q * 32 + lane;                    // this lane's row of A
        if (!drain_wait_cluster(&ctl.done, 0, wc, MPQ_TIMEOUT_MX)) *abort_flag = 1;
        if (!__any_sync(0xffffffffu, *abort_flag)) {
            tc_fence_after();
            const float bias = !MANY && a.bias && i < a.a_rows && a.split == 1 ? a.bias[i] : 0.0f;
            float *const part = reinterpret_cast<float *>(ring) + q * 32 + lane;
            const size_t size = (MANY ? a.a_rows - 1 : a.b_rows - 1) * a.ldy + (MANY ? a.b_rows : a.a_rows);
            // the warps of a quarter share its columns by sixteens (loading the next columns ahead of the
            // stores slows both forms down: 42.3 us instead of 37.2 for 2,785 x 10,304 x 448)
            const int step = blockDim.x > 192 ? 32 : 16;
            for (int j0 = warp < 6 ? 0 : 16; j0 < n_real; j0 += step) {
                float v[16];
                __syncwarp();
                tmem_ld_32x32b_x16(quarter + (uint32_t)j0, v);
                if (MANY) {                   // row i of the inputs, 16 consecutive channels
                    const int c = (int)n0 + j0;
                    if (a.bias) {
#pragma unroll
                        for (int j = 0; j < 16; ++j) v[j] += c + j < a.b_rows ? a.bias[c + j] : 0.0f;
                    }
                    T *const y = Y + i * a.ldy + c;
                    if (c + 16 <= a.b_rows) {
                        if (i < a.a_rows && MPQ_IN(i * a.ldy + c + 15, size)) store16(y, v);
                        continue;
                    }
#pragma unroll
                    for (int j = 0; j < 16; j += 4)
                        if (i < a.a_rows && c + j < a.b_rows && MPQ_IN(i * a.ldy + c + j + 3, size))
                            store4(y + j, v[j], v[j + 1], v[j + 2], v[j + 3]);
                } else if (!MANY && a.split > 1) {   // [token][128 channels]; the ring's copies have been read
#pragma unroll
                    for (int j = 0; j < 16; ++j) part[(j0 + j) * X_M] = v[j];
                } else if (!MANY && a.wide) {   // channel i of 16 tokens: by quads of lanes, 4 channels of 4
#pragma unroll
                    for (int j = 0; j < 16; ++j) v[j] += bias;
                    quad_transpose(v, lane);
                    const int c = i & ~3;
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        const int t = j0 + 4 * j + (lane & 3);
                        if (t < n_real && c < a.a_rows && MPQ_IN((n0 + t) * a.ldy + c + 3, size))
                            store4(Y + (n0 + t) * a.ldy + c, v[4 * j], v[4 * j + 1], v[4 * j + 2], v[4 * j + 3]);
                    }
                } else if (!MANY && i < a.a_rows) {  // channel i of 16 tokens
                    T *y = Y + (n0 + j0) * a.ldy + i;
                    const int n = n_real - j0;
#pragma unroll
                    for (int j = 0; j < 16; ++j, y += a.ldy)
                        if (j < n && MPQ_IN((n0 + j0 + j) * a.ldy + i, size)) *y = from_f32<T>(v[j] + bias);
                }
            }
            tc_fence_before();
        }
    }

    if (!MANY && a.split > 1) {
        cluster_sync();                  // every rank's sums are in its shared memory
        const JoinAt at{reinterpret_cast<const float *>(ring), n0, n_real, tile, rank};
        if (a.split == 2)
            join<T, 2>(a, Y, at);
        else if (a.split == 4)
            join<T, 4>(a, Y, at);
        else
            join<T, 8>(a, Y, at);
    }
    if (cluster)
        cluster_sync();                  // no rank leaves while its sums are read, or copies to it land
    else
        __syncthreads();
    if (warp == 1) {
        tc_fence_after();
        if (MANY)
            tmem_dealloc_pair(tmem, (uint32_t)a.cols);
        else
            tmem_dealloc(tmem, (uint32_t)a.cols);
    }
}

int pow2_at_least(int n, int least)
{
    int r = least;
    while (r < n) r <<= 1;
    return r;
}

template <typename T, bool MANY>
mpq_status launch_typed(const MxArgs &a, const void *A, const void *B, int row_bytes, dim3 grid,
                        int cluster, void *Y, cudaStream_t stream)
{
    CUtensorMap tmA, tmB;
    memset(&tmA, 0, sizeof(tmA));
    memset(&tmB, 0, sizeof(tmB));
    const cuuint64_t row = (cuuint64_t)row_bytes;
    const cuuint64_t da[2] = {row, (cuuint64_t)a.a_rows}, db[2] = {row, (cuuint64_t)a.b_rows}, st[1] = {row};
    const cuuint32_t ba[2] = {X_ROW, X_M};
    const cuuint32_t bb[2] = {X_ROW, (cuuint32_t)a.b_held};
    if (!encode_tile_map(&tmA, CU_TENSOR_MAP_DATA_TYPE_UINT8, 2, A, da, st, ba,
                         CU_TENSOR_MAP_SWIZZLE_128B) ||
        !encode_tile_map(&tmB, CU_TENSOR_MAP_DATA_TYPE_UINT8, 2, B, db, st, bb,
                         CU_TENSOR_MAP_SWIZZLE_128B)) {
        set_error("mx linear: tensor map encoding failed");
        return MPQ_ERR_CUDA;
    }
    const size_t smem = 1024 + X_CTRL_BYTES + (size_t)a.stages * stage_bytes(a);
    static std::atomic<int> limit[kMaxDevices];
    cudaError_t e = allow_smem(reinterpret_cast<const void *>(mx_linear_kernel<T, MANY>), limit, smem);
    if (e != cudaSuccess) return cuda_status(e, "cudaFuncSetAttribute");
    WaitCtl wc;
    const mpq_status ws = wait_ctl(&wc);
    if (ws != MPQ_OK) return ws;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = grid;
    // eight writers pay for wide tiles (256 columns: 6.0 us instead of 7.5 for 352 x 8,128 x 448), four for
    // narrow ones whose sums are joined by all warps (37 x 11,008 x 4,096: 7.8 us instead of 8.0)
    const bool four = MANY || a.n_tile <= 16 || (a.split > 1 && a.n_tile <= 64);
    cfg.blockDim = dim3(four ? 192 : X_THREADS, 1, 1);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = stream;
    cudaLaunchAttribute attr[2];
    attr[0] = after_previous_kernel();
    attr[1].id = cudaLaunchAttributeClusterDimension;
    attr[1].val.clusterDim.x = (unsigned)cluster;
    attr[1].val.clusterDim.y = 1;
    attr[1].val.clusterDim.z = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 2;
    e = cudaLaunchKernelEx(&cfg, mx_linear_kernel<T, MANY>, a, static_cast<T *>(Y), wc, tmA, tmB);
    return cuda_status(e != cudaSuccess ? e : cudaGetLastError(), "mx linear launch");
}

// CTAs of a cluster that split the K stages of few tokens' tiles: as many as leave every CTA resident, with
// two stages or more.
int few_split(long long tiles, int n, int k_stages, int sms)
{
    const long long resident = (long long)sms * (n <= 64 ? 2 : 1);
    int split = 1;
    while (split < X_MAX_SPLIT && tiles * split * 2 <= resident && k_stages >= split * 4) split *= 2;
    return split;
}

// The rows of B in a tile where A is the weights, 32 to 256 (n_tile), or none where the pairs' form
// (`pairs`: it may be taken) is expected to be faster.  The modelled time counts, for each round of resident
// CTAs, a start, the stages by their bytes and the columns on their way out, in units of about 10 ns; CTAs
// that share an SM take longer over the last two.  The constants are fitted to 500 timings of 110 sizes
// (17 <= T <= 4,096, 64 <= C, d <= 14,000): the choice costs 1% on average, 9% at worst, against the best
// of the forms.  Some of them, us, with 32 / 64 / 128 / 256 rows / pairs: 1,233 x 448 x 448 3.9, 4.1, 4.5,
// 6.2, 5.5; 128 x 4,096 x 4,096 8.5, 7.8, 7.7, -, -; 207 x 8,960 x 7,680 34, 18.3, 17.4, 14.6, -;
// 512 x 4,096 x 4,096 21.5, 11.6, 10.9, 10.9, 12.4; 1,024 x 4,096 x 4,096 41, 22.6, 21.3, 13.5, 13.2;
// 2,785 x 10,304 x 448 90, 51, 55, 37.4, 35.5.
int few_tile(int T, int C, int k_stages, int sms, bool pairs)
{
    const long long m_tiles = ((long long)C + X_M - 1) / X_M;
    auto rounds = [](long long ctas, long long at_once) { return (double)((ctas + at_once - 1) / at_once); };
    int best = 0;
    double least = HUGE_VAL;
    if (pairs) {
        const long long ctas = ((long long)T + 2 * X_M - 1) / (2 * X_M) * (((long long)C + X_N - 1) / X_N) * 2;
        least = rounds(ctas, std::max(2, sms / 2 * 2)) * (740.0 + 22.0 * k_stages);
    }
    for (int n = X_N; n >= 32; n /= 2) {
        const int width = std::min(n, (T + 15) / 16 * 16);
        const long long tiles = m_tiles * (((long long)T + n - 1) / n);
        const int split = few_split(tiles, width, k_stages, sms);
        const int share = width <= 64 && tiles * split > sms ? 2 : 1;
        const double t = rounds(tiles * split, (long long)sms * share) *
                             (485.0 + (k_stages + split - 1) / split * (128 + width) * share / 16.0 +
                              width * share) + (split > 1 ? 20.0 : 0.0);
        if (t < least) {
            best = width;
            least = t;
        }
    }
    return best;
}

// Stages that fit into `room` bytes of shared memory, and the tensor memory columns.
void size_ring(MxArgs &a, int room)
{
    a.stages = std::min(X_MAX_STAGES, (room - 1024 - X_CTRL_BYTES) / stage_bytes(a));
    a.acc_cols = pow2_at_least(a.n_tile, 32);
    a.cols = pow2_at_least(a.acc_cols + a.stages * sf_cols(a.n_tile), 32);
}

}  // namespace

mpq_status launch_mx_linear(const mpq_mx_matrix *xl, const void *X, const mpq_mx_matrix *wl,
                            const void *W, const float *bias, void *Y, int y_type, long long ldy,
                            cudaStream_t stream)
{
    MxArgs a = {};
    a.k_tiles = wl->k_tiles;
    a.k_stages = (wl->k_tiles + 1) / 2;
    a.bias = bias;
    a.ldy = ldy;
    const unsigned char *const x = static_cast<const unsigned char *>(X);
    const unsigned char *const w = static_cast<const unsigned char *>(W);
    const int T = xl->rows, C = wl->rows, sms = sm_count();
    const int four = 4 * type_size(y_type);
    a.wide = C % 4 == 0 && ldy % 4 == 0 && (uintptr_t)Y % four == 0;
    // (the pairs' writers hold 16 channels of a token each: 256 x 250 outputs, one by one, took 30 us)
    const int n = few_tile(T, C, a.k_stages, sms, T > X_N && a.wide && rows_aligned(Y, y_type, ldy));
    if (n == 0) {
        const long long n_cl = ((long long)C + X_N - 1) / X_N;
        const long long ctas = ((long long)T + 2 * X_M - 1) / (2 * X_M) * n_cl * 2;
        a.a_rows = T;
        a.b_rows = C;
        a.a_tiles = xl->row_tiles;
        a.a_scales = x + xl->off_scales;
        a.b_scales = w + wl->off_scales;
        a.n_tile = X_N;
        a.b_held = X_N / 2;
        a.split = 1;
        a.n_tiles = (int)n_cl;
        size_ring(a, max_smem_optin());
        if (ctas > 0x7fffffffLL) {
            set_error("mx linear: T = %d, C = %d are too large", T, C);
            return MPQ_ERR_UNSUPPORTED;
        }
        return by_type(y_type, [&](auto t) {
            return launch_typed<decltype(t), true>(a, X, W, wl->d_pad / 2, dim3((unsigned)ctas), 2, Y,
                                                   stream);
        });
    }
    a.a_rows = C;
    a.b_rows = T;
    a.a_tiles = wl->row_tiles;
    a.a_scales = w + wl->off_scales;
    a.b_scales = x + xl->off_scales;
    const long long m_tiles = ((long long)C + X_M - 1) / X_M;
    a.n_tile = a.b_held = n;
    // two CTAs share an SM where a ring of four stages leaves room for it (up to 64 tokens)
    const bool two = a.n_tile <= 64;
    size_ring(a, two ? 112 * 1024 : max_smem_optin());
    const long long n_tiles = ((long long)T + a.n_tile - 1) / a.n_tile;
    a.split = few_split(m_tiles * n_tiles, a.n_tile, a.k_stages, sms);
    if (n_tiles > 65535 || m_tiles * a.split > 0x7fffffffLL) {
        set_error("mx linear: T = %d, C = %d are too large", T, C);
        return MPQ_ERR_UNSUPPORTED;
    }
    return by_type(y_type, [&](auto t) {
        return launch_typed<decltype(t), false>(a, W, X, wl->d_pad / 2,
                                                dim3((unsigned)(m_tiles * a.split), (unsigned)n_tiles),
                                                a.split, Y, stream);
    });
}

}  // namespace mpq
