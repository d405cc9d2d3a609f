// Linear layer of microscaled 4-bit floats (mpq_mx_linear): Y[t][c] = sum_j x_tj w_cj + bias_c on the
// tensor cores' block-scaled MMAs (tcgen05.mma kind::mxf4).
//
// The weights' 128-channel row tiles are the MMA's A (M = 128), the tokens its B (N = 16 .. 256), so a
// handful of tokens costs no padding to 128.  A K stage is 256 elements: 128-byte rows of codes, as
// they lie in memory, by TMA into 128-byte-swizzled K-major tiles, and the scales of both, 512
// contiguous bytes per 128 rows x 128 elements, by bulk copies; one thread moves the scales from
// shared to tensor memory (each stage has columns of its own, reused when its MMAs are done) and
// issues the MMAs.  Accumulators are fp32 in tensor memory, one rounding (after the bias) on the way
// out.
//
// With few tokens the weights' bytes bound it (d / 2 + d / 32 a channel), and with few row tiles most
// SMs would idle: the K stages of a tile are then split over the CTAs of a cluster, which leave their
// sums in shared memory and join them there in the order of the ranks (so equal inputs give equal
// bits).  With many tokens shared-memory reads of the MMAs bound it: 128 + N rows of 32 bytes for 64
// elements of K, which 128 x 256 tiles bring to 3/4 of the 128 x 128 ones' per product.
//
// Roles: warp 0 copies, warp 1 issues MMAs, warps 2..5 (TMEM lane quarter warp % 4) write the outputs.
// Every wait is bounded.
#include <cuda.h>
#include <math.h>
#include <string.h>

#include <algorithm>

#include "elements.cuh"
#include "mpq_internal.cuh"
#include "pair_common.cuh"
#include "sm100.cuh"
#include "waits.cuh"

MPQ_CHECKED_UNIT("mx_linear.cu");

namespace mpq {
namespace {

using namespace sm100;

constexpr int X_M = 128;                 // channels of a tile
constexpr int X_N = 256;                 // most tokens of a tile
constexpr int X_ROW = 128;               // bytes of a row's codes in a stage: 256 elements
constexpr int X_SF = 512;                // bytes of a scale tile (128 rows x 128 elements)
constexpr int X_A_BYTES = X_M * X_ROW;
constexpr int X_MAX_STAGES = 8;
constexpr int X_THREADS = 192;
constexpr int X_MAX_SPLIT = 8;           // CTAs of a cluster

struct MxCtrl {
    uint64_t full[X_MAX_STAGES];         // a stage's tiles and scales have landed
    uint64_t empty[X_MAX_STAGES];        // the MMAs that read a stage completed
    uint64_t done;                       // every MMA completed
    uint32_t tmem_base;
    int abort;
};
constexpr int X_CTRL_BYTES = 1024;
static_assert(sizeof(MxCtrl) <= X_CTRL_BYTES, "control block");

struct MxArgs {
    int T, C;
    int n_tile;                          // tokens of a tile, a multiple of 16
    int stages, k_stages, k_tiles;       // ring, K stages of a row, scale tiles of a row
    int split;                           // CTAs that share a tile's K stages
    int acc_cols, cols;                  // TMEM columns: the accumulator's (scales follow), all
    const unsigned char *w_scales, *x_scales;
    const float *bias;
    long long ldy;
};

__host__ __device__ inline int sf_b_bytes(int n_tile) { return n_tile > 128 ? 4 * X_SF : 2 * X_SF; }
__host__ __device__ inline int stage_bytes(int n_tile)
{
    return X_A_BYTES + n_tile * X_ROW + 2 * X_SF + sf_b_bytes(n_tile);
}

template <typename T>
__global__ void __launch_bounds__(X_THREADS)
mx_linear_kernel(const MxArgs a, T *Y, WaitCtl wc, const __grid_constant__ CUtensorMap tmW,
                 const __grid_constant__ CUtensorMap tmX)
{
    extern __shared__ unsigned char raw[];
    const uint32_t raw_u32 = smem_u32(raw);
    unsigned char *const base = raw + ((1024u - (raw_u32 & 1023u)) & 1023u);
    MxCtrl &ctl = *reinterpret_cast<MxCtrl *>(base);
    unsigned char *const ring = base + X_CTRL_BYTES;
    const uint32_t ring_u32 = smem_u32(ring);
    volatile int *const abort_flag = &ctl.abort;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int sb = stage_bytes(a.n_tile);
    const int rank = a.split > 1 ? (int)cluster_ctarank() : 0;
    const int tile = (int)blockIdx.x / a.split;
    const long long n0 = (long long)blockIdx.y * a.n_tile;
    const int n_real = (int)min((long long)a.n_tile, a.T - n0);      // tokens of this tile
    const int k0 = (int)((long long)a.k_stages * rank / a.split);
    const int k1 = (int)((long long)a.k_stages * (rank + 1) / a.split);

    griddep_launch();
    if (threadIdx.x == 0) {
        for (int i = 0; i < a.stages; ++i) {
            mbar_init(&ctl.full[i], 1);
            mbar_init(&ctl.empty[i], 1);
        }
        mbar_init(&ctl.done, 1);
        ctl.abort = 0;
        fence_barrier_init();
        if (!MPQ_CHECK_SMEM_END(ring - raw + (size_t)a.stages * sb)) ctl.abort = 1;
        prefetch_tensormap(&tmW);
        prefetch_tensormap(&tmX);
    }
    if (warp == 1) tmem_alloc(&ctl.tmem_base, (uint32_t)a.cols);
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = ctl.tmem_base;
    griddep_wait();

    if (warp == 0) {
        // ---------------------------------------------------------------- copies
        if (lane == 0) {
            const int row_tiles = (n_real + 127) / 128;              // of the tokens' scales
            const size_t sf_a = (size_t)tile * a.k_tiles * X_SF;
            const size_t sf_b = (size_t)(n0 / 128) * a.k_tiles * X_SF;
            int issued = k0;
            for (int k = k0; k < k1; ++k) {
                const int i = k - k0, s = i % a.stages;
                if (i >= a.stages &&
                    !mbar_wait(&ctl.empty[s], (uint32_t)(i / a.stages - 1) & 1u, wc.budget)) {
                    *abort_flag = 1;
                    note_timeout(wc, MPQ_TIMEOUT_MX);
                }
                if (*abort_flag) break;
                const uint32_t at = ring_u32 + (uint32_t)(s * sb);
                const int kt = min(2, a.k_tiles - 2 * k);            // scale tiles of this stage
                if (!MPQ_CHECK(((k * X_ROW) & 15) == 0 && (at & 1023u) == 0u && kt > 0)) {
                    *abort_flag = 1;
                    break;
                }
                const uint32_t sfs = at + (uint32_t)(X_A_BYTES + a.n_tile * X_ROW);
                mbar_arrive_expect_tx(&ctl.full[s], (uint32_t)(X_A_BYTES + a.n_tile * X_ROW +
                                                               (1 + row_tiles) * kt * X_SF));
                tma_load_2d(at, &tmW, k * X_ROW, tile * X_M, &ctl.full[s]);
                tma_load_2d(at + X_A_BYTES, &tmX, k * X_ROW, (int)n0, &ctl.full[s]);
                bulk_load(sfs, a.w_scales + sf_a + (size_t)(2 * k) * X_SF, (uint32_t)(kt * X_SF),
                          &ctl.full[s]);
                for (int r = 0; r < row_tiles; ++r)
                    bulk_load(sfs + (uint32_t)((2 + 2 * r) * X_SF),
                              a.x_scales + sf_b + ((size_t)r * a.k_tiles + 2 * k) * X_SF,
                              (uint32_t)(kt * X_SF), &ctl.full[s]);
                issued = k + 1;
            }
            // no copy may land after the CTA is gone
            for (int k = max(k0, issued - a.stages); k < issued; ++k)
                drain_wait(&ctl.full[(k - k0) % a.stages], (uint32_t)((k - k0) / a.stages) & 1u, wc,
                           MPQ_TIMEOUT_MX);
        }
        __syncwarp();
    } else if (warp == 1) {
        // ---------------------------------------------------------------- MMAs
        if (lane == 0) {
            const int n = (n_real + 15) / 16 * 16;
            const int row_tiles = (n_real + 127) / 128;
            const uint32_t id0 = idesc_mxf4(X_M, n, 0), id2 = idesc_mxf4(X_M, n, 2);
            const int sf_cols = 8 + 8 * (a.n_tile > 128 ? 2 : 1);    // of a stage
            for (int k = k0; k < k1 && !*abort_flag; ++k) {
                const int i = k - k0, s = i % a.stages;
                if (!mbar_wait(&ctl.full[s], (uint32_t)(i / a.stages) & 1u, wc.budget)) {
                    *abort_flag = 1;
                    note_timeout(wc, MPQ_TIMEOUT_MX);
                    break;
                }
                tc_fence_after();
                const uint32_t at = ring_u32 + (uint32_t)(s * sb);
                const uint32_t sfs = at + (uint32_t)(X_A_BYTES + a.n_tile * X_ROW);
                const uint32_t ta = tmem + (uint32_t)(a.acc_cols + s * sf_cols), tb = ta + 8;
                const int kt = min(2, a.k_tiles - 2 * k);
                for (int j = 0; j < kt; ++j) {
                    tmem_copy_scales(ta + 4 * j, sfs + (uint32_t)(j * X_SF));
                    for (int r = 0; r < row_tiles; ++r)
                        tmem_copy_scales(tb + (uint32_t)((a.n_tile > 128 ? 8 : 4) * j + 4 * r),
                                         sfs + (uint32_t)((2 + 2 * r + j) * X_SF));
                }
                const uint64_t ad = smem_desc_sw128(at), bd = smem_desc_sw128(at + X_A_BYTES);
                for (int j = 0; j < 2 * kt; ++j) {
                    const uint64_t o = (uint64_t)(j * 2);            // 32 bytes, in 16 B units
                    mma_mxf4(tmem, ad + o, bd + o, (j & 1) ? id2 : id0, ta + 4 * (j >> 1),
                             tb + (uint32_t)((a.n_tile > 128 ? 8 : 4) * (j >> 1)),
                             i > 0 || j > 0 ? 1u : 0u);
                }
                mma_commit(&ctl.empty[s]);
            }
            // every MMA issued above completes before its sums are read or tensor memory released
            mma_commit(&ctl.done);
            drain_wait(&ctl.done, 0, wc, MPQ_TIMEOUT_MX);
        }
        __syncwarp();
    } else {
        // ---------------------------------------------------------------- outputs
        const int q = warp & 3, c = tile * X_M + q * 32 + lane;
        if (!drain_wait(&ctl.done, 0, wc, MPQ_TIMEOUT_MX)) *abort_flag = 1;
        if (!__any_sync(0xffffffffu, *abort_flag)) {
            tc_fence_after();
            const uint32_t from = tmem + ((uint32_t)(q * 32) << 16);
            const float bias = a.bias && c < a.C && a.split == 1 ? a.bias[c] : 0.0f;
            float *const part = reinterpret_cast<float *>(ring) + q * 32 + lane;
            for (int j0 = 0; j0 < n_real; j0 += 16) {
                float v[16];
                tmem_ld_32x32b_x16(from + (uint32_t)j0, v);
                if (a.split > 1) {       // [token][128 channels]; the ring's copies have been read
#pragma unroll
                    for (int j = 0; j < 16; ++j) part[(j0 + j) * X_M] = v[j];
                } else if (c < a.C) {
                    T *y = Y + (n0 + j0) * a.ldy + c;
#pragma unroll
                    for (int j = 0; j < 16; ++j)
                        if (j0 + j < n_real &&
                            MPQ_IN((n0 + j0 + j) * a.ldy + c, (a.T - 1) * a.ldy + a.C))
                            y[j * a.ldy] = from_f32<T>(v[j] + bias);
                }
            }
            tc_fence_before();
        }
    }

    if (a.split > 1) {
        cluster_sync();                  // every rank's sums are in its shared memory
        const float *const part = reinterpret_cast<const float *>(ring);
        const int quads = n_real * (X_M / 4);
        for (int i = (int)threadIdx.x + rank * X_THREADS; i < quads; i += a.split * X_THREADS) {
            const int t = i / (X_M / 4), cc = (i % (X_M / 4)) * 4, c = tile * X_M + cc;
            if (c >= a.C) continue;
            float v[4] = {0.0f, 0.0f, 0.0f, 0.0f};
            for (int r = 0; r < a.split; ++r) {
                const float4 p = ld_dsmem_f32x4(part + t * X_M + cc, (uint32_t)r);
                v[0] += p.x, v[1] += p.y, v[2] += p.z, v[3] += p.w;
            }
            T *y = Y + (n0 + t) * a.ldy + c;
#pragma unroll
            for (int e = 0; e < 4; ++e)
                if (c + e < a.C && MPQ_IN((n0 + t) * a.ldy + c + e, (a.T - 1) * a.ldy + a.C))
                    y[e] = from_f32<T>(v[e] + (a.bias ? a.bias[c + e] : 0.0f));
        }
        cluster_sync();                  // no rank leaves while its sums are read
    } else {
        __syncthreads();
    }
    if (warp == 1) {
        tc_fence_after();
        tmem_dealloc(tmem, (uint32_t)a.cols);
    }
}

int pow2_at_least(int n, int least)
{
    int r = least;
    while (r < n) r <<= 1;
    return r;
}

template <typename T>
mpq_status launch_typed(MxArgs &a, const mpq_mx_matrix *xl, const void *X, const mpq_mx_matrix *wl,
                        const void *W, void *Y, cudaStream_t stream)
{
    CUtensorMap tmW, tmX;
    memset(&tmW, 0, sizeof(tmW));
    memset(&tmX, 0, sizeof(tmX));
    const cuuint64_t row = (cuuint64_t)(wl->d_pad / 2);
    const cuuint64_t dw[2] = {row, (cuuint64_t)a.C}, dx[2] = {row, (cuuint64_t)a.T}, st[1] = {row};
    const cuuint32_t bw[2] = {X_ROW, X_M}, bx[2] = {X_ROW, (cuuint32_t)a.n_tile};
    if (!encode_tile_map(&tmW, CU_TENSOR_MAP_DATA_TYPE_UINT8, 2, W, dw, st, bw,
                         CU_TENSOR_MAP_SWIZZLE_128B) ||
        !encode_tile_map(&tmX, CU_TENSOR_MAP_DATA_TYPE_UINT8, 2, X, dx, st, bx,
                         CU_TENSOR_MAP_SWIZZLE_128B)) {
        set_error("mx linear: tensor map encoding failed");
        return MPQ_ERR_CUDA;
    }
    const size_t smem = 1024 + X_CTRL_BYTES + (size_t)a.stages * stage_bytes(a.n_tile);
    static std::atomic<int> limit[kMaxDevices];
    cudaError_t e = allow_smem(reinterpret_cast<const void *>(mx_linear_kernel<T>), limit, smem);
    if (e != cudaSuccess) return cuda_status(e, "cudaFuncSetAttribute");
    WaitCtl wc;
    const mpq_status ws = wait_ctl(&wc);
    if (ws != MPQ_OK) return ws;
    const long long tiles = ((long long)a.C + X_M - 1) / X_M;
    const long long token_tiles = ((long long)a.T + a.n_tile - 1) / a.n_tile;
    if (token_tiles > 65535) {
        set_error("mx linear: T = %d is too large", a.T);
        return MPQ_ERR_UNSUPPORTED;
    }
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)(tiles * a.split), (unsigned)token_tiles, 1);
    cfg.blockDim = dim3(X_THREADS, 1, 1);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = stream;
    cudaLaunchAttribute attr[2];
    attr[0] = after_previous_kernel();
    attr[1].id = cudaLaunchAttributeClusterDimension;
    attr[1].val.clusterDim.x = (unsigned)a.split;
    attr[1].val.clusterDim.y = 1;
    attr[1].val.clusterDim.z = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 2;
    e = cudaLaunchKernelEx(&cfg, mx_linear_kernel<T>, (const MxArgs)a, static_cast<T *>(Y), wc, tmW,
                           tmX);
    return cuda_status(e != cudaSuccess ? e : cudaGetLastError(), "mx linear launch");
}

}  // namespace

mpq_status launch_mx_linear(const mpq_mx_matrix *xl, const void *X, const mpq_mx_matrix *wl,
                            const void *W, const float *bias, void *Y, int y_type, long long ldy,
                            cudaStream_t stream)
{
    MxArgs a = {};
    a.T = xl->rows;
    a.C = wl->rows;
    a.n_tile = a.T >= X_N ? X_N : (a.T + 15) / 16 * 16;
    a.k_tiles = wl->k_tiles;
    a.k_stages = (wl->k_tiles + 1) / 2;
    a.w_scales = static_cast<const unsigned char *>(W) + wl->off_scales;
    a.x_scales = static_cast<const unsigned char *>(X) + xl->off_scales;
    a.bias = bias;
    a.ldy = ldy;
    // two CTAs share an SM where a ring of four stages leaves room for it (up to 64 tokens)
    const int sb = stage_bytes(a.n_tile);
    const bool two = a.n_tile <= 64;
    const int room = two ? 112 * 1024 : max_smem_optin();
    a.stages = std::min(X_MAX_STAGES, (room - 2048) / sb);
    a.acc_cols = pow2_at_least(a.n_tile, 32);
    a.cols = pow2_at_least(a.acc_cols + a.stages * (a.n_tile > 128 ? 24 : 16), 32);
    // clusters split the K stages while every CTA stays resident and has two stages or more
    const long long tiles = ((long long)a.C + X_M - 1) / X_M * ((a.T + a.n_tile - 1LL) / a.n_tile);
    const long long resident = (long long)sm_count() * (two ? 2 : 1);
    a.split = 1;
    while (a.split < X_MAX_SPLIT && tiles * a.split * 2 <= resident &&
           a.k_stages >= a.split * 4)
        a.split *= 2;
    return by_type(y_type, [&](auto t) {
        return launch_typed<decltype(t)>(a, xl, X, wl, W, Y, stream);
    });
}

}  // namespace mpq
