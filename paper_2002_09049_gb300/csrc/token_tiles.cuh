// The way out of a linear layer's tiles whose accumulators hold 128 channels on the tensor memory's lanes and
// tokens on its columns (mx_linear.cu, g4_tiles.cu): outputs by quads of channels, and the sums of a cluster
// that shares a tile's K, joined in the order of its ranks.
#pragma once

#include <algorithm>
#include <atomic>

#include "elements.cuh"
#include "mpq_internal.cuh"
#include "mx_ops.cuh"

namespace mpq {

constexpr int TOKEN_M = 128;             // channels of a tile
constexpr int TOKEN_MAX_SPLIT = 8;       // CTAs of a cluster that splits K

// tcgen05.alloc waits until the columns that it asks for are free, without a limit.  So CTAs whose columns do not fit
// beside one another must not come to one SM: two clusters that each hold what the other's CTA waits for would never
// end, nor would a kernel launched ahead that holds what the one before it waits for.  Shared memory keeps them apart: a
// CTA that takes more than half of the columns asks for TOKEN_ALONE_SMEM or more, one that takes half or less for
// TOKEN_HALF_SMEM or more, which two of them leave no third and none of the others room beside.  (The SM keeps
// 1 KB a CTA for itself.)
constexpr size_t TOKEN_SM_SMEM = 228 * 1024, TOKEN_KEPT_SMEM = 1024;
constexpr size_t TOKEN_HALF_SMEM = 96 * 1024, TOKEN_ALONE_SMEM = 132 * 1024;
constexpr int TOKEN_COLS = 512;          // columns of tensor memory
static_assert(TOKEN_ALONE_SMEM + TOKEN_HALF_SMEM + 2 * TOKEN_KEPT_SMEM > TOKEN_SM_SMEM, "one alone and half");
static_assert(3 * (TOKEN_HALF_SMEM + TOKEN_KEPT_SMEM) > TOKEN_SM_SMEM, "three halves");

// What a launch asks for: `smem` bytes and `cols` columns are what its CTA uses.
inline size_t token_smem(size_t smem, int cols)
{
    return std::max(smem, 2 * cols > TOKEN_COLS ? TOKEN_ALONE_SMEM : TOKEN_HALF_SMEM);
}
// Refuses a device whose SMs have other shared memory than this reckons with.
inline mpq_status token_check_sm()
{
    static std::atomic<int> good[kMaxDevices];
    int dev = 0, most = 0, kept = 0;
    cudaError_t e = cudaGetDevice(&dev);
    if (e == cudaSuccess && dev < kMaxDevices && good[dev].load(std::memory_order_relaxed)) return MPQ_OK;
    if (e == cudaSuccess) e = cudaDeviceGetAttribute(&most, cudaDevAttrMaxSharedMemoryPerMultiprocessor, dev);
    if (e == cudaSuccess) e = cudaDeviceGetAttribute(&kept, cudaDevAttrReservedSharedMemoryPerBlock, dev);
    if (e != cudaSuccess) return cuda_status(e, "shared memory of an SM");
    if ((size_t)most > TOKEN_SM_SMEM || (size_t)kept < TOKEN_KEPT_SMEM) {
        set_error("SMs of %d bytes of shared memory, %d kept a CTA, are not supported", most, kept);
        return MPQ_ERR_UNSUPPORTED;
    }
    if (dev < kMaxDevices) good[dev].store(1, std::memory_order_relaxed);
    return MPQ_OK;
}

// Outputs [tokens][channels], rows ldy apart; wide: they take 4 at a time.
struct TokenRows {
    int tokens, channels, wide;
    const float *bias;
    long long ldy;
};

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

// The sums of a cluster's R ranks, in rank order; four channels to a thread, eight loads in flight.  WHOLE: a thread's
// loads past the last are of the last again, so that none of them waits for a comparison.  The microscaled layer's up to
// 320 threads have few such (75 x 4,096 x 11,008, T x C x d, 9.9 us instead of 10.05, 256 x 4,096 x 4,096 8.5 instead
// of 9.1); of the 896 that the 4-bit integer layer has, most would load for nothing (75 x 4,096 x 11,008 14.4 us instead of
// 14.2, 500 x 1,024 x 4,096 10.8 instead of 10.55).
template <typename T, int R, bool WHOLE>
__device__ __forceinline__ void join(const TokenRows &a, T *Y, const JoinAt &at)
{
    constexpr int U = 8 / R;
    static_assert(TOKEN_MAX_SPLIT == 8, "ranks to join");
    const int quads = at.n_real * (TOKEN_M / 4), step = R * (int)blockDim.x;
    const size_t size = (a.tokens - 1) * a.ldy + a.channels;
    for (int i0 = (int)threadIdx.x + at.rank * (int)blockDim.x; i0 < quads; i0 += U * step) {
        float4 p[U][R];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int i = i0 + u * step;
            if (!WHOLE && i >= quads) break;
#pragma unroll
            for (int r = 0; r < R; ++r)
                p[u][r] = sm100::ld_dsmem_f32x4(at.part + (WHOLE ? min(i, quads - 1) : i) * 4, (uint32_t)r);
        }
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int i = i0 + u * step;
            if (!WHOLE && i >= quads) break;
            const int t = i / (TOKEN_M / 4), c = at.tile * TOKEN_M + (i % (TOKEN_M / 4)) * 4;
            if (i >= quads || c >= a.channels) continue;
            float v[4] = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
            for (int r = 0; r < R; ++r)
                v[0] += p[u][r].x, v[1] += p[u][r].y, v[2] += p[u][r].z, v[3] += p[u][r].w;
            if (a.bias) {
#pragma unroll
                for (int e = 0; e < 4; ++e) v[e] += c + e < a.channels ? a.bias[c + e] : 0.0f;
            }
            T *const y = Y + (at.n0 + t) * a.ldy + c;
            if (a.wide) {
                if (MPQ_IN((at.n0 + t) * a.ldy + c + 3, size)) store4(y, v[0], v[1], v[2], v[3]);
                continue;
            }
#pragma unroll
            for (int e = 0; e < 4; ++e)
                if (c + e < a.channels && MPQ_IN((at.n0 + t) * a.ldy + c + e, size)) y[e] = from_f32<T>(v[e]);
        }
    }
}

template <bool WHOLE, typename T>
__device__ __forceinline__ void join_split(const TokenRows &a, T *Y, const JoinAt &at, int split)
{
    if (split == 2)
        join<T, 2, WHOLE>(a, Y, at);
    else if (split == 4)
        join<T, 4, WHOLE>(a, Y, at);
    else
        join<T, 8, WHOLE>(a, Y, at);
}

}  // namespace mpq
