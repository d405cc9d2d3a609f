// Linear layer of weights in 4-bit integers (mpq_g4_linear): Y[t][c] = sum_j x_tj w_cj + bias_c, w = s (q - z) with
// s and z by groups of a row, rounded once to x's type.  (bf16 rounds the weight by 2^-9 of it at most, fp16 by
// 2^-12, beside the 1/30 of a group's largest that its codes are apart: what that buys is one sum over all of K, in
// the tensor cores' fp32.)  Many tokens: g4_tiles.cu.
//
// A few tokens, warp-level MMAs (m16n8k16): a tile's 16 rows are A, eight tokens B.  A lane's 16 bytes of a row hold,
// for each 32 elements, the eight that it multiplies in two MMAs: the codes become A's registers where they are,
// and x's registers are 16 consecutive bytes of its row.  Warps of a CTA take a row tile's tiles in turn and
// their sums are joined in shared memory in the warps' order.
#include <math.h>

#include <algorithm>

#include "g4.cuh"
#include "sm100.cuh"

MPQ_CHECKED_UNIT("g4_linear.cu");

namespace mpq {
namespace {

constexpr int FEW_WARPS = 8;
constexpr int FEW_TOKENS = 16;

template <typename T>
__device__ __forceinline__ void mma16816(float (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3,
                                         uint32_t b0, uint32_t b1)
{
    if constexpr (G4Pairs<T>::kBf16)
        asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, "
                     "{%8, %9}, {%0, %1, %2, %3};"
                     : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
                     : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
    else
        asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, "
                     "{%8, %9}, {%0, %1, %2, %3};"
                     : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
                     : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}

struct G4Args {
    mpq_g4_matrix L;
    const unsigned char *w;
    const float *bias;
    long long ldx, ldy;
    int T, y_type;
};

__device__ __forceinline__ void store_as(void *Y, int type, long long at, float v)
{
    if (type == MPQ_F32) static_cast<float *>(Y)[at] = v;
    else if (type == MPQ_F16) static_cast<__half *>(Y)[at] = from_f32<__half>(v);
    else static_cast<__nv_bfloat16 *>(Y)[at] = from_f32<__nv_bfloat16>(v);
}

// x's eight elements from p + j on, zeros from d on.
template <typename T, bool VEC>
__device__ __forceinline__ uint4 load_x(const T *p, int j, int d)
{
    if (VEC) return j < d ? *reinterpret_cast<const uint4 *>(p + j) : make_uint4(0, 0, 0, 0);
    const uint16_t *const h = reinterpret_cast<const uint16_t *>(p);
    uint32_t w[4];
#pragma unroll
    for (int i = 0; i < 4; ++i)
        w[i] = (j + 2 * i < d ? h[j + 2 * i] : 0u) | (j + 2 * i + 1 < d ? h[j + 2 * i + 1] : 0u) << 16;
    return make_uint4(w[0], w[1], w[2], w[3]);
}

// NT: tiles of eight tokens; GROUP: elements of a group; VEC: x's rows are 16-byte aligned, d a multiple of 8.
template <typename T, int NT, int GROUP, bool VEC>
__global__ void __launch_bounds__(FEW_WARPS * 32)
g4_few_kernel(const G4Args a, const T *X, void *Y)
{
    constexpr int N = 128 / GROUP;           // groups of a tile's row
    __shared__ float part[FEW_WARPS][NT * 8][17];
    sm100::griddep_launch();
    sm100::griddep_wait();
    const int warp = (int)threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, i = lane & 3;
    const long long n0 = (long long)blockIdx.y * (NT * 8);
    const unsigned char *const strip = a.w + (size_t)blockIdx.x * a.L.k_tiles * a.L.tile_bytes;
    float acc[NT][4];
#pragma unroll
    for (int n = 0; n < NT; ++n)
#pragma unroll
        for (int e = 0; e < 4; ++e) acc[n][e] = 0.0f;
    for (int kt = warp; kt < a.L.k_tiles; kt += FEW_WARPS) {
        const unsigned char *const tile = strip + (size_t)kt * a.L.tile_bytes;
        const uint4 wa = *reinterpret_cast<const uint4 *>(tile + g * 64 + i * 16);
        const uint4 wb = *reinterpret_cast<const uint4 *>(tile + (g + 8) * 64 + i * 16);
        const uint32_t qa[4] = {wa.x, wa.y, wa.z, wa.w}, qb[4] = {wb.x, wb.y, wb.z, wb.w};
        const uint16_t *const sc = reinterpret_cast<const uint16_t *>(tile + G4_CODES);
        const unsigned char *const zs = tile + G4_CODES + 32 * N;
        G4Scale ga, gb;
#pragma unroll
        for (int m = 0; m < 4; ++m) {
            if (m * 32 % GROUP == 0) {
                const int at = m * 32 / GROUP;
                ga = g4_scale<T>(sc[g * N + at], a.L.zeros ? zs[g * N + at] : G4_ZERO);
                gb = g4_scale<T>(sc[(g + 8) * N + at], a.L.zeros ? zs[(g + 8) * N + at] : G4_ZERO);
            }
            uint32_t pa[4], pb[4];
            g4_values<T>(qa[m], ga, pa);
            g4_values<T>(qb[m], gb, pb);
#pragma unroll
            for (int n = 0; n < NT; ++n) {
                const long long t = n0 + n * 8 + g;
                uint4 x = make_uint4(0, 0, 0, 0);
                if (t < a.T) x = load_x<T, VEC>(X + t * a.ldx, kt * 128 + m * 32 + i * 8, a.L.d);
                mma16816<T>(acc[n], pa[0], pb[0], pa[1], pb[1], x.x, x.y);
                mma16816<T>(acc[n], pa[2], pb[2], pa[3], pb[3], x.z, x.w);
            }
        }
    }
    // rows g and g + 8 of tokens 2 i and 2 i + 1
#pragma unroll
    for (int n = 0; n < NT; ++n)
#pragma unroll
        for (int e = 0; e < 4; ++e) part[warp][n * 8 + 2 * i + (e & 1)][g + (e >> 1) * 8] = acc[n][e];
    __syncthreads();
    for (int o = (int)threadIdx.x; o < NT * 8 * 16; o += FEW_WARPS * 32) {
        const int n = o >> 4, r = o & 15, c = (int)blockIdx.x * 16 + r;
        const long long t = n0 + n;
        if (t >= a.T || c >= a.L.rows) continue;
        float v = 0.0f;
#pragma unroll
        for (int w = 0; w < FEW_WARPS; ++w) v += part[w][n][r];
        if (a.bias) v += a.bias[c];
        if (MPQ_IN(t * a.ldy + c, (a.T - 1) * a.ldy + a.L.rows)) store_as(Y, a.y_type, t * a.ldy + c, v);
    }
}

template <typename T, int NT, bool VEC>
mpq_status launch_few(const G4Args &a, const T *X, void *Y, cudaStream_t stream)
{
    const dim3 grid((unsigned)a.L.row_tiles, (unsigned)((a.T + NT * 8 - 1) / (NT * 8)));
    auto *const kernel = a.L.group == 32   ? g4_few_kernel<T, NT, 32, VEC>
                         : a.L.group == 64 ? g4_few_kernel<T, NT, 64, VEC>
                                           : g4_few_kernel<T, NT, 128, VEC>;
    return launch_waiting(kernel, grid, dim3(FEW_WARPS * 32), 0, stream, "g4 linear launch", a, X, Y);
}

template <typename T>
mpq_status launch_typed(const G4Args &a, const T *X, int x_type, void *Y, cudaStream_t stream)
{
    const bool vec = rows_aligned(X, x_type, a.T > 1 ? a.ldx : 0) && a.L.d % 8 == 0;
    if (a.T <= 8) return vec ? launch_few<T, 1, true>(a, X, Y, stream) : launch_few<T, 1, false>(a, X, Y, stream);
    return vec ? launch_few<T, 4, true>(a, X, Y, stream) : launch_few<T, 4, false>(a, X, Y, stream);
}

}  // namespace

mpq_status launch_g4_linear(const void *X, int x_type, long long ldx, int T, const mpq_g4_matrix *L,
                            const void *W, const float *bias, void *Y, int y_type, long long ldy,
                            cudaStream_t stream)
{
    if (T > FEW_TOKENS) return launch_g4_tiles(X, x_type, ldx, T, L, W, bias, Y, y_type, ldy, stream);
    const G4Args a = {*L, static_cast<const unsigned char *>(W), bias, ldx, ldy, T, y_type};
    if (x_type == MPQ_F16) return launch_typed(a, static_cast<const __half *>(X), x_type, Y, stream);
    return launch_typed(a, static_cast<const __nv_bfloat16 *>(X), x_type, Y, stream);
}

}  // namespace mpq
