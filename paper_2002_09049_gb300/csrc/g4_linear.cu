// Linear layer of weights in 4-bit integers (mpq_g4_linear): Y[t][c] = sum_j x_tj w_cj + bias_c, w = s (q - z) with
// s and z by groups of a row, rounded once to x's type.  (bf16 rounds the weight by 2^-9 of it at most, fp16 by
// 2^-12, beside the 1/30 of a group's largest that its codes are apart: what that buys is one sum over all of K, in
// the tensor cores' fp32.)  Many tokens: g4_tiles.cu.
//
// A few tokens, warp-level MMAs (m16n8k16): a tile's 16 rows are A, eight tokens B.  A lane's 16 bytes of a row hold,
// for each 32 elements, the eight that it multiplies in two MMAs: the codes become A's registers where they are,
// and x's registers are 16 consecutive bytes of its row.  Warps of a CTA take a row tile's tiles in turn and
// their sums are joined in shared memory in the warps' order.
//
// Measured: 1 x 4,096 x 4,096 (T x C x d) 4.0 us (a launch, one round of loads, the join; the weights' bytes would take
// 1.3), 5 x 11,008 x 4,096 bf16 8.2, fp16 with zero points 9.6 (issue: 15 instructions for eight weights).
#include <math.h>

#include <algorithm>
#include <type_traits>

#include "g4.cuh"
#include "sm100.cuh"

MPQ_CHECKED_UNIT("g4_linear.cu");

namespace mpq {
namespace {

constexpr int FEW_WARPS = 8;

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

// The scales and zero points of a row's N groups in a tile, as they lie in memory.
template <int N>
struct Groups {
    uint32_t s[(N + 1) / 2], z;
    __device__ __forceinline__ void load(const unsigned char *scales, int row, int zeros)
    {
        const unsigned char *const ss = scales + row * 2 * N, *const zs = scales + 32 * N + row * N;
        z = 0x08080808u;
        if constexpr (N == 1) {
            s[0] = *reinterpret_cast<const uint16_t *>(ss);
            if (zeros) z = *zs;
        } else if constexpr (N == 2) {
            s[0] = *reinterpret_cast<const uint32_t *>(ss);
            if (zeros) z = *reinterpret_cast<const uint16_t *>(zs);
        } else {
            const uint2 w = *reinterpret_cast<const uint2 *>(ss);
            s[0] = w.x;
            s[1] = w.y;
            if (zeros) z = *reinterpret_cast<const uint32_t *>(zs);
        }
    }
    template <typename T>
    __device__ __forceinline__ G4Scale scale(int i) const
    {
        return g4_scale<T>(i & 1 ? s[i >> 1] >> 16 : s[i >> 1] & 0xffffu, z >> (8 * i) & 255u);
    }
};

// NT: tiles of eight tokens; GROUP: elements of a group; VEC: x's rows are 16-byte aligned, d a multiple of 8.  CROWD: more
// CTAs than two an SM, so three are to fit, with fewer loads ahead (5 x 11,008 x 4,096 9.1 -> 8.1 us; one token's 256 CTAs
// of 4,096 x 4,096 took 4.9 that way instead of 4.0).  Two fit otherwise: left to 255 registers, 64 x 4,096 x 4,096 took
// 19.4 us instead of 14.2.
template <typename T, int NT, int GROUP, bool VEC, bool CROWD>
__global__ void __launch_bounds__(FEW_WARPS * 32, CROWD ? 3 : 2)
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
    // U tiles' codes, scales and zero points are on their way before the first is used
    constexpr int U = NT == 1 && !CROWD ? 4 : 2;
    const unsigned char *const codes = strip + g * 64 + i * 16;
    for (int k0 = warp; k0 < a.L.k_tiles; k0 += U * FEW_WARPS) {
        uint4 wa[U], wb[U];
        Groups<N> ga[U], gb[U];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const size_t at = (size_t)min(k0 + u * FEW_WARPS, a.L.k_tiles - 1) * a.L.tile_bytes;
            wa[u] = *reinterpret_cast<const uint4 *>(codes + at);
            wb[u] = *reinterpret_cast<const uint4 *>(codes + at + 8 * 64);
            ga[u].load(strip + at + G4_CODES, g, a.L.zeros);
            gb[u].load(strip + at + G4_CODES, g + 8, a.L.zeros);
        }
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int kt = k0 + u * FEW_WARPS;
            if (kt >= a.L.k_tiles) break;
            const uint32_t qa[4] = {wa[u].x, wa[u].y, wa[u].z, wa[u].w}, qb[4] = {wb[u].x, wb[u].y, wb[u].z, wb[u].w};
            auto tile = [&](auto far) {
                G4Scale sa, sb;
#pragma unroll
                for (int m = 0; m < 4; ++m) {
                    if (m * 32 % GROUP == 0) {
                        sa = ga[u].template scale<T>(m * 32 / GROUP);
                        sb = gb[u].template scale<T>(m * 32 / GROUP);
                    }
                    uint32_t pa[4], pb[4];
                    g4_values<T, decltype(far)::value>(qa[m], sa, pa);
                    g4_values<T, decltype(far)::value>(qb[m], sb, pb);
#pragma unroll
                    for (int n = 0; n < NT; ++n) {
                        const long long t = n0 + n * 8 + g;
                        uint4 x = make_uint4(0, 0, 0, 0);
                        if (t < a.T) x = load_x<T, VEC>(X + t * a.ldx, kt * 128 + m * 32 + i * 8, a.L.d);
                        mma16816<T>(acc[n], pa[0], pb[0], pa[1], pb[1], x.x, x.y);
                        mma16816<T>(acc[n], pa[2], pb[2], pa[3], pb[3], x.z, x.w);
                    }
                }
            };
            if (g4_far<T>(ga[u].s) || g4_far<T>(gb[u].s))
                tile(std::true_type());
            else
                tile(std::false_type());
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

template <typename T, int NT, bool VEC, bool CROWD>
mpq_status launch_few(const G4Args &a, const T *X, void *Y, cudaStream_t stream)
{
    const dim3 grid((unsigned)a.L.row_tiles, (unsigned)((a.T + NT * 8 - 1) / (NT * 8)));
    auto *const kernel = a.L.group == 32   ? g4_few_kernel<T, NT, 32, VEC, CROWD>
                         : a.L.group == 64 ? g4_few_kernel<T, NT, 64, VEC, CROWD>
                                           : g4_few_kernel<T, NT, 128, VEC, CROWD>;
    return launch_waiting(kernel, grid, dim3(FEW_WARPS * 32), 0, stream, "g4 linear launch", a, X, Y);
}

template <typename T, int NT>
mpq_status launch_tokens(const G4Args &a, const T *X, bool vec, void *Y, cudaStream_t stream)
{
    const bool crowd = NT < 4 && a.L.row_tiles > 2 * sm_count();
    if (crowd) return vec ? launch_few<T, NT, true, NT < 4>(a, X, Y, stream) : launch_few<T, NT, false, NT < 4>(a, X, Y, stream);
    return vec ? launch_few<T, NT, true, false>(a, X, Y, stream) : launch_few<T, NT, false, false>(a, X, Y, stream);
}

template <typename T>
mpq_status launch_typed(const G4Args &a, const T *X, int x_type, void *Y, cudaStream_t stream)
{
    const bool vec = rows_aligned(X, x_type, a.T > 1 ? a.ldx : 0) && a.L.d % 8 == 0;
    if (a.T <= 8) return launch_tokens<T, 1>(a, X, vec, Y, stream);
    if (a.T <= 16) return launch_tokens<T, 2>(a, X, vec, Y, stream);
    return launch_tokens<T, 4>(a, X, vec, Y, stream);
}

// Whether this kernel's modelled time (us) is less than the tiles': a start, and what is longer of a warp's tiles one
// after another and of all tiles and CTAs, by the tokens of a CTA (8, 16 or 32).  Some timings, us, this kernel's and
// the tiles': 8 x 4,096 x 4,096 (T x C x d) 4.3, 8.2; 32 x 4,096 x 4,096 7.8, 9.0; 64 x 4,096 x 4,096 14.2, 9.3;
// 16 x 11,008 x 4,096 11.8, 14.9; 24 x 11,008 x 4,096 17.6, 14.9; 64 x 2,048 x 2,048 5.1, 7.4; 16 x 32,768 x 4,096
// 30.8, 27.5; 24 x 512 x 8,192 7.7, 8.4; 96 x 512 x 8,192 11.2, 9.6 (where the model is wrong).
bool few_tokens(int T, const mpq_g4_matrix *L)
{
    if (T > 128) return false;
    const int c = T <= 8 ? 0 : T <= 16 ? 1 : 2;
    constexpr double one[3] = {0.4, 0.6, 0.75}, tile[3] = {0.27e-3, 0.36e-3, 0.6e-3}, cta[3] = {0.6e-3, 1.5e-3, 2.3e-3};
    const double ctas = (double)L->row_tiles * ((T + 31) / 32);
    const double t = 2.0 + std::max((L->k_tiles + FEW_WARPS - 1) / FEW_WARPS * one[c], ctas * (L->k_tiles * tile[c] + cta[c]));
    return t < g4_tiles_time(T, L->rows, L->d);
}

}  // namespace

mpq_status launch_g4_linear(const void *X, int x_type, long long ldx, int T, const mpq_g4_matrix *L,
                            const void *W, const float *bias, void *Y, int y_type, long long ldy,
                            cudaStream_t stream)
{
    if (!few_tokens(T, L)) return launch_g4_tiles(X, x_type, ldx, T, L, W, bias, Y, y_type, ldy, stream);
    const G4Args a = {*L, static_cast<const unsigned char *>(W), bias, ldx, ldy, T, y_type};
    if (x_type == MPQ_F16) return launch_typed(a, static_cast<const __half *>(X), x_type, Y, stream);
    return launch_typed(a, static_cast<const __nv_bfloat16 *>(X), x_type, Y, stream);
}

}  // namespace mpq
