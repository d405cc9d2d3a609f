// A few tokens through a linear layer of weights in 4-bit integers, by warp-level MMAs (m16n8k16): the kernel of
// g4_linear.cu (weights' values rounded to x's type) and g4_linear_exact.cu (EXACT: the values themselves).
//
// A tile's 16 rows are A, eight tokens B.  A lane's 16 bytes of a row hold, for each 32 elements, the eight that it
// multiplies in two MMAs: the codes become A's registers where they are, and x's registers are 16 consecutive bytes of
// its row.  Warps of a CTA take a row tile's tiles in turn and their sums are joined in shared memory in the
// warps' order.  (EXACT with 32 tokens spills up to 19 words: it has its groups' sums beside all of K's.)
#pragma once

#include <type_traits>

#include "g4.cuh"
#include "sm100.cuh"

namespace mpq {

struct G4Args {
    mpq_g4_matrix L;
    const unsigned char *w;
    const float *bias;
    long long ldx, ldy;
    int T, y_type;
};

// The exact form (g4_linear_exact.cu).
mpq_status launch_few_exact(const G4Args &a, const void *X, int x_type, void *Y, cudaStream_t stream);

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

// EXACT: a group's operands are its q - z, whole numbers, and its sums of x (q - z), fp32, are added up times its scale.
// NT: tiles of eight tokens; GROUP: elements of a group; VEC: x's rows are 16-byte aligned, d a multiple of 8.  CROWD: more
// CTAs than two an SM, so three are to fit, with fewer loads ahead (5 x 11,008 x 4,096 9.1 -> 8.1 us; one token's 256 CTAs
// of 4,096 x 4,096 took 4.9 that way instead of 4.0).  Two fit otherwise: left to 255 registers, 64 x 4,096 x 4,096 took
// 19.4 us instead of 14.2.
template <typename T, int NT, int GROUP, bool VEC, bool CROWD, bool EXACT>
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
                float own[EXACT ? NT : 1][4];        // the group's sums
#pragma unroll
                for (int m = 0; m < 4; ++m) {
                    if (m * 32 % GROUP == 0) {
                        sa = ga[u].template scale<T>(m * 32 / GROUP);
                        sb = gb[u].template scale<T>(m * 32 / GROUP);
#pragma unroll
                        for (int n = 0; EXACT && n < NT; ++n)
#pragma unroll
                            for (int e = 0; e < 4; ++e) own[n][e] = 0.0f;
                    }
                    uint32_t pa[4], pb[4];
                    if constexpr (EXACT) {
                        g4_whole<T>(qa[m], sa.from, pa);
                        g4_whole<T>(qb[m], sb.from, pb);
                    } else {
                        g4_values<T, decltype(far)::value>(qa[m], sa, pa);
                        g4_values<T, decltype(far)::value>(qb[m], sb, pb);
                    }
#pragma unroll
                    for (int n = 0; n < NT; ++n) {
                        const long long t = n0 + n * 8 + g;
                        uint4 x = make_uint4(0, 0, 0, 0);
                        if (t < a.T) x = load_x<T, VEC>(X + t * a.ldx, kt * 128 + m * 32 + i * 8, a.L.d);
                        float(&to)[4] = EXACT ? own[EXACT ? n : 0] : acc[n];
                        mma16816<T>(to, pa[0], pb[0], pa[1], pb[1], x.x, x.y);
                        mma16816<T>(to, pa[2], pb[2], pa[3], pb[3], x.z, x.w);
                    }
                    if (EXACT && (m + 1) * 32 % GROUP == 0) {
                        const float fa = bf16_bits(sa.bits), fb = bf16_bits(sb.bits);
#pragma unroll
                        for (int n = 0; n < NT; ++n)
#pragma unroll
                            for (int e = 0; e < 4; ++e) acc[n][e] = fmaf(own[EXACT ? n : 0][e], e < 2 ? fa : fb, acc[n][e]);
                    }
                }
            };
            if (!EXACT && (g4_far<T>(ga[u].s) || g4_far<T>(gb[u].s)))
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

template <typename T, int NT, bool VEC, bool CROWD, bool EXACT>
mpq_status launch_few(const G4Args &a, const T *X, void *Y, cudaStream_t stream)
{
    const dim3 grid((unsigned)a.L.row_tiles, (unsigned)((a.T + NT * 8 - 1) / (NT * 8)));
    auto *const kernel = a.L.group == 32   ? g4_few_kernel<T, NT, 32, VEC, CROWD, EXACT>
                         : a.L.group == 64 ? g4_few_kernel<T, NT, 64, VEC, CROWD, EXACT>
                                           : g4_few_kernel<T, NT, 128, VEC, CROWD, EXACT>;
    return launch_waiting(kernel, grid, dim3(FEW_WARPS * 32), 0, stream, "g4 linear launch", a, X, Y);
}

template <typename T, int NT, bool EXACT>
mpq_status launch_tokens(const G4Args &a, const T *X, bool vec, void *Y, cudaStream_t stream)
{
    const bool crowd = NT < 4 && a.L.row_tiles > 2 * sm_count();
    if (crowd)
        return vec ? launch_few<T, NT, true, NT < 4, EXACT>(a, X, Y, stream)
                   : launch_few<T, NT, false, NT < 4, EXACT>(a, X, Y, stream);
    return vec ? launch_few<T, NT, true, false, EXACT>(a, X, Y, stream)
               : launch_few<T, NT, false, false, EXACT>(a, X, Y, stream);
}

template <typename T, bool EXACT>
mpq_status launch_typed(const G4Args &a, const T *X, int x_type, void *Y, cudaStream_t stream)
{
    const bool vec = rows_aligned(X, x_type, a.T > 1 ? a.ldx : 0) && a.L.d % 8 == 0;
    if (a.T <= 8) return launch_tokens<T, 1, EXACT>(a, X, vec, Y, stream);
    if (a.T <= 16) return launch_tokens<T, 2, EXACT>(a, X, vec, Y, stream);
    return launch_tokens<T, 4, EXACT>(a, X, vec, Y, stream);
}

template <bool EXACT>
mpq_status launch_few_tokens(const G4Args &a, const void *X, int x_type, void *Y, cudaStream_t stream)
{
    if (x_type == MPQ_F16) return launch_typed<__half, EXACT>(a, static_cast<const __half *>(X), x_type, Y, stream);
    return launch_typed<__nv_bfloat16, EXACT>(a, static_cast<const __nv_bfloat16 *>(X), x_type, Y, stream);
}

}  // namespace
}  // namespace mpq
