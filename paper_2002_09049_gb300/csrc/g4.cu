// Weights in 4-bit integers (mpq_g4_quantize, mpq_g4_dequantize): groups of 32, 64 or 128 elements of a row, a bf16
// scale and a zero point each.
//
// A thread has eight consecutive elements, a word of codes; 4, 8 or 16 threads share a group's range by
// shuffles; 256 threads make a tile of 16 rows x 128 elements, whose codes leave in order.  The quotient x / s has
// to be the correctly rounded one: two steps of Markstein's correction with the correctly rounded reciprocal (IBM
// J. Res. Dev. 34(1), 1990; kv_cache.cu has the argument), a division where the scale is so small or large
// that a remainder could leave the normal range.
//
// Memory-bound: an element's own bytes on one side, half a byte and its share of the scales on the other.
#include <math.h>
#include <string.h>

#include "g4.cuh"
#include "sm100.cuh"

MPQ_CHECKED_UNIT("g4.cu");

namespace mpq {
namespace {

constexpr int G4_THREADS = 256;              // of a tile: a word each
constexpr int G4_PITCH = 132;                // floats of a staged row: rows apart in the banks

__device__ __forceinline__ float bf16_rn(float v) { return __bfloat162float(__float2bfloat16_rn(v)); }

// RN(x / s), r = RN(1 / s).
__device__ __forceinline__ float quotient(float x, float s, float r)
{
    float y = __fmul_rn(x, r);
    y = __fmaf_rn(__fmaf_rn(-y, s, x), r, y);
    return __fmaf_rn(__fmaf_rn(-y, s, x), r, y);
}

// The nearest whole number (|y| below 2^22, ties to even).
__device__ __forceinline__ int whole(float y)
{
    return __float_as_int(__fadd_rn(y, 12582912.0f)) - __float_as_int(12582912.0f);
}

struct G4Group {
    float s;
    int z;
};

// The scale and zero point of a group of `threads` threads (4, 8 or 16 lanes of a warp).
__device__ __forceinline__ G4Group group_of(const float (&v)[8], int threads, int zeros)
{
    float hi = 0.0f, lo = 0.0f;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        hi = fmaxf(hi, v[i]);
        lo = fminf(lo, v[i]);
    }
    uint32_t top = top_bits(v);
    for (int o = 1; o < threads; o <<= 1) {
        hi = fmaxf(hi, __shfl_xor_sync(0xffffffffu, hi, o));
        lo = fminf(lo, __shfl_xor_sync(0xffffffffu, lo, o));
        top = max(top, __shfl_xor_sync(0xffffffffu, top, o));
    }
    constexpr float seventh = 1.0f / 7.0f, fifteenth = 1.0f / 15.0f;
    G4Group g;
    g.z = G4_ZERO;
    g.s = bf16_rn(zeros ? __fsub_rn(__fmul_rn(hi, fifteenth), __fmul_rn(lo, fifteenth))
                        : __fmul_rn(__uint_as_float(top), seventh));
    if (top >= 0x7f800000u) g.s = NAN;
    if (zeros && g.s > 0.0f) g.z = min(max(whole(fminf(__fdiv_rn(-lo, g.s), 32.0f)), 0), 15);
    return g;
}

// The word of a thread's eight codes.
__device__ __forceinline__ uint32_t codes_of(const float (&v)[8], const G4Group &g, int zeros)
{
    const int least = zeros ? 0 : 1;
    const bool plain = g.s >= 0x1p-100f && g.s <= 0x1p100f;
    const float r = plain ? __frcp_rn(g.s) : 0.0f;
    uint32_t w = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        int q = g.z;
        if (plain)
            q = min(max(whole(quotient(v[i], g.s, r)) + g.z, least), 15);
        else if (g.s > 0.0f)
            q = min(max(whole(fminf(fmaxf(__fdiv_rn(v[i], g.s), -32.0f), 32.0f)) + g.z, least), 15);
        w |= (uint32_t)q << g4_shift(i);
    }
    return w;
}

// VEC: rows are 16-byte aligned; else they pass through shared memory, a warp's accesses consecutive.
template <typename T, bool VEC>
__global__ void __launch_bounds__(G4_THREADS)
g4_quantize_kernel(const T *X, long long ldx, mpq_g4_matrix L, unsigned char *packed)
{
    __shared__ float stage[VEC ? 1 : 16 * G4_PITCH];
    sm100::griddep_launch();
    sm100::griddep_wait();
    const int rt = (int)blockIdx.x / L.k_tiles, kt = (int)blockIdx.x - rt * L.k_tiles;
    const int n = threadIdx.x & 15, in_tile = (int)threadIdx.x >> 4;
    const long long row0 = (long long)rt * 16;
    const int j0 = kt * 128 + n * 8;
    float v[8];
    if constexpr (VEC) {
        const long long row = row0 + in_tile;
        const bool real = row < L.rows;
        const T *const x = X + (real ? row : 0) * ldx + j0;
        if (real && j0 + 8 <= L.d) {
            load8(x, v);
        } else {
#pragma unroll
            for (int i = 0; i < 8; ++i) v[i] = real && j0 + i < L.d ? to_f32(x[i]) : 0.0f;
        }
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const int e = (int)threadIdx.x + i * G4_THREADS, r = e >> 7, j = e & 127;
            const bool real = row0 + r < L.rows && kt * 128 + j < L.d;
            stage[r * G4_PITCH + j] = real ? to_f32(X[(row0 + r) * ldx + kt * 128 + j]) : 0.0f;
        }
        __syncthreads();
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = stage[in_tile * G4_PITCH + n * 8 + i];
    }
    const int threads = L.group >> 3, groups = 128 / L.group;
    const G4Group g = group_of(v, threads, L.zeros);
    const uint32_t w = codes_of(v, g, L.zeros);
    const size_t at = (size_t)blockIdx.x * L.tile_bytes;
    unsigned char *const tile = packed + at;
    if (!MPQ_IN(at + L.tile_bytes - 1, L.bytes)) return;
    *reinterpret_cast<uint32_t *>(tile + in_tile * 64 + g4_word(n)) = w;
    if ((n & (threads - 1)) == 0) {
        const int i = in_tile * groups + n / threads;
        reinterpret_cast<__nv_bfloat16 *>(tile + G4_CODES)[i] = __float2bfloat16_rn(g.s);
        if (L.zeros) tile[G4_CODES + 32 * groups + i] = (unsigned char)g.z;
    }
}

template <typename T, bool VEC>
__global__ void __launch_bounds__(G4_THREADS)
g4_dequantize_kernel(const unsigned char *packed, mpq_g4_matrix L, T *Y, long long ldy)
{
    __shared__ float stage[VEC ? 1 : 16 * G4_PITCH];
    sm100::griddep_launch();
    sm100::griddep_wait();
    const int rt = (int)blockIdx.x / L.k_tiles, kt = (int)blockIdx.x - rt * L.k_tiles;
    const int n = threadIdx.x & 15, in_tile = (int)threadIdx.x >> 4;
    const long long row0 = (long long)rt * 16, row = row0 + in_tile;
    const int j0 = kt * 128 + n * 8, groups = 128 / L.group;
    const unsigned char *const tile = packed + (size_t)blockIdx.x * L.tile_bytes;
    const uint32_t w = *reinterpret_cast<const uint32_t *>(tile + in_tile * 64 + g4_word(n));
    const int at = in_tile * groups + n * 8 / L.group;
    const float s = bf16_bits(reinterpret_cast<const uint16_t *>(tile + G4_CODES)[at]);
    const int z = L.zeros ? tile[G4_CODES + 32 * groups + at] : G4_ZERO;
    float v[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = __fmul_rn((float)((int)(w >> g4_shift(i) & 15u) - z), s);
    const size_t size = (L.rows - 1) * ldy + L.d;
    if constexpr (VEC) {
        if (row >= L.rows || j0 >= L.d) return;
        T *const y = Y + row * ldy + j0;
        if (!MPQ_IN(row * ldy + min(j0 + 8, L.d) - 1, size)) return;
        if (j0 + 8 <= L.d) {
            store8(y, v);
        } else {
#pragma unroll
            for (int i = 0; i < 8; ++i)
                if (j0 + i < L.d) y[i] = from_f32<T>(v[i]);
        }
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) stage[in_tile * G4_PITCH + n * 8 + i] = v[i];
        __syncthreads();
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const int e = (int)threadIdx.x + i * G4_THREADS, r = e >> 7, j = e & 127;
            if (row0 + r < L.rows && kt * 128 + j < L.d && MPQ_IN((row0 + r) * ldy + kt * 128 + j, size))
                Y[(row0 + r) * ldy + kt * 128 + j] = from_f32<T>(stage[r * G4_PITCH + j]);
        }
    }
}

bool aligned(const void *p, int type, long long ld, int rows) { return rows_aligned(p, type, rows > 1 ? ld : 0); }

}  // namespace

mpq_status make_g4_layout(int rows, int d, int group, int zeros, mpq_g4_matrix *L)
{
    memset(L, 0, sizeof(*L));
    L->rows = rows;
    L->d = d;
    L->group = group;
    L->zeros = zeros;
    L->row_tiles = (int)(((long long)rows + 15) / 16);
    L->k_tiles = (d + 127) / 128;
    L->tile_bytes = G4_CODES + (zeros ? 48 : 32) * (128 / group);
    L->bytes = (size_t)L->row_tiles * L->k_tiles * L->tile_bytes;
    return MPQ_OK;
}

mpq_status launch_g4_quantize(const void *X, int x_type, long long ldx, const mpq_g4_matrix *L, void *packed,
                              cudaStream_t stream)
{
    const bool vec = aligned(X, x_type, ldx, L->rows);
    return by_type(x_type, [&](auto t) {
        using T = decltype(t);
        return launch_waiting(vec ? g4_quantize_kernel<T, true> : g4_quantize_kernel<T, false>,
                              dim3((unsigned)L->row_tiles * (unsigned)L->k_tiles), dim3(G4_THREADS), 0, stream,
                              "g4 quantize launch", static_cast<const T *>(X), ldx, *L,
                              static_cast<unsigned char *>(packed));
    });
}

mpq_status launch_g4_dequantize(const void *packed, const mpq_g4_matrix *L, void *Y, int y_type, long long ldy,
                                cudaStream_t stream)
{
    const bool vec = aligned(Y, y_type, ldy, L->rows);
    return by_type(y_type, [&](auto t) {
        using T = decltype(t);
        return launch_waiting(vec ? g4_dequantize_kernel<T, true> : g4_dequantize_kernel<T, false>,
                              dim3((unsigned)L->row_tiles * (unsigned)L->k_tiles), dim3(G4_THREADS), 0, stream,
                              "g4 dequantize launch", static_cast<const unsigned char *>(packed), *L,
                              static_cast<T *>(Y), ldy);
    });
}

}  // namespace mpq
