// Microscaled 4-bit floats (mpq_mx_quantize, mpq_mx_dequantize): blocks of 32 elements, each with the
// scale 2^e, e = floor(log2 amax) - 2, and E2M1 codes of x / 2^e.
//
// x / 2^e is exact (a power of two, and x has at most 24 significant bits; what falls below fp32's
// range is far below half the smallest level), so the one rounding of an element is the conversion to
// E2M1.  amax / 2^e lies in [4, 8): nothing but (6, 8) saturates.
//
// Memory-bound: an element costs its own bytes in and 17/32 of a byte out.  11,008 x 4,096 fp32 is quantised
// in 29.7 us and read back in 29.9 (204 MB each, 6.9 TB/s); 2,048 x 11,008 bf16 in 10.3 us (5.5 TB/s).
#include <math.h>
#include <string.h>

#include "elements.cuh"
#include "mpq_internal.cuh"
#include "sm100.cuh"

MPQ_CHECKED_UNIT("mx.cu");

namespace mpq {
namespace {

constexpr int MX_THREADS = 256;

// Byte of the scale of block b of row m (within its tile of 128 rows x 4 blocks).
__device__ __forceinline__ int scale_at(int m) { return (m & 31) * 16 + (m >> 5) * 4; }

// Eight levels, each in a nibble, from eight values in E2M1's range (saturating; none is NaN).
__device__ __forceinline__ uint32_t e2m1x8(const float (&v)[8])
{
    uint32_t r;
    asm("{\n\t.reg .b8 b0, b1, b2, b3;\n\t"
        "cvt.rn.satfinite.e2m1x2.f32 b0, %2, %1;\n\t"
        "cvt.rn.satfinite.e2m1x2.f32 b1, %4, %3;\n\t"
        "cvt.rn.satfinite.e2m1x2.f32 b2, %6, %5;\n\t"
        "cvt.rn.satfinite.e2m1x2.f32 b3, %8, %7;\n\t"
        "mov.b32 %0, {b0, b1, b2, b3};\n\t}"
        : "=r"(r)
        : "f"(v[0]), "f"(v[1]), "f"(v[2]), "f"(v[3]), "f"(v[4]), "f"(v[5]), "f"(v[6]), "f"(v[7]));
    return r;
}

__device__ __forceinline__ uint32_t e2m1x2(float a, float b)
{
    uint32_t r;
    asm("{\n\t.reg .b8 b0, z;\n\t"
        "mov.b16 {z, b0}, 0;\n\t"
        "cvt.rn.satfinite.e2m1x2.f32 b0, %2, %1;\n\t"
        "mov.b32 %0, {b0, z, z, z};\n\t}"
        : "=r"(r) : "f"(a), "f"(b));
    return r;
}

// The values of eight codes.
__device__ __forceinline__ void e2m1x8_values(uint32_t w, float (&v)[8])
{
    uint32_t h[4];
    asm("{\n\t.reg .b8 b0, b1, b2, b3;\n\t"
        "mov.b32 {b0, b1, b2, b3}, %4;\n\t"
        "cvt.rn.f16x2.e2m1x2 %0, b0;\n\t"
        "cvt.rn.f16x2.e2m1x2 %1, b1;\n\t"
        "cvt.rn.f16x2.e2m1x2 %2, b2;\n\t"
        "cvt.rn.f16x2.e2m1x2 %3, b3;\n\t}"
        : "=r"(h[0]), "=r"(h[1]), "=r"(h[2]), "=r"(h[3])
        : "r"(w));
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const float2 f = unpack2(h[i], __half());
        v[2 * i] = f.x;
        v[2 * i + 1] = f.y;
    }
}

// The thread's row and its group of elements of the row; rows past the matrix belong to its last row tile.
struct Place {
    long long row;
    int group;
};
__device__ __forceinline__ Place place()
{
    return {(long long)blockIdx.x * blockDim.y + threadIdx.y,
            (int)(blockIdx.y * blockDim.x + threadIdx.x)};
}

// Byte of the scale of a row's block in the packed buffer.
__device__ __forceinline__ size_t scale_byte(const mpq_mx_matrix &L, long long row, int block)
{
    return L.off_scales + ((size_t)(row >> 7) * L.k_tiles + (block >> 2)) * 512 +
           scale_at((int)(row & 127)) + (block & 3);
}

// The scale of a block (biased, as stored) from the bits of its largest magnitude: E = e + 127 is the
// exponent field less 2; below 2^-125 (subnormal or nearly) e stays at -127; 255 for infinities and NaN.
__device__ __forceinline__ uint32_t block_scale(uint32_t top)
{
    return top >= 0x7f800000u ? 255u : (uint32_t)max((int)(top >> 23) - 2, 0);
}

// The scales of four consecutive blocks (a word) from the lanes' own, P lanes a block; complete in every
// lane of the four blocks.
template <int P>
__device__ __forceinline__ uint32_t scale_word(uint32_t E, unsigned lane, unsigned lanes)
{
    uint32_t e = E << (8 * (lane / P & 3));
    e |= __shfl_xor_sync(lanes, e, P);
    return e | __shfl_xor_sync(lanes, e, 2 * P);
}

// Aligned rows: N consecutive elements a thread, 32 of 16-bit types (a block) or 16 (2,048 x 11,008 bf16:
// 10.9 us with 32, 13.5 with 16; 11,008 x 4,096 fp32: 29.7 us with 16, 34.0 with 32).
template <typename T, int N>
__global__ void __launch_bounds__(MX_THREADS)
mx_quantize_kernel(const T *X, long long ldx, mpq_mx_matrix L, unsigned char *packed)
{
    sm100::griddep_launch();
    sm100::griddep_wait();
    constexpr int P = 32 / N;            // threads of a block
    const Place at = place();
    const int j0 = at.group * N;
    // d_pad is a multiple of 128: the threads of a word of scales leave together
    if (j0 >= L.d_pad || at.row >= (long long)L.row_tiles * 128) return;
    const unsigned lane = (threadIdx.y * blockDim.x + threadIdx.x) & 31;
    const unsigned lanes = ((1u << 4 * P) - 1u) << (lane & ~(4 * P - 1));
    const bool real = at.row < L.rows;
    float v[N];
    const T *x = X + at.row * ldx + j0;
    if (real && j0 + N <= L.d) {
        if constexpr (N == 32) load32(x, v);
        else load16(x, v);
    } else {
#pragma unroll
        for (int i = 0; i < N; ++i) v[i] = real && j0 + i < L.d ? to_f32(x[i]) : 0.0f;
    }
    uint32_t top = top_bits(v);
    if constexpr (P == 2) top = max(top, __shfl_xor_sync(lanes, top, 1));
    const uint32_t E = block_scale(top);
    const float inv = __uint_as_float((254u - E) << 23);    // 2^-e, e <= 125
    uint32_t w[N / 8];
#pragma unroll
    for (int k = 0; k < N / 8; ++k) {
        float y[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) y[i] = v[8 * k + i] * inv;
        w[k] = E == 255u ? 0u : e2m1x8(y);
    }
    // (rows past the last fill what is left up to the scales with zero codes)
    const size_t to = (size_t)at.row * (L.d_pad / 2) + j0 / 2;
    if (to < L.off_scales) {
        if constexpr (N == 32)
            *reinterpret_cast<uint4 *>(packed + to) = make_uint4(w[0], w[1], w[2], w[3]);
        else
            *reinterpret_cast<uint2 *>(packed + to) = make_uint2(w[0], w[1]);
    }
    const uint32_t e = scale_word<P>(E, lane, lanes);
    if ((lane & (4 * P - 1)) == 0) {
        const size_t sc = scale_byte(L, at.row, j0 >> 5);
        if (MPQ_IN(sc + 3, L.bytes)) *reinterpret_cast<uint32_t *>(packed + sc) = e;
    }
}

// Other rows: a warp takes 128 elements of a row (a word of scales), so that its accesses stay together:
// quantising, a lane has four consecutive elements (156,090 x 230 fp32: 44 us; with 16 a thread, whose loads
// lie 64 bytes apart, 164).
template <typename T>
__global__ void __launch_bounds__(MX_THREADS)
mx_quantize_odd_kernel(const T *X, long long ldx, mpq_mx_matrix L, unsigned char *packed)
{
    sm100::griddep_launch();
    sm100::griddep_wait();
    const unsigned lane = threadIdx.x;
    const long long row = (long long)blockIdx.x * blockDim.z + threadIdx.z;
    const int kt = (int)(blockIdx.y * blockDim.y + threadIdx.y), j0 = kt * 128 + 4 * (int)lane;
    if (kt >= L.k_tiles || row >= (long long)L.row_tiles * 128) return;      // (a whole warp)
    const T *const x = X + row * ldx + j0;
    float v[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) v[i] = row < L.rows && j0 + i < L.d ? to_f32(x[i]) : 0.0f;
    uint32_t top = top_bits(v);
#pragma unroll
    for (int o = 1; o < 8; o <<= 1) top = max(top, __shfl_xor_sync(0xffffffffu, top, o));
    const uint32_t E = block_scale(top);
    const float inv = __uint_as_float((254u - E) << 23);
    const uint32_t c = E == 255u ? 0u : e2m1x2(v[0] * inv, v[1] * inv) | e2m1x2(v[2] * inv, v[3] * inv) << 8;
    const size_t to = (size_t)row * (L.d_pad / 2) + j0 / 2;
    if (to < L.off_scales) *reinterpret_cast<uint16_t *>(packed + to) = (uint16_t)c;
    const uint32_t e = scale_word<8>(E, lane, 0xffffffffu);
    if (lane == 0) {
        const size_t sc = scale_byte(L, row, 4 * kt);
        if (MPQ_IN(sc + 3, L.bytes)) *reinterpret_cast<uint32_t *>(packed + sc) = e;
    }
}

// 2^(E-127): subnormal for E = 0, NaN for 255.
__device__ __forceinline__ float scale_value(int E)
{
    return __uint_as_float(E == 255 ? 0x7fffffffu : E == 0 ? 0x00400000u : (uint32_t)E << 23);
}

// Aligned rows: 16 consecutive elements a thread.
template <typename T>
__global__ void __launch_bounds__(MX_THREADS)
mx_dequantize_kernel(const unsigned char *packed, mpq_mx_matrix L, T *Y, long long ldy)
{
    sm100::griddep_launch();
    sm100::griddep_wait();
    const Place at = place();
    const int j0 = at.group * 16;
    if (j0 >= L.d || at.row >= L.rows) return;
    const uint2 w = *reinterpret_cast<const uint2 *>(packed + at.row * (L.d_pad / 2) + j0 / 2);
    const float scale = scale_value(packed[scale_byte(L, at.row, at.group >> 1)]);
    float lo[8], hi[8], v[16];
    e2m1x8_values(w.x, lo);
    e2m1x8_values(w.y, hi);
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = __fmul_rn(lo[i], scale), v[8 + i] = __fmul_rn(hi[i], scale);
    T *y = Y + at.row * ldy + j0;
    if (!MPQ_IN(at.row * ldy + j0 + min(16, L.d - j0) - 1, (L.rows - 1) * ldy + L.d)) return;
    if (j0 + 16 <= L.d) {
        store16(y, v);
    } else {
#pragma unroll
        for (int i = 0; i < 16; ++i)
            if (j0 + i < L.d) y[i] = from_f32<T>(v[i]);
    }
}

// Other rows: 128 elements a warp, 32 consecutive ones (a block) at a time, one a lane, so that its stores
// are consecutive (16 of them a thread, 32 bytes apart, take 15 times as long).
template <typename T>
__global__ void __launch_bounds__(MX_THREADS)
mx_dequantize_odd_kernel(const unsigned char *packed, mpq_mx_matrix L, T *Y, long long ldy)
{
    sm100::griddep_launch();
    sm100::griddep_wait();
    const long long row = (long long)blockIdx.x * blockDim.z + threadIdx.z;
    const int kt = (int)(blockIdx.y * blockDim.y + threadIdx.y);
    if (kt >= L.k_tiles || row >= L.rows) return;
    const unsigned char *const codes = packed + row * (L.d_pad / 2) + kt * 64 + threadIdx.x / 2;
    const uint32_t scales = *reinterpret_cast<const uint32_t *>(packed + scale_byte(L, row, 4 * kt));
    uint32_t c[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) c[i] = codes[16 * i] >> (4 * (threadIdx.x & 1)) & 15u;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int j = kt * 128 + 32 * i + (int)threadIdx.x;
        // the level as an integer number of halves: m for m < 2, else (2 + (m & 1)) 2^(m/2 - 1)
        const unsigned m = c[i] & 7u;
        const float v = 0.5f * (float)(m < 2 ? m : (2u + (m & 1u)) << ((m >> 1) - 1));
        if (j < L.d && MPQ_IN(row * ldy + j, (L.rows - 1) * ldy + L.d))
            Y[row * ldy + j] = from_f32<T>(__fmul_rn(c[i] & 8u ? -v : v, scale_value(scales >> (8 * i) & 255u)));
    }
}

// Threads across a row of n groups (a power of two, 4 to 256), the rest down the rows.
dim3 mx_block(int n)
{
    int tx = 4;
    while (tx < MX_THREADS && tx < n) tx *= 2;
    return dim3((unsigned)tx, (unsigned)(MX_THREADS / tx), 1);
}

dim3 mx_grid(int n, long long rows, dim3 block)
{
    return dim3((unsigned)((rows + block.y - 1) / block.y), (unsigned)((n + (int)block.x - 1) / (int)block.x),
                1);
}

// A warp for 128 elements: warps across a row (a power of two, up to all), the rest down the rows.
dim3 odd_block(const mpq_mx_matrix *L)
{
    int ty = 1;
    while (ty < MX_THREADS / 32 && ty < L->k_tiles) ty *= 2;
    return dim3(32, (unsigned)ty, (unsigned)(MX_THREADS / 32 / ty));
}

dim3 odd_grid(const mpq_mx_matrix *L, long long rows, dim3 block)
{
    return dim3((unsigned)((rows + block.z - 1) / block.z),
                (unsigned)((L->k_tiles + (int)block.y - 1) / (int)block.y), 1);
}

// Rows of a matrix that take aligned accesses (one row needs no stride).
bool aligned(const void *p, int type, long long ld, int rows) { return rows_aligned(p, type, rows > 1 ? ld : 0); }

}  // namespace

mpq_status make_mx_layout(int rows, int d, mpq_mx_matrix *L)
{
    memset(L, 0, sizeof(*L));
    L->rows = rows;
    L->d = d;
    L->k_tiles = (d + 127) / 128;
    L->d_pad = L->k_tiles * 128;
    L->row_tiles = (int)(((long long)rows + 127) / 128);
    L->off_scales = ((size_t)rows * (L->d_pad / 2) + 511) / 512 * 512;
    L->bytes = L->off_scales + (size_t)L->row_tiles * L->k_tiles * 512;
    return MPQ_OK;
}

mpq_status launch_mx_quantize(const void *X, int x_type, long long ldx, const mpq_mx_matrix *L,
                              void *packed, cudaStream_t stream)
{
    const bool vec = aligned(X, x_type, ldx, L->rows);
    unsigned char *out = static_cast<unsigned char *>(packed);
    const long long rows = (long long)L->row_tiles * 128;
    return by_type(x_type, [&](auto t) {
        using T = decltype(t);
        constexpr int N = sizeof(T) == 2 ? 32 : 16;
        const T *const in = static_cast<const T *>(X);
        const dim3 block = vec ? mx_block(L->d_pad / N) : odd_block(L);
        const dim3 grid = vec ? mx_grid(L->d_pad / N, rows, block) : odd_grid(L, rows, block);
        return launch_waiting(vec ? mx_quantize_kernel<T, N> : mx_quantize_odd_kernel<T>, grid, block, 0,
                              stream, "mx quantize launch", in, ldx, *L, out);
    });
}

mpq_status launch_mx_dequantize(const void *packed, const mpq_mx_matrix *L, void *Y, int y_type,
                                long long ldy, cudaStream_t stream)
{
    const bool vec = aligned(Y, y_type, ldy, L->rows);
    const unsigned char *in = static_cast<const unsigned char *>(packed);
    return by_type(y_type, [&](auto t) {
        using T = decltype(t);
        const dim3 block = vec ? mx_block(L->d_pad / 16) : odd_block(L);
        const dim3 grid = vec ? mx_grid(L->d_pad / 16, L->rows, block) : odd_grid(L, L->rows, block);
        return launch_waiting(vec ? mx_dequantize_kernel<T> : mx_dequantize_odd_kernel<T>, grid, block, 0,
                              stream, "mx dequantize launch", in, *L, static_cast<T *>(Y), ldy);
    });
}

}  // namespace mpq
