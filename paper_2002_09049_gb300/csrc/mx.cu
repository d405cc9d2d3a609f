// Microscaled 4-bit floats (mpq_mx_quantize, mpq_mx_dequantize): blocks of 32 elements, each with the
// scale 2^e, e = floor(log2 amax) - 2, and E2M1 codes of x / 2^e.
//
// x / 2^e is exact (a power of two, and x has at most 24 significant bits; what falls below fp32's
// range is far below half the smallest level), so the one rounding of an element is the conversion to
// E2M1.  amax / 2^e lies in [4, 8): nothing but (6, 8) saturates.
//
// A thread takes 16 consecutive elements (one 32-byte access of 16-bit ones), two threads a block.
// Memory-bound: an element costs its own bytes in and 17/32 of a byte out.
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

// The thread's row and its 16-element group of the row (d_pad / 16 groups); rows past the matrix belong
// to its last row tile.
struct Place {
    long long row;
    int group;
};
__device__ __forceinline__ Place place()
{
    return {(long long)blockIdx.x * blockDim.y + threadIdx.y,
            (int)(blockIdx.y * blockDim.x + threadIdx.x)};
}

// Byte of the scale of a group's block in the packed buffer.
__device__ __forceinline__ size_t scale_byte(const mpq_mx_matrix &L, const Place &at)
{
    return L.off_scales + ((size_t)(at.row >> 7) * L.k_tiles + (at.group >> 3)) * 512 +
           scale_at((int)(at.row & 127)) + ((at.group >> 1) & 3);
}

template <typename T, bool VEC>
__global__ void __launch_bounds__(MX_THREADS)
mx_quantize_kernel(const T *X, long long ldx, mpq_mx_matrix L, unsigned char *packed)
{
    sm100::griddep_launch();
    sm100::griddep_wait();
    const Place at = place();
    const int j0 = at.group * 16;
    // d_pad / 16 is even: the two threads of a block leave together
    if (j0 >= L.d_pad || at.row >= (long long)L.row_tiles * 128) return;
    const unsigned pair = 3u << ((threadIdx.y * blockDim.x + threadIdx.x) & 30);
    const bool real = at.row < L.rows;
    float v[16];
    const T *x = X + at.row * ldx + j0;
    if (VEC && real && j0 + 16 <= L.d) {
        load16(x, v);
    } else {
#pragma unroll
        for (int i = 0; i < 16; ++i) v[i] = real && j0 + i < L.d ? to_f32(x[i]) : 0.0f;
    }
    uint32_t top = top_bits(v);
    top = max(top, __shfl_xor_sync(pair, top, 1));
    const bool bad = top >= 0x7f800000u;
    // E = e + 127: the exponent field less 2; below 2^-125 (subnormal or nearly) e stays at -127
    const int field = (int)(top >> 23);
    const int E = bad ? 255 : (field > 2 ? field - 2 : 0);
    const float inv = __uint_as_float((uint32_t)(254 - E) << 23);   // 2^-e, e <= 125
    float lo[8], hi[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) lo[i] = v[i] * inv, hi[i] = v[8 + i] * inv;
    // (rows past the last fill what is left up to the scales with zero codes)
    const size_t to = (size_t)at.row * (L.d_pad / 2) + j0 / 2;
    if (to < L.off_scales)
        *reinterpret_cast<uint2 *>(packed + to) =
            bad ? make_uint2(0, 0) : make_uint2(e2m1x8(lo), e2m1x8(hi));
    if ((at.group & 1) == 0) {
        const size_t sc = scale_byte(L, at);
        if (MPQ_IN(sc, L.bytes)) packed[sc] = (unsigned char)(real ? E : 0);
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
    const float scale = scale_value(packed[scale_byte(L, at)]);
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

// Other rows: a warp takes 512 elements of a row, 32 consecutive ones (a block) at a time, one a lane,
// so that its stores are consecutive (16 of them a thread 32 bytes apart take 15 times as long).
template <typename T>
__global__ void __launch_bounds__(MX_THREADS)
mx_dequantize_odd_kernel(const unsigned char *packed, mpq_mx_matrix L, T *Y, long long ldy)
{
    sm100::griddep_launch();
    sm100::griddep_wait();
    const int lane = threadIdx.x & 31;
    const long long row = blockIdx.x;
    const int j0 = ((int)blockIdx.y * (MX_THREADS / 32) + (int)(threadIdx.x >> 5)) * 512;
    const unsigned char *const codes = packed + row * (L.d_pad / 2);
    T *const y = Y + row * ldy;
#pragma unroll 4
    for (int j = j0 + lane; j < min(j0 + 512, L.d); j += 32) {
        const unsigned code = (codes[j >> 1] >> (4 * (j & 1))) & 15u;
        const float scale = scale_value(packed[scale_byte(L, {row, j >> 4})]);
        // the level as an integer number of halves: m for m < 2, else (2 + (m & 1)) 2^(m/2 - 1)
        const unsigned m = code & 7u;
        const float v = 0.5f * (float)(m < 2 ? m : (2u + (m & 1u)) << ((m >> 1) - 1));
        if (MPQ_IN(row * ldy + j, (L.rows - 1) * ldy + L.d))
            y[j] = from_f32<T>(__fmul_rn(code & 8u ? -v : v, scale));
    }
}

// Threads across a row (a power of two, 8 to 256), the rest down the rows.
dim3 mx_block(const mpq_mx_matrix *L)
{
    int tx = 8;
    while (tx < MX_THREADS && tx < L->d_pad / 16) tx *= 2;
    return dim3((unsigned)tx, (unsigned)(MX_THREADS / tx), 1);
}

dim3 mx_grid(const mpq_mx_matrix *L, long long rows, dim3 block)
{
    return dim3((unsigned)((rows + block.y - 1) / block.y),
                (unsigned)((L->d_pad / 16 + (int)block.x - 1) / (int)block.x), 1);
}

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
    const bool vec = rows_aligned(X, x_type, ldx);
    unsigned char *out = static_cast<unsigned char *>(packed);
    const dim3 block = mx_block(L), grid = mx_grid(L, (long long)L->row_tiles * 128, block);
    return by_type(x_type, [&](auto t) {
        using T = decltype(t);
        return launch_waiting(vec ? mx_quantize_kernel<T, true> : mx_quantize_kernel<T, false>, grid,
                              block, 0, stream, "mx quantize launch", static_cast<const T *>(X), ldx,
                              *L, out);
    });
}

mpq_status launch_mx_dequantize(const void *packed, const mpq_mx_matrix *L, void *Y, int y_type,
                                long long ldy, cudaStream_t stream)
{
    const bool vec = rows_aligned(Y, y_type, ldy);
    const unsigned char *in = static_cast<const unsigned char *>(packed);
    return by_type(y_type, [&](auto t) {
        using T = decltype(t);
        if (!vec)
            return launch_waiting(mx_dequantize_odd_kernel<T>,
                                  dim3((unsigned)L->rows, (unsigned)((L->d + MX_THREADS * 16 - 1) /
                                                                     (MX_THREADS * 16))),
                                  dim3(MX_THREADS), 0, stream, "mx dequantize launch", in, *L,
                                  static_cast<T *>(Y), ldy);
        const dim3 block = mx_block(L), grid = mx_grid(L, L->rows, block);
        return launch_waiting(mx_dequantize_kernel<T>, grid, block, 0, stream, "mx dequantize launch", in,
                              *L, static_cast<T *>(Y), ldy);
    });
}

}  // namespace mpq
