// Microscaled 4-bit floats (mpq_mx_quantize, mpq_mx_dequantize): blocks of 32 elements, each with the
// scale 2^e, e = floor(log2 amax) - 2, and E2M1 codes of x / 2^e.
//
// x / 2^e is exact (a power of two, and x has at most 24 significant bits; what falls below fp32's
// range is far below half the smallest level), so the one rounding of an element is the conversion to
// E2M1.  amax / 2^e lies in [4, 8): nothing but (6, 8) saturates.
//
// A thread takes 8 consecutive elements, 4 threads a block of 32, 16 threads the 128 elements of a
// scale tile's row.  Memory-bound: an element costs its own bytes in and 17/32 of a byte out.
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

// Rows a thread takes, blockDim.y apart: their loads are all on their way before the first is used
// (16 bytes a thread and row of 16-bit elements; one row is as much in fp32).
template <typename T>
constexpr int MX_ROWS = sizeof(T) == 4 ? 1 : 2;

// The thread's first row and its 8-element group of the rows (d_pad / 8 groups); rows past the matrix
// belong to its last row tile.
struct Place {
    long long row;
    int group;
};
template <int ROWS>
__device__ __forceinline__ Place place()
{
    return {(long long)blockIdx.x * (blockDim.y * ROWS) + threadIdx.y,
            (int)(blockIdx.y * blockDim.x + threadIdx.x)};
}

template <typename T, bool VEC>
__global__ void __launch_bounds__(MX_THREADS)
mx_quantize_kernel(const T *X, long long ldx, mpq_mx_matrix L, unsigned char *packed)
{
    sm100::griddep_launch();
    sm100::griddep_wait();
    constexpr int ROWS = MX_ROWS<T>;
    const Place at = place<ROWS>();
    const int j0 = at.group * 8;
    // d_pad / 8 is a multiple of 16: the 16 threads of a tile row leave together
    if (j0 >= L.d_pad) return;
    const unsigned half = (threadIdx.y * blockDim.x + threadIdx.x) & 16;   // of the warp
    const unsigned part = 0xffffu << half;
    float v[ROWS][8];
#pragma unroll
    for (int r = 0; r < ROWS; ++r) {
        const long long row = at.row + r * (int)blockDim.y;
        const bool real = row < L.rows;
        const T *x = X + row * ldx + j0;
        if (VEC && real && j0 + 8 <= L.d) {
            load8(x, v[r]);
        } else {
#pragma unroll
            for (int i = 0; i < 8; ++i) v[r][i] = real && j0 + i < L.d ? to_f32(x[i]) : 0.0f;
        }
    }
#pragma unroll
    for (int r = 0; r < ROWS; ++r) {
        const long long row = at.row + r * (int)blockDim.y;
        if (row >= (long long)L.row_tiles * 128) return;
        uint32_t top = top8(v[r]);
        top = max(top, __shfl_xor_sync(part, top, 1));
        top = max(top, __shfl_xor_sync(part, top, 2));
        const bool bad = top >= 0x7f800000u;
        // E = e + 127: the exponent field less 2; below 2^-125 (subnormal or nearly) e stays at -127
        const int field = (int)(top >> 23);
        const int E = bad ? 255 : (field > 2 ? field - 2 : 0);
        const float inv = __uint_as_float((uint32_t)(254 - E) << 23);   // 2^-e, e <= 125
#pragma unroll
        for (int i = 0; i < 8; ++i) v[r][i] *= inv;
        // (rows past the last fill what is left up to the scales with zero codes)
        const size_t to_codes = (size_t)row * (L.d_pad / 2) + j0 / 2;
        if (to_codes < L.off_scales)
            *reinterpret_cast<uint32_t *>(packed + to_codes) = bad ? 0u : e2m1x8(v[r]);
        if ((threadIdx.x & 3) == 0) {    // the block's scale: a tile row's four are consecutive bytes
            const size_t to = L.off_scales +
                              ((size_t)(row >> 7) * L.k_tiles + (at.group >> 4)) * 512 +
                              scale_at((int)(row & 127)) + ((at.group >> 2) & 3);
            if (MPQ_IN(to, L.bytes)) packed[to] = (unsigned char)(row < L.rows ? E : 0);
        }
    }
}

template <typename T, bool VEC>
__global__ void __launch_bounds__(MX_THREADS)
mx_dequantize_kernel(const unsigned char *packed, mpq_mx_matrix L, T *Y, long long ldy)
{
    sm100::griddep_launch();
    sm100::griddep_wait();
    const Place at = place<1>();
    const int j0 = at.group * 8;
    if (j0 >= L.d || at.row >= L.rows) return;
    const uint32_t w = sm100::ld_after_wait(
        reinterpret_cast<const unsigned *>(packed + at.row * (L.d_pad / 2) + j0 / 2));
    const uint32_t s = sm100::ld_after_wait(reinterpret_cast<const unsigned *>(
        packed + L.off_scales + ((size_t)(at.row >> 7) * L.k_tiles + (at.group >> 4)) * 512 +
        scale_at((int)(at.row & 127))));
    const int E = (int)((s >> (8 * ((at.group >> 2) & 3))) & 255u);
    float v[8];
    e2m1x8_values(w, v);
    // 2^(E-127) as two normal factors (E = 0 is subnormal, and 6 x 2^127 overflows in one step only
    // where the value does)
    const int h = E >> 1;
    const float f0 = E == 255 ? NAN : __uint_as_float((uint32_t)(h + 64) << 23);
    const float f1 = __uint_as_float((uint32_t)(E - h + 63) << 23);
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = __fmul_rn(__fmul_rn(v[i], f0), f1);
    T *y = Y + at.row * ldy + j0;
    if (!MPQ_IN(at.row * ldy + j0 + min(8, L.d - j0) - 1, (L.rows - 1) * ldy + L.d)) return;
    if (VEC && j0 + 8 <= L.d) {
        store8(y, v);
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (j0 + i < L.d) y[i] = from_f32<T>(v[i]);
    }
}

// Threads across a row (a multiple of 16, at most 256), the rest down the rows.
dim3 mx_block(const mpq_mx_matrix *L)
{
    int tx = 16;
    while (tx < MX_THREADS && tx < L->d_pad / 8) tx *= 2;
    return dim3((unsigned)tx, (unsigned)(MX_THREADS / tx), 1);
}

dim3 mx_grid(const mpq_mx_matrix *L, long long rows, dim3 block)
{
    return dim3((unsigned)((rows + block.y - 1) / block.y),
                (unsigned)((L->d_pad / 8 + (int)block.x - 1) / (int)block.x), 1);
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
    const dim3 block = mx_block(L);
    return by_type(x_type, [&](auto t) {
        using T = decltype(t);
        const dim3 grid = mx_grid(L, ((long long)L->row_tiles * 128 + MX_ROWS<T> - 1) / MX_ROWS<T>, block);
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
    const dim3 block = mx_block(L), grid = mx_grid(L, L->rows, block);
    return by_type(y_type, [&](auto t) {
        using T = decltype(t);
        return launch_waiting(vec ? mx_dequantize_kernel<T, true> : mx_dequantize_kernel<T, false>,
                              grid, block, 0, stream, "mx dequantize launch", in, *L,
                              static_cast<T *>(Y), ldy);
    });
}

}  // namespace mpq
