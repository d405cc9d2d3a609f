// Weights in 4-bit integers (mpq_g4_quantize, mpq_g4_dequantize): groups of 32, 64 or 128 elements of a row, a bf16
// scale and a zero point each.
//
// Quantising, a thread has 16 consecutive elements, two words of codes; 2, 4 or 8 threads share a group's range by
// shuffles.  Back, a thread has a word.  The quotient x / s has
// to be the correctly rounded one: a step of Markstein's correction with the correctly rounded reciprocal (IBM J.
// Res. Dev. 34(1), 1990), a division where the scale is so small or large that a remainder could leave the
// normal range.
//
// Memory-bound where elements are fp32: 11,008 x 4,096 is quantised in 31.3 us and read back in 31.4 (204 MB each, 6.5
// TB/s).  4,096 x 4,096 bf16 with zero points in groups of 64 takes 10.5 and 7.8 (42 MB each): quantising by its instructions.
// 16-bit types' ranges are found two elements an instruction, and quotients and their rounding too (one by one 13.6 us; with
// one word of codes a thread and a division's two corrections 19.2); two tiles a thread instead of four took 10.9.
#include <math.h>
#include <string.h>

#include <type_traits>

#include "g4.cuh"
#include "sm100.cuh"

MPQ_CHECKED_UNIT("g4.cu");

namespace mpq {
namespace {

constexpr int G4_THREADS = 256;              // of a tile: a word each
constexpr int G4_PITCH = 132;                // floats of a staged row: rows apart in the banks

__device__ __forceinline__ float bf16_rn(float v) { return __bfloat162float(__float2bfloat16_rn(v)); }

// RN(x / s) for an s of 8 significant bits, r = 1 / s to within 2^-22 of it.  x r is off by 2^-21 of it at most, its remainder
// x - y s is exact, and y + (x - y s) r by 2^-43 of it before its rounding.  With X and M whole numbers of 24 and 25 bits,
// M odd, and S of 8, X / S differs from M, a midpoint between two floats, by a multiple of 1 / S, and not by 0 (M S
// has an odd part of 25 bits or more): by 2^-33 of it or more, so the rounding is that of x / s.
__device__ __forceinline__ float quotient(float x, float s, float r)
{
    const float y = __fmul_rn(x, r);
    return __fmaf_rn(__fmaf_rn(-y, s, x), r, y);
}

__device__ __forceinline__ float near_reciprocal(float s)
{
    float r;
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(s));
    return r;
}

// For scales that quotient() is not for.  Functions of their own: a division's code among the quotients cost 2 of 11 us.
__device__ __noinline__ float divided(float x, float s) { return __fdiv_rn(x, s); }
__device__ __noinline__ uint32_t divided_codes(float2 a, float2 b, float2 c, float2 d, float s, int z, float least, float most)
{
    const float x[8] = {a.x, a.y, b.x, b.y, c.x, c.y, d.x, d.y};
    uint32_t w = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i)
        w |= (uint32_t)(z + (int)rintf(fminf(fmaxf(__fdiv_rn(x[i], s), least), most))) << g4_shift(i);
    return w;
}

// The nearest whole number (|y| below 2^22, ties to even).
__device__ __forceinline__ int whole(float y)
{
    return __float_as_int(__fadd_rn(y, 12582912.0f)) - __float_as_int(12582912.0f);
}

// A thread's 16 elements as they were read, and their range: the largest |x| (0 beside it), or with ZEROS the largest of x
// and 0 and the largest of -x and 0; NaN if an element is.
template <typename T>
struct Sixteen {
    uint32_t w[8];                           // two elements each

    using Two = std::conditional_t<std::is_same_v<T, __half>, __half2, __nv_bfloat162>;
    __device__ static __forceinline__ uint32_t more(uint32_t a, uint32_t b)
    {
        const Two m = __hmax2_nan(as(a), as(b));
        return *reinterpret_cast<const uint32_t *>(&m);
    }
    __device__ static __forceinline__ uint32_t less(uint32_t a, uint32_t b)
    {
        const Two m = __hmin2_nan(as(a), as(b));
        return *reinterpret_cast<const uint32_t *>(&m);
    }
    __device__ static __forceinline__ Two as(uint32_t v) { return *reinterpret_cast<Two *>(&v); }

    __device__ __forceinline__ void load(const T *x) { load_words(reinterpret_cast<const uint32_t *>(x), w); }
    __device__ __forceinline__ void pair(int i, float a, float b) { w[i] = pack2(a, b, T()); }
    __device__ __forceinline__ float2 pair(int i) const { return unpack2(w[i], T()); }

    template <bool ZEROS>
    __device__ __forceinline__ float2 range(int threads) const
    {
        constexpr uint32_t off = ZEROS ? 0xffffffffu : 0x7fff7fffu;
        uint32_t m = w[0] & off;
#pragma unroll
        for (int i = 1; i < 8; ++i) m = more(m, w[i] & off);
        if (ZEROS) {                         // the pairs' largest, and their least with its sign turned
            uint32_t l = w[0];
#pragma unroll
            for (int i = 1; i < 8; ++i) l = less(l, w[i]);
            m = more(__byte_perm(m, l, 0x5410) ^ 0x80000000u, __byte_perm(m, l, 0x7632) ^ 0x80000000u);
        }
#pragma unroll
        for (int o = 1; o < 8; o <<= 1) {
            if (o >= threads) break;
            m = more(m, __shfl_xor_sync(0xffffffffu, m, o));
        }
        if (ZEROS) return unpack2(more(m, 0u), T());
        return {unpack2(more(m, m >> 16), T()).x, 0.0f};
    }
};

template <>
struct Sixteen<float> {
    float v[16];

    __device__ static __forceinline__ float more(float a, float b, float c)
    {
        float m;
        asm("max.NaN.f32 %0, %1, %2, %3;" : "=f"(m) : "f"(a), "f"(b), "f"(c));
        return m;
    }
    __device__ static __forceinline__ float less(float a, float b, float c)
    {
        float m;
        asm("min.NaN.f32 %0, %1, %2, %3;" : "=f"(m) : "f"(a), "f"(b), "f"(c));
        return m;
    }

    __device__ __forceinline__ void load(const float *x) { load16(x, v); }
    __device__ __forceinline__ void pair(int i, float a, float b) { v[2 * i] = a, v[2 * i + 1] = b; }
    __device__ __forceinline__ float2 pair(int i) const { return {v[2 * i], v[2 * i + 1]}; }

    template <bool ZEROS>
    __device__ __forceinline__ float2 range(int threads) const
    {
        float m = ZEROS ? 0.0f : __uint_as_float(top_bits(v)), l = 0.0f;
        if (ZEROS) {
#pragma unroll
            for (int i = 0; i < 16; i += 2) {
                m = more(m, v[i], v[i + 1]);
                l = less(l, v[i], v[i + 1]);
            }
        }
        l = -l;
#pragma unroll
        for (int o = 1; o < 8; o <<= 1) {
            if (o >= threads) break;
            m = more(m, __shfl_xor_sync(0xffffffffu, m, o), 0.0f);
            if (ZEROS) l = more(l, __shfl_xor_sync(0xffffffffu, l, o), 0.0f);
        }
        return {m, l};
    }
};

struct G4Group {
    float s, r;
    int z;
    bool plain;                              // s lies where quotient() is exact; r is its reciprocal
};

// The scale and zero point of a group of `threads` threads (2, 4 or 8 lanes of a warp) of 16 elements.  The scale before its
// rounding is finite where all elements are.
template <bool ZEROS, typename T>
__device__ __forceinline__ G4Group group_of(const Sixteen<T> &v, int threads)
{
    const float2 m = v.template range<ZEROS>(threads);
    constexpr float seventh = 1.0f / 7.0f, fifteenth = 1.0f / 15.0f;
    const float s = ZEROS ? __fadd_rn(__fmul_rn(m.x, fifteenth), __fmul_rn(m.y, fifteenth)) : __fmul_rn(m.x, seventh);
    G4Group g;
    g.s = s < INFINITY ? bf16_rn(s) : NAN;
    g.plain = g.s >= 0x1p-100f && g.s <= 0x1p100f;
    g.r = near_reciprocal(g.s);
    g.z = G4_ZERO;
    if (ZEROS && g.s > 0.0f) {
        const float z = g.plain ? quotient(m.y, g.s, g.r) : divided(m.y, g.s);
        g.z = min(max(whole(fminf(z, 32.0f)), 0), 15);
    }
    return g;
}

// The word of the eight codes of pairs p .. p + 3.  1.5 * 2^23 + 16 is added to a quotient, which rounds it to the whole
// number in the sum's low bits, plus 16.  A scale that is a normal number is less than 2^-8 below its group's
// range / 7 or / 15, so |x / s| <= 7.03, or x / s in [-15.06, 15.06]: without zero points all codes are in the range.  With
// them z is the least element's quotient rounded, and no other rounds to less than -z, while the largest may come
// to 16.  Two sums' low halves lie in a word as two elements' codes do, so a word is four such pairs in their places,
// less what the 16s and z come to (all modulo 2^32).
template <bool ZEROS, typename T>
__device__ __forceinline__ uint32_t codes_of(const Sixteen<T> &v, int p, const G4Group &g)
{
    constexpr float big = 12582912.0f + 16.0f;
    if (!(g.s > 0.0f)) return (uint32_t)g.z * 0x11111111u;
    if (!g.plain)
        return divided_codes(v.pair(p), v.pair(p + 1), v.pair(p + 2), v.pair(p + 3), g.s, g.z,
                             ZEROS ? (float)-g.z : -7.0f, ZEROS ? (float)(15 - g.z) : 7.0f);
    uint32_t w = (uint32_t)(g.z - 16) * 0x11111111u;
    const uint32_t most = (uint32_t)(31 - g.z) * 0x10001u;
    const float2 s = {-g.s, -g.s}, r = {g.r, g.r};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const float2 x = v.pair(p + i);
        float2 y = mul2(x, r);               // quotient()
        y = fma2(fma2(y, s, x), r, y);
        y = add2(y, {big, big});
        const uint32_t two = __byte_perm(__float_as_uint(y.x), __float_as_uint(y.y), 0x5410);
        w += (ZEROS ? __vmins2(two, most) : two) << (4 * i);
    }
    return w;
}

// What a CTA has of a matrix: `most` tiles of 16 rows x 128 elements along a row from tile kt0 on, `here` of them there.
struct TileRun {
    int rt, kt0, here;
    long long row0;
};
__device__ __forceinline__ TileRun tile_run(const mpq_g4_matrix &L, int most)
{
    const int runs = (L.k_tiles + most - 1) / most, rt = (int)blockIdx.x / runs;
    const int kt0 = ((int)blockIdx.x - rt * runs) * most;
    return {rt, kt0, min(most, L.k_tiles - kt0), (long long)rt * 16};
}

// A thread has 16 elements of U tiles, and 128 threads a tile's 16 rows; the CTA's two halves take U tiles each.  VEC: rows
// are 16-byte aligned, and all of a thread's elements are on their way before the first is used; else (U = 1) rows
// pass through shared memory, a warp's accesses consecutive.  Four CTAs an SM: fp32 with zero points, 11,008 x 4,096, is
// 36.4 us with the two registers more that leave three, 33.6 with four.  (Four cost 16-bit rows with zero points two spilled
// words.)
template <typename T, bool VEC, bool ZEROS, int U>
__global__ void __launch_bounds__(G4_THREADS, U > 1 ? 4 : 1)
g4_quantize_kernel(const T *X, long long ldx, mpq_g4_matrix L, unsigned char *packed)
{
    static_assert(VEC || U == 1, "one staged tile of a half");
    __shared__ float stage[VEC ? 1 : 2 * 16 * G4_PITCH];
    sm100::griddep_launch();
    sm100::griddep_wait();
    const TileRun run = tile_run(L, 2 * U);
    const int part = (int)threadIdx.x >> 7, in_tile = ((int)threadIdx.x >> 3) & 15, n = 2 * (threadIdx.x & 7);
    const int k0 = run.kt0 + part * U;
    Sixteen<T> v[U];
    if constexpr (VEC) {
        const long long row = run.row0 + in_tile;
        const bool real = row < L.rows;
        const T *const x = X + (real ? row : 0) * ldx;
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int j = (k0 + u) * 128 + n * 8;
            if (real && j + 16 <= L.d) {
                v[u].load(x + j);
            } else {
#pragma unroll
                for (int i = 0; i < 8; ++i)
                    v[u].pair(i, real && j + 2 * i < L.d ? to_f32(x[j + 2 * i]) : 0.0f,
                              real && j + 2 * i + 1 < L.d ? to_f32(x[j + 2 * i + 1]) : 0.0f);
            }
        }
    } else {
#pragma unroll
        for (int i = 0; i < 16; ++i) {
            const int e = (int)threadIdx.x + i * G4_THREADS, r = e >> 8, j = e & 255;        // a row of both tiles
            const bool real = run.row0 + r < L.rows && run.kt0 * 128 + j < L.d;
            stage[((j >> 7) * 16 + r) * G4_PITCH + (j & 127)] =
                real ? to_f32(X[(run.row0 + r) * ldx + run.kt0 * 128 + j]) : 0.0f;
        }
        __syncthreads();
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const float *const at = stage + (part * 16 + in_tile) * G4_PITCH + n * 8 + 2 * i;
            v[0].pair(i, at[0], at[1]);
        }
    }
    const int threads = L.group >> 4, groups = 128 / L.group;
#pragma unroll
    for (int u = 0; u < U; ++u) {
        const G4Group g = group_of<ZEROS>(v[u], threads);
        const uint32_t w0 = codes_of<ZEROS>(v[u], 0, g), w1 = codes_of<ZEROS>(v[u], 4, g);
        const size_t at = ((size_t)run.rt * L.k_tiles + k0 + u) * L.tile_bytes;
        if (part * U + u >= run.here || !MPQ_IN(at + L.tile_bytes - 1, L.bytes)) return;
        unsigned char *const tile = packed + at;
        *reinterpret_cast<uint32_t *>(tile + in_tile * 64 + g4_word(n)) = w0;
        *reinterpret_cast<uint32_t *>(tile + in_tile * 64 + g4_word(n + 1)) = w1;
        if (((n >> 1) & (threads - 1)) == 0) {
            const int i = in_tile * groups + (n >> 1) / threads;
            reinterpret_cast<__nv_bfloat16 *>(tile + G4_CODES)[i] = __float2bfloat16_rn(g.s);
            if (ZEROS) tile[G4_CODES + 32 * groups + i] = (unsigned char)g.z;
        }
    }
}

template <typename T, bool VEC, int U>
__global__ void __launch_bounds__(G4_THREADS)
g4_dequantize_kernel(const unsigned char *packed, mpq_g4_matrix L, T *Y, long long ldy)
{
    static_assert(VEC || U == 1, "one staged tile");
    __shared__ float stage[VEC ? 1 : 16 * G4_PITCH];
    sm100::griddep_launch();
    sm100::griddep_wait();
    const TileRun run = tile_run(L, U);
    const int n = threadIdx.x & 15, in_tile = (int)threadIdx.x >> 4, groups = 128 / L.group;
    const long long row = run.row0 + in_tile;
    const int at = in_tile * groups + n * 8 / L.group;
    const size_t size = (L.rows - 1) * ldy + L.d;
    uint32_t w[U];
    float s[U];
    int z[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
        const unsigned char *const tile = packed + ((size_t)run.rt * L.k_tiles + run.kt0 + min(u, run.here - 1)) * L.tile_bytes;
        w[u] = *reinterpret_cast<const uint32_t *>(tile + in_tile * 64 + g4_word(n));
        s[u] = bf16_bits(reinterpret_cast<const uint16_t *>(tile + G4_CODES)[at]);
        z[u] = L.zeros ? tile[G4_CODES + 32 * groups + at] : G4_ZERO;
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
        float v[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = __fmul_rn((float)((int)(w[u] >> g4_shift(i) & 15u) - z[u]), s[u]);
        if constexpr (VEC) {
            const int j = (run.kt0 + u) * 128 + n * 8;
            if (row >= L.rows || j >= L.d || !MPQ_IN(row * ldy + min(j + 8, L.d) - 1, size)) return;
            T *const y = Y + row * ldy + j;
            if (j + 8 <= L.d) {
                store8(y, v);
            } else {
#pragma unroll
                for (int i = 0; i < 8; ++i)
                    if (j + i < L.d) y[i] = from_f32<T>(v[i]);
            }
        } else {
#pragma unroll
            for (int i = 0; i < 8; ++i) stage[in_tile * G4_PITCH + n * 8 + i] = v[i];
            __syncthreads();
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const int e = (int)threadIdx.x + i * G4_THREADS, r = e >> 7, j = run.kt0 * 128 + (e & 127);
                if (run.row0 + r < L.rows && j < L.d && MPQ_IN((run.row0 + r) * ldy + j, size))
                    Y[(run.row0 + r) * ldy + j] = from_f32<T>(stage[r * G4_PITCH + (e & 127)]);
            }
        }
    }
}

// Whether `each` tiles to a CTA leave every SM its fill of CTAs (`fill`).
bool by_many(const mpq_g4_matrix *L, bool vec, int each, int fill)
{
    return vec && (long long)L->row_tiles * ((L->k_tiles + each - 1) / each) >= (long long)fill * sm_count();
}
dim3 tile_grid(const mpq_g4_matrix *L, int each)
{
    return dim3((unsigned)L->row_tiles * (unsigned)((L->k_tiles + each - 1) / each));
}

template <typename T, bool ZEROS>
mpq_status quantize_typed(const void *X, bool vec, long long ldx, const mpq_g4_matrix *L, void *packed, cudaStream_t stream)
{
    constexpr int U = sizeof(T) == 2 ? 4 : 2;                // 128 bytes a thread on their way
    const bool many = by_many(L, vec, 2 * U, 16 / U);
    return launch_waiting(many  ? g4_quantize_kernel<T, true, ZEROS, U>
                          : vec ? g4_quantize_kernel<T, true, ZEROS, 1>
                                : g4_quantize_kernel<T, false, ZEROS, 1>,
                          tile_grid(L, many ? 2 * U : 2), dim3(G4_THREADS), 0, stream, "g4 quantize launch",
                          static_cast<const T *>(X), ldx, *L, static_cast<unsigned char *>(packed));
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
        return L->zeros ? quantize_typed<T, true>(X, vec, ldx, L, packed, stream)
                        : quantize_typed<T, false>(X, vec, ldx, L, packed, stream);
    });
}

mpq_status launch_g4_dequantize(const void *packed, const mpq_g4_matrix *L, void *Y, int y_type, long long ldy,
                                cudaStream_t stream)
{
    const bool vec = aligned(Y, y_type, ldy, L->rows);
    return by_type(y_type, [&](auto t) {
        using T = decltype(t);
        const int each = by_many(L, vec, 4, 8) ? 4 : 1;
        return launch_waiting(each > 1 ? g4_dequantize_kernel<T, true, 4>
                              : vec    ? g4_dequantize_kernel<T, true, 1>
                                       : g4_dequantize_kernel<T, false, 1>,
                              tile_grid(L, each), dim3(G4_THREADS), 0, stream,
                              "g4 dequantize launch", static_cast<const unsigned char *>(packed), *L,
                              static_cast<T *>(Y), ldy);
    });
}

}  // namespace mpq
