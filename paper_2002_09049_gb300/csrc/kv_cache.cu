// The few-bit key-value cache: quantising tokens as they are written (mpq_cache_write) and reading
// slots back (mpq_cache_read).
//
// A row is what one token keeps for one head (its key, or its value): s = max|x| (1 / Qmax), one fp32
// product, codes clamp(rint(x / s)) as Eq. 8's.  A thread takes 16 elements of a row, so dim / 16 threads
// (4, 8 or 16 of a warp) share its maximum by shuffles, and their codes leave in one store of 16 or 8 bytes
// a thread.  Writing, keys and values have threads of their own (1,999 tokens of 4 x 64 fp32 to 4 bits: 2.7 us,
// 3.5 with a key and a value row a thread; 32 elements a thread leave too few warps: 22.9 us instead of
// 15.7 for 8,192 tokens of 8 x 128 bf16, before the quotients below took one step); reading, a thread takes
// both.
//
// The quotient x / s has to be the correctly rounded one: 16-bit inputs meet near-ties all the time
// (elements whose ratio to the row's largest is a simple fraction: in 70% of a warp's 512 bf16 elements
// there is one, so that a screen with an exact way out gains nothing).  One correctly rounded reciprocal r
// a row, and Markstein's theorem (IBM J. Res. Dev. 34(1), 1990): a y within a unit in the last place of
// x / s gives RN(x / s) as RN(y + r (x - s y)), the remainder exact by a fused multiply-add.  RN(x r) is
// within 1.5 units, so one step (its remainder may have a bit too many, and is rounded) brings it within one,
// and the next is the quotient.  For elements and maxima of 11 bits or fewer the first step gives it already
// (all of them tried, with every rounding: tests/test_cache_quotient_steps.py).
// Rows whose scale is so small or large that r or a remainder could leave the normal range are divided.
//
// Memory-bound: an element's own bytes on one side, bits / 8 + 4 / dim bytes on the other; slots scatter
// rows of 32 to 256 bytes, whole sectors.  8,192 tokens of 8 x 128 bf16 to 8 bits: written in 12.6 us (51 MB,
// 4.0 TB/s; issue slots 74% busy), read back in 9.9 us (5.1 TB/s).
#include <math.h>
#include <string.h>

#include "elements.cuh"
#include "mpq_internal.cuh"
#include "sm100.cuh"

MPQ_CHECKED_UNIT("kv_cache.cu");

namespace mpq {
namespace {

constexpr int KV_THREADS = 256;

// A thread's place: token, head (blockIdx.y; writing, the heads' keys, then their values), and its first
// element of the row.
struct RowAt {
    int t, h, j0;
};
__device__ __forceinline__ bool row_at(int T, const mpq_kv_cache &L, RowAt &at)
{
    const int shift = L.dim == 64 ? 2 : L.dim == 128 ? 3 : 4;       // of dim / 16 threads a row
    at.t = (int)(blockIdx.x * (unsigned)(KV_THREADS >> shift) + (threadIdx.x >> shift));
    at.h = (int)blockIdx.y;
    at.j0 = (int)(threadIdx.x & ((1u << shift) - 1u)) * 16;
    return at.t < T;
}

// Index of a slot's key row among the cache's rows (its value row is heads * page further: head h + heads),
// or -1 for a slot outside the cache.
__device__ __forceinline__ long long cache_row(long long slot, const mpq_kv_cache &L, int page_shift, int h)
{
    if (slot < 0 || slot >= (long long)L.pages * L.page) return -1;
    const long long page = page_shift >= 0 ? slot >> page_shift : slot / L.page;
    return (page * 2 * L.heads + h) * L.page + (slot - page * L.page);
}

// max |x| of a row as bits (infinities and NaN above every finite value), over its `per` threads.
__device__ __forceinline__ uint32_t row_top(const float (&v)[16], unsigned per, unsigned lanes)
{
    uint32_t top = top_bits(v);
    for (unsigned o = 1; o < per; o <<= 1) top = max(top, __shfl_xor_sync(lanes, top, o));
    return top;
}

// Scales whose reciprocal, and whose quotients' remainders where the code is not 0, are normal.
constexpr float KV_LEAST = 0x1p-100f, KV_MOST = 0x1p100f;

// The codes of 16 elements, offset by Qmax + 1, in the low bits of each word, and the row's scale; STEPS
// corrections of a quotient.
template <int STEPS>
__device__ __forceinline__ float row_codes(const float (&v)[16], uint32_t top, int qmax,
                                           float inv_qmax, uint32_t (&u)[16])
{
    const float s = top >= 0x7f800000u ? NAN : __fmul_rn(__uint_as_float(top), inv_qmax);
    const int zero = qmax + 1;
    if (s >= KV_LEAST && s <= KV_MOST) {
        const float r = __frcp_rn(s);
        const float magic = 12582912.0f + (float)zero;  // 3 2^22 + offset: the sum's low bits are the code
#pragma unroll
        for (int i = 0; i < 16; ++i) {
            float y = __fmul_rn(v[i], r);
#pragma unroll
            for (int k = 0; k < STEPS; ++k) y = __fmaf_rn(__fmaf_rn(-y, s, v[i]), r, y);
            u[i] = __float_as_uint(__fadd_rn(y, magic));
        }
    } else {
#pragma unroll
        for (int i = 0; i < 16; ++i) u[i] = __float_as_uint(v[i]);
#pragma unroll 1
        for (int i = 0; i < 16; ++i) {
            uint32_t x = 0;
#pragma unroll
            for (int k = 0; k < 16; ++k) x = k == i ? u[k] : x;
            int q = 0;
            if (s > 0.0f) q = min(max(__float2int_rn(__fdiv_rn(__uint_as_float(x), s)), -qmax), qmax);
#pragma unroll
            for (int k = 0; k < 16; ++k)
                if (k == i) u[k] = (uint32_t)(q + zero);
        }
    }
    return s;
}

__device__ __forceinline__ uint32_t low_bytes(const uint32_t *u)
{
    return __byte_perm(__byte_perm(u[0], u[1], 0x0040), __byte_perm(u[2], u[3], 0x0040), 0x5410);
}

// Stores a thread's 16 codes and, by the row's first thread, its scale.
__device__ __forceinline__ void store_row(const uint32_t (&u)[16], float s, long long row, int j0,
                                          const mpq_kv_cache &L, unsigned char *codes, float *scales)
{
    if (!MPQ_IN(row, (size_t)L.pages * 2 * L.heads * L.page)) return;
    unsigned char *const out = codes + row * L.row_bytes;
    if (L.bits == 8) {
        *reinterpret_cast<uint4 *>(out + j0) = make_uint4(low_bytes(u), low_bytes(u + 4),
                                                          low_bytes(u + 8), low_bytes(u + 12));
    } else {
        uint32_t w[2] = {0, 0};
#pragma unroll
        for (int i = 0; i < 16; ++i) w[i >> 3] |= (u[i] & 15u) << (4 * (i & 7));
        *reinterpret_cast<uint2 *>(out + j0 / 2) = make_uint2(w[0], w[1]);
    }
    if (j0 == 0) scales[row] = s;
}

template <typename T, bool VEC>
__global__ void __launch_bounds__(KV_THREADS)
cache_write_kernel(const T *K, const T *V, long long ld_token, long long ld_head, int n,
                   const int64_t *slots, mpq_kv_cache L, int page_shift, float inv_qmax, unsigned char *codes,
                   float *scales)
{
    sm100::griddep_launch();
    sm100::griddep_wait();
    RowAt at;
    if (!row_at(n, L, at)) return;   // whole rows (dim / 16 threads) leave together
    const bool value = at.h >= L.heads;
    const T *const x = (value ? V : K) + ld_token * at.t + ld_head * (value ? at.h - L.heads : at.h) + at.j0;
    const long long slot = slots[at.t];
    float v[16];
    if (VEC) {
        load16(x, v);
    } else {
#pragma unroll
        for (int i = 0; i < 16; ++i) v[i] = to_f32(x[i]);
    }
    const long long row = cache_row(slot, L, page_shift, at.h);
    if (row < 0) return;
    const unsigned per = (unsigned)L.dim / 16;
    const unsigned lanes = ((1u << per) - 1u) << (threadIdx.x & 31 & ~(per - 1));
    const int qmax = (1 << (L.bits - 1)) - 1;
    uint32_t u[16];
    const float s = row_codes<sizeof(T) == 2 ? 1 : 2>(v, row_top(v, per, lanes), qmax, inv_qmax, u);
    store_row(u, s, row, at.j0, L, codes, scales);
}

// The values of 16 codes (four words, or two) with a scale.
__device__ __forceinline__ void row_values(uint4 w, float s, int bits, float (&v)[16])
{
    const uint32_t q[4] = {w.x, w.y, w.z, w.w};
    if (bits == 8) {
#pragma unroll
        for (int i = 0; i < 16; ++i)
            v[i] = s * (float)((int)((q[i >> 2] >> (8 * (i & 3))) & 255u) - 128);
    } else {
#pragma unroll
        for (int i = 0; i < 16; ++i) v[i] = s * (float)((int)((q[i >> 3] >> (4 * (i & 7))) & 15u) - 8);
    }
}

__device__ __forceinline__ uint4 load_codes(const unsigned char *row, int j0, int bits)
{
    if (bits == 8) return *reinterpret_cast<const uint4 *>(row + j0);
    const uint2 w = *reinterpret_cast<const uint2 *>(row + j0 / 2);
    return make_uint4(w.x, w.y, 0, 0);
}

template <typename T>
__global__ void __launch_bounds__(KV_THREADS)
cache_read_kernel(const int64_t *slots, int n, mpq_kv_cache L, int page_shift,
                  const unsigned char *codes, const float *scales, T *K, T *V)
{
    sm100::griddep_launch();
    sm100::griddep_wait();
    RowAt at;
    if (!row_at(n, L, at)) return;
    const long long row = cache_row(slots[at.t], L, page_shift, at.h);
    const long long v_row = row + (long long)L.heads * L.page;
    uint4 kw = make_uint4(0, 0, 0, 0), vw = make_uint4(0, 0, 0, 0);
    float ks = 0.0f, vs = 0.0f;      // (a slot outside the cache: zeros)
    if (row >= 0) {
        ks = scales[row];
        vs = scales[v_row];
        kw = load_codes(codes + row * L.row_bytes, at.j0, L.bits);
        vw = load_codes(codes + v_row * L.row_bytes, at.j0, L.bits);
    }
    float v[16];
    const size_t to = ((size_t)at.t * L.heads + at.h) * L.dim + at.j0;
    if (!MPQ_IN(to + 15, (size_t)n * L.heads * L.dim)) return;
    row_values(kw, ks, L.bits, v);
    store16(K + to, v);
    row_values(vw, vs, L.bits, v);
    store16(V + to, v);
}

// Blocks of KV_THREADS threads for T tokens' rows, by head.
dim3 kv_grid(int T, const mpq_kv_cache *L, int heads)
{
    const long long per_block = KV_THREADS / (L->dim / 16);
    return dim3((unsigned)((T + per_block - 1) / per_block), (unsigned)heads, 1);
}

// log2 of the page, -1 where it is no power of two.
int page_shift(const mpq_kv_cache *L)
{
    int s = 0;
    while (1 << s < L->page) ++s;
    return 1 << s == L->page ? s : -1;
}

}  // namespace

mpq_status make_cache_layout(int pages, int page, int heads, int dim, int bits, mpq_kv_cache *L)
{
    memset(L, 0, sizeof(*L));
    L->pages = pages;
    L->page = page;
    L->heads = heads;
    L->dim = dim;
    L->bits = bits;
    L->row_bytes = dim * bits / 8;
    const size_t rows = (size_t)pages * 2 * heads * page;
    L->codes_bytes = rows * L->row_bytes;
    L->scales_bytes = rows * sizeof(float);
    return MPQ_OK;
}

mpq_status launch_cache_write(const void *K, const void *V, int type, long long ld_token,
                              long long ld_head, int T, const int64_t *slots,
                              const mpq_kv_cache *L, void *codes, float *scales,
                              cudaStream_t stream)
{
    const bool vec = rows_aligned(K, type, ld_token) && rows_aligned(V, type, ld_head);
    return by_type(type, [&](auto t) {
        using E = decltype(t);
        return launch_waiting(vec ? cache_write_kernel<E, true> : cache_write_kernel<E, false>,
                              kv_grid(T, L, 2 * L->heads), dim3(KV_THREADS), 0, stream,
                              "cache write launch", static_cast<const E *>(K),
                              static_cast<const E *>(V), ld_token, ld_head, T, slots, *L,
                              page_shift(L), 1.0f / (float)((1 << (L->bits - 1)) - 1),
                              static_cast<unsigned char *>(codes), scales);
    });
}

mpq_status launch_cache_read(const int64_t *slots, int T, const mpq_kv_cache *L, const void *codes,
                             const float *scales, void *K, void *V, int type, cudaStream_t stream)
{
    return by_type(type, [&](auto t) {
        using E = decltype(t);
        return launch_waiting(cache_read_kernel<E>, kv_grid(T, L, L->heads), dim3(KV_THREADS), 0,
                              stream, "cache read launch", slots, T, *L, page_shift(L),
                              static_cast<const unsigned char *>(codes), scales,
                              static_cast<E *>(K), static_cast<E *>(V));
    });
}

}  // namespace mpq
