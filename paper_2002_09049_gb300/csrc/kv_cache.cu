// The few-bit key-value cache: quantising tokens as they are written (mpq_cache_write) and reading
// slots back (mpq_cache_read).
//
// A row is what one token keeps for one head (its key, or its value): s = max|x| (1 / Qmax), one fp32
// product, codes clamp(rint(x / s)) as Eq. 8's, by one correctly rounded division each.  A thread takes 8 elements
// of a row, so dim / 8 threads (8, 16 or 32 of a warp) share its maximum by shuffles, and its codes
// leave in one store of 8 or 4 bytes a thread.  Memory-bound: an element's own bytes on one side,
// bits / 8 + 4 / dim bytes on the other; slots scatter rows of 32 to 256 bytes, whole sectors.
#include <math.h>
#include <string.h>

#include "elements.cuh"
#include "mpq_internal.cuh"
#include "sm100.cuh"

MPQ_CHECKED_UNIT("kv_cache.cu");

namespace mpq {
namespace {

constexpr int KV_THREADS = 256;

// A thread's row: token, key or value, head, and its first element.
struct RowAt {
    int t, kv, h, j0;
};
__device__ __forceinline__ bool row_at(int T, const mpq_kv_cache &L, RowAt &at)
{
    const unsigned per = (unsigned)L.dim / 8;
    const unsigned r = blockIdx.x * (KV_THREADS / per) + threadIdx.x / per;
    const unsigned of_token = 2u * (unsigned)L.heads;
    at.t = (int)(r / of_token);
    const unsigned rest = r - (unsigned)at.t * of_token;
    at.kv = rest >= (unsigned)L.heads;
    at.h = (int)rest - at.kv * L.heads;
    at.j0 = (int)(threadIdx.x & (per - 1)) * 8;
    return at.t < T;
}

// Index of a slot's row among the cache's rows, or -1 for a slot outside it.
__device__ __forceinline__ long long cache_row(long long slot, const mpq_kv_cache &L, int kv, int h)
{
    if (slot < 0 || slot >= (long long)L.pages * L.page) return -1;
    const long long page = slot / L.page;
    return ((page * 2 + kv) * L.heads + h) * L.page + (slot - page * L.page);
}

template <typename T, bool VEC>
__global__ void __launch_bounds__(KV_THREADS)
cache_write_kernel(const T *K, const T *V, long long ld_token, long long ld_head, int n,
                   const int64_t *slots, mpq_kv_cache L, unsigned char *codes, float *scales)
{
    sm100::griddep_launch();
    sm100::griddep_wait();
    RowAt at;
    if (!row_at(n, L, at)) return;   // whole rows (dim / 8 threads) leave together
    const long long row = cache_row(slots[at.t], L, at.kv, at.h);
    if (row < 0) return;
    const T *x = (at.kv ? V : K) + ld_token * at.t + ld_head * at.h + at.j0;
    float v[8];
    if (VEC) {
        load8(x, v);
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = to_f32(x[i]);
    }
    // max |x| as bits (infinities and NaN above every finite value), over the row's threads
    uint32_t top = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) top = max(top, __float_as_uint(v[i]) & 0x7fffffffu);
    const unsigned per = (unsigned)L.dim / 8;
    const unsigned lanes = per == 32 ? 0xffffffffu : ((1u << per) - 1u)
                                                         << (threadIdx.x & 31 & ~(per - 1));
    for (unsigned o = 1; o < per; o <<= 1) top = max(top, __shfl_xor_sync(lanes, top, o));
    const int qmax = (1 << (L.bits - 1)) - 1;
    const bool bad = top >= 0x7f800000u;
    const float s = bad ? NAN : __fmul_rn(__uint_as_float(top), __fdiv_rn(1.0f, (float)qmax));
    uint32_t u[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        int q = 0;
        if (s > 0.0f) q = min(max(__float2int_rn(__fdiv_rn(v[i], s)), -qmax), qmax);
        u[i] = (uint32_t)(q + qmax + 1);
    }
    const size_t rows = (size_t)L.pages * 2 * L.heads * L.page;
    if (!MPQ_IN(row, rows)) return;
    unsigned char *out = codes + row * L.row_bytes;
    if (L.bits == 8) {
        *reinterpret_cast<uint2 *>(out + at.j0) =
            make_uint2(u[0] | u[1] << 8 | u[2] << 16 | u[3] << 24,
                       u[4] | u[5] << 8 | u[6] << 16 | u[7] << 24);
    } else {
        uint32_t w = 0;
#pragma unroll
        for (int i = 0; i < 8; ++i) w |= u[i] << (4 * i);
        *reinterpret_cast<uint32_t *>(out + at.j0 / 2) = w;
    }
    if (at.j0 == 0) scales[row] = s;
}

template <typename T>
__global__ void __launch_bounds__(KV_THREADS)
cache_read_kernel(const int64_t *slots, int n, mpq_kv_cache L, const unsigned char *codes,
                  const float *scales, T *K, T *V)
{
    sm100::griddep_launch();
    sm100::griddep_wait();
    RowAt at;
    if (!row_at(n, L, at)) return;
    const long long row = cache_row(slots[at.t], L, at.kv, at.h);
    float v[8];
    if (row < 0) {
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = 0.0f;
    } else {
        const float s = scales[row];
        const unsigned char *in = codes + row * L.row_bytes;
        if (L.bits == 8) {
            const uint2 w = *reinterpret_cast<const uint2 *>(in + at.j0);
#pragma unroll
            for (int i = 0; i < 8; ++i)
                v[i] = s * (float)((int)(((i < 4 ? w.x : w.y) >> (8 * (i & 3))) & 255u) - 128);
        } else {
            const uint32_t w = *reinterpret_cast<const uint32_t *>(in + at.j0 / 2);
#pragma unroll
            for (int i = 0; i < 8; ++i) v[i] = s * (float)((int)((w >> (4 * i)) & 15u) - 8);
        }
    }
    const size_t to = ((size_t)at.t * L.heads + at.h) * L.dim + at.j0;
    if (MPQ_IN(to + 7, (size_t)n * L.heads * L.dim)) store8((at.kv ? V : K) + to, v);
}

// Blocks of KV_THREADS threads for T tokens' rows.
unsigned kv_blocks(int T, const mpq_kv_cache *L)
{
    const long long per_block = KV_THREADS / (L->dim / 8);
    return (unsigned)(((long long)T * 2 * L->heads + per_block - 1) / per_block);
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
                              dim3(kv_blocks(T, L)), dim3(KV_THREADS), 0, stream,
                              "cache write launch", static_cast<const E *>(K),
                              static_cast<const E *>(V), ld_token, ld_head, T, slots, *L,
                              static_cast<unsigned char *>(codes), scales);
    });
}

mpq_status launch_cache_read(const int64_t *slots, int T, const mpq_kv_cache *L, const void *codes,
                             const float *scales, void *K, void *V, int type, cudaStream_t stream)
{
    return by_type(type, [&](auto t) {
        using E = decltype(t);
        return launch_waiting(cache_read_kernel<E>, dim3(kv_blocks(T, L)), dim3(KV_THREADS), 0,
                              stream, "cache read launch", slots, T, *L,
                              static_cast<const unsigned char *>(codes), scales,
                              static_cast<E *>(K), static_cast<E *>(V));
    });
}

}  // namespace mpq
