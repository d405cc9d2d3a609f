// Norms of queries and keys for each head and the position rotation in one pass (mpq_rotate).
//
// x' = x w / sqrt(mean x^2 + eps), then pairs (a, b) -> (a cos - b sin, b cos + a sin).  A position times a
// frequency in turns of 64 binary places is the angle's fraction of a turn, exact in wrapping integer
// arithmetic however far the position: no table, and no large argument to reduce.  Its nearest quarter turn
// is taken off before it is rounded to fp32 (24 bits of an angle below pi / 4: 2^-25 of a radian), and put back
// by exchanging cosine and sine.
//
// A CTA takes a token (several where a token has few rows): cosines and sines are made once, in shared memory,
// while the rows are on their way, and used by all heads (made by every row's own threads they cost more
// than the rows' traffic).  A row has dim / 16 threads of 16 elements: eight and the eight that they are paired
// with (their neighbours' form: sixteen consecutive ones), so a pair never leaves its thread.
#include <math.h>

#include <algorithm>

#include "elements.cuh"
#include "mpq_internal.cuh"
#include "sm100.cuh"

MPQ_CHECKED_UNIT("rotate.cu");

namespace mpq {
namespace {

constexpr int ROT_MAX_DIM = 512;

struct RotateArgs {
    mpq_rotate_rows part[2];             // queries, keys (heads 0: none)
    const int *positions;
    const uint64_t *turns;
    int T, dim, rot, shift, norm;
    int tokens;                          // of a CTA
    int per;                             // threads of a row, a power of two
    float eps, inv_dim;
};

// cos and sin of a fraction of a turn.
__device__ __forceinline__ float2 cos_sin(uint64_t turn)
{
    const uint32_t t = (uint32_t)(turn >> 32);
    const uint32_t q = (t + (1u << 29)) >> 30;                       // quarters, the nearest
    const float x = (float)(int)(t - (q << 30)) * 0x1p-31f;          // half turns, |x| <= 1/4
    float s, c;
    sincospif(x, &s, &c);
    if (q & 1) {
        const float y = c;
        c = -s;
        s = y;
    }
    return q & 2 ? make_float2(-c, -s) : make_float2(c, s);
}

// V elements from p on, to p on; VEC: 16-byte aligned.
template <bool VEC, int V, typename T>
__device__ __forceinline__ void load_v(const T *p, float (&v)[V])
{
    if constexpr (VEC) {
        load8(p, v);
    } else {
#pragma unroll
        for (int e = 0; e < V; ++e) v[e] = to_f32(p[e]);
    }
}
template <bool VEC, int V, typename T>
__device__ __forceinline__ void store_v(T *p, const float (&v)[V])
{
    if constexpr (VEC) {
        store8(p, v);
    } else {
#pragma unroll
        for (int e = 0; e < V; ++e) p[e] = from_f32<T>(v[e]);
    }
}

// A thread's U units of a row, each of V elements (a) and V more (b): rotated units first, their pairs
// numbered from V * unit on.
template <int V>
__device__ __forceinline__ void unit_at(int u, int rot, bool neighbours, int &ia, int &ib)
{
    const int turned = rot / 2 / V;
    if (!neighbours && u < turned) {
        ia = u * V;
        ib = rot / 2 + u * V;
    } else {                             // (u * 2 V: what is not turned follows what is)
        ia = u * 2 * V;
        ib = ia + V;
    }
}

template <typename T, int V, int U, bool NEIGHBOURS, bool VEC>
__global__ void __launch_bounds__(512)
rotate_kernel(const RotateArgs a)
{
    extern __shared__ float2 turned[];   // [tokens][rot / 2]
    sm100::griddep_launch();
    sm100::griddep_wait();
    const int t0 = (int)blockIdx.x * a.tokens, half = a.rot / 2, units = a.dim / (2 * V);
    const int tokens = min(a.tokens, a.T - t0);
    const int heads = a.part[0].heads + a.part[1].heads, rows = tokens * heads;
    const int slots = (int)blockDim.x / a.per, lane = (int)threadIdx.x & (a.per - 1);
    const int steps = (rows + slots - 1) / slots;        // (every thread takes part in every step's shuffles)
    for (int step = 0; step < steps; ++step) {
        const int row = step * slots + (int)threadIdx.x / a.per;
        const bool real = row < rows;
        const int tok = real ? row / heads : 0, h = real ? row - tok * heads : 0;
        const bool key = h >= a.part[0].heads;
        const mpq_rotate_rows &p = a.part[key ? 1 : 0];
        const int head = key ? h - a.part[0].heads : h;
        const T *const x = static_cast<const T *>(p.x) + p.ld_token * (t0 + tok) + p.ld_head * head;
        float va[U][V], vb[U][V];
#pragma unroll
        for (int i = 0; i < U; ++i) {
            const int u = lane + i * a.per;
#pragma unroll
            for (int e = 0; e < V; ++e) va[i][e] = vb[i][e] = 0.0f;
            if (!real || u >= units) continue;
            int ia, ib;
            unit_at<V>(u, a.rot, NEIGHBOURS, ia, ib);
            load_v<VEC>(x + ia, va[i]);
            load_v<VEC>(x + ib, vb[i]);
        }
        if (step == 0) {
            for (int i = (int)threadIdx.x; i < tokens * half; i += (int)blockDim.x) {
                const int tok = i / half, f = i - tok * half;
                const long long pos = (long long)a.positions[t0 + tok] + a.shift;
                turned[i] = cos_sin((uint64_t)pos * a.turns[f]);
            }
            __syncthreads();
        }
        float scale = 1.0f;
        if (a.norm) {
            auto squares = [&](float by) {
                float s = 0.0f;
#pragma unroll
                for (int i = 0; i < U; ++i)
#pragma unroll
                    for (int e = 0; e < V; ++e) {
                        const float fa = va[i][e] * by, fb = vb[i][e] * by;
                        s = fmaf(fa, fa, s);
                        s = fmaf(fb, fb, s);
                    }
                for (int o = 1; o < a.per; o <<= 1) s += __shfl_xor_sync(0xffffffffu, s, o);
                return s;
            };
            const float mean = fmaf(squares(1.0f), a.inv_dim, a.eps);
            scale = __frsqrt_rn(mean);
            // squares beyond fp32's range (elements above 2^60): again, of 2^-80 of them
            const bool big = isinf(mean);
            if (__any_sync(0xffffffffu, big)) {
                const float small = fmaf(squares(0x1p-80f), a.inv_dim, a.eps * 0x1p-80f * 0x1p-80f);
                if (big) scale = __frsqrt_rn(small) * 0x1p-80f;
            }
        }
        if (!real) continue;
        const long long to = p.ldy_token * (t0 + tok) + p.ldy_head * head;
        T *const y = static_cast<T *>(p.y) + to;
#pragma unroll
        for (int i = 0; i < U; ++i) {
            const int u = lane + i * a.per;
            if (u >= units) continue;
            int ia, ib;
            unit_at<V>(u, a.rot, NEIGHBOURS, ia, ib);
            if (a.norm) {
#pragma unroll
                for (int e = 0; e < V; ++e) {
                    va[i][e] *= scale;
                    vb[i][e] *= scale;
                    if (p.weight) {
                        va[i][e] *= p.weight[ia + e];
                        vb[i][e] *= p.weight[ib + e];
                    }
                }
            }
            if (u < half / V) {
                const float2 *const cs = turned + tok * half + u * V;
                if (NEIGHBOURS && V > 1) {
                    // pairs (va[0], va[1]), .., (vb[0], vb[1]), ..
#pragma unroll
                    for (int e = 0; e < V; e += 2) {
                        const float2 ca = cs[e / 2], cb = cs[V / 2 + e / 2];
                        float l = va[i][e], r = va[i][e + 1];
                        va[i][e] = l * ca.x - r * ca.y;
                        va[i][e + 1] = r * ca.x + l * ca.y;
                        l = vb[i][e], r = vb[i][e + 1];
                        vb[i][e] = l * cb.x - r * cb.y;
                        vb[i][e + 1] = r * cb.x + l * cb.y;
                    }
                } else {
#pragma unroll
                    for (int e = 0; e < V; ++e) {
                        const float2 c = cs[e];
                        const float l = va[i][e], r = vb[i][e];
                        va[i][e] = l * c.x - r * c.y;
                        vb[i][e] = r * c.x + l * c.y;
                    }
                }
            }
            if (!MPQ_CHECK(tok < tokens && ia + V <= a.dim && ib + V <= a.dim)) continue;
            store_v<VEC>(y + ia, va[i]);
            store_v<VEC>(y + ib, vb[i]);
        }
    }
}

// Strides and bases of rows that take 16-byte accesses.
bool wide_rows(const mpq_rotate_rows &p, int type, int T)
{
    if (p.heads == 0) return true;
    return rows_aligned(p.x, type, T > 1 ? p.ld_token : 0) && rows_aligned(p.x, type, p.heads > 1 ? p.ld_head : 0) &&
           rows_aligned(p.y, type, T > 1 ? p.ldy_token : 0) && rows_aligned(p.y, type, p.heads > 1 ? p.ldy_head : 0);
}

}  // namespace

mpq_status launch_rotate(const mpq_rotate_rows *q, const mpq_rotate_rows *k, int type, int T, int dim,
                         const int *positions, int shift, const uint64_t *turns, int rot, int neighbours,
                         int norm, float eps, cudaStream_t stream)
{
    RotateArgs a = {};
    a.part[0] = *q;
    if (k) a.part[1] = *k;
    a.positions = positions;
    a.turns = turns;
    a.T = T;
    a.dim = dim;
    a.rot = rot;
    a.shift = shift;
    a.norm = norm;
    a.eps = eps;
    a.inv_dim = 1.0f / (float)dim;
    // (the order of a row's sum goes by its sizes, not by its alignment)
    const bool wide = rot % 16 == 0 && dim % 16 == 0;
    const bool vec = wide_rows(a.part[0], type, T) && wide_rows(a.part[1], type, T);
    a.per = 32;
    if (wide)
        for (a.per = 1; a.per < dim / 16;) a.per *= 2;
    const int heads = a.part[0].heads + a.part[1].heads;
    const long long row_threads = (long long)heads * a.per;
    a.tokens = (int)std::max(1LL, std::min<long long>(256 / row_threads, T));
    const int threads = (int)std::min<long long>(512, (a.tokens * row_threads + 31) / 32 * 32);
    const dim3 grid((unsigned)((T + (long long)a.tokens - 1) / a.tokens));
    const size_t smem = (size_t)a.tokens * (rot / 2) * sizeof(float2);
    return by_type(type, [&](auto t) {
        using E = decltype(t);
        auto *const kernel =
            !wide ? (neighbours ? rotate_kernel<E, 1, 8, true, false> : rotate_kernel<E, 1, 8, false, false>)
            : vec ? (neighbours ? rotate_kernel<E, 8, 1, true, true> : rotate_kernel<E, 8, 1, false, true>)
                  : (neighbours ? rotate_kernel<E, 8, 1, true, false> : rotate_kernel<E, 8, 1, false, false>);
        return launch_waiting(kernel,
                              grid, dim3((unsigned)threads), smem, stream, "rotate launch", a);
    });
}

}  // namespace mpq
