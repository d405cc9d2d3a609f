// Norms of queries and keys for each head and the position rotation in one pass (mpq_rotate).
//
// x' = x w / sqrt(mean x^2 + eps), then pairs (a, b) -> (a cos - b sin, b cos + a sin).  A position times a
// frequency in turns of 64 binary places is the angle's fraction of a turn, exact in wrapping integer
// arithmetic however far the position: no table, and no large argument to reduce.  Its nearest quarter turn
// is taken off before it is rounded to fp32 (24 bits of an angle below pi / 4: 2^-25 of a radian), and put back
// by exchanging cosine and sine.
//
// A row has dim / 16 threads of 16 elements: eight and the eight that they are paired with (their neighbours' form:
// sixteen consecutive ones), so a pair never leaves its thread.  A CTA takes a token's rows at a time (those of
// several where a token has few), one token after another: the next one's elements are on their way while the
// last one is turned, and its cosines and sines -- made once for all heads, by every row's own threads they cost
// more than the rows' traffic -- are left in shared memory for it.
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
    int tokens, rows;                    // of a CTA at a time: tokens, a token's rows
    int groups;                          // of `tokens` tokens
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

// Where pair i's cosine and sine lie: eights 80 bytes apart, so that eight threads that read eight each, 16 bytes at a
// time, meet no bank twice.
template <int V>
__host__ __device__ constexpr int place(int i) { return V == 8 ? (i >> 3) * 10 + (i & 7) : i; }

template <int V>
__device__ __forceinline__ void take(const float2 *p, float2 (&cs)[V])
{
    if constexpr (V == 1) {
        cs[0] = *p;
    } else {
#pragma unroll
        for (int e = 0; e < V; e += 2) {
            const float4 f = *reinterpret_cast<const float4 *>(p + e);
            cs[e] = make_float2(f.x, f.y);
            cs[e + 1] = make_float2(f.z, f.w);
        }
    }
}

template <typename T, int V, int U, bool NEIGHBOURS, bool VEC>
__global__ void __launch_bounds__(512)
rotate_kernel(const RotateArgs a)
{
    extern __shared__ __align__(16) float2 turned[];     // [2][tokens][rot / 2], by place
    sm100::griddep_launch();
    sm100::griddep_wait();
    const int half = a.rot / 2, units = a.dim / (2 * V), entries = a.tokens * half, size = place<V>(entries);
    const int lane = (int)threadIdx.x & (a.per - 1), slot = (int)threadIdx.x / a.per;
    const int tok = slot / a.rows, row = (int)blockIdx.y * a.rows + slot - tok * a.rows;
    const int heads = a.part[0].heads + a.part[1].heads;
    const bool mine = tok < a.tokens && row < heads, key = row >= a.part[0].heads;
    const mpq_rotate_rows &p = a.part[key ? 1 : 0];
    const int head = key ? row - a.part[0].heads : row;
    const T *const x = static_cast<const T *>(p.x) + p.ld_head * head;
    T *const y = static_cast<T *>(p.y) + p.ldy_head * head;
    int ia[U], ib[U];
#pragma unroll
    for (int i = 0; i < U; ++i) unit_at<V>(lane + i * a.per, a.rot, NEIGHBOURS, ia[i], ib[i]);
    float va[U][V], vb[U][V], na[U][V], nb[U][V];        // this group's elements, the next one's
    auto fetch = [&](long long t) {
#pragma unroll
        for (int i = 0; i < U; ++i) {
#pragma unroll
            for (int e = 0; e < V; ++e) na[i][e] = nb[i][e] = 0.0f;
            if (!mine || t >= a.T || lane + i * a.per >= units) continue;
            load_v<VEC>(x + p.ld_token * t + ia[i], na[i]);
            load_v<VEC>(x + p.ld_token * t + ib[i], nb[i]);
        }
    };
    // a thread makes the same frequency's turns of every group (and others', where there are more than threads)
    const int own = (int)threadIdx.x, own_tok = half ? own / half : 0;
    const uint64_t own_turn = own < entries ? a.turns[own - own_tok * half] : 0;
    auto position = [&](int group) {
        const long long t = (long long)group * a.tokens + own_tok;
        return own < entries && t < a.T ? a.positions[t] : 0;
    };
    auto turn = [&](int group, int buffer, int at) {
        if (own < entries) turned[buffer * size + place<V>(own)] = cos_sin((uint64_t)((long long)at + a.shift) * own_turn);
        for (int i = own + (int)blockDim.x; i < entries; i += (int)blockDim.x) {
            const int k = i / half;
            const long long t = (long long)group * a.tokens + k;
            if (t >= a.T) continue;
            turned[buffer * size + place<V>(i)] =
                cos_sin((uint64_t)((long long)a.positions[t] + a.shift) * a.turns[i - k * half]);
        }
    };
    float wa[U][V], wb[U][V];            // the norm's weights
#pragma unroll
    for (int i = 0; i < U; ++i)
#pragma unroll
        for (int e = 0; e < V; ++e) {
            const bool has = mine && p.weight && lane + i * a.per < units;
            wa[i][e] = has ? p.weight[ia[i] + e] : 1.0f;
            wb[i][e] = has ? p.weight[ib[i] + e] : 1.0f;
        }
    fetch((long long)blockIdx.x * a.tokens + tok);
    turn((int)blockIdx.x, 0, position((int)blockIdx.x));
    int ahead = position((int)(blockIdx.x + gridDim.x));
    int buffer = 0;
    for (int group = (int)blockIdx.x; group < a.groups; group += (int)gridDim.x, buffer ^= 1) {
        const long long t = (long long)group * a.tokens + tok;
        const bool real = mine && t < a.T;
#pragma unroll
        for (int i = 0; i < U; ++i)
#pragma unroll
            for (int e = 0; e < V; ++e) va[i][e] = na[i][e], vb[i][e] = nb[i][e];
        __syncthreads();                 // the group's turns are there; the other buffer's have been used
        const int next = group + (int)gridDim.x;
        if (next < a.groups) {
            fetch((long long)next * a.tokens + tok);
            turn(next, buffer ^ 1, ahead);
            ahead = position(next + (int)gridDim.x);
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
#pragma unroll
        for (int i = 0; i < U; ++i) {
            const int u = lane + i * a.per;
            if (u >= units) continue;
            if (a.norm) {
#pragma unroll
                for (int e = 0; e < V; ++e) {
                    va[i][e] = va[i][e] * scale * wa[i][e];
                    vb[i][e] = vb[i][e] * scale * wb[i][e];
                }
            }
            if (u < half / V) {
                float2 cs[V];
                take<V>(turned + buffer * size + place<V>(tok * half + u * V), cs);
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
            if (!MPQ_CHECK(t < a.T && ia[i] + V <= a.dim && ib[i] + V <= a.dim)) continue;
            store_v<VEC>(y + p.ldy_token * t + ia[i], va[i]);
            store_v<VEC>(y + p.ldy_token * t + ib[i], vb[i]);
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
    // rows of up to 512 threads; a token of fewer than 256 shares its CTA
    a.rows = std::min(heads, 512 / a.per);
    a.tokens = (int)std::max(1LL, std::min<long long>(256 / (a.rows * a.per), T));
    a.groups = (int)((T + (long long)a.tokens - 1) / a.tokens);
    const int threads = (a.tokens * a.rows * a.per + 31) / 32 * 32, ys = (heads + a.rows - 1) / a.rows;
    const int resident = std::max(1, 1536 / threads) * sm_count();
    const dim3 grid((unsigned)std::min(a.groups, std::max(1, resident / ys)), (unsigned)ys);
    const size_t smem = 2 * (size_t)(wide ? place<8>(a.tokens * (rot / 2)) : a.tokens * (rot / 2)) * sizeof(float2);
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
