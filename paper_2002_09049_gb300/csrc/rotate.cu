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
//
// 8,192 tokens of 40 heads of 128 bf16 take 34.7 us (168 MB, 4.8 TB/s; without a norm 30.6, neighbours' pairs 44): a
// barrier a token, at which warps wait for the slowest (issue slots are 0.52 busy, with 290 warp instructions a token and
// four rows).  The 16-bit forms' 64 registers, for two CTAs of 512 threads, leave 12 to 16 bytes spilled.  A CTA a token, without
// loads ahead, took 62; one element after another instead of two at once, and cosines that eight threads read from
// the same banks, 49.
#include <math.h>

#include <algorithm>
#include <type_traits>

#include "elements.cuh"
#include "mpq_internal.cuh"
#include "sm100.cuh"

MPQ_CHECKED_UNIT("rotate.cu");

namespace mpq {
namespace {


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

// Where pair i's cosine lies, in floats, and how far its sine: eight cosines, eight sines and their negatives, such eights
// 112 bytes apart, so that eight threads that read theirs, 16 bytes at a time, meet no bank twice.
template <int V>
__host__ __device__ constexpr int place(int i) { return V == 8 ? (i >> 3) * 28 + (i & 7) : 2 * i; }
template <int V>
constexpr int kSine = V == 8 ? 8 : 1;

// (l, r) -> (l c - r s, r c + l s)
__device__ __forceinline__ void turn_pair(float &l, float &r, float c, float s)
{
    const float a = __fmaf_rn(r, -s, __fmul_rn(l, c));
    r = __fmaf_rn(l, s, __fmul_rn(r, c));
    l = a;
}

constexpr int ROT_DEPTH = 4;             // tokens of a thread's elements that are on their way or being turned (VEC)

template <typename T, int V, int U, bool NEIGHBOURS, bool VEC>
__global__ void __launch_bounds__(512, VEC && sizeof(T) == 2 ? 2 : 1)
rotate_kernel(const RotateArgs a)
{
    static_assert(!VEC || (V == 8 && U == 1), "the wide form");
    constexpr int CHUNKS = VEC ? 2 * V * (int)sizeof(T) / 16 : 1;        // of a thread and token, 16 bytes each
    extern __shared__ __align__(16) float turned[];      // cosines and sines [2][tokens][rot / 2], by place
    const int half = a.rot / 2, units = a.dim / (2 * V), entries = a.tokens * half, size = place<V>(entries);
    uint4 *const staged = reinterpret_cast<uint4 *>(turned + 2 * size);  // VEC: [ROT_DEPTH][CHUNKS][threads]
    sm100::griddep_launch();
    sm100::griddep_wait();
    const int lane = (int)threadIdx.x & (a.per - 1), slot = (int)threadIdx.x / a.per;
    const int tok = slot / a.rows, row = (int)blockIdx.y * a.rows + slot - tok * a.rows;
    const int heads = a.part[0].heads + a.part[1].heads;
    const bool mine = tok < a.tokens && row < heads, key = row >= a.part[0].heads;
    const mpq_rotate_rows &p = a.part[key ? 1 : 0];
    const int head = key ? row - a.part[0].heads : row;
    const int stride = (int)gridDim.x;
    // the token that is fetched next and the one that is turned, by addresses: both go on by a group of every CTA
    int t = (int)blockIdx.x * a.tokens + tok, t_next = t;
    const int t_step = stride * a.tokens;
    const T *x = static_cast<const T *>(p.x) + p.ld_head * head + p.ld_token * t;
    T *y = static_cast<T *>(p.y) + p.ldy_head * head + p.ldy_token * t;
    const long long x_step = p.ld_token * t_step, y_step = p.ldy_token * t_step;
    const float *const weight = p.weight;
    int ia[U], ib[U];
#pragma unroll
    for (int i = 0; i < U; ++i) unit_at<V>(lane + i * a.per, a.rot, NEIGHBOURS, ia[i], ib[i]);
    float va[U][V], vb[U][V];            // the group's elements
    // a token's elements on their way to shared memory (nothing where there is no such token)
    auto fetch = [&](int slot_at) {
        if constexpr (VEC) {
            const uint32_t bytes = mine && lane < units && t_next < a.T ? 16u : 0u;
#pragma unroll
            for (int c = 0; c < CHUNKS; ++c) {
                const int at = (c < CHUNKS / 2 ? ia[0] : ib[0]) + c % (CHUNKS / 2) * (16 / (int)sizeof(T));
                sm100::cp_async16(sm100::smem_u32(staged + (slot_at * CHUNKS + c) * (int)blockDim.x + (int)threadIdx.x),
                                  x + at, bytes);
            }
            sm100::cp_async_commit();
            x += x_step;
            t_next += t_step;
        }
    };
    auto take = [&](int slot_at) {
        if constexpr (VEC) {
            sm100::cp_async_wait<ROT_DEPTH - 2>();
            const uint4 *const q = staged + slot_at * CHUNKS * (int)blockDim.x + (int)threadIdx.x;
            if constexpr (sizeof(T) == 2) {
                load8(reinterpret_cast<const T *>(q), va[0]);
                load8(reinterpret_cast<const T *>(q + blockDim.x), vb[0]);
            } else {
#pragma unroll
                for (int c = 0; c < CHUNKS; ++c) {
                    const float4 f = *reinterpret_cast<const float4 *>(q + c * (int)blockDim.x);
                    float *const v = c < 2 ? va[0] + 4 * c : vb[0] + 4 * (c - 2);
                    v[0] = f.x, v[1] = f.y, v[2] = f.z, v[3] = f.w;
                }
            }
        } else {
#pragma unroll
            for (int i = 0; i < U; ++i) {
#pragma unroll
                for (int e = 0; e < V; ++e) va[i][e] = vb[i][e] = 0.0f;
                if (!mine || t >= a.T || lane + i * a.per >= units) continue;
#pragma unroll
                for (int e = 0; e < V; ++e) {
                    va[i][e] = to_f32(x[ia[i] + e]);
                    vb[i][e] = to_f32(x[ib[i] + e]);
                }
            }
            x += x_step;
        }
    };
    // a thread makes the same frequency's turns of every group (and others', where there are more than threads)
    const int own = (int)threadIdx.x, own_tok = half ? own / half : 0;
    const uint64_t own_turn = own < entries ? a.turns[own - own_tok * half] : 0;
    auto position = [&](int group) {
        const long long t = (long long)group * a.tokens + own_tok;
        return own < entries && t < a.T ? a.positions[t] : 0;
    };
    auto keep = [&](int buffer, int i, uint64_t turn) {
        const float2 c = cos_sin(turn);
        float *const to = turned + buffer * size + place<V>(i);
        to[0] = c.x;
        to[kSine<V>] = c.y;
        if (V == 8) to[16] = -c.y;
    };
    auto turn = [&](int group, int buffer, int at) {
        if (own < entries) keep(buffer, own, (uint64_t)((long long)at + a.shift) * own_turn);
        for (int i = own + (int)blockDim.x; i < entries; i += (int)blockDim.x) {
            const int k = i / half;
            const long long t = (long long)group * a.tokens + k;
            if (t < a.T) keep(buffer, i, (uint64_t)((long long)a.positions[t] + a.shift) * a.turns[i - k * half]);
        }
    };
    float wa[U][V], wb[U][V];            // the norm's weights
#pragma unroll
    for (int i = 0; i < U; ++i)
#pragma unroll
        for (int e = 0; e < V; ++e) {
            const bool has = mine && weight && lane + i * a.per < units;
            wa[i][e] = has ? weight[ia[i] + e] : 1.0f;
            wb[i][e] = has ? weight[ib[i] + e] : 1.0f;
        }
#pragma unroll
    for (int i = 0; i < ROT_DEPTH - 1; ++i) fetch(i);
    turn((int)blockIdx.x, 0, position((int)blockIdx.x));
    int ahead = position((int)blockIdx.x + stride);
    int buffer = 0, at = 0;
    for (int group = (int)blockIdx.x; group < a.groups;
         group += stride, buffer ^= 1, at = (at + 1) % ROT_DEPTH, t += t_step, y += y_step) {
        take(at);
        fetch((at + ROT_DEPTH - 1) % ROT_DEPTH);
        __syncthreads();                 // the group's turns are there; the other buffer's have been used
        if (group + stride < a.groups) {
            turn(group + stride, buffer ^ 1, ahead);
            ahead = position(group + 2 * stride);
        }
        float scale = 1.0f;
        if (a.norm) {
            auto squares = [&](auto small) {
                const float by = decltype(small)::value ? 0x1p-80f : 1.0f;
                float2 s = make_float2(0.0f, 0.0f);
#pragma unroll
                for (int i = 0; i < U; ++i) {
                    if constexpr (V == 8) {
#pragma unroll
                        for (int e = 0; e < V; e += 2) {
                            float2 fa = make_float2(va[i][e], va[i][e + 1]), fb = make_float2(vb[i][e], vb[i][e + 1]);
                            if (decltype(small)::value) {
                                fa = mul2(fa, make_float2(by, by));
                                fb = mul2(fb, make_float2(by, by));
                            }
                            s = fma2(fa, fa, s);
                            s = fma2(fb, fb, s);
                        }
                    } else {
                        s.x = __fmaf_rn(va[i][0] * by, va[i][0] * by, s.x);
                        s.y = __fmaf_rn(vb[i][0] * by, vb[i][0] * by, s.y);
                    }
                }
                float sum = s.x + s.y;
                for (int o = 1; o < a.per; o <<= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
                return sum;
            };
            const float mean = fmaf(squares(std::false_type()), a.inv_dim, a.eps);
            scale = __frsqrt_rn(mean);
            // squares beyond fp32's range (elements above 2^60): again, of 2^-80 of them
            const bool big = isinf(mean);
            if (__any_sync(0xffffffffu, big)) {
                const float small = fmaf(squares(std::true_type()), a.inv_dim, a.eps * 0x1p-80f * 0x1p-80f);
                if (big) scale = __frsqrt_rn(small) * 0x1p-80f;
            }
        }
        if (!mine || t >= a.T) continue;
#pragma unroll
        for (int i = 0; i < U; ++i) {
            const int u = lane + i * a.per;
            if (u >= units) continue;
            if (a.norm) {
                if constexpr (V == 8) {
                    const float2 k = make_float2(scale, scale);
#pragma unroll
                    for (int e = 0; e < V; e += 2) {
                        const float2 l = mul2(mul2(make_float2(va[i][e], va[i][e + 1]), k), make_float2(wa[i][e], wa[i][e + 1]));
                        const float2 r = mul2(mul2(make_float2(vb[i][e], vb[i][e + 1]), k), make_float2(wb[i][e], wb[i][e + 1]));
                        va[i][e] = l.x, va[i][e + 1] = l.y;
                        vb[i][e] = r.x, vb[i][e + 1] = r.y;
                    }
                } else {
                    va[i][0] = __fmul_rn(__fmul_rn(va[i][0], scale), wa[i][0]);
                    vb[i][0] = __fmul_rn(__fmul_rn(vb[i][0], scale), wb[i][0]);
                }
            }
            if (u < half / V) {
                const float *const cs = turned + buffer * size + place<V>(tok * half + u * V);
                float c[V], sn[V], ns[V];         // (cosines, sines, their negatives)
                if constexpr (V == 8) {
#pragma unroll
                    for (int e = 0; e < 8; e += 4) {
                        const float4 f = *reinterpret_cast<const float4 *>(cs + e);
                        const float4 h = *reinterpret_cast<const float4 *>(cs + 8 + e);
                        c[e] = f.x, c[e + 1] = f.y, c[e + 2] = f.z, c[e + 3] = f.w;
                        sn[e] = h.x, sn[e + 1] = h.y, sn[e + 2] = h.z, sn[e + 3] = h.w;
                        const float4 n = *reinterpret_cast<const float4 *>(cs + 16 + e);
                        ns[e] = n.x, ns[e + 1] = n.y, ns[e + 2] = n.z, ns[e + 3] = n.w;
                    }
                } else {
                    c[0] = cs[0];
                    sn[0] = cs[1];
                }
                if constexpr (NEIGHBOURS && V > 1) {
                    // pairs (va[0], va[1]), .., (vb[0], vb[1]), ..
#pragma unroll
                    for (int e = 0; e < V; e += 2) {
                        turn_pair(va[i][e], va[i][e + 1], c[e / 2], sn[e / 2]);
                        turn_pair(vb[i][e], vb[i][e + 1], c[V / 2 + e / 2], sn[V / 2 + e / 2]);
                    }
                } else if constexpr (V > 1) {
#pragma unroll
                    for (int e = 0; e < V; e += 2) {     // turn_pair's roundings, two at once
                        const float2 l = make_float2(va[i][e], va[i][e + 1]), r = make_float2(vb[i][e], vb[i][e + 1]);
                        const float2 k = make_float2(c[e], c[e + 1]), h = make_float2(sn[e], sn[e + 1]);
                        const float2 m = fma2(r, make_float2(ns[e], ns[e + 1]), mul2(l, k)), n = fma2(l, h, mul2(r, k));
                        va[i][e] = m.x, va[i][e + 1] = m.y;
                        vb[i][e] = n.x, vb[i][e + 1] = n.y;
                    }
                } else {
                    turn_pair(va[i][0], vb[i][0], c[0], sn[0]);
                }
            }
            if (!MPQ_CHECK(t < a.T && ia[i] + V <= a.dim && ib[i] + V <= a.dim)) continue;
            if constexpr (VEC) {
                store8(y + ia[i], va[i]);
                store8(y + ib[i], vb[i]);
            } else {
#pragma unroll
                for (int e = 0; e < V; ++e) {
                    y[ia[i] + e] = from_f32<T>(va[i][e]);
                    y[ib[i] + e] = from_f32<T>(vb[i][e]);
                }
            }
        }
    }
    sm100::cp_async_wait_all();
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
    // CTAs that are resident at once: 64 registers a thread in the wide 16-bit form, 128 in the others
    const int regs = wide && vec && type != MPQ_F32 ? 64 : 128;
    const int resident = std::max(1, 65536 / (regs * threads)) * sm_count();
    const dim3 grid((unsigned)std::min(a.groups, std::max(1, resident / ys)), (unsigned)ys);
    const int entries = a.tokens * (rot / 2);
    size_t smem = 2 * (size_t)(wide ? place<8>(entries) : place<1>(entries)) * sizeof(float);
    if (wide && vec) smem += (size_t)ROT_DEPTH * threads * 16 * type_size(type);
    return by_type(type, [&](auto t) {
        using E = decltype(t);
        auto *const kernel =
            !wide ? (neighbours ? rotate_kernel<E, 1, 8, true, false> : rotate_kernel<E, 1, 8, false, false>)
            : vec ? (neighbours ? rotate_kernel<E, 8, 1, true, true> : rotate_kernel<E, 8, 1, false, true>)
                  : (neighbours ? rotate_kernel<E, 8, 1, true, false> : rotate_kernel<E, 8, 1, false, false>);
        static std::atomic<int> limit[6][kMaxDevices];
        const cudaError_t e = allow_smem(reinterpret_cast<const void *>(kernel),
                                         limit[(wide ? vec ? 2 : 1 : 0) * 2 + neighbours], smem);
        if (e != cudaSuccess) return cuda_status(e, "cudaFuncSetAttribute");
        return launch_waiting(kernel, grid, dim3((unsigned)threads), smem, stream, "rotate launch", a);
    });
}

}  // namespace mpq
