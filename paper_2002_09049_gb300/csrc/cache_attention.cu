// Attention of one new token of every sequence over the few-bit key-value cache
// (mpq_cache_attention):
//   s_t = scale q . (sk_t kq_t),  o = sum_t 2^(s_t - M) sv_t vq_t / sum_t 2^(s_t - M)
// with s in the log2 domain, for the query heads of each key head.
//
// Bound by memory: a cached token's row costs dim * bits / 8 + 4 bytes and 4 dim operations for each
// query head that shares it.  So the codes go from memory to the registers that feed the MMAs with
// one stop: a lane copies (cp.async) exactly the chunks that its own fragments need into a ring of
// its warp's shared memory and reads them back itself, which takes no barrier and no bank conflict,
// and several 16-token stages are always in flight.  Codes become fp16 by setting them into the
// mantissa of 1024 (an exact conversion in one permute and one subtraction for two).
//
// Tokens and elements are the long sides of the warp MMAs (m16n8k16, fp16 in, fp32 sums), query heads
// the short one (8 or 16 of them, zero past the group), so that codes are converted once for all
// heads that share them:  S^T [16 tokens][8 heads] = K Q^T, then O^T [16 elements][8 heads] += V^T P^T.
// Which element an index of a contraction stands for is free, so a lane's k indices are the
// consecutive codes of its chunk, and an accumulator's rows are those of its V chunk.  P^T comes from
// S^T's layout by an 8 x 8 transpose.
//
// The weights P = 2^(s_t) sv_t carry the value scales, rounded to fp16 against a reference r within
// 2^14 of the largest so far (r moves when a weight passes it by 2^14: one vote a stage, and a
// rescale that long rows take a handful of times), so a token's precision does not hang on how large
// its values are.  The sum of the softmax keeps an fp32 maximum and sum per lane.
//
// The work is the list of (sequence, key head, 64 tokens) tiles, cut into equal ranges for the
// resident CTAs whatever the lengths are; the four warps of a CTA take every fourth stage of 16 tokens.
// A (sequence, head) whose tiles are in one range is finished there.  Else each range leaves its
// sums in the workspace, and the CTA that comes last joins them in the order of the ranges (so the
// result does not depend on which one it is).
#include <float.h>
#include <math.h>

#include <algorithm>

#include "elements.cuh"
#include "mpq_internal.cuh"
#include "pair_common.cuh"
#include "sm100.cuh"

MPQ_CHECKED_UNIT("cache_attention.cu");

namespace mpq {
namespace {

using namespace sm100;

constexpr int A_WARPS = 4;
constexpr int A_THREADS = A_WARPS * 32;
constexpr int A_STAGE = 16;                       // tokens of a warp's stage
constexpr int A_TILE = A_WARPS * A_STAGE;         // tokens of a tile
constexpr int A_MAX_CTAS = 2048;                  // counters at the head of the workspace
constexpr size_t A_COUNTERS = A_MAX_CTAS * sizeof(unsigned);
constexpr float A_SHIFT = 6.0f, A_MARGIN = 14.0f; // r = largest / 2^6; moves past r 2^14
constexpr int A_JOIN = 64;                        // ranges joined at a time

struct AttnArgs {
    const void *Q;
    long long q_stride;
    int q_aligned;               // 8-byte aligned rows
    int B, q_heads, group, blocks;   // blocks of query heads of a key head
    mpq_kv_cache L;
    const unsigned char *codes;
    const float *scales;
    const int *table;
    int cols;
    const int *lens;
    float scale_log2;
    int window;
    void *O;
    float *lse;
    unsigned char *workspace;
};

// What a kernel of (dim, bits, tiles of 8 query heads) needs.
template <int D, int BITS, int NT>
struct Shape {
    static constexpr int H = NT * 8;
    static constexpr int RB = D * BITS / 8;                   // bytes of a row
    static constexpr int CK = RB / 4 < 16 ? RB / 4 : 16;      // a lane's key chunk: bytes, chunks
    static constexpr int NK = RB / 4 / CK;
    static constexpr int CV = RB / 8 < 16 ? RB / 8 : 16;      // a lane's value chunk
    static constexpr int NV = RB / 8 / CV;
    static constexpr int K_BYTES = A_STAGE * RB;
    static constexpr int STAGE_BYTES = 2 * K_BYTES + 2 * A_STAGE * 4;   // rows and scales
    static constexpr int STAGES = RB <= 32 ? 8 : RB <= 64 ? 6 : RB <= 128 ? 4 : 3;
    static constexpr int RING = A_WARPS * STAGES * STAGE_BYTES;
    static constexpr int OUT_LD = D + 4;                      // a head's row of the warps' sums
    static constexpr int JOIN_BYTES = A_WARPS * H * (OUT_LD + 3) * 4;
    static constexpr int SMEM = RING > JOIN_BYTES ? RING : JOIN_BYTES;
    static constexpr int SLOT = H * (D + 3);                  // floats a range leaves
    static constexpr int CTAS = D * NT <= 128 ? 4 : D * NT <= 256 ? 3 : 2;   // resident per SM
};

__device__ __forceinline__ float ex2(float x)
{
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}

__device__ __forceinline__ void mma_16816(float (&c)[4], const uint32_t (&a)[4], uint32_t b0,
                                          uint32_t b1)
{
    asm volatile(
        "mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, "
        "{%0,%1,%2,%3};"
        : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
        : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}

__device__ __forceinline__ uint32_t transpose_8x8(uint32_t v)
{
    uint32_t r;
    asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(r) : "r"(v));
    return r;
}

// A pair of 16-bit halves 0x6400 | u (1024 + u in fp16) less 1024 + bias: the codes as fp16, exactly.
template <int BITS>
__device__ __forceinline__ uint32_t unbias(uint32_t v)
{
    const __half2 b = __float2half2_rn(BITS == 8 ? 1152.0f : 1032.0f);
    const __half2 r = __hsub2(*reinterpret_cast<const __half2 *>(&v), b);
    return *reinterpret_cast<const uint32_t *>(&r);
}

// 8 bits: codes of bytes 0, 1 (HI: 2, 3) of w.  4 bits: of nibbles J and J + 4.
template <int HI>
__device__ __forceinline__ uint32_t codes8(uint32_t w)
{
    return unbias<8>(__byte_perm(w, 0x64646464u, HI ? 0x4342 : 0x4140));
}
template <int J>
__device__ __forceinline__ uint32_t codes4(uint32_t w)
{
    return unbias<4>(((w >> (4 * J)) & 0x000f000fu) | 0x64006400u);
}

template <int BYTES>
__device__ __forceinline__ void copy_chunk(uint32_t dst, const void *src)
{
    if constexpr (BYTES == 16) {
        cp_async16(dst, src, 16);
    } else if constexpr (BYTES == 8) {
        asm volatile("cp.async.ca.shared.global [%0], [%1], 8;"
                     :: "r"(dst), "l"(__cvta_generic_to_global(src)) : "memory");
    } else {
        cp_async4(dst, src, 4);
    }
}

template <int BYTES>
__device__ __forceinline__ void read_chunk(uint32_t src, uint32_t (&w)[BYTES / 4])
{
    if constexpr (BYTES == 16)
        asm volatile("ld.shared.v4.u32 {%0, %1, %2, %3}, [%4];"
                     : "=r"(w[0]), "=r"(w[1]), "=r"(w[2]), "=r"(w[3]) : "r"(src) : "memory");
    else if constexpr (BYTES == 8)
        asm volatile("ld.shared.v2.u32 {%0, %1}, [%2];"
                     : "=r"(w[0]), "=r"(w[1]) : "r"(src) : "memory");
    else
        w[0] = ld_shared_u32(src);
}

// Attended tokens [first, end) of a sequence and its tiles.
struct Span {
    int first, end;
    __device__ int tile0() const { return first / A_TILE; }
    __device__ int tiles() const { return end > first ? (end + A_TILE - 1) / A_TILE - tile0() : 0; }
};

__device__ __forceinline__ Span span_of(const AttnArgs &a, int b)
{
    const long long room = (long long)a.cols * a.L.page;
    long long n = a.lens[b];
    n = n < 0 ? 0 : n > room ? room : n;
    const long long f = a.window > 0 && n > a.window ? n - a.window : 0;
    return {(int)f, (int)n};
}

// Sums of one range of a (sequence, head block): per head the reference of the weighted values, the
// maximum and the sum of the softmax, and the weighted values.
struct Joined {
    float ref, top, sum;
};

__device__ __forceinline__ float natural_lse(float top, float sum)
{
    return sum == 0.0f ? -INFINITY : (top + log2f(sum)) * 0.693147180559945f;
}

// v 2^(ref - top) / sum, in two steps so that neither factor leaves fp32's range first.
__device__ __forceinline__ float finish(float v, const Joined &j)
{
    if (j.sum == 0.0f) return 0.0f;
    const float h = ex2(0.5f * (j.ref - j.top));
    return v * h * h / j.sum;
}

template <typename T, int D, int BITS, int NT>
__global__ void __launch_bounds__(A_THREADS, Shape<D, BITS, NT>::CTAS)
cache_attention_kernel(const AttnArgs a)
{
    using S = Shape<D, BITS, NT>;
    constexpr int H = S::H;
    extern __shared__ __align__(16) unsigned char smem[];
    __shared__ long long sh_pre[A_WARPS];
    __shared__ long long sh_first;           // tiles of the sequences before sh_b
    __shared__ int sh_b, sh_last;
    __shared__ Joined sh_join[H];
    __shared__ float sh_factor[H][A_JOIN];
    griddep_launch();
    griddep_wait();
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, g = lane >> 2, c = lane & 3;
    const int units = a.L.heads * a.blocks;
    T *const O = static_cast<T *>(a.O);
    const size_t o_size = (size_t)a.B * a.q_heads * D;
    if (!MPQ_CHECK_SMEM_END(S::SMEM)) return;

    // ---- sequences with nothing to attend to --------------------------------------------------
    for (int b = blockIdx.x; b < a.B; b += gridDim.x) {
        if (span_of(a, b).tiles() > 0) continue;
        for (int i = tid; i < a.q_heads * D; i += A_THREADS)
            if (MPQ_IN((size_t)b * a.q_heads * D + i, o_size))
                O[(size_t)b * a.q_heads * D + i] = from_f32<T>(0.0f);
        if (a.lse)
            for (int i = tid; i < a.q_heads; i += A_THREADS)
                a.lse[(size_t)b * a.q_heads + i] = -INFINITY;
    }

    // ---- this CTA's range of the tiles, and the sequence it begins in -------------------------
    const int per = (a.B + A_THREADS - 1) / A_THREADS;
    const int b_lo = min(tid * per, a.B), b_hi = min(b_lo + per, a.B);
    long long mine = 0;
    for (int b = b_lo; b < b_hi; ++b) mine += (long long)span_of(a, b).tiles() * units;
    long long pre = mine;                    // inclusive prefix over the CTA's threads
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const long long v = __shfl_up_sync(0xffffffffu, pre, o);
        if (lane >= o) pre += v;
    }
    if (lane == 31) sh_pre[warp] = pre;
    __syncthreads();
    long long total = 0;
#pragma unroll
    for (int w = 0; w < A_WARPS; ++w) {
        if (w < warp) pre += sh_pre[w];
        total += sh_pre[w];
    }
    const long long ctas = min((long long)gridDim.x, total);
    if (blockIdx.x >= ctas) return;
    const long long r0 = total * blockIdx.x / ctas, r1 = total * (blockIdx.x + 1LL) / ctas;
    pre -= mine;
    if (r0 >= pre && r0 < pre + mine) {
        int b = b_lo;
        for (;; ++b) {
            const long long n = (long long)span_of(a, b).tiles() * units;
            if (r0 < pre + n) break;
            pre += n;
        }
        sh_b = b;
        sh_first = pre;
    }
    __syncthreads();
    int b = sh_b;
    long long first = sh_first;
    Span sp = span_of(a, b);

    const uint32_t ring = smem_u32(smem) + (uint32_t)(warp * S::STAGES * S::STAGE_BYTES);
    float *const join = reinterpret_cast<float *>(smem);          // [warp][H][OUT_LD]
    float *const join_stat = join + A_WARPS * H * S::OUT_LD;      // [warp][H][3]
    unsigned *const counters = reinterpret_cast<unsigned *>(a.workspace);
    float *const slots = reinterpret_cast<float *>(a.workspace + A_COUNTERS);

    for (long long at = r0; at < r1;) {
        // ---- the segment: tiles [t_lo, t_hi) of unit u of sequence b ----------------------------
        int nt = sp.tiles();
        while (at - first >= (long long)nt * units) {
            first += (long long)nt * units;
            sp = span_of(a, ++b);
            nt = sp.tiles();
        }
        const int u = (int)((at - first) / nt);
        const int t_lo = (int)(at - first - (long long)u * nt);
        const int t_hi = (int)min((long long)nt, t_lo + (r1 - at));
        const int kvh = u / a.blocks, head0 = (u - kvh * a.blocks) * H;   // within the group
        const int heads = min(H, a.group - head0);
        const int tok_lo = (sp.tile0() + t_lo) * A_TILE;
        const int tok_hi = min(sp.end, (sp.tile0() + t_hi) * A_TILE);

        // ---- the warp's ring of stages: 16 tokens each, every fourth ---------------------------
        const int *row_of_table = a.table + (size_t)b * a.cols;
        int f_tok = tok_lo + warp * A_STAGE;                  // next stage to fetch
        int f_col = f_tok / a.L.page, f_off = f_tok - f_col * a.L.page;
        int f_page = f_tok < tok_hi ? row_of_table[f_col] : -1;
        unsigned held = 0;                                    // bit per stage: it names a page
        int f_slot = 0;
        auto fetch = [&]() {
            const bool ok = f_tok < tok_hi && f_page >= 0 && f_page < a.L.pages;
            if (ok) {
                const size_t row = ((size_t)f_page * 2 * a.L.heads + kvh) * a.L.page + f_off;
                const size_t v_row = row + (size_t)a.L.heads * a.L.page;
                const uint32_t st = ring + (uint32_t)(f_slot * S::STAGE_BYTES);
                const unsigned char *kp = a.codes + row * S::RB, *vp = a.codes + v_row * S::RB;
#pragma unroll
                for (int r = 0; r < 2; ++r)
#pragma unroll
                    for (int i = 0; i < S::NK; ++i)
                        copy_chunk<S::CK>(st + (uint32_t)(((r * S::NK + i) * 32 + lane) * S::CK),
                                          kp + (g + 8 * r) * S::RB + (i * 4 + c) * S::CK);
#pragma unroll
                for (int r = 0; r < 4; ++r)
#pragma unroll
                    for (int i = 0; i < S::NV; ++i)
                        copy_chunk<S::CV>(st + (uint32_t)(S::K_BYTES + ((r * S::NV + i) * 32 + lane) *
                                                                           S::CV),
                                          vp + (2 * c + (r & 1) + 8 * (r >> 1)) * S::RB +
                                              (i * 8 + g) * S::CV);
                cp_async4(st + (uint32_t)(2 * S::K_BYTES + lane * 4),
                          a.scales + (lane < 16 ? row : v_row) + (lane & 15), 4);
            }
            cp_async_commit();
            held = ok ? held | (1u << f_slot) : held & ~(1u << f_slot);
            f_slot = f_slot + 1 == S::STAGES ? 0 : f_slot + 1;
            f_tok += A_TILE;
            f_off += A_TILE;
            while (f_off >= a.L.page) {
                f_off -= a.L.page;
                ++f_col;
            }
            f_page = f_tok < tok_hi ? row_of_table[f_col] : -1;
        };
#pragma unroll 1
        for (int i = 0; i < S::STAGES - 1; ++i) fetch();

        // ---- the queries: fp16 times a power of two, in the keys' element order -----------------
        constexpr int KSTEPS = D / 16;
        uint32_t qf[NT][KSTEPS][2];
        float qs[NT][2];                 // scale log2(e) / that power, of heads 2c and 2c + 1
#pragma unroll
        for (int n = 0; n < NT; ++n) {
            const int head = n * 8 + g;
            const T *q = static_cast<const T *>(a.Q) + a.q_stride * b +
                         (size_t)(kvh * a.group + head0 + head) * D;
            constexpr int CE = S::CK * 8 / BITS;        // elements of a key chunk
            float v[D / 4];
            float m = 0.0f;
#pragma unroll
            for (int i = 0; i < D / 4; i += 4) {
                const T *p = q + (i / CE * 4 + c) * CE + i % CE;
                if (head >= heads) {
                    v[i] = v[i + 1] = v[i + 2] = v[i + 3] = 0.0f;
                } else if (a.q_aligned) {
                    const uint2 w = *reinterpret_cast<const uint2 *>(p);
                    const float2 x = unpack2(w.x, T()), y = unpack2(w.y, T());
                    v[i] = x.x, v[i + 1] = x.y, v[i + 2] = y.x, v[i + 3] = y.y;
                } else {
#pragma unroll
                    for (int k = 0; k < 4; ++k) v[i + k] = to_f32(p[k]);
                }
            }
#pragma unroll
            for (int i = 0; i < D / 4; ++i) m = fmaxf(m, fabsf(v[i]));
            m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, 1));
            m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, 2));
            const int e = f16_scale_exp(m);
            const float up = pow2f(e), down = a.scale_log2 * pow2f(-e);
#pragma unroll
            for (int k = 0; k < KSTEPS; ++k) {
                // 8 bits: bytes 0..3 of a word.  4 bits: nibbles 0, 4 | 1, 5, then 2, 6 | 3, 7.
                const int w = BITS == 8 ? 4 * k : 8 * (k / 2) + 2 * (k & 1);
                const int i0 = w, i1 = BITS == 8 ? w + 1 : w + 4;
                const int i2 = BITS == 8 ? w + 2 : w + 1, i3 = BITS == 8 ? w + 3 : w + 5;
                qf[n][k][0] = pack2(v[i0] * up, v[i1] * up, __half());
                qf[n][k][1] = pack2(v[i2] * up, v[i3] * up, __half());
            }
            qs[n][0] = __shfl_sync(0xffffffffu, down, 8 * c);
            qs[n][1] = __shfl_sync(0xffffffffu, down, 8 * c + 4);
        }

        float o[NT][D / 16][4], ref[NT][2], top[NT][2], sum[NT][2];
#pragma unroll
        for (int n = 0; n < NT; ++n) {
#pragma unroll
            for (int i = 0; i < D / 16; ++i) o[n][i][0] = o[n][i][1] = o[n][i][2] = o[n][i][3] = 0.0f;
#pragma unroll
            for (int k = 0; k < 2; ++k) {
                ref[n][k] = top[n][k] = -FLT_MAX;
                sum[n][k] = 0.0f;
            }
        }

        int slot = 0;
#pragma unroll 1
        for (int tok = tok_lo + warp * A_STAGE; tok < tok_hi; tok += A_TILE) {
            cp_async_wait<S::STAGES - 2>();
            __syncwarp();                // every lane's copies (the scales are read across lanes);
            fetch();                     // all are done with the stage before, which this fills
            const bool ok = (held >> slot) & 1u;
            const uint32_t st = ring + (uint32_t)(slot * S::STAGE_BYTES);
            if (ok) {                    // warp-uniform
                // ---- S^T = K Q^T -----------------------------------------------------------------
                float s[NT][4];
#pragma unroll
                for (int n = 0; n < NT; ++n) s[n][0] = s[n][1] = s[n][2] = s[n][3] = 0.0f;
#pragma unroll
                for (int i = 0; i < S::NK; ++i) {
                    uint32_t ka[S::CK / 4], kb[S::CK / 4];
                    read_chunk<S::CK>(st + (uint32_t)((i * 32 + lane) * S::CK), ka);
                    read_chunk<S::CK>(st + (uint32_t)(((S::NK + i) * 32 + lane) * S::CK), kb);
#pragma unroll
                    for (int w = 0; w < S::CK / 4; ++w) {
                        if constexpr (BITS == 8) {
                            const uint32_t f[4] = {codes8<0>(ka[w]), codes8<0>(kb[w]),
                                                   codes8<1>(ka[w]), codes8<1>(kb[w])};
#pragma unroll
                            for (int n = 0; n < NT; ++n) {
                                const int k = i * (S::CK / 4) + w;
                                mma_16816(s[n], f, qf[n][k][0], qf[n][k][1]);
                            }
                        } else {
                            const uint32_t f0[4] = {codes4<0>(ka[w]), codes4<0>(kb[w]),
                                                    codes4<1>(ka[w]), codes4<1>(kb[w])};
                            const uint32_t f1[4] = {codes4<2>(ka[w]), codes4<2>(kb[w]),
                                                    codes4<3>(ka[w]), codes4<3>(kb[w])};
#pragma unroll
                            for (int n = 0; n < NT; ++n) {
                                const int k = 2 * (i * (S::CK / 4) + w);
                                mma_16816(s[n], f0, qf[n][k][0], qf[n][k][1]);
                                mma_16816(s[n], f1, qf[n][k + 1][0], qf[n][k + 1][1]);
                            }
                        }
                    }
                }
                // ---- weights: rows g and g + 8 of the stage, heads 2c and 2c + 1 ----------------
                const uint32_t sc = st + (uint32_t)(2 * S::K_BYTES);
                float sk[2], lv[2];
                bool in[2];
#pragma unroll
                for (int r = 0; r < 2; ++r) {
                    const int t = tok + g + 8 * r;
                    in[r] = t >= sp.first && t < sp.end;
                    sk[r] = __uint_as_float(ld_shared_u32(sc + (uint32_t)((g + 8 * r) * 4)));
                    lv[r] = log2f(__uint_as_float(ld_shared_u32(sc + (uint32_t)((16 + g + 8 * r) * 4))));
                }
                bool move = false;
                float w[NT][4];
#pragma unroll
                for (int n = 0; n < NT; ++n)
#pragma unroll
                    for (int k = 0; k < 4; ++k) {
                        const int r = k >> 1, h = k & 1;
                        s[n][k] = in[r] ? s[n][k] * (sk[r] * qs[n][h]) : -INFINITY;
                        w[n][k] = in[r] ? s[n][k] + lv[r] : -INFINITY;
                        move |= s[n][k] > top[n][h] + A_MARGIN || w[n][k] > ref[n][h] + A_MARGIN;
                    }
                if (__any_sync(0xffffffffu, move)) {
#pragma unroll
                    for (int n = 0; n < NT; ++n)
#pragma unroll
                        for (int h = 0; h < 2; ++h) {
                            const float t1 = fmaxf(top[n][h], fmaxf(s[n][h], s[n][2 + h]));
                            sum[n][h] *= ex2(top[n][h] - t1);
                            top[n][h] = t1;
                            float m = fmaxf(w[n][h], w[n][2 + h]);
                            m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, 4));
                            m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, 8));
                            m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, 16));
                            const float r1_ = fmaxf(ref[n][h], m - A_SHIFT);
                            const float f = ex2(ref[n][h] - r1_);
                            ref[n][h] = r1_;
#pragma unroll
                            for (int i = 0; i < D / 16; ++i) {
                                o[n][i][h] *= f;
                                o[n][i][2 + h] *= f;
                            }
                        }
                }
                uint32_t pf[NT][2];
#pragma unroll
                for (int n = 0; n < NT; ++n) {
#pragma unroll
                    for (int h = 0; h < 2; ++h)
                        sum[n][h] += ex2(s[n][h] - top[n][h]) + ex2(s[n][2 + h] - top[n][h]);
#pragma unroll
                    for (int r = 0; r < 2; ++r)
                        pf[n][r] = transpose_8x8(pack2(ex2(w[n][2 * r] - ref[n][0]),
                                                       ex2(w[n][2 * r + 1] - ref[n][1]), __half()));
                }
                // ---- O^T += V^T P^T --------------------------------------------------------------
#pragma unroll
                for (int i = 0; i < S::NV; ++i) {
                    uint32_t v[4][S::CV / 4];
#pragma unroll
                    for (int r = 0; r < 4; ++r)
                        read_chunk<S::CV>(st + (uint32_t)(S::K_BYTES +
                                                          ((r * S::NV + i) * 32 + lane) * S::CV),
                                          v[r]);
#pragma unroll
                    for (int w4 = 0; w4 < S::CV / 4; ++w4) {
#pragma unroll
                        for (int hi = 0; hi < 2; ++hi) {
                            // tokens 2c, 2c + 1 and 2c + 8, 2c + 9 of half a word's elements
                            if constexpr (BITS == 8) {
                                const uint32_t x = __byte_perm(v[0][w4], v[1][w4], hi ? 0x7362 : 0x5140);
                                const uint32_t y = __byte_perm(v[2][w4], v[3][w4], hi ? 0x7362 : 0x5140);
                                const uint32_t f[4] = {codes8<0>(x), codes8<1>(x), codes8<0>(y),
                                                       codes8<1>(y)};
                                const int m = (i * (S::CV / 4) + w4) * 2 + hi;
#pragma unroll
                                for (int n = 0; n < NT; ++n)
                                    mma_16816(o[n][m], f, pf[n][0], pf[n][1]);
                            } else {
                                const uint32_t x = __byte_perm(v[0][w4], v[1][w4], hi ? 0x7632 : 0x5410);
                                const uint32_t y = __byte_perm(v[2][w4], v[3][w4], hi ? 0x7632 : 0x5410);
                                const uint32_t f0[4] = {codes4<0>(x), codes4<1>(x), codes4<0>(y),
                                                        codes4<1>(y)};
                                const uint32_t f1[4] = {codes4<2>(x), codes4<3>(x), codes4<2>(y),
                                                        codes4<3>(y)};
                                const int m = (i * (S::CV / 4) + w4) * 4 + hi * 2;
#pragma unroll
                                for (int n = 0; n < NT; ++n) {
                                    mma_16816(o[n][m], f0, pf[n][0], pf[n][1]);
                                    mma_16816(o[n][m + 1], f1, pf[n][0], pf[n][1]);
                                }
                            }
                        }
                    }
                }
            }
            slot = slot + 1 == S::STAGES ? 0 : slot + 1;
        }
        cp_async_wait_all();

        // ---- the four warps' sums ---------------------------------------------------------------
#pragma unroll
        for (int n = 0; n < NT; ++n)
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                float t = top[n][h];
#pragma unroll
                for (int x = 4; x < 32; x <<= 1) t = fmaxf(t, __shfl_xor_sync(0xffffffffu, t, x));
                float l = sum[n][h] * ex2(top[n][h] - t);
#pragma unroll
                for (int x = 4; x < 32; x <<= 1) l += __shfl_xor_sync(0xffffffffu, l, x);
                top[n][h] = t;
                sum[n][h] = l;
            }
        __syncthreads();                 // the rings are free
#pragma unroll
        for (int n = 0; n < NT; ++n)
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const int head = n * 8 + 2 * c + h;
                if (g == 0) {
                    float *stat = join_stat + (warp * H + head) * 3;
                    stat[0] = ref[n][h];
                    stat[1] = top[n][h];
                    stat[2] = sum[n][h];
                }
                constexpr int CE = S::CV * 8 / BITS;    // elements of a value chunk
#pragma unroll
                for (int m = 0; m < D / 16; ++m)
#pragma unroll
                    for (int r = 0; r < 2; ++r) {
                        const int d = (m / (CE / 2) * 8 + g) * CE + 2 * (m % (CE / 2)) + r;
                        join[(warp * H + head) * S::OUT_LD + d] = o[n][m][2 * r + h];
                    }
            }
        __syncthreads();
        const bool whole = t_lo == 0 && t_hi == nt;
        if (tid < H) {
            Joined j = {-FLT_MAX, -FLT_MAX, 0.0f};
#pragma unroll
            for (int w = 0; w < A_WARPS; ++w) {
                j.ref = fmaxf(j.ref, join_stat[(w * H + tid) * 3]);
                j.top = fmaxf(j.top, join_stat[(w * H + tid) * 3 + 1]);
            }
#pragma unroll
            for (int w = 0; w < A_WARPS; ++w)
                j.sum += join_stat[(w * H + tid) * 3 + 2] *
                         ex2(join_stat[(w * H + tid) * 3 + 1] - j.top);
            sh_join[tid] = j;
        }
        __syncthreads();
        const size_t out_row = (size_t)b * a.q_heads + kvh * a.group + head0;
        float *const part = slots + (size_t)(2 * blockIdx.x + (t_lo == 0 ? 1 : 0)) * S::SLOT;
        for (int i = tid; i < heads * D; i += A_THREADS) {
            const int head = i / D, d = i - head * D;
            const Joined j = sh_join[head];
            float v = 0.0f;
#pragma unroll
            for (int w = 0; w < A_WARPS; ++w)
                v += join[(w * H + head) * S::OUT_LD + d] *
                     ex2(join_stat[(w * H + head) * 3] - j.ref);
            if (whole && MPQ_IN(out_row * D + i, o_size))
                O[out_row * D + i] = from_f32<T>(finish(v, j));
            else if (!whole && MPQ_IN(part + 3 * H + i - slots, 2 * gridDim.x * S::SLOT))
                __stcg(part + 3 * H + i, v);
        }
        if (whole) {
            if (a.lse && tid < heads)
                a.lse[out_row + tid] = natural_lse(sh_join[tid].top, sh_join[tid].sum);
            __syncthreads();             // the rings are filled again
        } else {
            if (tid < heads) {
                __stcg(part + tid, sh_join[tid].ref);
                __stcg(part + H + tid, sh_join[tid].top);
                __stcg(part + 2 * H + tid, sh_join[tid].sum);
            }
            // ---- the unit's ranges: c0 .. c1; the CTA that comes last joins them ------------------
            const long long g0 = first + (long long)u * nt;
            const int c0 = (int)(((g0 + 1) * ctas - 1) / total);
            const int c1 = (int)(((g0 + nt) * ctas - 1) / total);
            __threadfence();
            __syncthreads();
            if (tid == 0) {
                const unsigned n = atomicAdd(&counters[c0], 1u);
                sh_last = n == (unsigned)(c1 - c0);
                if (sh_last) counters[c0] = 0;
            }
            __syncthreads();
            if (sh_last) {
                __threadfence();
                // range i of the unit: the first leaves its sums in its second slot, the others in
                // their first
                auto slot_of = [&](int i) {
                    return slots + (size_t)(2 * (c0 + i) + (i == 0 ? 1 : 0)) * S::SLOT;
                };
                const int n = c1 - c0 + 1;
                for (int h = warp; h < heads; h += A_WARPS) {
                    Joined j = {-FLT_MAX, -FLT_MAX, 0.0f};
                    for (int i = lane; i < n; i += 32) {
                        j.ref = fmaxf(j.ref, __ldcg(slot_of(i) + h));
                        j.top = fmaxf(j.top, __ldcg(slot_of(i) + H + h));
                    }
#pragma unroll
                    for (int x = 1; x < 32; x <<= 1) {
                        j.ref = fmaxf(j.ref, __shfl_xor_sync(0xffffffffu, j.ref, x));
                        j.top = fmaxf(j.top, __shfl_xor_sync(0xffffffffu, j.top, x));
                    }
                    for (int i = lane; i < n; i += 32)
                        j.sum += __ldcg(slot_of(i) + 2 * H + h) *
                                 ex2(__ldcg(slot_of(i) + H + h) - j.top);
#pragma unroll
                    for (int x = 1; x < 32; x <<= 1)
                        j.sum += __shfl_xor_sync(0xffffffffu, j.sum, x);
                    if (lane == 0) sh_join[h] = j;
                }
                constexpr int MINE = H * D / A_THREADS;
                float acc[MINE];
#pragma unroll
                for (int k = 0; k < MINE; ++k) acc[k] = 0.0f;
                for (int i0 = 0; i0 < n; i0 += A_JOIN) {
                    const int m = min(A_JOIN, n - i0);
                    __syncthreads();
                    for (int i = tid; i < heads * A_JOIN; i += A_THREADS) {
                        const int h = i / A_JOIN, k = i % A_JOIN;
                        if (k < m)
                            sh_factor[h][k] = ex2(__ldcg(slot_of(i0 + k) + h) - sh_join[h].ref);
                    }
                    __syncthreads();
                    for (int k = 0; k < m; ++k) {
                        const float *p = slot_of(i0 + k) + 3 * H;
#pragma unroll
                        for (int e = 0; e < MINE; ++e) {
                            const int i = e * A_THREADS + tid;
                            if (i < heads * D) acc[e] += __ldcg(p + i) * sh_factor[i / D][k];
                        }
                    }
                }
#pragma unroll
                for (int e = 0; e < MINE; ++e) {
                    const int i = e * A_THREADS + tid;
                    if (i < heads * D && MPQ_IN(out_row * D + i, o_size))
                        O[out_row * D + i] = from_f32<T>(finish(acc[e], sh_join[i / D]));
                }
                if (a.lse && tid < heads)
                    a.lse[out_row + tid] = natural_lse(sh_join[tid].top, sh_join[tid].sum);
            }
            __syncthreads();
        }
        at += t_hi - t_lo;
    }
}

template <typename T, int D, int BITS, int NT>
mpq_status launch_shape(const AttnArgs &a, cudaStream_t stream)
{
    using S = Shape<D, BITS, NT>;
    static std::atomic<int> limit[kMaxDevices];
    const cudaError_t e = allow_smem(
        reinterpret_cast<const void *>(cache_attention_kernel<T, D, BITS, NT>), limit, S::SMEM);
    if (e != cudaSuccess) return cuda_status(e, "cudaFuncSetAttribute");
    // every tile that the tables could hold, at most as many CTAs as are resident and as the
    // workspace has room for
    const long long room = (long long)a.cols * a.L.page;
    const long long span = a.window > 0 ? std::min<long long>(room, a.window) + A_TILE : room;
    const long long tiles = (span + A_TILE - 1) / A_TILE;
    const long long fit =
        (long long)((MPQ_CACHE_WORKSPACE - A_COUNTERS) / (2 * S::SLOT * sizeof(float)));
    long long ctas = std::min<long long>((long long)sm_count() * S::CTAS, std::min<long long>(fit, A_MAX_CTAS));
    const long long most = tiles * a.L.heads * a.blocks;     // of one sequence
    if (most < ctas) ctas = std::min(ctas, std::max<long long>(1, most * a.B));
    return launch_waiting(cache_attention_kernel<T, D, BITS, NT>, dim3((unsigned)ctas),
                          dim3(A_THREADS), S::SMEM, stream, "cache attention launch", a);
}

template <typename T, int D, int BITS>
mpq_status launch_heads(AttnArgs &a, cudaStream_t stream)
{
    // 16 query heads a block where a group has more than 8: the codes are read and converted once
    // for twice the heads
    const int H = a.group > 8 ? 16 : 8;
    a.blocks = (a.group + H - 1) / H;
    return H == 16 ? launch_shape<T, D, BITS, 2>(a, stream) : launch_shape<T, D, BITS, 1>(a, stream);
}

template <typename T, int D>
mpq_status launch_bits(AttnArgs &a, cudaStream_t stream)
{
    return a.L.bits == 8 ? launch_heads<T, D, 8>(a, stream) : launch_heads<T, D, 4>(a, stream);
}

template <typename T>
mpq_status launch_dim(AttnArgs &a, cudaStream_t stream)
{
    if (a.L.dim == 64) return launch_bits<T, 64>(a, stream);
    if (a.L.dim == 128) return launch_bits<T, 128>(a, stream);
    return launch_bits<T, 256>(a, stream);
}

}  // namespace

mpq_status launch_cache_attention(const void *Q, int type, long long q_stride, int B, int q_heads,
                                  const mpq_kv_cache *L, const void *codes, const float *scales,
                                  const int *table, int cols, const int *lens, float scale,
                                  int window, void *O, float *lse, void *workspace,
                                  cudaStream_t stream)
{
    AttnArgs a = {};
    a.Q = Q;
    a.q_stride = q_stride;
    a.q_aligned = ((uintptr_t)Q & 7) == 0 && q_stride % 4 == 0;
    a.B = B;
    a.q_heads = q_heads;
    a.group = q_heads / L->heads;
    a.L = *L;
    a.codes = static_cast<const unsigned char *>(codes);
    a.scales = scales;
    a.table = table;
    a.cols = cols;
    a.lens = lens;
    a.scale_log2 = (float)((double)scale * 1.4426950408889634);
    a.window = window;
    a.O = O;
    a.lse = lse;
    a.workspace = static_cast<unsigned char *>(workspace);
    void *scratch = nullptr;
    if (!workspace) {
        mpq_status st = pool_scratch(&scratch, MPQ_CACHE_WORKSPACE, stream);
        if (st != MPQ_OK) return st;
        a.workspace = static_cast<unsigned char *>(scratch);
        st = cuda_status(cudaMemsetAsync(scratch, 0, A_COUNTERS, stream), "cudaMemsetAsync");
        if (st != MPQ_OK) {
            cudaFreeAsync(scratch, stream);
            return st;
        }
    }
    mpq_status st = type == MPQ_F16 ? launch_dim<__half>(a, stream)
                                    : launch_dim<__nv_bfloat16>(a, stream);
    if (scratch) {
        const mpq_status fr = cuda_status(cudaFreeAsync(scratch, stream), "cudaFreeAsync");
        if (st == MPQ_OK) st = fr;
    }
    return st;
}

}  // namespace mpq
