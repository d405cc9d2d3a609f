// Attention of one new token of every sequence over the few-bit key-value cache
// (mpq_cache_attention):
//   s_t = scale q . (sk_t kq_t),  o = sum_t 2^(s_t - M) sv_t vq_t / sum_t 2^(s_t - M)
// with s in the log2 domain, for the query heads of each key head.
//
// Bound by memory: a cached token's row costs dim * bits / 8 + 4 bytes and 4 dim operations for each
// query head that shares it.  A stage, 16 tokens of one page and head, is two tile copies (keys and
// values, contiguous in the cache) and a scale for each lane into a ring that each warp has for
// itself, so that several stages per warp are always in flight and no warp waits for another.  The
// copies swizzle the rows' 16-byte chunks, and the order of a stage's tokens in the MMAs is chosen so
// that both the keys' and the values' fragments are read without bank conflicts (row_of).  Codes become
// fp16 by setting them into the mantissa of 1024 (exact; one permute and one subtraction for two).
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
// The work is the list of every (sequence, key head)'s stages, cut into equal ranges for the resident
// warps whatever the lengths are.  A warp runs through its range on its own: its copies run ahead
// across the ends of rows, and a row that lies in one range is finished from registers.  Rows that
// several warps of a CTA share are joined in shared memory at the end; rows that several CTAs share
// leave their sums in the workspace, and the CTA that comes last joins them.  Sums are joined in the
// order of the ranges, so the result does not depend on who comes last.
//
// Measured, 8 key heads x 4 query heads of 128, 8 bits: 2 sequences of 131,072 tokens 93 us (554 MB, 6.0 TB/s;
// 4 bits: 92 us with half the bytes -- a stage is one chain of dependent steps, 565 warp instructions, and four
// warps a scheduler fill 0.58 of its issue slots); 96 sequences of 0 to 4,096, 32 us (a row's start and end cost
// four stages' time, ranges are ten stages long); one of 777 tokens 11.3 us, one of 64 6.6 (latency).  With 16
// query heads a key head 76 us instead of 54 (16 sequences of 8,192, 8 key heads of 128); with heads of 256 (4 key
// heads) 57, and 87 with 16 query heads.
#include <cuda.h>
#include <float.h>
#include <math.h>
#include <string.h>

#include <algorithm>

#include "elements.cuh"
#include "mpq_internal.cuh"
#include "pair_common.cuh"
#include "sm100.cuh"
#include "waits.cuh"

MPQ_CHECKED_UNIT("cache_attention.cu");

namespace mpq {
namespace {

using namespace sm100;

constexpr int A_STAGE = 16;                       // tokens of a stage
// Cuts of the work.  The geometric mean over 64 random batches (1 to 700 sequences of 8 to 60,000 tokens, all
// heads, widths and bits) is 16.2 us with these; A_ROW_COST 1, 2, 3, 5, 6, 8: 17.2, 16.4, 16.3, 16.1, 16.1, 16.2;
// A_WHOLE 6, 8, 14: 16.1, 16.2, 16.5; A_ROW 4, 9: 16.2; A_LEAST 1, 3: 16.1, 16.3 (two runs differ by 0.03).
constexpr int A_ROW_COST = 4;                     // what a row costs besides its stages, in stages
constexpr int A_LEAST = 2;                        // stages a warp is woken for
constexpr int A_ROW = 6;                          // most stages of a warp where each CTA takes one row
constexpr int A_WHOLE = 10;                       // most stages (and costs) of a row that a warp takes alone
constexpr int A_MAX_CTAS = 512;                   // counters at the head of the workspace
constexpr size_t A_COUNTERS = A_MAX_CTAS * sizeof(unsigned);
constexpr float A_SHIFT = 6.0f, A_MARGIN = 14.0f; // r = largest / 2^6; moves past r 2^14

struct AttnArgs {
    const void *Q;
    long long q_stride;
    int q_aligned;               // 8-byte aligned rows
    int page_shift;              // log2 of the page, -1 where it is no power of two
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
    static constexpr int K_BYTES = A_STAGE * RB;              // a stage's keys (and its values)
    static constexpr int BOX = RB < 128 ? RB : 128;           // bytes of a copied row: one swizzle span
    static constexpr int SCALE_BYTES = 2 * A_STAGE * 4;
    // warps of a CTA, one CTA per SM: 128, 168 or 255 registers a thread
    static constexpr int WARPS = D * NT <= 128 ? 16 : D * NT <= 256 ? 12 : 8;
    static constexpr int THREADS = WARPS * 32;
    static constexpr int ROOM = (222 * 1024 - 8192) / WARPS / (2 * K_BYTES + SCALE_BYTES + 8);
    static constexpr int STAGES = ROOM < 8 ? ROOM : 8;
    static_assert(STAGES >= 2, "a stage in use and one on its way");
    static constexpr int LD = D + 4;                          // (heads 2c apart: other banks)
    static constexpr int SUMS = H * (LD + 3);                 // floats of a row's sums: reference,
                                                              // maximum, sum by head, then values
    static constexpr int RING = STAGES * 2 * K_BYTES;
    static constexpr int WARP_BYTES = ((RING > SUMS * 4 ? RING : SUMS * 4) + 1023) / 1024 * 1024;
    static constexpr int OFF_SCALES = WARPS * WARP_BYTES;
    static constexpr int OFF_BARS = OFF_SCALES + WARPS * STAGES * SCALE_BYTES;
    static constexpr int SMEM = 1024 + OFF_BARS + WARPS * STAGES * 8;
};

// The token of a stage that row g (0..7) of an S^T tile stands for (row g + 8: that token + 8), and
// so, by twos, the tokens of the values' k indices.  With the copies' swizzles the 8 (or 16) lanes of
// one shared-memory access then read different banks: keys, g and g + 1 with all c; values, all c with
// neighbouring g.
__device__ __forceinline__ int row_of(int g) { return (g & 1) ? (g - 1) ^ 5 : g; }

// Byte of 16-byte chunk `ch` of row r of a stage's keys or values.
template <int RB>
__device__ __forceinline__ int chunk_at(int r, int ch)
{
    if (RB == 256) return (ch >> 3) * (A_STAGE * 128) + r * 128 + (((ch & 7) ^ (r & 7)) << 4);
    if (RB == 128) return r * 128 + ((ch ^ (r & 7)) << 4);
    if (RB == 64) return r * 64 + ((ch ^ ((r >> 1) & 3)) << 4);
    return r * 32 + ((ch ^ ((r >> 2) & 1)) << 4);
}

__device__ __forceinline__ float ex2(float x)
{
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}

__device__ __forceinline__ float lg2(float x)
{
    float y;
    asm("lg2.approx.f32 %0, %1;" : "=f"(y) : "f"(x));
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

// Codes as fp16, exactly: set into the mantissa of 1024, less 1024 and their offset.
// 8 bits: codes of bytes 0, 1 (HI: 2, 3) of w.
template <int HI>
__device__ __forceinline__ uint32_t codes8(uint32_t w)
{
    const uint32_t v = __byte_perm(w, 0x64646464u, HI ? 0x4342 : 0x4140);
    const __half2 r = __hsub2(*reinterpret_cast<const __half2 *>(&v), __float2half2_rn(1152.0f));
    return *reinterpret_cast<const uint32_t *>(&r);
}

// 4 bits: of nibbles J and J + 4 (an odd J sets 16 times the code: 1024 + 16 u, one fma from u - 8).
template <int J>
__device__ __forceinline__ uint32_t codes4(uint32_t w)
{
    const uint32_t x = J >= 2 ? w >> 8 : w;
    const uint32_t v = (x & (J & 1 ? 0x00f000f0u : 0x000f000fu)) | 0x64006400u;
    const __half2 h = *reinterpret_cast<const __half2 *>(&v);
    const __half2 r = J & 1 ? __hfma2(h, __float2half2_rn(0.0625f), __float2half2_rn(-72.0f))
                            : __hsub2(h, __float2half2_rn(1032.0f));
    return *reinterpret_cast<const uint32_t *>(&r);
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

// Attended tokens [first, end) of a sequence and its stages.
struct Span {
    int first, end;
    __device__ int stage0() const { return first / A_STAGE; }
    __device__ int stages() const
    {
        return end > first ? (end + A_STAGE - 1) / A_STAGE - stage0() : 0;
    }
};

__device__ __forceinline__ Span span_of(const AttnArgs &a, int b)
{
    const int room = a.cols * a.L.page;
    const int n = min(max(a.lens[b], 0), room);
    return {a.window > 0 ? max(n - a.window, 0) : 0, n};
}

// What one unit of a sequence of n stages counts in the work: its stages, and its own cost.
__device__ __forceinline__ int weight(int n) { return n > 0 ? n + A_ROW_COST : 0; }

// A row's place in the work: sequence, unit (key head and block of query heads), stages.
struct Row {
    int b, u, n;          // n: stages of each of the sequence's units
    Span sp;
    __device__ void next(const AttnArgs &a, int units)
    {
        if (++u < units) return;
        u = 0;
        do {
            sp = span_of(a, ++b);
            n = sp.stages();
        } while (n == 0);
    }
};

// Per head: the reference of the weighted values, the maximum and the sum of the softmax.
struct Stat {
    float ref, top, sum;
};

__device__ __forceinline__ float natural_lse(const Stat &s)
{
    return s.sum == 0.0f ? -INFINITY : (s.top + log2f(s.sum)) * 0.693147180559945f;
}

// 2^(ref - top) / sum, which makes weighted values outputs, as two factors (so that none leaves fp32's
// range before the product does); 0 where there was nothing to attend to.
__device__ __forceinline__ float2 to_output(const Stat &s)
{
    if (s.sum == 0.0f) return make_float2(0.0f, 0.0f);
    const float h = ex2(0.5f * (s.ref - s.top));
    return make_float2(h, h / s.sum);
}

// What a warp leaves for the others: up to two rows that it has a part of, the one its range begins
// in (kept in the workspace) and the one it ends in (in its shared memory).
struct Part {
    int b, u;             // b < 0: none
    int starts, ends;     // it holds the row's first stage, its last
};

// A load for L1's sake (of the 2 bytes at p; the value goes nowhere).
__device__ __forceinline__ void touch(const void *p)
{
    asm volatile("{\n\t.reg .u16 v;\n\tld.global.ca.u16 v, [%0];\n\t}" :: "l"(__cvta_generic_to_global(p))
                 : "memory");
}

// The sum of two parts' statistics.
__device__ __forceinline__ Stat add(const Stat &a, const Stat &b)
{
    const float t = fmaxf(a.top, b.top);
    return {fmaxf(a.ref, b.ref), t, a.sum * ex2(a.top - t) + b.sum * ex2(b.top - t)};
}

// The sum of the lanes' statistics, in every lane (the same bits: each step adds the same two).
__device__ __forceinline__ Stat add_lanes(Stat s)
{
#pragma unroll
    for (int x = 1; x < 32; x <<= 1)
        s = add(s, {__shfl_xor_sync(0xffffffffu, s.ref, x), __shfl_xor_sync(0xffffffffu, s.top, x),
                    __shfl_xor_sync(0xffffffffu, s.sum, x)});
    return s;
}

// a / b for a >= 0, b > 0: a 32-bit division where they allow it.
__device__ __forceinline__ long long quotient(long long a, long long b)
{
    return ((a | b) >> 32) == 0 ? (long long)((unsigned)a / (unsigned)b) : a / b;
}

// The cut of `total` stages into ranges for `n` workers (n <= total).  Where total / n workers hold a
// whole number of equal rows, so do their ranges.
struct Cut {
    long long total, n;
    __device__ long long begin(int w) const { return quotient(total * w, n); }
    __device__ int worker(long long stage) const { return (int)quotient((stage + 1) * n - 1, total); }
};

template <typename T, int D, int BITS, int NT>
__global__ void __launch_bounds__((Shape<D, BITS, NT>::THREADS), 1)
cache_attention_kernel(const AttnArgs a, WaitCtl wc, const __grid_constant__ CUtensorMap tm)
{
    using S = Shape<D, BITS, NT>;
    constexpr int H = S::H, W = S::WARPS, THREADS = S::THREADS;
    constexpr int E = D / 32;                    // values of a head that a lane joins
    extern __shared__ unsigned char raw[];
    __shared__ long long sh_pre[THREADS];        // stages before each thread's sequences
    __shared__ long long sh_warp[W];
    __shared__ int sh_some[W];
    __shared__ Part sh_part[2 * W];
    __shared__ int sh_open[2], sh_c0[2], sh_c1[2], sh_last[2];
    __shared__ __align__(16) float sh_slice[W][D];
    griddep_launch();
    const uint32_t raw_u32 = smem_u32(raw);
    unsigned char *const smem = raw + ((1024u - (raw_u32 & 1023u)) & 1023u);
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, g = lane >> 2, c = lane & 3;
    const int kr = row_of(g);
    unsigned char *const own = smem + warp * S::WARP_BYTES;
    const uint32_t ring = smem_u32(own);
    const uint32_t scales = smem_u32(smem) + (uint32_t)(S::OFF_SCALES + warp * S::STAGES * S::SCALE_BYTES);
    uint64_t *const bars = reinterpret_cast<uint64_t *>(smem + S::OFF_BARS) + warp * S::STAGES;
    if (!MPQ_CHECK_SMEM_END(smem - raw + S::OFF_BARS + W * S::STAGES * 8)) return;
    if (lane == 0) {
        for (int i = 0; i < S::STAGES; ++i) mbar_init(&bars[i], 1 + 32);   // the copies', the lanes' scales
        fence_barrier_init();
    }
    if (tid == 0) prefetch_tensormap(&tm);
    if (lane < 2) sh_part[2 * warp + lane].b = -1;
    const int units = a.L.heads * a.blocks;
    T *const O = static_cast<T *>(a.O);
    const size_t o_size = (size_t)a.B * a.q_heads * D;
    griddep_wait();

    // ---- the work: the stages before each sequence ------------------------------------------------
    // Up to 32 sequences: every warp looks at all of them, one a lane, and waits for no other.  More: each
    // thread at `per` of them.
    const bool few = a.B <= 32;
    const int per = few ? 1 : (a.B + THREADS - 1) / THREADS;
    Span lane_span = {0, 0};                     // (few) of sequence `lane`
    unsigned lane_pre = 0, lane_all = 0;         // (few) weight of a unit, before it and up to its end
    long long total;
    int some;                                    // sequences that have any
    if (few) {
        if (lane < a.B) lane_span = span_of(a, lane);
        const unsigned mine = (unsigned)weight(lane_span.stages());      // (32 of at most 2^26 + 4)
        lane_all = mine;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const unsigned v = __shfl_up_sync(0xffffffffu, lane_all, o);
            if (lane >= o) lane_all += v;
        }
        lane_pre = lane_all - mine;
        total = (long long)__shfl_sync(0xffffffffu, lane_all, 31) * units;
        some = __popc(__ballot_sync(0xffffffffu, mine > 0));
        if (warp == 0) sh_pre[lane] = (long long)lane_pre * units;       // (read after a barrier)
    } else {
        const int b_lo = min(tid * per, a.B), b_hi = min(b_lo + per, a.B);
        long long pre = 0;
        int live = 0;
        for (int b = b_lo; b < b_hi; ++b) {
            const int n = span_of(a, b).stages();
            pre += (long long)weight(n) * units;
            live += n > 0;
        }
        const long long mine = pre;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const long long v = __shfl_up_sync(0xffffffffu, pre, o);
            if (lane >= o) pre += v;
        }
        live = __reduce_add_sync(0xffffffffu, live);
        if (lane == 31) {
            sh_warp[warp] = pre;
            sh_some[warp] = live;
        }
        __syncthreads();
        total = 0;
        some = 0;
#pragma unroll
        for (int w = 0; w < W; ++w) {
            if (w < warp) pre += sh_warp[w];
            total += sh_warp[w];
            some += sh_some[w];
        }
        sh_pre[tid] = pre - mine;
        __syncthreads();
    }
    // sequences with nothing to attend to: a warp each
    auto empty_rows = [&]() {
        if (some == a.B) return;
        for (long long b = blockIdx.x + (long long)warp * gridDim.x; b < a.B;
             b += (long long)W * gridDim.x) {
            if (span_of(a, (int)b).stages() > 0) continue;
            const float zero[8] = {};
            for (int i = lane * 8; i < a.q_heads * D; i += 256)
                if (MPQ_IN(b * a.q_heads * D + i + 7, o_size)) store8(O + b * a.q_heads * D + i, zero);
            for (int i = lane; a.lse && i < a.q_heads; i += 32) a.lse[b * a.q_heads + i] = -INFINITY;
        }
    };
    // the warps that take part, and this one's range.  A CTA a row where there are no more rows than CTAs
    // and a warp then has A_ROW stages at most: joining CTAs takes longer than that (1 x 500 tokens 9.7 us,
    // 12.6 for the 1,024 that CTAs share).  A warp a row where there are more and they are short: nothing is
    // joined (96 x 64 tokens 11.3 us, 12.9 in ranges of two stages; 12 stages a row are too many: a case of 13 us
    // took 18).
    const long long rows = (long long)some * units;
    const bool by_row = rows <= gridDim.x && total <= rows * (W * A_ROW);
    const bool whole = rows > gridDim.x && rows <= (long long)gridDim.x * W && total <= rows * A_WHOLE;
    const int workers = by_row  ? (int)(rows * W)
                        : whole ? (int)rows
                                : (int)min((long long)gridDim.x * W, max(total / A_LEAST, 1LL));
    const int me = blockIdx.x * W + warp;
    if ((int)blockIdx.x * W >= workers || total == 0) {
        empty_rows();
        return;
    }
    const Cut cut = {total, workers};
    const long long r0 = me < workers ? cut.begin(me) : total;
    long long left = me < workers ? cut.begin(me + 1) - r0 : 0;

    unsigned *const counters = reinterpret_cast<unsigned *>(a.workspace);
    float *const cta_sums = reinterpret_cast<float *>(a.workspace + A_COUNTERS);      // [CTA][2]
    float *const warp_sums = cta_sums + (size_t)2 * gridDim.x * S::SUMS;             // [warp]
    bool dead = false;                           // a wait gave up: the outputs read NaN

    if (left > 0) {
        // ---- the sequence and unit that the range begins in ---------------------------------------
        Row at;
        int st;                                   // next stage of the row
        if (few) {
            at.b = __ffs((int)__ballot_sync(0xffffffffu, (long long)lane_all * units > r0)) - 1;
            at.sp.first = __shfl_sync(0xffffffffu, lane_span.first, at.b);
            at.sp.end = __shfl_sync(0xffffffffu, lane_span.end, at.b);
            at.n = at.sp.stages();
            const long long skip = r0 - (long long)__shfl_sync(0xffffffffu, lane_pre, at.b) * units;
            at.u = (int)quotient(skip, weight(at.n));
            st = (int)(skip - (long long)at.u * weight(at.n));
        } else {
            int lo = 0, hi = min(THREADS, a.B) - 1;   // the last thread whose sequences begin by r0
            while (lo < hi) {
                const int mid = (lo + hi + 1) / 2;
                if (sh_pre[mid] <= r0) lo = mid; else hi = mid - 1;
            }
            long long skip = r0 - sh_pre[lo];
            at.b = lo * per;
            for (;; ++at.b) {
                at.sp = span_of(a, at.b);
                at.n = at.sp.stages();
                const long long all = (long long)weight(at.n) * units;
                if (skip < all) break;
                skip -= all;
            }
            at.u = (int)quotient(skip, weight(at.n));
            st = (int)(skip - (long long)at.u * weight(at.n));
        }
        left -= max(0, A_ROW_COST - st);          // the row's own cost comes first
        st = max(0, st - A_ROW_COST);

        // ---- the ring: stages on their way, ahead of the row that is being worked on ---------------
        Row ahead = at;
        long long f_left = left;
        int f_st = st, f_i = 0, f_n = 0;          // next stage; place in the pages looked up, of f_n
        int f_blk = 0, f_off = 0;                 // this lane's, of stage f_st + lane: the keys' block
                                                  // (page x head) and place in the page
        unsigned f_ok = 0;                        // bit per lane: its stage names a page
        unsigned held = 0;                        // the same, bit per ring stage
        // A row's queries on their way to L1, before its stages are asked for (which they would wait
        // behind); nothing waits for them here.
        auto touch_queries = [&](const Row &r) {
            const int h0 = r.u % a.blocks * H, kv = r.u / a.blocks;
            const char *const q = reinterpret_cast<const char *>(
                static_cast<const T *>(a.Q) + a.q_stride * r.b + (size_t)(kv * a.group + h0) * D);
            const int bytes = min(H, a.group - h0) * D * (int)sizeof(T);
            for (int i = lane * 128; i < bytes; i += 32 * 128) touch(q + i);
        };
        auto fetch = [&](int to_slot) {
            if (f_left <= 0) return;
            if (f_i == f_n) {                     // look up the next 32 stages of the row
                if (f_st == ahead.n) {
                    f_left -= A_ROW_COST;
                    if (f_left <= 0) return;
                    ahead.next(a, units);
                    f_st = 0;
                    touch_queries(ahead);
                    if (lane == 0 && ahead.u == 0 && ahead.b + 1 < a.B)
                        touch(a.table + (size_t)(ahead.b + 1) * a.cols);
                }
                f_i = 0;
                f_n = min(32, ahead.n - f_st);
                const unsigned tok = (unsigned)(ahead.sp.stage0() + f_st + lane) * A_STAGE;
                const unsigned col = a.page_shift >= 0 ? tok >> a.page_shift : tok / (unsigned)a.L.page;
                const int page = lane < f_n ? a.table[(size_t)ahead.b * a.cols + col] : -1;
                const bool there = page >= 0 && page < a.L.pages;
                f_off = (int)(tok - col * (unsigned)a.L.page);
                f_blk = there ? page * 2 * a.L.heads + ahead.u / a.blocks : 0;
                f_ok = __ballot_sync(0xffffffffu, there);
            }
            const bool ok = (f_ok >> f_i) & 1u;
            if (ok && !wc.withhold) {             // (warp-uniform)
                const uint32_t to = ring + (uint32_t)(to_slot * 2 * S::K_BYTES);
                uint64_t *const bar = &bars[to_slot];
                const int blk = __shfl_sync(0xffffffffu, f_blk, f_i), off = __shfl_sync(0xffffffffu, f_off, f_i);
                if (lane == 0) {
                    mbar_arrive_expect_tx(bar, 2 * S::K_BYTES);
                    if (MPQ_CHECK((to & 255u) == 0u && off % A_STAGE == 0 && off < a.L.page)) {
#pragma unroll
                        for (int x = 0; x < S::RB; x += S::BOX) {
                            tma_load_3d(to + x * A_STAGE, &tm, x, off, blk, bar);
                            tma_load_3d(to + S::K_BYTES + x * A_STAGE, &tm, x, off, blk + a.L.heads, bar);
                        }
                    }
                }
                cp_async4(scales + (uint32_t)(to_slot * S::SCALE_BYTES + lane * 4),
                          a.scales + (long long)(blk + (lane < 16 ? 0 : a.L.heads)) * a.L.page + off +
                              (lane & 15),
                          4);
                cp_async_arrive(bar);
            }
            held = (held & ~(1u << to_slot)) | ((unsigned)ok << to_slot);
            ++f_i;
            ++f_st;
            --f_left;
        };
        touch_queries(at);
        __syncwarp();                             // the barriers are ready
#pragma unroll 1
        for (int i = 0; i < S::STAGES - 1; ++i) fetch(i);

        int slot = 0, fill = S::STAGES - 1;       // ring stages: the next to be used, to be filled
        unsigned parity = 0;                      // bit per ring stage: the phase of its next copies
#pragma unroll 1
        while (left > 0) {
            // ---- the queries of the row: fp16 times a power of two, in the keys' element order ------
            const int kvh = at.u / a.blocks, head0 = (at.u - kvh * a.blocks) * H;
            const int heads = min(H, a.group - head0);
            constexpr int KSTEPS = D / 16;
            uint32_t qf[NT][KSTEPS][2];
            float qs[NT][2];             // scale log2(e) / that power, of heads 2c and 2c + 1
#pragma unroll
            for (int n = 0; n < NT; ++n) {
                const int head = n * 8 + g;
                const T *q = static_cast<const T *>(a.Q) + a.q_stride * at.b +
                             (size_t)(kvh * a.group + head0 + head) * D;
                constexpr int CE = S::CK * 8 / BITS;    // elements of a key chunk
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

            float o[NT][D / 16][4];
            Stat sm[NT][2];
            float top_hi[NT][2], ref_hi[NT][2];  // the maximum and the reference move past these
#pragma unroll
            for (int n = 0; n < NT; ++n) {
#pragma unroll
                for (int i = 0; i < D / 16; ++i)
                    o[n][i][0] = o[n][i][1] = o[n][i][2] = o[n][i][3] = 0.0f;
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    sm[n][h] = {-FLT_MAX, -FLT_MAX, 0.0f};
                    top_hi[n][h] = ref_hi[n][h] = -FLT_MAX;
                }
            }
            const int st0 = st, st1 = (int)min((long long)at.n, st + left);
#pragma unroll 1
            for (; st < st1; ++st) {
                __syncwarp();            // all lanes are done with the stage before, which this fills
                fetch(fill);
                const int at_slot = fill = slot;
                slot = slot + 1 == S::STAGES ? 0 : slot + 1;
                if (!((held >> at_slot) & 1u)) continue;           // (warp-uniform)
                bool landed = !dead && mbar_wait(&bars[at_slot], (parity >> at_slot) & 1u, wc.budget);
                if (__any_sync(0xffffffffu, !landed)) {
                    // nothing more is asked for, and what is on its way lands before the warp goes on
                    if (!dead) note_timeout(wc, MPQ_TIMEOUT_ATTENTION);
                    dead = true;
                    f_left = 0;
                    held &= ~(1u << at_slot);
                    if (!wc.withhold)
                        drain_wait(&bars[at_slot], (parity >> at_slot) & 1u, wc, MPQ_TIMEOUT_ATTENTION);
                }
                parity ^= 1u << at_slot;
                if (dead) continue;
                const uint32_t from = ring + (uint32_t)(at_slot * 2 * S::K_BYTES);
                // ---- S^T = K Q^T -----------------------------------------------------------------
                float s[NT][4];
#pragma unroll
                for (int n = 0; n < NT; ++n) s[n][0] = s[n][1] = s[n][2] = s[n][3] = 0.0f;
#pragma unroll
                for (int i = 0; i < S::NK; ++i) {
                    uint32_t ka[S::CK / 4], kb[S::CK / 4];
                    const uint32_t k0 = from + (uint32_t)(chunk_at<S::RB>(kr, (i * 4 * S::CK + c * S::CK) / 16) +
                                                          c * S::CK % 16);
                    read_chunk<S::CK>(k0, ka);
                    read_chunk<S::CK>(k0 + 8 * S::BOX, kb);
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
                const uint32_t sc = scales + (uint32_t)(at_slot * S::SCALE_BYTES + kr * 4);
                    float sk[2], lv[2];
#pragma unroll
                    for (int r = 0; r < 2; ++r) {
                        sk[r] = __uint_as_float(ld_shared_u32(sc + 32 * r));
                        lv[r] = lg2(__uint_as_float(ld_shared_u32(sc + 64 + 32 * r)));
                    }
                    float w[NT][4];
#pragma unroll
                    for (int n = 0; n < NT; ++n)
#pragma unroll
                        for (int k = 0; k < 4; ++k) {
                            s[n][k] *= sk[k >> 1] * qs[n][k & 1];
                            w[n][k] = s[n][k] + lv[k >> 1];
                        }
                    const int t0 = (at.sp.stage0() + st) * A_STAGE;
                    if (t0 < at.sp.first || t0 + A_STAGE > at.sp.end) {    // tokens that are not attended to
#pragma unroll
                        for (int r = 0; r < 2; ++r) {
                            const int t = t0 + kr + 8 * r;
                            if (t >= at.sp.first && t < at.sp.end) continue;
#pragma unroll
                            for (int n = 0; n < NT; ++n)
                                s[n][2 * r] = s[n][2 * r + 1] = w[n][2 * r] = w[n][2 * r + 1] = -INFINITY;
                        }
                    }
                    bool move = false;
#pragma unroll
                    for (int n = 0; n < NT; ++n)
#pragma unroll
                        for (int h = 0; h < 2; ++h)
                            move |= fmaxf(s[n][h], s[n][2 + h]) > top_hi[n][h] ||
                                    fmaxf(w[n][h], w[n][2 + h]) > ref_hi[n][h];
                if (__any_sync(0xffffffffu, move)) {
#pragma unroll
                    for (int n = 0; n < NT; ++n)
#pragma unroll
                        for (int h = 0; h < 2; ++h) {
                            const float t1 = fmaxf(sm[n][h].top, fmaxf(s[n][h], s[n][2 + h]));
                            sm[n][h].sum *= ex2(sm[n][h].top - t1);
                            sm[n][h].top = t1;
                            float m = fmaxf(w[n][h], w[n][2 + h]);
                            m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, 4));
                            m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, 8));
                            m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, 16));
                            const float r1 = fmaxf(sm[n][h].ref, m - A_SHIFT);
                            const float f = ex2(sm[n][h].ref - r1);
                            sm[n][h].ref = r1;
                            top_hi[n][h] = t1 + A_MARGIN;
                            ref_hi[n][h] = r1 + A_MARGIN;
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
                        sm[n][h].sum += ex2(s[n][h] - sm[n][h].top) + ex2(s[n][2 + h] - sm[n][h].top);
#pragma unroll
                    for (int r = 0; r < 2; ++r)
                        pf[n][r] = transpose_8x8(pack2(ex2(w[n][2 * r] - sm[n][0].ref),
                                                       ex2(w[n][2 * r + 1] - sm[n][1].ref), __half()));
                }
                // ---- O^T += V^T P^T --------------------------------------------------------------
#pragma unroll
                for (int i = 0; i < S::NV; ++i) {
                    uint32_t v[4][S::CV / 4];
#pragma unroll
                    for (int r = 0; r < 2; ++r) {
                        const int tok = r ? 2 * c ^ 5 : 2 * c;           // row_of(2c), row_of(2c + 1)
                        const uint32_t v0 = from + (uint32_t)(S::K_BYTES + g * S::CV % 16 +
                                                              chunk_at<S::RB>(tok, (i * 8 * S::CV + g * S::CV) / 16));
                        read_chunk<S::CV>(v0, v[r]);
                        read_chunk<S::CV>(v0 + 8 * S::BOX, v[2 + r]);
                    }
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
            left -= st1 - st0;

            // ---- the end of the row, or of the range ------------------------------------------------
#pragma unroll
            for (int n = 0; n < NT; ++n)
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    float t = sm[n][h].top;
#pragma unroll
                    for (int x = 4; x < 32; x <<= 1) t = fmaxf(t, __shfl_xor_sync(0xffffffffu, t, x));
                    float l = sm[n][h].sum * ex2(sm[n][h].top - t);
#pragma unroll
                    for (int x = 4; x < 32; x <<= 1) l += __shfl_xor_sync(0xffffffffu, l, x);
                    sm[n][h].top = t;
                    sm[n][h].sum = dead ? NAN : l;
                }
            constexpr int CE = S::CV * 8 / BITS;        // elements of a value chunk, consecutive
            const bool starts = st0 == 0, ends = st1 == at.n;
            if (starts && ends) {
                const size_t row = (size_t)at.b * a.q_heads + kvh * a.group + head0;
#pragma unroll
                for (int n = 0; n < NT; ++n)
#pragma unroll
                    for (int h = 0; h < 2; ++h) {
                        const int head = n * 8 + 2 * c + h;
                        if (head >= heads) continue;
                        if (a.lse && g == 0) a.lse[row + head] = natural_lse(sm[n][h]);
                        const float2 f = to_output(sm[n][h]);
#pragma unroll
                        for (int i = 0; i < S::NV; ++i)
#pragma unroll
                            for (int k = 0; k < CE; k += 8) {
                                float v[8];
#pragma unroll
                                for (int e = 0; e < 8; ++e)
                                    v[e] = o[n][(i * CE + k + e) / 2][2 * (e & 1) + h] * f.x * f.y;
                                const size_t to = (row + head) * D + (i * 8 + g) * CE + k;
                                if (MPQ_IN(to + 7, o_size)) store8(O + to, v);
                            }
                    }
            } else {
                const bool last = left == 0 || (st1 == at.n && left <= A_ROW_COST);     // (then the ring is free)
                float *const to = last ? reinterpret_cast<float *>(own) : warp_sums + (size_t)me * S::SUMS;
                if (last) __syncwarp();
#pragma unroll
                for (int n = 0; n < NT; ++n)
#pragma unroll
                    for (int h = 0; h < 2; ++h) {
                        const int head = n * 8 + 2 * c + h;
                        if (g == 0) {
                            to[head] = sm[n][h].ref;
                            to[H + head] = sm[n][h].top;
                            to[2 * H + head] = sm[n][h].sum;
                        }
#pragma unroll
                        for (int i = 0; i < S::NV; ++i)
#pragma unroll
                            for (int k = 0; k < CE; k += 4) {
                                const int m = (i * CE + k) / 2;
                                *reinterpret_cast<float4 *>(to + 3 * H + head * S::LD + (i * 8 + g) * CE +
                                                            k) =
                                    make_float4(o[n][m][h], o[n][m][2 + h], o[n][m + 1][h],
                                                o[n][m + 1][2 + h]);
                            }
                    }
                if (lane == 0) sh_part[2 * warp + (last ? 1 : 0)] = {at.b, at.u, starts, ends};
            }
            if (st1 == at.n) left -= A_ROW_COST;
            if (left > 0) {
                at.next(a, units);
                st = 0;
            }
        }
    }
    empty_rows();
    __syncthreads();

    // ---- rows that several warps share: runs of parts of one row, in the order of the warps ------------
    // (every warp finds them for itself: lane p looks at part p)
    static_assert(2 * W <= 32, "one lane per part");
    const Part part = lane < 2 * W ? sh_part[lane] : Part{-1, 0, 0, 0};
    const unsigned live = __ballot_sync(0xffffffffu, part.b >= 0);
    if (live == 0) return;
    const int before = 31 - __clz((int)(live & ((1u << lane) - 1u)));       // the part before, or -1
    const int prev_b = __shfl_sync(0xffffffffu, part.b, before & 31);
    const int prev_u = __shfl_sync(0xffffffffu, part.u, before & 31);
    const unsigned firsts = __ballot_sync(
        0xffffffffu, part.b >= 0 && (before < 0 || prev_b != part.b || prev_u != part.u));
    const int first_part = __ffs((int)firsts) - 1, last_run = 31 - __clz((int)firsts);
    const int last_part = 31 - __clz((int)live);
    // the rows that other CTAs have parts of, the first run's (begun before) and the last one's, and
    // their CTAs: those of the workers of the row's first and last stage
    if (warp == W - 1 && lane < 2) {
        const Part p = sh_part[lane ? last_run : first_part];
        sh_open[lane] = lane ? p.starts && !sh_part[last_part].ends : !p.starts;
        if (sh_open[lane]) {
            long long g0 = sh_pre[p.b / per];
            for (int b = p.b / per * per; b < p.b; ++b)
                g0 += (long long)weight(span_of(a, b).stages()) * units;
            const int n = span_of(a, p.b).stages();
            g0 += (long long)p.u * weight(n) + A_ROW_COST;
            sh_c0[lane] = cut.worker(g0) / W;
            sh_c1[lane] = cut.worker(g0 + n - 1) / W;
        }
    }
    const float *const kept = warp_sums + (size_t)blockIdx.x * W * S::SUMS;
    // a warp takes a head of a run at a time, a lane the statistics of its part
    const float *const at = (lane & 1) ? reinterpret_cast<const float *>(smem + (lane >> 1) * S::WARP_BYTES)
                                       : kept + (size_t)(lane >> 1) * S::SUMS;
    int item = 0;
    for (unsigned rest = firsts; rest;) {
        const int p0 = __ffs((int)rest) - 1;
        rest &= rest - 1;
        const unsigned run = live & ~((1u << p0) - 1u) & (rest ? (rest & (0u - rest)) - 1u : ~0u);
        const Part lead = sh_part[p0];
        const bool starts = lead.starts, ends = sh_part[31 - __clz((int)run)].ends;
        const int head0 = lead.u % a.blocks * H, heads = min(H, a.group - head0);
        const int h0 = (warp + W - item % W) % W;        // this warp's first head of the run
        item += heads;
        for (int h = h0; h < heads; h += W) {
            Stat s = {-FLT_MAX, -FLT_MAX, 0.0f};
            if ((run >> lane) & 1u) s = {at[h], at[H + h], at[2 * H + h]};
            const float ref = s.ref;
            s = add_lanes(s);
            const float factor = ex2(ref - s.ref);
            float acc[E];
#pragma unroll
            for (int e = 0; e < E; ++e) acc[e] = 0.0f;
            unsigned left = run;
#pragma unroll 4
            for (int n = __popc(run); n > 0; --n) {
                const int i = __ffs((int)left) - 1;
                left &= left - 1;
                const float f = __shfl_sync(0xffffffffu, factor, i);
                const float *const q = reinterpret_cast<const float *>(
                    __shfl_sync(0xffffffffu, (unsigned long long)at, i)) + 3 * H + h * S::LD + lane;
#pragma unroll
                for (int e = 0; e < E; ++e) acc[e] += f * q[e * 32];
            }
            if (starts && ends) {
                const size_t row = (size_t)lead.b * a.q_heads + (lead.u / a.blocks) * a.group + head0 + h;
                const float2 f = to_output(s);
#pragma unroll
                for (int e = 0; e < E; ++e)
                    if (MPQ_IN(row * D + e * 32 + lane, o_size))
                        O[row * D + e * 32 + lane] = from_f32<T>(acc[e] * f.x * f.y);
                if (a.lse && lane == 0) a.lse[row] = natural_lse(s);
            } else {
                float *const to = cta_sums + (size_t)(2 * blockIdx.x + (starts ? 1 : 0)) * S::SUMS;
                if (lane == 0) {
                    __stcg(to + h, s.ref);
                    __stcg(to + H + h, s.top);
                    __stcg(to + 2 * H + h, s.sum);
                }
#pragma unroll
                for (int e = 0; e < E; ++e) __stcg(to + 3 * H + h * S::LD + e * 32 + lane, acc[e]);
            }
        }
    }

    // ---- rows that several CTAs share: this one's first run (begun before) and its last ---------------
    __syncthreads();
    if (tid < 2) {
        sh_last[tid] = 0;
        if (sh_open[tid]) {
            // (releases the CTA's sums, which the barrier ordered before it, and acquires the others')
            unsigned n;
            asm volatile("atom.add.acq_rel.gpu.u32 %0, [%1], 1;"
                         : "=r"(n) : "l"(&counters[sh_c0[tid]]) : "memory");
            sh_last[tid] = n == (unsigned)(sh_c1[tid] - sh_c0[tid]);
            if (sh_last[tid]) counters[sh_c0[tid]] = 0;
        }
    }
    __syncthreads();
#pragma unroll 1
    for (int k = 0; k < 2; ++k) {
        if (!sh_last[k]) continue;
        const Part p = sh_part[k ? last_run : first_part];
        const int head0 = p.u % a.blocks * H, heads = min(H, a.group - head0);
        const int n = sh_c1[k] - sh_c0[k] + 1;
        // the first CTA's sums are in its second place, the others' in their first
        const float *const base = cta_sums + (size_t)2 * sh_c0[k] * S::SUMS;
        auto sums = [&](int i) { return base + (size_t)(2 * i + (i == 0 ? 1 : 0)) * S::SUMS; };
        // several warps a head where there are more warps than heads, each a slice of the CTAs
        const int slices = max(1, W / heads);
        for (int i0 = 0; i0 < heads; i0 += W) {
            const int h = i0 + warp % heads, slice = heads > W ? 0 : warp / heads;
            const bool works = h < heads && slice < slices;
            Stat s = {0.0f, 0.0f, 0.0f};
            float acc[E];
#pragma unroll
            for (int e = 0; e < E; ++e) acc[e] = 0.0f;
            if (works) {
                s = {-FLT_MAX, -FLT_MAX, 0.0f};
                for (int i = lane; i < n; i += 32) {
                    const float *const q = sums(i) + h;
                    s = add(s, {__ldcg(q), __ldcg(q + H), __ldcg(q + 2 * H)});
                }
                s = add_lanes(s);
                const int lo = n * slice / slices, hi = n * (slice + 1) / slices;
#pragma unroll 4
                for (int i = lo; i < hi; ++i) {
                    const float *const q = sums(i);
                    const float f = ex2(__ldcg(q + h) - s.ref);
#pragma unroll
                    for (int e = 0; e < E; ++e) acc[e] += f * __ldcg(q + 3 * H + h * S::LD + e * 32 + lane);
                }
            }
            if (slices > 1) {
#pragma unroll
                for (int e = 0; e < E; ++e) sh_slice[warp][e * 32 + lane] = acc[e];
                __syncthreads();
                for (int j = 1; works && slice == 0 && j < slices; ++j)
#pragma unroll
                    for (int e = 0; e < E; ++e) acc[e] += sh_slice[j * heads + h][e * 32 + lane];
                __syncthreads();
            }
            if (works && slice == 0) {
                const size_t row = (size_t)p.b * a.q_heads + (p.u / a.blocks) * a.group + head0 + h;
                const float2 f = to_output(s);
#pragma unroll
                for (int e = 0; e < E; ++e)
                    if (MPQ_IN(row * D + e * 32 + lane, o_size))
                        O[row * D + e * 32 + lane] = from_f32<T>(acc[e] * f.x * f.y);
                if (a.lse && lane == 0) a.lse[row] = natural_lse(s);
            }
        }
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
    // the codes as rows of a page and head: [pages x 2 x heads][page][row] (a cache without pages is
    // never read; the map then names the workspace)
    CUtensorMap tm;
    memset(&tm, 0, sizeof(tm));
    const bool any = a.L.pages > 0;
    const cuuint64_t dims[3] = {(cuuint64_t)S::RB, (cuuint64_t)a.L.page,
                                any ? (cuuint64_t)a.L.pages * 2 * a.L.heads : 1};
    const cuuint64_t strides[2] = {(cuuint64_t)S::RB, (cuuint64_t)a.L.page * S::RB};
    const cuuint32_t box[3] = {(cuuint32_t)S::BOX, A_STAGE, 1};
    if (!encode_tile_map(&tm, CU_TENSOR_MAP_DATA_TYPE_UINT8, 3,
                         any ? (const void *)a.codes : (const void *)a.workspace, dims, strides, box,
                         S::BOX == 128  ? CU_TENSOR_MAP_SWIZZLE_128B
                         : S::BOX == 64 ? CU_TENSOR_MAP_SWIZZLE_64B
                                        : CU_TENSOR_MAP_SWIZZLE_32B)) {
        set_error("cache attention: tensor map encoding failed");
        return MPQ_ERR_CUDA;
    }
    WaitCtl wc;
    const mpq_status ws = wait_ctl(&wc);
    if (ws != MPQ_OK) return ws;
    // one CTA per SM, fewer where the tables cannot hold work for all their warps, but no fewer than rows (1 and
    // 4 sequences of 64 tokens 6.6 and 6.8 us, 8.2 and 10.0 with the CTAs that their stages wake); the
    // workspace has room for two rows' sums of each CTA and one of each warp
    const long long room = (long long)a.cols * a.L.page;
    const long long span = a.window > 0 ? std::min<long long>(room, a.window) + A_STAGE : room;
    const long long stages = (span + A_STAGE - 1) / A_STAGE * a.L.heads * a.blocks;   // of a sequence
    const long long fit =
        (long long)((MPQ_CACHE_WORKSPACE - A_COUNTERS) / ((2 + S::WARPS) * S::SUMS * sizeof(float)));
    const long long most = std::min<long long>(std::min<long long>(sm_count(), fit), A_MAX_CTAS);
    const long long wake = (long long)A_LEAST * S::WARPS;                 // stages that wake a CTA
    const long long rows = (long long)a.B * a.L.heads * a.blocks;
    const long long ctas = stages >= most * wake
                               ? most
                               : std::min(most, std::max(rows, (stages * a.B + wake - 1) / wake));
    return launch_waiting(cache_attention_kernel<T, D, BITS, NT>, dim3((unsigned)ctas),
                          dim3(S::THREADS), S::SMEM, stream, "cache attention launch", a, wc, tm);
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
    a.page_shift = -1;
    for (int i = 4; i <= 10; ++i)
        if (L->page == 1 << i) a.page_shift = i;
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
