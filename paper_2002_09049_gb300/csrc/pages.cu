// The pages of a cache's requests (mpq_pages_extend, mpq_pages_trim): which pages the requests' new tokens lie
// in, and which return, from lengths alone.
//
// Every CTA scans all requests -- pages and tokens before each, in sums that stop at 2^31 - 1 (saturating sums
// of non-negative numbers are associative) -- and leaves what its tokens need in shared memory; then a thread
// takes four consecutive tokens (pages, trimming) of the CTA's share, finds their request by bisection and
// walks on from there.  No CTA needs another's results: which page is the j-th given follows from the
// sums and the pool.  A new page's table entry is written with the token that is its first.  Where lengths or
// the count are updated in place, the last CTA to finish (a counter beside the count) writes them.
//
// Latency: 96 requests one token longer 5.0 us (a launch, the requests, two scans, a bisection, a table entry, a store,
// one after another), 1,024 prompts of 340,160 tokens 9.1 (4 MB out).
#include <limits.h>

#include <algorithm>

#include "elements.cuh"
#include "mpq_internal.cuh"
#include "sm100.cuh"

MPQ_CHECKED_UNIT("pages.cu");

namespace mpq {
namespace {

constexpr unsigned P_MOST = 0x7fffffffu;     // where sums stop: above every count, number and N
constexpr int P_EACH = 4;                    // tokens (pages) a thread takes at a time

struct PageArgs {
    int B, page, page_shift, cols, pages;    // page_shift: -1 where the page is no power of two
    const int *want, *lens;                  // add or keep
    int *new_lens, *count, *new_count;
    int in_place;                            // lens or count are: written by the last CTA
    long long N;
    int *taken;
};

// What a CTA keeps of request b: the number of its first token (page, trimming), its length, the
// number of its first new page; bit 31 of `first`: it is served.
struct Kept {
    int *start, *len;
    unsigned *first;
};

__device__ __forceinline__ unsigned add_most(unsigned a, unsigned b) { return min(a + b, P_MOST); }

__device__ __forceinline__ int div_page(const PageArgs &a, int n)
{
    return a.page_shift >= 0 ? n >> a.page_shift : n / a.page;
}
__device__ __forceinline__ int pages_of(const PageArgs &a, int n)      // n >= 0, n + page below 2^31
{
    return div_page(a, n + a.page - 1);
}

// The exclusive sum of a number over the CTA's threads, and the total.
__device__ __forceinline__ unsigned block_scan(unsigned own, unsigned &total, unsigned *warps)
{
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, n = (int)blockDim.x >> 5;
    auto warp_scan = [&](unsigned v) {
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const unsigned x = __shfl_up_sync(0xffffffffu, v, o);
            if (lane >= o) v = add_most(v, x);
        }
        return v;
    };
    const unsigned in = warp_scan(own);
    if (lane == 31) warps[warp] = in;
    __syncthreads();
    const unsigned w = warp_scan(lane < n ? warps[lane] : 0u);
    total = __shfl_sync(0xffffffffu, w, 31);
    const unsigned behind = __shfl_sync(0xffffffffu, w, max(warp - 1, 0));
    unsigned ex = __shfl_up_sync(0xffffffffu, in, 1);
    if (lane == 0) ex = 0;
    return warp == 0 ? ex : add_most(behind, ex);
}

// The last request that starts at or before number t.
__device__ __forceinline__ int request_of(const int *start, int B, int t)
{
    int lo = 0, hi = B;                      // start[lo] <= t < start[hi]
    while (hi - lo > 1) {
        const int m = (lo + hi) >> 1;
        if (start[m] <= t) lo = m; else hi = m;
    }
    return lo;
}

// True in the threads of the last CTA to come here (alone: at once).
__device__ __forceinline__ bool last_cta(int *counter)
{
    __shared__ int last;
    __syncthreads();
    if (threadIdx.x == 0) {
        __threadfence();
        last = atomicAdd(counter, 1) == (int)gridDim.x - 1;
        __threadfence();
    }
    __syncthreads();
    return last != 0;
}

// Every request's want and length into shared memory (where `start` and `len` will be), a warp's consecutive.
__device__ __forceinline__ void load_requests(const PageArgs &a, int *want, int *len)
{
    for (int b = (int)threadIdx.x; b < a.B; b += (int)blockDim.x) {
        want[b] = a.want[b];
        len[b] = a.lens[b];
    }
    __syncthreads();
}

// What a request asks of the pool: pages, and whether its length and numbers allow it.
struct Ask {
    int len, add, need;
    bool fits;
};
__device__ __forceinline__ Ask ask(const PageArgs &a, int want, int len)
{
    Ask r;
    r.len = len;
    r.add = max(want, 0);
    r.need = 0;
    r.fits = r.len >= 0 && (long long)r.len + r.add <= (long long)a.page * a.cols;
    if (r.fits) r.need = pages_of(a, r.len + r.add) - pages_of(a, r.len);
    return r;
}

__global__ void pages_extend_kernel(const PageArgs a, int *table, const int *pool, int64_t *slots,
                                    int *positions, long long share, int wide)
{
    extern __shared__ int kept[];
    __shared__ unsigned warps[2][32];    // (a scan after a scan has words of its own)
    const Kept k{kept, kept + a.B, reinterpret_cast<unsigned *>(kept + 2 * a.B)};
    sm100::griddep_launch();
    sm100::griddep_wait();
    const int have = min(max(a.count[0], 0), a.pages);
    load_requests(a, k.start, k.len);
    // the thread's requests: their tokens, then (which of them fit in N is known) their pages
    const int per = (a.B + (int)blockDim.x - 1) / (int)blockDim.x;
    const int b0 = min((int)threadIdx.x * per, a.B), b1 = min(b0 + per, a.B);
    unsigned all, ignored, tokens = 0;
    for (int b = b0; b < b1; ++b) tokens = add_most(tokens, (unsigned)max(k.start[b], 0));
    const unsigned t0 = block_scan(tokens, all, warps[0]), N = (unsigned)a.N;
    unsigned at = t0, need = 0;
    for (int b = b0; b < b1; ++b) {
        const Ask r = ask(a, k.start[b], k.len[b]);
        at = add_most(at, (unsigned)r.add);
        if (r.fits && at <= N) need = add_most(need, (unsigned)r.need);
    }
    unsigned before = block_scan(need, ignored, warps[1]);
    // the pages given: those of the last served request and all before it
    unsigned given = 0;
    const bool writer = !a.in_place && blockIdx.x == 0;
    at = t0;
    for (int b = b0; b < b1; ++b) {
        const Ask r = ask(a, k.start[b], k.len[b]);
        const unsigned end = add_most(at, (unsigned)r.add);
        const bool fits = r.fits && end <= N;
        const unsigned upto = add_most(before, fits ? (unsigned)r.need : 0u);
        const bool served = fits && (r.need == 0 || upto <= (unsigned)have);
        if (served) given = r.need ? upto : given;
        k.start[b] = (int)at;
        k.len[b] = r.len;
        k.first[b] = before | (served ? 0x80000000u : 0u);
        if (writer) {
            a.taken[b] = served ? r.add : 0;
            a.new_lens[b] = r.len + (served ? r.add : 0);
        }
        at = end;
        before = upto;
    }
    const int left = have - (int)__reduce_max_sync(0xffffffffu, given);
    if ((threadIdx.x & 31) == 0) warps[0][threadIdx.x >> 5] = (unsigned)left;
    __syncthreads();
    if (writer && threadIdx.x == 0) {
        unsigned least = warps[0][0];
        for (int i = 1; i < (int)blockDim.x >> 5; ++i) least = min(least, warps[0][i]);
        a.new_count[0] = (int)least;
        a.new_count[1] = 0;
    }

    // ---- the CTA's tokens
    const long long from = blockIdx.x * share, to = min(from + share, a.N);
    for (long long t0 = from + (long long)threadIdx.x * P_EACH; t0 < to; t0 += (long long)blockDim.x * P_EACH) {
        int64_t s[P_EACH];
        int p[P_EACH];
        int b = (unsigned)t0 < all && a.B > 0 ? request_of(k.start, a.B, (int)t0) : a.B;
#pragma unroll
        for (int i = 0; i < P_EACH; ++i) {
            const long long t = t0 + i;
            s[i] = -1;
            p[i] = 0;
            if (t >= to || (unsigned)t >= all) continue;
            while (b + 1 < a.B && k.start[b + 1] <= (int)t) ++b;
            const int len = k.len[b], at = len + (int)(t - k.start[b]);      // (wraps where len is at odds)
            p[i] = at;
            if (!(k.first[b] >> 31)) continue;
            const int col = div_page(a, at), held = pages_of(a, len), place = at - col * a.page;
            int page;
            if (col < held) {
                page = table[(size_t)b * a.cols + col];
            } else {
                const int j = (int)(k.first[b] & P_MOST) + col - held;
                page = pool[have - 1 - j];
                if (place == 0 && MPQ_IN((size_t)b * a.cols + col, (size_t)a.B * a.cols))
                    table[(size_t)b * a.cols + col] = page;
            }
            if (page >= 0) s[i] = (int64_t)page * a.page + place;
        }
        const int n = (int)min((long long)P_EACH, to - t0);
        if (wide && n == P_EACH && MPQ_IN(t0 + P_EACH - 1, a.N)) {   // (t0 is a multiple of P_EACH)
            longlong2 *const so = reinterpret_cast<longlong2 *>(slots + t0);
            so[0] = make_longlong2(s[0], s[1]);
            so[1] = make_longlong2(s[2], s[3]);
            *reinterpret_cast<int4 *>(positions + t0) = make_int4(p[0], p[1], p[2], p[3]);
            continue;
        }
        for (int i = 0; i < n; ++i) {
            if (!MPQ_IN(t0 + i, a.N)) continue;
            slots[t0 + i] = s[i];
            positions[t0 + i] = p[i];
        }
    }
    if (!a.in_place) return;
    if (gridDim.x > 1 && !last_cta(a.count + 1)) return;
    __syncthreads();                         // (alone: every read of the lengths is done)
    for (int b = (int)threadIdx.x; b < a.B; b += (int)blockDim.x) {
        const bool served = k.first[b] >> 31;
        const int add = max(a.want[b], 0);
        a.taken[b] = served ? add : 0;
        a.new_lens[b] = k.len[b] + (served ? add : 0);
    }
    if (threadIdx.x == 0) {
        unsigned least = warps[0][0];
        for (int i = 1; i < (int)blockDim.x >> 5; ++i) least = min(least, warps[0][i]);
        a.count[1] = 0;
        a.new_count[0] = (int)least;
        a.new_count[1] = 0;
    }
}

__global__ void pages_trim_kernel(const PageArgs a, const int *table, int *pool)
{
    extern __shared__ int kept[];            // start: the number of a request's first page that returns; len: its column
    __shared__ unsigned warps[2][32];    // (a scan after a scan has words of its own)
    const Kept k{kept, kept + a.B, nullptr};
    sm100::griddep_launch();
    sm100::griddep_wait();
    const int have = min(max(a.count[0], 0), a.pages);
    load_requests(a, k.start, k.len);
    const int per = (a.B + (int)blockDim.x - 1) / (int)blockDim.x;
    const int b0 = min((int)threadIdx.x * per, a.B), b1 = min(b0 + per, a.B);
    const int longest = a.page * a.cols;     // up to 2^30
    auto cut = [&](int want, int n, int &len, int &keep) {
        len = min(max(n, 0), longest);
        keep = min(max(want, 0), len);
    };
    unsigned back = 0;
    for (int b = b0; b < b1; ++b) {
        int len, keep;
        cut(k.start[b], k.len[b], len, keep);
        back = add_most(back, (unsigned)(pages_of(a, len) - pages_of(a, keep)));
    }
    unsigned all, before = block_scan(back, all, warps[0]);
    const bool writer = !a.in_place && blockIdx.x == 0;
    for (int b = b0; b < b1; ++b) {
        int len, keep;
        cut(k.start[b], k.len[b], len, keep);
        k.start[b] = (int)before;
        k.len[b] = pages_of(a, keep);
        before = add_most(before, (unsigned)(pages_of(a, len) - pages_of(a, keep)));
        if (writer) a.new_lens[b] = keep;
    }
    const int now = (int)min((long long)have + all, (long long)a.pages);
    if (writer && threadIdx.x == 0) {
        a.new_count[0] = now;
        a.new_count[1] = 0;
    }
    __syncthreads();
    const long long step = (long long)gridDim.x * blockDim.x * P_EACH;
    for (long long j0 = ((long long)blockIdx.x * blockDim.x + threadIdx.x) * P_EACH; j0 < all; j0 += step) {
        int b = request_of(k.start, a.B, (int)j0);
        for (int i = 0; i < P_EACH && j0 + i < all; ++i) {
            const int j = (int)j0 + i;
            while (b + 1 < a.B && k.start[b + 1] <= j) ++b;
            const long long to = (long long)have + all - 1 - j;
            if (to < a.pages && MPQ_IN(to, a.pages))
                pool[to] = table[(size_t)b * a.cols + k.len[b] + (j - k.start[b])];
        }
    }
    if (!a.in_place) return;
    if (gridDim.x > 1 && !last_cta(a.count + 1)) return;
    __syncthreads();
    for (int b = (int)threadIdx.x; b < a.B; b += (int)blockDim.x) {
        int len, keep;
        cut(a.want[b], a.lens[b], len, keep);
        a.new_lens[b] = keep;
    }
    if (threadIdx.x == 0) {
        a.count[1] = 0;
        a.new_count[0] = now;
        a.new_count[1] = 0;
    }
}

PageArgs page_args(const int *want, int B, int page, int cols, const int *lens, int *new_lens, int pages,
                   int *count, int *new_count)
{
    PageArgs a = {};
    a.B = B;
    a.page = page;
    int s = 0;
    while (s < 30 && 1 << s < page) ++s;
    a.page_shift = 1 << s == page ? s : -1;
    a.cols = cols;
    a.pages = pages;
    a.want = want;
    a.lens = lens;
    a.new_lens = new_lens;
    a.count = count;
    a.new_count = new_count;
    a.in_place = new_lens == lens || new_count == count;
    return a;
}

int page_threads(int B) { return B <= 1024 ? 256 : 1024; }

}  // namespace

mpq_status launch_pages_extend(const int *add, int B, int page, int cols, const int *lens, int *new_lens,
                               int *table, const int *pool, int pages, int *count, int *new_count,
                               int64_t *slots, int *positions, long long N, int *taken, cudaStream_t stream)
{
    PageArgs a = page_args(add, B, page, cols, lens, new_lens, pages, count, new_count);
    a.N = N;
    a.taken = taken;
    const int threads = page_threads(B);
    // a CTA scans every request: four CTAs of 256 threads an SM at most, two of 1,024
    const long long one = (long long)threads * P_EACH, most = (threads == 256 ? 4LL : 2LL) * sm_count();
    const long long share = std::max(one, ((N + most - 1) / most + one - 1) / one * one);
    const int grid = (int)std::max(1LL, (N + share - 1) / share);
    const int wide = ((uintptr_t)slots | (uintptr_t)positions) % 16 == 0;
    static_assert(P_EACH == 4, "the wide stores");
    const size_t smem = (size_t)B * 3 * sizeof(int);
    static std::atomic<int> limit[kMaxDevices];
    const cudaError_t e = allow_smem(reinterpret_cast<const void *>(pages_extend_kernel), limit, smem);
    if (e != cudaSuccess) return cuda_status(e, "cudaFuncSetAttribute");
    return launch_waiting(pages_extend_kernel, dim3((unsigned)grid), dim3((unsigned)threads), smem, stream,
                          "pages extend launch", a, table, pool, slots, positions, share, wide);
}

mpq_status launch_pages_trim(const int *keep, int B, int page, int cols, const int *lens, int *new_lens,
                             const int *table, int *pool, int pages, int *count, int *new_count,
                             cudaStream_t stream)
{
    const PageArgs a = page_args(keep, B, page, cols, lens, new_lens, pages, count, new_count);
    const int threads = page_threads(B);
    const long long one = (long long)threads * P_EACH, held = std::min((long long)pages, (long long)B * cols);
    const int grid = (int)std::min(std::max(1LL, (held + one - 1) / one), 2LL * sm_count());
    const size_t smem = (size_t)B * 2 * sizeof(int);
    static std::atomic<int> limit[kMaxDevices];
    const cudaError_t e = allow_smem(reinterpret_cast<const void *>(pages_trim_kernel), limit, smem);
    if (e != cudaSuccess) return cuda_status(e, "cudaFuncSetAttribute");
    return launch_waiting(pages_trim_kernel, dim3((unsigned)grid), dim3((unsigned)threads), smem, stream,
                          "pages trim launch", a, table, pool);
}

}  // namespace mpq
