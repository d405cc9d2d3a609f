// Host side of the few-bit serving entry points (include/mpq.h, "Serving in few bits"): argument
// validation, error reporting, dispatch to the kernel launchers.
#include <limits.h>
#include <math.h>

#include "api_common.cuh"
#include "elements.cuh"
#include "mpq_internal.cuh"

using namespace mpq;

static mpq_status check_type(int type, const char *what)
{
    REQUIRE(type_size(type) != 0, MPQ_ERR_INVALID_ARG,
            "%s = %d is not MPQ_F32, MPQ_F16 or MPQ_BF16", what, type);
    return MPQ_OK;
}

// A layout is one that its maker filled in (its fields are used unseen by the kernels).
static mpq_status check_mx(const mpq_mx_matrix *L, const char *what)
{
    REQUIRE(L, MPQ_ERR_INVALID_ARG, "%s must be non-NULL", what);
    mpq_mx_matrix own;
    const mpq_status st = mpq_mx_layout(L->rows, L->d, &own);
    if (st != MPQ_OK) return st;
    REQUIRE(own.d_pad == L->d_pad && own.row_tiles == L->row_tiles && own.k_tiles == L->k_tiles &&
                own.off_scales == L->off_scales && own.bytes == L->bytes,
            MPQ_ERR_INVALID_ARG, "%s is not one that mpq_mx_layout made", what);
    return MPQ_OK;
}

static mpq_status check_cache(const mpq_kv_cache *L)
{
    REQUIRE(L, MPQ_ERR_INVALID_ARG, "layout must be non-NULL");
    mpq_kv_cache own;
    const mpq_status st = mpq_cache_layout(L->pages, L->page, L->heads, L->dim, L->bits, &own);
    if (st != MPQ_OK) return st;
    REQUIRE(own.row_bytes == L->row_bytes && own.codes_bytes == L->codes_bytes &&
                own.scales_bytes == L->scales_bytes,
            MPQ_ERR_INVALID_ARG, "layout is not one that mpq_cache_layout made");
    return MPQ_OK;
}

static bool on(const void *p, size_t bytes) { return (uintptr_t)p % bytes == 0; }
static bool aligned16(const void *p) { return on(p, 16); }

extern "C" mpq_status mpq_mx_layout(int rows, int d, mpq_mx_matrix *layout)
{
    clear_error();
    REQUIRE(layout, MPQ_ERR_INVALID_ARG, "layout must be non-NULL");
    REQUIRE(rows >= 0, MPQ_ERR_INVALID_ARG, "rows = %d must be >= 0", rows);
    REQUIRE(d >= 1, MPQ_ERR_INVALID_ARG, "d = %d must be >= 1", d);
    REQUIRE(d <= MPQ_MX_MAX_DIM, MPQ_ERR_UNSUPPORTED, "d = %d exceeds MPQ_MX_MAX_DIM = %d", d,
            MPQ_MX_MAX_DIM);
    REQUIRE((long long)rows * d <= (1LL << 40), MPQ_ERR_UNSUPPORTED, "rows*d = %lld too large",
            (long long)rows * d);
    return make_mx_layout(rows, d, layout);
}

extern "C" mpq_status mpq_mx_quantize(const void *X, int x_type, long long ldx,
                                      const mpq_mx_matrix *layout, void *packed, void *stream)
{
    CallRange range_("mpq_mx_quantize");
    clear_error();
    mpq_status st = check_mx(layout, "layout");
    if (st == MPQ_OK) st = check_type(x_type, "x_type");
    if (st != MPQ_OK) return st;
    REQUIRE(ldx >= layout->d, MPQ_ERR_INVALID_ARG, "ldx = %lld must be >= d = %d", ldx, layout->d);
    if (layout->rows == 0) return MPQ_OK;
    REQUIRE(X && packed, MPQ_ERR_INVALID_ARG, "X and packed must be non-NULL");
    REQUIRE(on(X, type_size(x_type)), MPQ_ERR_INVALID_ARG, "X must be aligned to its elements");
    REQUIRE(aligned16(packed), MPQ_ERR_INVALID_ARG, "packed must be 16-byte aligned");
    return launch_mx_quantize(X, x_type, ldx, layout, packed, (cudaStream_t)stream);
}

extern "C" mpq_status mpq_mx_dequantize(const void *packed, const mpq_mx_matrix *layout, void *Y,
                                        int y_type, long long ldy, void *stream)
{
    CallRange range_("mpq_mx_dequantize");
    clear_error();
    mpq_status st = check_mx(layout, "layout");
    if (st == MPQ_OK) st = check_type(y_type, "y_type");
    if (st != MPQ_OK) return st;
    REQUIRE(ldy >= layout->d, MPQ_ERR_INVALID_ARG, "ldy = %lld must be >= d = %d", ldy, layout->d);
    if (layout->rows == 0) return MPQ_OK;
    REQUIRE(packed && Y, MPQ_ERR_INVALID_ARG, "packed and Y must be non-NULL");
    REQUIRE(on(Y, type_size(y_type)), MPQ_ERR_INVALID_ARG, "Y must be aligned to its elements");
    REQUIRE(aligned16(packed), MPQ_ERR_INVALID_ARG, "packed must be 16-byte aligned");
    return launch_mx_dequantize(packed, layout, Y, y_type, ldy, (cudaStream_t)stream);
}

extern "C" mpq_status mpq_mx_linear(const mpq_mx_matrix *x_layout, const void *X,
                                    const mpq_mx_matrix *w_layout, const void *W, const float *bias,
                                    void *Y, int y_type, long long ldy, void *stream)
{
    CallRange range_("mpq_mx_linear");
    clear_error();
    mpq_status st = check_mx(x_layout, "x_layout");
    if (st == MPQ_OK) st = check_mx(w_layout, "w_layout");
    if (st == MPQ_OK) st = check_type(y_type, "y_type");
    if (st != MPQ_OK) return st;
    REQUIRE(x_layout->d == w_layout->d, MPQ_ERR_INVALID_ARG,
            "the inputs have d = %d, the weights d = %d", x_layout->d, w_layout->d);
    REQUIRE(ldy >= w_layout->rows, MPQ_ERR_INVALID_ARG, "ldy = %lld must be >= C = %d", ldy,
            w_layout->rows);
    if (x_layout->rows == 0 || w_layout->rows == 0) return MPQ_OK;
    REQUIRE(X && W && Y, MPQ_ERR_INVALID_ARG, "X, W and Y must be non-NULL");
    REQUIRE(aligned16(X) && aligned16(W), MPQ_ERR_INVALID_ARG, "X and W must be 16-byte aligned");
    REQUIRE(on(bias, sizeof(float)) && on(Y, type_size(y_type)), MPQ_ERR_INVALID_ARG,
            "bias and Y must be aligned to their elements");
    return launch_mx_linear(x_layout, X, w_layout, W, bias, Y, y_type, ldy, (cudaStream_t)stream);
}

extern "C" mpq_status mpq_cache_layout(int pages, int page, int heads, int dim, int bits,
                                       mpq_kv_cache *layout)
{
    clear_error();
    REQUIRE(layout, MPQ_ERR_INVALID_ARG, "layout must be non-NULL");
    REQUIRE(pages >= 0, MPQ_ERR_INVALID_ARG, "pages = %d must be >= 0", pages);
    REQUIRE(page >= 1, MPQ_ERR_INVALID_ARG, "page = %d must be >= 1", page);
    REQUIRE(page % 16 == 0 && page <= 1024, MPQ_ERR_UNSUPPORTED,
            "page = %d must be a multiple of 16, at most 1024", page);
    REQUIRE(heads >= 1, MPQ_ERR_INVALID_ARG, "heads = %d must be >= 1", heads);
    REQUIRE(heads <= 1024, MPQ_ERR_UNSUPPORTED, "heads = %d exceeds 1024", heads);
    REQUIRE((long long)pages * 2 * heads <= INT_MAX, MPQ_ERR_UNSUPPORTED,
            "pages * 2 * heads = %lld too large", (long long)pages * 2 * heads);
    REQUIRE(dim >= 1, MPQ_ERR_INVALID_ARG, "dim = %d must be >= 1", dim);
    REQUIRE(dim == 64 || dim == 128 || dim == 256, MPQ_ERR_UNSUPPORTED,
            "dim = %d is not 64, 128 or 256", dim);
    REQUIRE(bits == 8 || bits == 4,
            bits < MPQ_MIN_BITS ? MPQ_ERR_INVALID_ARG : MPQ_ERR_UNSUPPORTED,
            "bits = %d is not 8 or 4", bits);
    return make_cache_layout(pages, page, heads, dim, bits, layout);
}

static mpq_status check_tokens(int T, const mpq_kv_cache *layout, int type)
{
    mpq_status st = check_cache(layout);
    if (st == MPQ_OK) st = check_type(type, "type");
    if (st != MPQ_OK) return st;
    REQUIRE(T >= 0, MPQ_ERR_INVALID_ARG, "T = %d must be >= 0", T);
    REQUIRE((long long)T * 2 * layout->heads <= INT_MAX, MPQ_ERR_UNSUPPORTED,
            "T * 2 * heads = %lld too large", (long long)T * 2 * layout->heads);
    return MPQ_OK;
}

extern "C" mpq_status mpq_cache_write(const void *K, const void *V, int type, long long ld_token,
                                      long long ld_head, int T, const int64_t *slots,
                                      const mpq_kv_cache *layout, void *codes, float *scales,
                                      void *stream)
{
    CallRange range_("mpq_cache_write");
    clear_error();
    const mpq_status st = check_tokens(T, layout, type);
    if (st != MPQ_OK) return st;
    REQUIRE(ld_token >= 0 && ld_head >= 0, MPQ_ERR_INVALID_ARG,
            "ld_token = %lld and ld_head = %lld must be >= 0", ld_token, ld_head);
    if (T == 0 || layout->pages == 0) return MPQ_OK;
    REQUIRE(K && V && slots && codes && scales, MPQ_ERR_INVALID_ARG,
            "K, V, slots, codes and scales must be non-NULL");
    REQUIRE(aligned16(codes), MPQ_ERR_INVALID_ARG, "codes must be 16-byte aligned");
    REQUIRE(on(K, type_size(type)) && on(V, type_size(type)) && on(slots, sizeof(int64_t)) &&
                on(scales, sizeof(float)),
            MPQ_ERR_INVALID_ARG, "K, V, slots and scales must be aligned to their elements");
    return launch_cache_write(K, V, type, ld_token, ld_head, T, slots, layout, codes, scales,
                              (cudaStream_t)stream);
}

extern "C" mpq_status mpq_cache_read(const int64_t *slots, int T, const mpq_kv_cache *layout,
                                     const void *codes, const float *scales, void *K, void *V,
                                     int type, void *stream)
{
    CallRange range_("mpq_cache_read");
    clear_error();
    const mpq_status st = check_tokens(T, layout, type);
    if (st != MPQ_OK) return st;
    if (T == 0) return MPQ_OK;
    REQUIRE(slots && K && V, MPQ_ERR_INVALID_ARG, "slots, K and V must be non-NULL");
    REQUIRE(layout->pages == 0 || (codes && scales), MPQ_ERR_INVALID_ARG,
            "codes and scales must be non-NULL");
    REQUIRE(aligned16(codes) && aligned16(K) && aligned16(V), MPQ_ERR_INVALID_ARG,
            "codes, K and V must be 16-byte aligned");
    REQUIRE(on(slots, sizeof(int64_t)) && on(scales, sizeof(float)), MPQ_ERR_INVALID_ARG,
            "slots and scales must be aligned to their elements");
    return launch_cache_read(slots, T, layout, codes, scales, K, V, type, (cudaStream_t)stream);
}

extern "C" mpq_status mpq_cache_attention(const void *Q, int type, long long q_stride, int B,
                                          int q_heads, const mpq_kv_cache *layout,
                                          const void *codes, const float *scales, const int *table,
                                          int table_cols, const int *lens, float scale, int window,
                                          void *O, float *lse, void *workspace,
                                          size_t workspace_bytes, void *stream)
{
    CallRange range_("mpq_cache_attention");
    clear_error();
    mpq_status st = check_cache(layout);
    if (st == MPQ_OK) st = check_type(type, "type");
    if (st != MPQ_OK) return st;
    REQUIRE(type != MPQ_F32, MPQ_ERR_UNSUPPORTED, "queries are MPQ_F16 or MPQ_BF16");
    REQUIRE(B >= 0, MPQ_ERR_INVALID_ARG, "B = %d must be >= 0", B);
    REQUIRE(q_heads >= layout->heads && q_heads % layout->heads == 0, MPQ_ERR_INVALID_ARG,
            "q_heads = %d must be a multiple of heads = %d", q_heads, layout->heads);
    REQUIRE((long long)q_heads * layout->dim <= INT_MAX, MPQ_ERR_UNSUPPORTED,
            "q_heads = %d is too large", q_heads);
    REQUIRE(q_stride >= 0, MPQ_ERR_INVALID_ARG, "q_stride = %lld must be >= 0", q_stride);
    REQUIRE(table_cols >= 0, MPQ_ERR_INVALID_ARG, "table_cols = %d must be >= 0", table_cols);
    // token indices of a sequence (and of the tiles past its end) are 32-bit
    REQUIRE((long long)table_cols * layout->page <= (1LL << 30), MPQ_ERR_UNSUPPORTED,
            "table_cols * page = %lld exceeds 2^30 tokens", (long long)table_cols * layout->page);
    REQUIRE(isfinite(scale), MPQ_ERR_NONFINITE, "scale is not finite");
    REQUIRE(window >= 0, MPQ_ERR_INVALID_ARG, "window = %d must be >= 0", window);
    if (B == 0) return MPQ_OK;
    REQUIRE(Q && lens && O, MPQ_ERR_INVALID_ARG, "Q, lens and O must be non-NULL");
    REQUIRE(table_cols == 0 || table, MPQ_ERR_INVALID_ARG, "table must be non-NULL");
    REQUIRE(layout->pages == 0 || (codes && scales), MPQ_ERR_INVALID_ARG,
            "codes and scales must be non-NULL");
    REQUIRE(aligned16(codes) && aligned16(scales) && aligned16(O) && aligned16(workspace),
            MPQ_ERR_INVALID_ARG, "codes, scales, O and workspace must be 16-byte aligned");
    REQUIRE(on(Q, type_size(type)) && on(table, sizeof(int)) && on(lens, sizeof(int)) && on(lse, sizeof(float)),
            MPQ_ERR_INVALID_ARG, "Q, table, lens and lse must be aligned to their elements");
    REQUIRE(!workspace || workspace_bytes >= MPQ_CACHE_WORKSPACE, MPQ_ERR_INVALID_ARG,
            "workspace of %zu bytes: %zu are needed", workspace_bytes, MPQ_CACHE_WORKSPACE);
    return launch_cache_attention(Q, type, q_stride, B, q_heads, layout, codes, scales, table,
                                  table_cols, lens, scale, window, O, lse, workspace,
                                  (cudaStream_t)stream);
}

extern "C" size_t mpq_cache_attention_workspace(void) { return MPQ_CACHE_WORKSPACE; }

static mpq_status check_g4(const mpq_g4_matrix *L, const char *what)
{
    REQUIRE(L, MPQ_ERR_INVALID_ARG, "%s must be non-NULL", what);
    mpq_g4_matrix own;
    const mpq_status st = mpq_g4_layout(L->rows, L->d, L->group, L->zeros, &own);
    if (st != MPQ_OK) return st;
    REQUIRE(own.row_tiles == L->row_tiles && own.k_tiles == L->k_tiles && own.tile_bytes == L->tile_bytes &&
                own.bytes == L->bytes,
            MPQ_ERR_INVALID_ARG, "%s is not one that mpq_g4_layout made", what);
    return MPQ_OK;
}

extern "C" mpq_status mpq_g4_layout(int rows, int d, int group, int zeros, mpq_g4_matrix *layout)
{
    clear_error();
    REQUIRE(layout, MPQ_ERR_INVALID_ARG, "layout must be non-NULL");
    REQUIRE(rows >= 0, MPQ_ERR_INVALID_ARG, "rows = %d must be >= 0", rows);
    REQUIRE(d >= 1, MPQ_ERR_INVALID_ARG, "d = %d must be >= 1", d);
    REQUIRE(d <= MPQ_MX_MAX_DIM, MPQ_ERR_UNSUPPORTED, "d = %d exceeds MPQ_MX_MAX_DIM = %d", d,
            MPQ_MX_MAX_DIM);
    REQUIRE((long long)rows * d <= (1LL << 40), MPQ_ERR_UNSUPPORTED, "rows*d = %lld too large",
            (long long)rows * d);
    REQUIRE(group >= 1, MPQ_ERR_INVALID_ARG, "group = %d must be >= 1", group);
    REQUIRE(group == 32 || group == 64 || group == 128, MPQ_ERR_UNSUPPORTED,
            "group = %d is not 32, 64 or 128", group);
    REQUIRE(zeros == 0 || zeros == 1, MPQ_ERR_INVALID_ARG, "zeros = %d is not 0 or 1", zeros);
    return make_g4_layout(rows, d, group, zeros, layout);
}

extern "C" mpq_status mpq_g4_quantize(const void *X, int x_type, long long ldx, const mpq_g4_matrix *layout,
                                      void *packed, void *stream)
{
    CallRange range_("mpq_g4_quantize");
    clear_error();
    mpq_status st = check_g4(layout, "layout");
    if (st == MPQ_OK) st = check_type(x_type, "x_type");
    if (st != MPQ_OK) return st;
    REQUIRE(ldx >= layout->d, MPQ_ERR_INVALID_ARG, "ldx = %lld must be >= d = %d", ldx, layout->d);
    if (layout->rows == 0) return MPQ_OK;
    REQUIRE(X && packed, MPQ_ERR_INVALID_ARG, "X and packed must be non-NULL");
    REQUIRE(on(X, type_size(x_type)), MPQ_ERR_INVALID_ARG, "X must be aligned to its elements");
    REQUIRE(aligned16(packed), MPQ_ERR_INVALID_ARG, "packed must be 16-byte aligned");
    return launch_g4_quantize(X, x_type, ldx, layout, packed, (cudaStream_t)stream);
}

extern "C" mpq_status mpq_g4_dequantize(const void *packed, const mpq_g4_matrix *layout, void *Y, int y_type,
                                        long long ldy, void *stream)
{
    CallRange range_("mpq_g4_dequantize");
    clear_error();
    mpq_status st = check_g4(layout, "layout");
    if (st == MPQ_OK) st = check_type(y_type, "y_type");
    if (st != MPQ_OK) return st;
    REQUIRE(ldy >= layout->d, MPQ_ERR_INVALID_ARG, "ldy = %lld must be >= d = %d", ldy, layout->d);
    if (layout->rows == 0) return MPQ_OK;
    REQUIRE(packed && Y, MPQ_ERR_INVALID_ARG, "packed and Y must be non-NULL");
    REQUIRE(on(Y, type_size(y_type)), MPQ_ERR_INVALID_ARG, "Y must be aligned to its elements");
    REQUIRE(aligned16(packed), MPQ_ERR_INVALID_ARG, "packed must be 16-byte aligned");
    return launch_g4_dequantize(packed, layout, Y, y_type, ldy, (cudaStream_t)stream);
}

static mpq_status g4_linear(const void *X, int x_type, long long ldx, int T, const mpq_g4_matrix *w_layout,
                            const void *W, const float *bias, void *Y, int y_type, long long ldy, int exact,
                            void *stream)
{
    clear_error();
    mpq_status st = check_g4(w_layout, "w_layout");
    if (st == MPQ_OK) st = check_type(x_type, "x_type");
    if (st == MPQ_OK) st = check_type(y_type, "y_type");
    if (st != MPQ_OK) return st;
    REQUIRE(x_type != MPQ_F32, MPQ_ERR_UNSUPPORTED, "inputs are MPQ_F16 or MPQ_BF16");
    REQUIRE(T >= 0, MPQ_ERR_INVALID_ARG, "T = %d must be >= 0", T);
    REQUIRE(T <= 1 << 20, MPQ_ERR_UNSUPPORTED, "T = %d exceeds 2^20", T);
    REQUIRE(ldx >= w_layout->d, MPQ_ERR_INVALID_ARG, "ldx = %lld must be >= d = %d", ldx, w_layout->d);
    REQUIRE(ldy >= w_layout->rows, MPQ_ERR_INVALID_ARG, "ldy = %lld must be >= C = %d", ldy, w_layout->rows);
    if (T == 0 || w_layout->rows == 0) return MPQ_OK;
    REQUIRE(X && W && Y, MPQ_ERR_INVALID_ARG, "X, W and Y must be non-NULL");
    REQUIRE(aligned16(W), MPQ_ERR_INVALID_ARG, "W must be 16-byte aligned");
    REQUIRE(on(X, type_size(x_type)) && on(bias, sizeof(float)) && on(Y, type_size(y_type)), MPQ_ERR_INVALID_ARG,
            "X, bias and Y must be aligned to their elements");
    return launch_g4_linear(X, x_type, ldx, T, w_layout, W, bias, Y, y_type, ldy, exact, (cudaStream_t)stream);
}

extern "C" mpq_status mpq_g4_linear(const void *X, int x_type, long long ldx, int T,
                                    const mpq_g4_matrix *w_layout, const void *W, const float *bias, void *Y,
                                    int y_type, long long ldy, void *stream)
{
    CallRange range_("mpq_g4_linear");
    return g4_linear(X, x_type, ldx, T, w_layout, W, bias, Y, y_type, ldy, 0, stream);
}

extern "C" mpq_status mpq_g4_linear_exact(const void *X, int x_type, long long ldx, int T,
                                          const mpq_g4_matrix *w_layout, const void *W, const float *bias,
                                          void *Y, int y_type, long long ldy, void *stream)
{
    CallRange range_("mpq_g4_linear_exact");
    return g4_linear(X, x_type, ldx, T, w_layout, W, bias, Y, y_type, ldy, 1, stream);
}

extern "C" mpq_status mpq_test_g4_form(int form, int tokens, int split)
{
    clear_error();
    REQUIRE(form >= 0 && form <= MPQ_G4_PAIRS, MPQ_ERR_INVALID_ARG, "form = %d is not one of MPQ_G4_*", form);
    const bool tiles = form == MPQ_G4_TILES;
    REQUIRE(!tiles || (tokens >= 16 && tokens <= 256 && tokens % 16 == 0), MPQ_ERR_INVALID_ARG,
            "tokens = %d is not a multiple of 16, 16..256", tokens);
    REQUIRE(!tiles || split == 1 || split == 2 || split == 4 || split == 8, MPQ_ERR_INVALID_ARG,
            "split = %d is not 1, 2, 4 or 8", split);
    set_g4_test_form({form, tiles ? tokens : 0, tiles ? split : 1});
    return MPQ_OK;
}

extern "C" mpq_status mpq_rotation_turns(const double *freq, int n, uint64_t *turns)
{
    clear_error();
    REQUIRE(n >= 0, MPQ_ERR_INVALID_ARG, "n = %d must be >= 0", n);
    REQUIRE(n == 0 || (freq && turns), MPQ_ERR_INVALID_ARG, "freq and turns must be non-NULL");
    constexpr double hi = 0x1.45f306dc9c883p-3, lo = -0x1.6b01ec5417056p-57;      // 1 / 2 pi = hi + lo
    for (int i = 0; i < n; ++i) {
        const double f = freq[i];
        REQUIRE(isfinite(f), MPQ_ERR_NONFINITE, "freq[%d] is not finite", i);
        REQUIRE(fabs(f) <= 0x1p32, MPQ_ERR_UNSUPPORTED, "freq[%d] = %g exceeds 2^32", i, f);
        // |f| / 2 pi: its places down to 2^-64, then what the product and 1 / 2 pi have below (under 2^-20)
        const double m = fabs(f), p = m * hi, rest = fma(m, hi, -p) + m * lo, frac = ldexp(p - floor(p), 64);
        const uint64_t whole = (uint64_t)frac;
        const uint64_t t = whole + (uint64_t)llrint(frac - (double)whole + ldexp(rest, 64));
        turns[i] = f < 0.0 ? 0 - t : t;
    }
    return MPQ_OK;
}

// One side of a rotation: heads, strides (those of the output without overlap), pointers.
static mpq_status check_rows(const mpq_rotate_rows *r, int type, int T, int dim, int norm, const char *what)
{
    REQUIRE(r->heads >= 0 && r->heads <= 65536, r->heads < 0 ? MPQ_ERR_INVALID_ARG : MPQ_ERR_UNSUPPORTED,
            "%s: heads = %d must be 0..65536", what, r->heads);
    if (T == 0 || r->heads == 0) return MPQ_OK;
    REQUIRE(r->x && r->y, MPQ_ERR_INVALID_ARG, "%s: x and y must be non-NULL", what);
    REQUIRE(on(r->x, type_size(type)) && on(r->y, type_size(type)) && on(r->weight, sizeof(float)),
            MPQ_ERR_INVALID_ARG, "%s: x, y and weight must be aligned to their elements", what);
    REQUIRE(norm || !r->weight, MPQ_ERR_INVALID_ARG, "%s: weights without a norm", what);
    REQUIRE(r->ld_token >= 0 && r->ld_head >= 0, MPQ_ERR_INVALID_ARG,
            "%s: ld_token = %lld and ld_head = %lld must be >= 0", what, r->ld_token, r->ld_head);
    const long long lt = r->ldy_token, lh = r->ldy_head;
    const bool apart = (T == 1 || lt >= dim) && (r->heads == 1 || lh >= dim) &&
                       (T == 1 || r->heads == 1 || lt >= lh * (r->heads - 1) + dim ||
                        lh >= lt * (T - 1) + dim);
    REQUIRE(apart, MPQ_ERR_INVALID_ARG, "%s: output rows overlap (ldy_token = %lld, ldy_head = %lld)", what, lt, lh);
    REQUIRE(r->x != r->y || ((T == 1 || lt == r->ld_token) && (r->heads == 1 || lh == r->ld_head)),
            MPQ_ERR_INVALID_ARG, "%s: in place with other strides", what);
    return MPQ_OK;
}

extern "C" mpq_status mpq_rotate(const mpq_rotate_rows *q, const mpq_rotate_rows *k, int type, int T, int dim,
                                 const int *positions, int shift, const uint64_t *turns, int rot,
                                 int neighbours, int norm, float eps, void *stream)
{
    CallRange range_("mpq_rotate");
    clear_error();
    mpq_status st = check_type(type, "type");
    if (st != MPQ_OK) return st;
    REQUIRE(q, MPQ_ERR_INVALID_ARG, "q must be non-NULL");
    REQUIRE(T >= 0, MPQ_ERR_INVALID_ARG, "T = %d must be >= 0", T);
    REQUIRE(T <= 1 << 30, MPQ_ERR_UNSUPPORTED, "T = %d exceeds 2^30", T);
    REQUIRE(dim >= 2 && dim % 2 == 0, MPQ_ERR_INVALID_ARG, "dim = %d must be even, >= 2", dim);
    REQUIRE(dim <= 512, MPQ_ERR_UNSUPPORTED, "dim = %d exceeds 512", dim);
    REQUIRE(rot >= 0 && rot % 2 == 0 && rot <= dim, MPQ_ERR_INVALID_ARG, "rot = %d must be even, 0..dim", rot);
    REQUIRE(neighbours == 0 || neighbours == 1, MPQ_ERR_INVALID_ARG, "neighbours = %d is not 0 or 1", neighbours);
    REQUIRE(norm == 0 || norm == 1, MPQ_ERR_INVALID_ARG, "norm = %d is not 0 or 1", norm);
    REQUIRE(!norm || isfinite(eps), MPQ_ERR_NONFINITE, "eps is not finite");
    REQUIRE(!norm || eps > 0.0f, MPQ_ERR_INVALID_ARG, "eps = %g must be > 0", eps);
    st = check_rows(q, type, T, dim, norm, "q");
    if (st == MPQ_OK && k) st = check_rows(k, type, T, dim, norm, "k");
    if (st != MPQ_OK) return st;
    if (T == 0 || q->heads + (k ? k->heads : 0) == 0) return MPQ_OK;
    REQUIRE(rot == 0 || (positions && turns), MPQ_ERR_INVALID_ARG, "positions and turns must be non-NULL");
    REQUIRE(on(positions, sizeof(int)) && on(turns, sizeof(uint64_t)), MPQ_ERR_INVALID_ARG,
            "positions and turns must be aligned to their elements");
    return launch_rotate(q, k, type, T, dim, positions, shift, turns, rot, neighbours, norm, eps,
                         (cudaStream_t)stream);
}

struct Range {
    const void *p;
    size_t bytes;
};

// Memory that a call reads or writes and memory that it writes, one of them empty or apart.
static bool apart(const Range &a, const Range &b)
{
    const uintptr_t x = (uintptr_t)a.p, y = (uintptr_t)b.p;
    return a.bytes == 0 || b.bytes == 0 || (x <= y ? y - x >= a.bytes : x - y >= b.bytes);
}

// Every output apart from every other and from every input (those that may be one are given once).
template <size_t I, size_t O>
static bool all_apart(const Range (&in)[I], const Range (&out)[O])
{
    for (size_t o = 0; o < O; ++o) {
        for (size_t i = 0; i < I; ++i)
            if (!apart(out[o], in[i])) return false;
        for (size_t i = 0; i < o; ++i)
            if (!apart(out[o], out[i])) return false;
    }
    return true;
}

// What extend and trim ask of a state.
static mpq_status check_pages(int B, int page, int cols, int pages)
{
    REQUIRE(B >= 0, MPQ_ERR_INVALID_ARG, "B = %d must be >= 0", B);
    REQUIRE(B <= MPQ_PAGES_MAX_REQUESTS, MPQ_ERR_UNSUPPORTED, "B = %d exceeds MPQ_PAGES_MAX_REQUESTS = %d", B,
            MPQ_PAGES_MAX_REQUESTS);
    REQUIRE(page >= 1, MPQ_ERR_INVALID_ARG, "page = %d must be >= 1", page);
    REQUIRE(cols >= 0, MPQ_ERR_INVALID_ARG, "cols = %d must be >= 0", cols);
    REQUIRE(page <= 1 << 30 && (long long)page * cols <= (1LL << 30), MPQ_ERR_UNSUPPORTED,
            "page * cols = %lld exceeds 2^30 tokens", (long long)page * cols);
    REQUIRE(pages >= 0, MPQ_ERR_INVALID_ARG, "pages = %d must be >= 0", pages);
    REQUIRE(pages <= 1 << 30, MPQ_ERR_UNSUPPORTED, "pages = %d exceeds 2^30", pages);
    return MPQ_OK;
}

extern "C" mpq_status mpq_pages_extend(const int *add, int B, int page, int cols, const int *lens,
                                       int *new_lens, int *table, const int *pool, int pages, int *count,
                                       int *new_count, int64_t *slots, int *positions, long long N,
                                       int *taken, void *stream)
{
    CallRange range_("mpq_pages_extend");
    clear_error();
    const mpq_status st = check_pages(B, page, cols, pages);
    if (st != MPQ_OK) return st;
    REQUIRE(N >= 0, MPQ_ERR_INVALID_ARG, "N = %lld must be >= 0", N);
    REQUIRE(N <= 1LL << 30, MPQ_ERR_UNSUPPORTED, "N = %lld exceeds 2^30", N);
    REQUIRE(count && new_count, MPQ_ERR_INVALID_ARG, "count and new_count must be non-NULL");
    REQUIRE(B == 0 || (add && lens && new_lens && taken), MPQ_ERR_INVALID_ARG,
            "add, lens, new_lens and taken must be non-NULL");
    REQUIRE(B == 0 || cols == 0 || table, MPQ_ERR_INVALID_ARG, "table must be non-NULL");
    REQUIRE(pages == 0 || pool, MPQ_ERR_INVALID_ARG, "pool must be non-NULL");
    REQUIRE(N == 0 || (slots && positions), MPQ_ERR_INVALID_ARG, "slots and positions must be non-NULL");
    REQUIRE(on(add, 4) && on(lens, 4) && on(new_lens, 4) && on(table, 4) && on(pool, 4) && on(count, 4) &&
                on(new_count, 4) && on(slots, 8) && on(positions, 4) && on(taken, 4),
            MPQ_ERR_INVALID_ARG, "every array must be aligned to its elements");
    const size_t b4 = (size_t)B * 4;
    const Range in[] = {{add, b4}, {pool, (size_t)pages * 4}, {lens, new_lens == lens ? 0 : b4},
                        {count, new_count == count ? 0u : 8u}};
    const Range out[] = {{new_lens, b4}, {new_count, 8}, {table, b4 * cols}, {slots, (size_t)N * 8},
                         {positions, (size_t)N * 4}, {taken, b4}};
    REQUIRE(all_apart(in, out), MPQ_ERR_INVALID_ARG, "an output overlaps another array");
    return launch_pages_extend(add, B, page, cols, lens, new_lens, table, pool, pages, count, new_count, slots,
                               positions, N, taken, (cudaStream_t)stream);
}

extern "C" mpq_status mpq_pages_trim(const int *keep, int B, int page, int cols, const int *lens, int *new_lens,
                                     const int *table, int *pool, int pages, int *count, int *new_count,
                                     void *stream)
{
    CallRange range_("mpq_pages_trim");
    clear_error();
    const mpq_status st = check_pages(B, page, cols, pages);
    if (st != MPQ_OK) return st;
    REQUIRE(count && new_count, MPQ_ERR_INVALID_ARG, "count and new_count must be non-NULL");
    REQUIRE(B == 0 || (keep && lens && new_lens), MPQ_ERR_INVALID_ARG, "keep, lens and new_lens must be non-NULL");
    REQUIRE(B == 0 || cols == 0 || table, MPQ_ERR_INVALID_ARG, "table must be non-NULL");
    REQUIRE(pages == 0 || pool, MPQ_ERR_INVALID_ARG, "pool must be non-NULL");
    REQUIRE(on(keep, 4) && on(lens, 4) && on(new_lens, 4) && on(table, 4) && on(pool, 4) && on(count, 4) &&
                on(new_count, 4),
            MPQ_ERR_INVALID_ARG, "every array must be aligned to its elements");
    const size_t b4 = (size_t)B * 4;
    const Range in[] = {{keep, b4}, {table, b4 * cols}, {lens, new_lens == lens ? 0 : b4},
                        {count, new_count == count ? 0u : 8u}};
    const Range out[] = {{new_lens, b4}, {new_count, 8}, {pool, (size_t)pages * 4}};
    REQUIRE(all_apart(in, out), MPQ_ERR_INVALID_ARG, "an output overlaps another array");
    return launch_pages_trim(keep, B, page, cols, lens, new_lens, table, pool, pages, count, new_count,
                             (cudaStream_t)stream);
}
