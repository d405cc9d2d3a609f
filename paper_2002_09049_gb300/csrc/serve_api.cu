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
