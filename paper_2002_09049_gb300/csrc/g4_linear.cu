// Linear layer of weights in 4-bit integers (mpq_g4_linear, mpq_g4_linear_exact): Y[t][c] = sum_j x_tj w_cj + bias_c,
// w = s (q - z) with s and z by groups of a row.  Which form a call takes; the forms: g4_few.cuh, g4_tiles.cu.
//
// mpq_g4_linear rounds w once to x's type.  (By 2^-9 of it at most in bf16, by 2^-12 of it or 2^-25 in fp16, beside the
// 1/30 of a group's largest that its codes are apart: what that buys is one operand a weight, and one sum over all of K
// in the tensor cores' fp32.)  In bf16 that is as much again as the rounding of 16-bit outputs, so the exact call has no
// rounding of weights at all.
//
// Measured (weights in L2, as they are from call to call; in brackets 20 layers' weights by turns, which come from memory),
// few tokens: 1 x 4,096 x 4,096 (T x C x d) 3.7 us (4.6: a launch, one round of loads, the join; the weights' bytes would
// take 1.3), 5 x 11,008 x 4,096 fp16 with zero points 9.1 (11.2: loads' latency, issue slots 0.45 busy with 15 instructions
// for eight weights, 688 CTAs on places for 456).  The models below were fitted to calls with weights in L2.
#include <math.h>

#include <algorithm>
#include <atomic>

#include "g4_few.cuh"

MPQ_CHECKED_UNIT("g4_linear.cu");

namespace mpq {
namespace {

// Whether this kernel's modelled time (us) is less than the tiles': a start, and what is longer of a warp's tiles one
// after another and of all tiles and CTAs, by the tokens of a CTA (8, 16 or 32).  Some timings, us, this kernel's and
// the tiles': 8 x 4,096 x 4,096 (T x C x d) 4.3, 8.2; 32 x 4,096 x 4,096 7.8, 9.0; 64 x 4,096 x 4,096 14.2, 9.3;
// 16 x 11,008 x 4,096 11.8, 14.9; 24 x 11,008 x 4,096 17.6, 14.9; 64 x 2,048 x 2,048 5.1, 7.4; 16 x 32,768 x 4,096
// 30.8, 27.5; 24 x 512 x 8,192 7.7, 8.4; 96 x 512 x 8,192 11.2, 9.6 (where the model is wrong).
bool few_tokens(int T, const mpq_g4_matrix *L, int terms)
{
    if (T > 128) return false;
    const int c = T <= 8 ? 0 : T <= 16 ? 1 : 2;
    constexpr double one[3] = {0.4, 0.6, 0.75}, tile[3] = {0.27e-3, 0.36e-3, 0.6e-3}, cta[3] = {0.6e-3, 1.5e-3, 2.3e-3};
    const double ctas = (double)L->row_tiles * ((T + 31) / 32);
    const double t = 2.0 + std::max((L->k_tiles + FEW_WARPS - 1) / FEW_WARPS * one[c], ctas * (L->k_tiles * tile[c] + cta[c]));
    return t < g4_tiles_time(T, L->rows, L->d, terms);
}

std::atomic<int> g_form{0};                  // a test's: form + 8 tokens + 4,096 split

}  // namespace

G4Form g4_test_form()
{
    const int f = g_form.load(std::memory_order_relaxed);
    return {f & 7, f >> 3 & 511, f >> 12};
}
void set_g4_test_form(const G4Form &f)
{
    g_form.store(f.form | f.tokens << 3 | f.split << 12, std::memory_order_relaxed);
}

mpq_status launch_g4_linear(const void *X, int x_type, long long ldx, int T, const mpq_g4_matrix *L,
                            const void *W, const float *bias, void *Y, int y_type, long long ldy, int exact,
                            cudaStream_t stream)
{
    const int form = g4_test_form().form;
    if (form ? form != MPQ_G4_FEW : !few_tokens(T, L, exact ? g4_terms(x_type, L) : 1))
        return launch_g4_tiles(X, x_type, ldx, T, L, W, bias, Y, y_type, ldy, exact, stream);
    const G4Args a = {*L, static_cast<const unsigned char *>(W), bias, ldx, ldy, T, y_type};
    return exact ? launch_few_exact(a, X, x_type, Y, stream) : launch_few_tokens<false>(a, X, x_type, Y, stream);
}

}  // namespace mpq
