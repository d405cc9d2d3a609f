// A few tokens through a linear layer with the values of 4-bit integer weights themselves (mpq_g4_linear_exact).
//
// The operands are the whole numbers q - z, and a group's sum of x (q - z) takes its scale in fp32: four FMAs a group and
// eight tokens in place of a multiplication for each pair of weights.
//
// Measured, beside the rounded values' kernel: 1 x 4,096 x 4,096 (T x C x d) bf16 3.5 us (3.7), 5 x 11,008 x 4,096 fp16 with
// zero points 7.3 (9.1: no product a pair of weights, and no second kind of scales), 16 x 11,008 x 4,096 bf16 12.3 (11.6: a
// group's sums of 16 tokens are as many FMAs as its weights are products).  With 20 layers' weights by turns, which come
// from memory, 4.4, 8.6 and 14.4.
#include "g4_few.cuh"

MPQ_CHECKED_UNIT("g4_linear_exact.cu");

namespace mpq {

mpq_status launch_few_exact(const G4Args &a, const void *X, int x_type, void *Y, cudaStream_t stream)
{
    return launch_few_tokens<true>(a, X, x_type, Y, stream);
}

}  // namespace mpq
