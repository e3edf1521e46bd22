// Products of a small head, few and short sums (small32.hip).
//
// What the tiles of product16.h cost before their first and after their last product is more than a small product takes, and so are the
// launches that bring its operands into bf16 planes.  Here a workgroup takes 32 x 32 results, its eight wavefronts share their sums, and operands
// go from memory into the fp32 form of the matrix instruction as they are: 1/16 of the bf16 form's rate, no piece of an fp32 number left out.  Bound by launches and
// the latency of loads: 256 x 512 -> 250 fp32, loss and gradients, 26 us in four kernels of 8, 3, 8 and 8.
#pragma once

#include "real16.h"

namespace dab {

struct Source32 {
    const void* p;
    int64_t ld;                      // elements between rows ([rows][k]) or between k ([k][rows])
    int rows;
    const int64_t* targets;          // k whose target has no loss are zeros (NULL: none)
    int64_t ignore_index;
    int V;
};
struct Small32 {
    Source32 A, B;
    int M, N, K, tiles_n;
    void* C;                         // results of dtype (DAB_F32 or DAB_BF16), rows ldc apart
    int64_t ldc;
    int dtype;
    // softmax: m is a token, n a word; gradients: m is a token, k a word, and rows of tokens without a loss are stored as zeros (NULL: none)
    const int64_t* targets;
    int64_t ignore_index;
    float2* stats;                   // [ceil(N / 32)][M]
    float* target_logit;
    const float* lse;
    const float* g;
};
constexpr int kSmallTile = 32;
// Estimated time of loss and gradients here, in microseconds (very large past the sizes that are taken).
double small32_us(int32_t dtype, int64_t T, int64_t D, int64_t V);
// Statistics of H W^T, P = g (softmax - onehot) as fp32 [T][ldc], and both gradients from it (one launch).
int launch_small_stats(const Small32& g, int32_t dtype, hipStream_t st);
int launch_small_softmax(const Small32& g, int32_t dtype, hipStream_t st);
int launch_small_gradients(const Small32& dw, const Small32& dh, int32_t dtype, hipStream_t st);

}  // namespace dab
