// Dense products on the matrix cores, for the training side of the real-valued layers:
//     C[m][n] = sum over pieces (a, b) and k of A_a[m][k] B_b[n][k],   fp32 accumulation.
// Either operand may be held with k contiguous ([rows][k], rows = m or n) or with its rows contiguous ([k][rows]): the second form is
// transposed on the way out of LDS (ds_read_b64_tr_b16), so that no operand is ever transposed in memory.  Operands are bf16, or fp32 in one
// of two forms: several bf16 planes whose sum they are, the product running over a list of pairs of planes (six for all of 24 bits), or as
// they are on the fp32 matrix instruction.  The first reaches 190 TFLOP/s of fp32 products, 1.4 times the second, but has the planes to write
// and read: it is for many rows.
//
// A workgroup of WM x WN wavefronts owns a TM x TN tile of C.  A step is 128 bytes of k: both operands' tiles go from memory straight into
// LDS (16 bytes a lane) while the steps before are multiplied; two buffers, one barrier a step (four buffers for a few tiles, which would wait
// for each step's copies).  The product is taken with B as the matrix core's left operand: register r of a lane is then column
// n = 4 (lane / 16) + r of row m = lane % 16, so that softmax sums over n stay in a lane but for two exchanges.
//
// Bound by the matrix cores at the clock that their power leaves (1.7 - 2.0 GHz in long products): 256 x 256 tiles of eight wavefronts, 64 x 128
// each, read 192 KB of LDS a step against 2048 clocks of products, 75 % of its bandwidth.  Measured: 16384 x 4096 -> 4096 from two
// operands in the form [k][rows] 410 us, 1340 TFLOP/s; logits of 8192 x 2048 -> 131072 with their softmax statistics 3.3 ms, 1330; a step that
// waited for its own LDS reads, its copies in a burst behind the barrier and addresses from vector registers had each cost 10 - 15 %.
#pragma once

#include "real16.h"

namespace dab {

struct Operand16 {
    const void* p;                   // bf16, or fp32 where the plan says so
    int64_t ld;                      // elements between rows ([rows][k]) or between k ([k][rows]), whole words of 32 bits
    int64_t plane;                   // elements between the planes
};

enum { kEpiStats = 0, kEpiSoftmax = 1, kEpiStore = 2 };

constexpr int kStepK = 64;           // k of a step of bf16 operands

struct Product16 {
    Operand16 A, B;
    int M, N, K;
    int tail;                        // kEpiStats, kEpiSoftmax: rows may hold anything behind K, not zeros up to 16 bytes
    int n_seg;                       // pairs of planes
    uint32_t seg_a, seg_b;           // plane of each pair, four bits a pair
    int tiles_m, tiles_n;
    int steps;                       // steps of a sum: n_seg * ceil(K / 64), fp32 ceil(K / 32)
    int whole, whole_xcd;            // tiles whose sum one workgroup takes, and how many of them an XCD does
    int rest, rest_xcd;              // the last tiles, in `shares` shares each, and shares an XCD takes
    int shares, share_steps;
    // kEpiStore: C (out_bf16 or fp32, rows ldc apart)
    void* C;
    int64_t ldc;
    int out_bf16;
    const float* add;                // fp32 [M][N] added to the sum, or NULL
                                     // (and `targets`, or NULL: rows m of tokens without a loss are stored as zeros)
    const float* factor;             // [2] what is stored is multiplied by the first, in P the weights by the second; or NULL
    float* part;                     // [rest][shares][tile] sums of the shares, in the order of the accumulators
    // kEpiStats, kEpiSoftmax: m is a token, n a word of the vocabulary, n0 the first word of this piece
    const int64_t* targets;
    int64_t ignore_index;
    int n0, V;
    float2* stats;                   // [ceil(N / stats_words16())][M] maximum and sum of exponentials
    float* target_logit;             // [M]
    const float* lse;
    const float* g;
    void* P;                         // bf16 [planes][M][ldp], or fp32 [M][ldp]
    int64_t ldp, p_plane;
    int p_planes;
};

// Tile of a product and how its sums are shared out (product16.hip).  kSmall 128 x 128, two workgroups on a compute unit; kDeep the same, one, four
// steps in LDS; kBig 256 x 256; of fp32 operands kF32 64 x 128, three workgroups, and kFew 32 x 128 for up to 32 rows and for few tiles.
enum class Tiles16 { kSmall, kDeep, kBig, kF32, kFew };
struct Plan16 {
    Tiles16 tiles;
    int steps, whole, rest, shares, share_steps;
    size_t part_bytes;
    double us;                       // estimated time
};
constexpr size_t kAnyShares16 = ~size_t{0};
// Of a product whose result is stored; share_bytes: room for the sums of shares (0: every sum whole in one workgroup).
Plan16 plan16(int M, int N, int K, int n_seg, size_t share_bytes);
// Of logits: a softmax needs its sums whole, and its kernels take the last round's big tiles in parts (kParts16) instead.
Plan16 plan16_logits(int M, int N, int K, int n_seg);
// The same two for fp32 operands.
Plan16 plan32(int M, int N, int K, size_t share_bytes);
inline Plan16 plan32_logits(int M, int N, int K) { return plan32(M, N, K, 0); }
// part_bytes: room at g.part; DAB_ERR_UNSUPPORTED if the plan's shares do not fit it.
int launch16(int epi, bool arc, bool brc, Product16 g, const Plan16& pl, size_t part_bytes, hipStream_t st);
int stats_words16(const Plan16& pl);           // words of the vocabulary per pair of the stats
int init_product16();
// fp32 rows ldp apart (a multiple of 4, zeros behind the last element), those of tokens without a loss cleared (targets may be NULL)
int launch_rows32(const float* X, int rows, int cols, int64_t ld, const int64_t* targets, int64_t ignore, int V, float* out, int64_t ldp,
                  hipStream_t st);
// bf16 planes [P][rows][ldp] of X [rows][cols], zeros up to ldp; rows whose target has no loss are zeros (targets may be NULL).  And, with
// `factor`, the significand (1 .. 2) of the first of the weights g of tokens with a loss that is no 0 and finite (1 if none is),
// and 1 over it.
int launch_planes16(const void* X, int32_t dtype, int rows, int cols, int64_t ld, const int64_t* targets, int64_t ignore, int V,
                    bf16* out, int64_t ldp, hipStream_t st, const float* g = nullptr, float* factor = nullptr);

}  // namespace dab
