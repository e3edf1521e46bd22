// Softmax cross entropy over a large vocabulary and its gradient, without the logits.
//
// loss: one product H W^T whose tiles leave only each token's maximum and sum of exponentials over a block of words, and the
// target's logit; a second, small kernel joins the blocks.  gradient: a piece of the vocabulary at a time, the product again, now
// written out as P = g (softmax - onehot), and the two products dW = P^T H (the piece's rows of dW, finished) and dH += P W
// (fp32 until the last piece).  8 T D V flops, two of them for taking the logits twice.  Bound by the matrix cores from a few hundred
// tokens on (8192 x 2048 -> 131072 in 13.4 ms, 1310 TFLOP/s over all four products; the library's own plain
// ones of these sizes reach 1140 to 1380), by reading W three times and writing dW once below
// (one token, 4096 -> 131072, 0.88 ms: 4.9 TB/s).  Small heads: small32.h.
#include "product16.h"
#include "small32.h"

namespace dab {

// The sum of exponentials of a set of words, from its own maximum to `top`.  A set without a maximum keeps its sum, which is 0 if all of
// its logits are minus infinity (exp of the difference would be undefined) and NaN if one of them is: maxima drop NaNs, sums never.
__device__ __forceinline__ float sum_at(float2 s, float top) { return s.x == -__builtin_inff() ? s.y : s.y * expf(s.x - top); }
// Maxima and sums of exponentials of two sets of words as those of both.
__device__ __forceinline__ float2 join_stats(float2 a, float2 b) {
    const float top = fmaxf(a.x, b.x);
    return float2{top, sum_at(a, top) + sum_at(b, top)};
}

// TT tokens a workgroup, 256 / TT threads each, eight pairs on their way at a time: many tokens take whole lines of the pairs, few
// the whole workgroup (one token, 131072 words: 100 us with eight threads).
template <int TT>
__global__ __launch_bounds__(256) void head_join_kernel(const float2* __restrict__ stats, const float* __restrict__ target_logit,
                                                        const int64_t* __restrict__ targets, int64_t ignore, int T, int V, int blocks,
                                                        float* __restrict__ loss, float* __restrict__ lse) {
    constexpr int kParts = 256 / TT;
    __shared__ float2 part[kParts][TT];
    const int tt = threadIdx.x % TT, u = threadIdx.x / TT, t = blockIdx.x * TT + tt;
    const float2 none = {-__builtin_inff(), 0.f};
    float2 all = none;
    if (t < T)
        for (int i = u; i < blocks; i += 8 * kParts) {
            float2 s[8];
            float top = all.x;
#pragma unroll
            for (int k = 0; k < 8; ++k) {
                s[k] = i + k * kParts < blocks ? stats[static_cast<int64_t>(i + k * kParts) * T + t] : none;
                top = fmaxf(top, s[k].x);
            }
            float sum = sum_at(all, top);
#pragma unroll
            for (int k = 0; k < 8; ++k) sum += sum_at(s[k], top);
            all = float2{top, sum};
        }
    part[u][tt] = all;
#pragma unroll
    for (int n = kParts / 2; n > 0; n /= 2) {
        __syncthreads();
        if (u < n) part[u][tt] = all = join_stats(all, part[u + n][tt]);
    }
    if (u != 0 || t >= T) return;
    const int64_t target = targets[t];
    const bool dead = no_loss(target, ignore, V);
    const float l = all.x + logf(all.y);
    lse[t] = dead ? 0.f : l;
    loss[t] = target == ignore ? 0.f : dead ? __builtin_nanf("") : l - target_logit[t];
}
static int launch_head_join(hipStream_t st, const float2* stats, const float* target_logit, const int64_t* targets, int64_t ignore, int T,
                            int V, int blocks, float* loss, float* lse) {
    if (T >= 2048) return launch(head_join_kernel<16>, dim3(ceil_div(T, 16)), dim3(256), 0, st, stats, target_logit, targets, ignore, T, V, blocks, loss, lse);
    return launch(head_join_kernel<4>, dim3(ceil_div(T, 4)), dim3(256), 0, st, stats, target_logit, targets, ignore, T, V, blocks, loss, lse);
}

// dH from the products with P's two planes, n entries of D a token.
__global__ __launch_bounds__(256) void head_unstack_kernel(const float* __restrict__ acc, int n, bf16* __restrict__ dH, int D,
                                                           const int64_t* __restrict__ targets, int64_t ignore, int V) {
    const int i = blockIdx.x * 256 + threadIdx.x;
    if (i < n) dH[i] = static_cast<bf16>(no_loss(targets[i / D], ignore, V) ? 0.f : acc[i] + acc[n + i]);
}

struct HeadPlan {
    bool small;                      // small32.h
    bool wide;                       // fp32 operands as they are
    int P;                           // planes
    int n_seg;
    int prob_planes;                 // planes of P
    bool stacked;                    // bf16, few tokens: P's two planes as twice the tokens in dH, and as two pairs in dW
    bool factored;                   // bf16, many tokens: the weights' factor (product16.h)
    bool h_direct, w_direct;
    bool tail;                       // rows that are read where they are and are no whole pieces of 16 bytes
    int64_t ldh, ldw;
    int piece, n_pieces;             // words of a piece
    int64_t ldp;
    Plan16 logits, dh, dw;           // of a piece (the last one may be smaller)
    size_t h_at, w_at, factor_at, stats_at, target_at, p_at, acc_at, part_at, part_bytes, bytes;
};

static bool head_sizes(int32_t T, int32_t D, int32_t V, int32_t dtype, int64_t ldh, int64_t ldw) {
    return (dtype == DAB_BF16 || dtype == DAB_F32) && ldh < (1 << 22) && ldw < (1 << 22) && T < (1 << 30) && V < (1 << 30) &&
           ceil_div64(T, 128) * ceil_div64(V, 128) < INT32_MAX / 64 && ceil_div64(T, 128) * ceil_div64(D, 128) < INT32_MAX / 1024;
}

// How the products of a head are done.  Measured, loss and gradients (tokens x width x words), small kernels, fp32 operands as they are, planes:
// fp32 256 x 512 x 250 27 us, 65, 95; 299 x 1504 x 628 75, 150, 194; 64 x 2048 x 64000 -, 632, 1734; 256 x 1024 x 16000 -, 281, 283;
// 1024 x 1024 x 16000 -, 1017, 664; 2048 x 1024 x 32000 -, 3931, 2495.  bf16, small kernels and tiles: 256 x 512 x 250 29 us, 42; 1 x 2083 x 256
// 54, 71; 75 x 931 x 901 51, 64; 51 x 1272 x 2602 130, 59; 1050 x 464 x 1060 113, 61.
enum class Route { kSmall, kWide, kPlanes };
static Route head_route(int32_t dtype, int64_t T, int64_t D, int64_t V) {
    const int t = static_cast<int>(T), d = static_cast<int>(D), v = static_cast<int>(V);
    const double small = small32_us(dtype, T, D, V);
    if (dtype == DAB_BF16) {
        const int planes = T <= 128 ? 2 : 1;                 // of P (head_plan)
        const double sums = 2 * plan16_logits(t, v, d, 1).us + plan16(v, d, t, planes, kAnyShares16).us + plan16(planes * t, d, v, 1, kAnyShares16).us;
        // (the estimates are those of a full chip, where steps take longer; H is copied)
        return small <= 22.5 + 0.78 * sums + 12e-6 * static_cast<double>(T * D) ? Route::kSmall : Route::kPlanes;
    }
    const double wide = 15.0 + 2 * plan32_logits(t, v, d).us + plan32(v, d, t, kAnyShares16).us + plan32(t, d, v, kAnyShares16).us;
    // (both calls write and read the planes of H and W)
    const double planes = 20.0 + 2 * plan16_logits(t, v, d, 6).us + plan16(v, d, t, 6, kAnyShares16).us + plan16(t, d, v, 6, kAnyShares16).us +
                          2.0 * static_cast<double>((T + V) * D) * 10 / 4e6;
    return small <= wide && small <= planes ? Route::kSmall : wide <= planes ? Route::kWide : Route::kPlanes;
}

// Pieces of up to 256 MB of P (`bytes` an entry), which is about what the memory-side cache holds, but no fewer than 1024 words, of equal size; rows of P stay within
// the offsets of the product's copies.
static void head_pieces(HeadPlan& p, int32_t T, int32_t D, int32_t V, int bytes) {
    int64_t words = (int64_t{256} << 20) / (static_cast<int64_t>(bytes) * T) / 1024 * 1024;
    if (words < 1024) words = 1024;
    if (words > (1 << 20)) words = 1 << 20;
    if (words > V) words = V;
    p.n_pieces = static_cast<int>(ceil_div64(V, words));
    p.piece = static_cast<int>(round_up(ceil_div64(V, p.n_pieces), 256));
    p.n_pieces = ceil_div(V, p.piece);
    p.ldp = p.piece;
}

static HeadPlan head_plan(int32_t T, int32_t D, int32_t V, int32_t dtype, int64_t ldh, int64_t ldw, bool gradient) {
    HeadPlan p{};
    size_t at = 0;
    auto room = [&at](int64_t bytes) {
        const size_t here = at;
        at += static_cast<size_t>(round_up(bytes, 256));
        return here;
    };
    const Route route = head_route(dtype, T, D, V);
    p.small = route == Route::kSmall;
    if (p.small) {
        if (gradient) {
            p.ldp = round_up(V, 4);
            p.p_at = room(T * p.ldp * 4);
        } else {
            p.stats_at = room(ceil_div64(V, kSmallTile) * T * 8);
            p.target_at = room(static_cast<int64_t>(T) * 4);
        }
        p.bytes = at;
        return p;
    }
    p.wide = route == Route::kWide;
    if (p.wide) {
        p.P = p.n_seg = p.prob_planes = 1;
        p.h_direct = !gradient, p.w_direct = true, p.tail = D % 4 != 0;
        p.ldh = p.h_direct ? ldh : round_up(D, 4), p.ldw = ldw;
        p.h_at = p.h_direct ? 0 : room(T * p.ldh * 4);
        if (!gradient) {
            p.logits = plan32_logits(T, V, D);
            p.stats_at = room((ceil_div64(V, stats_words16(p.logits)) + 8) * T * 8);
            p.target_at = room(static_cast<int64_t>(T) * 4);
        } else {
            head_pieces(p, T, D, V, 4);
            p.logits = plan32_logits(T, p.piece, D);
            p.dh = plan32(T, D, p.piece, kAnyShares16), p.dw = plan32(p.piece, D, T, kAnyShares16);
            p.p_at = room(static_cast<int64_t>(T) * p.ldp * 4);
            p.acc_at = room(p.n_pieces > 1 ? static_cast<int64_t>(T) * D * 4 : 0);
            p.part_bytes = p.dh.part_bytes > p.dw.part_bytes ? p.dh.part_bytes : p.dw.part_bytes;
            p.part_at = room(static_cast<int64_t>(p.part_bytes));
        }
        p.bytes = at;
        return p;
    }
    p.P = dtype_pieces(dtype);
    p.n_seg = p.P == 1 ? 1 : 6;
    // Rows of whole words are read where they are, though pieces of 16 bytes that cross lines cost the products more than aligned ones: loss
    // and gradients, copied | as they are: 100 x 1002 x 50000 249 | 157 us, 500 x 1002 x 50000 368 | 288, 2000 x 2050 x 32768 1183 | 1081,
    // 4000 x 1022 x 50000 1644 | 1652, 8000 x 1022 x 50000 3173 | 3287.
    auto direct = [&](int64_t ld) { return dtype == DAB_BF16 && ((D % 8 == 0 && ld % 8 == 0) || (D % 2 == 0 && ld % 2 == 0 && T <= 4096)); };
    p.w_direct = direct(ldw);
    // (a gradient reads H with the rows of ignored tokens cleared, whatever they hold)
    p.h_direct = !gradient && direct(ldh);
    p.tail = D % 8 != 0 && (p.w_direct || p.h_direct);
    p.ldh = p.h_direct ? ldh : round_up(D, 8);
    p.ldw = p.w_direct ? ldw : round_up(D, 8);
    p.h_at = p.h_direct ? 0 : room(static_cast<int64_t>(p.P) * T * p.ldh * 2);
    p.w_at = p.w_direct ? 0 : room(static_cast<int64_t>(p.P) * V * p.ldw * 2);
    if (!gradient) {
        p.logits = plan16_logits(T, V, D, p.n_seg);
        const int words = stats_words16(p.logits);
        p.stats_at = room((ceil_div64(V, words) + 8) * T * 8);
        p.target_at = room(static_cast<int64_t>(T) * 4);
    } else {
        // With many tokens the roundings of P to bf16 average out beside those of dH and dW; with few a row's largest entry is most of it, and
        // one rounding of that shows (relative error of one token's dH 0.4 % instead of 0.17 %).  Its second eight bits cost nothing there: the
        // products are bound by reading W and writing dW.
        p.stacked = p.P == 1 && T <= 128;
        // Of many tokens the weights are rounded with P, and one weight for all of them, a mean's 1 / N, is no bf16 number: the targets' terms,
        // -g but for little, would all be off by the same, up to 2^-8 of them.  So P is made with g over the significand of one of
        // them, powers of two then (but for a last bit of fp32), and dH and dW are multiplied by it in fp32.
        p.factored = p.P == 1 && !p.stacked;
        p.factor_at = p.factored ? room(8) : 0;
        p.prob_planes = p.stacked ? 2 : p.P;
        head_pieces(p, T, D, V, 2 * p.prob_planes);
        p.logits = plan16_logits(T, p.piece, D, p.n_seg);
        p.dh = plan16(p.stacked ? 2 * T : T, D, p.piece, p.n_seg, kAnyShares16);
        p.dw = plan16(p.piece, D, T, p.stacked ? 2 : p.n_seg, kAnyShares16);
        p.p_at = room(static_cast<int64_t>(p.prob_planes) * T * p.ldp * 2);
        p.acc_at = room(p.stacked ? int64_t{2} * T * D * 4 : p.n_pieces > 1 ? static_cast<int64_t>(T) * D * 4 : 0);
        p.part_bytes = p.dh.part_bytes > p.dw.part_bytes ? p.dh.part_bytes : p.dw.part_bytes;
        p.part_at = room(static_cast<int64_t>(p.part_bytes));
    }
    p.bytes = at;
    return p;
}

static int head_check(const void* H, int64_t ldh, const void* W, int64_t ldw, int32_t dtype, const void* targets, int32_t T, int32_t D,
                      int32_t V) {
    if (!H || !W || !targets) return DAB_ERR_NULL;
    if (T < 1 || D < 1 || V < 1 || ldh < D || ldw < D) return DAB_ERR_SHAPE;
    if (!head_sizes(T, D, V, dtype, ldh, ldw)) return DAB_ERR_UNSUPPORTED;
    if (misaligned(H, 16) || misaligned(W, 16) || misaligned(targets, 8)) return DAB_ERR_ALIGN;
    return DAB_OK;
}

static void head_segments(Product16& g, int n_seg) {
    // pairs of pieces in order of size; what is left out is below 2^-24 of a term
    g.n_seg = n_seg;
    if (n_seg > 1) g.seg_a = 0x201100, g.seg_b = 0x021010;
}

// The logits of small sizes: operands as they are.
static Small32 head_logits32(const void* H, int64_t ldh, const void* W, int64_t ldw, int32_t dtype, const int64_t* targets, int64_t ignore,
                             int T, int D, int V) {
    Small32 g{};
    g.A = {H, ldh, T, nullptr, 0, 0};
    g.B = {W, ldw, V, nullptr, 0, 0};
    g.M = T, g.N = V, g.K = D, g.tiles_n = ceil_div(V, kSmallTile);
    g.targets = targets, g.ignore_index = ignore;
    return g;
}

// The operands as bf16 planes, in the workspace where they are not already.
static int head_operands(const HeadPlan& p, const void* H, int64_t ldh, const void* W, int64_t ldw, int32_t dtype,
                         const int64_t* targets, int64_t ignore, int T, int D, int V, char* ws, hipStream_t st, Operand16* h, Operand16* w,
                         const float* g = nullptr) {
    *h = {H, p.ldh, static_cast<int64_t>(T) * p.ldh};
    *w = {W, p.ldw, static_cast<int64_t>(V) * p.ldw};
    if (p.wide) {
        if (!p.h_direct) {
            float* out = reinterpret_cast<float*>(ws + p.h_at);
            if (int rc = launch_rows32(static_cast<const float*>(H), T, D, ldh, targets, ignore, V, out, p.ldh, st)) return rc;
            h->p = out;
        }
        return DAB_OK;
    }
    if (!p.h_direct) {
        bf16* out = reinterpret_cast<bf16*>(ws + p.h_at);
        float* factor = g && p.factored ? reinterpret_cast<float*>(ws + p.factor_at) : nullptr;
        if (int rc = launch_planes16(H, dtype, T, D, ldh, targets, ignore, V, out, p.ldh, st, g, factor)) return rc;
        h->p = out;
    }
    if (!p.w_direct) {
        bf16* out = reinterpret_cast<bf16*>(ws + p.w_at);
        if (int rc = launch_planes16(W, dtype, V, D, ldw, nullptr, 0, 0, out, p.ldw, st)) return rc;
        w->p = out;
    }
    return DAB_OK;
}

}  // namespace dab

extern "C" size_t dab_head_loss_workspace_bytes(int32_t T, int32_t D, int32_t V, int32_t dtype, int64_t ldh, int64_t ldw) {
    using namespace dab;
    if (T < 1 || D < 1 || V < 1 || ldh < D || ldw < D || !head_sizes(T, D, V, dtype, ldh, ldw)) return 0;
    return head_plan(T, D, V, dtype, ldh, ldw, false).bytes;
}

extern "C" size_t dab_head_loss_gradient_workspace_bytes(int32_t T, int32_t D, int32_t V, int32_t dtype, int64_t ldh, int64_t ldw) {
    using namespace dab;
    if (T < 1 || D < 1 || V < 1 || ldh < D || ldw < D || !head_sizes(T, D, V, dtype, ldh, ldw)) return 0;
    return head_plan(T, D, V, dtype, ldh, ldw, true).bytes;
}

extern "C" int dab_head_loss(const void* H, int64_t ldh, const void* W, int64_t ldw, int32_t dtype, const int64_t* targets,
                             int64_t ignore_index, int32_t T, int32_t D, int32_t V, float* loss, float* lse, void* ws, size_t ws_bytes,
                             void* stream) {
    using namespace dab;
    if (!loss || !lse) return DAB_ERR_NULL;
    if (int rc = head_check(H, ldh, W, ldw, dtype, targets, T, D, V)) return rc;
    if (misaligned(loss, 4) || misaligned(lse, 4)) return DAB_ERR_ALIGN;
    const HeadPlan p = head_plan(T, D, V, dtype, ldh, ldw, false);
    if (!ws || ws_bytes < p.bytes || misaligned(ws, 256)) return DAB_ERR_WORKSPACE;
    if (int rc = ensure_device_ready()) return rc;
    const auto st = static_cast<hipStream_t>(stream);
    char* base = static_cast<char*>(ws);
    float2* stats = reinterpret_cast<float2*>(base + p.stats_at);
    float* target_logit = reinterpret_cast<float*>(base + p.target_at);
    if (p.small) {
        Small32 g = head_logits32(H, ldh, W, ldw, dtype, targets, ignore_index, T, D, V);
        g.stats = stats, g.target_logit = target_logit;
        if (int rc = launch_small_stats(g, dtype, st)) return rc;
        return launch_head_join(st, stats, target_logit, targets, ignore_index, T, V, ceil_div(V, kSmallTile), loss, lse);
    }
    Product16 g{};
    if (int rc = head_operands(p, H, ldh, W, ldw, dtype, targets, ignore_index, T, D, V, base, st, &g.A, &g.B)) return rc;
    g.M = T, g.N = V, g.K = D, g.V = V, g.tail = p.tail;
    head_segments(g, p.n_seg);
    g.targets = targets, g.ignore_index = ignore_index;
    g.stats = stats, g.target_logit = target_logit;
    if (int rc = launch16(kEpiStats, false, false, g, p.logits, 0, st)) return rc;
    const int blocks = ceil_div(V, stats_words16(p.logits));
    return launch_head_join(st, stats, target_logit, targets, ignore_index, T, V, blocks, loss, lse);
}

extern "C" int dab_head_loss_gradient(const void* H, int64_t ldh, const void* W, int64_t ldw, int32_t dtype, const int64_t* targets,
                                      int64_t ignore_index, const float* lse, const float* grad, int32_t T, int32_t D, int32_t V,
                                      void* dH, void* dW, void* ws, size_t ws_bytes, void* stream) {
    using namespace dab;
    if (!lse || !dH || !dW) return DAB_ERR_NULL;
    if (int rc = head_check(H, ldh, W, ldw, dtype, targets, T, D, V)) return rc;
    if (misaligned(lse, 4) || misaligned(grad, 4) || misaligned(dH, 16) || misaligned(dW, 16)) return DAB_ERR_ALIGN;
    const HeadPlan p = head_plan(T, D, V, dtype, ldh, ldw, true);
    if (!ws || ws_bytes < p.bytes || misaligned(ws, 256)) return DAB_ERR_WORKSPACE;
    if (int rc = ensure_device_ready()) return rc;
    const auto st = static_cast<hipStream_t>(stream);
    char* base = static_cast<char*>(ws);
    if (p.small) {
        float* P = reinterpret_cast<float*>(base + p.p_at);
        Small32 g = head_logits32(H, ldh, W, ldw, dtype, targets, ignore_index, T, D, V);
        g.C = P, g.ldc = p.ldp, g.lse = lse, g.g = grad;
        if (int rc = launch_small_softmax(g, dtype, st)) return rc;
        Small32 q{}, s{};
        q.A = {P, p.ldp, V, nullptr, 0, 0}, q.B = {H, ldh, D, targets, ignore_index, V};
        q.M = V, q.N = D, q.K = T, q.tiles_n = ceil_div(D, kSmallTile), q.C = dW, q.ldc = D, q.dtype = dtype;
        s.A = {P, p.ldp, T, nullptr, 0, 0}, s.B = {W, ldw, D, nullptr, 0, 0};
        s.M = T, s.N = D, s.K = V, s.tiles_n = q.tiles_n, s.C = dH, s.ldc = D, s.dtype = dtype;
        s.targets = targets, s.ignore_index = ignore_index;
        return launch_small_gradients(q, s, dtype, st);
    }
    Operand16 h, w;
    if (int rc = head_operands(p, H, ldh, W, ldw, dtype, targets, ignore_index, T, D, V, base, st, &h, &w, grad)) return rc;
    const float* factor = grad && p.factored ? reinterpret_cast<const float*>(base + p.factor_at) : nullptr;
    void* P = base + p.p_at;
    float* acc = reinterpret_cast<float*>(base + p.acc_at);
    const Operand16 probs = {P, p.ldp, static_cast<int64_t>(T) * p.ldp};
    const int64_t size = dtype_bytes(dtype);
    const int64_t w_size = p.wide ? 4 : 2;
    // (the last, smaller piece has its own plans; their shares have the room that the others' take)
    auto plan = [&](int M, int N, int K, int n_seg) { return p.wide ? plan32(M, N, K, p.part_bytes) : plan16(M, N, K, n_seg, p.part_bytes); };
    for (int i = 0; i < p.n_pieces; ++i) {
        const int v0 = i * p.piece, words = V - v0 < p.piece ? V - v0 : p.piece;
        const Operand16 wp = {static_cast<const char*>(w.p) + v0 * w.ld * w_size, w.ld, w.plane};
        // P of this piece; its columns past the last word are zeros
        Product16 g{};
        head_segments(g, p.n_seg);
        g.A = h, g.B = wp, g.M = T, g.N = words, g.K = D, g.tail = p.tail;
        g.targets = targets, g.ignore_index = ignore_index, g.n0 = v0, g.V = V, g.lse = lse, g.g = grad, g.factor = factor;
        g.P = P, g.ldp = p.ldp, g.p_plane = probs.plane, g.p_planes = p.prob_planes;
        if (int rc = launch16(kEpiSoftmax, false, false, g, p.wide ? plan32_logits(T, words, D) : plan16_logits(T, words, D, p.n_seg), 0, st)) return rc;
        // the piece's rows of dW
        Product16 q{};
        head_segments(q, p.n_seg);
        if (p.stacked) q.n_seg = 2, q.seg_a = 0x10, q.seg_b = 0;
        q.A = probs, q.B = h, q.M = words, q.N = D, q.K = T;
        q.C = static_cast<char*>(dW) + v0 * static_cast<int64_t>(D) * size, q.ldc = D, q.out_bf16 = dtype == DAB_BF16;
        q.factor = factor;
        q.part = reinterpret_cast<float*>(base + p.part_at);
        if (int rc = launch16(kEpiStore, true, true, q, plan(words, D, T, q.n_seg), p.part_bytes, st)) return rc;
        // its share of dH
        const bool last = i + 1 == p.n_pieces && !p.stacked;
        Product16 s{};
        head_segments(s, p.n_seg);
        s.A = probs, s.B = wp, s.M = p.stacked ? 2 * T : T, s.N = D, s.K = words;
        s.add = i ? acc : nullptr;
        s.C = last ? dH : acc, s.ldc = D, s.out_bf16 = last && dtype == DAB_BF16;
        if (last) s.targets = targets, s.ignore_index = ignore_index, s.V = V, s.factor = factor;
        s.part = q.part;
        if (int rc = launch16(kEpiStore, false, true, s, plan(s.M, D, words, p.n_seg), p.part_bytes, st)) return rc;
    }
    if (!p.stacked) return DAB_OK;
    return launch(head_unstack_kernel, dim3(ceil_div(T * D, 256)), dim3(256), 0, st, acc, T * D, static_cast<bf16*>(dH), D, targets, ignore_index, V);
}
