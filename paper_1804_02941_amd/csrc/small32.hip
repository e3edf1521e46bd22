// Products of few and short sums (small32.h).
#include "small32.h"

namespace dab {

constexpr int kSmallWaves = 8;

// Four k of a row as fp32, zeros past K.
template <typename T, bool RC>
__device__ __forceinline__ v4f four(const Source32& o, int row, int k, int K) {
    v4f v = v4f{0.f, 0.f, 0.f, 0.f};
    if constexpr (RC) {
#pragma unroll
        for (int c = 0; c < 4; ++c)
            if (k + c < K && !(o.targets && no_loss(o.targets[k + c], o.ignore_index, o.V)))
                v[c] = static_cast<float>(static_cast<const T*>(o.p)[(k + c) * o.ld + row]);
    } else {
        const T* from = static_cast<const T*>(o.p) + row * o.ld + k;
        if (k + 4 <= K) {
            typedef T v4t __attribute__((ext_vector_type(4)));
            const v4t got = *reinterpret_cast<const typename Unaligned<T, 4>::type*>(from);
            v = __builtin_convertvector(got, v4f);
        } else {
#pragma unroll
            for (int c = 0; c < 4; ++c)
                if (k + c < K) v[c] = static_cast<float>(from[c]);
        }
    }
    return v;
}

// The 32 x 32 results of a tile: thread t gets those of row t / 16 and columns 2 (t % 16), + 1.
template <typename TA, bool ARC, typename TB, bool BRC>
__device__ __forceinline__ float2 small_tile(const Small32& g, int m0, int n0, float (&sums)[kSmallWaves][32 * 34]) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int ra[2] = {min(m0 + (lane & 15), g.M - 1), min(m0 + 16 + (lane & 15), g.M - 1)};
    const int rb[2] = {min(n0 + (lane & 15), g.N - 1), min(n0 + 16 + (lane & 15), g.N - 1)};
    v4f acc[2][2] = {};
    // 16 k a turn, lane l four of them from 4 (l / 16) on; the next turn's are on their way
    v4f a[2], b[2];
    int k = wave * 16 + (lane >> 4) * 4;
#pragma unroll
    for (int u = 0; u < 2; ++u) a[u] = four<TA, ARC>(g.A, ra[u], k, g.K), b[u] = four<TB, BRC>(g.B, rb[u], k, g.K);
    for (int turn = wave * 16; turn < g.K; turn += kSmallWaves * 16) {
        v4f na[2], nb[2];
        k += kSmallWaves * 16;
#pragma unroll
        for (int u = 0; u < 2; ++u) na[u] = four<TA, ARC>(g.A, ra[u], k, g.K), nb[u] = four<TB, BRC>(g.B, rb[u], k, g.K);
#pragma unroll
        for (int c = 0; c < 4; ++c)
#pragma unroll
            for (int i = 0; i < 2; ++i)
#pragma unroll
                for (int j = 0; j < 2; ++j) acc[i][j] = __builtin_amdgcn_mfma_f32_16x16x4f32(b[i][c], a[j][c], acc[i][j], 0, 0, 0);
#pragma unroll
        for (int u = 0; u < 2; ++u) a[u] = na[u], b[u] = nb[u];
    }
#pragma unroll
    for (int i = 0; i < 2; ++i)
#pragma unroll
        for (int j = 0; j < 2; ++j)
#pragma unroll
            for (int r = 0; r < 4; ++r) sums[wave][(j * 16 + (lane & 15)) * 34 + i * 16 + (lane >> 4) * 4 + r] = acc[i][j][r];
    __syncthreads();
    float2 v = {0.f, 0.f};
    const int at = (threadIdx.x >> 4) * 34 + (threadIdx.x & 15) * 2;
#pragma unroll
    for (int w = 0; w < kSmallWaves; ++w) v.x += sums[w][at], v.y += sums[w][at + 1];
    return v;
}

template <typename T>
__global__ __launch_bounds__(64 * kSmallWaves) void small_stats_kernel(Small32 g) {
    __shared__ float sums[kSmallWaves][32 * 34];
    const int tm = blockIdx.x / g.tiles_n, tn = blockIdx.x - tm * g.tiles_n;
    const float2 v = small_tile<T, false, T, false>(g, tm * 32, tn * 32, sums);
    const int m = tm * 32 + (threadIdx.x >> 4), n = tn * 32 + (threadIdx.x & 15) * 2;
    const float x = n < g.N ? v.x : -__builtin_inff(), y = n + 1 < g.N ? v.y : -__builtin_inff();
    float big = fmaxf(x, y);
#pragma unroll
    for (int d = 1; d < 16; d *= 2) big = fmaxf(big, __shfl_xor(big, d));
    const float at = big == -__builtin_inff() ? 0.f : big;
    float sum = __expf(x - at) + __expf(y - at);
#pragma unroll
    for (int d = 1; d < 16; d *= 2) sum += __shfl_xor(sum, d);
    if (m >= g.M) return;
    if ((threadIdx.x & 15) == 0) g.stats[static_cast<int64_t>(tn) * g.M + m] = float2{big, sum};
    const int64_t t = g.targets[m];
    if (n < g.N && t == n) g.target_logit[m] = v.x;
    if (n + 1 < g.N && t == n + 1) g.target_logit[m] = v.y;
}

template <typename T>
__global__ __launch_bounds__(64 * kSmallWaves) void small_softmax_kernel(Small32 g) {
    __shared__ float sums[kSmallWaves][32 * 34];
    const int tm = blockIdx.x / g.tiles_n, tn = blockIdx.x - tm * g.tiles_n;
    const float2 v = small_tile<T, false, T, false>(g, tm * 32, tn * 32, sums);
    const int m = tm * 32 + (threadIdx.x >> 4), n = tn * 32 + (threadIdx.x & 15) * 2;
    if (m >= g.M || n >= g.N) return;
    const int64_t t = g.targets[m];
    const bool dead = no_loss(t, g.ignore_index, g.N);
    const float lse = dead ? 0.f : g.lse[m], w = dead ? 0.f : g.g ? g.g[m] : 1.f;
    float* to = static_cast<float*>(g.C) + m * g.ldc + n;
    to[0] = dead ? 0.f : w * (__expf(v.x - lse) - (t == n ? 1.f : 0.f));
    if (n + 1 < g.N) to[1] = dead ? 0.f : w * (__expf(v.y - lse) - (t == n + 1 ? 1.f : 0.f));
}

__device__ __forceinline__ void small_store(const Small32& g, int m0, int n0, float2 v) {
    const int m = m0 + (threadIdx.x >> 4), n = n0 + (threadIdx.x & 15) * 2;
    if (m >= g.M) return;
    // (not its product: P's zeros times a word that is no number are not 0)
    if (g.targets && no_loss(g.targets[m], g.ignore_index, g.K)) v = float2{0.f, 0.f};
#pragma unroll
    for (int u = 0; u < 2; ++u) {
        if (n + u >= g.N) return;
        const float y = u ? v.y : v.x;
        if (g.dtype == DAB_BF16) static_cast<bf16*>(g.C)[m * g.ldc + n + u] = static_cast<bf16>(y);
        else static_cast<float*>(g.C)[m * g.ldc + n + u] = y;
    }
}

// The tiles of dW = P^T H, then those of dH = P W.
template <typename T>
__global__ __launch_bounds__(64 * kSmallWaves) void small_gradients_kernel(Small32 dw, Small32 dh, int tiles_w) {
    __shared__ float sums[kSmallWaves][32 * 34];
    if (static_cast<int>(blockIdx.x) < tiles_w) {
        const int tm = blockIdx.x / dw.tiles_n, tn = blockIdx.x - tm * dw.tiles_n;
        small_store(dw, tm * 32, tn * 32, small_tile<float, true, T, true>(dw, tm * 32, tn * 32, sums));
    } else {
        const int b = blockIdx.x - tiles_w, tm = b / dh.tiles_n, tn = b - tm * dh.tiles_n;
        small_store(dh, tm * 32, tn * 32, small_tile<float, false, T, true>(dh, tm * 32, tn * 32, sums));
    }
}

// Time of loss and gradients here, in microseconds: the launches, the products at what single loads bring the matrix cores, the longest chains of
// loads (words in dH, width in the logits), the tiles of dW and of the rest.  Fitted to 25 fp32 and 44 bf16 heads of up to 4096 of anything,
// all of them within a quarter.
double small32_us(int32_t dtype, int64_t T, int64_t D, int64_t V) {
    if (T > 4096 || D > 4096 || V > 4096) return 1e30;
    const double products = static_cast<double>(T * D * V) / (int64_t{1} << 29), tiles = static_cast<double>(V * D + T * D + 2 * T * V) / (1024 * 768);
    if (dtype == DAB_BF16) return 14.5 + 17.0 * products + 0.011 * (V + D) + 0.014 * T + 13.0 * tiles;
    return 14.0 + 55.0 * products + 0.012 * (V + D) + 0.006 * T + 4.0 * tiles;
}

static unsigned small_tiles(const Small32& g) { return static_cast<unsigned>(ceil_div(g.M, kSmallTile) * g.tiles_n); }

int launch_small_stats(const Small32& g, int32_t dtype, hipStream_t st) {
    return launch(dtype == DAB_F32 ? small_stats_kernel<float> : small_stats_kernel<bf16>, dim3(small_tiles(g)), dim3(64 * kSmallWaves), 0, st, g);
}
int launch_small_softmax(const Small32& g, int32_t dtype, hipStream_t st) {
    return launch(dtype == DAB_F32 ? small_softmax_kernel<float> : small_softmax_kernel<bf16>, dim3(small_tiles(g)), dim3(64 * kSmallWaves), 0, st, g);
}
int launch_small_gradients(const Small32& dw, const Small32& dh, int32_t dtype, hipStream_t st) {
    const int tiles_w = static_cast<int>(small_tiles(dw));
    return launch(dtype == DAB_F32 ? small_gradients_kernel<float> : small_gradients_kernel<bf16>, dim3(tiles_w + small_tiles(dh)),
                  dim3(64 * kSmallWaves), 0, st, dw, dh, tiles_w);
}
}  // namespace dab
