// What the calls with adapters share (adapters.hip, w4.hip).
#pragma once

#include "lanes.h"
#include "real16.h"

namespace dab {

struct Adapters {
    const int32_t* ids;
    const float* scale;              // or null: 1
    int T, n, r;
};

// A token's adapter, -1 for none.
__device__ __forceinline__ int adapter_of(const Adapters& a, int64_t t) {
    const int id = t < a.T ? a.ids[t] : -1;
    return static_cast<uint32_t>(id) < static_cast<uint32_t>(a.n) ? id : -1;
}
__device__ __forceinline__ float scale_of(const Adapters& a, int id) { return a.scale ? a.scale[id] : 1.f; }

// N neighbouring elements as they are: all of them in the row, or zeros past its end.
template <typename T, int N>
struct Some {
    typedef typename Unaligned<T, N>::type V;
    V v;
    __device__ __forceinline__ void load(const T* row, int c) { v = *reinterpret_cast<const V*>(row + c); }
    // (past the caches: what nobody reads again soon)
    __device__ __forceinline__ void load_once(const T* row, int c) { v = __builtin_nontemporal_load(reinterpret_cast<const V*>(row + c)); }
    __device__ __forceinline__ void load(const T* row, int c, int cols) {
        if (c + N <= cols) {
            load(row, c);
        } else {
#pragma unroll
            for (int i = 0; i < N; ++i) v[i] = c + i < cols ? row[c + i] : static_cast<T>(0.f);
        }
    }
    // those from column c on, or the row's last N where fewer are left (of rows of N columns at least)
    __device__ __forceinline__ void load_last(const T* row, int c, int cols) {
        if (cols < N) load(row, c, cols);
        else load(row, min(c, cols - N));
    }
    __device__ __forceinline__ float operator[](int i) const { return static_cast<float>(v[i]); }
};
template <typename T>
using Eight = Some<T, 8>;

// Rows of kNarrow columns and more are read eight at a time throughout: the last eight of a row, some of them a second time, where fewer are left.
constexpr int kNarrow = 8;

// Few tokens: a workgroup of four wavefronts takes one row of a token's adapter, a lane eight k of 2048 at a time, four of those turns in flight.  (A
// wavefront a row: seven fp32 tokens, 8 rows of 9111, 6.8 us.)
constexpr int kFewTokens = 64, kFewWaves = 4;
template <typename T>
__device__ __forceinline__ void shrink_few(const T* __restrict__ X, int64_t ldx, const T* __restrict__ A, int K, const Adapters& a, bool scaled,
                                           int64_t at, float* __restrict__ U) {
    __shared__ float part[kFewWaves];
    const int64_t t = at / a.r;
    const int row = static_cast<int>(at - t * a.r), id = adapter_of(a, t);
    if (id < 0) {
        if (threadIdx.x == 0) U[at] = 0.f;
        return;
    }
    const T *x = X + t * ldx, *w = A + (static_cast<int64_t>(id) * a.r + row) * K;
    float sum = 0.f;
    for (int64_t k0 = threadIdx.x * 8; k0 < K; k0 += 8192) {
        Eight<T> p[4], q[4];
#pragma unroll
        for (int u = 0; u < 4; ++u) {
            const int64_t k = k0 + u * 2048;
            p[u].v = {}, q[u].v = {};
            if (k < K) p[u].load_last(x, static_cast<int>(k), K), q[u].load_last(w, static_cast<int>(k), K);
        }
#pragma unroll
        for (int u = 0; u < 4; ++u) {
            // (the last few k: those of the last eight that no lane before has)
            const int64_t k = k0 + u * 2048;
            const int again = K >= 8 && k < K ? static_cast<int>(k) - (K - 8) : 0;
            if (again > 0)
#pragma unroll
                for (int i = 0; i < 8; ++i)
                    if (i < again) p[u].v[i] = q[u].v[i] = static_cast<T>(0.f);
        }
#pragma unroll
        for (int u = 0; u < 4; ++u)
#pragma unroll
            for (int i = 0; i < 8; ++i) sum += p[u][i] * q[u][i];
    }
    sum = lanes_sum<6>(sum);
    if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = sum;
    __syncthreads();
    if (threadIdx.x != 0) return;
    sum = (part[0] + part[1]) + (part[2] + part[3]);
    U[at] = scaled ? sum * scale_of(a, id) : sum;
}

// The adapters of the tokens behind a 4-bit product (w4.hip).
struct W4Adapters {
    Adapters a;
    float* U;                        // times the adapters' scales
    const void *A, *B;
};
// The product alone (w null), or with the tokens' adapters behind it.  Of up to kFewTokens tokens it makes U itself, in the launch that lays
// the tokens out; of more U is there already.
int w4_product(const void* X, int32_t dtype, int64_t ldx, const uint8_t* Q, const uint8_t* S, int32_t B, int32_t K, int32_t F, void* Y, void* ws,
               size_t ws_bytes, hipStream_t st, const W4Adapters* w = nullptr);

}  // namespace dab
