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

// Eight neighbouring elements as they are, all of them in the row.
template <typename T>
struct Eight {
    typename Unaligned<T, 8>::type v;
    __device__ __forceinline__ void load(const T* row, int c) { v = *reinterpret_cast<const typename Unaligned<T, 8>::type*>(row + c); }
    __device__ __forceinline__ float operator[](int i) const { return static_cast<float>(v[i]); }
};

// Few tokens: a wavefront takes one row of a token's adapter, its lanes eight k of 512, four of those turns in flight.
constexpr int kFewTokens = 64;
template <typename T>
__device__ __forceinline__ void shrink_few(const T* __restrict__ X, int64_t ldx, const T* __restrict__ A, int K, const Adapters& a, bool scaled,
                                           int64_t at, float* __restrict__ U) {
    const int lane = threadIdx.x & 63;
    const int64_t t = at / a.r;
    const int row = static_cast<int>(at - t * a.r), id = adapter_of(a, t);
    float sum = 0.f;
    if (id >= 0) {
        const T *x = X + t * ldx, *w = A + (static_cast<int64_t>(id) * a.r + row) * K;
        int64_t k0 = 0;
        for (; k0 + 2048 <= K; k0 += 2048) {
            Eight<T> p[4], q[4];
#pragma unroll
            for (int u = 0; u < 4; ++u) {
                const int k = static_cast<int>(k0) + u * 512 + lane * 8;
                p[u].load(x, k), q[u].load(w, k);
            }
#pragma unroll
            for (int u = 0; u < 4; ++u)
#pragma unroll
                for (int i = 0; i < 8; ++i) sum += p[u][i] * q[u][i];
        }
        for (k0 += lane * 8; k0 < K; k0 += 512) {
            float p[8], q[8];
            load8(x, static_cast<int>(k0), K, p), load8(w, static_cast<int>(k0), K, q);
#pragma unroll
            for (int i = 0; i < 8; ++i) sum += p[i] * q[i];
        }
        if (scaled) sum *= scale_of(a, id);
    }
    sum = lanes_sum<6>(sum);
    if (lane == 0) U[at] = sum;
}

// U of any number of tokens (adapters.hip).
template <typename T>
int shrink(const T* X, int64_t ldx, const T* A, int K, const Adapters& a, bool scaled, float* U, hipStream_t st);

// What all calls with adapters refuse alike.
int check_adapters(const void* X, int32_t dtype, int64_t ldx, const int32_t* ids, const void* A, const void* B, const float* scale, int32_t T, int32_t K,
                   int32_t F, int32_t n, int32_t r);

}  // namespace dab
