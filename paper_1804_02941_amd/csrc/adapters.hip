// Products of low rank beside a shared projection: every token takes the pair of matrices of its adapter, or none (include/dab.h).
//
//     U = X A_i^T,  Y = base + s_i U B_i;    V = s_i dY B_i^T,  dX = base + V A_i,  dA_i = V^T X,  dB_i = s_i U^T dY
//
// A and B are r long rows per adapter, so that forward and backward are the same three products: `shrink` (long rows times long rows, r
// results a token), `expand` (r numbers a token times long rows) and `outer` (the sum over an adapter's tokens of r numbers times a long row).  Each is
// bound by its long rows in memory: 2 r operations an element.  Tokens come in any order; a tile of sixteen takes its adapters one after the other,
// and what a token is not to take is left out by selection, not by a product with zero, so that no adapter's infinities and NaN
// reach another's tokens.
#include <algorithm>

#include "lanes.h"
#include "real16.h"

namespace dab {

typedef _Float16 v8h __attribute__((ext_vector_type(8)));

struct Adapters {
    const int32_t* ids;
    const float* scale;              // or null: 1
    int T, n, r;
};

__device__ __forceinline__ int adapter_of(const Adapters& a, int64_t t) {
    const int id = t < a.T ? a.ids[t] : -1;
    return static_cast<uint32_t>(id) < static_cast<uint32_t>(a.n) ? id : -1;
}
__device__ __forceinline__ float scale_of(const Adapters& a, int id) { return a.scale ? a.scale[id] : 1.f; }

// ---------------------------------------------------------------- shrink
// Eight k as the matrix cores take them: 16-bit numbers as they are, fp32 ones for eight products of four k.
template <typename T>
struct Long;
template <>
struct Long<float> {
    float v[8];
    __device__ __forceinline__ void load(const float* row, int k, int K) { load8(row, k, K, v); }
    static __device__ __forceinline__ v4f mul(const Long& a, const Long& b, v4f c) {
#pragma unroll
        for (int i = 0; i < 8; ++i) c = __builtin_amdgcn_mfma_f32_16x16x4f32(a.v[i], b.v[i], c, 0, 0, 0);
        return c;
    }
};
template <typename T, typename V>
__device__ __forceinline__ void load_raw(const T* row, int k, int K, V* v) {
    if (k + 8 <= K) {
        *v = *reinterpret_cast<const typename Unaligned<T, 8>::type*>(row + k);
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) (*v)[i] = k + i < K ? row[k + i] : static_cast<T>(0.f);
    }
}
template <>
struct Long<bf16> {
    v8bf v;
    __device__ __forceinline__ void load(const bf16* row, int k, int K) { load_raw(row, k, K, &v); }
    static __device__ __forceinline__ v4f mul(const Long& a, const Long& b, v4f c) { return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a.v, b.v, c, 0, 0, 0); }
};
template <>
struct Long<f16> {
    v8h v;
    __device__ __forceinline__ void load(const f16* row, int k, int K) { load_raw(row, k, K, &v); }
    static __device__ __forceinline__ v4f mul(const Long& a, const Long& b, v4f c) { return __builtin_amdgcn_mfma_f32_16x16x32_f16(a.v, b.v, c, 0, 0, 0); }
};

// Many tokens: a workgroup takes sixteen of them and 16 RT of the r rows, its wavefronts every eighth step of 32 k.
constexpr int kShrinkWaves = 8;
template <typename T, int RT>
__global__ __launch_bounds__(64 * kShrinkWaves) void shrink_kernel(const T* __restrict__ X, int64_t ldx, const T* __restrict__ A, int K, Adapters a,
                                                                   int scaled, float* __restrict__ U) {
    __shared__ float sums[kShrinkWaves][RT][16][17];
    DAB_RESERVE_VGPRS();
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, m = lane & 15, g = lane >> 4;
    const int64_t t0 = static_cast<int64_t>(blockIdx.x) * 16, t = t0 + m;
    const int r0 = blockIdx.y * 16 * RT, id = adapter_of(a, t);
    const T* x = X + (t < a.T ? t : a.T - 1) * ldx;
    v4f out[RT];
#pragma unroll
    for (int j = 0; j < RT; ++j) out[j] = v4f{0.f, 0.f, 0.f, 0.f};
    bool waiting = id >= 0;
    while (__any(waiting)) {
        const int now = __shfl(id, __ffsll(static_cast<unsigned long long>(__ballot(waiting))) - 1);
        const T* rows = A + static_cast<int64_t>(now) * a.r * K;
        v4f acc[RT];
#pragma unroll
        for (int j = 0; j < RT; ++j) acc[j] = v4f{0.f, 0.f, 0.f, 0.f};
        for (int64_t k0 = wave * 32; k0 < K; k0 += kShrinkWaves * 32) {
            const int k = static_cast<int>(k0) + g * 8;
            Long<T> xv;
            xv.load(x, k, K);
#pragma unroll
            for (int j = 0; j < RT; ++j) {
                Long<T> av;
                av.load(rows + static_cast<int64_t>(min(r0 + j * 16 + m, a.r - 1)) * K, k, K);
                acc[j] = Long<T>::mul(av, xv, acc[j]);
            }
        }
        if (id == now) {
#pragma unroll
            for (int j = 0; j < RT; ++j) out[j] = acc[j];
            waiting = false;
        }
    }
#pragma unroll
    for (int j = 0; j < RT; ++j)
#pragma unroll
        for (int v = 0; v < 4; ++v) sums[wave][j][m][g * 4 + v] = out[j][v];       // [token][row]
    __syncthreads();
    for (int i = threadIdx.x; i < RT * 256; i += 64 * kShrinkWaves) {
        const int j = i >> 8, token = (i >> 4) & 15, row = r0 + j * 16 + (i & 15);
        if (t0 + token >= a.T || row >= a.r) continue;
        float u = 0.f;
#pragma unroll
        for (int w = 0; w < kShrinkWaves; ++w) u += sums[w][j][token][i & 15];
        if (scaled) {
            const int who = adapter_of(a, t0 + token);
            u = who >= 0 ? u * scale_of(a, who) : 0.f;
        }
        U[(t0 + token) * a.r + row] = u;
    }
}

// Few tokens: a wavefront takes one row of a token's adapter.
template <typename T>
__global__ __launch_bounds__(256) void shrink_few_kernel(const T* __restrict__ X, int64_t ldx, const T* __restrict__ A, int K, Adapters a, int scaled,
                                                         float* __restrict__ U) {
    const int lane = threadIdx.x & 63;
    const int64_t at = static_cast<int64_t>(blockIdx.x) * 4 + (threadIdx.x >> 6);
    if (at >= static_cast<int64_t>(a.T) * a.r) return;
    const int64_t t = at / a.r;
    const int row = static_cast<int>(at - t * a.r), id = adapter_of(a, t);
    float sum = 0.f;
    if (id >= 0) {
        const T *x = X + t * ldx, *w = A + (static_cast<int64_t>(id) * a.r + row) * K;
        for (int64_t k0 = lane * 8; k0 < K; k0 += 512) {
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

// ---------------------------------------------------------------- expand
struct Base {
    const void* p;                   // or null
    int64_t ld;
    int dtype;
};
__device__ __forceinline__ void load_base(const Base& b, int64_t t, int f, int F, float (&v)[8]) {
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = 0.f;
    if (!b.p) return;
    if (b.dtype == DAB_F32) load8(static_cast<const float*>(b.p) + t * b.ld, f, F, v);
    else if (b.dtype == DAB_BF16) load8(static_cast<const bf16*>(b.p) + t * b.ld, f, F, v);
    else load8(static_cast<const f16*>(b.p) + t * b.ld, f, F, v);
}

// Many tokens: a wavefront takes sixteen of them and 128 columns, lane l the eight columns 8 (l % 16) .. of tokens 4 (l / 16) .. + 3.  In
// fp32 on the matrix cores, whatever the type: U is fp32, and the products are few.
constexpr int kExpandWaves = 4;
template <typename T>
__global__ __launch_bounds__(64 * kExpandWaves) void expand_kernel(const float* __restrict__ U, const T* __restrict__ B, int F, Adapters a, int scaled,
                                                                   Base base, T* Y) {
    DAB_RESERVE_VGPRS();
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, m = lane & 15, g = lane >> 4;
    const int64_t t0 = static_cast<int64_t>(blockIdx.x) * 16;
    const int64_t f64 = (static_cast<int64_t>(blockIdx.y) * kExpandWaves + wave) * 128 + m * 8;
    if (f64 - m * 8 >= F) return;
    const int f = static_cast<int>(f64);
    const int id = adapter_of(a, t0 + m);
    const float s = id >= 0 && scaled ? scale_of(a, id) : 1.f;
    v4f out[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) out[j] = v4f{0.f, 0.f, 0.f, 0.f};
    bool waiting = id >= 0;
    while (__any(waiting)) {
        const int now = __shfl(id, __ffsll(static_cast<unsigned long long>(__ballot(waiting))) - 1);
        const T* rows = B + static_cast<int64_t>(now) * a.r * F;
        v4f acc[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) acc[j] = v4f{0.f, 0.f, 0.f, 0.f};
        for (int q = 0; q < a.r; q += 4) {
            const int row = q + g;
            float b[8] = {};
            float u = 0.f;
            if (row < a.r) {
                load8(rows + static_cast<int64_t>(row) * F, f, F, b);
                if (id == now) u = U[(t0 + m) * a.r + row] * s;
            }
#pragma unroll
            for (int j = 0; j < 8; ++j) acc[j] = __builtin_amdgcn_mfma_f32_16x16x4f32(u, b[j], acc[j], 0, 0, 0);
        }
        // (of the tokens in this lane's results)
#pragma unroll
        for (int v = 0; v < 4; ++v) {
            const bool mine = __shfl(id, 4 * g + v) == now;
#pragma unroll
            for (int j = 0; j < 8; ++j) out[j][v] = mine ? acc[j][v] : out[j][v];
        }
        waiting = waiting && id != now;
    }
    if (f >= F) return;
#pragma unroll
    for (int v = 0; v < 4; ++v) {
        const int64_t t = t0 + 4 * g + v;
        if (t >= a.T) break;
        float y[8];
        load_base(base, t, f, F, y);
#pragma unroll
        for (int j = 0; j < 8; ++j) y[j] += out[j][v];
        store8(Y + t * F, f, F, y);
    }
}

// Few tokens: a lane takes eight columns of one.
template <typename T>
__global__ __launch_bounds__(64) void expand_few_kernel(const float* __restrict__ U, const T* __restrict__ B, int F, Adapters a, int scaled, Base base,
                                                        T* Y) {
    const int64_t t = blockIdx.y, f64 = (static_cast<int64_t>(blockIdx.x) * 64 + threadIdx.x) * 8;
    if (f64 >= F) return;
    const int f = static_cast<int>(f64), id = adapter_of(a, t);
    float y[8], v[8] = {};
    load_base(base, t, f, F, y);
    if (id >= 0) {
        const T* rows = B + static_cast<int64_t>(id) * a.r * F;
        const float s = scaled ? scale_of(a, id) : 1.f;
        for (int row = 0; row < a.r; ++row) {
            float b[8];
            load8(rows + static_cast<int64_t>(row) * F, f, F, b);
            const float u = U[t * a.r + row] * s;
#pragma unroll
            for (int i = 0; i < 8; ++i) v[i] += u * b[i];
        }
#pragma unroll
        for (int i = 0; i < 8; ++i) y[i] += v[i];
    }
    store8(Y + t * F, f, F, y);
}

// ---------------------------------------------------------------- outer
// A workgroup takes 128 columns, 16 RT of the r rows, a share of the tokens and every slices-th adapter; of each adapter that has tokens in its share
// its wavefronts take every eighth four of them, and add up in LDS.  parts: [share][adapter][r][columns], have: [share][adapter], 1
// where the share has tokens of the adapter (other parts are not written).
constexpr int kOuterWaves = 8, kOuterMaxAdapters = 65536;
struct Outer {
    int cols, tokens, slices;        // columns, tokens of a share (a multiple of 32), slices of the adapters
    int64_t ldx;
    int32_t* have;
};
template <typename T, int RT>
__global__ __launch_bounds__(64 * kOuterWaves) void outer_kernel(const float* __restrict__ V, const T* __restrict__ X, Adapters a, int scaled, Outer o,
                                                                 float* __restrict__ parts) {
    extern __shared__ uint32_t present[];                    // a bit for every adapter
    __shared__ float sums[kOuterWaves / 2][16][132];
    DAB_RESERVE_VGPRS();
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, m = lane & 15, g = lane >> 4;
    const int tiles = (o.cols + 127) >> 7, tile = blockIdx.x % tiles, rb = blockIdx.x / tiles;
    const int share = blockIdx.y, slice = blockIdx.z, r0 = rb * 16 * RT;
    const int64_t first = static_cast<int64_t>(share) * o.tokens, last = min(first + o.tokens, static_cast<int64_t>(a.T));
    const int words = (a.n + 31) >> 5;
    for (int i = threadIdx.x; i < words; i += 64 * kOuterWaves) present[i] = 0;
    __syncthreads();
    for (int64_t t = first + threadIdx.x; t < last; t += 64 * kOuterWaves) {
        const int id = adapter_of(a, t);
        if (id >= 0) atomicOr(&present[id >> 5], 1u << (id & 31));
    }
    __syncthreads();
    if (tile == 0 && rb == 0)
        for (int i = slice + threadIdx.x * o.slices; i < a.n; i += 64 * kOuterWaves * o.slices)
            o.have[static_cast<int64_t>(share) * a.n + i] = (present[i >> 5] >> (i & 31)) & 1u;
    const int c = tile * 128 + m * 8;
    for (int id = slice; id < a.n; id += o.slices) {
        if (!((present[id >> 5] >> (id & 31)) & 1u)) continue;              // (the same for the whole workgroup)
        const float s = scaled ? scale_of(a, id) : 1.f;
        v4f acc[RT][8];
#pragma unroll
        for (int j = 0; j < RT; ++j)
#pragma unroll
            for (int i = 0; i < 8; ++i) acc[j][i] = v4f{0.f, 0.f, 0.f, 0.f};
        for (int64_t t1 = first + wave * 4; t1 < last; t1 += kOuterWaves * 4) {
            const int64_t t = t1 + g;
            const bool mine = t < last && a.ids[t] == id;
            if (!__any(mine)) continue;
            float x[8] = {}, v[RT];
#pragma unroll
            for (int j = 0; j < RT; ++j) v[j] = 0.f;
            if (mine) {
                if (c < o.cols) load8(X + t * o.ldx, c, o.cols, x);
#pragma unroll
                for (int j = 0; j < RT; ++j)
                    if (r0 + j * 16 + m < a.r) v[j] = V[t * a.r + r0 + j * 16 + m] * s;
            }
#pragma unroll
            for (int j = 0; j < RT; ++j)
#pragma unroll
                for (int i = 0; i < 8; ++i) acc[j][i] = __builtin_amdgcn_mfma_f32_16x16x4f32(v[j], x[i], acc[j][i], 0, 0, 0);
        }
        // rows 4 g + v of 16, columns 8 m + i of 128: added up in a fixed order, the upper wavefronts' onto the lower ones'
#pragma unroll
        for (int j = 0; j < RT; ++j) {
#pragma unroll
            for (int half = kOuterWaves / 2; half >= 1; half /= 2) {
                if (wave >= half && wave < 2 * half)
#pragma unroll
                    for (int i = 0; i < 8; ++i)
#pragma unroll
                        for (int v = 0; v < 4; ++v) sums[wave - half][4 * g + v][m * 8 + i] = acc[j][i][v];
                __syncthreads();
                if (wave < half)
#pragma unroll
                    for (int i = 0; i < 8; ++i)
#pragma unroll
                        for (int v = 0; v < 4; ++v) acc[j][i][v] += sums[wave][4 * g + v][m * 8 + i];
                __syncthreads();
            }
            if (wave == 0 && c < o.cols)
#pragma unroll
                for (int v = 0; v < 4; ++v) {
                    const int row = r0 + j * 16 + 4 * g + v;
                    if (row >= a.r) break;
                    float w[8];
#pragma unroll
                    for (int i = 0; i < 8; ++i) w[i] = acc[j][i][v];
                    store8(parts + ((static_cast<int64_t>(share) * a.n + id) * a.r + row) * o.cols, c, o.cols, w);
                }
        }
    }
}

// The shares' parts added in a fixed order; zeros for an adapter without tokens.
__global__ __launch_bounds__(256) void outer_join_kernel(const float* __restrict__ parts, const int32_t* __restrict__ have, int shares, int n,
                                                         int64_t size, float* __restrict__ out) {
    const int64_t at = (static_cast<int64_t>(blockIdx.x) * 256 + threadIdx.x) * 4;
    const int id = blockIdx.y;
    if (at >= size) return;
    const int left = static_cast<int>(min(size - at, int64_t{4}));
    float v[4] = {};
    for (int s = 0; s < shares; ++s) {
        const int64_t who = static_cast<int64_t>(s) * n + id;
        if (!have[who]) continue;
        const float* from = parts + who * size + at;
        if (left == 4) {
            const auto got = *reinterpret_cast<const Unaligned<float, 4>::type*>(from);
#pragma unroll
            for (int i = 0; i < 4; ++i) v[i] += got[i];
        } else {
            for (int i = 0; i < left; ++i) v[i] += from[i];
        }
    }
    float* to = out + static_cast<int64_t>(id) * size + at;
    for (int i = 0; i < left; ++i) to[i] = v[i];
}

// ---------------------------------------------------------------- host side
constexpr int kFewTokens = 64;       // up to these, a wavefront or a lane per token and row
constexpr int kMaxRank = 256;

template <typename T>
static int shrink(const T* X, int64_t ldx, const T* A, int K, const Adapters& a, bool scaled, float* U, hipStream_t st) {
    if (a.T <= kFewTokens)
        return launch(shrink_few_kernel<T>, dim3(static_cast<unsigned>(ceil_div64(static_cast<int64_t>(a.T) * a.r, 4))), dim3(256), 0, st, X, ldx, A, K, a,
                      static_cast<int>(scaled), U);
    const unsigned tiles = static_cast<unsigned>(ceil_div64(a.T, 16));
    const dim3 block(64 * kShrinkWaves);
    const int s = scaled;
    if (a.r <= 16) return launch(shrink_kernel<T, 1>, dim3(tiles), block, 0, st, X, ldx, A, K, a, s, U);
    if (a.r <= 32) return launch(shrink_kernel<T, 2>, dim3(tiles), block, 0, st, X, ldx, A, K, a, s, U);
    return launch(shrink_kernel<T, 4>, dim3(tiles, ceil_div(a.r, 64)), block, 0, st, X, ldx, A, K, a, s, U);
}

template <typename T>
static int expand(const float* U, const T* B, int F, const Adapters& a, bool scaled, const Base& base, T* Y, hipStream_t st) {
    if (a.T <= kFewTokens)
        return launch(expand_few_kernel<T>, dim3(static_cast<unsigned>(ceil_div64(F, 512)), a.T), dim3(64), 0, st, U, B, F, a, static_cast<int>(scaled),
                      base, Y);
    return launch(expand_kernel<T>, dim3(static_cast<unsigned>(ceil_div64(a.T, 16)), static_cast<unsigned>(ceil_div64(F, 128 * kExpandWaves))),
                  dim3(64 * kExpandWaves), 0, st, U, B, F, a, static_cast<int>(scaled), base, Y);
}

struct OuterPlan {
    int shares, tokens, slices, rt;
    size_t parts, have;              // bytes, multiples of 256
};
static OuterPlan outer_plan(int T, int n, int r, int cols) {
    OuterPlan p{};
    p.rt = r <= 16 ? 1 : r <= 32 ? 2 : 4;
    const int64_t tiles = static_cast<int64_t>(ceil_div(cols, 128)) * ceil_div(r, 16 * p.rt), part = static_cast<int64_t>(n) * r * cols * 4;
    // about two workgroups for every compute unit, shares of at least 128 tokens, parts of at most 256 MB
    int64_t shares = ceil_div64(2 * kNumCU, tiles);
    shares = std::min<int64_t>(shares, ceil_div64(T, 128));
    shares = std::max<int64_t>(1, std::min<int64_t>(shares, (int64_t{256} << 20) / part));
    p.tokens = static_cast<int>(round_up(ceil_div64(T, shares), 32));
    p.shares = static_cast<int>(ceil_div64(T, p.tokens));
    p.slices = static_cast<int>(std::max<int64_t>(1, std::min<int64_t>(std::min(n, 1024), 2 * kNumCU / (tiles * p.shares))));
    p.parts = round_up(part * p.shares, 256), p.have = round_up(static_cast<int64_t>(p.shares) * n * 4, 256);
    return p;
}
template <typename T>
static int outer(const float* V, const T* X, int64_t ldx, int cols, const Adapters& a, bool scaled, float* out, char* ws, hipStream_t st) {
    const OuterPlan p = outer_plan(a.T, a.n, a.r, cols);
    Outer o{};
    o.cols = cols, o.tokens = p.tokens, o.slices = p.slices, o.ldx = ldx, o.have = reinterpret_cast<int32_t*>(ws + p.parts);
    float* parts = reinterpret_cast<float*>(ws);
    const int64_t x = static_cast<int64_t>(ceil_div(cols, 128)) * ceil_div(a.r, 16 * p.rt);
    const dim3 grid(static_cast<unsigned>(x), p.shares, p.slices), block(64 * kOuterWaves);
    const size_t lds = static_cast<size_t>(ceil_div(a.n, 32)) * 4;
    const int s = scaled;
    int rc;
    if (p.rt == 1) rc = launch(outer_kernel<T, 1>, grid, block, lds, st, V, X, a, s, o, parts);
    else if (p.rt == 2) rc = launch(outer_kernel<T, 2>, grid, block, lds, st, V, X, a, s, o, parts);
    else rc = launch(outer_kernel<T, 4>, grid, block, lds, st, V, X, a, s, o, parts);
    if (rc) return rc;
    const int64_t size = static_cast<int64_t>(a.r) * cols;
    return launch(outer_join_kernel, dim3(static_cast<unsigned>(ceil_div64(size, 1024)), a.n), dim3(256), 0, st, static_cast<const float*>(parts),
                  static_cast<const int32_t*>(o.have), p.shares, a.n, size, out);
}

static int check_adapters(const void* X, int32_t dtype, int64_t ldx, const int32_t* ids, const void* A, const void* B, const float* scale, int32_t T,
                          int32_t K, int32_t F, int32_t n, int32_t r) {
    if (!X || !ids || !A || !B) return DAB_ERR_NULL;
    if (T < 1 || K < 1 || F < 1 || n < 1 || r < 1 || ldx < K) return DAB_ERR_SHAPE;
    if (!real_dtype(dtype) || K > (1 << 24) || F > (1 << 24) || n > 65535 || r > kMaxRank || T > (1 << 25)) return DAB_ERR_UNSUPPORTED;
    if (misaligned(X, 16) || misaligned(A, 16) || misaligned(B, 16) || misaligned(ids, 4) || misaligned(scale, 4)) return DAB_ERR_ALIGN;
    return DAB_OK;
}
static int check_base(const void* base, int32_t dtype, int64_t ld, int32_t cols, int32_t own_dtype) {
    if (!base) return DAB_OK;
    if (ld < cols) return DAB_ERR_SHAPE;
    if (dtype != DAB_F32 && dtype != own_dtype) return DAB_ERR_UNSUPPORTED;
    return misaligned(base, 16) ? DAB_ERR_ALIGN : DAB_OK;
}

}  // namespace dab

extern "C" int dab_adapters(const void* X, int32_t dtype, int64_t ldx, const int32_t* ids, const void* A, const void* B, const float* scale, int32_t T,
                            int32_t K, int32_t F, int32_t n, int32_t r, const void* base, int32_t base_dtype, int64_t ldbase, void* Y, float* U,
                            void* stream) {
    using namespace dab;
    if (int rc = check_adapters(X, dtype, ldx, ids, A, B, scale, T, K, F, n, r)) return rc;
    if (!Y || !U) return DAB_ERR_NULL;
    if (int rc = check_base(base, base_dtype, ldbase, F, dtype)) return rc;
    if (misaligned(Y, 16) || misaligned(U, 4)) return DAB_ERR_ALIGN;
    const Adapters a{ids, scale, T, n, r};
    const auto st = static_cast<hipStream_t>(stream);
    const auto go = [&](auto* t) -> int {
        typedef std::remove_pointer_t<decltype(t)> E;
        if (int rc = shrink(static_cast<const E*>(X), ldx, static_cast<const E*>(A), K, a, false, U, st)) return rc;
        return expand(static_cast<const float*>(U), static_cast<const E*>(B), F, a, true, Base{base, ldbase, base_dtype}, static_cast<E*>(Y), st);
    };
    if (dtype == DAB_F32) return go(static_cast<float*>(nullptr));
    if (dtype == DAB_BF16) return go(static_cast<bf16*>(nullptr));
    return go(static_cast<f16*>(nullptr));
}

extern "C" size_t dab_adapters_gradient_workspace_bytes(int32_t T, int32_t K, int32_t F, int32_t n, int32_t r) {
    using namespace dab;
    if (T < 1 || K < 1 || F < 1 || n < 1 || r < 1 || K > (1 << 24) || F > (1 << 24) || n > 65535 || r > kMaxRank || T > (1 << 25)) return 0;
    const OuterPlan p = outer_plan(T, n, r, K), q = outer_plan(T, n, r, F);
    return static_cast<size_t>(round_up(static_cast<int64_t>(T) * r * 4, 256)) + std::max(p.parts + p.have, q.parts + q.have);
}

extern "C" int dab_adapters_gradient(const void* dY, int64_t lddy, const void* X, int32_t dtype, int64_t ldx, const float* U, const int32_t* ids,
                                     const void* A, const void* B, const float* scale, int32_t T, int32_t K, int32_t F, int32_t n, int32_t r,
                                     const void* base, int32_t base_dtype, int64_t ldbase, void* dX, float* dA, float* dB, void* ws, size_t ws_bytes,
                                     void* stream) {
    using namespace dab;
    if (int rc = check_adapters(X, dtype, ldx, ids, A, B, scale, T, K, F, n, r)) return rc;
    if (!dY || !U || !dA || !dB || (base && !dX)) return DAB_ERR_NULL;
    if (lddy < F) return DAB_ERR_SHAPE;
    if (int rc = check_base(base, base_dtype, ldbase, K, dtype)) return rc;
    if (misaligned(dY, 16) || misaligned(dX, 16) || misaligned(U, 4) || misaligned(dA, 4) || misaligned(dB, 4)) return DAB_ERR_ALIGN;
    const size_t need = dab_adapters_gradient_workspace_bytes(T, K, F, n, r);
    if (!ws || ws_bytes < need || misaligned(ws, 256)) return DAB_ERR_WORKSPACE;
    const Adapters a{ids, scale, T, n, r};
    const auto st = static_cast<hipStream_t>(stream);
    float* V = static_cast<float*>(ws);
    char* rest = static_cast<char*>(ws) + round_up(static_cast<int64_t>(T) * r * 4, 256);
    const auto go = [&](auto* t) -> int {
        typedef std::remove_pointer_t<decltype(t)> E;
        const E *x = static_cast<const E*>(X), *dy = static_cast<const E*>(dY), *up = static_cast<const E*>(B), *down = static_cast<const E*>(A);
        if (int rc = shrink(dy, lddy, up, F, a, true, V, st)) return rc;
        if (int rc = outer(U, dy, lddy, F, a, true, dB, rest, st)) return rc;
        if (int rc = outer(static_cast<const float*>(V), x, ldx, K, a, false, dA, rest, st)) return rc;
        if (!dX) return DAB_OK;
        return expand(static_cast<const float*>(V), down, K, a, false, Base{base, ldbase, base_dtype}, static_cast<E*>(dX), st);
    };
    if (dtype == DAB_F32) return go(static_cast<float*>(nullptr));
    if (dtype == DAB_BF16) return go(static_cast<bf16*>(nullptr));
    return go(static_cast<f16*>(nullptr));
}

namespace dab {
// Workspace of the served call: the projection's own, its sums in fp32, and U.
struct ServeSpace {
    size_t product, base, u;
};
static ServeSpace serve_space(int32_t B, int32_t K, int32_t F, int32_t r, int32_t dtype, int64_t ldx) {
    return {static_cast<size_t>(round_up(static_cast<int64_t>(dab_w4_matvec_workspace_bytes(B, K, F, dtype, ldx)), 256)),
            static_cast<size_t>(round_up(static_cast<int64_t>(B) * F * 4, 256)), static_cast<size_t>(round_up(static_cast<int64_t>(B) * r * 4, 256))};
}
}  // namespace dab

extern "C" size_t dab_w4_adapters_workspace_bytes(int32_t B, int32_t K, int32_t F, int32_t r, int32_t dtype, int64_t ldx) {
    using namespace dab;
    if (B < 1 || K < 1 || F < 1 || r < 1 || !real_dtype(dtype)) return 0;
    const ServeSpace s = serve_space(B, K, F, r, dtype, ldx);
    return s.product + s.base + s.u;
}

extern "C" int dab_w4_adapters(const void* X, int32_t dtype, int64_t ldx, const uint8_t* Q, const uint8_t* S, const int32_t* ids, const void* A,
                               const void* Bt, const float* scale, int32_t B, int32_t K, int32_t F, int32_t n, int32_t r, void* Y, void* ws,
                               size_t ws_bytes, void* stream) {
    using namespace dab;
    if (int rc = check_adapters(X, dtype, ldx, ids, A, Bt, scale, B, K, F, n, r)) return rc;
    if (!Q || !S || !Y) return DAB_ERR_NULL;
    if (B > 65535 || F > 65535 * 16) return DAB_ERR_UNSUPPORTED;
    if (misaligned(Q, 16) || misaligned(S, 16) || misaligned(Y, 16)) return DAB_ERR_ALIGN;
    const ServeSpace s = serve_space(B, K, F, r, dtype, ldx);
    if (!ws || ws_bytes < s.product + s.base + s.u || misaligned(ws, 256)) return DAB_ERR_WORKSPACE;
    char* at = static_cast<char*>(ws);
    float *base = reinterpret_cast<float*>(at + s.product), *U = reinterpret_cast<float*>(at + s.product + s.base);
    if (int rc = w4_product(X, dtype, ldx, Q, S, B, K, F, base, DAB_F32, ws, s.product, stream)) return rc;
    return dab_adapters(X, dtype, ldx, ids, A, Bt, scale, B, K, F, n, r, base, DAB_F32, F, Y, U, stream);
}
