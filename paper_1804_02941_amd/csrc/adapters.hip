// Products of low rank beside a shared projection: every token takes the pair of matrices of its adapter, or none (include/dab.h).
//
//     U = X A_i^T,  Y = base + s_i U B_i;    V = s_i dY B_i^T,  dX = base + V A_i,  dA_i = V^T X,  dB_i = s_i U^T dY
//
// A and B are r long rows per adapter, so that forward and backward are the same three products: `shrink` (long rows times long rows, r
// results a token), `expand` (r numbers a token times long rows) and `outer` (the sum over an adapter's tokens of r numbers times a long row).  Each is
// bound by its long rows in memory: 2 r operations an element.  Tokens come in any order; a tile of sixteen takes its adapters one after the other,
// and what a token is not to take is left out by selection, not by a product with zero, so that no adapter's infinities and NaN
// reach another's tokens.  8192 tokens of four adapters, 4096 -> 4096, r = 16, bf16: U and Y 46 us (207 MB, 4.5 TB/s), V and dX the same, dA and dB 34
// (132 MB, 3.9) and 6 for joining shares.
#include <algorithm>

#include "adapters.h"

namespace dab {

typedef _Float16 v8h __attribute__((ext_vector_type(8)));

// ---------------------------------------------------------------- shrink
// Eight k as the matrix cores take them: 16-bit numbers as they are, fp32 ones for eight products of four k.  ODD: 16-bit rows at odd distances, every
// other one of which lies two bytes behind a multiple of four, where 16 bytes a lane from sixteen rows are slow: there the four words that hold an eight's
// first seven are read, and the eighth alone, nothing outside the matrix.  1024 tokens, 4095 k, bf16: r = 16 13.7 us (27.2 from the rows as they are, 4094
// k 11.9), r = 32 17.0 (39.3), r = 64 27.2 (63.5); 8192 tokens with 4095 columns of Y, r = 16: 67.5 (85).
template <typename T, bool ODD>
struct Long;
template <>
struct Long<float, false> {
    typedef float v8f __attribute__((ext_vector_type(8)));
    v8f v;
    __device__ __forceinline__ void clear() { v = {}; }
    __device__ __forceinline__ void load(const float* row, int k) { v = *reinterpret_cast<const Unaligned<float, 8>::type*>(row + k); }
    static __device__ __forceinline__ v4f mul(const Long& a, const float*, const Long& b, const float*, v4f c) {
#pragma unroll
        for (int i = 0; i < 8; ++i) c = __builtin_amdgcn_mfma_f32_16x16x4f32(a.v[i], b.v[i], c, 0, 0, 0);
        return c;
    }
};
__device__ __forceinline__ v4f mul_eights(v8bf a, v8bf b, v4f c) { return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0); }
__device__ __forceinline__ v4f mul_eights(v8h a, v8h b, v4f c) { return __builtin_amdgcn_mfma_f32_16x16x32_f16(a, b, c, 0, 0, 0); }
template <typename T>
struct Long<T, false> {
    typedef T v8 __attribute__((ext_vector_type(8)));
    v8 v;
    __device__ __forceinline__ void clear() { v = {}; }
    __device__ __forceinline__ void load(const T* row, int k) { v = *reinterpret_cast<const typename Unaligned<T, 8>::type*>(row + k); }
    static __device__ __forceinline__ v4f mul(const Long& a, const T*, const Long& b, const T*, v4f c) { return mul_eights(a.v, b.v, c); }
};
template <typename T>
struct Long<T, true> {
    typedef T v8 __attribute__((ext_vector_type(8)));
    v4u32 words;
    uint32_t last;
    __device__ __forceinline__ void clear() { words = v4u32{0, 0, 0, 0}, last = 0; }
    // (only rows behind the first lie so: there is an element before theirs)
    __device__ __forceinline__ void load(const T* row, int k) {
        words = *reinterpret_cast<const Unaligned<uint32_t, 4>::type*>(row - (reinterpret_cast<uintptr_t>(row) >> 1 & 1) + k);
        last = __builtin_bit_cast(uint16_t, row[k + 7]);
    }
    __device__ __forceinline__ v8 eight(const T* row) const {
        const uint32_t by = static_cast<uint32_t>(reinterpret_cast<uintptr_t>(row)) & 2u;
        v4u32 v;
#pragma unroll
        for (int i = 0; i < 4; ++i) v[i] = __builtin_amdgcn_alignbyte(i < 3 ? words[(i + 1) & 3] : last, words[i], by);
        return __builtin_bit_cast(v8, v);
    }
    static __device__ __forceinline__ v4f mul(const Long& a, const T* row_a, const Long& b, const T* row_b, v4f c) {
        return mul_eights(a.eight(row_a), b.eight(row_b), c);
    }
};

// Many tokens: a workgroup takes sixteen of them and 16 RT of the r rows, its wavefronts every eighth stretch of 128 k (RT = 1, 16-bit types), whose
// loads are in flight at once.  Those of the next stretch are asked for ahead of its products, but each eight's stand under a condition of their own, so that the
// compiler does not know how many are on their way and waits for all of them: stretches do not overlap.  This lane's sums over its
// wavefront's k: rows 4 (lane / 16) .. + 3 of each sixteen from r0 on, of token lane % 16.
// (sixteen wavefronts a tile where tiles do not fill the chip: 1024 x 4096 bf16 11.5 us, with eight 11.1.)
constexpr int kShrinkWaves = 8;
template <typename T, int RT, bool ODD>
__device__ __forceinline__ void shrink_tile(const T* __restrict__ x, const T* __restrict__ A, int K, const Adapters& a, int id, int r0, v4f (&out)[RT]) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, m = lane & 15, g = lane >> 4;
#pragma unroll
    for (int j = 0; j < RT; ++j) out[j] = v4f{0.f, 0.f, 0.f, 0.f};
    bool waiting = id >= 0;
    while (__any(waiting)) {
        const int now = __shfl(id, __ffsll(static_cast<unsigned long long>(__ballot(waiting))) - 1);
        const T* rows = A + static_cast<int64_t>(now) * a.r * K;
        v4f acc[RT];
#pragma unroll
        for (int j = 0; j < RT; ++j) acc[j] = v4f{0.f, 0.f, 0.f, 0.f};
        const T* mine[RT];
#pragma unroll
        for (int j = 0; j < RT; ++j) mine[j] = rows + static_cast<int64_t>(min(r0 + j * 16 + m, a.r - 1)) * K;
        // a stretch of k: its loads, then, with those of the next one on their way, its products
        constexpr int kAhead = RT == 1 ? 8 / static_cast<int>(sizeof(T)) - ODD : RT == 2 && sizeof(T) == 2 && !ODD ? 2 : 1, kStep = kShrinkWaves * 32 * kAhead;
        struct Stretch {
            Long<T, ODD> x[kAhead], a[kAhead][RT];
            // (eights that the row does not hold whole are zeros here)
            __device__ __forceinline__ void load(const T* from, const T* const (&rows)[RT], int64_t k0, int g, int K) {
#pragma unroll
                for (int u = 0; u < kAhead; ++u) {
                    const int64_t k = k0 + u * 32 + g * 8;
                    x[u].clear();
#pragma unroll
                    for (int j = 0; j < RT; ++j) a[u][j].clear();
                    if (k + 8 <= K) {
                        x[u].load(from, static_cast<int>(k));
#pragma unroll
                        for (int j = 0; j < RT; ++j) a[u][j].load(rows[j], static_cast<int>(k));
                    }
                }
            }
        };
        int64_t k0 = wave * 32 * kAhead;
        if (k0 < K) {
            Stretch cur, next;
            cur.load(x, mine, k0, g, K);
            for (; k0 < K; k0 += kStep) {
                const bool more = k0 + kStep < K;
                if (more) next.load(x, mine, k0 + kStep, g, K);
#pragma unroll
                for (int u = 0; u < kAhead; ++u)
#pragma unroll
                    for (int j = 0; j < RT; ++j) acc[j] = Long<T, ODD>::mul(cur.a[u][j], mine[j], cur.x[u], x, acc[j]);
                if (more) cur = next;
            }
        }
        if ((K & 7) != 0 && wave == kShrinkWaves - 1) {
            // the last few of a row: those of its last eight that no eight before holds
            const int again = g == 0 ? 8 - (K & 7) : 8;
            Long<T, false> xv, av;
            xv.load(x, K - 8);
#pragma unroll
            for (int i = 0; i < 8; ++i) xv.v[i] = i < again ? static_cast<T>(0.f) : xv.v[i];
#pragma unroll
            for (int j = 0; j < RT; ++j) {
                av.load(mine[j], K - 8);
#pragma unroll
                for (int i = 0; i < 8; ++i) av.v[i] = i < again ? static_cast<T>(0.f) : av.v[i];
                acc[j] = Long<T, false>::mul(av, mine[j], xv, x, acc[j]);
            }
        }
        if (id == now) {
#pragma unroll
            for (int j = 0; j < RT; ++j) out[j] = acc[j];
            waiting = false;
        }
    }
}
// The wavefronts' sums added up in LDS: put(token, row, sum) for each of the tile's.
template <int RT, typename Put>
__device__ __forceinline__ void shrink_join(const v4f (&out)[RT], float (&sums)[kShrinkWaves][RT][16][17], Put put) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, m = lane & 15, g = lane >> 4;
#pragma unroll
    for (int j = 0; j < RT; ++j)
#pragma unroll
        for (int v = 0; v < 4; ++v) sums[wave][j][m][g * 4 + v] = out[j][v];       // [token][row]
    __syncthreads();
    for (int i = threadIdx.x; i < RT * 256; i += 64 * kShrinkWaves) {
        const int j = i >> 8, token = (i >> 4) & 15;
        float u = 0.f;
#pragma unroll
        for (int w = 0; w < kShrinkWaves; ++w) u += sums[w][j][token][i & 15];
        put(token, j * 16 + (i & 15), u);
    }
}
template <typename T, int RT, bool ODD>
__global__ __launch_bounds__(64 * kShrinkWaves, RT == 4 && (ODD || sizeof(T) == 4) ? 2 : 4) void shrink_kernel(const T* __restrict__ X, int64_t ldx,
                                                                                                  const T* __restrict__ A, int K, Adapters a, int scaled,
                                                                                                  float* __restrict__ U) {
    __shared__ float sums[kShrinkWaves][RT][16][17];
    DAB_RESERVE_VGPRS();
    const int64_t t0 = static_cast<int64_t>(blockIdx.x) * 16, t = t0 + (threadIdx.x & 15);
    const int r0 = blockIdx.y * 16 * RT;
    v4f out[RT];
    shrink_tile<T, RT, ODD>(X + min(t, static_cast<int64_t>(a.T) - 1) * ldx, A, K, a, adapter_of(a, t), r0, out);
    shrink_join<RT>(out, sums, [&](int token, int row, float u) {
        if (t0 + token >= a.T || r0 + row >= a.r) return;
        const int who = adapter_of(a, t0 + token);
        U[(t0 + token) * a.r + r0 + row] = who < 0 ? 0.f : scaled ? u * scale_of(a, who) : u;
    });
}

// Rows of fewer than eight k: a thread takes a token and a row.
template <typename T>
__global__ __launch_bounds__(256) void shrink_narrow_kernel(const T* __restrict__ X, int64_t ldx, const T* __restrict__ A, int K, Adapters a, int scaled,
                                                            float* __restrict__ U) {
    const int64_t all = static_cast<int64_t>(a.T) * a.r;
    for (int64_t at = static_cast<int64_t>(blockIdx.x) * 256 + threadIdx.x; at < all; at += static_cast<int64_t>(gridDim.x) * 256) {
        const int64_t t = at / a.r, row = at - t * a.r;
        const int id = adapter_of(a, t);
        float u = 0.f;
        if (id >= 0) {
            for (int k = 0; k < K; ++k) u += static_cast<float>(X[t * ldx + k]) * static_cast<float>(A[(static_cast<int64_t>(id) * a.r + row) * K + k]);
            if (scaled) u *= scale_of(a, id);
        }
        U[at] = u;
    }
}

template <typename T>
__global__ __launch_bounds__(256) void shrink_few_kernel(const T* __restrict__ X, int64_t ldx, const T* __restrict__ A, int K, Adapters a, int scaled,
                                                         float* __restrict__ U) {
    DAB_RESERVE_VGPRS();
    shrink_few(X, ldx, A, K, a, scaled != 0, blockIdx.x, U);
}

// ---------------------------------------------------------------- expand
struct Base {
    const void* p;                   // or null
    int64_t ld;
    int dtype;                       // fp32, or the tokens'
};

// An element behind a place that all lanes share, by less than 2^32 bytes: the address is that place's scalar registers and 32 bits a lane.
template <typename T>
__device__ __forceinline__ T* past(T* shared, uint32_t elements) {
    typedef std::conditional_t<std::is_const_v<T>, const char, char> Byte;
    return reinterpret_cast<T*>(reinterpret_cast<Byte*>(shared) + static_cast<uint32_t>(elements * static_cast<uint32_t>(sizeof(T))));
}
// Values of N columns, without the first `again` of them.  Past the caches, which keep what the sums over tokens read next instead (8192 x 4096 bf16: 34
// us for those, 36.7 with ordinary stores, and 46.4 for the tile's own launch, 47.3).
template <typename T, int N>
__device__ __forceinline__ void store_own(T* to, int again, const float (&w)[N]) {
    if (again == 0) {
        typename Unaligned<T, N>::type v;
#pragma unroll
        for (int i = 0; i < N; ++i) v[i] = static_cast<T>(w[i]);
        __builtin_nontemporal_store(v, reinterpret_cast<typename Unaligned<T, N>::type*>(to));
    } else {
#pragma unroll
        for (int i = 1; i < N; ++i)
            if (i >= again) to[i] = static_cast<T>(w[i]);
    }
}

// Many tokens: a wavefront takes sixteen and 128 columns, lane l the columns 8 (l % 16) .. of tokens 4 (l / 16) .. + 3.  In fp32 on the
// matrix cores, whatever the type: U is fp32, and the products are few.  All that sixteen of the r rows need is in flight at once, base ahead of it.
// id: the adapter of token lane % 16; u_of(row): its U, times its scale.
template <typename T, typename TB, typename UOf>
__device__ __forceinline__ void expand_tile(const T* __restrict__ B, int F, const Adapters& a, const TB* base, int64_t ldbase, T* Y, int64_t t0, int64_t f0,
                                            int id, UOf u_of) {
    const int lane = threadIdx.x & 63, m = lane & 15, g = lane >> 4;
    // (a lane whose eight columns pass the row's end takes the last eight, and stores those that are its own)
    const int f = min(static_cast<int>(f0) + m * 8, F - 8), again = static_cast<int>(f0) + m * 8 - f;
    // one adapter after the other, -1 among them; of sequences' tokens there is one
    bool waiting = true;
    while (__any(waiting)) {
        const int now = __builtin_amdgcn_readfirstlane(__shfl(id, __ffsll(static_cast<unsigned long long>(__ballot(waiting))) - 1));
        waiting = waiting && id != now;
        Eight<TB> y[4];
        bool mine[4];
#pragma unroll
        for (int v = 0; v < 4; ++v) {
            mine[v] = __shfl(id, 4 * g + v) == now && t0 + 4 * g + v < a.T && again < 8;
            y[v].v = {};
            if (base && mine[v]) y[v].load_once(past(base + t0 * ldbase, (4 * g + v) * static_cast<uint32_t>(ldbase) + f), 0);
        }
        v4f out[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) out[j] = v4f{0.f, 0.f, 0.f, 0.f};
        if (now >= 0) {
            const T* rows = B + static_cast<int64_t>(now) * a.r * F;
            for (int q0 = 0; q0 < a.r; q0 += 16) {
                Eight<T> b[4];
                float u[4];
#pragma unroll
                for (int q = 0; q < 4; ++q) {
                    const int row = q0 + 4 * q + g;
                    b[q].v = {}, u[q] = 0.f;
                    if (row < a.r) {
                        b[q].load(past(rows, static_cast<uint32_t>(row) * F + f), 0);
                        if (id == now) u[q] = u_of(row);
                    }
                }
#pragma unroll
                for (int q = 0; q < 4; ++q)
#pragma unroll
                    for (int j = 0; j < 8; ++j) out[j] = __builtin_amdgcn_mfma_f32_16x16x4f32(u[q], b[q][j], out[j], 0, 0, 0);
            }
        }
#pragma unroll
        for (int v = 0; v < 4; ++v) {
            if (!mine[v]) continue;
            float w[8];
#pragma unroll
            for (int j = 0; j < 8; ++j) w[j] = y[v][j] + out[j][v];
            store_own(past(Y + t0 * F, (4 * g + v) * static_cast<uint32_t>(F) + f), again, w);
        }
    }
}

// 8192 x 4096 bf16, r = 16, base added: 34.3 us, 3.9 TB/s.  Measured and left: tiles of 16 x 64 40.6 us, base and U on their way before the ids 39 (registers),
// several tiles a wavefront with the next one's loads ahead 74 (registers), products in bf16 pieces of U 42 (registers).
constexpr int kExpandWaves = 4;
template <typename T, typename TB>
__global__ __launch_bounds__(64 * kExpandWaves, sizeof(TB) == 4 ? 3 : 4) void expand_kernel(const float* __restrict__ U, const T* __restrict__ B, int F,
                                                                                        Adapters a, int scaled, const TB* base, int64_t ldbase, T* Y) {
    DAB_RESERVE_VGPRS();
    const int64_t t0 = (static_cast<int64_t>(blockIdx.z) * gridDim.y + blockIdx.y) * 16;
    const int64_t f0 = (static_cast<int64_t>(blockIdx.x) * kExpandWaves + (threadIdx.x >> 6)) * 128;
    if (f0 >= F || t0 >= a.T) return;
    const int64_t t = t0 + (threadIdx.x & 15);
    const int id = adapter_of(a, t);
    const float s = id >= 0 && scaled ? scale_of(a, id) : 1.f;
    expand_tile<T, TB>(B, F, a, base, ldbase, Y, t0, f0, id, [&](int row) { return U[t * a.r + row] * s; });
}

// Columns 2 d and 2 d + 1 of eight rows' eight columns, as the matrix cores take the rows: eight numbers of a column a lane.
__device__ __forceinline__ void columns(const v4u32 (&x)[8], int d, v8bf* even, v8bf* odd) {
    v4u32 p, q;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        p[i] = __builtin_amdgcn_perm(x[2 * i + 1][d], x[2 * i][d], 0x05040100u);
        q[i] = __builtin_amdgcn_perm(x[2 * i + 1][d], x[2 * i][d], 0x07060302u);
    }
    *even = __builtin_bit_cast(v8bf, p), *odd = __builtin_bit_cast(v8bf, q);
}

// The same tile on the bf16 matrix instruction, with U as three bf16 numbers in LDS, [piece][token][row], whose sum it is, so that products stay exact.  Of
// the 32 numbers that an instruction adds up the first sixteen are one piece times sixteen rows, the others another piece times the
// same rows; eight rows of eight columns are transposed in a lane's registers.
template <int RT>
struct Pieces {
    static constexpr int kRow = 16 * RT + 8;
    __attribute__((aligned(16))) bf16 v[3][16][kRow];
};
template <typename TB, int RT>
__device__ __forceinline__ void expand_tile16(const bf16* __restrict__ B, int F, const Adapters& a, const TB* base, int64_t ldbase, bf16* Y, int64_t t0,
                                              int64_t f0, int id, const Pieces<RT>& u) {
    const int lane = threadIdx.x & 63, m = lane & 15, g = lane >> 4;
    const int f = min(static_cast<int>(f0) + m * 8, F - 8), again = static_cast<int>(f0) + m * 8 - f;
    bool waiting = true;
    while (__any(waiting)) {
        // (offsets are made anew where they are used: kept over the columns they take the registers of the loads)
        uint32_t step_base = static_cast<uint32_t>(ldbase), step_y = F;
        asm volatile("" : "+s"(step_base), "+s"(step_y));
        const int now = __builtin_amdgcn_readfirstlane(__shfl(id, __ffsll(static_cast<unsigned long long>(__ballot(waiting))) - 1));
        waiting = waiting && id != now;
        Eight<TB> y[4];
        bool mine[4];
#pragma unroll
        for (int v = 0; v < 4; ++v) {
            mine[v] = __shfl(id, 4 * g + v) == now && t0 + 4 * g + v < a.T && again < 8;
            y[v].v = {};
            if (base && mine[v]) y[v].load_once(past(base + t0 * ldbase, (4 * g + v) * step_base + f), 0);
        }
        v4f out[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) out[j] = v4f{0.f, 0.f, 0.f, 0.f};
        if (now >= 0) {
            const bf16* rows = B + static_cast<int64_t>(now) * a.r * F;
            for (int q0 = 0; q0 < a.r; q0 += 16) {
                const int row0 = q0 + 8 * (g & 1);
                uint32_t step = F;
                asm volatile("" : "+s"(step));
                v4u32 b[8];
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    b[e] = v4u32{0, 0, 0, 0};
                    if (row0 + e < a.r) {
                        Eight<bf16> w;
                        w.load(past(rows, static_cast<uint32_t>(row0 + e) * step + f), 0);
                        b[e] = __builtin_bit_cast(v4u32, w.v);
                    }
                }
                v8bf p = *reinterpret_cast<const v8bf*>(&u.v[g < 2 ? 0 : 1][m][row0]), q = *reinterpret_cast<const v8bf*>(&u.v[2][m][row0]);
                if (id != now) p = v8bf{}, q = v8bf{};
                if (g >= 2) q = v8bf{};
#pragma unroll
                for (int d = 0; d < 4; ++d) {
                    v8bf even, odd;
                    columns(b, d, &even, &odd);
                    out[2 * d] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(p, even, out[2 * d], 0, 0, 0);
                    out[2 * d + 1] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(p, odd, out[2 * d + 1], 0, 0, 0);
                    out[2 * d] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(q, even, out[2 * d], 0, 0, 0);
                    out[2 * d + 1] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(q, odd, out[2 * d + 1], 0, 0, 0);
                }
            }
        }
#pragma unroll
        for (int v = 0; v < 4; ++v) {
            if (!mine[v]) continue;
            float w[8];
#pragma unroll
            for (int j = 0; j < 8; ++j) w[j] = y[v][j] + out[j][v];
            store_own(past(Y + t0 * F, (4 * g + v) * step_y + f), again, w);
        }
    }
}

// Both in one launch, for tiles that fill the chip: a workgroup's eight wavefronts share the tile's k, then its columns, with U in LDS between.  U goes out
// as well (times the scale where `scaled`).  What is left above the time of its bytes: all workgroups are resident at once and read, then write, in step.
template <typename T, typename TB, int RT, bool ODD>
__global__ __launch_bounds__(64 * kShrinkWaves, sizeof(T) == 4 || (RT == 4 && ODD) ? 2 : 4) void shrink_expand_kernel(
    const T* __restrict__ X, int64_t ldx, const T* __restrict__ A, int K, const T* __restrict__ B, int F, Adapters a, int scaled, float* __restrict__ U,
    const TB* base, int64_t ldbase, T* Y) {
    constexpr bool k16 = std::is_same_v<T, bf16> && sizeof(TB) == 2;          // (with an fp32 base its registers are not left)
    struct Floats {
        float v[16][16 * RT + 1];
    };
    __shared__ float sums[kShrinkWaves][RT][16][17];
    __shared__ std::conditional_t<k16, Pieces<RT>, Floats> kept;
    DAB_RESERVE_VGPRS();
    const int m = threadIdx.x & 15;
    const int64_t t0 = static_cast<int64_t>(blockIdx.x) * 16;
    const int id = adapter_of(a, t0 + m);
    v4f out[RT];
    shrink_tile<T, RT, ODD>(X + min(t0 + m, static_cast<int64_t>(a.T) - 1) * ldx, A, K, a, id, 0, out);
    shrink_join<RT>(out, sums, [&](int token, int row, float u) {
        const int who = adapter_of(a, t0 + token);
        const float by = who < 0 ? 0.f : u * scale_of(a, who);
        if constexpr (k16) {
#pragma unroll
            for (int p = 0; p < 3; ++p) kept.v[p][token][row] = piece_of(row < a.r ? by : 0.f, p);
        } else {
            kept.v[token][row] = by;
        }
        if (t0 + token < a.T && row < a.r) U[(t0 + token) * a.r + row] = scaled ? by : who < 0 ? 0.f : u;
    });
    __syncthreads();
    for (int64_t f0 = static_cast<int64_t>(threadIdx.x >> 6) * 128; f0 < F; f0 += 128 * kShrinkWaves) {
        if constexpr (k16) expand_tile16<TB, RT>(B, F, a, base, ldbase, Y, t0, f0, id, kept);
        else expand_tile<T, TB>(B, F, a, base, ldbase, Y, t0, f0, id, [&](int row) { return kept.v[m][row]; });
    }
}

// Rows of fewer than eight columns: a thread takes a token.
template <typename T, typename TB>
__global__ __launch_bounds__(256) void expand_narrow_kernel(const float* __restrict__ U, const T* __restrict__ B, int F, Adapters a, int scaled,
                                                            const TB* base, int64_t ldbase, T* Y) {
    const int64_t t = static_cast<int64_t>(blockIdx.x) * 256 + threadIdx.x;
    if (t >= a.T) return;
    const int id = adapter_of(a, t);
    const float s = id >= 0 && scaled ? scale_of(a, id) : 1.f;
    for (int f = 0; f < F; ++f) {
        float v = 0.f;
        if (id >= 0)
            for (int row = 0; row < a.r; ++row) v += (U[t * a.r + row] * s) * static_cast<float>(B[(static_cast<int64_t>(id) * a.r + row) * F + f]);
        Y[t * F + f] = static_cast<T>((base ? static_cast<float>(base[t * ldbase + f]) : 0.f) + v);
    }
}

// Few tokens: a lane takes eight columns of one, the last eight of a row, and stores those that are its own, where fewer are left (read one by one there,
// r = 24, rows of 8005 and 2672, bf16: 10.4 us on average, now 6.5).
template <typename T, typename TB>
__global__ __launch_bounds__(64) void expand_few_kernel(const float* __restrict__ U, const T* __restrict__ B, int F, Adapters a, int scaled,
                                                        const TB* base, int64_t ldbase, T* Y) {
    DAB_RESERVE_VGPRS();
    const int64_t t = blockIdx.y, f64 = (static_cast<int64_t>(blockIdx.x) * 64 + threadIdx.x) * 8;
    if (f64 >= F) return;
    const int id = adapter_of(a, t);
    const T* rows = B + static_cast<int64_t>(max(id, 0)) * a.r * F;
    const float s = id >= 0 && scaled ? scale_of(a, id) : 1.f;
    const float* u = U + t * a.r;
    const int r = id >= 0 ? a.r : 0;
    if (F < kNarrow) {
        for (int c = 0; c < F; ++c) {
            float v = 0.f;
            for (int row = 0; row < r; ++row) v += (u[row] * s) * static_cast<float>(rows[static_cast<int64_t>(row) * F + c]);
            Y[t * F + c] = static_cast<T>((base ? static_cast<float>(base[t * ldbase + c]) : 0.f) + v);
        }
        return;
    }
    const int f = static_cast<int>(min(f64, static_cast<int64_t>(F) - 8)), again = static_cast<int>(f64) - f;
    Eight<TB> y;
    y.v = {};
    if (base) y.load(base + t * ldbase, f);
    float v[8] = {};
#pragma unroll 8
    for (int row = 0; row < r; ++row) {
        Eight<T> b;
        b.load(rows + static_cast<int64_t>(row) * F, f);
        const float by = u[row] * s;
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] += by * b[i];
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] += y[i];
    store_own(Y + t * F + f, again, v);
}

// ---------------------------------------------------------------- outer
// Both gradients of the adapters in one launch: a workgroup takes 128 columns of one, sixteen of the r rows, a share of the tokens and every
// slices-th adapter.  Of each adapter that has tokens in its share they are listed, dealt out to the wavefronts and the sums added up in LDS (every
// wavefront its own stretch of the tokens instead, so that half of them wait where sequences are short: 41 us instead of 35).  With one
// share that is the gradient; else it goes to parts: [share][adapter][r][columns], and have: [share][adapter] is 1 where the share has
// tokens of the adapter (other parts are not written).  Sixteen rows a workgroup whatever the rank, each of which reads X and dY again: these sums of r = 64,
// four adapters, took 84 us, with 32 rows 84 and a longer join, with 64 rows 102 (registers); they take 80 now, of f16, on the fp32 instruction, 128.
// bf16 products with three pieces of V instead of fp32 ones: 49 -> 37 us.
constexpr int kOuterWaves = 8, kOuterIds = 2048;
template <typename T>
struct OuterSide {
    const float* V;                  // [tokens][r]
    const T* X;
    int64_t ldx;
    int cols, scaled;
    float* out;                      // the gradient, or parts
};
template <typename T>
struct Outer {
    OuterSide<T> side[2];
    int tiles0, tiles;               // column tiles of the first side, of both
    int tokens, shares, slices;      // tokens of a share (a multiple of 32); slices of the adapters
    int32_t* have;
};
template <typename T>
__global__ __launch_bounds__(64 * kOuterWaves) void outer_kernel(const Adapters a, const Outer<T> o) {
    extern __shared__ uint32_t present[];                    // a bit for every adapter
    __shared__ float sums[kOuterWaves][8][132];
    __shared__ int ids[kOuterIds];
    __shared__ __attribute__((aligned(16))) uint16_t list[kOuterIds];
    __shared__ int counts[kOuterWaves];
    DAB_RESERVE_VGPRS();
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), m = lane & 15, g = lane >> 4;
    const int rb = blockIdx.x / o.tiles, tile2 = blockIdx.x - rb * o.tiles;
    const bool second = tile2 >= o.tiles0;
    const OuterSide<T> side = o.side[second];
    const int tile = second ? tile2 - o.tiles0 : tile2, share = blockIdx.y, slice = blockIdx.z, r0 = rb * 16, cols = side.cols;
    const int64_t first = static_cast<int64_t>(share) * o.tokens;
    const int count = static_cast<int>(min(static_cast<int64_t>(o.tokens), a.T - first));
    const int words = (a.n + 31) >> 5;
    const bool kept = count <= kOuterIds;                    // the share's ids in LDS
    for (int i = threadIdx.x; i < words; i += 64 * kOuterWaves) present[i] = 0;
    __syncthreads();
    for (int t = threadIdx.x; t < count; t += 64 * kOuterWaves) {
        const int id = adapter_of(a, first + t);
        if (kept) ids[t] = id;
        if (id >= 0) atomicOr(&present[id >> 5], 1u << (id & 31));
    }
    __syncthreads();
    if (o.shares > 1 && tile2 == 0 && rb == 0)
        for (int i = slice + threadIdx.x * o.slices; i < a.n; i += 64 * kOuterWaves * o.slices)
            o.have[static_cast<int64_t>(share) * a.n + i] = (present[i >> 5] >> (i & 31)) & 1u;
    const bool whole = tile * 128 + 128 <= cols;
    const int c = min(tile * 128 + m * 8, cols - 8), again = tile * 128 + m * 8 - c;         // (as in expand)
    const T* x0 = side.X + first * side.ldx;
    const float* v0 = side.V + first * a.r;
    for (int id = slice; id < a.n; id += o.slices) {
        const bool none = !((present[id >> 5] >> (id & 31)) & 1u);          // (the same for the whole workgroup)
        if (none && o.shares > 1) continue;
        const float s = side.scaled && !none ? scale_of(a, id) : 1.f;       // (zeros stay zeros)
        v4f acc[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) acc[i] = v4f{0.f, 0.f, 0.f, 0.f};
        for (int w0 = none ? count : 0; w0 < count; w0 += kOuterIds) {
            // the adapter's tokens among the next ones, in their order
            uint64_t hits[kOuterIds / 64 / kOuterWaves];
            int found = 0;
#pragma unroll
            for (int k = 0; k < kOuterIds / 64 / kOuterWaves; ++k) {
                const int t = w0 + (wave * (kOuterIds / 64 / kOuterWaves) + k) * 64 + lane;
                hits[k] = __ballot(t < count && (kept ? ids[t] : a.ids[first + t]) == id);
                found += __popcll(hits[k]);
            }
            if (lane == 0) counts[wave] = found;
            __syncthreads();
            int before = 0, c_tokens = 0;
#pragma unroll
            for (int k = 0; k < kOuterWaves; ++k) {
                if (k == wave) before = c_tokens;
                c_tokens += counts[k];
            }
#pragma unroll
            for (int k = 0; k < kOuterIds / 64 / kOuterWaves; ++k) {
                if ((hits[k] >> lane) & 1)
                    list[before + __popcll(hits[k] & ((uint64_t{1} << lane) - 1))] =
                        static_cast<uint16_t>((wave * (kOuterIds / 64 / kOuterWaves) + k) * 64 + lane);
                before += __popcll(hits[k]);
            }
            __syncthreads();
            if constexpr (std::is_same_v<T, bf16>) {
                // 32 tokens a step and wavefront, eight of them a lane: V as the sum of three bf16 numbers, eight rows of eight columns transposed in
                // the lane's registers
                for (int i0 = 0; i0 < c_tokens; i0 += 32 * kOuterWaves) {
                    const int p0 = i0 + (g * kOuterWaves + wave) * 8;
                    if (!__any(p0 < c_tokens)) continue;
                    const v4u32 eight = *reinterpret_cast<const v4u32*>(&list[min(p0, kOuterIds - 8)]);
                    v4u32 x[8];
                    float v[8];
#pragma unroll
                    for (int e = 0; e < 8; ++e) {
                        const int64_t t = w0 + ((eight[e / 2] >> (16 * (e & 1))) & 0xffffu);
                        Eight<bf16> w;
                        w.v = {}, v[e] = 0.f;
                        if (p0 + e < c_tokens) {
                            w.load(x0 + t * side.ldx, c);
                            if (r0 + m < a.r) v[e] = v0[t * a.r + r0 + m];
                        }
                        x[e] = __builtin_bit_cast(v4u32, w.v);
                    }
                    v8bf p[3];
#pragma unroll
                    for (int k = 0; k < 3; ++k)
#pragma unroll
                        for (int e = 0; e < 8; ++e) p[k][e] = piece_of(v[e], k);
#pragma unroll
                    for (int d = 0; d < 4; ++d) {
                        v8bf even, odd;
                        columns(x, d, &even, &odd);
#pragma unroll
                        for (int k = 0; k < 3; ++k) {
                            acc[2 * d] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(p[k], even, acc[2 * d], 0, 0, 0);
                            acc[2 * d + 1] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(p[k], odd, acc[2 * d + 1], 0, 0, 0);
                        }
                    }
                }
            } else {
                // four tokens a step and wavefront, one a lane, several steps in flight
                constexpr int kAhead = 4;
                for (int i0 = 0; i0 < c_tokens; i0 += 4 * kOuterWaves * kAhead) {
                    Eight<T> x[kAhead];
                    float v[kAhead];
#pragma unroll
                    for (int u = 0; u < kAhead; ++u) {
                        const int p0 = i0 + (u * kOuterWaves + wave) * 4 + g;
                        x[u].v = {}, v[u] = 0.f;
                        if (p0 < c_tokens) {
                            const int64_t t = w0 + list[p0];
                            x[u].load(x0 + t * side.ldx, c);
                            if (r0 + m < a.r) v[u] = v0[t * a.r + r0 + m];
                        }
                    }
#pragma unroll
                    for (int u = 0; u < kAhead; ++u)
                        if (i0 + (u * kOuterWaves + wave) * 4 < c_tokens)
#pragma unroll
                            for (int i = 0; i < 8; ++i) acc[i] = __builtin_amdgcn_mfma_f32_16x16x4f32(v[u], x[u][i], acc[i], 0, 0, 0);
                }
            }
        }
        // rows 4 g + v of 16, columns 8 m + i of 128: every wavefront's into LDS, then a thread adds up four columns
        float* out = side.out + (static_cast<int64_t>(o.shares > 1 ? share : 0) * a.n + id) * a.r * cols;
#pragma unroll
        for (int j = 0; j < 2; ++j) {                        // (eight of the rows at a time: those of v = 0 and 1, then of 2 and 3)
            if (!none)
#pragma unroll
                for (int i = 0; i < 8; i += 4)
#pragma unroll
                    for (int h = 0; h < 2; ++h) {
                        const int v = 2 * j + h;
                        if (again == 0) {
                            *reinterpret_cast<v4f*>(&sums[wave][2 * g + h][m * 8 + i]) =
                                v4f{acc[i][v], acc[i + 1][v], acc[i + 2][v], acc[i + 3][v]};
                        } else if (again < 8) {
#pragma unroll
                            for (int k = 0; k < 4; ++k)
                                if (i + k >= again) sums[wave][2 * g + h][m * 8 + i + k - again] = acc[i + k][v];
                        }
                    }
            __syncthreads();
            const int at = threadIdx.x >> 5, col = (threadIdx.x & 31) * 4, row = r0 + 4 * (at >> 1) + 2 * j + (at & 1);
            if (at < 8 && row < a.r) {
                v4f w = v4f{0.f, 0.f, 0.f, 0.f};
                if (!none)
#pragma unroll
                    for (int k = 0; k < kOuterWaves; ++k) w += *reinterpret_cast<const v4f*>(&sums[k][at][col]);
                float* to = out + static_cast<int64_t>(row) * cols + tile * 128 + col;
                if (whole) {
                    *reinterpret_cast<Unaligned<float, 4>::type*>(to) = w * s;
                } else {
#pragma unroll
                    for (int i = 0; i < 4; ++i)
                        if (tile * 128 + col + i < cols) to[i] = w[i] * s;
                }
            }
            __syncthreads();
        }
    }
}

// Rows of fewer than eight columns: a workgroup takes a row of an adapter.
template <typename T>
__global__ __launch_bounds__(256) void outer_narrow_kernel(const Adapters a, const OuterSide<T> side) {
    __shared__ float sums[4];
    const int row = blockIdx.x, id = blockIdx.y;
    for (int c = 0; c < side.cols; ++c) {
        float v = 0.f;
        bool any = false;
        for (int64_t t = threadIdx.x; t < a.T; t += 256)
            if (a.ids[t] == id) v += side.V[t * a.r + row] * static_cast<float>(side.X[t * side.ldx + c]), any = true;
        v = lanes_sum<6>(v);
        if ((threadIdx.x & 63) == 0) sums[threadIdx.x >> 6] = v;
        any = __syncthreads_or(any);
        if (threadIdx.x == 0)
            side.out[(static_cast<int64_t>(id) * a.r + row) * side.cols + c] =
                any ? ((sums[0] + sums[1]) + (sums[2] + sums[3])) * (side.scaled ? scale_of(a, id) : 1.f) : 0.f;
        __syncthreads();
    }
}

// The shares' parts of both gradients added in a fixed order; zeros for an adapter without tokens.
struct Join {
    const float* parts[2];
    float* out[2];
    int64_t size[2];                 // of an adapter
    unsigned blocks0;                // workgroups of the first
    const int32_t* have;
    int shares, n;
};
// (a lane four neighbouring elements, the workgroup's four wavefronts every fourth share: whether it has a part is waited for, then the part, share by share,
// 5.6 us for 15 MB)
__global__ __launch_bounds__(256) void outer_join_kernel(const Join j) {
    __shared__ v4f sums[3][64];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const bool second = blockIdx.x >= j.blocks0;
    const int64_t at = (static_cast<int64_t>(second ? blockIdx.x - j.blocks0 : blockIdx.x) * 64 + lane) * 4, size = j.size[second];
    const int id = blockIdx.y, left = static_cast<int>(max(min(size - at, int64_t{4}), int64_t{0}));
    v4f v = v4f{0.f, 0.f, 0.f, 0.f};
#pragma unroll 4
    for (int s = wave; s < j.shares; s += 4) {
        const int64_t who = static_cast<int64_t>(s) * j.n + id;
        if (!j.have[who]) continue;
        const float* from = j.parts[second] + who * size + at;
        if (left == 4) {
            v += static_cast<v4f>(*reinterpret_cast<const Unaligned<float, 4>::type*>(from));
        } else {
            for (int i = 0; i < left; ++i) v[i] += from[i];
        }
    }
    if (wave) sums[wave - 1][lane] = v;
    __syncthreads();
    if (wave) return;
    v = (v + sums[0][lane]) + (sums[1][lane] + sums[2][lane]);
    float* to = j.out[second] + static_cast<int64_t>(id) * size + at;
    for (int i = 0; i < left; ++i) to[i] = v[i];
}

// ---------------------------------------------------------------- host side
constexpr int kMaxRank = 256, kAdapterCols = 1 << 21;         // (a row block of an adapter and sixteen tokens stay below 2^32 bytes)
constexpr int64_t kAdapterLd = 1 << 25;

static bool odd_rows(int64_t ldx, int K) { return ((ldx | K) & 1) != 0; }

template <typename T>
static int shrink(const T* X, int64_t ldx, const T* A, int K, const Adapters& a, bool scaled, float* U, hipStream_t st) {
    // A workgroup for every token and row, or for sixteen tokens: the one's time grows with tokens, rows and k, the other's with k alone until its workgroups
    // fill the chip.  bf16, r = 16, rows of 4096: 128 tokens 5.2 us and 10.8, 256 8.7 and 10.8, 512 14.1 and 11.0; of 1024, 256 tokens 6.0 and 4.9.  The
    // limit is that of rows of up to some 8192 and too high for longer ones (with the 1100 columns of Y behind it, tokens in four runs of one adapter
    // each: 8192, 288 tokens 19 us and 37, 576 24 and 21; 16384, 544 35 and 66, 1088 56 and 37; 65536, 1040 200 and 232, 4080 820 and 240).
    if (static_cast<int64_t>(a.T) * a.r <= 1024 + K)
        return launch(shrink_few_kernel<T>, dim3(a.T * a.r), dim3(64 * kFewWaves), 0, st, X, ldx, A, K, a, static_cast<int>(scaled), U);
    const unsigned tiles = static_cast<unsigned>(ceil_div64(a.T, 16));
    const dim3 block(64 * kShrinkWaves);
    const int s = scaled;
    if (K < kNarrow)
        return launch(shrink_narrow_kernel<T>, dim3(static_cast<unsigned>(std::min<int64_t>(ceil_div64(static_cast<int64_t>(a.T) * a.r, 256), 1 << 20))), dim3(256),
                      0, st, X, ldx, A, K, a, s, U);
    const auto go = [&](auto odd) {
        constexpr bool ODD = sizeof(T) == 2 && decltype(odd)::value;
        if (a.r <= 16) return launch(shrink_kernel<T, 1, ODD>, dim3(tiles), block, 0, st, X, ldx, A, K, a, s, U);
        if (a.r <= 32) return launch(shrink_kernel<T, 2, ODD>, dim3(tiles), block, 0, st, X, ldx, A, K, a, s, U);
        return launch(shrink_kernel<T, 4, ODD>, dim3(tiles, ceil_div(a.r, 64)), block, 0, st, X, ldx, A, K, a, s, U);
    };
    return odd_rows(ldx, K) ? go(std::true_type{}) : go(std::false_type{});
}

template <typename T, typename TB>
static int expand_from(const float* U, const T* B, int F, const Adapters& a, bool scaled, const Base& base, T* Y, hipStream_t st) {
    const TB* p = static_cast<const TB*>(base.p);
    const int s = scaled;
    if (a.T <= kFewTokens)
        return launch(expand_few_kernel<T, TB>, dim3(static_cast<unsigned>(ceil_div64(F, 512)), a.T), dim3(64), 0, st, U, B, F, a, s, p, base.ld, Y);
    if (F < kNarrow)
        return launch(expand_narrow_kernel<T, TB>, dim3(static_cast<unsigned>(ceil_div64(a.T, 256))), dim3(256), 0, st, U, B, F, a, s, p, base.ld, Y);
    // (token tiles along y and z: more than 65535 of them)
    const int64_t tiles = ceil_div64(a.T, 16);
    const dim3 grid(static_cast<unsigned>(ceil_div64(F, 128 * kExpandWaves)), static_cast<unsigned>(std::min<int64_t>(tiles, 32768)),
                    static_cast<unsigned>(ceil_div64(tiles, 32768))), block(64 * kExpandWaves);
    return launch(expand_kernel<T, TB>, grid, block, 0, st, U, B, F, a, s, p, base.ld, Y);
}
template <typename T>
static int expand(const float* U, const T* B, int F, const Adapters& a, bool scaled, const Base& base, T* Y, hipStream_t st) {
    return base.p && base.dtype == DAB_F32 ? expand_from<T, float>(U, B, F, a, scaled, base, Y, st) : expand_from<T, T>(U, B, F, a, scaled, base, Y, st);
}

// U and Y (or V and dX): one launch of up to 64 rows where the tiles fill the chip, or the columns are one round of a workgroup's wavefronts.  8192 tokens,
// 4096 -> 4096, r = 16, bf16: 46 us, in two launches 22 + 34; 1999 tokens, 777 -> 301, r = 5, f16: 8.7, 4.8 + 5.5.
template <typename T, typename TB, int RT>
static int shrink_expand_from(const T* X, int64_t ldx, const T* A, int K, const T* B, int F, const Adapters& a, bool scaled, float* U, const Base& base, T* Y,
                              hipStream_t st) {
    const auto go = [&](auto odd) {
        constexpr bool ODD = sizeof(T) == 2 && decltype(odd)::value;
        return launch(shrink_expand_kernel<T, TB, RT, ODD>, dim3(static_cast<unsigned>(ceil_div64(a.T, 16))), dim3(64 * kShrinkWaves), 0, st, X, ldx, A, K, B, F,
                      a, static_cast<int>(scaled), U, static_cast<const TB*>(base.p), base.ld, Y);
    };
    return odd_rows(ldx, K) ? go(std::true_type{}) : go(std::false_type{});
}
template <typename T>
static int shrink_expand(const T* X, int64_t ldx, const T* A, int K, const T* B, int F, const Adapters& a, bool scaled, float* U, const Base& base, T* Y,
                         hipStream_t st) {
    const int64_t tiles = ceil_div64(a.T, 16);
    if (a.T > kFewTokens && a.r <= 64 && K >= kNarrow && F >= kNarrow && (tiles >= kNumCU || F <= 128 * kShrinkWaves)) {
        const bool wide = base.p && base.dtype == DAB_F32 && sizeof(T) == 2;
        if (wide) {
            if (a.r <= 16) return shrink_expand_from<T, float, 1>(X, ldx, A, K, B, F, a, scaled, U, base, Y, st);
            if (a.r <= 32) return shrink_expand_from<T, float, 2>(X, ldx, A, K, B, F, a, scaled, U, base, Y, st);
            return shrink_expand_from<T, float, 4>(X, ldx, A, K, B, F, a, scaled, U, base, Y, st);
        }
        if (a.r <= 16) return shrink_expand_from<T, T, 1>(X, ldx, A, K, B, F, a, scaled, U, base, Y, st);
        if (a.r <= 32) return shrink_expand_from<T, T, 2>(X, ldx, A, K, B, F, a, scaled, U, base, Y, st);
        return shrink_expand_from<T, T, 4>(X, ldx, A, K, B, F, a, scaled, U, base, Y, st);
    }
    if (int rc = shrink(X, ldx, A, K, a, scaled, U, st)) return rc;
    return expand(static_cast<const float*>(U), B, F, a, !scaled, base, Y, st);
}

struct OuterPlan {
    int shares, tokens, slices, tiles0, tiles, row_blocks;
    size_t parts0, parts1, have;     // bytes, multiples of 256
    size_t bytes() const { return parts0 + parts1 + have; }
};
static OuterPlan outer_plan(int T, int n, int r, int cols0, int cols1) {
    OuterPlan p{};
    p.row_blocks = ceil_div(r, 16), p.tiles0 = ceil_div(cols0, 128), p.tiles = p.tiles0 + ceil_div(cols1, 128);
    const int64_t blocks = static_cast<int64_t>(p.tiles) * p.row_blocks, row = static_cast<int64_t>(n) * r * 4;
    // about two workgroups for every compute unit, shares of at least 128 tokens, parts of at most 256 MB
    int64_t shares = ceil_div64(2 * kNumCU, blocks);
    shares = std::min<int64_t>(shares, ceil_div64(T, 128));
    shares = std::max<int64_t>(1, std::min<int64_t>(shares, (int64_t{256} << 20) / (row * (static_cast<int64_t>(cols0) + cols1))));
    p.tokens = static_cast<int>(round_up(ceil_div64(T, shares), 32));
    p.shares = static_cast<int>(ceil_div64(T, p.tokens));
    p.slices = static_cast<int>(std::max<int64_t>(1, std::min<int64_t>(std::min(n, 1024), 2 * kNumCU / (blocks * p.shares))));
    if (p.shares > 1)
        p.parts0 = round_up(row * cols0 * p.shares, 256), p.parts1 = round_up(row * cols1 * p.shares, 256), p.have = round_up(static_cast<int64_t>(p.shares) * n * 4, 256);
    return p;
}
// Both sides of the gradients: out[i] = sum over adapter i's tokens of V^T X, times scale[i] where `scaled`.
template <typename T>
static int outer(const OuterSide<T> (&sides)[2], const Adapters& a, char* ws, hipStream_t st) {
    OuterSide<T> wide[2];
    int n = 0;
    for (const OuterSide<T>& s : sides) {
        if (s.cols >= kNarrow) wide[n++] = s;
        else if (int rc = launch(outer_narrow_kernel<T>, dim3(a.r, a.n), dim3(256), 0, st, a, s)) return rc;
    }
    if (n == 0) return DAB_OK;
    if (n == 1) wide[1] = wide[0], wide[1].cols = 0;
    const OuterPlan p = outer_plan(a.T, a.n, a.r, wide[0].cols, wide[1].cols);
    Outer<T> o{};
    Join j{};
    j.out[0] = wide[0].out, j.out[1] = wide[1].out;
    if (p.shares > 1) {
        wide[0].out = reinterpret_cast<float*>(ws), wide[1].out = reinterpret_cast<float*>(ws + p.parts0);
        o.have = reinterpret_cast<int32_t*>(ws + p.parts0 + p.parts1);
    }
    o.side[0] = wide[0], o.side[1] = wide[1], o.tiles0 = p.tiles0, o.tiles = p.tiles, o.tokens = p.tokens, o.shares = p.shares, o.slices = p.slices;
    const dim3 grid(static_cast<unsigned>(static_cast<int64_t>(p.tiles) * p.row_blocks), p.shares, p.slices), block(64 * kOuterWaves);
    const size_t lds = static_cast<size_t>(ceil_div(a.n, 32)) * 4;
    const int rc = launch(outer_kernel<T>, grid, block, lds, st, a, o);
    if (rc || p.shares == 1) return rc;
    j.parts[0] = wide[0].out, j.parts[1] = wide[1].out, j.have = o.have, j.shares = p.shares, j.n = a.n;
    j.size[0] = static_cast<int64_t>(a.r) * wide[0].cols, j.size[1] = static_cast<int64_t>(a.r) * wide[1].cols;
    j.blocks0 = static_cast<unsigned>(ceil_div64(j.size[0], 256));
    return launch(outer_join_kernel, dim3(j.blocks0 + static_cast<unsigned>(ceil_div64(j.size[1], 256)), a.n), dim3(256), 0, st, j);
}
// (rows that the narrow kernels take are no part of the plan)
static size_t outer_bytes(int T, int n, int r, int F, int K) {
    if (F < kNarrow && K < kNarrow) return 0;
    return F < kNarrow ? outer_plan(T, n, r, K, 0).bytes() : outer_plan(T, n, r, F, K < kNarrow ? 0 : K).bytes();
}

static int check_adapters(const void* X, int32_t dtype, int64_t ldx, const int32_t* ids, const void* A, const void* B, const float* scale, int32_t T, int32_t K,
                   int32_t F, int32_t n, int32_t r) {
    if (!X || !ids || !A || !B) return DAB_ERR_NULL;
    if (T < 1 || K < 1 || F < 1 || n < 1 || r < 1 || ldx < K) return DAB_ERR_SHAPE;
    if (!real_dtype(dtype) || K > kAdapterCols || F > kAdapterCols || n > 65535 || r > kMaxRank || T > (1 << 25) || ldx > kAdapterLd)
        return DAB_ERR_UNSUPPORTED;
    if (misaligned(X, 16) || misaligned(A, 16) || misaligned(B, 16) || misaligned(ids, 4) || misaligned(scale, 4)) return DAB_ERR_ALIGN;
    return DAB_OK;
}
static int check_base(const void* base, int32_t dtype, int64_t ld, int32_t cols, int32_t own_dtype) {
    if (!base) return DAB_OK;
    if (ld < cols) return DAB_ERR_SHAPE;
    if ((dtype != DAB_F32 && dtype != own_dtype) || ld > kAdapterLd) return DAB_ERR_UNSUPPORTED;
    return misaligned(base, 16) ? DAB_ERR_ALIGN : DAB_OK;
}
// An output over base: only element by element, which the same lane reads before it writes.
static bool over_base(const void* out, int32_t dtype, const void* base, int32_t base_dtype, int32_t T, int32_t cols, int64_t ld) {
    if (!out || !base || (out == base && base_dtype == dtype && (ld == cols || T == 1))) return false;
    return meet({out, T, cols, cols, dtype_bytes(dtype)}, {base, T, cols, ld, dtype_bytes(base_dtype)});
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
    // (X is read for other columns of Y)
    if (meet({Y, T, F, F, dtype_bytes(dtype)}, {X, T, K, ldx, dtype_bytes(dtype)})) return DAB_ERR_UNSUPPORTED;
    if (over_base(Y, dtype, base, base_dtype, T, F, ldbase)) return DAB_ERR_UNSUPPORTED;
    const Adapters a{ids, scale, T, n, r};
    const auto st = static_cast<hipStream_t>(stream);
    const auto go = [&](auto* t) -> int {
        typedef std::remove_pointer_t<decltype(t)> E;
        return shrink_expand(static_cast<const E*>(X), ldx, static_cast<const E*>(A), K, static_cast<const E*>(B), F, a, false, U,
                             Base{base, ldbase, base_dtype}, static_cast<E*>(Y), st);
    };
    if (dtype == DAB_F32) return go(static_cast<float*>(nullptr));
    if (dtype == DAB_BF16) return go(static_cast<bf16*>(nullptr));
    return go(static_cast<f16*>(nullptr));
}

extern "C" size_t dab_adapters_gradient_workspace_bytes(int32_t T, int32_t K, int32_t F, int32_t n, int32_t r) {
    using namespace dab;
    if (T < 1 || K < 1 || F < 1 || n < 1 || r < 1 || K > kAdapterCols || F > kAdapterCols || n > 65535 || r > kMaxRank || T > (1 << 25)) return 0;
    return static_cast<size_t>(round_up(static_cast<int64_t>(T) * r * 4, 256)) + outer_bytes(T, n, r, F, K);
}

extern "C" int dab_adapters_gradient(const void* dY, int64_t lddy, const void* X, int32_t dtype, int64_t ldx, const float* U, const int32_t* ids,
                                     const void* A, const void* B, const float* scale, int32_t T, int32_t K, int32_t F, int32_t n, int32_t r,
                                     const void* base, int32_t base_dtype, int64_t ldbase, void* dX, float* dA, float* dB, void* ws, size_t ws_bytes,
                                     void* stream) {
    using namespace dab;
    if (int rc = check_adapters(X, dtype, ldx, ids, A, B, scale, T, K, F, n, r)) return rc;
    if (!dY || !U || !dA || !dB || (base && !dX)) return DAB_ERR_NULL;
    if (lddy < F) return DAB_ERR_SHAPE;
    if (lddy > kAdapterLd) return DAB_ERR_UNSUPPORTED;
    if (int rc = check_base(base, base_dtype, ldbase, K, dtype)) return rc;
    if (misaligned(dY, 16) || misaligned(dX, 16) || misaligned(U, 4) || misaligned(dA, 4) || misaligned(dB, 4)) return DAB_ERR_ALIGN;
    // (X and dY are read again behind dX)
    const int64_t size = dtype_bytes(dtype);
    if (dX && (meet({dX, T, K, K, size}, {X, T, K, ldx, size}) || meet({dX, T, K, K, size}, {dY, T, F, lddy, size}))) return DAB_ERR_UNSUPPORTED;
    if (over_base(dX, dtype, base, base_dtype, T, K, ldbase)) return DAB_ERR_UNSUPPORTED;
    const size_t need = dab_adapters_gradient_workspace_bytes(T, K, F, n, r);
    if (!ws || ws_bytes < need || misaligned(ws, 256)) return DAB_ERR_WORKSPACE;
    const Adapters a{ids, scale, T, n, r};
    const auto st = static_cast<hipStream_t>(stream);
    float* V = static_cast<float*>(ws);
    char* rest = static_cast<char*>(ws) + round_up(static_cast<int64_t>(T) * r * 4, 256);
    const auto go = [&](auto* t) -> int {
        typedef std::remove_pointer_t<decltype(t)> E;
        const E *x = static_cast<const E*>(X), *dy = static_cast<const E*>(dY), *up = static_cast<const E*>(B), *down = static_cast<const E*>(A);
        if (int rc = dX ? shrink_expand(dy, lddy, up, F, down, K, a, true, V, Base{base, ldbase, base_dtype}, static_cast<E*>(dX), st)
                        : shrink(dy, lddy, up, F, a, true, V, st))
            return rc;
        return outer<E>({{U, dy, lddy, F, 1, dB}, {V, x, ldx, K, 0, dA}}, a, rest, st);
    };
    if (dtype == DAB_F32) return go(static_cast<float*>(nullptr));
    if (dtype == DAB_BF16) return go(static_cast<bf16*>(nullptr));
    return go(static_cast<f16*>(nullptr));
}

// Workspace of the product with adapters: the product's own, then U.
static size_t w4_own_bytes(int32_t B, int32_t K, int32_t F, int32_t dtype, int64_t ldx) {
    return static_cast<size_t>(dab::round_up(static_cast<int64_t>(dab_w4_matvec_workspace_bytes(B, K, F, dtype, ldx)), 256));
}
extern "C" size_t dab_w4_adapters_workspace_bytes(int32_t B, int32_t K, int32_t F, int32_t r, int32_t dtype, int64_t ldx) {
    if (B < 1 || K < 1 || F < 1 || r < 1 || !dab::real_dtype(dtype)) return 0;
    return w4_own_bytes(B, K, F, dtype, ldx) + static_cast<size_t>(dab::round_up(static_cast<int64_t>(B) * r * 4, 256));
}

extern "C" int dab_w4_adapters(const void* X, int32_t dtype, int64_t ldx, const uint8_t* Q, const uint8_t* S, const int32_t* ids, const void* A,
                               const void* Bt, const float* scale, int32_t B, int32_t K, int32_t F, int32_t n, int32_t r, void* Y, void* ws,
                               size_t ws_bytes, void* stream) {
    using namespace dab;
    if (int rc = check_adapters(X, dtype, ldx, ids, A, Bt, scale, B, K, F, n, r)) return rc;
    if (!Q || !S || !Y) return DAB_ERR_NULL;
    if (B > 65535 || F > 65535 * 16) return DAB_ERR_UNSUPPORTED;
    if (misaligned(Q, 16) || misaligned(S, 16) || misaligned(Y, 16)) return DAB_ERR_ALIGN;
    if (!ws || ws_bytes < dab_w4_adapters_workspace_bytes(B, K, F, r, dtype, ldx) || misaligned(ws, 256)) return DAB_ERR_WORKSPACE;
    if (meet({Y, B, F, F, dtype_bytes(dtype)}, {X, B, K, ldx, dtype_bytes(dtype)})) return DAB_ERR_UNSUPPORTED;
    const size_t product = w4_own_bytes(B, K, F, dtype, ldx);
    float* U = reinterpret_cast<float*>(static_cast<char*>(ws) + product);
    const W4Adapters w{Adapters{ids, scale, B, n, r}, U, A, Bt};
    const auto st = static_cast<hipStream_t>(stream);
    if (B > kFewTokens) {
        int rc;
        if (dtype == DAB_F32) rc = shrink(static_cast<const float*>(X), ldx, static_cast<const float*>(A), K, w.a, true, U, st);
        else if (dtype == DAB_BF16) rc = shrink(static_cast<const bf16*>(X), ldx, static_cast<const bf16*>(A), K, w.a, true, U, st);
        else rc = shrink(static_cast<const f16*>(X), ldx, static_cast<const f16*>(A), K, w.a, true, U, st);
        if (rc) return rc;
    }
    return w4_product(X, dtype, ldx, Q, S, B, K, F, Y, ws, product, st, &w);
}
