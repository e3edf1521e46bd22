// Weights in 4 bits: laying out, reading back, and products of a few tokens with them.
//
// The product reads 0.53 bytes a weight and is bound by that (one bf16 token, 4096 -> 131072, 49 us: 5.8 TB/s; 4096 -> 4096 3.9, little more than
// a launch).  A vector multiply-add per weight would
// already exceed the vector units' rate at one token, so the matrix cores do it at any number of tokens: a wavefront holds 16 rows of
// weights as the left operand of 16 x 16 x 32 products, converted from 4 bits to bf16 and scaled by one instruction per two weights, and up to
// 16 columns of tokens as the right one.  A token whose numbers are wider than bf16 takes two or three columns, one per piece;
// the columns of a token are added up at the end.  The layout (include/dab.h) gives every lane the 32 weights of one group,
// so that a load is 16 bytes a lane and a kilobyte a wavefront, and a lane has one scale for them; the order of the weights within
// the sum is then that of the lanes, which the tokens' loads follow.
#include "adapters.h"

namespace dab {

constexpr int kW4MaxWaves = 8;       // wavefronts per workgroup

// ---------------------------------------------------------------- laying out
// Both directions: a workgroup takes 16 rows x 512 weights, a wavefront 128 of them.  A lane holds four neighbouring weights of a row, 32 lanes a
// row of the block, so that rows are read and written in whole lines; the packed block passes through LDS on its way.  (A wavefront that
// takes the 512 by itself waits four times as long for its loads: 1836 x 624 bf16 laid out and read back, 17 + 11 us instead of 6 + 5.)  Rows
// of one or two blocks: four or two times 16 of them.  Bound by memory from a few thousand rows on: 4096 x 9216 fp32 laid out in 39 us, read
// back in 33, 4.4 and 5.2 TB/s.
constexpr int kW4PackWaves = 4;      // blocks that share a word of scales
struct W4Place {
    int tile, step, j, kt, slot;     // 16 rows, 512 weights of them, which 128 of those and of all; the tile's place in the workgroup
    __device__ __forceinline__ W4Place(int Kt) {
        const int wave = threadIdx.x >> 6, shift = Kt == 1 ? 0 : Kt == 2 ? 1 : 2;
        slot = wave >> shift, tile = blockIdx.y * (kW4PackWaves >> shift) + slot, step = blockIdx.x;
        j = wave & ((1 << shift) - 1), kt = step * kW4PackWaves + j;
    }
    static dim3 grid(int F, int Kt) { return dim3(ceil_div(Kt, kW4PackWaves), ceil_div(F, Kt == 1 ? 64 : Kt == 2 ? 32 : 16)); }
};

template <typename T>
__device__ __forceinline__ v4f load4(const T* row, int c, int cols) {
    typedef T v4t __attribute__((ext_vector_type(4)));
    v4f v = v4f{0.f, 0.f, 0.f, 0.f};
    if (c + 4 <= cols) {
        const v4t got = *reinterpret_cast<const typename Unaligned<T, 4>::type*>(row + c);
        return __builtin_convertvector(got, v4f);
    }
#pragma unroll
    for (int i = 0; i < 4; ++i)
        if (c + i < cols) v[i] = static_cast<float>(row[c + i]);
    return v;
}

// (six wavefronts on a SIMD asked for, or else the compiler takes all rows at once, in 238 registers)
template <typename T>
__global__ __launch_bounds__(64 * kW4PackWaves, 6) void w4_pack_kernel(const T* __restrict__ W, int F, int K, int64_t ldw, int Kt, int K4,
                                                                    uint8_t* __restrict__ Q, uint8_t* __restrict__ S) {
    __shared__ __attribute__((aligned(16))) uint16_t codes[kW4PackWaves][512];     // [group][row][four weights]: a block's kilobyte
    __shared__ __attribute__((aligned(4))) uint8_t scales[kW4PackWaves][64][kW4PackWaves];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const W4Place at(Kt);
    const int tile = at.tile, kt = at.kt;
    if (kt < Kt && tile * 16 < F) {
        const int k = kt * 128 + (lane & 31) * 4, group = (lane & 31) >> 3;
        v4f v[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const int row = tile * 16 + 2 * i + (lane >> 5);
            v[i] = v4f{0.f, 0.f, 0.f, 0.f};
            if (row < F) v[i] = load4(W + row * ldw, k, K);
        }
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const int r = 2 * i + (lane >> 5);
            // the largest magnitude, as bits, of the eight lanes of a group
            uint32_t m = 0;
#pragma unroll
            for (int u = 0; u < 4; ++u) m = max(m, __float_as_uint(v[i][u]) & 0x7fffffffu);
            m = max(m, static_cast<uint32_t>(__builtin_amdgcn_update_dpp(0, static_cast<int>(m), 0xB1, 0xf, 0xf, true)));    // lane ^ 1
            m = max(m, static_cast<uint32_t>(__builtin_amdgcn_update_dpp(0, static_cast<int>(m), 0x4E, 0xf, 0xf, true)));    // lane ^ 2
            m = max(m, static_cast<uint32_t>(__builtin_amdgcn_update_dpp(0, static_cast<int>(m), 0x141, 0xf, 0xf, true)));   // the other four
            const bool finite = m < 0x7f800000u;
            const int e = group_exponent<2>(finite ? m : 0);
            const float inv = pow2f(-e);
            uint32_t word = 0;
#pragma unroll
            for (int u = 0; u < 4; ++u) {
                const float a = fabsf(v[i][u] * inv);
                // to the nearest level, in the middle to the even code
                uint32_t code = (a > 0.25f) + (a >= 0.75f) + (a > 1.25f) + (a >= 1.75f) + (a > 2.5f) + (a >= 3.5f) + (a > 5.f);
                code |= (__float_as_uint(v[i][u]) >> 31) << 3;
                word |= (finite ? code : 7u) << (4 * u);
            }
            codes[wave][(group * 16 + r) * 8 + (lane & 7)] = static_cast<uint16_t>(word);
            if ((lane & 7) == 0) scales[at.slot][group * 16 + r][at.j] = static_cast<uint8_t>(finite ? e + 127 : 255);
        }
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        __builtin_nontemporal_store(reinterpret_cast<const v4u32*>(codes[wave])[lane],
                                    reinterpret_cast<v4u32*>(Q + ((static_cast<int64_t>(tile) * Kt + kt) * 64 + lane) * 16));
    }
    __syncthreads();
    if (at.j == 0 && tile * 16 < F) {
        // (17, the scale of zeros, for blocks past the last one)
        const uint32_t all = *reinterpret_cast<const uint32_t*>(scales[at.slot][lane]);
        const int n = Kt - at.step * kW4PackWaves;
        const uint32_t past = n >= kW4PackWaves ? 0u : ~0u << (8 * n);
        *reinterpret_cast<uint32_t*>(S + ((static_cast<int64_t>(tile) * K4 + at.step) * 64 + lane) * 4) = (all & ~past) | (17u * 0x01010101u & past);
    }
}

// The scale of block j of four from its byte, as the conversions take it.
__device__ __forceinline__ float scale_of(uint32_t codes, int j) {
    const uint32_t s = (codes >> (8 * j)) & 255u;
    return __builtin_bit_cast(float, s == 255u ? 0x7fc00000u : s << 23);
}

__global__ __launch_bounds__(64 * kW4PackWaves) void w4_unpack_kernel(const uint8_t* __restrict__ Q, const uint8_t* __restrict__ S, int F,
                                                                      int K, int Kt, int K4, float* __restrict__ W) {
    __shared__ __attribute__((aligned(16))) uint16_t codes[kW4PackWaves][512];
    __shared__ uint8_t scales[kW4PackWaves][64];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const W4Place at(Kt);
    const int tile = at.tile, kt = at.kt;
    if (kt >= Kt || tile * 16 >= F) return;                  // (a wavefront works alone: no barrier below)
    const v4u32 q = *reinterpret_cast<const v4u32*>(Q + ((static_cast<int64_t>(tile) * Kt + kt) * 64 + lane) * 16);
    scales[wave][lane] = S[((static_cast<int64_t>(tile) * K4 + at.step) * 64 + lane) * 4 + at.j];
    reinterpret_cast<v4u32*>(codes[wave])[lane] = q;
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    const int k = kt * 128 + (lane & 31) * 4, group = (lane & 31) >> 3;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const int r = 2 * i + (lane >> 5), row = tile * 16 + r;
        const uint32_t word = codes[wave][(group * 16 + r) * 8 + (lane & 7)], s = scales[wave][group * 16 + r];
        const float scale = s == 255u ? __builtin_nanf("") : pow2f(static_cast<int>(s) - 127);
        v4f v;
#pragma unroll
        for (int u = 0; u < 4; ++u) {
            const uint32_t c = word >> (4 * u), m = c & 7u;
            // 0, 1/2, then (2 + last bit) 2^(upper bits - 2)
            const float a = m < 2 ? 0.5f * static_cast<float>(m) : static_cast<float>(2u + (m & 1u)) * pow2f(static_cast<int>(m >> 1) - 2);
            v[u] = (c & 8u ? -a : a) * scale;
        }
        if (row >= F) continue;
        float* to = W + static_cast<int64_t>(row) * K;
        if (k + 4 <= K) {
            *reinterpret_cast<Unaligned<float, 4>::type*>(to + k) = v;
        } else {
#pragma unroll
            for (int u = 0; u < 4; ++u)
                if (k + u < K) to[k + u] = v[u];
        }
    }
}

// ---------------------------------------------------------------- tokens as the matrix cores take them
// [pass][block of 128 k][i][column tile][lane] pieces of 16 bytes: column c = 16 tile + lane % 16 is piece c / nb of token c % nb of the pass, and
// the piece holds its k = 128 block + 32 (lane / 16) + 8 i .. + 7; zeros past the last column and the last k.  A wavefront's load of them is a
// kilobyte in a row; from the tokens' own rows it would touch 16 rows in four places each.  Little more than a launch: 7 x 9111 fp32 2.7 us.
struct W4Tokens {
    int B, K;
    int64_t ldx;
    int Kt, nb, P, tiles;            // blocks of 128 k; tokens of a pass, pieces, column tiles
};
template <typename T>
__device__ __forceinline__ void w4_tokens(const T* __restrict__ X, const W4Tokens& g, int block, int pass, bf16* __restrict__ out) {
    const int at = block * 256 + threadIdx.x, lane = at & 63, frag = at >> 6;
    const int i4 = frag / g.tiles, t = frag - i4 * g.tiles, kt = i4 >> 2, i = i4 & 3;
    if (kt >= g.Kt) return;
    const int b0 = pass * g.nb, n = min(g.nb, g.B - b0), c = t * 16 + (lane & 15), p = c / n, b = c - p * n;
    float v[8] = {};
    const int k = kt * 128 + (lane >> 4) * 32 + 8 * i;
    if (p < g.P && k < g.K) load8(X + (b0 + b) * g.ldx, k, g.K, v);
    v8bf o;
#pragma unroll
    for (int u = 0; u < 8; ++u) o[u] = piece_of(v[u], p);
    *reinterpret_cast<v8bf*>(out + ((static_cast<int64_t>(pass) * g.Kt * 4 * g.tiles + frag) * 64 + lane) * 8) = o;
}
template <typename T>
__global__ __launch_bounds__(256) void w4_tokens_kernel(const T* __restrict__ X, int B, int K, int64_t ldx, int Kt, int nb, int P,
                                                        int tiles, bf16* __restrict__ out) {
    w4_tokens(X, W4Tokens{B, K, ldx, Kt, nb, P, tiles}, blockIdx.x, blockIdx.y, out);
}
// The same beside U of the few tokens' adapters (shrink_few), in workgroups behind the layout's.
template <typename T>
__global__ __launch_bounds__(256) void w4_tokens_shrink_kernel(const T* __restrict__ X, W4Tokens g, int blocks, bf16* __restrict__ out, const T* __restrict__ A,
                                                               Adapters a, float* __restrict__ U) {
    DAB_RESERVE_VGPRS();
    const int pass = blockIdx.x / max(blocks, 1), passes = (g.B + g.nb - 1) / g.nb;
    if (blocks > 0 && pass < passes) {
        w4_tokens(X, g, blockIdx.x - pass * blocks, pass, out);
        return;
    }
    shrink_few(X, g.ldx, A, g.K, a, true, static_cast<int64_t>(blockIdx.x) - blocks * passes, U);
}

// ---------------------------------------------------------------- product
struct W4Geom {
    int F, K, Kt, K4;
    int Ft, ks, groups;              // 16-row tiles, wavefronts that share a group of tiles, groups of a workgroup
    int B, nb, P;                    // tokens in all and per pass over the weights, pieces
    int64_t ldx;                     // of tokens that are read where they are
    int dtype;                       // of the output
};

// Eight weights as bf16, times a power of two.
__device__ __forceinline__ v8bf weights8(uint32_t q, float scale) {
    v8bf a;
    const v2bf w0 = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(q, scale, 0), w1 = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(q, scale, 1);
    const v2bf w2 = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(q, scale, 2), w3 = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(q, scale, 3);
    a[0] = w0[0], a[1] = w0[1], a[2] = w1[0], a[3] = w1[1], a[4] = w2[0], a[5] = w2[1], a[6] = w3[0], a[7] = w3[1];
    return a;
}

// A wavefront's share of a step: 512 weights of each of its TB tiles, five loads a tile.
template <int TB>
struct Step4 {
    v4u32 q[TB][4];
    uint32_t codes[TB];
    __device__ __forceinline__ void load(const uint8_t* __restrict__ Q, const uint8_t* __restrict__ S, const W4Geom& g, int tile, int s,
                                         int lane) {
#pragma unroll
        for (int t = 0; t < TB; ++t) {
            const int64_t tl = min(tile + t, g.Ft - 1);      // (a tile past the last is read from the last and not used)
            codes[t] = __builtin_nontemporal_load(reinterpret_cast<const uint32_t*>(S + (tl * g.K4 + s) * 256 + lane * 4));
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const int kt = min(4 * s + j, g.Kt - 1);     // (likewise: its tokens are zeros)
                q[t][j] = __builtin_nontemporal_load(reinterpret_cast<const v4u32*>(Q + (tl * g.Kt + kt) * 1024 + lane * 16));
            }
        }
    }
};

// LANES lanes share a token's eight columns: the shares of the sums, the pieces of the token and the adapter's rows are dealt out to them, ROWS
// rows a lane read at once.
template <typename T, int LANES, int ROWS>
struct W4Rows {
    Eight<T> b[ROWS];
    float u[ROWS];
    int id;
    __device__ __forceinline__ void load(const W4Adapters& w, int64_t t, int f, int F, int lane) {
        id = adapter_of(w.a, t);
#pragma unroll
        for (int q = 0; q < ROWS; ++q) {
            const int row = q * LANES + lane;
            b[q].v = {}, u[q] = 0.f;
            if (id >= 0 && row < w.a.r) {
                b[q].load_last(static_cast<const T*>(w.B) + (static_cast<int64_t>(id) * w.a.r + row) * F, f, F);
                u[q] = w.U[t * w.a.r + row];
            }
        }
    }
    // y += the lane's part of U_t B_i
    __device__ __forceinline__ void add(const W4Adapters& w, int64_t t, int f, int F, int lane, float (&y)[8]) const {
        if (id < 0) return;
        float v[8] = {};
#pragma unroll
        for (int q = 0; q < ROWS; ++q)
#pragma unroll
            for (int i = 0; i < 8; ++i) v[i] += u[q] * b[q][i];
        const T* rows = static_cast<const T*>(w.B) + static_cast<int64_t>(id) * w.a.r * F;
#pragma unroll 4
        for (int row = ROWS * LANES + lane; row < w.a.r; row += LANES) {
            Eight<T> c;
            c.load_last(rows + static_cast<int64_t>(row) * F, f, F);
            const float by = w.U[t * w.a.r + row];
#pragma unroll
            for (int i = 0; i < 8; ++i) v[i] += by * c[i];
        }
        if (F >= 8) own_first(max(f - (F - 8), 0), v);
#pragma unroll
        for (int i = 0; i < 8; ++i) y[i] += v[i];
    }
};
struct NoAdapters {};

// ROWS: bf16 tokens in rows of their own, X; else as w4_tokens_kernel lays them out.  TA: the type of the
// adapters that are added to the tokens' sums, and of Y then; or NoAdapters.
template <int NCT, int TB, bool ROWS, typename TA>
__global__ __launch_bounds__(64 * kW4MaxWaves) void w4_matvec_kernel(const bf16* __restrict__ X, const uint8_t* __restrict__ Q,
                                                                     const uint8_t* __restrict__ S, W4Geom g, void* __restrict__ Y,
                                                                     const W4Adapters w) {
    extern __shared__ float sums[];                          // [wavefront][tile][column][16 rows]
    DAB_RESERVE_VGPRS();
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int group = __builtin_amdgcn_readfirstlane(wave / g.ks), part = wave - group * g.ks;
    const int tile0 = blockIdx.x * g.groups * TB, tile = tile0 + group * TB;
    const int b0 = blockIdx.y * g.nb, nb = min(g.nb, g.B - b0), cols = nb * g.P;
    constexpr bool kAdapt = !std::is_same_v<TA, NoAdapters>;
    // Where registers are left the adapter's number and first rows are read before the product, by eight lanes each (one token, 4096 x 4096: 4.6 us, 4.4
    // without an adapter; read behind the product 6.3 to 7.3); else behind it, by two (32 tokens, 16384 x 4096: 14.4 us, 13.8 without).
    constexpr bool kEarly = NCT * TB <= 4;
    constexpr int kLanes = kEarly ? 8 : 2;
    std::conditional_t<kAdapt, W4Rows<std::conditional_t<kAdapt, TA, float>, kLanes, kEarly ? 2 : 4>, NoAdapters> early;
    const int eights = g.groups * TB * 2, units = eights * nb * kLanes;        // eight rows of a token a unit

    v4f acc[TB][NCT];
#pragma unroll
    for (int t = 0; t < NCT; ++t)
#pragma unroll
        for (int u = 0; u < TB; ++u) acc[u][t] = v4f{0.f, 0.f, 0.f, 0.f};
    // (columns past the last read the first one's token; their results are not used)
    const bf16* x0 = ROWS ? X + (b0 + ((lane & 15) < cols ? lane & 15 : 0)) * g.ldx
                          : X + static_cast<int64_t>(blockIdx.y) * g.Kt * (4 * NCT * 512) + lane * 8;
    const bool some = tile < g.Ft && part < g.K4;
    Step4<TB> now, next;
    if (some) now.load(Q, S, g, tile, part, lane);
    if constexpr (kAdapt && kEarly) {
        const int unit = threadIdx.x / kLanes, f = tile0 * 16 + unit % eights * 8;
        if (static_cast<int>(threadIdx.x) < units && f < g.F) early.load(w, b0 + unit / eights, f, g.F, threadIdx.x % kLanes);
    }
    if (some) {
        for (int s = part; s < g.K4; s += g.ks) {
            const bool more = s + g.ks < g.K4;
            if (more) next.load(Q, S, g, tile, s + g.ks, lane);
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const int kt = 4 * s + j;
                v8bf x[4][NCT];
                if constexpr (ROWS) {
                    const int k = kt * 128 + (lane >> 4) * 32;
#pragma unroll
                    for (int i = 0; i < 4; ++i) x[i][0] = *reinterpret_cast<const v8bf*>(x0 + min(k + 8 * i, g.K - 8));
                    if (kt * 128 + 128 > g.K) {
                        // past the last element: zeros, whatever was loaded
#pragma unroll
                        for (int i = 0; i < 4; ++i)
                            if (k + 8 * i >= g.K) x[i][0] = v8bf{};
                    }
                } else {
#pragma unroll
                    for (int i = 0; i < 4; ++i)
#pragma unroll
                        for (int t = 0; t < NCT; ++t) x[i][t] = *reinterpret_cast<const v8bf*>(x0 + (static_cast<int64_t>(min(kt, g.Kt - 1)) * 4 + i) * (NCT * 512) + t * 512);
                    if (kt >= g.Kt) {
#pragma unroll
                        for (int i = 0; i < 4; ++i)
#pragma unroll
                            for (int t = 0; t < NCT; ++t) x[i][t] = v8bf{};
                    }
                }
#pragma unroll
                for (int u = 0; u < TB; ++u) {
                    const float scale = scale_of(now.codes[u], j);
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        const v8bf a = weights8(now.q[u][j][i], scale);
#pragma unroll
                        for (int t = 0; t < NCT; ++t) acc[u][t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, x[i][t], acc[u][t], 0, 0, 0);
                    }
                }
            }
            if (more) now = next;
        }
    }
#pragma unroll
    for (int u = 0; u < TB; ++u)
#pragma unroll
        for (int t = 0; t < NCT; ++t)
            *reinterpret_cast<v4f*>(sums + (((wave * TB + u) * NCT + t) * 16 + (lane & 15)) * 16 + (lane >> 4) * 4) = acc[u][t];
    __syncthreads();
    // the shares of a tile and the pieces of a token, added in a fixed order
    const int rows = g.groups * TB * 16;
    if constexpr (kAdapt) {
        for (int i = threadIdx.x; i < units; i += blockDim.x) {
            const int unit = i / kLanes, l = i % kLanes, b = unit / eights, row = (unit - b * eights) * 8, tl = row >> 4, grp = tl / TB, u = tl - grp * TB;
            const int f = tile0 * 16 + row;
            if (f >= g.F) continue;
            const int64_t t = b0 + b;
            if (!kEarly || i != static_cast<int>(threadIdx.x)) early.load(w, t, f, g.F, l);
            float y[8] = {};
            for (int k = l; k < g.ks * g.P; k += kLanes) {
                const int p = k / g.ks;
                const v4f* at = reinterpret_cast<const v4f*>(sums + (((grp * g.ks + k - p * g.ks) * TB + u) * NCT * 16 + p * nb + b) * 16 + (row & 15));
#pragma unroll
                for (int e = 0; e < 4; ++e) y[e] += at[0][e], y[4 + e] += at[1][e];
            }
            early.add(w, t, f, g.F, l, y);
#pragma unroll
            for (int e = 0; e < 8; ++e) y[e] = lanes_sum<kEarly ? 3 : 1>(y[e]);
            if (l == 0) store8(static_cast<TA*>(Y) + t * g.F, f, g.F, y);
        }
        return;
    }
    for (int i = threadIdx.x; i < rows * nb; i += blockDim.x) {
        const int b = i / rows, row = i - b * rows, r = row & 15, tl = row >> 4, grp = tl / TB, u = tl - grp * TB;
        const int f = tile0 * 16 + row;
        float y = 0.f;
        for (int p = g.P - 1; p >= 0; --p)
            for (int k = 0; k < g.ks; ++k) y += sums[(((grp * g.ks + k) * TB + u) * NCT * 16 + p * nb + b) * 16 + r];
        if (f >= g.F) continue;
        const int64_t at = static_cast<int64_t>(b0 + b) * g.F + f;
        if (g.dtype == DAB_F32) static_cast<float*>(Y)[at] = y;
        else if (g.dtype == DAB_BF16) static_cast<bf16*>(Y)[at] = static_cast<bf16>(y);
        else static_cast<f16*>(Y)[at] = static_cast<f16>(y);
    }
}

// Columns of tokens that a pass over the weights takes, and its tokens.
constexpr int kW4Columns = 48;
static int w4_tokens(int B, int P) { return ceil_div(B, ceil_div(B, kW4Columns / P)); }
// Aligned bf16 tokens of one column tile are read where they are, others from the workspace.
static bool w4_rows(int32_t B, int32_t K, int32_t dtype, int64_t ldx) { return dtype == DAB_BF16 && B <= 16 && K % 8 == 0 && ldx % 8 == 0; }

template <int NCT, int TB, bool ROWS>
static int launch_matvec(const W4Geom& g, hipStream_t st, const bf16* X, const uint8_t* Q, const uint8_t* S, void* Y, const W4Adapters* w) {
    const int waves = g.ks * g.groups;
    const dim3 grid(ceil_div(g.Ft, g.groups * TB), ceil_div(g.B, g.nb)), block(64 * waves);
    const size_t lds = static_cast<size_t>(waves) * TB * NCT * 1024;
    if (!w) return launch(w4_matvec_kernel<NCT, TB, ROWS, NoAdapters>, grid, block, lds, st, X, Q, S, g, Y, W4Adapters{});
    if constexpr (!ROWS) {
        if (g.dtype == DAB_F32) return launch(w4_matvec_kernel<NCT, TB, ROWS, float>, grid, block, lds, st, X, Q, S, g, Y, *w);
        if (g.dtype == DAB_F16) return launch(w4_matvec_kernel<NCT, TB, ROWS, f16>, grid, block, lds, st, X, Q, S, g, Y, *w);
    }
    return launch(w4_matvec_kernel<NCT, TB, ROWS, bf16>, grid, block, lds, st, X, Q, S, g, Y, *w);
}
static int launch_matvec(const W4Geom& g, int columns, int TB, bool rows, hipStream_t st, const bf16* X, const uint8_t* Q, const uint8_t* S,
                         void* Y, const W4Adapters* w) {
    if (rows) return TB == 2 ? launch_matvec<1, 2, true>(g, st, X, Q, S, Y, w) : launch_matvec<1, 1, true>(g, st, X, Q, S, Y, w);
    if (columns == 1) return TB == 2 ? launch_matvec<1, 2, false>(g, st, X, Q, S, Y, w) : launch_matvec<1, 1, false>(g, st, X, Q, S, Y, w);
    if (columns == 2)
        return TB == 4   ? launch_matvec<2, 4, false>(g, st, X, Q, S, Y, w)
               : TB == 2 ? launch_matvec<2, 2, false>(g, st, X, Q, S, Y, w)
                         : launch_matvec<2, 1, false>(g, st, X, Q, S, Y, w);
    return TB == 2 ? launch_matvec<3, 2, false>(g, st, X, Q, S, Y, w) : launch_matvec<3, 1, false>(g, st, X, Q, S, Y, w);
}

}  // namespace dab

extern "C" int dab_w4_pack(const void* W, int32_t dtype, int32_t F, int32_t K, int64_t ldw, uint8_t* Q, uint8_t* S, void* stream) {
    using namespace dab;
    if (!W || !Q || !S) return DAB_ERR_NULL;
    if (F < 1 || K < 1 || ldw < K) return DAB_ERR_SHAPE;
    if (!real_dtype(dtype) || K > INT32_MAX - 512 || F > 65535 * 16) return DAB_ERR_UNSUPPORTED;
    if (misaligned(W, 16) || misaligned(Q, 16) || misaligned(S, 16)) return DAB_ERR_ALIGN;
    const int Kt = ceil_div(K, 128), K4 = ceil_div(Kt, 4);
    const dim3 grid = W4Place::grid(F, Kt), block(64 * kW4PackWaves);
    const auto st = static_cast<hipStream_t>(stream);
    if (dtype == DAB_F32) return launch(w4_pack_kernel<float>, grid, block, 0, st, static_cast<const float*>(W), F, K, ldw, Kt, K4, Q, S);
    if (dtype == DAB_BF16) return launch(w4_pack_kernel<bf16>, grid, block, 0, st, static_cast<const bf16*>(W), F, K, ldw, Kt, K4, Q, S);
    return launch(w4_pack_kernel<f16>, grid, block, 0, st, static_cast<const f16*>(W), F, K, ldw, Kt, K4, Q, S);
}

extern "C" int dab_w4_unpack(const uint8_t* Q, const uint8_t* S, int32_t F, int32_t K, float* W, void* stream) {
    using namespace dab;
    if (!W || !Q || !S) return DAB_ERR_NULL;
    if (F < 1 || K < 1) return DAB_ERR_SHAPE;
    if (K > INT32_MAX - 512 || F > 65535 * 16) return DAB_ERR_UNSUPPORTED;
    if (misaligned(W, 16) || misaligned(Q, 16) || misaligned(S, 16)) return DAB_ERR_ALIGN;
    const int Kt = ceil_div(K, 128), K4 = ceil_div(Kt, 4);
    return launch(w4_unpack_kernel, W4Place::grid(F, Kt), dim3(64 * kW4PackWaves), 0, static_cast<hipStream_t>(stream), Q, S, F, K, Kt, K4, W);
}

extern "C" size_t dab_w4_matvec_workspace_bytes(int32_t B, int32_t K, int32_t F, int32_t dtype, int64_t ldx) {
    using namespace dab;
    if (B < 1 || K < 1 || F < 1 || !real_dtype(dtype) || w4_rows(B, K, dtype, ldx)) return 0;
    const int P = dtype_pieces(dtype), nb = w4_tokens(B, P);
    return static_cast<size_t>(ceil_div(B, nb)) * ceil_div(K, 128) * 4 * ceil_div(nb * P, 16) * 1024;
}

namespace dab {

int w4_product(const void* X, int32_t dtype, int64_t ldx, const uint8_t* Q, const uint8_t* S, int32_t B, int32_t K, int32_t F, void* Y, void* ws,
               size_t ws_bytes, hipStream_t st, const W4Adapters* w) {
    if (!X || !Q || !S || !Y) return DAB_ERR_NULL;
    if (B < 1 || K < 1 || F < 1 || ldx < K) return DAB_ERR_SHAPE;
    if (!real_dtype(dtype) || K > (1 << 26) || B > 65535 || F > 65535 * 16) return DAB_ERR_UNSUPPORTED;
    if (misaligned(X, 16) || misaligned(Q, 16) || misaligned(S, 16) || misaligned(Y, 16)) return DAB_ERR_ALIGN;
    const size_t need = dab_w4_matvec_workspace_bytes(B, K, F, dtype, ldx);
    if (need && (!ws || ws_bytes < need || misaligned(ws, 256))) return DAB_ERR_WORKSPACE;

    W4Geom g{};
    g.F = F, g.K = K, g.Kt = ceil_div(K, 128), g.K4 = ceil_div(g.Kt, 4);
    g.Ft = ceil_div(F, 16), g.B = B, g.P = dtype_pieces(dtype), g.nb = w4_tokens(B, g.P);
    // Tiles of a wavefront: with one they are spread furthest, with more the tokens are loaded less often.  One token, 4096 weights a row:
    // 4096 rows 3.9 us with one and 5.5 with two, 16384 rows 10.8 and 9.1, 131072 rows 63 and 52.4; two columns of tokens, 4096 rows
    // of 4096: 8.0, 9.8 with two, 4099 rows of 9111 19.9, 15.4, 20.4 with four, 32768 rows of 4096 34, 26, 24.5; three, 4096 rows of 4096
    // 9.6 and 10.8, (four tiles and three columns do not fit the registers).
    const int columns = ceil_div(g.nb * g.P, 16);
    const int TB = columns == 1   ? (g.Ft >= 1024 ? 2 : 1)
                   : columns == 2 ? (g.Ft >= 1024 ? 4 : g.Ft >= 128 && g.K4 > 8 ? 2 : 1)
                                  : (g.Ft >= 512 ? 2 : 1);
    // Shares of a row's sum: for one column of tokens until there are 24 wavefronts for every compute unit (131072 rows, two tiles: 58.6 us
    // with one share, 52.4, 53.7, 54.8 with eight; 4096 rows, one tile: 7.7, 5.3, 4.1, 3.9), for more, which are bound by the tokens'
    // loads, until there are eight (32768 rows of 4096, two columns: 43, 28, 24.5, 27.4; 65536 of 8192 124, 129, 138, 160).
    const int enough = columns == 1 ? 24 * kNumCU : 8 * kNumCU;
    g.ks = 1;
    while (g.ks < 8 && g.ks * 2 <= g.K4 && g.Ft / TB * g.ks < enough) g.ks *= 2;
    // groups of a workgroup: eight wavefronts, fewer where that leaves compute units without one (30 tokens, 1024 x 1024: 11.8 -> 7.1)
    g.groups = 8 / g.ks;
    while (g.groups > 1 && ceil_div(g.Ft, g.groups * TB) < kNumCU) g.groups /= 2;
    g.dtype = dtype;
    const bf16* x = static_cast<const bf16*>(X);
    g.ldx = ldx;
    const int blocks = need ? static_cast<int>(ceil_div64(static_cast<int64_t>(g.Kt) * 4 * columns, 4)) : 0, passes = ceil_div(B, g.nb);
    const W4Tokens to{B, K, ldx, g.Kt, g.nb, g.P, columns};
    bf16* out = static_cast<bf16*>(ws);
    const auto prepare = [&](auto* t) -> int {
        typedef std::remove_pointer_t<decltype(t)> T;
        const T* from = static_cast<const T*>(X);
        if (w && B <= kFewTokens) {
            const int64_t rows = static_cast<int64_t>(B) * w->a.r;
            return launch(w4_tokens_shrink_kernel<T>, dim3(static_cast<unsigned>(static_cast<int64_t>(blocks) * passes + rows)), dim3(256), 0, st, from, to,
                          blocks, out, static_cast<const T*>(w->A), w->a, w->U);
        }
        return need ? launch(w4_tokens_kernel<T>, dim3(blocks, passes), dim3(256), 0, st, from, B, K, ldx, g.Kt, g.nb, g.P, columns, out)
                    : static_cast<int>(DAB_OK);
    };
    // (U of many tokens is the caller's work)
    if (need || (w && B <= kFewTokens))
        if (int rc = dtype == DAB_F32   ? prepare(static_cast<float*>(nullptr))
                     : dtype == DAB_F16 ? prepare(static_cast<f16*>(nullptr))
                                        : prepare(static_cast<bf16*>(nullptr)))
            return rc;
    return launch_matvec(g, columns, TB, !need, st, need ? out : x, Q, S, Y, w);
}

}  // namespace dab

extern "C" int dab_w4_matvec(const void* X, int32_t dtype, int64_t ldx, const uint8_t* Q, const uint8_t* S, int32_t B, int32_t K,
                             int32_t F, void* Y, void* ws, size_t ws_bytes, void* stream) {
    return dab::w4_product(X, dtype, ldx, Q, S, B, K, F, Y, ws, ws_bytes, static_cast<hipStream_t>(stream));
}
