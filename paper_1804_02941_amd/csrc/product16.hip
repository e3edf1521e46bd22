// Host side of the bf16 products (product16.h): tile and split of a product, launches, and the kernels around it.
#include "product16.h"

namespace dab {

// ---------------------------------------------------------------- the product
__device__ __forceinline__ void wait_and_meet() {
    asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)\n\ts_barrier" ::: "memory");
}

static __device__ const uint32_t g_zeros16[4] = {0, 0, 0, 0};

typedef __attribute__((address_space(3))) uint32_t lds_u32;
typedef __attribute__((address_space(1))) const uint32_t glb_u32;

// One operand's tile of ROWS x 64 k in LDS.
template <int ROWS, bool RC, int NW>
struct Tile16 {
    static constexpr int kBytes = ROWS * kStepK * 2;
    static constexpr int kCopies = kBytes / 1024 / NW;       // of one wavefront
    static constexpr int kChunks = RC ? ROWS / 8 : 8;        // 16-byte pieces of a row of the tile in LDS
    static constexpr int kLdsRows = 64 / kChunks;            // rows of it that one copy fills

    // Where the lane's piece of copy c comes from: row and column in the tile (in elements of its two directions).
    // A row's pieces are permuted so that the reads below meet no bank twice; a copy's lanes are in order in LDS, so the
    // permutation is one of the addresses in memory.
    static __device__ __forceinline__ void source(int copy, int lane, int* lds_row, int* elem) {
        const int r = copy * kLdsRows + lane / kChunks, phys = lane % kChunks;
        *lds_row = r;
        if constexpr (RC) *elem = (phys ^ (((r & 3) | ((r >> 3) & 1) << 2) << 1)) * 8;
        else *elem = (phys ^ ((r >> 1) & 7)) * 8;
    }
};

template <int ROWS, bool RC, int NW>
struct Loader16 {
    using Tl = Tile16<ROWS, RC, NW>;
    uint32_t off[Tl::kCopies];                               // bytes from the tile's origin, the same every step
    int wave, lane;

    // rows: how many of the operand's rows are left from the tile's first on; rows past them are read from the last one
    // (their results are not used)
    __device__ __forceinline__ void init(int w, int l, int64_t ld, int rows) {
        wave = w, lane = l;
#pragma unroll
        for (int c = 0; c < Tl::kCopies; ++c) {
            int r, e;
            Tl::source(w * Tl::kCopies + c, l, &r, &e);
            if constexpr (RC) off[c] = static_cast<uint32_t>((r * ld + min(e, (rows - 1) & ~7)) * 2);
            else off[c] = static_cast<uint32_t>((min(r, rows - 1) * ld + e) * 2);
        }
    }
    // origin: the tile's first element of this step; k_left: k that are left from there on
    __device__ __forceinline__ void copy(const bf16* origin, int k_left, char* lds) const {
        const char* base = reinterpret_cast<const char*>(origin);
#pragma unroll
        for (int c = 0; c < Tl::kCopies; ++c) {
            const char* src = base + off[c];
            if (k_left < kStepK) {
                int r, e;
                Tl::source(wave * Tl::kCopies + c, lane, &r, &e);
                if ((RC ? r : e) >= k_left) src = reinterpret_cast<const char*>(g_zeros16);
            }
            __builtin_amdgcn_global_load_lds((glb_u32*)src, (lds_u32*)(lds + (wave * Tl::kCopies + c) * 1024), 16, 0, 0);
        }
    }
};

// Fragments of 16 rows x 32 k: lane l holds row l % 16, k = 8 (l / 16) .. + 7.
template <int ROWS, bool RC>
struct Reader16 {
    uint32_t at[RC ? 8 : 2];
    // row0: this wavefront's first row in the tile
    template <int NFRAG>
    __device__ __forceinline__ void init(int lane, int row0) {
        if constexpr (RC) {
            // a group of 16 lanes reads 4 k x 16 rows, a lane 4 neighbouring rows of one k, and gets the four k of its row
            const int s = lane & 15, g = lane >> 4, key = (s >> 2) | (g & 1) << 2;
#pragma unroll
            for (int j = 0; j < NFRAG; ++j)
                at[j] = (g * 8 + (s >> 2)) * (ROWS * 2) + (((row0 >> 4) + j) ^ key) * 32 + (s & 3) * 8;
        } else {
            const int row = row0 + (lane & 15), key = (lane & 15) >> 1;
#pragma unroll
            for (int kk = 0; kk < 2; ++kk) at[kk] = row * 128 + (((kk * 4 + (lane >> 4)) ^ key) * 16);
        }
    }
    __device__ __forceinline__ v8bf read(const char* lds, int kk, int j) const {
        if constexpr (RC) {
            typedef short v4s __attribute__((ext_vector_type(4)));
            typedef __attribute__((address_space(3))) v4s lds_v4s;
            union { v4s h[2]; v8bf v; } u;
            const char* p = lds + at[j] + kk * 32 * (ROWS * 2);
            u.h[0] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_v4s*)p);
            u.h[1] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_v4s*)(p + 4 * (ROWS * 2)));
            return u.v;
        } else {
            return *reinterpret_cast<const v8bf*>(lds + at[kk] + j * 16 * 128);
        }
    }
};

template <int EPI, int TM, int TN, int WM, int WN, bool ARC, bool BRC>
__global__ __launch_bounds__(64 * WM * WN) void product16_kernel(Product16 g) {
    constexpr int NW = WM * WN, FM = TM / WM / 16, FN = TN / WN / 16;
    using TA = Tile16<TM, ARC, NW>;
    using TB = Tile16<TN, BRC, NW>;
    constexpr int kBuf = TA::kBytes + TB::kBytes;
    extern __shared__ __attribute__((aligned(1024))) char lds[];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);

    // consecutive workgroups go to the XCDs in turn: each XCD gets neighbouring tiles, eight rows of tiles at a time, so
    // that what runs on it together shares operands in its L2
    const int unit = (blockIdx.x & 7) * g.per_xcd + (blockIdx.x >> 3);
    const int tiles = g.tiles_m * g.tiles_n;
    if (unit >= tiles * g.splits) return;
    const int share = unit / tiles, tile = unit - share * tiles;
    const int band = tile / (8 * g.tiles_n), in_band = tile - band * 8 * g.tiles_n;
    const int bm = min(8, g.tiles_m - band * 8);
    const int tn = in_band / bm, tm = band * 8 + in_band - tn * bm;
    const int m0 = tm * TM, n0 = tn * TN;
    const int wm = wave % WM, wn = wave / WM;

    Loader16<TM, ARC, NW> la;
    Loader16<TN, BRC, NW> lb;
    la.init(wave, lane, g.A.ld, g.M - m0);
    lb.init(wave, lane, g.B.ld, g.N - n0);
    const bf16* a0 = g.A.p + (ARC ? m0 : m0 * g.A.ld);
    const bf16* b0 = g.B.p + (BRC ? n0 : n0 * g.B.ld);
    const int64_t ka = ARC ? g.A.ld : 1, kb = BRC ? g.B.ld : 1;

    const int first = share * g.steps_per_split, last = min(first + g.steps_per_split, g.steps);
    const int per_seg = g.steps / g.n_seg;
    int seg = first / per_seg, k = (first - seg * per_seg) * kStepK;
    auto fetch = [&](char* buf) {
        la.copy(a0 + g.seg_a[seg] * g.A.plane + k * ka, g.K - k, buf);
        lb.copy(b0 + g.seg_b[seg] * g.B.plane + k * kb, g.K - k, buf + TA::kBytes);
        k += kStepK;
        if (k >= g.K) k = 0, ++seg;
    };

    Reader16<TM, ARC> ra;
    Reader16<TN, BRC> rb;
    ra.template init<FM>(lane, wm * FM * 16);
    rb.template init<FN>(lane, wn * FN * 16);

    v4f acc[FN][FM];
#pragma unroll
    for (int i = 0; i < FN; ++i)
#pragma unroll
        for (int j = 0; j < FM; ++j) acc[i][j] = v4f{0.f, 0.f, 0.f, 0.f};

    fetch(lds);
    wait_and_meet();
    for (int s = first; s < last; ++s) {
        char* cur = lds + ((s - first) & 1) * kBuf;
        if (s + 1 < last) fetch(lds + ((s + 1 - first) & 1) * kBuf);
#pragma unroll
        for (int kk = 0; kk < 2; ++kk) {
            v8bf a[FM], b[FN];
#pragma unroll
            for (int j = 0; j < FM; ++j) a[j] = ra.read(cur, kk, j);
#pragma unroll
            for (int i = 0; i < FN; ++i) b[i] = rb.read(cur + TA::kBytes, kk, i);
#pragma unroll
            for (int i = 0; i < FN; ++i)
#pragma unroll
                for (int j = 0; j < FM; ++j) acc[i][j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(b[i], a[j], acc[i][j], 0, 0, 0);
        }
        wait_and_meet();
    }

    const int mw = m0 + wm * FM * 16 + (lane & 15), nw = n0 + wn * FN * 16 + (lane >> 4) * 4;
#pragma unroll
    for (int j = 0; j < FM; ++j) {
        const int m = mw + j * 16;
        const bool in = m < g.M;
        if constexpr (EPI == kEpiStats) {
            // maximum and sum of exponentials of this wavefront's words, one pair per token
            float big = -__builtin_inff();
#pragma unroll
            for (int i = 0; i < FN; ++i)
#pragma unroll
                for (int r = 0; r < 4; ++r)
                    if (nw + i * 16 + r < g.N) big = fmaxf(big, acc[i][j][r]);
            big = fmaxf(big, __shfl_xor(big, 16));
            big = fmaxf(big, __shfl_xor(big, 32));
            float sum = 0.f;
            const float at = big == -__builtin_inff() ? 0.f : big;
#pragma unroll
            for (int i = 0; i < FN; ++i)
#pragma unroll
                for (int r = 0; r < 4; ++r)
                    if (nw + i * 16 + r < g.N) sum += __expf(acc[i][j][r] - at);
            sum += __shfl_xor(sum, 16);
            sum += __shfl_xor(sum, 32);
            if (in && lane < 16) g.stats[static_cast<int64_t>(tn * WN + wn) * g.M + m] = float2{big, sum};
            const int64_t t = in ? g.targets[m] : -1;
            if (in && t >= nw && t < g.N) {
                const int d = static_cast<int>(t) - nw;
#pragma unroll
                for (int i = 0; i < FN; ++i)
#pragma unroll
                    for (int r = 0; r < 4; ++r)
                        if (d == i * 16 + r) g.target_logit[m] = acc[i][j][r];
            }
        } else if constexpr (EPI == kEpiSoftmax) {
            if (in) {
                const int64_t t = g.targets[m];
                const bool dead = no_loss(t, g.ignore_index, g.V);
                const float lse = dead ? 0.f : g.lse[m], w = dead ? 0.f : g.g ? g.g[m] : 1.f;
                const int d = dead ? -1 : static_cast<int>(t) - g.n0;
                bf16* row = g.P + m * g.ldp + nw;
#pragma unroll
                for (int i = 0; i < FN; ++i) {
                    float p[4];
#pragma unroll
                    for (int r = 0; r < 4; ++r) {
                        const int n = nw + i * 16 + r;
                        p[r] = dead || n >= g.N ? 0.f : w * (__expf(acc[i][j][r] - lse) - (n == d ? 1.f : 0.f));
                    }
                    typedef __bf16 v4bf __attribute__((ext_vector_type(4)));
                    for (int q = 0; q < g.p_planes; ++q) {
                        v4bf o;
#pragma unroll
                        for (int r = 0; r < 4; ++r) o[r] = piece_of(p[r], q);
                        *reinterpret_cast<v4bf*>(row + q * g.p_plane + i * 16) = o;
                    }
                }
            }
        } else {
            if (in) {
#pragma unroll
                for (int i = 0; i < FN; ++i) {
                    const int n = nw + i * 16;
                    if (n >= g.N) continue;
                    v4f v = acc[i][j];
                    if (g.splits > 1) {
                        float* to = g.part + (static_cast<int64_t>(share) * g.M + m) * g.N + n;
                        if ((g.N & 3) == 0) *reinterpret_cast<v4f*>(to) = v;
                        else
                            for (int r = 0; r < 4; ++r)
                                if (n + r < g.N) to[r] = v[r];
                        continue;
                    }
                    if (g.add) {
                        const float* from = g.add + static_cast<int64_t>(m) * g.N + n;
                        for (int r = 0; r < 4; ++r)
                            if (n + r < g.N) v[r] += from[r];
                    }
                    if (g.out_bf16) {
                        bf16* to = static_cast<bf16*>(g.C) + m * g.ldc + n;
                        typedef __bf16 v4bf __attribute__((ext_vector_type(4)));
                        if (g.vec) *reinterpret_cast<v4bf*>(to) = v4bf{static_cast<bf16>(v[0]), static_cast<bf16>(v[1]), static_cast<bf16>(v[2]), static_cast<bf16>(v[3])};
                        else
                            for (int r = 0; r < 4; ++r)
                                if (n + r < g.N) to[r] = static_cast<bf16>(v[r]);
                    } else {
                        float* to = static_cast<float*>(g.C) + m * g.ldc + n;
                        if (g.vec) *reinterpret_cast<v4f*>(to) = v;
                        else
                            for (int r = 0; r < 4; ++r)
                                if (n + r < g.N) to[r] = v[r];
                    }
                }
            }
        }
    }
}


// ---------------------------------------------------------------- operands as bf16 planes
template <typename T, int P>
__global__ __launch_bounds__(256) void planes16_kernel(const T* __restrict__ X, int rows, int cols, int64_t ld, int vec,
                                                       const int64_t* __restrict__ targets, int64_t ignore, int V,
                                                       bf16* __restrict__ out, int ldp, int64_t chunks) {
    const int per_row = ldp >> 3;
    for (int64_t i = static_cast<int64_t>(blockIdx.x) * 256 + threadIdx.x; i < chunks; i += static_cast<int64_t>(gridDim.x) * 256) {
        const int64_t row = i / per_row;
        const int c = static_cast<int>(i - row * per_row) * 8;
        float v[8] = {};
        if (!targets || !no_loss(targets[row], ignore, V)) load8(X + row * ld, c, cols, vec, v);
#pragma unroll
        for (int p = 0; p < P; ++p) {
            v8bf o;
#pragma unroll
            for (int u = 0; u < 8; ++u) o[u] = piece_of(v[u], p);
            *reinterpret_cast<v8bf*>(out + p * (static_cast<int64_t>(rows) * ldp) + row * ldp + c) = o;
        }
    }
}

int launch_planes16(const void* X, int32_t dtype, int rows, int cols, int64_t ld, const int64_t* targets, int64_t ignore, int V,
                    bf16* out, int64_t ldp, hipStream_t st) {
    const int64_t chunks = rows * (ldp >> 3);
    const int64_t blocks = ceil_div64(chunks, 256);
    const dim3 grid(static_cast<unsigned>(blocks < 8192 ? blocks : 8192)), block(256);
    const int vec = ld * dtype_bytes(dtype) % 16 == 0, l = static_cast<int>(ldp);
    if (dtype == DAB_F32) return launch(planes16_kernel<float, 3>, grid, block, 0, st, static_cast<const float*>(X), rows, cols, ld, vec, targets, ignore, V, out, l, chunks);
    if (dtype == DAB_F16) return launch(planes16_kernel<f16, 2>, grid, block, 0, st, static_cast<const f16*>(X), rows, cols, ld, vec, targets, ignore, V, out, l, chunks);
    return launch(planes16_kernel<bf16, 1>, grid, block, 0, st, static_cast<const bf16*>(X), rows, cols, ld, vec, targets, ignore, V, out, l, chunks);
}

// ---------------------------------------------------------------- shares of a sum, added in a fixed order
__global__ __launch_bounds__(256) void join16_kernel(const float* __restrict__ part, int splits, int64_t n, const float* add,
                                                     void* C, int out_bf16) {
    for (int64_t i = static_cast<int64_t>(blockIdx.x) * 256 + threadIdx.x; i < n; i += static_cast<int64_t>(gridDim.x) * 256) {
        float v = add ? add[i] : 0.f;
        for (int s = 0; s < splits; ++s) v += part[s * n + i];
        if (out_bf16) static_cast<bf16*>(C)[i] = static_cast<bf16>(v);
        else static_cast<float*>(C)[i] = v;
    }
}

// ---------------------------------------------------------------- plan and launch
constexpr int kBigM = 256, kBigN = 256, kBigWM = 4, kBigWN = 2;
constexpr int kSmallM = 128, kSmallN = 128, kSmallWM = 2, kSmallWN = 2;
constexpr size_t lds_bytes16(int tm, int tn) { return static_cast<size_t>(2) * (tm + tn) * kStepK * 2; }

Plan16 plan16(int M, int N, int K, int n_seg, bool can_split) {
    Plan16 pl{};
    pl.steps = n_seg * ceil_div(K, kStepK);
    const int64_t big = static_cast<int64_t>(ceil_div(M, kBigM)) * ceil_div(N, kBigN);
    pl.big = big >= kNumCU * 3 / 4;
    pl.splits = 1;
    if (!pl.big && can_split) {
        const int64_t tiles = static_cast<int64_t>(ceil_div(M, kSmallM)) * ceil_div(N, kSmallN);
        int64_t s = 2 * kNumCU / tiles;
        if (s > pl.steps / 4) s = pl.steps / 4;
        pl.splits = static_cast<int>(s < 1 ? 1 : s);
    }
    pl.steps_per_split = ceil_div(pl.steps, pl.splits);
    pl.splits = ceil_div(pl.steps, pl.steps_per_split);
    pl.part_bytes = pl.splits > 1 ? static_cast<size_t>(pl.splits) * M * N * sizeof(float) : 0;
    return pl;
}

int stats_words16(const Plan16& pl) { return pl.big ? kBigN / kBigWN : kSmallN / kSmallWN; }

template <int EPI, bool ARC, bool BRC>
static auto kernel16(bool big) {
    return big ? product16_kernel<EPI, kBigM, kBigN, kBigWM, kBigWN, ARC, BRC>
               : product16_kernel<EPI, kSmallM, kSmallN, kSmallWM, kSmallWN, ARC, BRC>;
}

int launch16(int epi, bool arc, bool brc, Product16 g, const Plan16& pl, hipStream_t st) {
    const int tm = pl.big ? kBigM : kSmallM, tn = pl.big ? kBigN : kSmallN;
    g.tiles_m = ceil_div(g.M, tm), g.tiles_n = ceil_div(g.N, tn);
    g.splits = pl.splits, g.steps_per_split = pl.steps_per_split, g.steps = pl.steps;
    const int64_t units = static_cast<int64_t>(g.tiles_m) * g.tiles_n * g.splits;
    if (units > INT32_MAX / 2) return DAB_ERR_UNSUPPORTED;
    g.per_xcd = static_cast<int>(ceil_div64(units, kNumXCD));
    const auto kernel = epi == kEpiStats ? kernel16<kEpiStats, false, false>(pl.big)
                        : epi == kEpiSoftmax ? kernel16<kEpiSoftmax, false, false>(pl.big)
                        : arc ? kernel16<kEpiStore, true, true>(pl.big)
                              : kernel16<kEpiStore, false, true>(pl.big);
    if (brc != (epi == kEpiStore)) return DAB_ERR_UNSUPPORTED;
    const int threads = 64 * (pl.big ? kBigWM * kBigWN : kSmallWM * kSmallWN);
    if (int rc = launch(kernel, dim3(g.per_xcd * kNumXCD), dim3(threads), lds_bytes16(tm, tn), st, g)) return rc;
    if (pl.splits == 1) return DAB_OK;
    const int64_t n = static_cast<int64_t>(g.M) * g.N, blocks = ceil_div64(n, 256);
    return launch(join16_kernel, dim3(static_cast<unsigned>(blocks < 8192 ? blocks : 8192)), dim3(256), 0, st, g.part, g.splits, n,
                  g.add, g.C, g.out_bf16);
}

int init_product16() {
    for (int big = 0; big < 2; ++big)
        for (const auto k : {kernel16<kEpiStats, false, false>(big), kernel16<kEpiSoftmax, false, false>(big),
                             kernel16<kEpiStore, true, true>(big), kernel16<kEpiStore, false, true>(big)}) {
            const size_t lds = big ? lds_bytes16(kBigM, kBigN) : lds_bytes16(kSmallM, kSmallN);
            const hipError_t e = hipFuncSetAttribute(reinterpret_cast<const void*>(k), hipFuncAttributeMaxDynamicSharedMemorySize,
                                                     static_cast<int>(lds));
            if (e != hipSuccess) return hip_failed(e);
        }
    return DAB_OK;
}

}  // namespace dab

// ---------------------------------------------------------------- the weight gradient from a saved input
namespace dab {
struct GradPlan {
    Plan16 pl;
    bool direct;                     // dY is read where it is
    int64_t ldy, ldx;
    size_t x_at, y_at, part_at, bytes;
};
static GradPlan grad_plan(int32_t rows, int32_t cols, int32_t F, int32_t dtype, int64_t lddy) {
    GradPlan p{};
    const int P = dtype_pieces(dtype);
    p.direct = dtype == DAB_BF16 && F % 8 == 0 && lddy % 8 == 0;
    p.ldx = round_up(cols, 32);
    p.ldy = p.direct ? lddy : round_up(F, 8);
    p.pl = plan16(F, cols, rows, P, true);
    p.x_at = 0;
    p.y_at = round_up(static_cast<int64_t>(rows) * p.ldx * 2, 256);
    p.part_at = p.y_at + (p.direct ? 0 : round_up(static_cast<int64_t>(P) * rows * p.ldy * 2, 256));
    p.bytes = p.part_at + p.pl.part_bytes;
    return p;
}
static bool grad_sizes(int32_t rows, int32_t cols, int32_t F, int32_t dtype, int64_t lddy) {
    return real_dtype(dtype) && lddy < (1 << 23) && F < (1 << 23) && cols < (1 << 23) &&
           ceil_div64(F, 128) * ceil_div64(cols, 128) < INT32_MAX / 64;
}
}  // namespace dab

extern "C" size_t dab_ckpt8_weight_gradient_workspace_bytes(int32_t rows, int32_t cols, int32_t F, int32_t dtype, int64_t lddy) {
    using namespace dab;
    if (rows < 1 || cols < 1 || F < 1 || lddy < F || !grad_sizes(rows, cols, F, dtype, lddy)) return 0;
    return grad_plan(rows, cols, F, dtype, lddy).bytes;
}

extern "C" int dab_ckpt8_weight_gradient(const void* dY, int32_t dtype, int64_t lddy, const int8_t* Q, const uint8_t* S, int32_t rows,
                                         int32_t cols, int32_t F, float* dW, void* ws, size_t ws_bytes, void* stream) {
    using namespace dab;
    if (!dY || !Q || !S || !dW) return DAB_ERR_NULL;
    if (rows < 1 || cols < 1 || F < 1 || lddy < F) return DAB_ERR_SHAPE;
    if (!grad_sizes(rows, cols, F, dtype, lddy)) return DAB_ERR_UNSUPPORTED;
    if (misaligned(dY, 16) || misaligned(Q, 16) || misaligned(dW, 16)) return DAB_ERR_ALIGN;
    const GradPlan p = grad_plan(rows, cols, F, dtype, lddy);
    if (!ws || ws_bytes < p.bytes || misaligned(ws, 256)) return DAB_ERR_WORKSPACE;
    if (int rc = ensure_device_ready()) return rc;
    const auto st = static_cast<hipStream_t>(stream);
    char* base = static_cast<char*>(ws);
    bf16* x = reinterpret_cast<bf16*>(base + p.x_at);
    if (int rc = dab_ckpt8_restore(Q, S, rows, cols, x, DAB_BF16, p.ldx, stream)) return rc;
    const bf16* y = static_cast<const bf16*>(dY);
    if (!p.direct) {
        bf16* out = reinterpret_cast<bf16*>(base + p.y_at);
        if (int rc = launch_planes16(dY, dtype, rows, F, lddy, nullptr, 0, 0, out, p.ldy, st)) return rc;
        y = out;
    }
    Product16 g{};
    g.A = {y, p.ldy, static_cast<int64_t>(rows) * p.ldy};
    g.B = {x, p.ldx, 0};
    g.M = F, g.N = cols, g.K = rows;
    g.n_seg = dtype_pieces(dtype);
    for (int i = 0; i < g.n_seg; ++i) g.seg_a[i] = static_cast<uint8_t>(i);
    g.C = dW, g.ldc = cols, g.vec = cols % 4 == 0;
    g.part = reinterpret_cast<float*>(base + p.part_at);
    return launch16(kEpiStore, true, true, g, p.pl, st);
}
