// The products of product16.h: kernels, their tiles and shares, launches, the operands they need laid out, and the weight gradient
// from a saved input, which is one of them.
#include "product16.h"

#include <type_traits>

namespace dab {

// ---------------------------------------------------------------- the product
// Waits until no more than N of the wavefront's copies are on their way and its LDS reads have arrived, and for the other wavefronts.
template <int N = 0>
__device__ __forceinline__ void wait_and_meet() {
    asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" : : "n"(N) : "memory");
}

typedef __attribute__((address_space(3))) uint32_t lds_u32;
// A byte offset past every tile: a load from there gives zeros.  What a tile's offsets reach stays below it (ld < 2^22).
constexpr uint32_t kPast16 = 0x80000000u;
constexpr int kParts16 = 4;          // of a big tile in the last round of a product whose sums are not shared out

// One operand's tile of ROWS x 128 bytes of k (64 bf16 or 32 fp32), from memory into LDS.
template <typename E, int ROWS, bool RC, int NW>
struct Loader16 {
    static constexpr int kE = sizeof(E), kPer = 16 / kE, kStep = 128 / kE;
    static constexpr int kBytes = ROWS * 128;
    static constexpr int kCopies = kBytes / 1024 / NW;       // of one wavefront, a kilobyte each
    static constexpr int kChunks = RC ? ROWS / kPer : 8;     // 16-byte pieces of a row of the tile in LDS
    static constexpr int kLdsRows = 64 / kChunks;            // rows of it that one copy fills
    static_assert((ROWS & (ROWS - 1)) == 0 && (!RC || kE == 4 || ROWS >= 128), "the permutation stays within a row's pieces");
    static_assert(RC || kCopies == 1 || kCopies % 2 == 0, "the permutation of a row's pieces repeats every second copy");
    uint32_t off[kCopies];                                   // bytes from the tile's origin, the same every step
    uint64_t past[2];                                        // lanes whose k are past K in the last step, even and odd copies
    uint32_t reach;                                          // bytes of a k's rows ([k][rows]), or of all rows but the last
    __amdgpu_buffer_rsrc_t rsrc;
    int wave;

    // Bytes of n elements, in whole words of 32 bits (an odd number of bf16 has room behind it).
    static __device__ __forceinline__ uint32_t words(uint32_t n) { return kE == 4 ? n * 4 : (n + 1) / 2 * 4; }
    // A row's pieces are permuted in LDS so that the reads below meet no bank twice.  A copy's lanes are in order in LDS, so the
    // permutation is one of the addresses in memory.  rows: how many of the operand's rows are left from the tile's first on.
    __device__ __forceinline__ void init(int w, int lane, int64_t ld, int rows, int K) {
        wave = w;
        const int n = rows < ROWS ? rows : ROWS;
        reach = RC ? words(n) : (n - 1) * static_cast<uint32_t>(ld) * kE;
#pragma unroll
        for (int c = 0; c < kCopies; ++c) {
            const int r = (w * kCopies + c) * kLdsRows + lane / kChunks, phys = lane % kChunks;
            int e;
            if constexpr (RC) {
                const int key = (kE == 2 ? ((r & 3) | ((r >> 3) & 1) << 2) << 1 : ((r >> 2) & 3) << 2) & (kChunks - 1);
                e = (phys ^ key) * kPer;
                off[c] = e < rows ? static_cast<uint32_t>((r * ld + e) * kE) : kPast16;
            } else {
                e = (phys ^ ((r >> 1) & 7)) * kPer;
                off[c] = r < rows ? static_cast<uint32_t>((r * ld + e) * kE) : kPast16;
                if (c < 2) past[c] = __ballot(K % kStep != 0 && e >= K % kStep);
            }
        }
    }
    // origin: the tile's first element of this step; left: k from there on (none: zeros).
    // Nothing behind the operand's last word is read.  Rows past K are past the end of the buffer in one form, offsets of their own in the other.
    __device__ __forceinline__ void aim(const E* origin, int left, int64_t ld) {
        const uint32_t end = RC ? (left - 1) * (static_cast<uint32_t>(ld) * kE) + reach : reach + words(left);
        const uint32_t bytes = left <= 0 ? 0u : left <= kStep ? end : kPast16;
        rsrc = __builtin_amdgcn_make_buffer_rsrc(const_cast<E*>(origin), 0, static_cast<int>(bytes), 0x00020000);
    }
    __device__ __forceinline__ void copy(int c, bool last_k, char* lds) const {
        uint32_t o = off[c];
        if constexpr (!RC) o = __builtin_amdgcn_inverse_ballot_w64(last_k ? past[c & 1] : 0) ? kPast16 : o;
        // (in assembly because the compiler would have every later LDS read wait for the copy; what may be read is behind wait_and_meet())
#pragma clang diagnostic push
#pragma clang diagnostic ignored "-Winline-asm"               // (m0 is named as clobbered, which nothing else here uses)
        asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tbuffer_load_dwordx4 %1, %2, 0 offen lds"
                     : : "s"(static_cast<uint32_t>(reinterpret_cast<uintptr_t>((lds_u32*)(lds + (wave * kCopies + c) * 1024)))), "v"(o), "s"(rsrc) : "m0");
#pragma clang diagnostic pop
    }
};

// Fragments of 16 rows, half a step of k: lane l holds row l % 16 and 16 bytes of k from piece l / 16 of the half on, eight bf16 or four fp32.
template <typename E, int ROWS, bool RC, int NFRAG>
struct Reader16 {
    static constexpr bool kWide = sizeof(E) == 4;
    using Frag = std::conditional_t<kWide, v4f, v8bf>;
    static constexpr int kPitch = ROWS * static_cast<int>(sizeof(E));   // bytes of a k in the form [k][rows]
    uint32_t at[RC ? NFRAG : 2];
    // row0: this wavefront's first row in the tile
    __device__ __forceinline__ void init(int lane, int row0) {
        const int s = lane & 15, g = lane >> 4;
        if constexpr (RC) {
#pragma unroll
            for (int j = 0; j < NFRAG; ++j) {
                const int block = (row0 >> 4) + j;
                if constexpr (kWide) {
                    at[j] = g * 4 * kPitch + (block ^ (g & (ROWS / 16 - 1))) * 64 + s * 4;
                } else {
                    // a group of 16 lanes reads 4 k x 16 rows, a lane 4 neighbouring rows of one k, and gets the four k of its row
                    at[j] = (g * 8 + (s >> 2)) * kPitch + (block ^ ((s >> 2) | (g & 1) << 2)) * 32 + (s & 3) * 8;
                }
            }
        } else {
            const int row = row0 + s, key = s >> 1;
#pragma unroll
            for (int kk = 0; kk < 2; ++kk) at[kk] = row * 128 + (((kk * 4 + g) ^ key) * 16);
        }
    }
    __device__ __forceinline__ Frag read(const char* lds, int kk, int j) const {
        if constexpr (RC && kWide) {
            v4f v;
#pragma unroll
            for (int c = 0; c < 4; ++c) v[c] = *reinterpret_cast<const float*>(lds + at[j] + (kk * 16 + c) * kPitch);
            return v;
        } else if constexpr (RC) {
            typedef short v4s __attribute__((ext_vector_type(4)));
            typedef __attribute__((address_space(3))) v4s lds_v4s;
            union { v4s h[2]; v8bf v; } u;
            const char* p = lds + at[j] + kk * 32 * kPitch;
            u.h[0] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_v4s*)p);
            u.h[1] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_v4s*)(p + 4 * kPitch));
            return u.v;
        } else {
            return *reinterpret_cast<const Frag*>(lds + at[kk] + j * 16 * 128);
        }
    }
};
// One half step's product of two fragments (which k a lane holds does not matter as long as both operands agree).
__device__ __forceinline__ v4f multiply16(v8bf a, v8bf b, v4f c) { return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0); }
__device__ __forceinline__ v4f multiply16(v4f a, v4f b, v4f c) {
#pragma unroll
    for (int u = 0; u < 4; ++u) c = __builtin_amdgcn_mfma_f32_16x16x4f32(a[u], b[u], c, 0, 0, 0);
    return c;
}

// Four neighbouring columns of the result.
template <typename T>
__device__ __forceinline__ void store4(T* to, v4f v, int columns) {
    typedef T v4t __attribute__((ext_vector_type(4)));
    const v4t out = __builtin_convertvector(v, v4t);
    if (columns >= 4) {
        *reinterpret_cast<typename Unaligned<T, 4>::type*>(to) = out;
        return;
    }
#pragma unroll
    for (int r = 0; r < 4; ++r)
        if (r < columns) to[r] = out[r];
}
// What a row's sums become as they are stored: times the factor, or zeros, of a token without a loss (not its products: P's zeros times a word
// that is no number are not 0).
struct RowEnd {
    float factor;
    bool none;
    __device__ __forceinline__ RowEnd(const Product16& g, int m)
        : factor(g.factor ? *g.factor : 1.f), none(g.targets && no_loss(g.targets[m], g.ignore_index, g.V)) {}
};
__device__ __forceinline__ void store16(const Product16& g, int m, int n, v4f v, RowEnd end) {
    if (n >= g.N) return;
    if (g.add) {
        const float* from = g.add + static_cast<int64_t>(m) * g.N + n;
#pragma unroll
        for (int r = 0; r < 4; ++r) v[r] += n + r < g.N ? from[r] : 0.f;
    }
    v = end.none ? v4f{0.f, 0.f, 0.f, 0.f} : v * end.factor;
    if (g.out_bf16) store4(static_cast<bf16*>(g.C) + m * g.ldc + n, v, g.N - n);
    else store4(static_cast<float*>(g.C) + m * g.ldc + n, v, g.N - n);
}

// 16 rows of a wavefront's result through LDS (its own part, 16 rows x FN x 16 columns), so that rows are stored in whole lines instead of
// a quarter of one: one token's dW, 131072 x 4096 bf16, 431 -> 220 us.  put(): this lane's four columns of block i, as
// they are stored; flush(): rows in order, 16 bytes a lane.  A row's 16-byte pieces are permuted so that neither meets a bank twice.
template <typename T, int FN>
struct Rows16 {
    static constexpr int kRow = FN * 16 * static_cast<int>(sizeof(T)), kChunks = kRow / 16, kLanes = kChunks < 64 ? kChunks : 64;
    char* lds;
    int lane;
    __device__ __forceinline__ void put(int i, v4f v) const {
        typedef T v4t __attribute__((ext_vector_type(4)));
        const int row = lane & 15, byte = (i * 16 + (lane >> 4) * 4) * static_cast<int>(sizeof(T));
        *reinterpret_cast<v4t*>(lds + row * kRow + (((byte >> 4) ^ row) & (kChunks - 1)) * 16 + (byte & 15)) = __builtin_convertvector(v, v4t);
    }
    // row0: address of the first row's first column; columns: how many there are from it on
    __device__ __forceinline__ void flush(T* row0, int64_t ld, int rows, int columns) const {
        const int c = lane % kLanes;
#pragma unroll
        for (int r0 = 0; r0 < 16; r0 += 64 / kLanes) {
            const int r = r0 + lane / kLanes;
            const v4u32 v = *reinterpret_cast<const v4u32*>(lds + r * kRow + ((c ^ r) & (kChunks - 1)) * 16);
            constexpr int kElems = 16 / static_cast<int>(sizeof(T));
            const int left = columns - c * kElems;
            T* to = row0 + r * ld + c * kElems;
            if (r >= rows) continue;
            if (left >= kElems) {
                *reinterpret_cast<Unaligned<uint32_t, 4>::type*>(to) = v;
            } else {
                // the last columns of a row whose number is no multiple of a piece's
#pragma unroll
                for (int u = 0; u < kElems; ++u) {
                    const uint32_t bits = sizeof(T) == 4 ? v[u & 3] : v[(u >> 1) & 3] >> (16 * (u & 1));
                    if (u < left) {
                        if constexpr (sizeof(T) == 4) to[u] = __uint_as_float(bits);
                        else to[u] = __builtin_bit_cast(T, static_cast<uint16_t>(bits));
                    }
                }
            }
        }
    }
};

// NS: steps in LDS.  TAIL: the operands' rows may hold anything behind K.  PARTS: the tile is one of that many, one above the other, of a tile of the last round.
template <typename E, int EPI, int TM, int TN, int WM, int WN, bool ARC, bool BRC, int NS, bool TAIL = false, int PARTS = 1>
__device__ __forceinline__ void product16(const Product16& g) {
    constexpr int NW = WM * WN, FM = TM / WM / 16, FN = TN / WN / 16;
    using LA = Loader16<E, TM, ARC, NW>;
    using LB = Loader16<E, TN, BRC, NW>;
    constexpr int kStep = LA::kStep, kE = sizeof(E);
    constexpr int kBuf = LA::kBytes + LB::kBytes;
    extern __shared__ __attribute__((aligned(1024))) char lds[];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);

    // Consecutive workgroups go to the XCDs in turn: each XCD gets neighbouring tiles, eight rows of tiles at a time, so
    // that what runs on it together shares operands in its L2.  The tiles that would leave a last round half empty are taken in shares.
    // (quotients come from vector instructions; what is made of them here has to be scalar)
    int tile, first = 0, last = g.steps, share = -1, part = 0;
    if (PARTS == 1 && static_cast<int>(blockIdx.x) < 8 * g.whole_xcd) {
        tile = (blockIdx.x & 7) * g.whole_xcd + (blockIdx.x >> 3);
        if (tile >= g.whole) return;
    } else {
        const int b = blockIdx.x - 8 * g.whole_xcd, unit = (b & 7) * g.rest_xcd + (b >> 3);
        if (unit >= g.rest * g.shares) return;
        const int sh = __builtin_amdgcn_readfirstlane(unit / g.rest);
        tile = g.whole + unit - sh * g.rest;
        if (PARTS > 1) part = sh;
        else if (g.shares > 1) share = sh, first = sh * g.share_steps, last = min(first + g.share_steps, g.steps);
    }
    const int band = __builtin_amdgcn_readfirstlane(tile / (8 * g.tiles_n)), in_band = tile - band * 8 * g.tiles_n;
    const int bm = min(8, g.tiles_m - band * 8);
    const int tn = __builtin_amdgcn_readfirstlane(in_band / bm), tm = band * 8 + in_band - tn * bm;
    const int m0 = (tm * PARTS + part) * TM, n0 = tn * TN;
    if (PARTS > 1 && m0 >= g.M) return;
    const int wm = wave % WM, wn = wave / WM;

    LA la;
    LB lb;
    la.init(wave, lane, g.A.ld, g.M - m0, g.K);
    lb.init(wave, lane, g.B.ld, g.N - n0, g.K);
    const E* a0 = static_cast<const E*>(g.A.p) + (ARC ? m0 : m0 * g.A.ld);
    const E* b0 = static_cast<const E*>(g.B.p) + (BRC ? n0 : n0 * g.B.ld);
    const int64_t ka = kStep * (ARC ? g.A.ld : 1), kb = kStep * (BRC ? g.B.ld : 1);   // a step further

    const int per_seg = __builtin_amdgcn_readfirstlane(g.steps / g.n_seg);
    // the step that is fetched next: how many are left, its pair of planes, its operands and k left there
    int to_fetch = last - first, seg = __builtin_amdgcn_readfirstlane(first / per_seg), k_left = g.K - (first - seg * per_seg) * kStep;
    const E* pa = a0 + ((g.seg_a >> (4 * seg)) & 15) * g.A.plane + (first - seg * per_seg) * ka;
    const E* pb = b0 + ((g.seg_b >> (4 * seg)) & 15) * g.B.plane + (first - seg * per_seg) * kb;
    bool last_k = false;
    auto aim = [&] {
        const int left = to_fetch > 0 ? k_left : 0;
        la.aim(pa, left, g.A.ld);
        lb.aim(pb, left, g.B.ld);
        last_k = k_left < kStep;
        --to_fetch, k_left -= kStep, pa += ka, pb += kb;
        if (k_left <= 0 && to_fetch > 0) {
            ++seg, k_left = g.K;
            pa = a0 + ((g.seg_a >> (4 * seg)) & 15) * g.A.plane;
            pb = b0 + ((g.seg_b >> (4 * seg)) & 15) * g.B.plane;
        }
    };
    auto fetch = [&](char* buf) {
#pragma unroll
        for (int c = 0; c < LA::kCopies; ++c) la.copy(c, last_k, buf);
#pragma unroll
        for (int c = 0; c < LB::kCopies; ++c) lb.copy(c, last_k, buf + LA::kBytes);
    };

    // An operand that is read where it is has rows of whole words, not of whole pieces: what the last piece of a row holds behind K is
    // cleared in LDS, in both operands (one's zeros would not do: the other's may be a NaN).
    const int tail = TAIL && g.tail && last == g.steps ? static_cast<int>(LB::words(g.K % LB::kPer) / 4) : 0;
    auto clear = [&](char* buf) {
        const int piece = g.K % kStep / LB::kPer;
        for (int r = threadIdx.x; r < TM + TN; r += 64 * NW) {
            // (B's rows follow A's, and both begin a permutation: TM is a multiple of 16)
            uint32_t* at = reinterpret_cast<uint32_t*>(buf + r * 128 + (piece ^ ((r >> 1) & 7)) * 16);
            for (int u = tail; u < 4; ++u) at[u] = 0;
        }
        wait_and_meet<(NS - 2) * (LA::kCopies + LB::kCopies)>();
    };

    Reader16<E, TM, ARC, FM> ra;
    Reader16<E, TN, BRC, FN> rb;
    ra.init(lane, wm * FM * 16);
    rb.init(lane, wn * FN * 16);

    // (a scalar load: an earlier launch has written it)
    auto factor_of = [&](int which) {
        typedef const __attribute__((address_space(4))) float scalar_f32;
        return g.factor ? reinterpret_cast<scalar_f32*>(reinterpret_cast<uintptr_t>(g.factor))[which] : 1.f;
    };
    float factor = EPI == kEpiStore ? factor_of(0) : 1.f;

    v4f acc[FN][FM];
#pragma unroll
    for (int i = 0; i < FN; ++i)
#pragma unroll
        for (int j = 0; j < FM; ++j) acc[i][j] = v4f{0.f, 0.f, 0.f, 0.f};
    typename decltype(ra)::Frag a[2][FM], b[2][FN];
    // Half a step: its products, and among them the reads of the next half's fragments (early, so that they have arrived by its
    // end) and, COPY, the copies of a later step, one at a time: a burst of either would hold up the products behind it.
    auto half = [&](auto copy_c, int set, const char* buf, int kk, char* to) {
        constexpr bool COPY = decltype(copy_c)::value;
        constexpr int kCopies = LA::kCopies + LB::kCopies, kEarly = FN / 2;
#pragma unroll
        for (int i = 0; i < FN; ++i) {
            if constexpr (COPY)
#pragma unroll
                for (int c = kCopies * i / FN; c < kCopies * (i + 1) / FN; ++c) {
                    if (c < LA::kCopies) la.copy(c, last_k, to);
                    else lb.copy(c - LA::kCopies, last_k, to + LA::kBytes);
                }
            if (i < kEarly) {
#pragma unroll
                for (int j = FM * i / kEarly; j < FM * (i + 1) / kEarly; ++j) a[set ^ 1][j] = ra.read(buf, kk, j);
#pragma unroll
                for (int u = 2 * i; u < 2 * i + 2; ++u) b[set ^ 1][u] = rb.read(buf + LA::kBytes, kk, u);
            }
#pragma unroll
            for (int j = 0; j < FM; ++j) acc[i][j] = multiply16(b[set][i], a[set][j], acc[i][j]);
            __builtin_amdgcn_sched_barrier(0);
        }
    };
    using yes = std::integral_constant<bool, true>;
    using no = std::integral_constant<bool, false>;

    // NS buffers of a step.  While a half step is multiplied from registers, the next one's fragments are read; behind the one barrier of a
    // step, in its middle, the next step has landed (those after it may be on their way) and its own buffer has been read by all, so step NS further on
    // is fetched into it.
    constexpr int kInFlight = LA::kCopies + LB::kCopies;     // copies of a wavefront for a step
    if constexpr (NS == 2) {
        aim();
        fetch(lds);
        wait_and_meet();
        aim();
        fetch(lds + kBuf);
    } else {
#pragma unroll
        for (int i = 0; i < NS; ++i) {
            aim();
            fetch(lds + i * kBuf);
        }
        wait_and_meet<(NS - 1) * kInFlight>();
    }
    if constexpr (EPI == kEpiStore) asm volatile("" : "+s"(factor));   // (arrived by now; the compiler would load it at the end)
    if (TAIL && tail && last - first == 1) clear(lds);
#pragma unroll
    for (int j = 0; j < FM; ++j) a[0][j] = ra.read(lds, 0, j);
#pragma unroll
    for (int i = 0; i < FN; ++i) b[0][i] = rb.read(lds + LA::kBytes, 0, i);
    auto step = [&](auto end_c, int s) {
        char* cur = lds + ((s - first) & (NS - 1)) * kBuf;
        char* other = lds + ((s + 1 - first) & (NS - 1)) * kBuf;
        aim();
        half(no{}, 0, cur, 1, cur);
        wait_and_meet<(NS - 2) * kInFlight>();
        if (decltype(end_c)::value && tail && s + 2 == last) clear(other);
        half(yes{}, 1, other, 0, cur);
    };
    int s = first;
    for (; s < last - (TAIL ? 2 : 0); ++s) step(no{}, s);
    // (apart from the others: with the question in all of them the logits' products took 3 % longer)
    if (TAIL)
        for (; s < last; ++s) step(yes{}, s);
    // (copies and reads past the last step: zeros, and not used; the wavefront waits for them before it ends)
    wait_and_meet();

    const int mw = m0 + wm * FM * 16 + (lane & 15), nb = n0 + wn * FN * 16, nw = nb + (lane >> 4) * 4;
    const bool full = n0 + TN <= g.N;                        // no column past the last one
    char* mine = lds + wave * (16 * FN * 16 * 4);
    // what a token's row needs, all of it requested before the first is used
    int64_t target[FM];
    float lse[FM], weight[FM];
    if constexpr (EPI != kEpiStore) {
        if constexpr (EPI == kEpiSoftmax) factor = factor_of(1);
#pragma unroll
        for (int j = 0; j < FM; ++j) {
            const int m = min(mw + j * 16, g.M - 1);
            target[j] = g.targets[m];
            if constexpr (EPI == kEpiSoftmax) lse[j] = g.lse[m], weight[j] = g.g ? g.g[m] * factor : 1.f;
        }
    }
#pragma unroll
    for (int j = 0; j < FM; ++j) {
        const int m = mw + j * 16, mj = m0 + wm * FM * 16 + j * 16;
        const bool in = m < g.M;
        if constexpr (EPI == kEpiStats) {
            // maximum and sum of exponentials of this wavefront's words, one pair per token
            if (!full) {
#pragma unroll
                for (int i = 0; i < FN; ++i)
#pragma unroll
                    for (int r = 0; r < 4; ++r)
                        if (nw + i * 16 + r >= g.N) acc[i][j][r] = -__builtin_inff();
            }
            float big = -__builtin_inff();
#pragma unroll
            for (int i = 0; i < FN; ++i) big = fmaxf(fmaxf(fmaxf(big, acc[i][j][0]), fmaxf(acc[i][j][1], acc[i][j][2])), acc[i][j][3]);
            big = fmaxf(big, __shfl_xor(big, 16));
            big = fmaxf(big, __shfl_xor(big, 32));
            const float at = big == -__builtin_inff() ? 0.f : big;
            float sum = 0.f;
#pragma unroll
            for (int i = 0; i < FN; ++i) {
                float four = 0.f;
#pragma unroll
                for (int r = 0; r < 4; ++r) four += __expf(acc[i][j][r] - at);
                sum += four;
            }
            sum += __shfl_xor(sum, 16);
            sum += __shfl_xor(sum, 32);
            if (in && lane < 16) g.stats[static_cast<int64_t>(tn * WN + wn) * g.M + m] = float2{big, sum};
            const int64_t t = target[j];
            if (in && t >= nw && t < g.N) {
                const int d = static_cast<int>(t) - nw;
#pragma unroll
                for (int i = 0; i < FN; ++i)
#pragma unroll
                    for (int r = 0; r < 4; ++r)
                        if (d == i * 16 + r) g.target_logit[m] = acc[i][j][r];
            }
        } else if constexpr (EPI == kEpiSoftmax) {
            const int64_t t = target[j];
            const bool dead = !in || no_loss(t, g.ignore_index, g.V);
            const float base = dead ? 0.f : lse[j], w = dead ? 0.f : weight[j];
            // the target's column, counted from this lane's first
            const int64_t d64 = dead ? -1 : t - g.n0 - nw;
            const int d = d64 < 0 || d64 >= FN * 16 ? -1 : static_cast<int>(d64);
            const bool hit = __ballot(d >= 0) != 0;
#pragma unroll
            for (int i = 0; i < FN; ++i) {
                v4f p;
#pragma unroll
                for (int r = 0; r < 4; ++r) p[r] = __expf(acc[i][j][r] - base);
                if (hit) {
#pragma unroll
                    for (int r = 0; r < 4; ++r) p[r] -= d == i * 16 + r ? 1.f : 0.f;
                }
                p *= w;
                if (!full || dead) {
#pragma unroll
                    for (int r = 0; r < 4; ++r) p[r] = dead || nw + i * 16 + r >= g.N ? 0.f : p[r];
                }
                acc[i][j] = p;
            }
            if constexpr (kE == 4) {
                const Rows16<float, FN> out{mine, lane};
#pragma unroll
                for (int i = 0; i < FN; ++i) out.put(i, acc[i][j]);
                out.flush(static_cast<float*>(g.P) + mj * g.ldp + nb, g.ldp, g.M - mj, FN * 16);
                continue;
            }
            const Rows16<bf16, FN> out{mine, lane};
            for (int q = 0; q < g.p_planes; ++q) {
#pragma unroll
                for (int i = 0; i < FN; ++i) {
                    out.put(i, acc[i][j]);
                    if (q + 1 < g.p_planes)
#pragma unroll
                        for (int r = 0; r < 4; ++r) acc[i][j][r] -= static_cast<float>(static_cast<bf16>(acc[i][j][r]));
                }
                out.flush(static_cast<bf16*>(g.P) + q * g.p_plane + mj * g.ldp + nb, g.ldp, g.M - mj, FN * 16);
            }
        } else if (share >= 0) {
#pragma unroll
            for (int i = 0; i < FN; ++i)
                *reinterpret_cast<v4f*>(g.part + ((static_cast<int64_t>(tile - g.whole) * g.shares + share) * (FN * FM) + i * FM + j) * (256 * NW) +
                                        threadIdx.x * 4) = acc[i][j];
        } else if (!g.add) {
            if (g.factor) {
#pragma unroll
                for (int i = 0; i < FN; ++i) acc[i][j] *= factor;
            }
            if (g.targets && no_loss(g.targets[min(m, g.M - 1)], g.ignore_index, g.V)) {
#pragma unroll
                for (int i = 0; i < FN; ++i) acc[i][j] = v4f{0.f, 0.f, 0.f, 0.f};
            }
            if (g.out_bf16) {
                const Rows16<bf16, FN> out{mine, lane};
#pragma unroll
                for (int i = 0; i < FN; ++i) out.put(i, acc[i][j]);
                out.flush(static_cast<bf16*>(g.C) + mj * g.ldc + nb, g.ldc, g.M - mj, g.N - nb);
            } else {
                const Rows16<float, FN> out{mine, lane};
#pragma unroll
                for (int i = 0; i < FN; ++i) out.put(i, acc[i][j]);
                out.flush(static_cast<float*>(g.C) + mj * g.ldc + nb, g.ldc, g.M - mj, g.N - nb);
            }
        } else if (in) {
            const RowEnd end(g, m);
#pragma unroll
            for (int i = 0; i < FN; ++i) store16(g, m, nw + i * 16, acc[i][j], end);
        }
    }
}

template <int EPI, int TM, int TN, int WM, int WN, bool ARC, bool BRC>
__global__ __launch_bounds__(64 * WM * WN, WM * WN / 4) void product16_kernel(Product16 g) {
    product16<bf16, EPI, TM, TN, WM, WN, ARC, BRC, 2>(g);
}
// Logits whose operands' rows may hold anything behind K; and, as sums that a softmax needs whole are not shared out, whose big tiles of the last round
// are taken in four parts.
template <int EPI, int TM, int TN, int WM, int WN>
__global__ __launch_bounds__(64 * WM * WN, WM * WN / 4) void product16_ends_kernel(Product16 g) {
    if constexpr (TM == 256)
        if (static_cast<int>(blockIdx.x) >= 8 * g.whole_xcd) {
            product16<bf16, EPI, TM / kParts16, TN, WM, WN, false, false, 2, true, kParts16>(g);
            return;
        }
    product16<bf16, EPI, TM, TN, WM, WN, false, false, 2, true>(g);
}
// For no more tiles than compute units: with one workgroup on each, a step of the small tile takes as long as its copies, so four
// steps are on their way instead of two.
template <int EPI, int TM, int TN, int WM, int WN, bool ARC, bool BRC>
__global__ __launch_bounds__(64 * WM * WN, WM * WN / 4) void product16_deep_kernel(Product16 g) {
    product16<bf16, EPI, TM, TN, WM, WN, ARC, BRC, 4>(g);
}
template <int EPI, int TM, int TN, int WM, int WN>
__global__ __launch_bounds__(64 * WM * WN, WM * WN / 4) void product16_deep_ends_kernel(Product16 g) {
    product16<bf16, EPI, TM, TN, WM, WN, false, false, 4, true>(g);
}
// fp32 operands as they are, on the matrix cores' fp32 form.
template <int EPI, int TM, int TN, int WM, int WN, bool ARC, bool BRC>
__global__ __launch_bounds__(64 * WM * WN, WM * WN / 4) void product32_kernel(Product16 g) {
    product16<float, EPI, TM, TN, WM, WN, ARC, BRC, 2, !BRC>(g);
}

// The shares of a tile's sums, added in a fixed order.  A workgroup takes one 16 x 16 block of every wavefront; eight shares
// are on their way at a time.
template <int TM, int TN, int WM, int WN>
__global__ __launch_bounds__(64 * WM * WN) void join16_kernel(Product16 g) {
    DAB_RESERVE_VGPRS();
    constexpr int NW = WM * WN, FM = TM / WM / 16, FN = TN / WN / 16;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int rest_tile = blockIdx.x / (FN * FM), block = blockIdx.x - rest_tile * (FN * FM), i = block / FM, j = block - i * FM;
    const int tile = g.whole + rest_tile;
    const int band = tile / (8 * g.tiles_n), in_band = tile - band * 8 * g.tiles_n, bm = min(8, g.tiles_m - band * 8);
    const int tn = in_band / bm, tm = band * 8 + in_band - tn * bm;
    const int n = tn * TN + (wave / WM * FN + i) * 16 + (lane >> 4) * 4, m = tm * TM + (wave % WM * FM + j) * 16 + (lane & 15);
    if (m >= g.M || n >= g.N) return;
    const RowEnd end(g, m);                                  // (requested before the sums)
    constexpr int64_t kNext = static_cast<int64_t>(FN * FM) * 256 * NW;
    const float* from = g.part + static_cast<int64_t>(rest_tile) * g.shares * kNext + block * (256 * NW) + threadIdx.x * 4;
    v4f v = v4f{0.f, 0.f, 0.f, 0.f};
    for (int s = 0; s < g.shares; s += 8) {
        v4f got[8];
#pragma unroll
        for (int u = 0; u < 8; ++u) got[u] = *reinterpret_cast<const v4f*>(from + min(s + u, g.shares - 1) * kNext);
#pragma unroll
        for (int u = 0; u < 8; ++u)
            if (s + u < g.shares) v += got[u];
    }
    store16(g, m, n, v, end);
}

// ---------------------------------------------------------------- operands as bf16 planes
// (bound by memory: 8192 x 2048 bf16 rows with some cleared 12 us, 5.5 TB/s; the weights' factor is found by a workgroup of its own in front of
// the others, 1024 tokens at a time: behind them it ended last, 14.5 us)
__device__ __forceinline__ void weights_factor(const float* __restrict__ g, const int64_t* __restrict__ targets, int64_t ignore, int V, int rows,
                                               float* __restrict__ factor) {
    __shared__ int found[4];
    float by = 1.f;
    for (int64_t t0 = 0; t0 < rows; t0 += 1024) {
        int first = INT32_MAX;
#pragma unroll
        for (int u = 3; u >= 0; --u) {
            const int t = static_cast<int>(min(t0 + u * 256 + threadIdx.x, static_cast<int64_t>(rows) - 1));
            const uint32_t size = __float_as_uint(g[t]) & 0x7fffffffu;
            // (0, subnormal numbers, infinities and NaN have no significand to divide by)
            if (!no_loss(targets[t], ignore, V) && size >= 0x00800000u && size < 0x7f800000u) first = t;
        }
#pragma unroll
        for (int d = 1; d < 64; d *= 2) first = min(first, __shfl_xor(first, d));
        if ((threadIdx.x & 63) == 0) found[threadIdx.x >> 6] = first;
        __syncthreads();
        first = min(min(found[0], found[1]), min(found[2], found[3]));
        __syncthreads();
        if (first == INT32_MAX) continue;
        by = __uint_as_float((__float_as_uint(g[first]) & 0x007fffffu) | 0x3f800000u);
        break;
    }
    if (threadIdx.x == 0) factor[0] = by, factor[1] = 1.f / by;
}
template <typename T, int P>
__global__ __launch_bounds__(256) void planes16_kernel(const T* __restrict__ X, int rows, int cols, int64_t ld,
                                                       const int64_t* __restrict__ targets, int64_t ignore, int V,
                                                       bf16* __restrict__ out, int ldp, int64_t chunks, unsigned blocks,
                                                       const float* __restrict__ g, float* __restrict__ factor) {
    const unsigned lead = gridDim.x - blocks;
    if (blockIdx.x < lead) {
        weights_factor(g, targets, ignore, V, rows, factor);
        return;
    }
    const int per_row = ldp >> 3;
    for (int64_t i = static_cast<int64_t>(blockIdx.x - lead) * 256 + threadIdx.x; i < chunks; i += static_cast<int64_t>(blocks) * 256) {
        const int64_t row = i / per_row;
        const int c = static_cast<int>(i - row * per_row) * 8;
        float v[8] = {};
        if (!targets || !no_loss(targets[row], ignore, V)) load8(X + row * ld, c, cols, v);
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
                    bf16* out, int64_t ldp, hipStream_t st, const float* g, float* factor) {
    const int64_t chunks = rows * (ldp >> 3);
    const unsigned blocks = static_cast<unsigned>(ceil_div64(chunks, 256) < 8192 ? ceil_div64(chunks, 256) : 8192);
    const dim3 grid(blocks + (factor ? 1 : 0)), block(256);
    const int l = static_cast<int>(ldp);
    if (dtype == DAB_F32) return launch(planes16_kernel<float, 3>, grid, block, 0, st, static_cast<const float*>(X), rows, cols, ld, targets, ignore, V, out, l, chunks, blocks, g, factor);
    return launch(planes16_kernel<bf16, 1>, grid, block, 0, st, static_cast<const bf16*>(X), rows, cols, ld, targets, ignore, V, out, l, chunks, blocks, g, factor);
}

// fp32 rows [rows][cols] as they are, ldp apart (a multiple of 4, zeros behind the last element); those of tokens without a loss cleared
// (targets may be NULL).
__global__ __launch_bounds__(256) void rows32_kernel(const float* __restrict__ X, int cols, int64_t ld, const int64_t* __restrict__ targets,
                                                     int64_t ignore, int V, float* __restrict__ out, int ldp, int64_t chunks) {
    const int per_row = ldp >> 2;
    for (int64_t i = static_cast<int64_t>(blockIdx.x) * 256 + threadIdx.x; i < chunks; i += static_cast<int64_t>(gridDim.x) * 256) {
        const int64_t row = i / per_row;
        const int c = static_cast<int>(i - row * per_row) * 4;
        const float* from = X + row * ld + c;
        v4f v = v4f{0.f, 0.f, 0.f, 0.f};
        if (!targets || !no_loss(targets[row], ignore, V)) {
            if (c + 4 <= cols) {
                v = *reinterpret_cast<const Unaligned<float, 4>::type*>(from);
            } else {
#pragma unroll
                for (int u = 0; u < 4; ++u)
                    if (c + u < cols) v[u] = from[u];
            }
        }
        *reinterpret_cast<v4f*>(out + row * ldp + c) = v;
    }
}
int launch_rows32(const float* X, int rows, int cols, int64_t ld, const int64_t* targets, int64_t ignore, int V, float* out, int64_t ldp,
                  hipStream_t st) {
    const int64_t chunks = rows * (ldp >> 2), blocks = ceil_div64(chunks, 256);
    return launch(rows32_kernel, dim3(static_cast<unsigned>(blocks < 8192 ? blocks : 8192)), dim3(256), 0, st, X, cols, ld, targets, ignore, V,
                  out, static_cast<int>(ldp), chunks);
}

// ---------------------------------------------------------------- plan and launch
constexpr int kBigM = 256, kBigN = 256, kBigWM = 4, kBigWN = 2;
constexpr int kSmallM = 128, kSmallN = 128, kSmallWM = 2, kSmallWN = 2;
constexpr int kF32M = 64, kF32N = 128, kF32WM = 2, kF32WN = 2;
// of up to 32 rows, and of few tiles (one token's logits, 64000 x 2048: with 64 rows 142 us, which is the matrix cores', with these 88)
constexpr int kFewM = 32, kFewN = 128, kFewWM = 1, kFewWN = 4;
constexpr bool wide16(Tiles16 kind) { return kind == Tiles16::kF32 || kind == Tiles16::kFew; }
constexpr int tile_m16(Tiles16 kind) {
    return kind == Tiles16::kBig ? kBigM : kind == Tiles16::kF32 ? kF32M : kind == Tiles16::kFew ? kFewM : kSmallM;
}
constexpr int tile_n16(Tiles16 kind) {
    return kind == Tiles16::kBig ? kBigN : kind == Tiles16::kF32 ? kF32N : kind == Tiles16::kFew ? kFewN : kSmallN;
}
constexpr size_t lds_bytes16(Tiles16 kind) { return (kind == Tiles16::kDeep ? size_t{4} : size_t{2}) * (tile_m16(kind) + tile_n16(kind)) * 128; }

// Time of a product in one kind of tiles, in microseconds: rounds of workgroups over the compute units, the last of them in shares (or, of
// logits, parts of tiles) where that takes less.
static Plan16 plan16_of(Tiles16 kind, int M, int N, int K, int n_seg, size_t share_bytes, bool logits) {
    // Workgroups that a compute unit runs together; a step's time with all of them there, that of one alone (fp32 products are bound by the
    // matrix cores, which the workgroups share), and that of a tile's beginning and end: those of long sums on a full chip, of
    // the deep form of few tiles.
    struct Cost {
        int together;
        double step, alone, ends;
    };
    const Cost cost = kind == Tiles16::kBig    ? Cost{1, 1.6, 1.6, 5.0}
                      : kind == Tiles16::kDeep ? Cost{1, 0.6, 0.6, 4.0}
                      : kind == Tiles16::kF32  ? Cost{3, 3.0, 1.1, 4.0}
                      : kind == Tiles16::kFew  ? Cost{3, 1.6, 0.7, 4.0}
                                               : Cost{2, 1.1, 1.1, 3.0};
    const int slots = kNumCU * cost.together;
    const int64_t tile_bytes = static_cast<int64_t>(tile_m16(kind)) * tile_n16(kind) * 4;
    Plan16 pl{};
    pl.tiles = kind;
    pl.steps = n_seg * ceil_div(K, wide16(kind) ? kStepK / 2 : kStepK);
    const int64_t tiles = static_cast<int64_t>(ceil_div(M, tile_m16(kind))) * ceil_div(N, tile_n16(kind));
    auto round = [&](int64_t units, int steps) {
        const int on_one = ceil_div(static_cast<int>(units), kNumCU);
        return steps * (on_one >= cost.together ? cost.step : cost.alone + (cost.step - cost.alone) * (on_one - 1) / cost.together) + cost.ends;
    };
    const int64_t rounds = tiles / slots;
    pl.whole = static_cast<int>(rounds * slots), pl.rest = static_cast<int>(tiles - pl.whole);
    pl.shares = 1, pl.share_steps = pl.steps;
    pl.us = rounds * round(slots, pl.steps);
    if (kind == Tiles16::kDeep && rounds > 0) pl.us = 1e30;
    if (pl.rest == 0) return pl;
    double best = round(pl.rest, pl.steps);
    for (int s = 2; s <= 64 && pl.rest * s <= slots && s * 4 <= pl.steps && static_cast<size_t>(pl.rest * s * tile_bytes) <= share_bytes; ++s) {
        const int per = ceil_div(pl.steps, s), n = ceil_div(pl.steps, per);
        if (n != s) continue;
        // the join: a launch, and the sums written and read once
        const double us = round(pl.rest * s, per) + 4.0 + 2.0 * pl.rest * s * tile_bytes / 4e6;
        if (us < best) best = us, pl.shares = s, pl.share_steps = per;
    }
    if (kind == Tiles16::kBig && logits) {
        // a quarter of a tile: two fifths of its time, as all its columns are fetched and read
        const double us = ceil_div(pl.rest * kParts16, slots) * (pl.steps * 0.65 + 4.0);
        if (us < best) best = us, pl.shares = kParts16;
    }
    pl.us += best;
    if (pl.shares == 1) pl.whole = static_cast<int>(tiles), pl.rest = 0;
    pl.part_bytes = pl.shares > 1 && !logits ? static_cast<size_t>(pl.rest) * pl.shares * tile_bytes : 0;
    return pl;
}

static Plan16 plan16_best(int M, int N, int K, int n_seg, size_t share_bytes, bool logits) {
    Plan16 best = plan16_of(Tiles16::kBig, M, N, K, n_seg, share_bytes, logits);
    for (const Tiles16 kind : {Tiles16::kSmall, Tiles16::kDeep}) {
        const Plan16 pl = plan16_of(kind, M, N, K, n_seg, share_bytes, logits);
        if (pl.us < best.us) best = pl;
    }
    return best;
}
Plan16 plan16(int M, int N, int K, int n_seg, size_t share_bytes) { return plan16_best(M, N, K, n_seg, share_bytes, false); }
Plan16 plan16_logits(int M, int N, int K, int n_seg) { return plan16_best(M, N, K, n_seg, 0, true); }

Plan16 plan32(int M, int N, int K, size_t share_bytes) {
    const Plan16 few = plan16_of(Tiles16::kFew, M, N, K, 1, share_bytes, false), all = plan16_of(Tiles16::kF32, M, N, K, 1, share_bytes, false);
    return few.us < all.us ? few : all;
}

int stats_words16(const Plan16& pl) {
    return pl.tiles == Tiles16::kF32   ? kF32N / kF32WN
           : pl.tiles == Tiles16::kFew ? kFewN / kFewWN
           : pl.tiles == Tiles16::kBig ? kBigN / kBigWN
                                       : kSmallN / kSmallWN;
}

template <int EPI, bool ARC, bool BRC>
static auto kernel16(Tiles16 kind, bool ends) {
    if constexpr (EPI != kEpiStore)
        if (ends && !wide16(kind))
            return kind == Tiles16::kBig    ? product16_ends_kernel<EPI, kBigM, kBigN, kBigWM, kBigWN>
                   : kind == Tiles16::kDeep ? product16_deep_ends_kernel<EPI, kSmallM, kSmallN, kSmallWM, kSmallWN>
                                            : product16_ends_kernel<EPI, kSmallM, kSmallN, kSmallWM, kSmallWN>;
    return kind == Tiles16::kF32    ? product32_kernel<EPI, kF32M, kF32N, kF32WM, kF32WN, ARC, BRC>
           : kind == Tiles16::kFew  ? product32_kernel<EPI, kFewM, kFewN, kFewWM, kFewWN, ARC, BRC>
           : kind == Tiles16::kBig  ? product16_kernel<EPI, kBigM, kBigN, kBigWM, kBigWN, ARC, BRC>
           : kind == Tiles16::kDeep ? product16_deep_kernel<EPI, kSmallM, kSmallN, kSmallWM, kSmallWN, ARC, BRC>
                                    : product16_kernel<EPI, kSmallM, kSmallN, kSmallWM, kSmallWN, ARC, BRC>;
}

int launch16(int epi, bool arc, bool brc, Product16 g, const Plan16& pl, size_t part_bytes, hipStream_t st) {
    const bool big = pl.tiles == Tiles16::kBig;
    const int tm = tile_m16(pl.tiles), tn = tile_n16(pl.tiles);
    g.tiles_m = ceil_div(g.M, tm), g.tiles_n = ceil_div(g.N, tn);
    if (static_cast<int64_t>(g.tiles_m) * g.tiles_n > INT32_MAX / 64) return DAB_ERR_UNSUPPORTED;
    g.steps = pl.steps, g.whole = pl.whole, g.rest = pl.rest, g.shares = pl.shares, g.share_steps = pl.share_steps;
    g.whole_xcd = ceil_div(g.whole, kNumXCD), g.rest_xcd = ceil_div(g.rest * g.shares, kNumXCD);
    // (the sums of shares go to g.part: never past the room that the caller has there)
    if (epi == kEpiStore && g.shares > 1 && static_cast<uint64_t>(g.rest) * g.shares * tm * tn * 4 > part_bytes) return DAB_ERR_UNSUPPORTED;
    const bool ends = g.tail || g.shares > 1;
    const auto kernel = epi == kEpiStats ? kernel16<kEpiStats, false, false>(pl.tiles, ends)
                        : epi == kEpiSoftmax ? kernel16<kEpiSoftmax, false, false>(pl.tiles, ends)
                        : arc ? kernel16<kEpiStore, true, true>(pl.tiles, false)
                              : kernel16<kEpiStore, false, true>(pl.tiles, false);
    if (brc != (epi == kEpiStore)) return DAB_ERR_UNSUPPORTED;
    const int threads = 64 * (big ? kBigWM * kBigWN : kSmallWM * kSmallWN);
    if (int rc = launch(kernel, dim3((g.whole_xcd + g.rest_xcd) * kNumXCD), dim3(threads), lds_bytes16(pl.tiles), st, g)) return rc;
    if (pl.shares == 1 || epi != kEpiStore) return DAB_OK;
    const int blocks = tm * tn / 256 / (threads / 64);   // 16 x 16 blocks of a wavefront
    const auto join = pl.tiles == Tiles16::kF32   ? join16_kernel<kF32M, kF32N, kF32WM, kF32WN>
                      : pl.tiles == Tiles16::kFew ? join16_kernel<kFewM, kFewN, kFewWM, kFewWN>
                      : big                       ? join16_kernel<kBigM, kBigN, kBigWM, kBigWN>
                                                  : join16_kernel<kSmallM, kSmallN, kSmallWM, kSmallWN>;
    return launch(join, dim3(g.rest * blocks), dim3(threads), 0, st, g);
}

int init_product16() {
    for (const Tiles16 kind : {Tiles16::kSmall, Tiles16::kDeep, Tiles16::kBig, Tiles16::kF32, Tiles16::kFew})
        for (const auto k : {kernel16<kEpiStats, false, false>(kind, false), kernel16<kEpiSoftmax, false, false>(kind, false),
                             kernel16<kEpiStats, false, false>(kind, true), kernel16<kEpiSoftmax, false, false>(kind, true),
                             kernel16<kEpiStore, true, true>(kind, false), kernel16<kEpiStore, false, true>(kind, false)}) {
            const hipError_t e = hipFuncSetAttribute(reinterpret_cast<const void*>(k), hipFuncAttributeMaxDynamicSharedMemorySize,
                                                     static_cast<int>(lds_bytes16(kind)));
            if (e != hipSuccess) return hip_failed(e);
        }
    return DAB_OK;
}

}  // namespace dab

// ---------------------------------------------------------------- the weight gradient from a saved input
namespace dab {

// Both operands of it in one launch: the saved input as bf16 [rows][32 groups], which is exact, by the first `x_blocks` workgroups; dY as P
// planes by the others (none where it is read as it is).  Bound by memory: 16384 x 4096 of the input in 32 us, 6.3 TB/s.
template <typename T, int P>
__global__ __launch_bounds__(256) void grad_operands_kernel(const int8_t* __restrict__ Q, const uint8_t* __restrict__ S, int64_t x_chunks,
                                                            bf16* __restrict__ X, unsigned x_blocks, const T* __restrict__ dY, int rows, int F,
                                                            int64_t ld, bf16* __restrict__ Y, int ldp) {
    if (blockIdx.x < x_blocks) {
        for (int64_t i = static_cast<int64_t>(blockIdx.x) * 256 + threadIdx.x; i < x_chunks; i += static_cast<int64_t>(x_blocks) * 256) {
            const uint64_t word = reinterpret_cast<const uint64_t*>(Q)[i];
            const int code = S[i >> 2];
            const float scale = code == 255 ? __builtin_nanf("") : pow2f(code - 127);
            v8bf o;
#pragma unroll
            for (int u = 0; u < 8; ++u) o[u] = static_cast<bf16>(static_cast<float>(static_cast<int8_t>(word >> (8 * u))) * scale);
            reinterpret_cast<v8bf*>(X)[i] = o;
        }
        return;
    }
    const int per_row = ldp >> 3;
    const int64_t chunks = static_cast<int64_t>(rows) * per_row, step = static_cast<int64_t>(gridDim.x - x_blocks) * 256;
    for (int64_t i = static_cast<int64_t>(blockIdx.x - x_blocks) * 256 + threadIdx.x; i < chunks; i += step) {
        const int64_t row = i / per_row;
        const int c = static_cast<int>(i - row * per_row) * 8;
        float v[8];
        load8(dY + row * ld, c, F, v);
#pragma unroll
        for (int p = 0; p < P; ++p) {
            v8bf o;
#pragma unroll
            for (int u = 0; u < 8; ++u) o[u] = piece_of(v[u], p);
            *reinterpret_cast<v8bf*>(Y + p * (static_cast<int64_t>(rows) * ldp) + row * ldp + c) = o;
        }
    }
}

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
    p.pl = plan16(F, cols, rows, P, kAnyShares16);
    p.x_at = 0;
    p.y_at = round_up(static_cast<int64_t>(rows) * p.ldx * 2, 256);
    p.part_at = p.y_at + (p.direct ? 0 : round_up(static_cast<int64_t>(P) * rows * p.ldy * 2, 256));
    p.bytes = p.part_at + p.pl.part_bytes;
    return p;
}
static bool grad_sizes(int32_t rows, int32_t cols, int32_t F, int32_t dtype, int64_t lddy) {
    return real_dtype(dtype) && rows <= INT32_MAX - (kStepK - 1) && lddy < (1 << 22) && F < (1 << 22) && cols < (1 << 22) &&
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
    const bf16* y = static_cast<const bf16*>(dY);
    bf16* out = reinterpret_cast<bf16*>(base + p.y_at);
    const int64_t x_chunks = rows * (p.ldx / 8), y_chunks = p.direct ? 0 : rows * (p.ldy / 8);
    auto blocks = [](int64_t chunks) { return static_cast<unsigned>(ceil_div64(chunks, 256) < 8192 ? ceil_div64(chunks, 256) : 8192); };
    const unsigned x_blocks = blocks(x_chunks);
    const dim3 grid(x_blocks + blocks(y_chunks)), block(256);
    const int ldy = static_cast<int>(p.ldy);
    int rc;
    if (dtype == DAB_F32) rc = launch(grad_operands_kernel<float, 3>, grid, block, 0, st, Q, S, x_chunks, x, x_blocks, static_cast<const float*>(dY), rows, F, lddy, out, ldy);
    else if (dtype == DAB_F16) rc = launch(grad_operands_kernel<f16, 2>, grid, block, 0, st, Q, S, x_chunks, x, x_blocks, static_cast<const f16*>(dY), rows, F, lddy, out, ldy);
    else rc = launch(grad_operands_kernel<bf16, 1>, grid, block, 0, st, Q, S, x_chunks, x, x_blocks, static_cast<const bf16*>(dY), rows, F, lddy, out, ldy);
    if (rc) return rc;
    if (!p.direct) y = out;
    Product16 g{};
    g.A = {y, p.ldy, static_cast<int64_t>(rows) * p.ldy};
    g.B = {x, p.ldx, 0};
    g.M = F, g.N = cols, g.K = rows;
    g.n_seg = dtype_pieces(dtype);
    g.seg_a = 0x210;                 // pieces of dY in turn, with the one plane of X
    g.C = dW, g.ldc = cols;
    g.part = reinterpret_cast<float*>(base + p.part_at);
    return launch16(kEpiStore, true, true, g, p.pl, p.bytes - p.part_at, st);
}
