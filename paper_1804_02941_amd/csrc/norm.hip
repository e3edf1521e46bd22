// The root-mean-square norm: forward with the residual's addition and a copy of the output in 8 bits, and its gradients.
//
//     h = x + r (rounded to the tensors' type),  y = gain h / sqrt(mean(h^2) + eps)
//     n = h rstd,  w = gain dy:   dx = rstd (w - n mean(w n)) + dh,   dgain = sum over rows of dy n
//
// One pass over memory each: 2^LOG lanes hold a row in registers, eight neighbouring values at a time, from the load to the store, so that
// the sum over the row costs no second read.  Bound by memory: 16384 x 4096 bf16 with residual and bytes 121 us, 5.0 TB/s, its gradients 102 + 5, 5.1
// (a copy of 2 GB reaches 4.92); counters: 269 MB read and 338 written, what the formulas need.  A lane loads its vectors one after the other and waits for
// each (row8 branches on short rows, and H, which may be X, is stored between): rows that fill the chip hide that, a few MB do not (346 x 6128 fp32 8.9 us,
// 17 MB; gradients of 1999 x 1003 fp32 9.5 and 2.9, 24 MB).
#include "lanes.h"
#include "real16.h"

namespace dab {

constexpr int kNormThreads = 256;    // of a workgroup, unless a row takes more

struct NormGeom {
    int rows, cols, groups;          // groups of 32 of a row
    int64_t ldx, ldr;                // of x and r, or of dy and h
    int64_t ldd;                     // of dh
    float eps;
};

// Eight values of a row from column c on.  Where fewer are left they are the row's last eight, the first again_of() of which another lane has: loads
// without a branch for each value (one by one, every row of 8192 x 4095 waited for them: its gradients 93 us and 12 for joining, now 59 and 5; 8192 x 4096 54 and
// 5).  Shorter rows: zeros behind them.
__device__ __forceinline__ int place_of(int c, int cols) { return cols < 8 ? c : min(c, cols - 8); }
__device__ __forceinline__ int again_of(int c, int cols) { return c - place_of(c, cols); }
template <typename T>
__device__ __forceinline__ void row8(const T* row, int c, int cols, float (&v)[8]) {
    if (cols < 8) {
        load8(row, c, cols, v);
    } else {
        const auto eight = *reinterpret_cast<const typename Unaligned<T, 8>::type*>(row + place_of(c, cols));
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = static_cast<float>(eight[i]);
    }
}
// Zeros in place of another lane's.
__device__ __forceinline__ void drop(int again, float (&v)[8]) {
    if (again > 0)
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = i < again ? 0.f : v[i];
}
template <typename T>
__device__ __forceinline__ void put8(T* row, int c, int cols, const float (&v)[8]) {
    const int again = again_of(c, cols);
    if (again == 0) {
        store8(row, c, cols, v);
    } else {
#pragma unroll
        for (int i = 1; i < 8; ++i)
            if (i >= again) row[c - again + i] = static_cast<T>(v[i]);
    }
}

// The sum over the 2^LOG lanes of a row; buffer: one of two, so that a barrier stands between a value's last reader and its next writer.
template <int LOG>
__device__ __forceinline__ float row_sum(float v, float (&part)[2][16], int buffer) {
    v = lanes_sum<(LOG < 6 ? LOG : 6)>(v);
    if constexpr (LOG > 6) {
        constexpr int kWaves = 1 << (LOG - 6);
        const int wave = threadIdx.x >> 6;
        if ((threadIdx.x & 63) == 0) part[buffer][wave] = v;
        __syncthreads();
        const int first = wave & ~(kWaves - 1);
        v = 0.f;
#pragma unroll
        for (int i = 0; i < kWaves; ++i) v += part[buffer][first + i];
    }
    return v;
}

// Eight values of y as bytes with their group's scale, as dab_ckpt8_save() writes them.
__device__ __forceinline__ void save_eight(const float (&y)[8], int64_t row_groups, int c, int8_t* __restrict__ Q, uint8_t* __restrict__ S) {
    const uint32_t m = group_max(y);
    uint64_t word = 0;
    int code = 255;
    if (m < 0x7f800000u) {
        const int e = group_exponent<6>(m);
        const float inv = pow2f(-e);
        code = e + 127;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const int q = static_cast<int>(fminf(fmaxf(rintf(y[i] * inv), -127.f), 127.f));
            word |= static_cast<uint64_t>(static_cast<uint8_t>(q)) << (8 * i);
        }
    }
    *reinterpret_cast<uint64_t*>(Q + row_groups * 32 + c) = word;
    if ((c & 31) == 0) S[row_groups + (c >> 5)] = static_cast<uint8_t>(code);
}

// Rows of at most 8 NV 2^LOG values.  Lane i of a row holds the eights i, i + 2^LOG, ..  Four eights a lane where rows fill the chip; fewer of them are
// spread over as many lanes as a row has eights (one row of 4096: 2.4 us, with four eights a lane 4.4).
template <typename T, int LOG, int NV>
__global__ __launch_bounds__(LOG > 8 ? 1 << LOG : kNormThreads) void norm_kernel(const T* X, const T* R, const float* __restrict__ gain, NormGeom g,
                                                                                T* H, T* Y, int8_t* Q, uint8_t* S, float* rstd) {
    __shared__ float part[2][16];
    DAB_RESERVE_VGPRS();
    constexpr int kLanes = 1 << LOG, kRows = LOG > 8 ? 1 : kNormThreads >> LOG;
    const int lane = threadIdx.x & (kLanes - 1);
    const int64_t row = static_cast<int64_t>(blockIdx.x) * kRows + (threadIdx.x >> LOG);
    const bool live = row < g.rows;
    float h[NV][8];
    float sum = 0.f;
#pragma unroll
    for (int j = 0; j < NV; ++j) {
        const int c = (j * kLanes + lane) * 8;
#pragma unroll
        for (int i = 0; i < 8; ++i) h[j][i] = 0.f;
        if (live && c < g.cols) {
            row8(X + row * g.ldx, c, g.cols, h[j]);
            if (R) {
                float r[8];
                row8(R + row * g.ldr, c, g.cols, r);
#pragma unroll
                for (int i = 0; i < 8; ++i) h[j][i] = static_cast<float>(static_cast<T>(h[j][i] + r[i]));
                put8(H + row * g.cols, c, g.cols, h[j]);
            }
            drop(again_of(c, g.cols), h[j]);
        }
#pragma unroll
        for (int i = 0; i < 8; ++i) sum += h[j][i] * h[j][i];
    }
    sum = row_sum<LOG>(sum, part, 0);
    const float scale = 1.f / sqrtf(sum / static_cast<float>(g.cols) + g.eps);
    if (!live) return;
    if (lane == 0) rstd[row] = scale;
#pragma unroll
    for (int j = 0; j < NV; ++j) {
        const int c = (j * kLanes + lane) * 8;
        float y[8] = {};
        if (c < g.cols) {
            row8(gain, c, g.cols, y);
#pragma unroll
            for (int i = 0; i < 8; ++i) y[i] = (h[j][i] * scale) * y[i];
            if (Y) put8(Y + row * g.cols, c, g.cols, y);
        }
        // (the four lanes of a group are all here, those past the row's end with zeros)
        if (Q && c < g.groups * 32) {
            if (c < g.cols) own_first(again_of(c, g.cols), y);
            save_eight(y, row * g.groups, c, Q, S);
        }
    }
}

// Rows that no workgroup holds: read twice, the second time what the first has written where there is a residual.
template <typename T>
__global__ __launch_bounds__(1024) void norm_long_kernel(const T* X, const T* R, const float* __restrict__ gain, NormGeom g, T* H, T* Y, int8_t* Q,
                                                         uint8_t* S, float* rstd) {
    __shared__ float part[2][16];
    const int64_t row = blockIdx.x;
    const T* x = X + row * g.ldx;
    T* hout = H + row * g.cols;                              // (not used without a residual)
    float sum = 0.f;
    for (int64_t c0 = threadIdx.x * 8; c0 < g.cols; c0 += 8192) {
        const int c = static_cast<int>(c0);
        float h[8];
        row8(x, c, g.cols, h);
        if (R) {
            float r[8];
            row8(R + row * g.ldr, c, g.cols, r);
#pragma unroll
            for (int i = 0; i < 8; ++i) h[i] = static_cast<float>(static_cast<T>(h[i] + r[i]));
            put8(hout, c, g.cols, h);
        }
        drop(again_of(c, g.cols), h);
#pragma unroll
        for (int i = 0; i < 8; ++i) sum += h[i] * h[i];
    }
    sum = row_sum<10>(sum, part, 0);
    const float scale = 1.f / sqrtf(sum / static_cast<float>(g.cols) + g.eps);
    if (threadIdx.x == 0) rstd[row] = scale;
    for (int64_t c0 = threadIdx.x * 8; c0 < static_cast<int64_t>(g.groups) * 32; c0 += 8192) {
        const int c = static_cast<int>(c0);
        float h[8] = {}, y[8] = {};
        if (c < g.cols) {
            row8(R ? static_cast<const T*>(hout) : x, c, g.cols, h);
            row8(gain, c, g.cols, y);
#pragma unroll
            for (int i = 0; i < 8; ++i) y[i] = (h[i] * scale) * y[i];
            if (Y) put8(Y + row * g.cols, c, g.cols, y);
            own_first(again_of(c, g.cols), y);
        }
        if (Q) save_eight(y, row * g.groups, c, Q, S);
    }
}

// ---------------------------------------------------------------- gradients
// Columns of a part of dgain, with up to three behind the row's, so that every part is read in fours.
__host__ __device__ __forceinline__ int64_t part_ld(int cols) { return (static_cast<int64_t>(cols) + 3) & ~int64_t{3}; }

// A workgroup takes rows blockIdx.x, + gridDim.x, .. (times the rows that it holds at once) and keeps its part of dgain in registers meanwhile, that of
// its rows' lanes together in LDS at the end; norm_join_kernel adds the workgroups' parts in a fixed order.  (Every row's lanes with a part of their
// own: 1999 x 1003 fp32 11.8 us and 37 for joining 2000 parts, now 9.5 and 2.9.)  Two eights a lane: gain and the part of dgain stay in registers too.
template <typename T, int LOG, int NV>
__global__ __launch_bounds__(LOG > 8 ? 1 << LOG : kNormThreads) void norm_grad_kernel(const T* dY, const T* H, const float* __restrict__ gain,
                                                                                     const float* __restrict__ rstd, const T* dH, NormGeom g, T* dX,
                                                                                     float* __restrict__ parts) {
    __shared__ float part[2][16];
    DAB_RESERVE_VGPRS();
    constexpr int kLanes = 1 << LOG, kRows = LOG > 8 ? 1 : kNormThreads >> LOG;
    const int lane = threadIdx.x & (kLanes - 1), slot = threadIdx.x >> LOG;
    float dg[NV][8], gn[NV][8];
#pragma unroll
    for (int j = 0; j < NV; ++j) {
        const int c = (j * kLanes + lane) * 8;
#pragma unroll
        for (int i = 0; i < 8; ++i) dg[j][i] = 0.f, gn[j][i] = 0.f;
        if (c < g.cols) row8(gain, c, g.cols, gn[j]), drop(again_of(c, g.cols), gn[j]);
    }
    int buffer = 0;
    for (int64_t row0 = static_cast<int64_t>(blockIdx.x) * kRows; row0 < g.rows; row0 += static_cast<int64_t>(gridDim.x) * kRows, buffer ^= 1) {
        const int64_t row = row0 + slot;
        const bool live = row < g.rows;
        const float s = live ? rstd[row] : 0.f;
        float n[NV][8], w[NV][8];
        float dot = 0.f;
#pragma unroll
        for (int j = 0; j < NV; ++j) {
            const int c = (j * kLanes + lane) * 8;
#pragma unroll
            for (int i = 0; i < 8; ++i) n[j][i] = 0.f, w[j][i] = 0.f;
            if (live && c < g.cols) {
                row8(dY + row * g.ldx, c, g.cols, w[j]);
                row8(H + row * g.ldr, c, g.cols, n[j]);
                drop(again_of(c, g.cols), w[j]);
            }
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                n[j][i] *= s;
                dg[j][i] += w[j][i] * n[j][i];
                w[j][i] *= gn[j][i];
                dot += w[j][i] * n[j][i];
            }
        }
        dot = row_sum<LOG>(dot, part, buffer) / static_cast<float>(g.cols);
        if (!live) continue;
#pragma unroll
        for (int j = 0; j < NV; ++j) {
            const int c = (j * kLanes + lane) * 8;
            if (c >= g.cols) continue;
            float d[8] = {};
            if (dH) row8(dH + row * g.ldd, c, g.cols, d);
#pragma unroll
            for (int i = 0; i < 8; ++i) d[i] += (w[j][i] - n[j][i] * dot) * s;
            put8(dX + row * g.cols, c, g.cols, d);
        }
    }
    float* to = parts + static_cast<int64_t>(blockIdx.x) * part_ld(g.cols);
    if constexpr (kRows == 1) {
#pragma unroll
        for (int j = 0; j < NV; ++j) {
            const int c = (j * kLanes + lane) * 8;
            if (c < g.cols) put8(to, c, g.cols, dg[j]);
        }
    } else {
        constexpr int kCols = kLanes * NV * 8;
        __shared__ float all[kRows][kCols];
#pragma unroll
        for (int j = 0; j < NV; ++j) {
            const int c = (j * kLanes + lane) * 8;
            if (c < g.cols) put8(all[slot], c, g.cols, dg[j]);
        }
        __syncthreads();
        for (int c = threadIdx.x; c < g.cols; c += kNormThreads) {
            float v = 0.f;
#pragma unroll
            for (int i = 0; i < kRows; ++i) v += all[i][c];
            to[c] = v;
        }
    }
}

// Few rows: a workgroup takes rows, for dX, or 32 columns, for dgain, which needs no sum over a row: one launch, nothing to join, and dY and H read twice.
// first: the number of the launch's first workgroup (dX over dY or H: one launch for the columns, another one behind it for the rows).
template <typename T, int LOG, int NV>
__global__ __launch_bounds__(LOG > 8 ? 1 << LOG : kNormThreads) void norm_grad_few_kernel(const T* dY, const T* H, const float* __restrict__ gain,
                                                                                         const float* __restrict__ rstd, const T* dH, NormGeom g, T* dX,
                                                                                         float* __restrict__ dgain, int row_blocks, int first) {
    constexpr int kLanes = 1 << LOG, kRows = LOG > 8 ? 1 : kNormThreads >> LOG, kThreads = kLanes * kRows;
    __shared__ float part[2][16];
    __shared__ float sums[kThreads / 4][33];
    DAB_RESERVE_VGPRS();
    const int block = blockIdx.x + first;
    if (block >= row_blocks) {
        // four lanes for a row's 32 columns
        const int c0 = (block - row_blocks) * 32, c = c0 + (threadIdx.x & 3) * 8, slice = threadIdx.x >> 2;
        float v[8] = {};
        if (c < g.cols) {
#pragma unroll 4
            for (int64_t row = slice; row < g.rows; row += kThreads / 4) {
                float w[8], n[8];
                const float s = rstd[row];
                row8(dY + row * g.ldx, c, g.cols, w), row8(H + row * g.ldr, c, g.cols, n);
#pragma unroll
                for (int i = 0; i < 8; ++i) v[i] += w[i] * (n[i] * s);
            }
            own_first(again_of(c, g.cols), v);
        }
#pragma unroll
        for (int i = 0; i < 8; ++i) sums[slice][(threadIdx.x & 3) * 8 + i] = v[i];
        __syncthreads();
        // eight slices by each half wavefront, then those sums
        const int col = threadIdx.x & 31, share = threadIdx.x >> 5;
        float w = 0.f;
#pragma unroll
        for (int i = 0; i < 8; ++i) w += sums[share * 8 + i][col];
        __syncthreads();
        sums[share][col] = w;
        __syncthreads();
        if (share != 0 || c0 + col >= g.cols) return;
        w = 0.f;
#pragma unroll
        for (int i = 0; i < kThreads / 32; ++i) w += sums[i][col];
        dgain[c0 + col] = w;
        return;
    }
    const int lane = threadIdx.x & (kLanes - 1);
    const int64_t row = static_cast<int64_t>(block) * kRows + (threadIdx.x >> LOG);
    const bool live = row < g.rows;
    const float s = live ? rstd[row] : 0.f;
    float n[NV][8], w[NV][8], d[NV][8];
    float dot = 0.f;
#pragma unroll
    for (int j = 0; j < NV; ++j) {
        const int c = (j * kLanes + lane) * 8;
        float gn[8] = {};
#pragma unroll
        for (int i = 0; i < 8; ++i) n[j][i] = 0.f, w[j][i] = 0.f, d[j][i] = 0.f;
        if (live && c < g.cols) {
            row8(gain, c, g.cols, gn);
            row8(dY + row * g.ldx, c, g.cols, w[j]);
            row8(H + row * g.ldr, c, g.cols, n[j]);
            if (dH) row8(dH + row * g.ldd, c, g.cols, d[j]);
            drop(again_of(c, g.cols), w[j]), drop(again_of(c, g.cols), gn);
        }
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            n[j][i] *= s;
            w[j][i] *= gn[i];
            dot += w[j][i] * n[j][i];
        }
    }
    dot = row_sum<LOG>(dot, part, 0) / static_cast<float>(g.cols);
    if (!live) return;
#pragma unroll
    for (int j = 0; j < NV; ++j) {
        const int c = (j * kLanes + lane) * 8;
        if (c >= g.cols) continue;
#pragma unroll
        for (int i = 0; i < 8; ++i) d[j][i] += (w[j][i] - n[j][i] * dot) * s;
        put8(dX + row * g.cols, c, g.cols, d[j]);
    }
}

// Rows that no workgroup holds: the workgroup's part of dgain lies in its row of `parts` meanwhile.
template <typename T>
__global__ __launch_bounds__(1024) void norm_grad_long_kernel(const T* dY, const T* H, const float* __restrict__ gain, const float* __restrict__ rstd,
                                                              const T* dH, NormGeom g, T* dX, float* parts) {
    __shared__ float part[2][16];
    DAB_RESERVE_VGPRS();
    float* to = parts + static_cast<int64_t>(blockIdx.x) * part_ld(g.cols);
    int buffer = 0;
    for (int64_t row = blockIdx.x; row < g.rows; row += gridDim.x, buffer ^= 1) {
        const float s = rstd[row];
        float dot = 0.f;
        for (int64_t c0 = threadIdx.x * 8; c0 < g.cols; c0 += 8192) {
            const int c = static_cast<int>(c0);
            float w[8], n[8], gn[8], dg[8] = {};
            row8(dY + row * g.ldx, c, g.cols, w), row8(H + row * g.ldr, c, g.cols, n), row8(gain, c, g.cols, gn);
            if (row != blockIdx.x) row8(static_cast<const float*>(to), c, g.cols, dg);
            drop(again_of(c, g.cols), w), drop(again_of(c, g.cols), gn);
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                n[i] *= s;
                dg[i] += w[i] * n[i];
                dot += (w[i] * gn[i]) * n[i];
            }
            put8(to, c, g.cols, dg);
        }
        dot = row_sum<10>(dot, part, buffer) / static_cast<float>(g.cols);
        for (int64_t c0 = threadIdx.x * 8; c0 < g.cols; c0 += 8192) {
            const int c = static_cast<int>(c0);
            float w[8], n[8], gn[8], d[8] = {};
            row8(dY + row * g.ldx, c, g.cols, w), row8(H + row * g.ldr, c, g.cols, n), row8(gain, c, g.cols, gn);
            if (dH) row8(dH + row * g.ldd, c, g.cols, d);
#pragma unroll
            for (int i = 0; i < 8; ++i) d[i] += (w[i] * gn[i] - (n[i] * s) * dot) * s;
            put8(dX + row * g.cols, c, g.cols, d);
        }
    }
}

// dgain[c] = sum over the parts: 32 columns a workgroup, 128 threads that share the parts of four columns, so that a thread's few loads are in flight
// together (1024 parts of 4096: 5.1 us).
__global__ __launch_bounds__(1024) void norm_join_kernel(const float* __restrict__ parts, int n, int cols, float* __restrict__ dgain) {
    __shared__ float sums[128][33];
    DAB_RESERVE_VGPRS();
    const int slice = threadIdx.x >> 3, c = blockIdx.x * 32 + (threadIdx.x & 7) * 4;
    float v[4] = {0.f, 0.f, 0.f, 0.f};
    if (c < cols) {
        const float* from = parts + c;
        const int64_t ld = part_ld(cols);
#pragma unroll 8
        for (int i = slice; i < n; i += 128) {
            const v4f got = *reinterpret_cast<const v4f*>(from + i * ld);
#pragma unroll
            for (int k = 0; k < 4; ++k) v[k] += got[k];
        }
    }
#pragma unroll
    for (int k = 0; k < 4; ++k) sums[slice][(threadIdx.x & 7) * 4 + k] = v[k];
    __syncthreads();
    // eight slices by each wavefront half, then the sixteen that are left
    const int col = threadIdx.x & 31, part = threadIdx.x >> 5;
    float w = 0.f;
    if (part < 16)
#pragma unroll
        for (int i = 0; i < 8; ++i) w += sums[part * 8 + i][col];
    __syncthreads();
    if (part < 16) sums[part][col] = w;
    __syncthreads();
    if (part != 0 || blockIdx.x * 32 + col >= cols) return;
    w = 0.f;
#pragma unroll
    for (int i = 0; i < 16; ++i) w += sums[i][col];
    dgain[blockIdx.x * 32 + col] = w;
}

// ---------------------------------------------------------------- host side
// Lanes of a row (their logarithm) and eights of a lane; log 0: the kernels for long rows.
struct NormForm {
    int log, nv;
};
static NormForm norm_form(int cols, int max_nv) {
    const int eights = ceil_div(cols, 8);
    NormForm f{2, 1};
    while (f.log < 6 && (1 << f.log) < eights) ++f.log;
    while (f.nv < max_nv && (f.nv << f.log) < eights) f.nv *= 2;
    while (f.log < 10 && (f.nv << f.log) < eights) ++f.log;
    if ((static_cast<int64_t>(f.nv) << f.log) < eights) f.log = 0;
    return f;
}
static int norm_rows(NormForm f) { return f.log == 0 || f.log > 8 ? 1 : kNormThreads >> f.log; }
static int norm_threads(NormForm f) { return f.log == 0 ? 1024 : f.log > 8 ? 1 << f.log : kNormThreads; }
constexpr int kNormNV = 4, kNormGradNV = 2;
constexpr int64_t kNormFew = 256 * 4096;

template <typename T>
struct NormArgs {
    const T *X, *R;
    const float* gain;
    NormGeom g;
    T *H, *Y;
    int8_t* Q;
    uint8_t* S;
    float* rstd;
};
template <typename T, int LOG, int NV>
static int norm_launch(const NormArgs<T>& a, NormForm f, hipStream_t st) {
    const dim3 grid(static_cast<unsigned>(ceil_div64(a.g.rows, norm_rows(f)))), block(norm_threads(f));
    return launch(norm_kernel<T, LOG, NV>, grid, block, 0, st, a.X, a.R, a.gain, a.g, a.H, a.Y, a.Q, a.S, a.rstd);
}
template <typename T>
static int norm_launch(const NormArgs<T>& a, hipStream_t st) {
    // (rows that do not fill the chip: as many lanes as a row has eights)
    const bool few = static_cast<int64_t>(a.g.rows) * a.g.cols <= kNormFew;
    const NormForm f = few ? norm_form(a.g.cols, a.g.cols <= 8192 ? 1 : kNormNV) : norm_form(a.g.cols, kNormNV);
    switch (f.log) {
        case 0: return launch(norm_long_kernel<T>, dim3(a.g.rows), dim3(1024), 0, st, a.X, a.R, a.gain, a.g, a.H, a.Y, a.Q, a.S, a.rstd);
        case 2: return norm_launch<T, 2, 1>(a, f, st);
        case 3: return norm_launch<T, 3, 1>(a, f, st);
        case 4: return norm_launch<T, 4, 1>(a, f, st);
        case 5: return norm_launch<T, 5, 1>(a, f, st);
        case 6: return f.nv == 1 ? norm_launch<T, 6, 1>(a, f, st) : f.nv == 2 ? norm_launch<T, 6, 2>(a, f, st) : norm_launch<T, 6, 4>(a, f, st);
        case 7: return f.nv == 1 ? norm_launch<T, 7, 1>(a, f, st) : norm_launch<T, 7, 4>(a, f, st);
        case 8: return f.nv == 1 ? norm_launch<T, 8, 1>(a, f, st) : norm_launch<T, 8, 4>(a, f, st);
        case 9: return f.nv == 1 ? norm_launch<T, 9, 1>(a, f, st) : norm_launch<T, 9, 4>(a, f, st);
        default: return f.nv == 1 ? norm_launch<T, 10, 1>(a, f, st) : norm_launch<T, 10, 4>(a, f, st);
    }
}

template <typename T>
struct NormGradArgs {
    const T *dY, *H;
    const float *gain, *rstd;
    const T* dH;
    NormGeom g;
    T* dX;
    float *dgain, *parts;
    int blocks;
};
template <typename T, int LOG, int NV>
static int norm_grad_launch(const NormGradArgs<T>& a, NormForm f, hipStream_t st) {
    return launch(norm_grad_kernel<T, LOG, NV>, dim3(a.blocks), dim3(norm_threads(f)), 0, st, a.dY, a.H, a.gain, a.rstd, a.dH, a.g, a.dX, a.parts);
}
// Workgroups of the gradient's kernel: what the chip holds at once, fewer where there are fewer rows: half as many as these would fill, once that leaves
// one for every other compute unit, so that half the parts are joined (both kernels, us: 1999 x 1003 fp32 15.0 and 13.9, 512 x 4096 bf16 12.9 and
// 12.4, 1000 x 2000 11.4 and 11.8; below, 100 x 16384 12.6 and 13.4; a quarter as many is slower throughout).
static int norm_grad_blocks(int rows, NormForm f) {
    const int64_t n = ceil_div64(rows, norm_rows(f)), most = 1024 / norm_threads(f) * int64_t{kNumCU};
    if (n <= 2) return 1;
    if (n >= most) return static_cast<int>(most);
    return static_cast<int>(n <= kNumCU ? n : (n + 1) / 2);
}
// Up to this many rows, and elements: the columns' workgroups are few and read every row.  us, one launch and two: 5 x 2000 fp32 6.1 and 9.0, 512 x 2000
// bf16 8.5 and 9.6, 512 x 4096 8.7 and 12.6, 128 x 16384 8.8 and 14.6; past them, 1024 x 2000 16.3 and 12.5, 512 x 16384 25.9 and 20.4.
static bool norm_grad_few(int rows, int cols) { return rows <= 512 && cols <= 16384 && rows * cols <= 1 << 21; }
template <typename T, int LOG, int NV>
static int norm_grad_few_launch(const NormGradArgs<T>& a, hipStream_t st) {
    const NormForm f{LOG, NV};
    const int rows = static_cast<int>(ceil_div64(a.g.rows, norm_rows(f))), columns = ceil_div(a.g.cols, 32);
    const auto go = [&](int first, int blocks) {
        return launch(norm_grad_few_kernel<T, LOG, NV>, dim3(blocks), dim3(norm_threads(f)), 0, st, a.dY, a.H, a.gain, a.rstd, a.dH, a.g, a.dX, a.dgain, rows,
                      first);
    };
    if (a.dX != a.dY && a.dX != a.H) return go(0, rows + columns);
    const int rc = go(rows, columns);
    return rc ? rc : go(0, rows);
}
template <typename T>
static int norm_grad_few_launch(const NormGradArgs<T>& a, hipStream_t st) {
    const NormForm f = norm_form(a.g.cols, a.g.cols <= 8192 ? 1 : 2);
    switch (f.log) {
        case 2: return norm_grad_few_launch<T, 2, 1>(a, st);
        case 3: return norm_grad_few_launch<T, 3, 1>(a, st);
        case 4: return norm_grad_few_launch<T, 4, 1>(a, st);
        case 5: return norm_grad_few_launch<T, 5, 1>(a, st);
        case 6: return norm_grad_few_launch<T, 6, 1>(a, st);
        case 7: return norm_grad_few_launch<T, 7, 1>(a, st);
        case 8: return norm_grad_few_launch<T, 8, 1>(a, st);
        case 9: return norm_grad_few_launch<T, 9, 1>(a, st);
        default: return f.nv == 1 ? norm_grad_few_launch<T, 10, 1>(a, st) : norm_grad_few_launch<T, 10, 2>(a, st);
    }
}
template <typename T>
static int norm_grad_launch(NormGradArgs<T> a, hipStream_t st) {
    if (norm_grad_few(a.g.rows, a.g.cols)) return norm_grad_few_launch(a, st);
    const NormForm f = norm_form(a.g.cols, kNormGradNV);
    int rc;
    // (the part of a workgroup that has all rows is the gradient)
    if (a.blocks == 1) a.parts = a.dgain;
    switch (f.log) {
        case 0: rc = launch(norm_grad_long_kernel<T>, dim3(a.blocks), dim3(1024), 0, st, a.dY, a.H, a.gain, a.rstd, a.dH, a.g, a.dX, a.parts); break;
        case 2: rc = norm_grad_launch<T, 2, 1>(a, f, st); break;
        case 3: rc = norm_grad_launch<T, 3, 1>(a, f, st); break;
        case 4: rc = norm_grad_launch<T, 4, 1>(a, f, st); break;
        case 5: rc = norm_grad_launch<T, 5, 1>(a, f, st); break;
        case 6: rc = f.nv == 1 ? norm_grad_launch<T, 6, 1>(a, f, st) : norm_grad_launch<T, 6, 2>(a, f, st); break;
        case 7: rc = norm_grad_launch<T, 7, 2>(a, f, st); break;
        case 8: rc = norm_grad_launch<T, 8, 2>(a, f, st); break;
        case 9: rc = norm_grad_launch<T, 9, 2>(a, f, st); break;
        default: rc = norm_grad_launch<T, 10, 2>(a, f, st);
    }
    if (rc || a.blocks == 1) return rc;
    return launch(norm_join_kernel, dim3(ceil_div(a.g.cols, 32)), dim3(1024), 0, st, static_cast<const float*>(a.parts), a.blocks, a.g.cols, a.dgain);
}

constexpr int kNormMaxCols = 1 << 26;
// An output over an input: only element by element, which the same lane reads before it writes.
static bool crosses(const void* out, const void* in, int rows, int cols, int64_t ld, int64_t size) {
    return out && in && !(out == in && (ld == cols || rows == 1)) && meet({out, rows, cols, cols, size}, {in, rows, cols, ld, size});
}

}  // namespace dab

extern "C" int dab_rms_norm(const void* X, int32_t dtype, int64_t ldx, const void* R, int64_t ldr, const float* gain, float eps, int32_t rows,
                            int32_t cols, void* H, void* Y, int8_t* Q, uint8_t* S, float* rstd, void* stream) {
    using namespace dab;
    if (!X || !gain || !rstd || (R && !H) || (!Y && !Q) || (Q == nullptr) != (S == nullptr)) return DAB_ERR_NULL;
    if (rows < 1 || cols < 1 || ldx < cols || (R && ldr < cols) || !(eps >= 0.f)) return DAB_ERR_SHAPE;
    if (!real_dtype(dtype) || cols > kNormMaxCols) return DAB_ERR_UNSUPPORTED;
    if (misaligned(X, 16) || misaligned(R, 16) || misaligned(H, 16) || misaligned(Y, 16) || misaligned(Q, 16) || misaligned(gain, 4) ||
        misaligned(rstd, 4))
        return DAB_ERR_ALIGN;
    const int64_t size = dtype_bytes(dtype);
    if (R && (crosses(H, X, rows, cols, ldx, size) || crosses(H, R, rows, cols, ldr, size))) return DAB_ERR_UNSUPPORTED;
    if (crosses(Y, X, rows, cols, ldx, size) || crosses(Y, R, rows, cols, ldr, size)) return DAB_ERR_UNSUPPORTED;
    // (h is kept for the gradient)
    if (R && Y && meet({H, rows, cols, cols, size}, {Y, rows, cols, cols, size})) return DAB_ERR_UNSUPPORTED;
    NormGeom g{};
    g.rows = rows, g.cols = cols, g.groups = ceil_div(cols, 32), g.ldx = ldx, g.ldr = ldr, g.eps = eps;
    const auto st = static_cast<hipStream_t>(stream);
    const auto go = [&](auto* t) {
        typedef std::remove_pointer_t<decltype(t)> T;
        const NormArgs<T> a{static_cast<const T*>(X), static_cast<const T*>(R), gain, g, static_cast<T*>(H), static_cast<T*>(Y), Q, S, rstd};
        return norm_launch(a, st);
    };
    if (dtype == DAB_F32) return go(static_cast<float*>(nullptr));
    if (dtype == DAB_BF16) return go(static_cast<bf16*>(nullptr));
    return go(static_cast<f16*>(nullptr));
}

extern "C" size_t dab_rms_norm_gradient_workspace_bytes(int32_t rows, int32_t cols) {
    using namespace dab;
    if (rows < 1 || cols < 1 || cols > kNormMaxCols || norm_grad_few(rows, cols)) return 0;
    const NormForm f = norm_form(cols, kNormGradNV);
    const int blocks = norm_grad_blocks(rows, f);
    return blocks == 1 ? 0 : static_cast<size_t>(blocks) * part_ld(cols) * 4;
}

extern "C" int dab_rms_norm_gradient(const void* dY, int64_t lddy, const void* H, int64_t ldh, int32_t dtype, const float* gain, const float* rstd,
                                     const void* dH, int64_t lddh, int32_t rows, int32_t cols, void* dX, float* dgain, void* ws, size_t ws_bytes,
                                     void* stream) {
    using namespace dab;
    if (!dY || !H || !gain || !rstd || !dX || !dgain) return DAB_ERR_NULL;
    if (rows < 1 || cols < 1 || lddy < cols || ldh < cols || (dH && lddh < cols)) return DAB_ERR_SHAPE;
    if (!real_dtype(dtype) || cols > kNormMaxCols) return DAB_ERR_UNSUPPORTED;
    if (misaligned(dY, 16) || misaligned(H, 16) || misaligned(dH, 16) || misaligned(dX, 16) || misaligned(gain, 4) || misaligned(rstd, 4) ||
        misaligned(dgain, 4))
        return DAB_ERR_ALIGN;
    const int64_t size = dtype_bytes(dtype);
    if (crosses(dX, dY, rows, cols, lddy, size) || crosses(dX, H, rows, cols, ldh, size) || crosses(dX, dH, rows, cols, lddh, size)) return DAB_ERR_UNSUPPORTED;
    const size_t need = dab_rms_norm_gradient_workspace_bytes(rows, cols);
    if (need && (!ws || ws_bytes < need || misaligned(ws, 256))) return DAB_ERR_WORKSPACE;
    NormGeom g{};
    g.rows = rows, g.cols = cols, g.groups = ceil_div(cols, 32), g.ldx = lddy, g.ldr = ldh, g.ldd = lddh;
    const int blocks = norm_grad_blocks(rows, norm_form(cols, kNormGradNV));
    const auto st = static_cast<hipStream_t>(stream);
    const auto go = [&](auto* t) {
        typedef std::remove_pointer_t<decltype(t)> T;
        const NormGradArgs<T> a{static_cast<const T*>(dY), static_cast<const T*>(H), gain, rstd, static_cast<const T*>(dH), g,
                                static_cast<T*>(dX), dgain, static_cast<float*>(ws), blocks};
        return norm_grad_launch(a, st);
    };
    if (dtype == DAB_F32) return go(static_cast<float*>(nullptr));
    if (dtype == DAB_BF16) return go(static_cast<bf16*>(nullptr));
    return go(static_cast<f16*>(nullptr));
}
