// A step of Adam with decoupled weight decay over many tensors at once, its two states in 32 bits or in 8 (formats: include/dab.h).
//
//     m = b1 m + (1 - b1) g,  v = b2 v + (1 - b2) g^2,  p = p (1 - lr wd) - lr / (1 - b1^t) m / (sqrt(v / (1 - b2^t)) + eps)
//
// One pass over memory: a lane holds eight neighbouring elements of everything, four lanes a group of 32 that shares a scale.  One launch
// for all tensors: a table in device memory, written once by kernels that get the addresses with their launch (nothing is copied to the device, so
// that it may be made in a captured graph too), says which stretch of which tensor a workgroup takes.  Bound by memory: 28 bytes an element with
// fp32 gradients and states (8.5 M of them 50 us, 4.8 TB/s), 16.1 with bf16 gradients, 8-bit states and a bf16 copy (75.5 M 237 to 263 us, 4.6 to 5.1).
// 96 tensors of a few thousand elements: 5.8 us, with the tensors among the arguments, 32 a launch, 21.6.  What is left are reads that wait for one
// another behind the launch: the tensor's number, the tensor, scale, rate and step where they are in device memory, the gradient, the weights, the states (their
// addresses come out of the table, so that the compiler takes them for generic ones, and each stands under a branch).
#include <cmath>

#include "real16.h"

namespace dab {

constexpr int kAdamThreads = 256;
constexpr int kAdamFill = 32;                    // tensors that a launch writes into the table: what its arguments hold

struct AdamTensor {
    float* P;
    const void* G;
    void *M, *V;                                 // fp32, or codes
    uint8_t *MS, *VS;                            // their scales
    void* copy;
    int64_t n;
    uint64_t place;
    float decay;
    int16_t kind;                                // 3 * (8-bit states) + type of the gradient
    int16_t copy_dtype;
    uint32_t first, blocks;                      // workgroups
};
// The table: the tensors, then for every workgroup its tensor's number.
struct AdamFill {
    int first, count;
    AdamTensor t[kAdamFill];
};
static_assert(sizeof(AdamFill) <= 4000, "arguments of a launch");
struct AdamStep {
    double lr, b1, b2;
    double rise1, rise2;                         // 1 - b1^t, 1 - b2^t, where the step is known
    const float* lr_dev;
    const int64_t* step_dev;
    const float* grad_scale;
    uint64_t seed;
    int64_t step;
    float c_b1, c_g1, c_b2, c_g2, eps;           // b1, 1 - b1, b2, 1 - b2 as they multiply
    int turns;                                   // eights of a lane
};

__global__ __launch_bounds__(256) void adamw_table_kernel(const AdamFill f, AdamTensor* __restrict__ tensors, uint32_t* __restrict__ of) {
    const AdamTensor& t = f.t[blockIdx.x];
    const uint32_t which = f.first + blockIdx.x;
    if (threadIdx.x == 0) tensors[which] = t;
    for (uint32_t i = threadIdx.x; i < t.blocks; i += 256) of[t.first + i] = which;
}

// 32 bits, mixed: two multiplications by odd numbers (digits of pi and of the golden ratio), each after the upper half is brought down.
__device__ __host__ __forceinline__ uint32_t mix32(uint32_t x) {
    x ^= x >> 16;
    x *= 0x85A308D3u;
    x ^= x >> 15;
    x *= 0x9E3779B1u;
    return x ^ (x >> 16);
}

// b^n for whole n >= 0.
__device__ __host__ __forceinline__ double whole_power(double b, int64_t n) {
    double r = 1.0;
    for (; n > 0; n >>= 1, b *= b)
        if (n & 1) r *= b;
    return r;
}

// The exponent that a group shares, from the bits of its largest magnitude: floor(log2), one more where that lies above the last code; -100 for zeros.
template <int BITS>
__device__ __forceinline__ int state_exponent(uint32_t m) {
    return min(max(static_cast<int>((m + (1u << (23 - BITS)) - 1u) >> 23) - 127, -100), 120);
}

// The code of a magnitude x 2^-f: its upper bits as a float whose exponents end at 15 (below 2^-14: whole multiples of the smallest step), after what is
// dropped and 16 bits of chance are added up.
template <int BITS>
__device__ __forceinline__ uint32_t state_code(float y, uint32_t chance) {
    constexpr int kDrop = 23 - BITS;
    const uint32_t whole = y >= 0x1p-14f ? __float_as_uint(y) - (112u << 23) : static_cast<uint32_t>(y * 0x1p37f);
    return min((whole + (chance << (kDrop - 16))) >> kDrop, (16u << BITS) - 1u);
}
// The magnitude of a code, before the group's scale.
template <int BITS>
__device__ __forceinline__ float state_value(uint32_t code) {
    const float low = static_cast<float>(code) * (0x1p-14f / (1 << BITS));           // (right where the exponent is 0)
    return code < (1u << BITS) ? low : __uint_as_float((code << (23 - BITS)) + (112u << 23));
}
__device__ __forceinline__ float state_scale(uint32_t s) { return s == 255u ? __builtin_nanf("") : pow2f(static_cast<int>(s) - 127); }

template <bool SIGNED>
__device__ __forceinline__ void read_state(uint64_t word, float scale, float (&v)[8]) {
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const uint32_t c = static_cast<uint32_t>(word >> (8 * i)) & 255u;
        if constexpr (SIGNED) v[i] = state_value<3>(c & 127u) * (c & 128u ? -scale : scale);
        else v[i] = state_value<4>(c) * scale;
    }
}
// Eight values as codes, and their group's scale byte; chance(i): 16 bits.
template <bool SIGNED, typename Chance>
__device__ __forceinline__ uint64_t write_state(const float (&v)[8], Chance chance, uint32_t* scale) {
    const uint32_t m = group_max(v);
    if (m >= 0x7f800000u) {
        *scale = 255u;
        return 0;
    }
    const int f = state_exponent<SIGNED ? 3 : 4>(m);
    *scale = static_cast<uint32_t>(f + 127);
    const float inv = pow2f(-f);
    uint64_t word = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const float y = fabsf(v[i]) * inv;
        uint32_t c = state_code<SIGNED ? 3 : 4>(y, chance(i));
        // (a root that is not zero stays so: it stands below a quotient)
        if constexpr (SIGNED) c |= (__float_as_uint(v[i]) >> 31) << 7;
        else if (v[i] > 0.f) c = max(c, 1u);
        word |= static_cast<uint64_t>(c) << (8 * i);
    }
    return word;
}

struct AdamRates {
    float c_b1, c_g1, c_b2, c_g2, eps, keep, first, root;   // ..., 1 - lr wd, lr / (1 - b1^t), 1 / sqrt(1 - b2^t)
    float scale;                                            // of the gradients
    uint32_t key;                                           // of (seed, step)
};

// Eight elements from `at` on.
template <typename TG, bool EIGHT>
__device__ __forceinline__ void adam_eight(const AdamTensor& t, const AdamRates& r, int64_t at) {
    const int left = static_cast<int>(t.n - at < 8 ? t.n - at : 8);     // (below 1 in the last group of codes)
    float g[8], p[8], m[8], v[8];
    load8(static_cast<const TG*>(t.G) + at, 0, left, g);
    load8(t.P + at, 0, left, p);
    if constexpr (EIGHT) {
        const uint64_t qm = *reinterpret_cast<const uint64_t*>(static_cast<const uint8_t*>(t.M) + at);
        const uint64_t qv = *reinterpret_cast<const uint64_t*>(static_cast<const uint8_t*>(t.V) + at);
        read_state<true>(qm, state_scale(t.MS[at >> 5]), m), read_state<false>(qv, state_scale(t.VS[at >> 5]), v);
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            if (i >= left) m[i] = v[i] = 0.f;
            v[i] *= v[i];
        }
    } else {
        load8(static_cast<const float*>(t.M) + at, 0, left, m), load8(static_cast<const float*>(t.V) + at, 0, left, v);
    }
    float root[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const float gi = g[i] * r.scale;
        m[i] = r.c_b1 * m[i] + r.c_g1 * gi;
        v[i] = r.c_b2 * v[i] + (r.c_g2 * gi) * gi;
        root[i] = sqrtf(v[i]);
        p[i] = p[i] * r.keep - (r.first * m[i]) / (root[i] * r.root + r.eps);
    }
    store8(t.P + at, 0, left, p);
    if (t.copy) {
        if (t.copy_dtype == DAB_BF16) store8(static_cast<bf16*>(t.copy) + at, 0, left, p);
        else store8(static_cast<f16*>(t.copy) + at, 0, left, p);
    }
    if constexpr (EIGHT) {
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (i >= left) m[i] = root[i] = 0.f;
        const uint64_t place = t.place + static_cast<uint64_t>(at);
        const uint32_t low = static_cast<uint32_t>(place), key = mix32(static_cast<uint32_t>(place >> 32) + r.key);
        uint32_t chance[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) chance[i] = mix32(low + i + key);
        uint32_t ms, vs;
        const uint64_t qm = write_state<true>(m, [&](int i) { return chance[i] & 0xffffu; }, &ms);
        const uint64_t qv = write_state<false>(root, [&](int i) { return chance[i] >> 16; }, &vs);
        *reinterpret_cast<uint64_t*>(static_cast<uint8_t*>(t.M) + at) = qm;
        *reinterpret_cast<uint64_t*>(static_cast<uint8_t*>(t.V) + at) = qv;
        if ((at & 31) == 0) t.MS[at >> 5] = static_cast<uint8_t>(ms), t.VS[at >> 5] = static_cast<uint8_t>(vs);
    } else {
        store8(static_cast<float*>(t.M) + at, 0, left, m), store8(static_cast<float*>(t.V) + at, 0, left, v);
    }
}

__global__ __launch_bounds__(kAdamThreads) void adamw_kernel(const AdamTensor* __restrict__ tensors, const uint32_t* __restrict__ of, const AdamStep a) {
    DAB_RESERVE_VGPRS();
    const AdamTensor t = tensors[__builtin_amdgcn_readfirstlane(of[blockIdx.x])];
    AdamRates r;
    r.c_b1 = a.c_b1, r.c_g1 = a.c_g1, r.c_b2 = a.c_b2, r.c_g2 = a.c_g2, r.eps = a.eps;
    r.scale = a.grad_scale ? *a.grad_scale : 1.f;
    if (!(fabsf(r.scale) < __builtin_inff())) return;                   // a scale that is no number: no step
    const double lr = a.lr_dev ? static_cast<double>(*a.lr_dev) : a.lr;
    int64_t step = a.step;
    double rise1 = a.rise1, rise2 = a.rise2;
    if (a.step_dev) step = *a.step_dev, rise1 = 1.0 - whole_power(a.b1, step), rise2 = 1.0 - whole_power(a.b2, step);
    r.keep = static_cast<float>(1.0 - lr * static_cast<double>(t.decay));
    r.first = static_cast<float>(lr / rise1);
    r.root = static_cast<float>(1.0 / sqrt(rise2));
    r.key = mix32(static_cast<uint32_t>(a.seed) + mix32(static_cast<uint32_t>(a.seed >> 32) + mix32(static_cast<uint32_t>(step))));
    const int64_t end = t.kind < 3 ? t.n : (t.n + 31) & ~int64_t{31};
    int64_t at = static_cast<int64_t>(blockIdx.x - t.first) * a.turns * (kAdamThreads * 8) + threadIdx.x * 8;
    for (int turn = 0; turn < a.turns; ++turn, at += kAdamThreads * 8) {
        if (at >= end) return;
        switch (t.kind) {
            case 0: adam_eight<float, false>(t, r, at); break;
            case 1: adam_eight<bf16, false>(t, r, at); break;
            case 2: adam_eight<f16, false>(t, r, at); break;
            case 3: adam_eight<float, true>(t, r, at); break;
            case 4: adam_eight<bf16, true>(t, r, at); break;
            default: adam_eight<f16, true>(t, r, at);
        }
    }
}

template <typename T, bool SIGNED>
__global__ __launch_bounds__(kAdamThreads) void state8_restore_kernel(const uint8_t* __restrict__ Q, const uint8_t* __restrict__ S, int64_t n,
                                                                      T* __restrict__ X) {
    const int64_t at = (static_cast<int64_t>(blockIdx.x) * kAdamThreads + threadIdx.x) * 8;
    if (at >= n) return;
    float v[8];
    read_state<SIGNED>(*reinterpret_cast<const uint64_t*>(Q + at), state_scale(S[at >> 5]), v);
    store8(X + at, 0, static_cast<int>(n - at < 8 ? n - at : 8), v);
}

template <bool SIGNED>
__global__ __launch_bounds__(kAdamThreads) void state8_save_kernel(const float* __restrict__ X, int64_t n, uint8_t* __restrict__ Q,
                                                                   uint8_t* __restrict__ S) {
    const int64_t at = (static_cast<int64_t>(blockIdx.x) * kAdamThreads + threadIdx.x) * 8;
    if (at >= ((n + 31) & ~int64_t{31})) return;
    float v[8];
    load8(X + at, 0, static_cast<int>(n - at < 8 ? n - at : 8), v);
    if constexpr (!SIGNED) {
        // (a root has no sign: what is below zero counts as zero, a NaN stays one)
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = v[i] < 0.f ? 0.f : v[i];
    }
    uint32_t scale;
    const uint64_t q = write_state<SIGNED>(v, [](int) { return 0x8000u; }, &scale);
    *reinterpret_cast<uint64_t*>(Q + at) = q;
    if ((at & 31) == 0) S[at >> 5] = static_cast<uint8_t>(scale);
}

static int check_state8(const void* Q, const void* S, int64_t n, const void* X) {
    if (!Q || !S || !X) return DAB_ERR_NULL;
    if (n < 1) return DAB_ERR_SHAPE;
    if (n > (int64_t{1} << 34)) return DAB_ERR_UNSUPPORTED;
    return misaligned(Q, 16) || misaligned(X, 16) ? DAB_ERR_ALIGN : DAB_OK;
}
static dim3 state8_grid(int64_t n) { return dim3(static_cast<unsigned>(ceil_div64(n, kAdamThreads * 8))); }

template <typename T>
static int restore_state8(const uint8_t* Q, const uint8_t* S, int64_t n, bool with_sign, void* X, hipStream_t st) {
    const dim3 grid = state8_grid(n), block(kAdamThreads);
    if (with_sign) return launch(state8_restore_kernel<T, true>, grid, block, 0, st, Q, S, n, static_cast<T*>(X));
    return launch(state8_restore_kernel<T, false>, grid, block, 0, st, Q, S, n, static_cast<T*>(X));
}

static int check_job(const dab_adamw_job& j) {
    if (!j.P || !j.G || !j.M || !j.V || (j.bits == 8 && (!j.MS || !j.VS))) return DAB_ERR_NULL;
    if (j.n < 1 || (j.place & 31) != 0 || !std::isfinite(j.weight_decay)) return DAB_ERR_SHAPE;
    if (!real_dtype(j.grad_dtype) || (j.bits != 8 && j.bits != 32) || j.n > (int64_t{1} << 34)) return DAB_ERR_UNSUPPORTED;
    if (j.copy && j.copy_dtype != DAB_BF16 && j.copy_dtype != DAB_F16) return DAB_ERR_UNSUPPORTED;
    if (misaligned(j.P, 16) || misaligned(j.G, 16) || misaligned(j.M, 16) || misaligned(j.V, 16) || misaligned(j.copy, 16)) return DAB_ERR_ALIGN;
    return DAB_OK;
}

// Eights of a lane: four once the chip is full of workgroups several times over.
static int adam_turns(const dab_adamw_job* jobs, int32_t n) {
    int64_t all = 0;
    for (int32_t i = 0; i < n; ++i) all += ceil_div64(jobs[i].n, kAdamThreads * 8);
    return all > 8 * 8 * kNumCU ? 4 : 1;
}
static int64_t adam_blocks(int64_t n, int turns) { return ceil_div64(n, static_cast<int64_t>(kAdamThreads) * 8 * turns); }
static int64_t adam_table_bytes(int32_t n_jobs, int64_t workgroups) { return round_up(n_jobs * static_cast<int64_t>(sizeof(AdamTensor)) + 4 * workgroups, 256); }
constexpr int64_t kAdamMost = int64_t{1} << 23;  // workgroups

}  // namespace dab

extern "C" int dab_adamw_plan_of(const dab_adamw_job* jobs, int32_t n_jobs, dab_adamw_plan* plan) {
    using namespace dab;
    if (!jobs || !plan) return DAB_ERR_NULL;
    if (n_jobs < 1) return DAB_ERR_SHAPE;
    for (int32_t i = 0; i < n_jobs; ++i)
        if (int rc = check_job(jobs[i])) return rc;
    const int turns = adam_turns(jobs, n_jobs);
    int64_t blocks = 0;
    for (int32_t i = 0; i < n_jobs; ++i) blocks += adam_blocks(jobs[i].n, turns);
    if (blocks > kAdamMost) return DAB_ERR_UNSUPPORTED;
    plan->n_jobs = n_jobs, plan->turns = turns, plan->workgroups = static_cast<int32_t>(blocks);
    plan->table_bytes = adam_table_bytes(n_jobs, blocks);
    return DAB_OK;
}

extern "C" int dab_adamw_table(const dab_adamw_job* jobs, const dab_adamw_plan* plan, void* table, size_t table_bytes, void* stream) {
    using namespace dab;
    if (!jobs || !plan || !table) return DAB_ERR_NULL;
    dab_adamw_plan now;
    if (int rc = dab_adamw_plan_of(jobs, plan->n_jobs, &now)) return rc;
    if (now.turns != plan->turns || now.workgroups != plan->workgroups) return DAB_ERR_SHAPE;
    if (static_cast<int64_t>(table_bytes) < now.table_bytes || misaligned(table, 256)) return DAB_ERR_WORKSPACE;
    AdamTensor* tensors = static_cast<AdamTensor*>(table);
    uint32_t* of = reinterpret_cast<uint32_t*>(tensors + now.n_jobs);
    int64_t blocks = 0;
    for (int32_t i0 = 0; i0 < now.n_jobs; i0 += kAdamFill) {
        AdamFill f{};
        f.first = i0, f.count = now.n_jobs - i0 < kAdamFill ? now.n_jobs - i0 : kAdamFill;
        for (int k = 0; k < f.count; ++k) {
            const dab_adamw_job& j = jobs[i0 + k];
            AdamTensor& t = f.t[k];
            t.P = j.P, t.G = j.G, t.M = j.M, t.V = j.V, t.MS = j.MS, t.VS = j.VS, t.copy = j.copy, t.n = j.n, t.place = j.place;
            t.decay = j.weight_decay, t.kind = static_cast<int16_t>((j.bits == 8 ? 3 : 0) + j.grad_dtype), t.copy_dtype = static_cast<int16_t>(j.copy_dtype);
            t.first = static_cast<uint32_t>(blocks), t.blocks = static_cast<uint32_t>(adam_blocks(j.n, now.turns));
            blocks += t.blocks;
        }
        if (int rc = launch(adamw_table_kernel, dim3(f.count), dim3(256), 0, static_cast<hipStream_t>(stream), f, tensors, of)) return rc;
    }
    return DAB_OK;
}

extern "C" int dab_adamw(const void* table, size_t table_bytes, const dab_adamw_plan* plan, const dab_adamw_step* s, void* stream) {
    using namespace dab;
    if (!table || !plan || !s) return DAB_ERR_NULL;
    if (plan->n_jobs < 1 || plan->workgroups < plan->n_jobs || plan->workgroups > kAdamMost || (plan->turns != 1 && plan->turns != 4)) return DAB_ERR_SHAPE;
    if (static_cast<int64_t>(table_bytes) < adam_table_bytes(plan->n_jobs, plan->workgroups) || misaligned(table, 256)) return DAB_ERR_WORKSPACE;
    const bool rates = s->beta1 >= 0. && s->beta1 < 1. && s->beta2 >= 0. && s->beta2 < 1. && s->eps >= 0. && std::isfinite(s->eps);
    if (!rates || (!s->lr_dev && !std::isfinite(s->lr)) || (!s->step_dev && s->step < 1)) return DAB_ERR_SHAPE;
    if (misaligned(s->lr_dev, 4) || misaligned(s->step_dev, 8) || misaligned(s->grad_scale, 4)) return DAB_ERR_ALIGN;
    AdamStep a{};
    a.lr = s->lr, a.b1 = s->beta1, a.b2 = s->beta2, a.step = s->step, a.lr_dev = s->lr_dev, a.step_dev = s->step_dev;
    a.rise1 = 1.0 - whole_power(s->beta1, s->step), a.rise2 = 1.0 - whole_power(s->beta2, s->step);
    a.grad_scale = s->grad_scale, a.seed = s->seed, a.turns = plan->turns;
    a.c_b1 = static_cast<float>(s->beta1), a.c_g1 = static_cast<float>(1.0 - s->beta1);
    a.c_b2 = static_cast<float>(s->beta2), a.c_g2 = static_cast<float>(1.0 - s->beta2), a.eps = static_cast<float>(s->eps);
    const AdamTensor* tensors = static_cast<const AdamTensor*>(table);
    return launch(adamw_kernel, dim3(plan->workgroups), dim3(kAdamThreads), 0, static_cast<hipStream_t>(stream), tensors,
                  reinterpret_cast<const uint32_t*>(tensors + plan->n_jobs), a);
}

extern "C" int dab_state8_restore(const uint8_t* Q, const uint8_t* S, int64_t n, int32_t is_signed, void* X, int32_t dtype, void* stream) {
    using namespace dab;
    if (int rc = check_state8(Q, S, n, X)) return rc;
    if (!real_dtype(dtype)) return DAB_ERR_UNSUPPORTED;
    const auto st = static_cast<hipStream_t>(stream);
    if (dtype == DAB_F32) return restore_state8<float>(Q, S, n, is_signed != 0, X, st);
    if (dtype == DAB_BF16) return restore_state8<bf16>(Q, S, n, is_signed != 0, X, st);
    return restore_state8<f16>(Q, S, n, is_signed != 0, X, st);
}

extern "C" int dab_state8_save(const float* X, int64_t n, int32_t is_signed, uint8_t* Q, uint8_t* S, void* stream) {
    using namespace dab;
    if (int rc = check_state8(Q, S, n, X)) return rc;
    const auto st = static_cast<hipStream_t>(stream);
    const dim3 grid = state8_grid((n + 31) & ~int64_t{31}), block(kAdamThreads);
    if (is_signed) return launch(state8_save_kernel<true>, grid, block, 0, st, X, n, Q, S);
    return launch(state8_save_kernel<false>, grid, block, 0, st, X, n, Q, S);
}
