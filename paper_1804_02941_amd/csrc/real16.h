// Element types, groups of 32 values with one power of two, and matrix-core forms of the calls on real-valued layers
// (ckpt.hip, w4.hip, head.hip, product16.h).  gfx950 only.
#pragma once

#include "dab_internal.h"

namespace dab {

typedef __bf16 bf16;
typedef _Float16 f16;
typedef __bf16 v8bf __attribute__((ext_vector_type(8)));
typedef __bf16 v2bf __attribute__((ext_vector_type(2)));
typedef float v4f __attribute__((ext_vector_type(4)));
typedef uint32_t v4u32 __attribute__((ext_vector_type(4)));
typedef uint32_t v2u32 __attribute__((ext_vector_type(2)));

inline bool real_dtype(int32_t t) { return t == DAB_F32 || t == DAB_BF16 || t == DAB_F16; }
inline int64_t dtype_bytes(int32_t t) { return t == DAB_F32 ? 4 : 2; }
// bf16 numbers whose sum a value of the type is, exactly (24, 8 and 11 significant bits in pieces of 8)
inline int dtype_pieces(int32_t t) { return t == DAB_F32 ? 3 : t == DAB_F16 ? 2 : 1; }
inline int64_t round_up(int64_t v, int64_t m) { return (v + m - 1) / m * m; }
inline int64_t ceil_div64(int64_t a, int64_t b) { return (a + b - 1) / b; }
// Whether the bytes of two matrices, first to last, meet.
struct Extent {
    const void* p;
    int64_t rows, cols, ld, size;
    uintptr_t first() const { return reinterpret_cast<uintptr_t>(p); }
    uintptr_t end() const { return first() + static_cast<uintptr_t>(((rows - 1) * ld + cols) * size); }
};
inline bool meet(const Extent& a, const Extent& b) { return a.first() < b.end() && b.first() < a.end(); }

// 2^e as fp32 for -126 <= e <= 127.
__device__ __forceinline__ float pow2f(int e) { return __builtin_bit_cast(float, static_cast<uint32_t>(e + 127) << 23); }

// Vectors of elements at any address of theirs: the memory system takes 16 bytes a lane at any alignment (rows whose distance is odd cost a
// line more here and there, not eight loads for one).
template <typename T, int N>
struct Unaligned {
    typedef T type __attribute__((ext_vector_type(N), aligned(sizeof(T))));
};

// Eight elements of a row from column c on as fp32, zeros past the row's end.
template <typename T>
__device__ __forceinline__ void load8(const T* row, int c, int cols, float (&v)[8]) {
    if (c + 8 <= cols) {
        typedef typename Unaligned<T, 4>::type v4t;
        typedef typename Unaligned<T, 8>::type v8t;
        if constexpr (sizeof(T) == 4) {
            const v4t a = *reinterpret_cast<const v4t*>(row + c), b = *reinterpret_cast<const v4t*>(row + c + 4);
#pragma unroll
            for (int i = 0; i < 4; ++i) v[i] = a[i], v[4 + i] = b[i];
        } else {
            const v8t a = *reinterpret_cast<const v8t*>(row + c);
#pragma unroll
            for (int i = 0; i < 8; ++i) v[i] = static_cast<float>(a[i]);
        }
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = c + i < cols ? static_cast<float>(row[c + i]) : 0.f;
    }
}

// The same eight back; what lies past the row's end is not written.
template <typename T>
__device__ __forceinline__ void store8(T* row, int c, int cols, const float (&v)[8]) {
    if (c + 8 <= cols) {
        typedef typename Unaligned<T, 4>::type v4t;
        typedef typename Unaligned<T, 8>::type v8t;
        if constexpr (sizeof(T) == 4) {
            *reinterpret_cast<v4t*>(row + c) = v4t{v[0], v[1], v[2], v[3]};
            *reinterpret_cast<v4t*>(row + c + 4) = v4t{v[4], v[5], v[6], v[7]};
        } else {
            v8t a;
#pragma unroll
            for (int i = 0; i < 8; ++i) a[i] = static_cast<T>(v[i]);
            *reinterpret_cast<v8t*>(row + c) = a;
        }
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (c + i < cols) row[c + i] = static_cast<T>(v[i]);
    }
}

// Eight values without the first `again`, the others moved to the front, zeros behind them.
__device__ __forceinline__ void own_first(int again, float (&y)[8]) {
    if (again == 0) return;
#pragma unroll
    for (int by = 4; by > 0; by >>= 1)
        if (again & by)
#pragma unroll
            for (int i = 0; i < 8; ++i) y[i] = i + by < 8 ? y[(i + by) & 7] : 0.f;
}

// Largest magnitude, as bits (those of a NaN are larger than those of any number), over the four lanes that hold a group.
__device__ __forceinline__ uint32_t group_max(const float (&v)[8]) {
    uint32_t m = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) m = max(m, __builtin_bit_cast(uint32_t, v[i]) & 0x7fffffffu);
    m = max(m, static_cast<uint32_t>(__builtin_amdgcn_update_dpp(0, static_cast<int>(m), 0xB1, 0xf, 0xf, true)));   // lane ^ 1
    m = max(m, static_cast<uint32_t>(__builtin_amdgcn_update_dpp(0, static_cast<int>(m), 0x4E, 0xf, 0xf, true)));   // lane ^ 2
    return m;
}

// Exponent of a group from its largest magnitude: floor(log2) - TOP, kept within -110 .. 120 so that every scaled value and
// every restored one is a normal bf16 number, one more where the largest scaled value would round past the format's last.
template <int TOP>
__device__ __forceinline__ int group_exponent(uint32_t m) {
    if (m == 0) return -110;
    int e = min(max(static_cast<int>(m >> 23) - 127 - TOP, -110), 120);
    const float at = __builtin_bit_cast(float, m) * pow2f(-e);
    if (TOP == 6 ? at >= 127.5f : at > 7.f) ++e;
    return e;
}

// Whether a token has no part in the loss.
__device__ __forceinline__ bool no_loss(int64_t target, int64_t ignore, int V) { return target == ignore || target < 0 || target >= V; }

// x without what a bf16 number does not hold.
__device__ __forceinline__ float cut16(float x) { return __uint_as_float(__float_as_uint(x) & 0xffff0000u); }
// Piece `which` of the bf16 numbers whose sum x is: x rounded, what is left rounded, what is left then.  Numbers that would round to infinity are
// cut instead, and so is what is left of them, so that no sum of their pieces passes fp32's last number; of an infinity and of a NaN nothing
// is left behind the first piece (their difference would be undefined).
__device__ __forceinline__ bf16 piece_of(float x, int which) {
    const uint32_t size = __float_as_uint(x) & 0x7fffffffu;
    const bool finite = size < 0x7f800000u, last = finite && size >= 0x7f7f8000u;
    const bf16 a = static_cast<bf16>(last ? cut16(x) : x);
    if (which == 0) return a;
    const float r = finite ? x - static_cast<float>(a) : 0.f;
    const bf16 b = static_cast<bf16>(last ? cut16(r) : r);
    if (which == 1) return b;
    return static_cast<bf16>(r - static_cast<float>(b));
}

}  // namespace dab
