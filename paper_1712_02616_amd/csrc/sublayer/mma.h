// Fragments of the matrix instructions: 16 bytes per lane whatever the type,
// 8 16-bit elements for one 16x16x32 instruction, or 4 fp32 for four 16x16x4
// ones, whose k indices are those that the lanes hold (any order of the sum
// over k will do, the same for both operands).  Lane l holds row (or column)
// l % 16 and the 16 bytes number l / 16 of 64; of a result, column l % 16 and
// rows 4*(l / 16) to + 3.
#pragma once

#include "common.h"

namespace iabn_impl {

typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

template <int DT>
struct Mma;
template <>
struct Mma<IABN_BF16> {
    typedef __bf16 frag __attribute__((ext_vector_type(8)));
    static __device__ __forceinline__ f32x4 run(u32x4 a, u32x4 b, f32x4 c) {
        return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(frag, a),
                                                       __builtin_bit_cast(frag, b), c, 0, 0, 0);
    }
};
template <>
struct Mma<IABN_F16> {
    typedef _Float16 frag __attribute__((ext_vector_type(8)));
    static __device__ __forceinline__ f32x4 run(u32x4 a, u32x4 b, f32x4 c) {
        return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(frag, a),
                                                      __builtin_bit_cast(frag, b), c, 0, 0, 0);
    }
};
template <>
struct Mma<IABN_F32> {
    static __device__ __forceinline__ f32x4 run(u32x4 a, u32x4 b, f32x4 c) {
#pragma unroll
        for (int j = 0; j < 4; ++j)
            c = __builtin_amdgcn_mfma_f32_16x16x4f32(__builtin_bit_cast(f32x4, a)[j],
                                                     __builtin_bit_cast(f32x4, b)[j], c, 0, 0, 0);
        return c;
    }
};

// 16 bytes of consecutive elements at element alignment.
template <int DT, int HINT>
__device__ __forceinline__ u32x4 load16(const typename Elem<DT>::T* p) {
    using T = typename Elem<DT>::T;
    typedef T vec __attribute__((ext_vector_type(16 / sizeof(T))));
    typedef T mem __attribute__((ext_vector_type(16 / sizeof(T)), aligned(sizeof(T))));
    const mem* const q = reinterpret_cast<const mem*>(p);
    const vec v = HINT == kStream ? __builtin_nontemporal_load(q) : *q;
    return __builtin_bit_cast(u32x4, v);
}

// The same where those past the first n are zero and not read.
template <int DT>
__device__ __forceinline__ u32x4 load16_first(const typename Elem<DT>::T* p, int64_t n) {
    using T = typename Elem<DT>::T;
    constexpr int E = 16 / sizeof(T);
    if (n >= E) return load16<DT, kCached>(p);
    typedef T vec __attribute__((ext_vector_type(E)));
    vec v = {};
#pragma unroll
    for (int j = 0; j < E; ++j)
        if (j < n) v[j] = p[j];
    return __builtin_bit_cast(u32x4, v);
}

}  // namespace iabn_impl
