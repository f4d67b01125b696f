// Definitions shared by the kernels of a transformer's feed-forward sublayer:
// accesses of 8 elements at any alignment, sums over a wave and a block, the
// counter-based generator of the dropout, and what the host side hands to the
// kernels.
#pragma once

#include "common.h"

namespace iabn_impl {

// ---------------------------------------------------------------- chunks

// A chunk is 8 consecutive elements of a row.  Rows need not start on a
// 16-byte boundary (odd widths, tensors that are offset): the accesses are
// declared at element alignment, which the hardware takes in one instruction
// per 16 bytes.  The last chunk of a row may hold fewer elements and moves
// one by one.
constexpr int kChunk = 8;

// Chunks of a row of C elements, C < 2^31 (C + 7 in an int would overflow for the
// last seven widths).
constexpr int chunks_of(int64_t C) { return static_cast<int>((C + kChunk - 1) / kChunk); }
static_assert(chunks_of((int64_t(1) << 31) - 1) == 1 << 28 && chunks_of((int64_t(1) << 31) - 8) == (1 << 28) - 1, "");

template <int DT>
struct ChunkOf {
    using T = typename Elem<DT>::T;
    typedef T vec __attribute__((ext_vector_type(8)));
    typedef T mem __attribute__((ext_vector_type(8), aligned(sizeof(T))));
};

// Elements [at, at + n) of `base`, n <= 8; the rest of the chunk is zero.
template <int DT, int HINT>
__device__ __forceinline__ typename ChunkOf<DT>::vec load_chunk(const void* __restrict__ base,
                                                                int64_t at, int n) {
    using T = typename ChunkOf<DT>::T;
    const T* p = static_cast<const T*>(base) + at;
    typename ChunkOf<DT>::vec v = {};
    if (n >= kChunk) {
        const auto* q = reinterpret_cast<const typename ChunkOf<DT>::mem*>(p);
        if constexpr (HINT == kStream) v = __builtin_nontemporal_load(q);
        else v = *q;
    } else {
#pragma unroll
        for (int j = 0; j < kChunk; ++j)
            if (j < n) v[j] = p[j];
    }
    return v;
}

template <int DT, int HINT>
__device__ __forceinline__ void store_chunk(void* __restrict__ base, int64_t at, int n,
                                            const float (&f)[kChunk]) {
    using T = typename ChunkOf<DT>::T;
    T* p = static_cast<T*>(base) + at;
    typedef float vf __attribute__((ext_vector_type(8)));
    vf w;
#pragma unroll
    for (int j = 0; j < kChunk; ++j) w[j] = f[j];
    const typename ChunkOf<DT>::vec v = __builtin_convertvector(w, typename ChunkOf<DT>::vec);
    if (n >= kChunk) {
        auto* q = reinterpret_cast<typename ChunkOf<DT>::mem*>(p);
        if constexpr (HINT == kStream) __builtin_nontemporal_store(static_cast<typename ChunkOf<DT>::mem>(v), q);
        else *q = v;
    } else {
#pragma unroll
        for (int j = 0; j < kChunk; ++j)
            if (j < n) p[j] = v[j];
    }
}

template <int DT>
__device__ __forceinline__ void widen(const typename ChunkOf<DT>::vec& v, float (&f)[kChunk]) {
    typedef float vf __attribute__((ext_vector_type(8)));
    const vf w = __builtin_convertvector(v, vf);
#pragma unroll
    for (int j = 0; j < kChunk; ++j) f[j] = w[j];
}

// The chunks of a row over the threads that hold it.  A load under a branch is
// waited for where the branches join, so where a row does not fill its threads
// (kPartial) every thread loads 8 elements of it whatever it has of them, the
// last 8 where its chunk ends beyond the row, and they are put in their place
// when they are used (place_chunk).  kFull: every thread has a whole chunk, and
// nothing is masked; kShort: rows of fewer than 8 elements, one by one.
enum RowFill { kFull, kPartial, kShort };

struct RowChunk {
    int col;   // the chunk's first element
    int from;  // the first element to load
    int n;     // elements inside the row (0 for a thread that has none)
};
template <int FILL>
__device__ __forceinline__ RowChunk row_chunk(int chunk, int C) {
    const int col = chunk * kChunk;
    if constexpr (FILL == kFull) return {col, col, kChunk};
    return {col, FILL == kShort ? col : min(col, C - kChunk), max(min(kChunk, C - col), 0)};
}
template <int DT, int HINT, int FILL>
__device__ __forceinline__ typename ChunkOf<DT>::vec load_row_chunk(const void* __restrict__ base,
                                                                    int64_t row, const RowChunk& c) {
    return load_chunk<DT, HINT>(base, row + c.from, FILL == kShort ? c.n : kChunk);
}
template <int DT, int HINT, int FILL>
__device__ __forceinline__ void store_row_chunk(void* __restrict__ base, int64_t row, const RowChunk& c,
                                                const float (&v)[kChunk]) {
    store_chunk<DT, HINT>(base, row + c.col, FILL == kFull ? kChunk : c.n, v);
}

// The loaded elements in their place: those before the chunk's leave, zeros
// follow the row's last.  A shift by 8 - n elements, in steps of 8, 4, 2 and 1.
template <int DT, int FILL>
__device__ __forceinline__ typename ChunkOf<DT>::vec place_chunk(typename ChunkOf<DT>::vec v,
                                                                 const RowChunk& c) {
    if constexpr (FILL != kPartial) return v;
    const int shift = kChunk - c.n;
    typename ChunkOf<DT>::vec w;
#pragma unroll
    for (int step = kChunk; step >= 1; step >>= 1) {
#pragma unroll
        for (int j = 0; j < kChunk; ++j) {
            const auto moved = j + step < kChunk ? v[j + step < kChunk ? j + step : 0]
                                                 : static_cast<typename ChunkOf<DT>::T>(0.0f);
            w[j] = shift & step ? moved : v[j];
        }
        v = w;
    }
    return v;
}
// v where it is inside the row, else 0.
template <int FILL>
__device__ __forceinline__ float inside_row(const RowChunk& c, int j, float v) {
    return FILL == kFull || j < c.n ? v : 0.0f;
}

// ---------------------------------------------------------------- sums

template <int CTRL, int ROW_MASK>
__device__ __forceinline__ float dpp_f32(float v) {
    return __builtin_bit_cast(
        float, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, v), CTRL, ROW_MASK, 0xF, true));
}

// Sum over the 64 lanes of a wave (every lane active), in every lane; the
// steps of the double form in common.h.
__device__ __forceinline__ float wave_sum_f32(float v) {
    v += dpp_f32<0x111, 0xF>(v);
    v += dpp_f32<0x112, 0xF>(v);
    v += dpp_f32<0x114, 0xF>(v);
    v += dpp_f32<0x118, 0xF>(v);
    v += dpp_f32<0x142, 0xA>(v);
    v += dpp_f32<0x143, 0xC>(v);
    return __builtin_bit_cast(float,
                              __builtin_amdgcn_readlane(__builtin_bit_cast(int, v), 63));
}

constexpr int kMaxRowWaves = 16;

// One or two sums over the waves of a row's threads, each in a fixed order, in
// every thread.  One wave needs no more than its DPP steps.  More waves exchange
// their sums through `slot`, with one barrier: consecutive sums of a block
// have to use different slots, and a slot may come again after one other.
struct alignas(8) SumSlot {
    float a[kMaxRowWaves], b[kMaxRowWaves];
};

// Sum over each row of 16 lanes, in its lane 15, read from the first row.
__device__ __forceinline__ float row16_sum_f32(float v) {
    v += dpp_f32<0x111, 0xF>(v);
    v += dpp_f32<0x112, 0xF>(v);
    v += dpp_f32<0x114, 0xF>(v);
    v += dpp_f32<0x118, 0xF>(v);
    return __builtin_bit_cast(float,
                              __builtin_amdgcn_readlane(__builtin_bit_cast(int, v), 15));
}

// Before a block's first row_sum2 (with a barrier between): the places of
// waves that the block does not have.
__device__ __forceinline__ void clear_slots(SumSlot* slots, int n) {
    for (int i = threadIdx.x; i < n * 2 * kMaxRowWaves; i += blockDim.x)
        reinterpret_cast<float*>(slots)[i] = 0.0f;
    __syncthreads();
}

template <bool ONE_WAVE>
__device__ __forceinline__ float row_sum(float a, SumSlot& slot) {
    a = wave_sum_f32(a);
    if constexpr (!ONE_WAVE) {
        if (lane_id() == 0) slot.a[threadIdx.x / kWave] = a;
        __syncthreads();
        a = row16_sum_f32(slot.a[lane_id() % kMaxRowWaves]);
    }
    return a;
}

template <bool ONE_WAVE>
__device__ __forceinline__ void row_sum2(float& a, float& b, SumSlot& slot) {
    a = wave_sum_f32(a);
    b = wave_sum_f32(b);
    if constexpr (!ONE_WAVE) {
        const int w = threadIdx.x / kWave;
        if (lane_id() == 0) {
            slot.a[w] = a;
            slot.b[w] = b;
        }
        __syncthreads();
        a = row16_sum_f32(slot.a[lane_id() % kMaxRowWaves]);
        b = row16_sum_f32(slot.b[lane_id() % kMaxRowWaves]);
    }
}

// ---------------------------------------------------------------- dropout

// What a dropout keeps: element (row, col) of a [rows, C] tensor belongs to
// lane col % 8 of the group row * ceil(C / 8) + col / 8, and is kept where
// the lane's 16 random bits are >= threshold = p in 2^-16ths; then it is
// scaled by 1 / (1 - threshold / 65536).  The bits of a group are the
// Philox4x32-10 output (Salmon, Moraes, Dror, Shaw, "Parallel random numbers:
// as easy as 1, 2, 3", SC11) for the counter (group, offset) and the key
// seed: a function of the element's place alone, so the backward makes them
// again and no mask is stored.  8 elements per generator call: its 20
// products of 32x32 bits are the kernels' largest integer work.
struct Dropout {
    uint32_t threshold;  // 0: keeps everything
    float scale;
    uint64_t seed, offset;
};

__device__ __forceinline__ void philox(uint64_t group, uint64_t offset, uint64_t seed,
                                       uint32_t (&w)[4]) {
    uint32_t c0 = static_cast<uint32_t>(group), c1 = static_cast<uint32_t>(group >> 32);
    uint32_t c2 = static_cast<uint32_t>(offset), c3 = static_cast<uint32_t>(offset >> 32);
    uint32_t k0 = static_cast<uint32_t>(seed), k1 = static_cast<uint32_t>(seed >> 32);
#pragma unroll
    for (int i = 0; i < 10; ++i) {
        const uint64_t a = uint64_t(0xD2511F53u) * c0, b = uint64_t(0xCD9E8D57u) * c2;
        const uint32_t n0 = static_cast<uint32_t>(b >> 32) ^ c1 ^ k0;
        const uint32_t n2 = static_cast<uint32_t>(a >> 32) ^ c3 ^ k1;
        c1 = static_cast<uint32_t>(b);
        c3 = static_cast<uint32_t>(a);
        c0 = n0;
        c2 = n2;
        k0 += 0x9E3779B9u;
        k1 += 0xBB67AE85u;
    }
    w[0] = c0;
    w[1] = c1;
    w[2] = c2;
    w[3] = c3;
}

// The factors of a group's 8 elements are applied as a choice, not a product,
// so that a dropped infinity or NaN is 0.
__device__ __forceinline__ void drop_group(const Dropout& d, uint64_t group, float (&v)[kChunk]) {
    uint32_t w[4];
    philox(group, d.offset, d.seed, w);
#pragma unroll
    for (int j = 0; j < kChunk; ++j) {
        const uint32_t bits = (j & 1) ? w[j >> 1] >> 16 : w[j >> 1] & 0xFFFFu;
        v[j] = bits >= d.threshold ? v[j] * d.scale : 0.0f;
    }
}

// ---------------------------------------------------------------- norms around a block

// r = alpha*x + beta*gate*D(post(h)),  u = pre(r)   (iabn_resnorm_forward)
struct ResnormArgs {
    const void *x, *h;       // [R, C]; h may be null: r = alpha*x
    void *r, *u;             // [R, C]; either may be null
    const void* gate;        // [groups, C] or null
    const float *post_w, *post_b, *pre_w, *pre_b;  // [C] or null
    float *post_stats, *pre_stats;                 // [2, R] or null
    int post, pre;           // iabn_norm_t
    float alpha, beta, eps, inv_c;
    Dropout drop;
    int64_t R, gate_rows;    // rows that share a row of the gate
    int C, chunks;           // chunks = ceil(C / 8)
};

// The backward's rows over its blocks: `groups` of group_rows rows (those of
// a row of the gate, or all rows), each cut into per_group segments; a block
// takes `segs` consecutive segments, one where a group has several.
struct ResnormSplit {
    int64_t groups, group_rows;
    int per_group, segs, blocks;
};

struct ResnormBwdArgs {
    const void *dr, *du, *r, *h;
    void *dx, *dh;
    const void* gate;
    const float *post_w, *post_b, *pre_w;
    const float *post_stats, *pre_stats;  // [2, R]
    void* dgate;                          // [groups, C] or null
    float *dpost_w, *dpost_b, *dpre_w, *dpre_b;  // [C] or null
    int post, pre;
    float alpha, beta, inv_c;
    Dropout drop;
    int64_t R, gate_rows;  // rows that share a row of the gate
    int C, chunks;
    bool gate_each_row;  // every row has its own gate: its gradient is no sum
    ResnormSplit split;
    float* part;   // [4][blocks][C]: post_w, post_b, pre_w, pre_b
    float* gpart;  // [blocks][C]: the gate's, where per_group > 1
};

// Zeroes a buffer of whole elements with a kernel (a captured graph replays it).
void launch_zero(void* p, int64_t bytes, hipStream_t st);

bool launch_dropout(int dtype, const void* x, void* y, int64_t R, int C, const Dropout& d,
                    hipStream_t st);
bool launch_resnorm_fwd(int dtype, const ResnormArgs& a, hipStream_t st);
bool launch_resnorm_bwd(int dtype, const ResnormBwdArgs& a, hipStream_t st);

// Threads of a row, and how many chunks each holds.
struct RowShape {
    int waves, k;
};
// one_wave: the most chunks of a thread for which a row stays in one wave.
inline RowShape row_shape(int chunks, int one_wave) {
    for (int k = 1; k <= one_wave; ++k)
        if (chunks <= k * kWave) return {1, k};
    const int k = chunks <= kMaxRowWaves * kWave ? 1 : 2;
    return {(chunks + k * kWave - 1) / (k * kWave), k};
}

// Rows of one wave: up to 2 chunks a thread in the forward ((32768, 1024) fp16,
// all parts: 62 us, 69 in two waves); 1 in the backward, whose columns' sums take
// 40 registers a chunk (the same rows 93 us and 11 for the sums in two waves, 108
// and 5 in one; bf16 with RMS norms 86 and 11, 101 and 5).
constexpr int kFwdOneWave = 2, kBwdOneWave = 1;

}  // namespace iabn_impl
