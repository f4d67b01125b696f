// Products over groups of rows: those of routed experts.  The pairs (token, slot) are
// sorted by expert (a plan: routed.h); expert e has the sorted rows
// offsets[e] .. offsets[e + 1], and weights of its own.
//
//   up, dh:   X's rows are tokens, gathered by the plan's order; down, dx: X's rows are
//             sorted ones.  Y is the expert's weights.
//   dW:       the sum over k is over the expert's rows; one operand's are tokens.
//
// A block finds its expert from the offsets (which only the GPU knows): a wave
// adds up how many tiles each expert has.  The numbers of a plan are held to their
// ranges where they are used, so that a wrong one reads a wrong row of the right
// matrix.
#pragma once

#include <type_traits>

#include "ffn.h"
#include "routed.h"

namespace iabn_impl {

// The kinds of products over groups: kOverGroups + a GemmKind, where dW's x is the
// tokens' operand, or its y.
constexpr int kOverGroups = 10, kGroupDwTokensY = kOverGroups + kGemmDw + 1;

struct GroupArgs : GemmArgs {
    const int32_t *offsets, *order, *by_size;
    const float* weights;    // [M, k]: down, dh
    float* dots;             // dh: [P][ceil(F/64)], sums of h*(dy Wd) over 64 columns
    iabn_divmagic_t top;     // k
    int32_t E, P;
    int64_t expert_stride;   // elements from one expert's matrix to the next one's
};
template <int KIND>
using ArgsOf = std::conditional_t<(KIND < kOverGroups), GemmArgs, GroupArgs>;

// The tokens of a group's rows.
struct Tokens {
    const int32_t* order;  // from the group's first row
    uint32_t pairs;
    iabn_divmagic_t top;
    __device__ __forceinline__ uint32_t pair(uint32_t entry) const { return min(entry, pairs - 1); }
    __device__ __forceinline__ uint32_t of(uint32_t entry) const { return iabn_divmagic_div(pair(entry), top); }
    __device__ __forceinline__ int64_t operator()(int64_t row) const { return of(order[row]); }
};

__device__ __forceinline__ float pair_weight(const GroupArgs& a, const Tokens& tokens, int64_t m, int64_t M) {
    return m < M ? a.weights[tokens.pair(tokens.order[m])] : 0.0f;
}

__device__ __forceinline__ void rows_of(const int32_t* offsets, int e, int P, int& first, int& rows) {
    first = min(max(offsets[e], 0), P);
    rows = max(min(offsets[e + 1], P) - first, 0);
}

// A tile's number for a block's: runs of `run` consecutive tiles stay on one XCD
// (its L2 holds what they share), the runs go round the XCDs (experts differ in how
// many rows they have).
__device__ __forceinline__ uint32_t spread(uint32_t block, uint32_t n, uint32_t run) {
    const uint32_t round = run * kXcds, whole = n / round * round;
    if (block < whole) {
        const uint32_t x = block % kXcds, j = block / kXcds;
        return j / run * round + x * run + j % run;
    }
    const uint32_t left = n - whole, b = block - whole, x = b % kXcds, j = b / kXcds;
    return whole + x * (left / kXcds) + min(x, left % kXcds) + j;
}

// Tile `t` of tiles_m x tiles_n, in strips of a few tiles of m.
__device__ __forceinline__ void strip_of(uint32_t t, int tiles_m, int tiles_n, int strip_height, int& tm, int& tn) {
    const uint32_t strip = t / (strip_height * tiles_n), in = t - strip * (strip_height * tiles_n);
    const uint32_t height = min(static_cast<uint32_t>(strip_height), tiles_m - strip * strip_height);
    tn = static_cast<int>(in / height);
    tm = static_cast<int>(strip * strip_height + in % height);
}

// The expert that tile number t of the launch (tiles_n tiles for every TM of an
// expert's rows) belongs to, and the tile's number in it; false past the last.
template <int CTRL>
__device__ __forceinline__ int shifted(int v) {
    return __builtin_amdgcn_update_dpp(0, v, CTRL, 0xF, 0xF, true);
}
struct Group {
    int expert, first, rows;
    uint32_t tile;
};
template <int TM>
__device__ __forceinline__ bool find_group(const int32_t* offsets, int E, int P, uint32_t tiles_n, uint32_t run,
                                           Group& g) {
    const int each = (E + kWave - 1) / kWave, e0 = static_cast<int>(lane_id()) * each, e1 = min(e0 + each, E);
    int tiles = 0;
    for (int e = e0; e < e1; ++e) {
        int first, rows;
        rows_of(offsets, e, P, first, rows);
        tiles += (rows + TM - 1) / TM;
    }
    // The sum over the lanes up to each: in rows of 16, then over the rows' ends.
    int upto = tiles;
    upto += shifted<0x111>(upto);
    upto += shifted<0x112>(upto);
    upto += shifted<0x114>(upto);
    upto += shifted<0x118>(upto);
    {
        const int row = static_cast<int>(lane_id()) / 16;
        const int end0 = __builtin_amdgcn_readlane(upto, 15), end1 = __builtin_amdgcn_readlane(upto, 31),
                  end2 = __builtin_amdgcn_readlane(upto, 47);
        upto += (row > 0 ? end0 : 0) + (row > 1 ? end1 : 0) + (row > 2 ? end2 : 0);
    }
    const uint32_t total = static_cast<uint32_t>(__builtin_amdgcn_readlane(upto, kWave - 1)) * tiles_n;
    if (blockIdx.x >= total) return false;
    const uint32_t t = run ? spread(blockIdx.x, total, run) : blockIdx.x;
    const int m = static_cast<int>(t / tiles_n);
    const uint64_t has = __ballot(upto - tiles <= m && m < upto);
    const int lane = __builtin_ctzll(has);
    int before = upto - tiles, expert = e0, first = 0, rows = 0;
    for (int e = e0; e < e1; ++e) {
        rows_of(offsets, e, P, first, rows);
        const int n = (rows + TM - 1) / TM;
        expert = e;
        if (m < before + n) break;
        before += n;
    }
    g.expert = __builtin_amdgcn_readlane(expert, lane);
    g.first = __builtin_amdgcn_readlane(first, lane);
    g.rows = __builtin_amdgcn_readlane(rows, lane);
    g.tile = t - static_cast<uint32_t>(__builtin_amdgcn_readlane(before, lane)) * tiles_n;
    return true;
}

// A pair's term of its token's sum (y, dx), between the product that forms it and the
// kernel that adds the terms up.  fp32 for fp32; else the upper 24 bits of it, 16 in
// `high` and 8 in `low`: with fp32's range, and so many digits that they do not show
// beside the result's rounding.  (In the storage type y of (4096, 8 of 64 experts,
// 2048 -> 1024) bf16 is off by 2.9e-3 in root mean square, with these by 2.3e-3,
// which h's rounding leaves, at 26 us of 545 more.)
template <int DT>
__device__ __forceinline__ void store_terms(void* high, void* low, int64_t at, int n, const float (&v)[kChunk]) {
    if constexpr (DT == IABN_F32) {
        store_chunk<IABN_F32, kCached>(high, at, n, v);
    } else {
        typedef uint16_t high_t __attribute__((ext_vector_type(8)));
        typedef uint16_t high_mem __attribute__((ext_vector_type(8), aligned(2)));
        typedef uint8_t low_t __attribute__((ext_vector_type(8)));
        typedef uint8_t low_mem __attribute__((ext_vector_type(8), aligned(1)));
        high_t h;
        low_t l;
#pragma unroll
        for (int j = 0; j < kChunk; ++j) {
            const uint32_t bits = __builtin_bit_cast(uint32_t, v[j]) + (v[j] == v[j] ? 0x80u : 0u);
            h[j] = static_cast<uint16_t>(bits >> 16);
            l[j] = static_cast<uint8_t>(bits >> 8);
        }
        uint16_t* const ph = static_cast<uint16_t*>(high) + at;
        uint8_t* const pl = static_cast<uint8_t*>(low) + at;
        if (n >= kChunk) {
            *reinterpret_cast<high_mem*>(ph) = h;
            *reinterpret_cast<low_mem*>(pl) = l;
        } else {
#pragma unroll
            for (int j = 0; j < kChunk; ++j)
                if (j < n) ph[j] = h[j], pl[j] = l[j];
        }
    }
}
// The bits of kChunk terms as they are loaded, and the terms.
template <int DT>
struct Terms {
    typename ChunkOf<IABN_F32>::vec v;
    __device__ __forceinline__ void load(const void* high, const void*, int64_t at, int n) {
        v = load_chunk<IABN_F32, kStream>(high, at, n);
    }
    __device__ __forceinline__ void get(float (&f)[kChunk]) const { widen<IABN_F32>(v, f); }
};
struct Terms24 {
    typedef uint16_t high_t __attribute__((ext_vector_type(8)));
    typedef uint8_t low_t __attribute__((ext_vector_type(8)));
    high_t h;
    low_t l;
    __device__ __forceinline__ void load(const void* high, const void* low, int64_t at, int n) {
        typedef uint16_t high_mem __attribute__((ext_vector_type(8), aligned(2)));
        typedef uint8_t low_mem __attribute__((ext_vector_type(8), aligned(1)));
        const uint16_t* const ph = static_cast<const uint16_t*>(high) + at;
        const uint8_t* const pl = static_cast<const uint8_t*>(low) + at;
        h = {}, l = {};
        if (n >= kChunk) {
            h = __builtin_nontemporal_load(reinterpret_cast<const high_mem*>(ph));
            l = __builtin_nontemporal_load(reinterpret_cast<const low_mem*>(pl));
        } else {
#pragma unroll
            for (int j = 0; j < kChunk; ++j)
                if (j < n) h[j] = ph[j], l[j] = pl[j];
        }
    }
    __device__ __forceinline__ void get(float (&f)[kChunk]) const {
#pragma unroll
        for (int j = 0; j < kChunk; ++j)
            f[j] = __builtin_bit_cast(float, static_cast<uint32_t>(h[j]) << 16 | static_cast<uint32_t>(l[j]) << 8);
    }
};
template <>
struct Terms<IABN_F16> : Terms24 {};
template <>
struct Terms<IABN_BF16> : Terms24 {};

// A group's operand: its two matrices in registers (an array that is indexed by a
// register would go through scratch memory).
struct GroupOperand {
    const void *p0, *p1;
    int64_t ld;
};
__device__ __forceinline__ const void* matrix(const Operand& o, int q) { return o.p[q]; }
__device__ __forceinline__ const void* matrix(const GroupOperand& o, int q) {
    const uint64_t a = reinterpret_cast<uint64_t>(o.p0), b = reinterpret_cast<uint64_t>(o.p1);
    return reinterpret_cast<const void*>(q ? b : a);
}

// What a block's group is: its rows or its part of k, its weights, its outputs.
struct Entered {
    GroupOperand x, y;
    int64_t rows;  // of the group: M, or K of dW
    int64_t row0;  // the group's first sorted row
    int64_t out;   // elements from the outputs' first one (dW)
};
constexpr int kGroupStrip = 8;
template <int DT, int KIND, int TM>
__device__ __forceinline__ bool enter_group(const GroupArgs& a, int tiles_m, int tiles_n, int& tm, int& tn,
                                            Entered& in, Tokens& tokens) {
    using T = typename Elem<DT>::T;
    // (Runs of the largest tile, one on each of an XCD's CUs; of 16 no other times, of 64
    // 2115 us for the backward of 8192 tokens instead of 2025.)
    constexpr uint32_t kRun = TM == 256 ? 32 : 64;
    const auto from = [](const Operand& o, int64_t by) -> GroupOperand {
        return {static_cast<const T*>(o.p[0]) + by, static_cast<const T*>(o.p[1]) + by, o.ld};
    };
    int first, rows;
    if constexpr (KIND == kOverGroups + kGemmDw || KIND == kGroupDwTokensY) {
        // The experts with the longest sums first: what is left at the end is short
        // (two skewed choices, gate and up, (8192, 8 of 64 experts, 2048 -> 1024) bf16: 739
        // and 820 us in the order of the experts, 710 and 711 so).
        const uint32_t t = spread(blockIdx.x, gridDim.x, kRun), per = tiles_m * tiles_n, nth = t / per;
        const uint32_t e = min(static_cast<uint32_t>(a.by_size[nth]), static_cast<uint32_t>(a.E - 1));
        strip_of(t - nth * per, tiles_m, tiles_n, kGroupStrip, tm, tn);
        rows_of(a.offsets, static_cast<int>(e), a.P, first, rows);
        first = __builtin_amdgcn_readfirstlane(first), rows = __builtin_amdgcn_readfirstlane(rows);
        in.x = from(a.x, KIND == kGroupDwTokensY ? first * a.x.ld : 0);
        in.y = from(a.y, KIND == kGroupDwTokensY ? 0 : first * a.y.ld);
        in.out = e * a.expert_stride;
    } else {
        Group g;
        if (!find_group<TM>(a.offsets, a.E, a.P, tiles_n, kRun, g)) return false;
        first = g.first, rows = g.rows;
        strip_of(g.tile, (rows + TM - 1) / TM, tiles_n, kGroupStrip, tm, tn);
        constexpr bool kSorted = KIND == kOverGroups + kGemmDown || KIND == kOverGroups + kGemmDx;
        in.x = from(a.x, kSorted ? first * a.x.ld : 0);
        in.y = from(a.y, g.expert * a.expert_stride);
        in.out = 0;
    }
    in.rows = rows, in.row0 = first;
    tokens = {a.order + first, static_cast<uint32_t>(a.P), a.top};
    return true;
}

// The products of routed experts (`kind`: one over groups).  Of a few tokens, the
// second one goes to `part`, [splits][P][N] fp32, not weighted.
template <int DT>
void launch_grouped(int kind, const GroupArgs& a, int products, hipStream_t st);
template <int DT>
void launch_grouped_few(int kind, const GroupArgs& a, hipStream_t st);

extern template void launch_grouped<IABN_F32>(int, const GroupArgs&, int, hipStream_t);
extern template void launch_grouped<IABN_F16>(int, const GroupArgs&, int, hipStream_t);
extern template void launch_grouped<IABN_BF16>(int, const GroupArgs&, int, hipStream_t);
extern template void launch_grouped_few<IABN_F32>(int, const GroupArgs&, hipStream_t);
extern template void launch_grouped_few<IABN_F16>(int, const GroupArgs&, hipStream_t);
extern template void launch_grouped_few<IABN_BF16>(int, const GroupArgs&, hipStream_t);

// The tile of a grouped product.
TileSize plan_grouped(int dtype, GemmKind kind, bool direct, int64_t P, int64_t E, int64_t M, int64_t N, int64_t K,
                      int products);

// Whether the forward takes the few tokens' kernels, over how many blocks their
// second product's sum is split.
bool few_pairs(int64_t M);
int plan_grouped_few(int64_t P, int64_t E, int64_t N, int64_t K, int dtype);

// y_t = sum over the slots s of the terms of its pairs' rows (place[t*k + s]),
// weighted where `weights` is not null: [splits][P][C] of fp32 then, else [P][C]
// as store_terms leaves them.
struct CombineArgs {
    const void *terms, *low;
    const int32_t* place;
    const float* weights;
    void* y;
    int64_t M, C;
    int32_t k, P, splits;
};
void launch_combine(int dtype, const CombineArgs& a, hipStream_t st);

// dweights[i] = sum of the n dots of pair i's row, 0 where it has none.
void launch_dots(const float* dots, const int32_t* place, float* dweights, int64_t P, int64_t n, hipStream_t st);

}  // namespace iabn_impl
