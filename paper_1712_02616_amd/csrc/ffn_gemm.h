// The block's matrix products on the matrix cores: tiles of TM x TN outputs,
// K in steps of 128 bytes per row, both operands staged through LDS.
//
// A block's waves each own WM x WN outputs in 16x16 accumulators (fp32).  The
// operand with the n index (the weights, mostly) takes the first place of the
// matrix instruction, so that a lane's 4 results are consecutive in n, which
// is how every output is stored.
//
// The fragment of an instruction is 16 bytes per lane whatever the type: 8
// 16-bit elements, one 16x16x32 instruction; or 4 fp32, four 16x16x4
// instructions, whose k indices are those that the lanes hold (any order of
// the sum over k will do, the same for both operands).
#pragma once

#include "ffn.h"

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

constexpr int kRowBytes = 128;  // of K per LDS row (k contiguous)
constexpr int kSteps = 2;       // fragments of 64 bytes of K in it
// kGemmUp's tile: a wave's span of n holds the gate's columns in its first
// half and the same columns of the up projection in its second.
constexpr int kSpan = 64;

// 16 bytes of consecutive elements at element alignment; those past the
// first n are zero and not read.
template <int DT>
__device__ __forceinline__ u32x4 load16(const typename Elem<DT>::T* p, int64_t n) {
    using T = typename Elem<DT>::T;
    constexpr int E = 16 / sizeof(T);
    typedef T vec __attribute__((ext_vector_type(E)));
    typedef T mem __attribute__((ext_vector_type(E), aligned(sizeof(T))));
    if (n >= E) return __builtin_bit_cast(u32x4, static_cast<vec>(*reinterpret_cast<const mem*>(p)));
    vec v = {};
#pragma unroll
    for (int j = 0; j < E; ++j)
        if (j < n) v[j] = p[j];
    return __builtin_bit_cast(u32x4, v);
}

// One operand's tile of ROWS x 128 bytes of K: from memory to registers, to
// LDS, and fragments from there.  KS: k strided in memory (and in LDS, where
// the transposing read turns it).
//
// LDS, k contiguous: a row's eight 16-byte chunks are permuted by the row, so
// that the 16 rows that one read takes fall on all 64 banks.  k strided: a
// row is one k; 32-byte chunks (fp32: 64) are permuted so that the k that one
// read takes fall on different banks.
template <int DT, bool KS, int ROWS, int THREADS, bool DUAL>
struct Stage {
    using T = typename Elem<DT>::T;
    static constexpr int E = 16 / sizeof(T);
    static constexpr int BK = kRowBytes / sizeof(T);
    static constexpr int kBytes = ROWS * kRowBytes;
    static constexpr int kLoads = kBytes / 16 / THREADS;
    static constexpr int kPerRow = KS ? ROWS / E : 8;  // 16-byte chunks of a row of memory
    static_assert(kLoads * 16 * THREADS == kBytes, "a tile is whole accesses");

    u32x4 r[kLoads];

    static __device__ __forceinline__ uint32_t swizzle(int k) {
        return DT == IABN_F32 ? (k >> 2) & 3 : ((k >> 1) & 4) | (k & 3);
    }

    // rows: how many of the operand's rows there are from row0 on.
    __device__ __forceinline__ void load(const Operand& o, int seg, int64_t row0, int64_t rows,
                                         int64_t k0, int64_t K) {
#pragma unroll
        for (int i = 0; i < kLoads; ++i) {
            const int idx = threadIdx.x + i * THREADS, line = idx / kPerRow, c = idx % kPerRow;
            if constexpr (KS) {
                const T* p = static_cast<const T*>(o.p[seg]) + (k0 + line) * o.ld + row0 + c * E;
                r[i] = load16<DT>(p, k0 + line < K ? rows - c * E : 0);
            } else {
                int row = line;
                if constexpr (DUAL) {
                    seg = line % kSpan / (kSpan / 2);
                    row = line / kSpan * (kSpan / 2) + line % (kSpan / 2);
                }
                const T* p = static_cast<const T*>(o.p[seg]) + (row0 + row) * o.ld + k0 + c * E;
                r[i] = load16<DT>(p, row < rows ? K - k0 - c * E : 0);
            }
        }
    }

    __device__ __forceinline__ void store(char* lds) const {
#pragma unroll
        for (int i = 0; i < kLoads; ++i) {
            const int idx = threadIdx.x + i * THREADS, line = idx / kPerRow, c = idx % kPerRow;
            uint32_t at;
            if constexpr (!KS)
                at = line * kRowBytes + ((c ^ ((line >> 1) & 7)) << 4);
            else if constexpr (DT == IABN_F32)
                at = line * ROWS * 4 + (((c >> 2) ^ swizzle(line)) << 6) + ((c & 3) << 4);
            else
                at = line * ROWS * 2 + (((c >> 1) ^ swizzle(line)) << 5) + ((c & 1) << 4);
            *reinterpret_cast<u32x4*>(lds + at) = r[i];
        }
    }

    // The fragment of rows row..row+15 for step s.
    static __device__ __forceinline__ u32x4 frag(const char* lds, int row, int s) {
        const int i = lane_id() & 15, g = lane_id() >> 4;
        if constexpr (!KS) {
            const int line = row + i;
            return *reinterpret_cast<const u32x4*>(
                lds + line * kRowBytes + (((s * 4 + g) ^ ((line >> 1) & 7)) << 4));
        } else if constexpr (DT == IABN_F32) {
            f32x4 v;
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const int k = 16 * s + 4 * g + j;
                v[j] = *reinterpret_cast<const float*>(lds + k * ROWS * 4 +
                                                       (((row >> 4) ^ swizzle(k)) << 6) + i * 4);
            }
            return __builtin_bit_cast(u32x4, v);
        } else {
            // A transposing read: of 16 lanes, lane i gives the address of 4
            // columns of row k = i/4 and gets column i of the 4 rows.
            typedef short s16x4 __attribute__((ext_vector_type(4)));
            typedef s16x4 __attribute__((address_space(3))) lds_t;
            s16x4 half[2];
#pragma unroll
            for (int j = 0; j < 2; ++j) {
                const int k = 32 * s + 8 * g + 4 * j + (i >> 2);
                const char* at = lds + k * ROWS * 2 + (((row >> 4) ^ swizzle(k)) << 5) + ((i & 3) << 3);
                half[j] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_t*)(at));
            }
            return __builtin_bit_cast(
                u32x4, __builtin_shufflevector(half[0], half[1], 0, 1, 2, 3, 4, 5, 6, 7));
        }
    }
};

// 4 consecutive elements, of which n are inside.
template <int DT>
__device__ __forceinline__ void store4(void* base, int64_t at, int64_t n, const f32x4& v) {
    using T = typename Elem<DT>::T;
    typedef T vec __attribute__((ext_vector_type(4)));
    typedef T mem __attribute__((ext_vector_type(4), aligned(sizeof(T))));
    T* p = static_cast<T*>(base) + at;
    const vec w = __builtin_convertvector(v, vec);
    if (n >= 4) {
        *reinterpret_cast<mem*>(p) = w;
    } else {
#pragma unroll
        for (int j = 0; j < 4; ++j)
            if (j < n) p[j] = w[j];
    }
}

template <int DT>
__device__ __forceinline__ f32x4 load4(const void* base, int64_t at, int64_t n) {
    using T = typename Elem<DT>::T;
    typedef T vec __attribute__((ext_vector_type(4)));
    typedef T mem __attribute__((ext_vector_type(4), aligned(sizeof(T))));
    const T* p = static_cast<const T*>(base) + at;
    vec v = {};
    if (n >= 4) {
        v = *reinterpret_cast<const mem*>(p);
    } else {
#pragma unroll
        for (int j = 0; j < 4; ++j)
            if (j < n) v[j] = p[j];
    }
    return __builtin_convertvector(v, f32x4);
}

template <int KIND>
struct KindOf {
    static constexpr bool kDual = KIND == kGemmUp;
    static constexpr bool kXStrided = KIND == kGemmDw;
    static constexpr bool kYStrided = KIND == kGemmDh || KIND == kGemmDx || KIND == kGemmDw;
    static constexpr int kSegs = KIND == kGemmDx ? 2 : 1;  // products that add up
};

template <int DT, int KIND, int TM, int TN, int WAVES_M, int WAVES_N>
__global__ __launch_bounds__(WAVES_M* WAVES_N* kWave) void gemm_kernel(GemmArgs a, int tiles_m,
                                                                        int tiles_n) {
    using Kind = KindOf<KIND>;
    constexpr int kT = WAVES_M * WAVES_N * kWave;
    constexpr int WM = TM / WAVES_M, WN = TN / WAVES_N, NM = WM / 16, NN = WN / 16;
    static_assert(!Kind::kDual || WN == kSpan, "a wave holds both projections of its columns");
    using SX = Stage<DT, Kind::kXStrided, TM, kT, false>;
    using SY = Stage<DT, Kind::kYStrided, TN, kT, Kind::kDual>;
    constexpr int BK = SX::BK;
    __shared__ __align__(16) char lds[2][SX::kBytes + SY::kBytes];

    const int tile = blockIdx.x;
    const int64_t m0 = int64_t(tile % tiles_m) * TM;
    constexpr int kCols = Kind::kDual ? TN / 2 : TN;  // columns of the output
    const int64_t n0 = int64_t(tile / tiles_m) * kCols;
    const int z = blockIdx.z;
    const int wave = threadIdx.x / kWave, wm = wave / WAVES_N * WM, wn = wave % WAVES_N * WN;

    f32x4 acc[NM][NN] = {};
    SX sx;
    SY sy;
    const int64_t per_seg = (a.K + BK - 1) / BK, tiles_k = per_seg * Kind::kSegs;
    const auto load = [&](int64_t kt) {
        const int seg = Kind::kSegs > 1 ? (kt >= per_seg ? 1 : 0) : z;
        const int64_t k0 = (Kind::kSegs > 1 && seg ? kt - per_seg : kt) * BK;
        sx.load(a.x, seg, m0, a.M - m0, k0, a.K);
        sy.load(a.y, seg, n0, a.N - n0, k0, a.K);
    };
    if (tiles_k > 0) {
        load(0);
        sx.store(lds[0]);
        sy.store(lds[0] + SX::kBytes);
    }
    __syncthreads();
    for (int64_t kt = 0; kt < tiles_k; ++kt) {
        const char* const cur = lds[kt & 1];
        if (kt + 1 < tiles_k) load(kt + 1);
#pragma unroll
        for (int s = 0; s < kSteps; ++s) {
            u32x4 fy[NN];
#pragma unroll
            for (int j = 0; j < NN; ++j) fy[j] = SY::frag(cur + SX::kBytes, wn + j * 16, s);
#pragma unroll
            for (int i = 0; i < NM; ++i) {
                const u32x4 fx = SX::frag(cur, wm + i * 16, s);
#pragma unroll
                for (int j = 0; j < NN; ++j) acc[i][j] = Mma<DT>::run(fy[j], fx, acc[i][j]);
            }
        }
        if (kt + 1 < tiles_k) {
            char* const next = lds[(kt + 1) & 1];
            sx.store(next);
            sy.store(next + SX::kBytes);
        }
        __syncthreads();
    }

    // A lane holds row m and 4 consecutive n of every accumulator.
    const int lm = lane_id() & 15, ln = (lane_id() >> 4) * 4;
#pragma unroll
    for (int i = 0; i < NM; ++i) {
        const int64_t m = m0 + wm + i * 16 + lm;
        if (m >= a.M) continue;
        if constexpr (KIND == kGemmUp) {
#pragma unroll
            for (int j = 0; j < NN / 2; ++j) {
                const int64_t n = n0 + wn / 2 + j * 16 + ln, left = a.N - n, at = m * a.N + n;
                if (left <= 0) continue;
                const f32x4 g = acc[i][j], u = acc[i][j + NN / 2];
                f32x4 h;
#pragma unroll
                for (int q = 0; q < 4; ++q) {
                    float v, d;
                    activate(a.act, a.slope, g[q], v, d);
                    h[q] = v * u[q];
                }
                store4<DT>(a.out[0], at, left, h);
                if (a.dg) {
                    store4<DT>(a.dg, at, left, g);
                    store4<DT>(a.du, at, left, u);
                }
            }
        } else {
#pragma unroll
            for (int j = 0; j < NN; ++j) {
                const int64_t n = n0 + wn + j * 16 + ln, left = a.N - n, at = m * a.N + n;
                if (left <= 0) continue;
                if constexpr (KIND == kGemmDh) {
                    const f32x4 g = load4<DT>(a.g, at, left), u = load4<DT>(a.u, at, left);
                    f32x4 dg, du, h;
#pragma unroll
                    for (int q = 0; q < 4; ++q) {
                        float v, d;
                        activate(a.act, a.slope, g[q], v, d);
                        dg[q] = acc[i][j][q] * u[q] * d;
                        du[q] = acc[i][j][q] * v;
                        h[q] = v * u[q];
                    }
                    store4<DT>(a.dg, at, left, dg);
                    store4<DT>(a.du, at, left, du);
                    store4<DT>(a.out[0], at, left, h);
                } else {
                    store4<DT>(a.out[z], at, left, acc[i][j]);
                }
            }
        }
    }
}

template <int DT, int KIND, int TM, int TN, int WAVES_M, int WAVES_N>
void launch_tiles(const GemmArgs& a, int products, hipStream_t st) {
    constexpr int kCols = KindOf<KIND>::kDual ? TN / 2 : TN;
    const int64_t tm = (a.M + TM - 1) / TM, tn = (a.N + kCols - 1) / kCols;
    gemm_kernel<DT, KIND, TM, TN, WAVES_M, WAVES_N>
        <<<dim3(static_cast<uint32_t>(tm * tn), 1, products), WAVES_M * WAVES_N * kWave, 0, st>>>(
            a, static_cast<int>(tm), static_cast<int>(tn));
}

// Tiles of 256x256 where there are enough of them for every CU, else of 128x128.
template <int DT, int KIND>
void launch_kind(const GemmArgs& a, int products, hipStream_t st) {
    constexpr int kCols = KindOf<KIND>::kDual ? 128 : 256;
    const int64_t big = (a.M + 255) / 256 * ((a.N + kCols - 1) / kCols) * products;
    if (big >= 192) launch_tiles<DT, KIND, 256, 256, 2, 4>(a, products, st);
    else launch_tiles<DT, KIND, 128, 128, 2, 2>(a, products, st);
}

template <int DT>
bool launch_gemm(GemmKind kind, const GemmArgs& a, int products, hipStream_t st) {
    switch (kind) {
        case kGemmUp: launch_kind<DT, kGemmUp>(a, products, st); return true;
        case kGemmDown: launch_kind<DT, kGemmDown>(a, products, st); return true;
        case kGemmDh: launch_kind<DT, kGemmDh>(a, products, st); return true;
        case kGemmDx: launch_kind<DT, kGemmDx>(a, products, st); return true;
        case kGemmDw: launch_kind<DT, kGemmDw>(a, products, st); return true;
    }
    return false;
}

}  // namespace iabn_impl
