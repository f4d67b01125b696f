// The block's matrix products on the matrix cores: tiles of TM x TN outputs,
// K in steps of 128 bytes per row, both operands staged through two LDS
// buffers: while the waves multiply out of one, the next step's tiles arrive
// in the other.  Operands whose addresses are whole dwords go straight from
// memory to LDS (DMA); others, and a last step that K does not fill, go through
// registers, which hold zeros for what is not there.
//
// A block's waves each own WM x WN outputs in 16x16 accumulators (fp32).  The
// operand with the n index (the weights, mostly) takes the first place of the
// matrix instruction, so that a lane's 4 results are consecutive in n, which
// is how every output is stored.
//
// Bound by the matrix cores at the clock that their power leaves, which falls in
// a long run of products (random values; the fastest of 20 passes and the
// median; a large library product 1.39-1.61 PFLOP/s NT, 1.2-1.37 NN, 1.05-1.16
// TN).  bf16: dx (8192, 2x10240 -> 4096) 1.000 and 1.027 ms, 1.37 and 1.34
// PFLOP/s; both projections (4096, 2048 -> 2x8192) 239 and 274 us, 1.15 and 1.00
// (200 MB of results leave in that time, of which a 256x256 tile, alone on its
// CU, hides none); the weights' gradients over 8192 tokens 1.36 and 1.32 (gate
// and up), 1.08 and 1.02 (down); dh with the gating's gradient (8192, 4096 ->
// 10240) 633 and 643 us, 1.09 and 1.07 (840 MB in its epilogue); the down
// projection (4096, 8192 -> 2048) 110 and 119 us, 1.25 and 1.15.  fp32, the sizes
// of that forward: 1.94 and 0.95 ms, 141 and 144 TFLOP/s (the library 153).
#pragma once

#include "groups.h"
#include "mma.h"

namespace iabn_impl {

constexpr int kRowBytes = 128;  // of K per LDS row (k contiguous)
constexpr int kSteps = 2;       // fragments of 64 bytes of K in it
// kGemmUp's tile: a wave's span of n holds the gate's columns in its first
// half and the same columns of the up projection in its second.
constexpr int kSpan = 64;

// One operand's tile of ROWS x 128 bytes of K: from memory to LDS, and
// fragments from there.  KS: k strided in memory (and in LDS, where the
// transposing read turns it).
//
// The tile's 16-byte chunks lie in LDS in the order of the threads that bring
// them, THREADS chunks at a time; which chunk of the line a thread brings is
// permuted.  k contiguous: a line is a row, its eight chunks are permuted by
// the row, so that the 16 rows that one read takes fall on all 64 banks.  k
// strided: a line is one k; 32-byte pairs of chunks (fp32: 64-byte fours) are
// permuted so that the k that one read takes fall on different banks.
//
// GATHER: the operand's rows (k strided: its k) are tokens, in the order of a plan
// (groups.h).
template <int DT, bool KS, int ROWS, int THREADS, bool DUAL, bool GATHER = false>
struct Stage {
    using T = typename Elem<DT>::T;
    static constexpr int E = 16 / sizeof(T);
    static constexpr int BK = kRowBytes / sizeof(T);
    static constexpr int kBytes = ROWS * kRowBytes;
    static constexpr int kLoads = kBytes / 16 / THREADS;
    static constexpr int kPerLine = KS ? ROWS / E : 8;  // chunks
    static_assert(kLoads * 16 * THREADS == kBytes, "a tile is whole accesses");
    // A thread's chunks stand at one place of lines that are this far apart.
    static constexpr int kLineStep = THREADS / kPerLine;
    static_assert(THREADS % kPerLine == 0, "");

    static __device__ __forceinline__ uint32_t swizzle(int line) {
        if constexpr (!KS) return (line >> 1) & 7;
        else if constexpr (DT == IABN_F32) return (line >> 2) & (ROWS == 32 ? 1 : 3);
        // (Lines of 64 elements are half a round of the banks, of 32 a quarter.)
        else if constexpr (ROWS == 32) return (line >> 3) & 1;
        else if constexpr (ROWS == 64) return ((line >> 2) & 2) | ((line >> 1) & 1);
        else return ((line >> 1) & 4) | (line & 3);
    }
    static __device__ __forceinline__ int first_line() { return threadIdx.x / kPerLine; }
    // The chunk of its i-th line that this thread brings (the same one of each
    // where the permutation does not tell lines that are a step apart).
    static __device__ __forceinline__ int chunk(int i) {
        constexpr int kGroup = !KS ? 1 : DT == IABN_F32 ? 4 : 2;
        const int line = first_line() + (kLineStep % 16 == 0 ? 0 : i * kLineStep);
        return static_cast<int>((threadIdx.x % kPerLine) ^ (swizzle(line) * kGroup));
    }
    // The matrix and the row in it of a line (k contiguous).
    static __device__ __forceinline__ int row_of(int line) {
        return DUAL ? line / kSpan * (kSpan / 2) + line % (kSpan / 2) : line;
    }
    static __device__ __forceinline__ int matrix_of(int line, int seg) {
        return DUAL ? line % kSpan / (kSpan / 2) : seg;
    }

    // Through registers.  rows: how many of the operand's rows there are from
    // row0 on.
    u32x4 r[kLoads];
    template <typename Op>
    __device__ __forceinline__ void load(const Op& o, int seg, int64_t row0, int64_t rows,
                                         int64_t k0, int64_t K, const Tokens& tokens = {}) {
#pragma unroll
        for (int i = 0; i < kLoads; ++i) {
            const int line = first_line() + i * kLineStep, c = chunk(i) * E;
            const T* p = static_cast<const T*>(matrix(o, KS ? seg : matrix_of(line, seg)));
            if constexpr (KS && GATHER)
                r[i] = load16_first<DT>(p + tokens(min(k0 + line, K - 1)) * o.ld + row0 + c,
                                        k0 + line < K ? rows - c : 0);
            else if constexpr (GATHER)
                r[i] = load16_first<DT>(p + tokens(row0 + min(int64_t(row_of(line)), rows - 1)) * o.ld + k0 + c,
                                        row_of(line) < rows ? K - k0 - c : 0);
            else if constexpr (KS)
                r[i] = load16_first<DT>(p + (k0 + line) * o.ld + row0 + c, k0 + line < K ? rows - c : 0);
            else
                r[i] = load16_first<DT>(p + (row0 + row_of(line)) * o.ld + k0 + c,
                                  row_of(line) < rows ? K - k0 - c : 0);
        }
    }
    __device__ __forceinline__ void store(char* lds) const {
#pragma unroll
        for (int i = 0; i < kLoads; ++i)
            *reinterpret_cast<u32x4*>(lds + (threadIdx.x + i * THREADS) * 16) = r[i];
    }

    // Straight to LDS, a whole step of K.  Rows past the operand's read its
    // last ones (the results that they go into are not stored).
    uint64_t base[2];      // the tile's first element of each matrix
    uint32_t off[kLoads];  // bytes from the step's first element
    // (k strided, GATHER: the next step's entries of the plan.)
    uint32_t entry[KS && GATHER ? kLoads : 1];
    template <typename Op>
    __device__ __forceinline__ void prepare(const Op& o, int64_t row0, int64_t rows, const Tokens& tokens = {}) {
#pragma unroll
        for (int q = 0; q < 2; ++q) {
            // (Kept in scalar registers, not loaded from the arguments at each step.)
            const uint64_t p = reinterpret_cast<uint64_t>(static_cast<const T*>(matrix(o, q)) +
                                                          (KS ? row0 : GATHER ? 0 : row0 * o.ld));
            base[q] = static_cast<uint32_t>(__builtin_amdgcn_readfirstlane(static_cast<int>(p))) |
                      uint64_t(static_cast<uint32_t>(__builtin_amdgcn_readfirstlane(static_cast<int>(p >> 32)))) << 32;
        }
#pragma unroll
        for (int i = 0; i < kLoads; ++i) {
            const int line = first_line() + i * kLineStep, c = chunk(i) * E;
            if constexpr (KS && GATHER) {
                off[i] = static_cast<uint32_t>((c < rows ? c : 0) * sizeof(T));
            } else if constexpr (KS) {
                off[i] = static_cast<uint32_t>((line * o.ld + (c < rows ? c : 0)) * sizeof(T));
            } else if constexpr (GATHER) {
                const int64_t row = min(static_cast<int64_t>(row_of(line)), rows - 1);
                off[i] = static_cast<uint32_t>((tokens(row0 + row) * o.ld + c) * sizeof(T));
            } else {
                const int64_t row = min(static_cast<int64_t>(row_of(line)), rows - 1);
                off[i] = static_cast<uint32_t>((row * o.ld + c) * sizeof(T));
            }
        }
    }
    // GATHER with k strided: the entries that the step at k0 takes, a step ahead of its fetch.
    __device__ __forceinline__ void look_up(int64_t k0, int64_t K, const Tokens& tokens) {
        if constexpr (KS && GATHER)
#pragma unroll
            for (int i = 0; i < kLoads; ++i)
                entry[i] = tokens.order[min(k0 + first_line() + i * kLineStep, K - 1)];
    }
    // K >= 0: lines of k from there on (strided) are fetched as zeros, by offsets that
    // lie outside of the buffer (row0: the tile's first column).
    static constexpr uint32_t kOutside = 0xfffff000;
    template <int FROM, int TO, typename Op>
    __device__ __forceinline__ void fetch(const Op& o, int seg, int64_t k0, char* lds, const Tokens& tokens,
                                          int64_t K, int64_t row0) const {
#if defined(__HIP_DEVICE_COMPILE__)  // (the host's pass does not know the buffer types)
        typedef __attribute__((address_space(3))) void lds_t;
        const uint64_t at = KS && GATHER ? 0 : (KS ? k0 * o.ld : k0) * sizeof(T);
        const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
        uint32_t bytes = 0xffffffff;
        if (KS && K >= 0) {
            const uint64_t left = static_cast<uint64_t>(((K - k0) * o.ld - row0) * static_cast<int64_t>(sizeof(T)));
            bytes = GATHER || left > kOutside ? kOutside : static_cast<uint32_t>(left);
        }
#pragma unroll
        for (int i = FROM; i < TO; ++i) {
            // (A wave's lines are of one matrix: a wave covers 8 lines or fewer.)
            const int which =
                DUAL ? __builtin_amdgcn_readfirstlane(matrix_of(first_line() + i * kLineStep, seg)) : seg;
            const __amdgpu_buffer_rsrc_t rsrc = __builtin_amdgcn_make_buffer_rsrc(
                reinterpret_cast<void*>((which ? base[1] : base[0]) + at), 0, static_cast<int>(bytes), 0x00027000);
            uint32_t from = off[i];
            if constexpr (KS && GATHER) {
                from += tokens.of(entry[i]) * static_cast<uint32_t>(o.ld * static_cast<int64_t>(sizeof(T)));
                if (K >= 0 && k0 + first_line() + i * kLineStep >= K) from = kOutside;
            }
            __builtin_amdgcn_raw_ptr_buffer_load_lds(
                rsrc, (lds_t*)(lds + (wave * kWave + (i - FROM) * THREADS) * 16), 16, from, 0, 0, 0);
        }
#endif
    }

    // The fragment of rows row..row+15 for step s.
    static __device__ __forceinline__ u32x4 frag(const char* lds, int row, int s) {
        const int i = lane_id() & 15, g = lane_id() >> 4;
        if constexpr (!KS) {
            const int line = row + i;
            return *reinterpret_cast<const u32x4*>(
                lds + line * kRowBytes + (((s * 4 + g) ^ swizzle(line)) << 4));
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

template <int KIND>
struct KindOf {
    static constexpr bool kGroups = KIND >= kOverGroups;
    static constexpr GemmKind kBase = static_cast<GemmKind>(
        !kGroups ? KIND : KIND == kGroupDwTokensY ? static_cast<int>(kGemmDw) : KIND - kOverGroups);
    static constexpr bool kDual = kBase == kGemmUp;
    static constexpr bool kXStrided = kBase == kGemmDw;
    static constexpr bool kYStrided = kBase == kGemmDh || kBase == kGemmDx || kBase == kGemmDw;
    static constexpr int kSegs = kBase == kGemmDx ? 2 : 1;  // products that add up
    // The operand whose rows (strided: k) are tokens.
    static constexpr bool kGatherY = KIND == kGroupDwTokensY;
    static constexpr bool kGatherX = kGroups && !kGatherY && kBase != kGemmDown && kBase != kGemmDx;
};

// The tile of a block.  The hardware hands consecutive blocks to the XCDs in
// turn; each XCD takes a contiguous range of tiles, in strips of kStrip tiles
// of m, so that the tiles that run on it at one time share rows of both
// operands in its L2.
constexpr int kStrip = 8;
__device__ __forceinline__ void tile_of(int tiles_m, int tiles_n, int& tm, int& tn) {
    const uint32_t n = gridDim.x, x = blockIdx.x % kXcds, j = blockIdx.x / kXcds;
    const uint32_t t = x * (n / kXcds) + min(x, n % kXcds) + j;
    const uint32_t strip = t / (kStrip * tiles_n), in = t - strip * (kStrip * tiles_n);
    const uint32_t height = min(static_cast<uint32_t>(kStrip), tiles_m - strip * kStrip);
    tn = static_cast<int>(in / height);
    tm = static_cast<int>(strip * kStrip + in % height);
}

// KIND: a GemmKind, or one of the kinds over groups of rows (groups.h).
template <int DT, int KIND, int TM, int TN, int WAVES_M, int WAVES_N, bool DMA>
__global__ __launch_bounds__(WAVES_M* WAVES_N* kWave) void gemm_kernel(ArgsOf<KIND> a, int tiles_m,
                                                                        int tiles_n) {
    using Kind = KindOf<KIND>;
    constexpr bool kGroups = Kind::kGroups;
    constexpr GemmKind kBase = Kind::kBase;
    constexpr int kT = WAVES_M * WAVES_N * kWave;
    constexpr int WM = TM / WAVES_M, WN = TN / WAVES_N, NM = WM / 16, NN = WN / 16;
    static_assert(!Kind::kDual || WN == kSpan, "a wave holds both projections of its columns");
    using SX = Stage<DT, Kind::kXStrided, TM, kT, false, Kind::kGatherX>;
    using SY = Stage<DT, Kind::kYStrided, TN, kT, Kind::kDual, Kind::kGatherY>;
    constexpr int BK = SX::BK;
    // Two buffers, of which one is multiplied while the other fills.
    constexpr int kBuffer = SX::kBytes + SY::kBytes;
    __shared__ __align__(16) char lds[2 * kBuffer];
    char *const lds0 = lds, *const lds1 = lds + kBuffer;

    int tm, tn;
    Tokens tokens = {};
    Entered group = {};
    if constexpr (kGroups) {
        if (!enter_group<DT, KIND, TM>(a, tiles_m, tiles_n, tm, tn, group, tokens)) return;
        (kBase == kGemmDw ? a.K : a.M) = group.rows;
    } else {
        tile_of(tiles_m, tiles_n, tm, tn);
    }
    const auto operand = [](const auto& whole, const auto& own) -> const auto& {
        if constexpr (kGroups) return own;
        else return whole;
    };
    const auto &x = operand(a.x, group.x), &y = operand(a.y, group.y);
    const int64_t m0 = int64_t(tm) * TM;
    constexpr int kCols = Kind::kDual ? TN / 2 : TN;  // columns of the output
    const int64_t n0 = int64_t(tn) * kCols;
    const int z = blockIdx.z;
    const int wave = threadIdx.x / kWave, wm = wave / WAVES_N * WM, wn = wave % WAVES_N * WN;

    f32x4 acc[NM][NN] = {};
    SX sx;
    SY sy;
    // A step goes in phases, each of one half of K and (in the largest tile) one
    // half of a wave's rows of x: its fragments, and their products.
    constexpr bool kAhead = NM * NN > 16;
    constexpr int kHalves = kAhead ? 2 : 1, kPhases = kSteps * kHalves, NH = NM / kHalves;
    // The largest tile over groups: the last one of an expert's rows often holds no
    // more than half of them.  Every wave then has rows of both halves of the tile,
    // so that the phases of the empty half are left out (32768 pairs of 64 experts, up
    // projection: 328 us, 315 without them).
    constexpr bool kShort = kGroups && kBase != kGemmDw && kAhead;
    const auto acc_row = [&](int g) __attribute__((always_inline)) {  // of accumulators g
        return kShort ? g / NH * (TM / 2) + wave / WAVES_N * (WM / 2) + g % NH * 16 : wm + g * 16;
    };
    u32x4 fy[kSteps][NN], fx[2][NH];
    const auto read = [&](const char* __restrict__ buf, int phase) __attribute__((always_inline)) {
        const int s = phase / kHalves, h = phase % kHalves;
        if (h == 0)
#pragma unroll
            for (int j = 0; j < NN; ++j) fy[s][j] = SY::frag(buf + SX::kBytes, wn + j * 16, s);
#pragma unroll
        for (int i = 0; i < NH; ++i) fx[phase & 1][i] = SX::frag(buf, acc_row(h * NH + i), s);
    };
    const auto products = [&](int phase) __attribute__((always_inline)) {
        const int s = phase / kHalves, h = phase % kHalves;
#pragma unroll
        for (int i = 0; i < NH; ++i)
#pragma unroll
            for (int j = 0; j < NN; ++j)
                acc[h * NH + i][j] = Mma<DT>::run(fy[s][j], fx[phase & 1][i], acc[h * NH + i][j]);
    };
    // fp32 over groups: a long sum of parts, of kLong steps each, so that its roundings
    // grow with the number of parts and not with K: y of (1500, 2 of 8 experts, 1024 ->
    // 4096) is off by 5.2e-7 in root mean square and dx by 4.3e-7, 1.4e-6 and 1.7e-6 in
    // one sum, for at most 2% more time (up projection of (333, 2 of 7, 1000 -> 731) 41.3
    // -> 43.0 us).  (Not in dW, whose sums over an expert's rows are shorter, and which
    // would take 11% more.  As a loop in a loop 4 to 10% more.)
    constexpr bool kParts = kGroups && DT == IABN_F32 && kBase != kGemmDw;
    constexpr int kLong = 8;
    f32x4 parts[kParts ? NM : 1][kParts ? NN : 1] = {};
    const auto end_part = [&]() __attribute__((always_inline)) {
        if constexpr (kParts)
#pragma unroll
            for (int i = 0; i < NM; ++i)
#pragma unroll
                for (int j = 0; j < NN; ++j) parts[i][j] += acc[i][j], acc[i][j] = f32x4{};
    };
    // Steps of K: whole ones that go straight to LDS, those of the first
    // product and then those of the second, and the others, through
    // registers.  This block's share of them all: [lo, hi) and [from, to).
    // (A strided operand whose last chunk of a row reaches into the next one may
    // not fetch its last row.)
    constexpr int E = SX::E;
    const bool reaches = (Kind::kXStrided && a.M % E != 0) || (Kind::kYStrided && a.N % E != 0);
    // (dW over groups: its sums end anywhere.  Where nothing reaches, the last step is
    // fetched too, and its lines past the sum's end as zeros.)
    constexpr bool kFill = kGroups && kBase == kGemmDw;
    const int whole = !DMA ? 0 : static_cast<int>(kFill && !reaches ? (a.K + BK - 1) / BK : (a.K - (reaches ? 1 : 0)) / BK), steps = whole * Kind::kSegs;
    const int per_seg = static_cast<int>((a.K + BK - 1) / BK) - whole, rest = per_seg * Kind::kSegs;
    const int64_t all = steps + rest;
    const int begin = static_cast<int>(all * blockIdx.y / gridDim.y);
    const int end = static_cast<int>(all * (blockIdx.y + 1) / gridDim.y);
    const int lo = min(begin, steps), hi = min(end, steps);
    const int from = max(begin - steps, 0), to = max(end - steps, 0);
    if constexpr (DMA) {
        const auto seg_of = [&](int kt) { return Kind::kSegs > 1 ? (kt >= whole ? 1 : 0) : z; };
        const auto k_of = [&](int kt) { return int64_t(Kind::kSegs > 1 && kt >= whole ? kt - whole : kt) * BK; };
        const auto fetch = [&](int kt, char* buf) __attribute__((always_inline)) {
            const int seg = seg_of(kt);
            const int64_t k0 = k_of(kt);
            sx.template fetch<0, SX::kLoads>(x, seg, k0, buf, tokens, kFill ? a.K : -1, m0);
            sy.template fetch<0, SY::kLoads>(y, seg, k0, buf + SX::kBytes, tokens, kFill ? a.K : -1, n0);
            sx.look_up(k0 + BK, a.K, tokens);
            sy.look_up(k0 + BK, a.K, tokens);
        };
        // At `meet` what was fetched has arrived (each wave has waited for its
        // own) and the reads of the buffer to be filled next have ended.  The
        // largest tile, alone on its CU, goes in phases: the fragments of one
        // are read while the one before is multiplied (all reads of a step first
        // would spill: (4096, 2048 -> 2x8192) bf16 517 us instead of 280, the
        // products of two sums (8192, 2x10240 -> 4096) 3098 instead of 1020),
        // those of the next step's first phase while this one's last is, so that
        // products run on both sides of the barrier (237 us instead of 243 in a
        // first pass; nothing in a long run, where the clock has fallen).  Of the
        // smaller tiles two or more share a CU; there every read of a step before
        // its first product is better ((4096, 1024) fp16 weights' gradients of
        // 2085 tokens 37 us against 40).
        const auto meet = []() __attribute__((always_inline)) {
            __builtin_amdgcn_s_waitcnt(0x0070);  // vmcnt(0) lgkmcnt(0)
            asm volatile("" ::: "memory");
            __builtin_amdgcn_s_barrier();
            asm volatile("" ::: "memory");
        };
        const auto turn = [&](int kt, char* __restrict__ cur, char* __restrict__ next) __attribute__((always_inline)) {
            if constexpr (kAhead) {
#pragma unroll
                for (int p = 0; p + 1 < kPhases; ++p) {
                    read(cur, p + 1);
                    products(p);
                    __builtin_amdgcn_sched_barrier(0);  // (products stay on their side)
                }
                meet();
                if (kt + 2 < hi) fetch(kt + 2, cur);
                if (kt + 1 < hi) read(next, 0);
                products(kPhases - 1);
                __builtin_amdgcn_sched_barrier(0);
            } else {
                meet();
                if (kt + 1 < hi) fetch(kt + 1, next);
#pragma unroll
                for (int p = 0; p < kPhases; ++p) read(cur, p);
                __builtin_amdgcn_sched_barrier(0);
#pragma unroll
                for (int p = 0; p < kPhases; ++p) products(p);
            }
        };
        // (The buffers are told apart, restrict, so that the compiler does not
        // make the reads of one wait for what arrives in the other.)
        const auto round = [&](int kt, char* __restrict__ b0, char* __restrict__ b1) __attribute__((always_inline)) {
            turn(kt, b0, b1);
            if (kt + 1 < hi) turn(kt + 1, b1, b0);
        };
        sx.prepare(x, m0, a.M - m0, tokens);
        sy.prepare(y, n0, a.N - n0, tokens);
        if (kGroups && lo < hi) {
            sx.look_up(int64_t(lo) * BK, a.K, tokens);
            sy.look_up(int64_t(lo) * BK, a.K, tokens);
        }
        if constexpr (kShort) {
            // Over groups a step's tiles come from farther away (an expert's weights
            // serve few rows): its fetch is cut in two, and the first part of the
            // next but one starts as soon as it has been read, in the middle of a
            // step: X's first half of rows, and all of Y, whose fragments are held for
            // the second half.  (Up projection of 512 rows of each of 64 experts, 2048
            // -> 2x1024: 238 us instead of 254.  In dW, with parts by k: dy's 345 us
            // instead of 317.)
            constexpr int kXPart = SX::kLoads / 2, kXHalf = SX::kBytes / 2;
            const auto first_part = [&](int kt, char* x0, char* yb) __attribute__((always_inline)) {
                sx.template fetch<0, kXPart>(x, seg_of(kt), k_of(kt), x0, tokens, -1, m0);
                sy.template fetch<0, SY::kLoads>(y, seg_of(kt), k_of(kt), yb, tokens, -1, n0);
            };
            const auto second_part = [&](int kt, char* x1) __attribute__((always_inline)) {
                sx.template fetch<kXPart, SX::kLoads>(x, seg_of(kt), k_of(kt), x1, tokens, -1, m0);
            };
            // Phase p: half p/2 of X's rows (in xr), half p%2 of k.
            const auto take = [&](const char* __restrict__ xr, const char* __restrict__ yr, int p) __attribute__((always_inline)) {
                if (p < kSteps)
#pragma unroll
                    for (int j = 0; j < NN; ++j) fy[p][j] = SY::frag(yr, wn + j * 16, p);
#pragma unroll
                for (int i = 0; i < NH; ++i) fx[p & 1][i] = SX::frag(xr, acc_row(i), p % kSteps);
            };
            const auto multiply = [&](int p) __attribute__((always_inline)) {
                const int h = p / kSteps, k = p % kSteps;
#pragma unroll
                for (int i = 0; i < NH; ++i)
#pragma unroll
                    for (int j = 0; j < NN; ++j)
                        acc[h * NH + i][j] = Mma<DT>::run(fy[k][j], fx[p & 1][i], acc[h * NH + i][j]);
                __builtin_amdgcn_sched_barrier(0);  // (products stay on their side)
            };
            // All waves: their reads of LDS have ended, and all but their last `left`
            // fetches have arrived.
            const auto meet_but = [](auto left) __attribute__((always_inline)) {
                __builtin_amdgcn_s_waitcnt(0x0070 | (left & 15) | (left >> 4 << 14));
                asm volatile("" ::: "memory");
                __builtin_amdgcn_s_barrier();
                asm volatile("" ::: "memory");
            };
            using std::integral_constant;
            constexpr integral_constant<int, 63> kAny;
            constexpr integral_constant<int, kXPart + SY::kLoads> kFirst;
            constexpr integral_constant<int, SX::kLoads + SY::kLoads> kStepLoads;
            constexpr integral_constant<int, 0> kNone;
            // (The parts of both buffers are told apart as the buffers are above.)
            const auto split_turn = [&](int kt, char* __restrict__ x0, char* __restrict__ x1, char* __restrict__ yb,
                                        char* __restrict__ next_x, char* __restrict__ next_y,
                                        auto tall) __attribute__((always_inline)) {
                const bool more = kt + 2 < hi;
                take(x0, yb, 1);
                multiply(0);
                if constexpr (tall) {
                    meet_but(kAny);
                    if (more) first_part(kt + 2, x0, yb);
                    take(x1, yb, 2);
                    multiply(1);
                    take(x1, yb, 3);
                    multiply(2);
                    if (more) meet_but(kFirst);
                    else meet_but(kNone);
                    if (more) second_part(kt + 2, x1);
                } else {
                    meet_but(kNone);
                    if (more) first_part(kt + 2, x0, yb);
                }
                if (kt + 1 < hi) take(next_x, next_y, 0);
                multiply(tall ? 3 : 1);
            };
            const auto split_round = [&](int kt, char* __restrict__ x0, char* __restrict__ x1, char* __restrict__ ya,
                                         char* __restrict__ x2, char* __restrict__ x3, char* __restrict__ yb,
                                         auto tall) __attribute__((always_inline)) {
                split_turn(kt, x0, x1, ya, x2, yb, tall);
                if (kt + 1 < hi) split_turn(kt + 1, x2, x3, yb, x0, ya, tall);
            };
            const auto run = [&](auto tall) __attribute__((always_inline)) {
                char *const ya = lds0 + SX::kBytes, *const yb = lds1 + SX::kBytes;
                if (lo >= hi) return;
                first_part(lo, lds0, ya);
                if (tall) second_part(lo, lds0 + kXHalf);
                if (lo + 1 < hi) {
                    first_part(lo + 1, lds1, yb);
                    if (tall) second_part(lo + 1, lds1 + kXHalf);
                    if (tall) meet_but(kStepLoads);
                    else meet_but(kFirst);
                } else {
                    meet_but(kNone);
                }
                take(lds0, ya, 0);
                for (int kt = lo; kt < hi; kt += 2)
                    split_round(kt, lds0, lds0 + kXHalf, ya, lds1, lds1 + kXHalf, yb, tall);
            };
            if (a.M - m0 > TM / 2) run(std::true_type());
            else run(std::false_type());
        } else {
            if (lo < hi) fetch(lo, lds0);
            if (kAhead && lo < hi) {
                meet();
                if (lo + 1 < hi) fetch(lo + 1, lds1);
                read(lds0, 0);
            }
            for (int kt = lo; kt < hi; kt += 2) {
                round(kt, lds0, lds1);
                if (kParts && (kt - lo) % kLong == kLong - 2) end_part();
            }
        }
        __syncthreads();
    }
    if (from < to) {
        const auto load = [&](int kt) __attribute__((always_inline)) {
            const int seg = Kind::kSegs > 1 ? (kt >= per_seg ? 1 : 0) : z;
            const int64_t k0 = int64_t(whole + (Kind::kSegs > 1 && seg ? kt - per_seg : kt)) * BK;
            sx.load(x, seg, m0, a.M - m0, k0, a.K, tokens);
            sy.load(y, seg, n0, a.N - n0, k0, a.K, tokens);
        };
        const auto store = [&](char* buf) __attribute__((always_inline)) {
            sx.store(buf);
            sy.store(buf + SX::kBytes);
            __syncthreads();
        };
        const auto multiply = [&](const char* buf) __attribute__((always_inline)) {
#pragma unroll
            for (int p = 0; p < kPhases; ++p) {
                read(buf, p);
                products(p);
            }
        };
        load(from);
        store(lds0);
        for (int kt = from; kt < to; kt += 2) {
            if (kt + 1 < to) load(kt + 1);
            multiply(lds0);
            if (kt + 1 >= to) break;
            store(lds1);
            if (kt + 2 < to) load(kt + 2);
            multiply(lds1);
            if (kt + 2 < to) store(lds0);
            if (kParts && (kt - from) % kLong == kLong - 2) end_part();
        }
    }
    if constexpr (kParts)
#pragma unroll
        for (int i = 0; i < NM; ++i)
#pragma unroll
            for (int j = 0; j < NN; ++j) acc[i][j] += parts[i][j];

    // The results, through LDS: a lane holds a row and 4 consecutive columns of
    // each accumulator; it gets chunks of 8 columns, which it finishes and
    // stores as one access, 128 bytes of a row by 8 lanes.  Each wave has
    // kPass rows of 16 accumulators at a time in its own part.
    __syncthreads();
    constexpr int kPass = NM < 4 ? NM : 4, kPart = kPass * 16 * WN;
    static_assert(WAVES_M * WAVES_N * kPart * 4 <= 2 * kBuffer && NM % kPass == 0 && WN == 64, "");
    float* const part = reinterpret_cast<float*>(lds) + wave * kPart;
    const auto at = [](int row, int col) {  // 16-byte units permuted by the row
        return row * WN + (((col >> 2) ^ (row & 15)) << 2);
    };
    // A lane's c-th chunk of the rows of pass p.
    constexpr int kCh = (Kind::kDual ? WN / 2 : WN) / kChunk;  // chunks of a row
    constexpr int kTurns = kPass * 16 * kCh / kWave;
    static_assert(kTurns * kWave == kPass * 16 * kCh && (kBase != kGemmDh || kTurns % 2 == 0), "");
    struct Place {
        int row, col, inside;
        int64_t out, m;
    };
    const auto place = [&](int p, int c) {
        const int at_c = c * kWave + static_cast<int>(lane_id());
        Place r;
        r.row = at_c / kCh, r.col = at_c % kCh * kChunk;
        const int64_t m = m0 + (kShort ? acc_row(p + r.row / 16) + r.row % 16 : wm + p * 16 + r.row), n = n0 + (Kind::kDual ? wn / 2 : wn) + r.col;
        r.m = m;
        r.inside = m < a.M ? static_cast<int>(max(min(a.N - n, int64_t(kChunk)), int64_t(0))) : 0;
        r.out = kGroups ? (kBase == kGemmDw ? group.out : group.row0 * a.N) + m * a.N + n : m * a.N + n;
        return r;
    };
    // kGemmDh: g and u of the next chunks are on their way while one is finished.
    typedef typename ChunkOf<DT>::vec chunk_t;
    const auto load_gu = [&](int p, int c, chunk_t (&v)[2]) {
        const Place at_c = place(p, c);
        v[0] = load_chunk<DT, kStream>(a.g, at_c.out, at_c.inside);
        v[1] = load_chunk<DT, kStream>(a.u, at_c.out, at_c.inside);
    };
#pragma unroll
    for (int p = 0; p < NM; p += kPass) {
        if (kShort && m0 + acc_row(p) - acc_row(0) >= a.M) break;  // (a half that is empty)
        constexpr int kLook = kGroups && kTurns % 4 == 0 ? 4 : 2;
        chunk_t gu[kLook][2];
        if constexpr (kBase == kGemmDh)
#pragma unroll
            for (int q = 0; q < kLook; ++q) load_gu(p, q, gu[q]);
        const int lm = lane_id() & 15, ln = (lane_id() >> 4) * 4;
#pragma unroll
        for (int i = 0; i < kPass; ++i)
#pragma unroll
            for (int j = 0; j < NN; ++j)
                *reinterpret_cast<f32x4*>(part + at(i * 16 + lm, j * 16 + ln)) = acc[p + i][j];
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        __builtin_amdgcn_wave_barrier();
        const auto read = [&](int row, int col, float (&v)[kChunk]) {
            const f32x4 lo = *reinterpret_cast<const f32x4*>(part + at(row, col));
            const f32x4 hi = *reinterpret_cast<const f32x4*>(part + at(row, col + 4));
#pragma unroll
            for (int q = 0; q < 4; ++q) v[q] = lo[q], v[q + 4] = hi[q];
        };
        if constexpr (kBase == kGemmDh) {
#pragma unroll 1
            for (int c = 0; c < kTurns; c += kLook)
#pragma unroll
                for (int q = 0; q < kLook; ++q) {
                    const auto raw_g = gu[q][0], raw_u = gu[q][1];
                    const Place at_c = place(p, c + q);
                    if (c + q + kLook < kTurns) load_gu(p, c + q + kLook, gu[q]);
                    if (!kGroups && at_c.inside <= 0) continue;
                    float v[kChunk], g[kChunk], u[kChunk], dg[kChunk], du[kChunk], h[kChunk];
                    read(at_c.row, at_c.col, v);
                    widen<DT>(raw_g, g);
                    widen<DT>(raw_u, u);
                    if constexpr (kGroups) {
                        // The gradients of a pair's weight (the sum over the row of h and
                        // dy Wd, of which this is 64 columns') and of its projections.
                        const float w = pair_weight(a, tokens, at_c.m, a.M);
                        float dot = 0.0f;
                        gate_backward<DT>(a.act, a.slope, v, g, u, dg, du, h);
#pragma unroll
                        for (int j = 0; j < kChunk; ++j) {
                            if (j < at_c.inside) dot = fmaf(h[j], v[j], dot);
                            dg[j] *= w, du[j] *= w, h[j] *= w;
                        }
                        dot += dpp_f32<0xB1, 0xF>(dot);
                        dot += dpp_f32<0x4E, 0xF>(dot);
                        dot += dpp_f32<0x141, 0xF>(dot);
                        if (at_c.inside <= 0) continue;
                        if (at_c.col == 0)
                            a.dots[(group.row0 + at_c.m) * ((a.N + WN - 1) / WN) + (n0 + wn) / WN] = dot;
                    } else {
                        gate_backward<DT>(a.act, a.slope, v, g, u, dg, du, h);
                    }
                    store_chunk<DT, kCached>(a.dg, at_c.out, at_c.inside, dg);
                    store_chunk<DT, kCached>(a.du, at_c.out, at_c.inside, du);
                    store_chunk<DT, kCached>(a.out[0], at_c.out, at_c.inside, h);
                }
        } else {
#pragma unroll 1
            for (int c = 0; c < kTurns; ++c) {
                const Place at_c = place(p, c);
                if (at_c.inside <= 0) continue;
                float v[kChunk];
                read(at_c.row, at_c.col, v);
                if constexpr (kBase == kGemmUp) {
                    float u[kChunk], h[kChunk];
                    read(at_c.row, at_c.col + WN / 2, u);
                    gate_forward<DT>(a.act, a.slope, v, u, h);
                    store_chunk<DT, kCached>(a.out[0], at_c.out, at_c.inside, h);
                    if (a.dg) {
                        store_chunk<DT, kStream>(a.dg, at_c.out, at_c.inside, v);
                        store_chunk<DT, kStream>(a.du, at_c.out, at_c.inside, u);
                    }
                } else if (!kGroups && gridDim.y > 1) {
                    store_chunk<IABN_F32, kCached>(
                        a.part, (int64_t(blockIdx.y) * gridDim.z + z) * a.M * a.N + at_c.out, at_c.inside, v);
                } else {
                    if constexpr (kGroups && kBase == kGemmDown) {
                        const float w = pair_weight(a, tokens, at_c.m, a.M);
#pragma unroll
                        for (int j = 0; j < kChunk; ++j) v[j] *= w;
                    }
                    if constexpr (kGroups && (kBase == kGemmDown || kBase == kGemmDx))
                        store_terms<DT>(a.out[0], a.out[1], at_c.out, at_c.inside, v);
                    else
                        store_chunk<DT, kCached>(z ? a.out[1] : a.out[0], at_c.out, at_c.inside, v);
                }
            }
        }
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        __builtin_amdgcn_wave_barrier();
    }
}

template <int DT, int KIND, int TM, int TN, int WAVES_M, int WAVES_N, bool DMA>
void launch_tiles(const GemmArgs& a, int products, hipStream_t st) {
    constexpr int kCols = KindOf<KIND>::kDual ? TN / 2 : TN;
    const int64_t tm = (a.M + TM - 1) / TM, tn = (a.N + kCols - 1) / kCols;
    gemm_kernel<DT, KIND, TM, TN, WAVES_M, WAVES_N, DMA>
        <<<dim3(static_cast<uint32_t>(tm * tn), a.splits, products), WAVES_M * WAVES_N * kWave, 0, st>>>(
            a, static_cast<int>(tm), static_cast<int>(tn));
}

// Whether an operand's tiles can go straight to LDS: its addresses are whole
// dwords, a row of it holds a chunk, and a tile's offsets fit 31 bits.
template <int DT>
bool fetchable(const Operand& o, int64_t row) {
    constexpr int64_t es = sizeof(typename Elem<DT>::T), E = 16 / es;
    if (row < E || o.ld * es % 4 != 0 || o.ld * es * 256 >= int64_t(1) << 31) return false;
    for (const void* p : o.p)
        if (reinterpret_cast<uintptr_t>(p) % 4 != 0) return false;
    return true;
}

template <int DT, int KIND, bool DMA>
void launch_planned(GemmArgs a, int products, hipStream_t st) {
    const GemmPlan plan = plan_gemm(DT, static_cast<GemmKind>(KIND), DMA, a.M, a.N, a.K, products);
    a.splits = plan.splits;
    switch (plan.tile) {
        case kTile256:
            // (Through registers, and in fp32, it would spill them.)
            if constexpr (DMA && DT != IABN_F32) launch_tiles<DT, KIND, 256, 256, 2, 4, DMA>(a, products, st);
            break;
        case kTile128:
            // (Through registers, two blocks of 64x128 take less: the plan's costs.)
            if constexpr (DMA) launch_tiles<DT, KIND, 128, 128, 2, 2, DMA>(a, products, st);
            break;
        case kTile64: launch_tiles<DT, KIND, 64, 128, 2, 2, DMA>(a, products, st); break;
        case kTile32: launch_tiles<DT, KIND, 32, 128, 2, 2, DMA>(a, products, st); break;
    }
    if (a.splits > 1) launch_join(DT, a, products, st);
}

template <int DT, int KIND>
void launch_kind(const GemmArgs& a, int products, hipStream_t st) {
    if (fetchable<DT>(a.x, KindOf<KIND>::kXStrided ? a.M : a.K) &&
        fetchable<DT>(a.y, KindOf<KIND>::kYStrided ? a.N : a.K))
        launch_planned<DT, KIND, true>(a, products, st);
    else
        launch_planned<DT, KIND, false>(a, products, st);
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
