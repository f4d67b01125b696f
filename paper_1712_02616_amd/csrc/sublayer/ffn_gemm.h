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

#include "ffn.h"
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
template <int DT, bool KS, int ROWS, int THREADS, bool DUAL>
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
    __device__ __forceinline__ void load(const Operand& o, int seg, int64_t row0, int64_t rows,
                                         int64_t k0, int64_t K) {
#pragma unroll
        for (int i = 0; i < kLoads; ++i) {
            const int line = first_line() + i * kLineStep, c = chunk(i) * E;
            const T* p = static_cast<const T*>(o.p[KS ? seg : matrix_of(line, seg)]);
            if constexpr (KS)
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
    __device__ __forceinline__ void prepare(const Operand& o, int64_t row0, int64_t rows) {
#pragma unroll
        for (int q = 0; q < 2; ++q) {
            // (Kept in scalar registers, not loaded from the arguments at each step.)
            const uint64_t p = reinterpret_cast<uint64_t>(static_cast<const T*>(o.p[q]) + row0 * (KS ? 1 : o.ld));
            base[q] = static_cast<uint32_t>(__builtin_amdgcn_readfirstlane(static_cast<int>(p))) |
                      uint64_t(static_cast<uint32_t>(__builtin_amdgcn_readfirstlane(static_cast<int>(p >> 32)))) << 32;
        }
#pragma unroll
        for (int i = 0; i < kLoads; ++i) {
            const int line = first_line() + i * kLineStep, c = chunk(i) * E;
            if constexpr (KS) {
                off[i] = static_cast<uint32_t>((line * o.ld + (c < rows ? c : 0)) * sizeof(T));
            } else {
                const int64_t row = min(static_cast<int64_t>(row_of(line)), rows - 1);
                off[i] = static_cast<uint32_t>((row * o.ld + c) * sizeof(T));
            }
        }
    }
    __device__ __forceinline__ void fetch(const Operand& o, int seg, int64_t k0, char* lds) const {
#if defined(__HIP_DEVICE_COMPILE__)  // (the host's pass does not know the buffer types)
        typedef __attribute__((address_space(3))) void lds_t;
        const uint64_t at = (KS ? k0 * o.ld : k0) * sizeof(T);
        const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
#pragma unroll
        for (int i = 0; i < kLoads; ++i) {
            // (A wave's lines are of one matrix: a wave covers 8 lines or fewer.)
            const int which =
                DUAL ? __builtin_amdgcn_readfirstlane(matrix_of(first_line() + i * kLineStep, seg)) : seg;
            const __amdgpu_buffer_rsrc_t rsrc = __builtin_amdgcn_make_buffer_rsrc(
                reinterpret_cast<void*>((which ? base[1] : base[0]) + at), 0, 0xffffffff, 0x00027000);
            __builtin_amdgcn_raw_ptr_buffer_load_lds(
                rsrc, (lds_t*)(lds + (wave * kWave + i * THREADS) * 16), 16, off[i], 0, 0, 0);
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
    static constexpr bool kDual = KIND == kGemmUp;
    static constexpr bool kXStrided = KIND == kGemmDw;
    static constexpr bool kYStrided = KIND == kGemmDh || KIND == kGemmDx || KIND == kGemmDw;
    static constexpr int kSegs = KIND == kGemmDx ? 2 : 1;  // products that add up
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

template <int DT, int KIND, int TM, int TN, int WAVES_M, int WAVES_N, bool DMA>
__global__ __launch_bounds__(WAVES_M* WAVES_N* kWave) void gemm_kernel(GemmArgs a, int tiles_m,
                                                                        int tiles_n) {
    using Kind = KindOf<KIND>;
    constexpr int kT = WAVES_M * WAVES_N * kWave;
    constexpr int WM = TM / WAVES_M, WN = TN / WAVES_N, NM = WM / 16, NN = WN / 16;
    static_assert(!Kind::kDual || WN == kSpan, "a wave holds both projections of its columns");
    using SX = Stage<DT, Kind::kXStrided, TM, kT, false>;
    using SY = Stage<DT, Kind::kYStrided, TN, kT, Kind::kDual>;
    constexpr int BK = SX::BK;
    // Two buffers, of which one is multiplied while the other fills.
    constexpr int kBuffer = SX::kBytes + SY::kBytes;
    __shared__ __align__(16) char lds[2 * kBuffer];
    char *const lds0 = lds, *const lds1 = lds + kBuffer;

    int tm, tn;
    tile_of(tiles_m, tiles_n, tm, tn);
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
    u32x4 fy[kSteps][NN], fx[2][NH];
    const auto read = [&](const char* __restrict__ buf, int phase) __attribute__((always_inline)) {
        const int s = phase / kHalves, h = phase % kHalves;
        if (h == 0)
#pragma unroll
            for (int j = 0; j < NN; ++j) fy[s][j] = SY::frag(buf + SX::kBytes, wn + j * 16, s);
#pragma unroll
        for (int i = 0; i < NH; ++i) fx[phase & 1][i] = SX::frag(buf, wm + (h * NH + i) * 16, s);
    };
    const auto products = [&](int phase) __attribute__((always_inline)) {
        const int s = phase / kHalves, h = phase % kHalves;
#pragma unroll
        for (int i = 0; i < NH; ++i)
#pragma unroll
            for (int j = 0; j < NN; ++j)
                acc[h * NH + i][j] = Mma<DT>::run(fy[s][j], fx[phase & 1][i], acc[h * NH + i][j]);
    };
    // Steps of K: whole ones that go straight to LDS, those of the first
    // product and then those of the second, and the others, through
    // registers.  This block's share of them all: [lo, hi) and [from, to).
    // (A strided operand whose last chunk of a row reaches into the next one may
    // not fetch its last row.)
    constexpr int E = SX::E;
    const bool reaches = (Kind::kXStrided && a.M % E != 0) || (Kind::kYStrided && a.N % E != 0);
    const int whole = DMA ? static_cast<int>((a.K - (reaches ? 1 : 0)) / BK) : 0, steps = whole * Kind::kSegs;
    const int per_seg = static_cast<int>((a.K + BK - 1) / BK) - whole, rest = per_seg * Kind::kSegs;
    const int64_t all = steps + rest;
    const int begin = static_cast<int>(all * blockIdx.y / gridDim.y);
    const int end = static_cast<int>(all * (blockIdx.y + 1) / gridDim.y);
    const int lo = min(begin, steps), hi = min(end, steps);
    const int from = max(begin - steps, 0), to = max(end - steps, 0);
    if constexpr (DMA) {
        const auto fetch = [&](int kt, char* buf) __attribute__((always_inline)) {
            const int seg = Kind::kSegs > 1 ? (kt >= whole ? 1 : 0) : z;
            const int64_t k0 = int64_t(Kind::kSegs > 1 && seg ? kt - whole : kt) * BK;
            sx.fetch(a.x, seg, k0, buf);
            sy.fetch(a.y, seg, k0, buf + SX::kBytes);
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
        sx.prepare(a.x, m0, a.M - m0);
        sy.prepare(a.y, n0, a.N - n0);
        if (lo < hi) fetch(lo, lds0);
        if (kAhead && lo < hi) {
            meet();
            if (lo + 1 < hi) fetch(lo + 1, lds1);
            read(lds0, 0);
        }
        for (int kt = lo; kt < hi; kt += 2) round(kt, lds0, lds1);
        __syncthreads();
    }
    if (from < to) {
        const auto load = [&](int kt) __attribute__((always_inline)) {
            const int seg = Kind::kSegs > 1 ? (kt >= per_seg ? 1 : 0) : z;
            const int64_t k0 = int64_t(whole + (Kind::kSegs > 1 && seg ? kt - per_seg : kt)) * BK;
            sx.load(a.x, seg, m0, a.M - m0, k0, a.K);
            sy.load(a.y, seg, n0, a.N - n0, k0, a.K);
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
        }
    }

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
    static_assert(kTurns * kWave == kPass * 16 * kCh && (KIND != kGemmDh || kTurns % 2 == 0), "");
    struct Place {
        int row, col, inside;
        int64_t out;
    };
    const auto place = [&](int p, int c) {
        const int at_c = c * kWave + static_cast<int>(lane_id());
        Place r;
        r.row = at_c / kCh, r.col = at_c % kCh * kChunk;
        const int64_t m = m0 + wm + p * 16 + r.row, n = n0 + (Kind::kDual ? wn / 2 : wn) + r.col;
        r.inside = m < a.M ? static_cast<int>(max(min(a.N - n, int64_t(kChunk)), int64_t(0))) : 0;
        r.out = m * a.N + n;
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
        chunk_t gu[2][2];
        if constexpr (KIND == kGemmDh) {
            load_gu(p, 0, gu[0]);
            load_gu(p, 1, gu[1]);
        }
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
        if constexpr (KIND == kGemmDh) {
#pragma unroll 1
            for (int c = 0; c < kTurns; c += 2)
#pragma unroll
                for (int q = 0; q < 2; ++q) {
                    const auto raw_g = gu[q][0], raw_u = gu[q][1];
                    const Place at_c = place(p, c + q);
                    if (c + q + 2 < kTurns) load_gu(p, c + q + 2, gu[q]);
                    if (at_c.inside <= 0) continue;
                    float v[kChunk], g[kChunk], u[kChunk], dg[kChunk], du[kChunk], h[kChunk];
                    read(at_c.row, at_c.col, v);
                    widen<DT>(raw_g, g);
                    widen<DT>(raw_u, u);
                    gate_backward<DT>(a.act, a.slope, v, g, u, dg, du, h);
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
                if constexpr (KIND == kGemmUp) {
                    float u[kChunk], h[kChunk];
                    read(at_c.row, at_c.col + WN / 2, u);
                    gate_forward<DT>(a.act, a.slope, v, u, h);
                    store_chunk<DT, kCached>(a.out[0], at_c.out, at_c.inside, h);
                    if (a.dg) {
                        store_chunk<DT, kStream>(a.dg, at_c.out, at_c.inside, v);
                        store_chunk<DT, kStream>(a.du, at_c.out, at_c.inside, u);
                    }
                } else if (gridDim.y > 1) {
                    store_chunk<IABN_F32, kCached>(
                        a.part, (int64_t(blockIdx.y) * gridDim.z + z) * a.M * a.N + at_c.out, at_c.inside, v);
                } else {
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
