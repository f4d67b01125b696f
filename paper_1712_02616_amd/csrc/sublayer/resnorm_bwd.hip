// Backward of the norms around a block (resnorm_fwd.hip).  Per row, with
// rhat, hhat the normalised rows of r and h (from the saved statistics; (v - mean)*rho,
// whose subtraction loses nothing where the mean is large against the spread, as
// v*rho - mean*rho would):
//
//   a  = du*w',  g = dr + rho'*(a - [mean a] - rhat*mean(a*rhat))
//   dx = alpha*g,  e = beta*g*D,  dn = e*gate
//   b  = dn*w,   dh = rho*(b - [mean b] - hhat*mean(b*hhat))
//
// ([.]: layer norms only), and over the rows dw' = sum du*rhat, db' = sum du,
// dw = sum dn*hhat, db = sum dn, and over the rows of a gate dgate = sum e*n.
//
// Bound by HBM traffic: dr, du, r, h in and dx, dh out, 6 row-sized
// transfers, all of them once: the threads of a row keep it in registers over
// the two sums, and keep its columns' sums over the rows in registers from
// row to row, so the vectors' gradients cost no second reading.  A block
// therefore goes through many rows (a segment); the next row's loads are
// issued before this row's sums (two rows ahead were no faster).  Each block
// leaves its columns' sums in the workspace and a second kernel adds the
// blocks' in double, in a fixed order.  (A wave adds at most 1024 rows in fp32: more
// rows are more blocks.)
//
// bf16, RMS norms, gate and dropout: (16384, 2048) 82 us and 7 for the sums,
// against 71 us for its 403 MB of HBM traffic at 5.7 TB/s; it reads 279 MB and
// writes 166, of which 19 are the columns' sums and 13 registers that are spilled
// for a third wave per SIMD (rows that fill their
// threads are not masked, sums that a norm does not need are left out, the
// branch's scale goes with the dropout's); (65536, 512), the same traffic, 82 and
// 5, and 68 and 5 with no more than the norm before the next block.  (1031, 1501)
// fp32 21 and 4: four rows one after the other in each of 258 blocks.  Rows of
// 4097 to 8192 have 128 registers per thread: (4096, 8192) bf16 125 us, 171 with a
// row ahead; those of up to 16384 spill: (2048, 16384) 450 us.
#include "sublayer.h"

namespace iabn_impl {
namespace {

// ONE_WAVE: a block is kRows rows at a time of one wave each.
constexpr int kRows = 4;

template <int DT, int K>
struct RowRegs {
    typename ChunkOf<DT>::vec dr[K], du[K], r[K], h[K];
    float pre_mean, pre_rstd, post_mean, post_rstd;
};

// (`zero` is 0 in a vector register: a row's statistics come by vector loads, in
// the order of the others.  By scalar ones, which the wait for LDS waits for
// too, or when they are needed, they cost a round trip to memory per row:
// (1031, 1501) fp32 22 us.)
template <int DT, int K, int FILL, bool POST, bool PRE>
__device__ __forceinline__ void load_row(const ResnormBwdArgs& a, int64_t row, const RowChunk (&c)[K],
                                         int zero, RowRegs<DT, K>& x) {
    const int64_t base = row * a.C;
    if constexpr (PRE) {
        x.pre_mean = a.pre_stats[row + zero];
        x.pre_rstd = a.pre_stats[a.R + row + zero];
    }
    if constexpr (POST) {
        if (a.post != IABN_NORM_NONE) {
            x.post_mean = a.post_stats[row + zero];
            x.post_rstd = a.post_stats[a.R + row + zero];
        }
    }
#pragma unroll
    for (int k = 0; k < K; ++k) {
        if (a.dr) x.dr[k] = load_row_chunk<DT, kStream, FILL>(a.dr, base, c[k]);
        if constexpr (PRE) {
            x.du[k] = load_row_chunk<DT, kStream, FILL>(a.du, base, c[k]);
            x.r[k] = load_row_chunk<DT, kStream, FILL>(a.r, base, c[k]);
        }
        if constexpr (POST) {
            if (a.h) x.h[k] = load_row_chunk<DT, kStream, FILL>(a.h, base, c[k]);
        }
    }
}

// Adds up the block's columns' sums and leaves them at `out`: the threads of
// one row at a time hold every column once; kRows waves add theirs in LDS.
template <int K, bool ONE_WAVE, typename Put>
__device__ __forceinline__ void flush(float (&acc)[K][kChunk], const RowChunk (&c)[K], float* lds, Put put) {
    if constexpr (ONE_WAVE) {
        const int w = threadIdx.x / kWave;
#pragma unroll
        for (int k = 0; k < K; ++k) {
            __syncthreads();
#pragma unroll
            for (int j = 0; j < kChunk; ++j) lds[(w * kChunk + j) * kWave + lane_id()] = acc[k][j];
            __syncthreads();
            if (w == 0) {
#pragma unroll
                for (int j = 0; j < kChunk; ++j) {
                    float s = acc[k][j];
                    for (int i = 1; i < kRows; ++i) s += lds[(i * kChunk + j) * kWave + lane_id()];
                    acc[k][j] = s;
                }
                put(c[k].n, c[k].col, acc[k]);
            }
        }
    } else {
#pragma unroll
        for (int k = 0; k < K; ++k) put(c[k].n, c[k].col, acc[k]);
    }
#pragma unroll
    for (int k = 0; k < K; ++k)
#pragma unroll
        for (int j = 0; j < kChunk; ++j) acc[k][j] = 0.0f;
}

template <int DT, int K, bool ONE_WAVE, int FILL, bool POST, bool PRE, int THREADS>
__global__ __launch_bounds__(THREADS, !ONE_WAVE && THREADS == 256 && FILL == kFull && DT != IABN_F32 ? 3 : 1)
void resnorm_bwd_kernel(ResnormBwdArgs a, int waves) {
    __shared__ SumSlot slots[4];
    if constexpr (!ONE_WAVE) clear_slots(slots, 4);
    __shared__ float lds[ONE_WAVE ? kRows * kWave * kChunk : 1];
    const int t = ONE_WAVE ? lane_id() : threadIdx.x, T = ONE_WAVE ? kWave : waves * kWave;
    const int first = ONE_WAVE ? threadIdx.x / kWave : 0;
    constexpr int kStep = ONE_WAVE ? kRows : 1;
    // The widest rows' threads have 128 registers: no row ahead, and the weights
    // come from the caches for each row.
    constexpr bool kLean = THREADS > 512;
    RowChunk c[K];
#pragma unroll
    for (int k = 0; k < K; ++k) c[k] = row_chunk<FILL>(t + k * T, a.C);
    const auto vector = [&](const float* v, int k, float (&out)[kChunk]) {
        widen<IABN_F32>(place_chunk<IABN_F32, FILL>(load_row_chunk<IABN_F32, kCached, FILL>(v, 0, c[k]), c[k]), out);
    };
    const auto values = [&](const typename ChunkOf<DT>::vec& v, int k, float (&out)[kChunk]) {
        widen<DT>(place_chunk<DT, FILL>(v, c[k]), out);
    };
    // The columns' sums: dw, db, dgate; dw', db'.
    float sw[POST ? K : 1][kChunk] = {}, sb[POST ? K : 1][kChunk] = {}, sg[POST ? K : 1][kChunk] = {};
    float tw[PRE ? K : 1][kChunk] = {}, tb[PRE ? K : 1][kChunk] = {};
    // The vectors, in registers for all rows.
    float pre_w[PRE ? K : 1][kChunk], post_w[POST ? K : 1][kChunk];
    if constexpr (PRE) {
#pragma unroll
        for (int k = 0; k < K; ++k) {
#pragma unroll
            for (int j = 0; j < kChunk; ++j) pre_w[k][j] = 1.0f;
            if (a.pre_w && !kLean) vector(a.pre_w, k, pre_w[k]);
        }
    }
    if constexpr (POST) {
#pragma unroll
        for (int k = 0; k < K; ++k) {
#pragma unroll
            for (int j = 0; j < kChunk; ++j) post_w[k][j] = 1.0f;
            if (a.post_w && !kLean) vector(a.post_w, k, post_w[k]);
        }
    }
    int zero = 0;
    asm volatile("" : "+v"(zero));
    const int64_t seg_rows = (a.split.group_rows + a.split.per_group - 1) / a.split.per_group;
    int par = 0;  // alternates the slots of consecutive rows
    Dropout dropped = a.drop;
    dropped.scale *= a.beta;

    for (int s = 0; s < a.split.segs; ++s) {
        const int64_t seg = int64_t(blockIdx.x) * a.split.segs + s, group = seg / a.split.per_group;
        if (group >= a.split.groups) break;
        const int64_t in_group = (seg - group * a.split.per_group) * seg_rows, at = group * a.split.group_rows;
        const int64_t lo = at + min(in_group, a.split.group_rows);
        const int64_t hi = at + min(in_group + seg_rows, a.split.group_rows);
        typename ChunkOf<DT>::vec gate[POST ? K : 1];  // the segment's (or each row's)
        if constexpr (POST) {
            if (a.gate && lo + first < hi)
#pragma unroll
                for (int k = 0; k < K; ++k)
                    gate[k] = load_row_chunk<DT, kCached, FILL>(a.gate, (lo + first) / a.gate_rows * a.C, c[k]);
        }
        RowRegs<DT, K> x;
        if (!kLean && lo + first < hi) load_row<DT, K, FILL, POST, PRE>(a, lo + first, c, zero, x);
        for (int64_t row = lo + first; row < hi; row += kStep) {
            if constexpr (kLean) load_row<DT, K, FILL, POST, PRE>(a, row, c, zero, x);
            float g[K][kChunk];
#pragma unroll
            for (int k = 0; k < K; ++k) {
                if (a.dr) values(x.dr[k], k, g[k]);
                else
#pragma unroll
                    for (int j = 0; j < kChunk; ++j) g[k][j] = 0.0f;
            }
            typename ChunkOf<DT>::vec raw_h[POST ? K : 1];
            float rhat[PRE ? K : 1][kChunk], rdu[PRE ? K : 1][kChunk];
#pragma unroll
            for (int k = 0; k < K; ++k) {
                if constexpr (POST) raw_h[k] = x.h[k];
                if constexpr (PRE) {
                    values(x.r[k], k, rhat[k]);
                    values(x.du[k], k, rdu[k]);
                }
            }
            const float pre_mean = x.pre_mean, pre_rstd = x.pre_rstd;
            const float post_mean = x.post_mean, post_rstd = x.post_rstd;
            // The next row is on its way while this one is worked on.
            if (!kLean && row + kStep < hi) load_row<DT, K, FILL, POST, PRE>(a, row + kStep, c, zero, x);
            if constexpr (PRE) {
                const float mean = pre_mean, rstd = pre_rstd;
                float (&hat)[K][kChunk] = rhat, (&d)[K][kChunk] = rdu, s1 = 0.0f, s2 = 0.0f;
                if (a.dpre_b) {
#pragma unroll
                    for (int k = 0; k < K; ++k)
#pragma unroll
                        for (int j = 0; j < kChunk; ++j) tb[k][j] += d[k][j];
                }
#pragma unroll
                for (int k = 0; k < K; ++k) {
                    if (kLean && a.pre_w) vector(a.pre_w, k, pre_w[k]);
#pragma unroll
                    for (int j = 0; j < kChunk; ++j) {
                        hat[k][j] = inside_row<FILL>(c[k], j, (hat[k][j] - mean) * rstd);
                        tw[k][j] = fmaf(d[k][j], hat[k][j], tw[k][j]);
                        d[k][j] *= pre_w[k][j];
                        s2 = fmaf(d[k][j], hat[k][j], s2);
                    }
                }
                if (a.pre == IABN_NORM_LAYER) {
#pragma unroll
                    for (int k = 0; k < K; ++k)
#pragma unroll
                        for (int j = 0; j < kChunk; ++j) s1 += d[k][j];
                    row_sum2<ONE_WAVE>(s1, s2, slots[par]);
                    s1 *= -rstd * a.inv_c;
#pragma unroll
                    for (int k = 0; k < K; ++k)
#pragma unroll
                        for (int j = 0; j < kChunk; ++j) g[k][j] += s1;
                } else {
                    s2 = row_sum<ONE_WAVE>(s2, slots[par]);
                }
                s2 *= -rstd * a.inv_c;
#pragma unroll
                for (int k = 0; k < K; ++k)
#pragma unroll
                    for (int j = 0; j < kChunk; ++j)
                        g[k][j] = fmaf(rstd, d[k][j], fmaf(s2, hat[k][j], g[k][j]));
            }
            const int64_t base = row * a.C;
            if (a.dx) {
#pragma unroll
                for (int k = 0; k < K; ++k) {
                    float o[kChunk];
#pragma unroll
                    for (int j = 0; j < kChunk; ++j) o[j] = a.alpha * g[k][j];
                    store_row_chunk<DT, kStream, FILL>(a.dx, base, c[k], o);
                }
            }
            if constexpr (POST) {
                float hat[K][kChunk], s1 = 0.0f, s2 = 0.0f, mean = 0.0f, rstd = 1.0f;
                if (a.post != IABN_NORM_NONE) {
                    mean = post_mean;
                    rstd = post_rstd;
                }
#pragma unroll
                for (int k = 0; k < K; ++k) {
                    if (a.h) values(raw_h[k], k, hat[k]);
                    if (kLean && a.post_w) vector(a.post_w, k, post_w[k]);
                    // From here g is e = beta*g*D, then dn, then dn*w.
#pragma unroll
                    for (int j = 0; j < kChunk; ++j) {
                        hat[k][j] = a.h ? inside_row<FILL>(c[k], j, (hat[k][j] - mean) * rstd) : 0.0f;
                        if constexpr (FILL != kFull) g[k][j] = inside_row<FILL>(c[k], j, g[k][j]);
                    }
                    if (a.drop.threshold)
                        drop_group(dropped, static_cast<uint64_t>(row * a.chunks + c[k].col / kChunk), g[k]);
                    else
#pragma unroll
                        for (int j = 0; j < kChunk; ++j) g[k][j] *= a.beta;
                    if (a.gate) {
                        float gv[kChunk], o[kChunk], bv[kChunk] = {};
                        if (a.post_b) vector(a.post_b, k, bv);
                        values(gate[k], k, gv);
                        if (a.gate_each_row && row + kStep < hi)
                            gate[k] = load_row_chunk<DT, kStream, FILL>(a.gate, (row + kStep) * a.C, c[k]);
#pragma unroll
                        for (int j = 0; j < kChunk; ++j) {
                            o[j] = g[k][j] * fmaf(hat[k][j], post_w[k][j], bv[j]);
                            sg[k][j] += o[j];
                            g[k][j] *= gv[j];
                        }
                        if (a.dgate && a.gate_each_row)
                            store_row_chunk<DT, kStream, FILL>(a.dgate, base, c[k], o);
                    }
                    if (a.post != IABN_NORM_NONE) {
                        if (a.dpost_b) {
#pragma unroll
                            for (int j = 0; j < kChunk; ++j) sb[k][j] += g[k][j];
                        }
#pragma unroll
                        for (int j = 0; j < kChunk; ++j) {
                            sw[k][j] = fmaf(g[k][j], hat[k][j], sw[k][j]);
                            g[k][j] *= post_w[k][j];
                            s2 = fmaf(g[k][j], hat[k][j], s2);
                        }
                    }
                }
                if (a.post != IABN_NORM_NONE) {
                    if (a.post == IABN_NORM_LAYER) {
#pragma unroll
                        for (int k = 0; k < K; ++k)
#pragma unroll
                            for (int j = 0; j < kChunk; ++j) s1 += g[k][j];
                        row_sum2<ONE_WAVE>(s1, s2, slots[2 + par]);
                    } else {
                        s2 = row_sum<ONE_WAVE>(s2, slots[2 + par]);
                    }
                    s1 *= -rstd * a.inv_c;
                    s2 *= -rstd * a.inv_c;
#pragma unroll
                    for (int k = 0; k < K; ++k)
#pragma unroll
                        for (int j = 0; j < kChunk; ++j)
                            g[k][j] = fmaf(s2, hat[k][j], fmaf(rstd, g[k][j], s1));
                }
                if (a.dh)
#pragma unroll
                    for (int k = 0; k < K; ++k) store_row_chunk<DT, kStream, FILL>(a.dh, base, c[k], g[k]);
            }
            par ^= 1;
        }
        if constexpr (POST) {
            if (a.dgate && !a.gate_each_row) {
                const int64_t out = (a.split.per_group == 1 ? group : int64_t(blockIdx.x)) * a.C;
                flush<K, ONE_WAVE>(sg, c, lds, [&](int m, int c, float (&v)[kChunk]) {
                    if (a.split.per_group == 1) store_chunk<DT, kStream>(a.dgate, out + c, m, v);
                    else store_chunk<IABN_F32, kCached>(a.gpart, out + c, m, v);
                });
            }
        }
    }
    const auto put = [&](int which) {
        return [=](int m, int c, float (&v)[kChunk]) {
            store_chunk<IABN_F32, kCached>(a.part, (int64_t(which) * a.split.blocks + blockIdx.x) * a.C + c, m, v);
        };
    };
    if constexpr (POST) {
        if (a.dpost_w) flush<K, ONE_WAVE>(sw, c, lds, put(0));
        if (a.dpost_b) flush<K, ONE_WAVE>(sb, c, lds, put(1));
    }
    if constexpr (PRE) {
        if (a.dpre_w) flush<K, ONE_WAVE>(tw, c, lds, put(2));
        if (a.dpre_b) flush<K, ONE_WAVE>(tb, c, lds, put(3));
    }
}

// out[c] = sum over `count` rows of part[., c], in double.  A block takes 32
// columns; 8 of its threads share a column.
constexpr int kSumCols = 32;
constexpr int64_t kMaxSumGroups = 1 << 15;  // of a launch; more take turns

template <int DT>
__device__ __forceinline__ void column_sum(const float* __restrict__ part, int count, int C,
                                           void* __restrict__ out) {
    __shared__ double lds[kThreads];
    const int c = blockIdx.x * kSumCols + threadIdx.x % kSumCols, y = threadIdx.x / kSumCols;
    constexpr int kY = kThreads / kSumCols;
    double s = 0.0;
    if (c < C) {
#pragma unroll 8
        for (int i = y; i < count; i += kY) s += part[int64_t(i) * C + c];
    }
    lds[threadIdx.x] = s;
    __syncthreads();
    if (y == 0 && c < C) {
        for (int i = 1; i < kY; ++i) s += lds[i * kSumCols + threadIdx.x];
        static_cast<typename Elem<DT>::T*>(out)[c] =
            static_cast<typename Elem<DT>::T>(static_cast<float>(s));
    }
}

// Grid: (columns, the 4 vectors and then the gate's groups).
template <int DT>
__global__ __launch_bounds__(kThreads) void resnorm_bwd_sum_kernel(ResnormBwdArgs a) {
    if (blockIdx.y < 4) {
        float* const out = blockIdx.y == 0   ? a.dpost_w
                           : blockIdx.y == 1 ? a.dpost_b
                           : blockIdx.y == 2 ? a.dpre_w
                                             : a.dpre_b;
        if (out)
            column_sum<IABN_F32>(a.part + int64_t(blockIdx.y) * a.split.blocks * a.C, a.split.blocks, a.C, out);
    } else {
        for (int64_t g = blockIdx.y - 4; g < a.split.groups; g += gridDim.y - 4) {
            column_sum<DT>(a.gpart + g * a.split.per_group * a.C, a.split.per_group, a.C,
                           static_cast<typename Elem<DT>::T*>(a.dgate) + g * a.C);
            __syncthreads();
        }
    }
}

template <int DT, int FILL, bool POST, bool PRE>
void launch_filled(const ResnormBwdArgs& a, const RowShape& s, hipStream_t st) {
    const dim3 grid(static_cast<uint32_t>(a.split.blocks));
    const int threads = s.waves == 1 ? kRows * kWave : s.waves * kWave;
    // (The registers of a thread follow from the most threads that a block may have.)
    if (s.waves == 1)
        resnorm_bwd_kernel<DT, 1, true, FILL, POST, PRE, kRows * kWave><<<grid, threads, 0, st>>>(a, 1);
    else if constexpr (FILL != kShort) {
        if (s.waves <= 4)
            resnorm_bwd_kernel<DT, 1, false, FILL, POST, PRE, 256><<<grid, threads, 0, st>>>(a, s.waves);
        else if (s.waves <= 8)
            resnorm_bwd_kernel<DT, 1, false, FILL, POST, PRE, 512><<<grid, threads, 0, st>>>(a, s.waves);
        else if (s.k == 1)
            resnorm_bwd_kernel<DT, 1, false, FILL, POST, PRE, 1024><<<grid, threads, 0, st>>>(a, s.waves);
        else
            resnorm_bwd_kernel<DT, 2, false, FILL, POST, PRE, 1024><<<grid, threads, 0, st>>>(a, s.waves);
    }
}

template <int DT, bool POST, bool PRE>
void launch_rows(const ResnormBwdArgs& a, hipStream_t st) {
    const RowShape s = row_shape(a.chunks, kBwdOneWave);
    if (a.C < kChunk) launch_filled<DT, kShort, POST, PRE>(a, s, st);
    else if (a.C == s.waves * s.k * kWave * kChunk) launch_filled<DT, kFull, POST, PRE>(a, s, st);
    else launch_filled<DT, kPartial, POST, PRE>(a, s, st);
}

template <int DT>
void launch(const ResnormBwdArgs& a, hipStream_t st) {
    const bool post = a.dh || a.dgate || a.dpost_w || a.dpost_b, pre = a.du != nullptr;
    if (post && pre) launch_rows<DT, true, true>(a, st);
    else if (post) launch_rows<DT, true, false>(a, st);
    else if (pre) launch_rows<DT, false, true>(a, st);
    else launch_rows<DT, false, false>(a, st);
    const bool gate = a.dgate && a.split.per_group > 1 && !a.gate_each_row;
    if (a.dpost_w || a.dpost_b || a.dpre_w || a.dpre_b || gate) {
        const dim3 grid((a.C + kSumCols - 1) / kSumCols,
                        4 + (gate ? static_cast<uint32_t>(min(a.split.groups, kMaxSumGroups)) : 0u));
        resnorm_bwd_sum_kernel<DT><<<grid, kThreads, 0, st>>>(a);
    }
}

}  // namespace

bool launch_resnorm_bwd(int dtype, const ResnormBwdArgs& a, hipStream_t st) {
    switch (dtype) {
        case IABN_F32: launch<IABN_F32>(a, st); return true;
        case IABN_F16: launch<IABN_F16>(a, st); return true;
        case IABN_BF16: launch<IABN_BF16>(a, st); return true;
        default: return false;
    }
}

}  // namespace iabn_impl
