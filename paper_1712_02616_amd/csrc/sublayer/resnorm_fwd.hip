// Forward of the norms around a block, fused with its gate, residual scale
// and dropout:
//
//   n = post(h),  r = alpha*x + beta*gate*D(n),  u = pre(r)
//
// where a norm is hat*w + b with hat = v*rho (rms, rho = (mean v^2 + eps)^-1/2)
// or hat = (v - mean)*rho (layer, the variance about the mean).  r and u of a
// row are written by the threads that read its x and h, which hold the row in
// registers from the first sum to the last: every tensor crosses HBM once, the
// 4 row-sized transfers that the operator cannot do without.  The variance is
// summed about the mean, from the registers (a row whose mean is large against
// its spread loses nothing); sums are fp32 over at most 16 elements of a
// thread, then a tree over its waves.
//
// Rows of up to 1024 elements are one wave's, whose sums need no barrier
// ((32768, 1024) fp16, both norms layer norms, a gate per sample, dropout:
// 61 us, 69 in two waves); wider ones have a block of their own.  That case is
// bound by its arithmetic (vector instructions in 0.79 of the busy cycles) as much
// as by HBM, where its 270 MB (each tensor once) take 47 us at 5.7 TB/s.  (16384,
// 2048) bf16, the same traffic, takes 60 us with RMS norms, a gate and dropout,
// and 46, 5.8 TB/s, with no more than the sum and the RMS norm before the next
// block.  One row of 2048 bf16: 2.5 us, a launch.
#include "sublayer.h"

namespace iabn_impl {
namespace {

// hat*w + b over the row in v; the statistics.
template <int K, bool ONE_WAVE, int FILL>
__device__ __forceinline__ void norm_row(float (&v)[K][kChunk], const RowChunk (&c)[K],
                                         int kind, const float* __restrict__ w,
                                         const float* __restrict__ b, float eps, float inv_c,
                                         SumSlot (&slots)[2], float& mean, float& rstd) {
    float s = 0.0f;
    mean = 0.0f;
    if (kind == IABN_NORM_LAYER) {
#pragma unroll
        for (int k = 0; k < K; ++k)
#pragma unroll
            for (int j = 0; j < kChunk; ++j) s += v[k][j];  // past the row: 0
        s = row_sum<ONE_WAVE>(s, slots[0]);
        mean = s * inv_c;
#pragma unroll
        for (int k = 0; k < K; ++k)
#pragma unroll
            for (int j = 0; j < kChunk; ++j) v[k][j] = inside_row<FILL>(c[k], j, v[k][j] - mean);
    }
    s = 0.0f;
#pragma unroll
    for (int k = 0; k < K; ++k)
#pragma unroll
        for (int j = 0; j < kChunk; ++j) s = fmaf(v[k][j], v[k][j], s);
    s = row_sum<ONE_WAVE>(s, slots[1]);
    rstd = 1.0f / sqrtf(fmaf(s, inv_c, eps));
#pragma unroll
    for (int k = 0; k < K; ++k) {
        float wv[kChunk], bv[kChunk];
        if (w) widen<IABN_F32>(place_chunk<IABN_F32, FILL>(load_row_chunk<IABN_F32, kCached, FILL>(w, 0, c[k]), c[k]), wv);
        if (b) widen<IABN_F32>(place_chunk<IABN_F32, FILL>(load_row_chunk<IABN_F32, kCached, FILL>(b, 0, c[k]), c[k]), bv);
#pragma unroll
        for (int j = 0; j < kChunk; ++j) {
            v[k][j] *= rstd;
            if (w) v[k][j] *= wv[j];
            if (b) v[k][j] += bv[j];
        }
    }
}

// A block is one row of `waves` waves, or (ONE_WAVE) kRows rows of one wave each.
constexpr int kRows = 4;

template <int DT, int K, bool ONE_WAVE, int FILL, int THREADS>
__global__ __launch_bounds__(THREADS) void resnorm_fwd_kernel(ResnormArgs a, int waves) {
    __shared__ SumSlot slots[4];
    if constexpr (!ONE_WAVE) clear_slots(slots, 4);
    const int t = ONE_WAVE ? lane_id() : threadIdx.x, T = ONE_WAVE ? kWave : waves * kWave;
    RowChunk c[K];
#pragma unroll
    for (int k = 0; k < K; ++k) c[k] = row_chunk<FILL>(t + k * T, a.C);
    Dropout dropped = a.drop;
    dropped.scale *= a.beta;
    for (int64_t row = ONE_WAVE ? int64_t(blockIdx.x) * kRows + threadIdx.x / kWave : blockIdx.x;
         row < a.R; row += int64_t(gridDim.x) * (ONE_WAVE ? kRows : 1)) {
        const int64_t base = row * a.C;
        typename ChunkOf<DT>::vec xr[K], hr[K], gr[K];
#pragma unroll
        for (int k = 0; k < K; ++k) {
            xr[k] = load_row_chunk<DT, kStream, FILL>(a.x, base, c[k]);
            if (a.h) hr[k] = load_row_chunk<DT, kStream, FILL>(a.h, base, c[k]);
            if (a.gate) gr[k] = load_row_chunk<DT, kCached, FILL>(a.gate, row / a.gate_rows * a.C, c[k]);
        }
        float v[K][kChunk];
        if (a.h) {
#pragma unroll
            for (int k = 0; k < K; ++k) widen<DT>(place_chunk<DT, FILL>(hr[k], c[k]), v[k]);
            if (a.post != IABN_NORM_NONE) {
                float mean, rstd;
                norm_row<K, ONE_WAVE, FILL>(v, c, a.post, a.post_w, a.post_b, a.eps, a.inv_c,
                                      reinterpret_cast<SumSlot(&)[2]>(slots[0]), mean, rstd);
                if (a.post_stats && t == 0) {
                    a.post_stats[row] = mean;
                    a.post_stats[a.R + row] = rstd;
                }
            }
        }
#pragma unroll
        for (int k = 0; k < K; ++k) {
            float xv[kChunk];
            widen<DT>(place_chunk<DT, FILL>(xr[k], c[k]), xv);
            if (a.h) {
                if (a.drop.threshold)
                    drop_group(dropped, static_cast<uint64_t>(row * a.chunks + c[k].col / kChunk), v[k]);
                else
#pragma unroll
                    for (int j = 0; j < kChunk; ++j) v[k][j] *= a.beta;
                if (a.gate) {
                    float gv[kChunk];
                    widen<DT>(place_chunk<DT, FILL>(gr[k], c[k]), gv);
#pragma unroll
                    for (int j = 0; j < kChunk; ++j) v[k][j] = fmaf(v[k][j], gv[j], a.alpha * xv[j]);
                } else {
#pragma unroll
                    for (int j = 0; j < kChunk; ++j) v[k][j] = fmaf(a.alpha, xv[j], v[k][j]);
                }
                if constexpr (FILL != kFull)
#pragma unroll
                    for (int j = 0; j < kChunk; ++j) v[k][j] = inside_row<FILL>(c[k], j, v[k][j]);
            } else {
#pragma unroll
                for (int j = 0; j < kChunk; ++j) v[k][j] = a.alpha * xv[j];
            }
            if (a.r) store_row_chunk<DT, kStream, FILL>(a.r, base, c[k], v[k]);
        }
        if (a.u) {
            float mean, rstd;
            norm_row<K, ONE_WAVE, FILL>(v, c, a.pre, a.pre_w, a.pre_b, a.eps, a.inv_c,
                                  reinterpret_cast<SumSlot(&)[2]>(slots[2]), mean, rstd);
            if (a.pre_stats && t == 0) {
                a.pre_stats[row] = mean;
                a.pre_stats[a.R + row] = rstd;
            }
#pragma unroll
            for (int k = 0; k < K; ++k) store_row_chunk<DT, kStream, FILL>(a.u, base, c[k], v[k]);
        }
        // The next row's first sum may take the slot that this row's last did.
        if constexpr (!ONE_WAVE) __syncthreads();
    }
}

constexpr int64_t kMaxBlocks = 1 << 20;  // (a launch holds fewer than 2^32 threads)

template <int DT, int FILL>
void launch_filled(const ResnormArgs& a, const RowShape& s, const dim3& grid, hipStream_t st) {
    const int threads = s.waves == 1 ? kRows * kWave : s.waves * kWave;
    if (s.waves == 1 && s.k == 1)
        resnorm_fwd_kernel<DT, 1, true, FILL, kRows * kWave><<<grid, threads, 0, st>>>(a, 1);
    else if constexpr (FILL != kShort) {
        if (s.waves == 1)
            resnorm_fwd_kernel<DT, 2, true, FILL, kRows * kWave><<<grid, threads, 0, st>>>(a, 1);
        else if (s.k == 1)
            resnorm_fwd_kernel<DT, 1, false, FILL, 1024><<<grid, threads, 0, st>>>(a, s.waves);
        else
            resnorm_fwd_kernel<DT, 2, false, FILL, 1024><<<grid, threads, 0, st>>>(a, s.waves);
    }
}

template <int DT>
void launch(const ResnormArgs& a, hipStream_t st) {
    const RowShape s = row_shape(a.chunks, kFwdOneWave);
    const int64_t rows = s.waves == 1 ? kRows : 1, want = (a.R + rows - 1) / rows;
    const dim3 grid(static_cast<uint32_t>(want < kMaxBlocks ? want : kMaxBlocks));
    if (a.C < kChunk) launch_filled<DT, kShort>(a, s, grid, st);
    else if (a.C == s.waves * s.k * kWave * kChunk) launch_filled<DT, kFull>(a, s, grid, st);
    else launch_filled<DT, kPartial>(a, s, grid, st);
}

}  // namespace

bool launch_resnorm_fwd(int dtype, const ResnormArgs& a, hipStream_t st) {
    switch (dtype) {
        case IABN_F32: launch<IABN_F32>(a, st); return true;
        case IABN_F16: launch<IABN_F16>(a, st); return true;
        case IABN_BF16: launch<IABN_BF16>(a, st); return true;
        default: return false;
    }
}

}  // namespace iabn_impl
