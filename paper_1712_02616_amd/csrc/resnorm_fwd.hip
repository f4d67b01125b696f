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
#include "sublayer.h"

namespace iabn_impl {
namespace {

// hat*w + b over the row in v; the statistics.
template <int K, bool ONE_WAVE>
__device__ __forceinline__ void norm_row(float (&v)[K][kChunk], const int (&n)[K],
                                         const int (&col)[K], int kind, const float* __restrict__ w,
                                         const float* __restrict__ b, float eps, float inv_c,
                                         int waves, SumSlot (&slots)[2], float& mean, float& rstd) {
    float s = 0.0f, none = 0.0f;
    mean = 0.0f;
    if (kind == IABN_NORM_LAYER) {
#pragma unroll
        for (int k = 0; k < K; ++k)
#pragma unroll
            for (int j = 0; j < kChunk; ++j) s += v[k][j];  // past the row: 0
        row_sum2<ONE_WAVE>(s, none, slots[0], waves);
        mean = s * inv_c;
#pragma unroll
        for (int k = 0; k < K; ++k)
#pragma unroll
            for (int j = 0; j < kChunk; ++j) v[k][j] = j < n[k] ? v[k][j] - mean : 0.0f;
    }
    s = none = 0.0f;
#pragma unroll
    for (int k = 0; k < K; ++k)
#pragma unroll
        for (int j = 0; j < kChunk; ++j) s = fmaf(v[k][j], v[k][j], s);
    row_sum2<ONE_WAVE>(s, none, slots[1], waves);
    rstd = 1.0f / sqrtf(fmaf(s, inv_c, eps));
#pragma unroll
    for (int k = 0; k < K; ++k) {
        float wv[kChunk], bv[kChunk];
        if (w) widen<IABN_F32>(load_chunk<IABN_F32, kCached>(w, col[k], n[k]), wv);
        if (b) widen<IABN_F32>(load_chunk<IABN_F32, kCached>(b, col[k], n[k]), bv);
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

template <int DT, int K, bool ONE_WAVE>
__global__ __launch_bounds__(ONE_WAVE ? kRows * kWave : kMaxRowWaves * kWave)
void resnorm_fwd_kernel(ResnormArgs a, int waves) {
    __shared__ SumSlot slots[4];
    const int t = ONE_WAVE ? lane_id() : threadIdx.x, T = ONE_WAVE ? kWave : waves * kWave;
    for (int64_t row = ONE_WAVE ? int64_t(blockIdx.x) * kRows + threadIdx.x / kWave : blockIdx.x;
         row < a.R; row += int64_t(gridDim.x) * (ONE_WAVE ? kRows : 1)) {
        const int64_t base = row * a.C;
        int n[K], col[K];
        typename ChunkOf<DT>::vec xr[K], hr[K], gr[K];
#pragma unroll
        for (int k = 0; k < K; ++k) {
            const int c = t + k * T;
            // A thread past the row loads and stores nothing.
            n[k] = max(min(kChunk, a.C - c * kChunk), 0);
            col[k] = c * kChunk;
            xr[k] = load_chunk<DT, kStream>(a.x, base + col[k], n[k]);
            if (a.h) hr[k] = load_chunk<DT, kStream>(a.h, base + col[k], n[k]);
        }
        float v[K][kChunk];
        if (a.h) {
#pragma unroll
            for (int k = 0; k < K; ++k) {
                if (a.gate)
                    gr[k] = load_chunk<DT, kCached>(a.gate, row / a.gate_rows * a.C + col[k], n[k]);
                widen<DT>(hr[k], v[k]);
            }
            if (a.post != IABN_NORM_NONE) {
                float mean, rstd;
                norm_row<K, ONE_WAVE>(v, n, col, a.post, a.post_w, a.post_b, a.eps, a.inv_c, waves,
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
            widen<DT>(xr[k], xv);
            if (a.h) {
                if (a.drop.threshold)
                    drop_group(a.drop, static_cast<uint64_t>(row * a.chunks + col[k] / kChunk), v[k]);
                if (a.gate) {
                    float gv[kChunk];
                    widen<DT>(gr[k], gv);
#pragma unroll
                    for (int j = 0; j < kChunk; ++j) v[k][j] *= gv[j];
                }
#pragma unroll
                for (int j = 0; j < kChunk; ++j)
                    v[k][j] = j < n[k] ? fmaf(a.beta, v[k][j], a.alpha * xv[j]) : 0.0f;
            } else {
#pragma unroll
                for (int j = 0; j < kChunk; ++j) v[k][j] = a.alpha * xv[j];
            }
            if (a.r) store_chunk<DT, kStream>(a.r, base + col[k], n[k], v[k]);
        }
        if (a.u) {
            float mean, rstd;
            norm_row<K, ONE_WAVE>(v, n, col, a.pre, a.pre_w, a.pre_b, a.eps, a.inv_c, waves,
                                  reinterpret_cast<SumSlot(&)[2]>(slots[2]), mean, rstd);
            if (a.pre_stats && t == 0) {
                a.pre_stats[row] = mean;
                a.pre_stats[a.R + row] = rstd;
            }
#pragma unroll
            for (int k = 0; k < K; ++k) store_chunk<DT, kStream>(a.u, base + col[k], n[k], v[k]);
        }
        // The next row's first sum may take the slot that this row's last did.
        if constexpr (!ONE_WAVE) __syncthreads();
    }
}

constexpr int64_t kMaxBlocks = 1 << 20;  // (a launch holds fewer than 2^32 threads)

template <int DT>
void launch(const ResnormArgs& a, hipStream_t st) {
    const RowShape s = row_shape(a.chunks);
    const int64_t rows = s.waves == 1 ? kRows : 1, want = (a.R + rows - 1) / rows;
    const dim3 grid(static_cast<uint32_t>(want < kMaxBlocks ? want : kMaxBlocks));
    if (s.waves == 1)
        resnorm_fwd_kernel<DT, 1, true><<<grid, kRows * kWave, 0, st>>>(a, 1);
    else if (s.k == 1)
        resnorm_fwd_kernel<DT, 1, false><<<grid, s.waves * kWave, 0, st>>>(a, s.waves);
    else
        resnorm_fwd_kernel<DT, 2, false><<<grid, s.waves * kWave, 0, st>>>(a, s.waves);
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
