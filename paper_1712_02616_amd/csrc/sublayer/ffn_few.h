// The block's forward for few tokens (serving): the weights' traffic is all
// that counts, so every weight goes from memory to the matrix cores' registers
// once, with no LDS between: a wave holds 16 columns of the output (kGemmUp:
// of both projections) for up to 64 tokens, whose x it reads from the caches
// in the same layout.  The waves of a block share their columns and split K,
// line by line of 128 bytes, so that a block reads each row of the weights in
// long runs; their sums meet in LDS.
//
// Bound by HBM: one token (4096 -> 2x10240) bf16 34 us for 168 MB, 4.9 TB/s, and
// 16 us for the 84 MB back, 5.3; 24 tokens (2048 -> 2x8192) fp16 17 us, 4.0, and
// back 12 and 4 to join, where the tokens' h, read by every block, is more
// traffic than the weights.  The weights' loads keep lines in the caches: a line
// is two loads (one token: 32 and 16 us, non-temporal 35 and 21).
#pragma once

#include "ffn.h"
#include "mma.h"

namespace iabn_impl {

// Lines of 128 bytes of every row in a batch; a wave has two batches in flight
// (four lines spill: one
// token 41 us instead of 34, 24 tokens 32 instead of 16).
constexpr int kFewLines = 2;

template <int DT, int KIND, int MT>
__global__ __launch_bounds__(512) void few_kernel(GemmArgs a) {
    using T = typename Elem<DT>::T;
    constexpr int E = 16 / sizeof(T), kLine = 128 / sizeof(T);
    constexpr int NW = KIND == kGemmUp ? 2 : 1;  // matrices of weights
    extern __shared__ __align__(16) char lds[];

    const int waves = blockDim.x / kWave, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
    const int i = lane_id() & 15, g = lane_id() >> 4;
    const int64_t n0 = int64_t(blockIdx.x) * 16;
    const T *w[NW], *x[MT];
#pragma unroll
    for (int q = 0; q < NW; ++q)
        w[q] = static_cast<const T*>(a.y.p[q]) + min(n0 + i, a.N - 1) * a.y.ld + g * E;
#pragma unroll
    for (int t = 0; t < MT; ++t)
        x[t] = static_cast<const T*>(a.x.p[0]) + min(int64_t(t * 16 + i), a.M - 1) * a.x.ld + g * E;

    f32x4 acc[NW][MT] = {};
    // This block's share of K in lines, and the whole ones of it.
    const int64_t all = (a.K + kLine - 1) / kLine, first = all * blockIdx.y / gridDim.y;
    const int64_t last = all * (blockIdx.y + 1) / gridDim.y, lines = min(last, a.K / kLine);
    // Batches of kFewLines lines, the next one's loads before this one's products.
    struct Batch {
        u32x4 w[kFewLines][2][NW], x[kFewLines][2][MT];
    };
    const auto load = [&](Batch& b, int64_t l) {
#pragma unroll
        for (int c = 0; c < kFewLines; ++c)
#pragma unroll
            for (int s = 0; s < 2; ++s) {
                const int64_t k = (l + c * waves) * kLine + s * 4 * E;
#pragma unroll
                for (int q = 0; q < NW; ++q) b.w[c][s][q] = load16<DT, kCached>(w[q] + k);
#pragma unroll
                for (int t = 0; t < MT; ++t) b.x[c][s][t] = load16<DT, kCached>(x[t] + k);
            }
    };
    const auto multiply = [&](const Batch& b) {
#pragma unroll
        for (int c = 0; c < kFewLines; ++c)
#pragma unroll
            for (int s = 0; s < 2; ++s)
#pragma unroll
                for (int t = 0; t < MT; ++t)
#pragma unroll
                    for (int q = 0; q < NW; ++q)
                        acc[q][t] = Mma<DT>::run(b.w[c][s][q], b.x[c][s][t], acc[q][t]);
    };
    const int64_t span = (kFewLines - 1) * waves, stride = kFewLines * waves;
    int64_t l = first + wave;
    if (l + span < lines) {
        Batch b0, b1;
        load(b0, l);
        for (;;) {
            l += stride;
            if (l + span >= lines) {
                multiply(b0);
                break;
            }
            load(b1, l);
            multiply(b0);
            l += stride;
            if (l + span >= lines) {
                multiply(b1);
                break;
            }
            load(b0, l);
            multiply(b1);
        }
    }
    // What is left: line by line, and the last one's end.
    for (; l < last; l += waves) {
#pragma unroll
        for (int s = 0; s < 2; ++s) {
            const int64_t k = l * kLine + s * 4 * E, left = a.K - k - g * E;
            u32x4 fw[NW];
#pragma unroll
            for (int q = 0; q < NW; ++q) fw[q] = load16_first<DT>(w[q] + k, left);
#pragma unroll
            for (int t = 0; t < MT; ++t) {
                const u32x4 fx = load16_first<DT>(x[t] + k, left);
#pragma unroll
                for (int q = 0; q < NW; ++q) acc[q][t] = Mma<DT>::run(fw[q], fx, acc[q][t]);
            }
        }
    }

    f32x4* const part = reinterpret_cast<f32x4*>(lds);  // [wave][q][t][lane]
#pragma unroll
    for (int q = 0; q < NW; ++q)
#pragma unroll
        for (int t = 0; t < MT; ++t)
            part[((wave * NW + q) * MT + t) * kWave + lane_id()] = acc[q][t];
    __syncthreads();
    if (wave >= MT) return;
    const int64_t m = wave * 16 + i, n = n0 + g * 4, left = a.N - n, at = m * a.N + n;
    f32x4 sum[NW] = {};
    for (int v = 0; v < waves; ++v)
#pragma unroll
        for (int q = 0; q < NW; ++q) sum[q] += part[((v * NW + q) * MT + wave) * kWave + lane_id()];
    if (m >= a.M) return;
    const auto put = [&](void* to, const float (&v)[4]) {
#pragma unroll
        for (int j = 0; j < 4; ++j)
            if (j < left) static_cast<T*>(to)[at + j] = static_cast<T>(v[j]);
    };
    float v[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) v[j] = sum[0][j];
    if constexpr (KIND == kGemmUp) {
        float u[4], h[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) u[j] = sum[NW - 1][j];
        gate_forward<DT>(a.act, a.slope, v, u, h);
        put(a.out[0], h);
        if (a.dg) {
            put(a.dg, v);
            put(a.du, u);
        }
    } else if (gridDim.y > 1) {
        float* const to = a.part + int64_t(blockIdx.y) * a.M * a.N + at;
#pragma unroll
        for (int j = 0; j < 4; ++j)
            if (j < left) to[j] = v[j];
    } else {
        put(a.out[0], v);
    }
}

template <int DT, int KIND, int MT>
void launch_few_tiles(GemmArgs a, hipStream_t st) {
    a.splits = KIND == kGemmDown ? plan_few(a.N, a.K, DT) : 1;
    constexpr int kLine = 128 / sizeof(typename Elem<DT>::T), NW = KIND == kGemmUp ? 2 : 1;
    const int64_t blocks = (a.N + 15) / 16, lines = (a.K + kLine - 1) / kLine;
    // Waves of a block: enough for about 2048 in all, each with a batch of
    // lines at least, and as many as there are tiles of tokens to finish.
    int waves = MT;
    while (waves < 8 && blocks * a.splits * waves < 2048 && waves * 2 * kFewLines * a.splits <= lines) waves *= 2;
    const size_t lds = static_cast<size_t>(waves) * NW * MT * kWave * sizeof(f32x4);
    few_kernel<DT, KIND, MT>
        <<<dim3(static_cast<uint32_t>(blocks), a.splits), waves * kWave, lds, st>>>(a);
    if (a.splits > 1) launch_join(DT, a, 1, st);
}

template <int DT, int KIND>
void launch_few_kind(const GemmArgs& a, hipStream_t st) {
    if (a.M <= 16) launch_few_tiles<DT, KIND, 1>(a, st);
    else if (a.M <= 32) launch_few_tiles<DT, KIND, 2>(a, st);
    else launch_few_tiles<DT, KIND, 4>(a, st);
}

template <int DT>
bool launch_few(GemmKind kind, const GemmArgs& a, hipStream_t st) {
    if (kind == kGemmUp) launch_few_kind<DT, kGemmUp>(a, st);
    else if (kind == kGemmDown) launch_few_kind<DT, kGemmDown>(a, st);
    else return false;
    return true;
}

}  // namespace iabn_impl
