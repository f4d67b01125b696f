// Routed experts: how their products are cut, and the kernels that join the rows
// of a token's pairs.
#include "checks.h"
#include "groups.h"

namespace iabn_impl {
namespace {

// (A launch holds fewer than 2^32 threads.)
uint32_t blocks_for(int64_t want) { return static_cast<uint32_t>(want < 1 << 22 ? want : 1 << 22); }

// A thread has 8 columns of a token; the slots are added in their order.  Bound
// by the terms' traffic.
template <int DT, bool FEW>
__global__ __launch_bounds__(kThreads) void combine_kernel(CombineArgs a, int chunks) {
    constexpr int TERM = FEW ? IABN_F32 : DT;
    for (int64_t c = int64_t(blockIdx.x) * kThreads + threadIdx.x; c < a.M * chunks; c += int64_t(gridDim.x) * kThreads) {
        const int64_t t = c / chunks, col = (c - t * chunks) * kChunk;
        const int n = static_cast<int>(min(a.C - col, int64_t(kChunk)));
        float sum[kChunk] = {};
        for (int s = 0; s < a.k; ++s) {
            const uint32_t p = static_cast<uint32_t>(a.place[t * a.k + s]);
            if (p >= static_cast<uint32_t>(a.P)) continue;
            if constexpr (FEW) {
                const float w = a.weights[t * a.k + s];
                float term[kChunk] = {};
                for (int q = 0; q < a.splits; ++q) {
                    float v[kChunk];
                    widen<TERM>(load_chunk<TERM, kCached>(a.terms, (int64_t(q) * a.P + p) * a.C + col, n), v);
#pragma unroll
                    for (int j = 0; j < kChunk; ++j) term[j] += v[j];
                }
#pragma unroll
                for (int j = 0; j < kChunk; ++j) sum[j] = fmaf(w, term[j], sum[j]);
            } else {
                float v[kChunk];
                widen<TERM>(load_chunk<TERM, kStream>(a.terms, p * a.C + col, n), v);
#pragma unroll
                for (int j = 0; j < kChunk; ++j) sum[j] += v[j];
            }
        }
        store_chunk<DT, kCached>(a.y, t * a.C + col, n, sum);
    }
}

// 16 lanes have a pair.
__global__ __launch_bounds__(kThreads) void dots_kernel(const float* dots, const int32_t* place, float* dweights,
                                                        int64_t P, int64_t n) {
    constexpr int kPairs = kThreads / 16;  // of a block
    for (int64_t base = int64_t(blockIdx.x) * kPairs; base < P; base += int64_t(gridDim.x) * kPairs) {
        const int64_t own = base + threadIdx.x / 16, i = min(own, P - 1);
        const uint32_t p = static_cast<uint32_t>(place[i]);
        float sum = 0.0f;
        if (p < static_cast<uint32_t>(P))
            for (int64_t j = threadIdx.x % 16; j < n; j += 16) sum += dots[p * n + j];
        sum += dpp_f32<0xB1, 0xF>(sum);
        sum += dpp_f32<0x4E, 0xF>(sum);
        sum += dpp_f32<0x141, 0xF>(sum);
        sum += dpp_f32<0x140, 0xF>(sum);
        if (own < P && threadIdx.x % 16 == 0) dweights[i] = sum;
    }
}

template <int DT>
void combine(const CombineArgs& a, hipStream_t st) {
    const int64_t chunks = div_up(a.C, kChunk);
    const dim3 grid(blocks_for(div_up(a.M * chunks, kThreads)));
    if (a.weights) combine_kernel<DT, true><<<grid, kThreads, 0, st>>>(a, static_cast<int>(chunks));
    else combine_kernel<DT, false><<<grid, kThreads, 0, st>>>(a, static_cast<int>(chunks));
}

}  // namespace

void launch_combine(int dtype, const CombineArgs& a, hipStream_t st) {
    switch (dtype) {
        case IABN_F32: combine<IABN_F32>(a, st); break;
        case IABN_F16: combine<IABN_F16>(a, st); break;
        default: combine<IABN_BF16>(a, st); break;
    }
}

void launch_dots(const float* dots, const int32_t* place, float* dweights, int64_t P, int64_t n, hipStream_t st) {
    dots_kernel<<<dim3(blocks_for(div_up(P, kThreads / 16))), kThreads, 0, st>>>(dots, place, dweights, P, n);
}

bool few_pairs(int64_t M, int64_t, int64_t) { return M <= kFewRows; }

int plan_grouped_few(int64_t P, int64_t E, int64_t N, int64_t K, int dtype) {
    const int64_t blocks = div_up(N, 16) * (E < P ? E : P), lines = div_up(K, dtype == IABN_F32 ? 32 : 64);
    if (blocks >= 192) return 1;
    int64_t s = 512 / blocks;
    if (s > 16) s = 16;
    if (s > lines / 16) s = lines / 16;
    return s < 2 ? 1 : static_cast<int>(s);
}

}  // namespace iabn_impl
