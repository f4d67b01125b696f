// Routed experts: how their products are cut, and the kernels that join the rows
// of a token's pairs.
#include "checks.h"
#include "groups.h"

namespace iabn_impl {
namespace {

constexpr int64_t kCUs = 256;
constexpr int kMaxSplits = 16;

// (A launch holds fewer than 2^32 threads.)
uint32_t blocks_for(int64_t want) { return static_cast<uint32_t>(want < 1 << 22 ? want : 1 << 22); }

// A thread has 8 columns of a token; the slots are added in their order.  Bound by the
// terms' traffic: 4096 tokens' 8 terms of 2048, bf16, 35 us for 218 MB, 6.2 TB/s; one
// token's, in fp32, 3.8 us (5.2 with one slot on its way at a time).
template <int DT, bool FEW>
__global__ __launch_bounds__(kThreads) void combine_kernel(CombineArgs a, int chunks) {
    constexpr int kSlots = 4;
    for (int64_t c = int64_t(blockIdx.x) * kThreads + threadIdx.x; c < a.M * chunks; c += int64_t(gridDim.x) * kThreads) {
        const int64_t t = c / chunks, col = (c - t * chunks) * kChunk;
        const int n = static_cast<int>(min(a.C - col, int64_t(kChunk)));
        float sum[kChunk] = {};
        for (int s0 = 0; s0 < a.k; s0 += kSlots) {
            // The places, then the terms of several slots on their way together.
            uint32_t p[kSlots];
            float w[kSlots];
            Terms<FEW ? IABN_F32 : DT> term[kSlots];
#pragma unroll
            for (int q = 0; q < kSlots; ++q) {
                p[q] = s0 + q < a.k ? static_cast<uint32_t>(a.place[t * a.k + s0 + q]) : 0xFFFFFFFFu;
                w[q] = FEW && s0 + q < a.k ? a.weights[t * a.k + s0 + q] : 1.0f;
            }
            for (int split = 0; split < (FEW ? a.splits : 1); ++split) {
#pragma unroll
                for (int q = 0; q < kSlots; ++q)
                    term[q].load(a.terms, a.low, (int64_t(split) * a.P + p[q]) * a.C + col,
                                 p[q] < static_cast<uint32_t>(a.P) ? n : 0);
#pragma unroll
                for (int q = 0; q < kSlots; ++q) {
                    float v[kChunk];
                    term[q].get(v);
#pragma unroll
                    for (int j = 0; j < kChunk; ++j)
                        sum[j] = p[q] < static_cast<uint32_t>(a.P) ? FEW ? fmaf(w[q], v[j], sum[j]) : sum[j] + v[j] : sum[j];
                }
            }
        }
        store_chunk<DT, kCached>(a.y, t * a.C + col, n, sum);
    }
}

// 16 lanes have a pair.  (65536 pairs of 16 dots: 4.7 us.)
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

// By the tokens, which no expert has more rows than (where none has it twice).  Few
// tokens' kernels and tiles take (us, forward, 16 / 40 / 56 / 64 tokens): bf16 8 of 64
// experts (2048 -> 1024) 143 / 161 / 175 / 181 and 147 / 162 / 164 / 164; 2 of 8 (2048
// -> 4096) 95 / 97 / 104 / 113 and 128 / 117 / 118 / 132; fp16 4 of 32 (1024 -> 2048) 81
// / 85 / 91 / 95 and 86 / 90 / 91 / 91; fp32 2 of 7 (1000 -> 731) 30 / 39 / 40 / 69 and
// 51 each.  One token of the first: 32 and 48.  What is faster goes by the rows of an
// expert and its weights' bytes; one limit on tokens lies between: from 40 to 56
// tokens the tiles would take up to 11 us less of the first, above it the few tokens'
// kernels up to 19 less of the second (at 64).
constexpr int64_t kFewTokens = 56;
bool few_pairs(int64_t M) { return M <= kFewTokens; }

// Blocks of 16 columns over K: split like those of one matrix (plan_few), where they
// are fewer than three quarters of the CUs.
int plan_grouped_few(int64_t P, int64_t E, int64_t N, int64_t K, int dtype) {
    const int64_t blocks = div_up(N, 16) * (E < P ? E : P), lines = div_up(K, dtype == IABN_F32 ? 32 : 64);
    if (blocks >= kCUs * 3 / 4) return 1;
    int64_t s = kCUs * 2 / blocks;
    if (s > kMaxSplits) s = kMaxSplits;
    if (s > lines / 16) s = lines / 16;
    return s < 2 ? 1 : static_cast<int>(s);
}

}  // namespace iabn_impl
