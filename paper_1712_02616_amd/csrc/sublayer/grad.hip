// The norm over a list of gradients, and the gradients clipped to it:
//
//   norm = sqrt(sum over all of g^2),   out = g*min(1, max_norm/(norm + 1e-6))
//
// A block takes a piece of one tensor, which it finds among its launch's pieces.
// Squares are formed and added in 64 bits, so that neither an overflow of a
// square nor the length of a sum costs digits (two 64-bit instructions an element,
// a third of the time that its bytes take); the pieces' sums are added up in
// their order by one more block.  403 million bf16 values: 132 us and 4 to join, 6.1
// TB/s, and 277 to clip, 5.8 of which the caches have a part.  198 thousand fp32
// ones: 3.7, 1.5 and 3.8 us, three launches.
#include "routed.h"

namespace iabn_impl {
namespace {

// The tensor of piece b, and the piece [from, to) of it.
__device__ __forceinline__ int tensor_of(const GradArgs& a, int b, int64_t& from, int64_t& to) {
    int lo = 0, hi = a.count;  // first[lo] <= b < first[hi]
    while (hi - lo > 1) {
        const int mid = (lo + hi) / 2;
        if (a.first[mid] <= b) lo = mid;
        else hi = mid;
    }
    from = int64_t(b - a.first[lo]) * a.piece;
    to = min(from + a.piece, a.n[lo]);
    return lo;
}

__device__ __forceinline__ double block_sum(double v, double (&slots)[kWaves]) {
#pragma unroll
    for (int d = 1; d < kWave; d *= 2) v += __shfl_xor(v, d);
    if (lane_id() == 0) slots[threadIdx.x / kWave] = v;
    __syncthreads();
    double sum = 0.0;
#pragma unroll
    for (int w = 0; w < kWaves; ++w) sum += slots[w];
    return sum;
}

template <int DT>
__device__ __forceinline__ double squares(const void* p, int64_t from, int64_t to) {
    double sum = 0.0;
    for (int64_t at = from + int64_t(threadIdx.x) * kChunk; at < to; at += kThreads * kChunk) {
        float v[kChunk];
        widen<DT>(load_chunk<DT, kCached>(p, at, static_cast<int>(min(to - at, int64_t(kChunk)))), v);
#pragma unroll
        for (int j = 0; j < kChunk; ++j) {
            const double d = v[j];
            sum = fma(d, d, sum);
        }
    }
    return sum;
}

__global__ __launch_bounds__(kThreads) void grad_norm_kernel(GradArgs a) {
    __shared__ double slots[kWaves];
    int64_t from, to;
    const int t = tensor_of(a, blockIdx.x, from, to);
    double sum;
    switch (a.dtype[t]) {
        case IABN_F32: sum = squares<IABN_F32>(a.in[t], from, to); break;
        case IABN_F16: sum = squares<IABN_F16>(a.in[t], from, to); break;
        default: sum = squares<IABN_BF16>(a.in[t], from, to); break;
    }
    sum = block_sum(sum, slots);
    if (threadIdx.x == 0) a.part[blockIdx.x] = sum;
}

__global__ __launch_bounds__(kThreads) void grad_join_kernel(const double* part, int64_t n, float* norm) {
    __shared__ double slots[kWaves];
    double sum = 0.0;
    constexpr int kAhead = 8;  // on their way at a time
    for (int64_t i = threadIdx.x; i < n; i += kAhead * kThreads) {
        double v[kAhead];
#pragma unroll
        for (int q = 0; q < kAhead; ++q) v[q] = i + q * kThreads < n ? part[i + q * kThreads] : 0.0;
#pragma unroll
        for (int q = 0; q < kAhead; ++q) sum += v[q];
    }
    sum = block_sum(sum, slots);
    if (threadIdx.x == 0) *norm = static_cast<float>(sqrt(sum));
}

// By factor*2^power.
template <int DT>
__device__ __forceinline__ void scale(const void* in, void* out, int64_t from, int64_t to, float factor, int power) {
    for (int64_t at = from + int64_t(threadIdx.x) * kChunk; at < to; at += kThreads * kChunk) {
        const int n = static_cast<int>(min(to - at, int64_t(kChunk)));
        float v[kChunk];
        widen<DT>(load_chunk<DT, kStream>(in, at, n), v);
#pragma unroll
        for (int j = 0; j < kChunk; ++j) v[j] = ldexpf(v[j] * factor, power);
        store_chunk<DT, kStream>(out, at, n, v);
    }
}

__global__ __launch_bounds__(kThreads) void grad_clip_kernel(GradArgs a) {
    int64_t from, to;
    // (From the last piece on: the caches hold what the norm read last.  403 million
    // bf16 values: 277 us, and 132 for the norm; 309 and 118 where the norm's loads
    // are non-temporal.)
    const int t = tensor_of(a, gridDim.x - 1 - blockIdx.x, from, to);
    const double norm = *a.norm, limit = a.max_norm;
    // (No limit clips nothing, an infinite norm neither; a NaN stays one.)
    const double ratio = limit == __builtin_inf() && norm == norm ? 1.0 : limit / (norm + 1e-6);
    // (Below 2^-126 an fp32 factor would have fewer digits: the power of two is apart.)
    int power = 0;
    const double digits = ratio > 0.0 && ratio < 0x1p-126 ? frexp(ratio, &power) : ratio;
    const float factor = ratio >= 1.0 ? 1.0f : static_cast<float>(digits);
    if (factor == 1.0f && power == 0 && a.in[t] == a.out[t]) return;
    switch (a.dtype[t]) {
        case IABN_F32: scale<IABN_F32>(a.in[t], a.out[t], from, to, factor, power); break;
        case IABN_F16: scale<IABN_F16>(a.in[t], a.out[t], from, to, factor, power); break;
        default: scale<IABN_BF16>(a.in[t], a.out[t], from, to, factor, power); break;
    }
}

}  // namespace

void launch_grad_norm(const GradArgs& a, hipStream_t st) {
    grad_norm_kernel<<<a.first[a.count], kThreads, 0, st>>>(a);
}
void launch_grad_join(const double* part, int64_t n, float* norm, hipStream_t st) {
    grad_join_kernel<<<1, kThreads, 0, st>>>(part, n, norm);
}
void launch_grad_clip(const GradArgs& a, hipStream_t st) {
    grad_clip_kernel<<<a.first[a.count], kThreads, 0, st>>>(a);
}

}  // namespace iabn_impl
