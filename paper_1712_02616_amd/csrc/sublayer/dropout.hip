// Dropout whose mask is a function of (seed, offset, place): y = D(x).
//
// Bound by HBM traffic, 2 bytes in and 2 out per 16-bit element, as long as one
// generator call (20 products of 32x32 bits) serves 8 elements.  A thread moves
// one chunk of 8: its 16 bytes are one access, and its group's bits need no
// exchange.  (32768, 2048) bf16: 45 us, 5.9 TB/s; (64, 1024) fp16 2.4 us, a
// launch.
#include "sublayer.h"

namespace iabn_impl {
namespace {

constexpr int64_t kMaxBlocks = 1 << 22;

template <int DT>
__global__ __launch_bounds__(kThreads) void dropout_kernel(const void* x, void* y, int64_t groups,
                                                           int C, int chunks, Dropout d) {
    for (int64_t g = int64_t(blockIdx.x) * kThreads + threadIdx.x; g < groups;
         g += int64_t(gridDim.x) * kThreads) {
        int64_t at = g * kChunk;
        int n = kChunk;
        if (C % kChunk != 0) {  // uniform
            const int64_t row = g / chunks;
            const int c = static_cast<int>(g - row * chunks);
            at = row * C + c * kChunk;
            n = min(kChunk, C - c * kChunk);
        }
        const auto raw = load_chunk<DT, kStream>(x, at, n);
        float v[kChunk];
        widen<DT>(raw, v);
        drop_group(d, static_cast<uint64_t>(g), v);
        store_chunk<DT, kStream>(y, at, n, v);
    }
}

template <typename T>
__global__ __launch_bounds__(kThreads) void zero_kernel(T* p, int64_t n) {
    for (int64_t i = int64_t(blockIdx.x) * kThreads + threadIdx.x; i < n;
         i += int64_t(gridDim.x) * kThreads)
        p[i] = 0;
}

}  // namespace

void launch_zero(void* p, int64_t bytes, hipStream_t st) {
    const int64_t n = bytes / 2, blocks = (n + kThreads - 1) / kThreads;
    if (n == 0) return;
    zero_kernel<<<dim3(static_cast<uint32_t>(blocks < 4096 ? blocks : 4096)), kThreads, 0, st>>>(
        static_cast<uint16_t*>(p), n);
}

bool launch_dropout(int dtype, const void* x, void* y, int64_t R, int C, const Dropout& d,
                    hipStream_t st) {
    const int chunks = chunks_of(C);
    const int64_t groups = R * chunks, blocks = (groups + kThreads - 1) / kThreads;
    // (A launch holds fewer than 2^32 threads.)
    const dim3 grid(static_cast<uint32_t>(blocks < kMaxBlocks ? blocks : kMaxBlocks));
    switch (dtype) {
        case IABN_F32:
            dropout_kernel<IABN_F32><<<grid, kThreads, 0, st>>>(x, y, groups, C, chunks, d);
            return true;
        case IABN_F16:
            dropout_kernel<IABN_F16><<<grid, kThreads, 0, st>>>(x, y, groups, C, chunks, d);
            return true;
        case IABN_BF16:
            dropout_kernel<IABN_BF16><<<grid, kThreads, 0, st>>>(x, y, groups, C, chunks, d);
            return true;
        default: return false;
    }
}

}  // namespace iabn_impl
