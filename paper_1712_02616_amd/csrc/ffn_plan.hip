// How the gated feed-forward block's products are cut (the tiles and the split
// of the sum over k), and the kernel that joins a split sum.
#include "ffn.h"

namespace iabn_impl {
namespace {

constexpr int64_t kCUs = 256;

int64_t div_up(int64_t a, int64_t b) { return (a + b - 1) / b; }

int64_t tiles(TileSize t, GemmKind kind, int64_t M, int64_t N, int products) {
    const int64_t tm = t == kTile256 ? 256 : t == kTile128 ? 128 : 64;
    const int64_t tn = (t == kTile256 ? 256 : 128) / (kind == kGemmUp ? 2 : 1);
    return div_up(M, tm) * div_up(N, tn) * products;
}

template <int DT>
__global__ __launch_bounds__(kThreads) void join_kernel(GemmArgs a) {
    const int64_t n = a.M * a.N, c = int64_t(blockIdx.x) * kThreads + threadIdx.x;
    const int64_t at = c * kChunk;
    if (at >= n) return;
    const int inside = static_cast<int>(min(n - at, int64_t(kChunk)));
    const int z = blockIdx.z;
    float sum[kChunk] = {};
    for (int s = 0; s < a.splits; ++s) {
        float v[kChunk];
        widen<IABN_F32>(load_chunk<IABN_F32, kCached>(a.part, (int64_t(s) * gridDim.z + z) * n + at, inside), v);
#pragma unroll
        for (int j = 0; j < kChunk; ++j) sum[j] += v[j];
    }
    store_chunk<DT, kCached>(z ? a.out[1] : a.out[0], at, inside, sum);
}

}  // namespace

TileSize gemm_tile(int, GemmKind kind, int64_t M, int64_t N, int products) {
    if (tiles(kTile256, kind, M, N, products) >= 192) return kTile256;
    if (tiles(kTile128, kind, M, N, products) >= 192) return kTile128;
    return kTile64;
}

int gemm_splits(int dtype, GemmKind kind, int64_t M, int64_t N, int64_t K, int products) {
    if (kind == kGemmUp || kind == kGemmDh || M == 0 || N == 0) return 1;
    const int64_t step = dtype == IABN_F32 ? 32 : 64;  // of K
    int64_t blocks, least;                             // steps of a split, at least
    if (few_rows(kind, M)) {
        blocks = div_up(N, 16);
        least = 16;
    } else {
        blocks = tiles(gemm_tile(dtype, kind, M, N, products), kind, M, N, products);
        least = 8;
    }
    if (blocks >= kCUs * 3 / 4) return 1;
    int64_t s = kCUs * 2 / blocks;
    if (s > kMaxSplits) s = kMaxSplits;
    if (s > div_up(K, step) / least) s = div_up(K, step) / least;
    return s < 2 ? 1 : static_cast<int>(s);
}

void launch_join(int dtype, const GemmArgs& a, int products, hipStream_t st) {
    const dim3 grid(static_cast<uint32_t>(div_up(div_up(a.M * a.N, kChunk), kThreads)), 1, products);
    switch (dtype) {
        case IABN_F32: join_kernel<IABN_F32><<<grid, kThreads, 0, st>>>(a); break;
        case IABN_F16: join_kernel<IABN_F16><<<grid, kThreads, 0, st>>>(a); break;
        default: join_kernel<IABN_BF16><<<grid, kThreads, 0, st>>>(a); break;
    }
}

}  // namespace iabn_impl
