// How the gated feed-forward block's products are cut (the tiles and the split
// of the sum over k), and the kernel that joins a split sum.
#include "ffn.h"

namespace iabn_impl {
namespace {

constexpr int64_t kCUs = 256;
constexpr int kMaxSplits = 16;

int64_t div_up(int64_t a, int64_t b) { return (a + b - 1) / b; }

// The time of a step of 128 bytes of K with 1, 2, 3 and 4 blocks on a CU, and
// of each block's ends (us, measured at full grids of each).  16-bit: the
// larger tile reads half of LDS per product but holds a CU alone; two blocks
// of 128x128 hide each other's waits (0.68 us for both, 0.67 for one).  fp32
// is bound by the matrix cores at every size: the tiles matter where they do
// not fill the last round.  Through registers, 128x128 is no choice: 1.5, 3.0, 4.4,
// 5.9 us a step (fp32 2.65, 5.2, 7.8, 10.4), more than two blocks of 64x128 at every
// number of blocks, and the same ends.
struct TileCost {
    float step[4], ends;
};
// [fp32][direct][tile]
constexpr TileCost kCost[2][2][4] = {
    {{{{0, 0, 0, 0}, 0}, {{0, 0, 0, 0}, 0}, {{1.1f, 1.3f, 2.0f, 2.6f}, 1}, {{0.9f, 1.1f, 1.4f, 2.2f}, 0.5f}},
     {{{1.27f, 2.54f, 3.81f, 5.08f}, 8}, {{0.67f, 0.68f, 1.36f, 1.4f}, 1.6f}, {{0.32f, 0.55f, 0.75f, 1.16f}, 0.8f}, {{0.26f, 0.45f, 0.68f, 0.87f}, 0.4f}}},
    {{{{0, 0, 0, 0}, 0}, {{0, 0, 0, 0}, 0}, {{1.6f, 2.6f, 4.8f, 5.0f}, 2}, {{1.0f, 1.6f, 2.25f, 3.2f}, 1}},
     {{{0, 0, 0, 0}, 0}, {{2.05f, 3.7f, 7.2f, 7.4f}, 4}, {{1.1f, 1.93f, 2.8f, 3.9f}, 2}, {{0.63f, 1.02f, 1.5f, 1.95f}, 1}}}};
constexpr float kGatingEnds = 3.0f;  // kGemmDh's end is so much longer
// 16-bit rows at odd addresses, through registers: the loads are what a step
// takes, and a strided operand's are so much slower ((1777, 4003 -> 1501) fp16
// dx: 211 us in 64x128 tiles of four splits, 511 in 32x128 ones of one).
constexpr float kStridedLoads = 2.5f;
// Joining split sums: a launch, and the sums written and read.
constexpr float kJoinUs = 3.0f, kJoinBytesPerUs = 4e6f;

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

GemmPlan plan_gemm(int dtype, GemmKind kind, bool direct, int64_t M, int64_t N, int64_t K, int products) {
    const int64_t step = dtype == IABN_F32 ? 32 : 64;
    const int64_t steps = div_up(K, step) * (kind == kGemmDx ? 2 : 1);
    const bool splittable = kind != kGemmUp && kind != kGemmDh;
    GemmPlan best = {kTile128, 1};
    float best_us = 0.0f;
    for (TileSize t : {kTile256, kTile128, kTile64, kTile32}) {
        const TileCost& cost = kCost[dtype == IABN_F32][direct][t];
        if (cost.ends == 0.0f) continue;
        const int64_t tm = t == kTile256 ? 256 : t == kTile128 ? 128 : t == kTile64 ? 64 : 32;
        const int64_t tn = (t == kTile256 ? 256 : 128) / (kind == kGemmUp ? 2 : 1);
        const int64_t tiles = div_up(M, tm) * div_up(N, tn) * products;
        for (int s = 1; s <= (splittable ? kMaxSplits : 1) && s <= steps; s *= 2) {
            const int64_t on_cu = div_up(tiles * s, kCUs);  // blocks that the busiest CU gets
            const float full = static_cast<float>((on_cu - 1) / 4);
            const float slow = dtype != IABN_F32 && !direct && kind >= kGemmDh ? kStridedLoads : 1.0f;
            const float per_step = slow * (full * cost.step[3] + cost.step[(on_cu - 1) % 4]);
            const float ends = cost.ends * (kind == kGemmDh ? kGatingEnds : 1.0f);
            float us = static_cast<float>(div_up(steps, s)) * per_step + static_cast<float>(on_cu) * ends;
            if (s > 1) us += kJoinUs + 8.0f * s * M * N * products / kJoinBytesPerUs;
            if (best_us == 0.0f || us < best_us) {
                best_us = us;
                best = {t, s};
            }
        }
    }
    return best;
}

// Blocks of 16 columns over K, for few tokens: where there are fewer of them
// than CUs, K is split for about two blocks a CU, of 16 lines of 128 bytes at
// least ((24 tokens, 8192 -> 2048) fp16: 20.3 us -> 12.1 and 3.9 to join).
int plan_few(int64_t N, int64_t K, int dtype) {
    const int64_t blocks = div_up(N, 16), lines = div_up(K, dtype == IABN_F32 ? 32 : 64);
    if (blocks >= kCUs * 3 / 4) return 1;
    int64_t s = kCUs * 2 / blocks;
    if (s > kMaxSplits) s = kMaxSplits;
    if (s > lines / 16) s = lines / 16;
    return s < 2 ? 1 : static_cast<int>(s);
}

size_t part_bytes(int dtype, GemmKind kind, int64_t M, int64_t N, int64_t K, int products) {
    if (M == 0 || N == 0 || K == 0) return 0;
    int splits = 1;
    if (few_rows(kind, M)) {
        splits = plan_few(N, K, dtype);
    } else {
        for (bool direct : {false, true}) {
            const int s = plan_gemm(dtype, kind, direct, M, N, K, products).splits;
            splits = splits < s ? s : splits;
        }
    }
    return splits > 1 ? static_cast<size_t>(splits) * products * M * N * sizeof(float) : 0;
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
