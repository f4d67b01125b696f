// The plan of the experts' products: the M*k pairs (token, slot) sorted by expert,
// pairs of one expert in their own order (a counting sort, the same result
// whatever the order in which blocks run).
//
// Each wave has a contiguous part of the pairs.  It counts its experts in LDS;
// the counts of the waves, and of the blocks before this one, say where its
// pairs of an expert begin; then it goes through them again, 64 at a time, and a
// pair's place among those is the number of lanes before it with the same expert
// (found bit by bit of the expert's number).  Up to kPlanPairs pairs are one
// block and one launch; more are counted by a launch of their own, and every block
// adds up the counts before its own (blocks*E integers from the caches).  65536 pairs
// of 64 experts: 3 and 7 us (16 with one count on its way at a time and blocks of 256
// threads); 8 pairs 3.3, a launch.
#include "routed.h"

namespace iabn_impl {
namespace {

constexpr int kPlanThreads = 512, kPlanWaves = kPlanThreads / kWave;
constexpr int kPlanPairs = 2048;    // of a block, while there are fewer blocks than
constexpr int kMaxPlanBlocks = 256;

// Whether it is an expert at all (any other number: the pair is left out).
__device__ __forceinline__ bool routed(int e, int E) { return e >= 0 && e < E; }

// [P) of block b, wave w.
__device__ __forceinline__ void span_of(const PlanArgs& a, int wave, int& from, int& to) {
    const int64_t begin = int64_t(blockIdx.x) * a.span, end = min(begin + a.span, int64_t(a.P));
    const int64_t per = a.span / kPlanWaves;
    from = static_cast<int>(min(begin + wave * per, end));
    to = static_cast<int>(min(begin + (wave + 1) * per, end));
}

// Counts the experts of a wave's pairs in LDS; a lane has eight on their way.
__device__ __forceinline__ void count_span(const PlanArgs& a, int32_t* counts, int from, int to) {
    for (int base = from; base < to; base += 8 * kWave) {
        int e[8];
#pragma unroll
        for (int q = 0; q < 8; ++q) {
            const int i = base + q * kWave + static_cast<int>(lane_id());
            e[q] = i < to ? a.experts[i] : -1;
        }
#pragma unroll
        for (int q = 0; q < 8; ++q)
            if (routed(e[q], a.E)) atomicAdd(&counts[e[q]], 1);
    }
}

__global__ __launch_bounds__(kPlanThreads) void plan_count_kernel(PlanArgs a) {
    extern __shared__ int32_t counts[];  // [E]
    for (int e = threadIdx.x; e < a.E; e += kPlanThreads) counts[e] = 0;
    __syncthreads();
    int from, to;
    span_of(a, threadIdx.x / kWave, from, to);
    count_span(a, counts, from, to);
    __syncthreads();
    for (int e = threadIdx.x; e < a.E; e += kPlanThreads)
        a.counts[int64_t(blockIdx.x) * a.E + e] = counts[e];
}

// The sum over the lanes before this one; in `total` that over all.
__device__ __forceinline__ int wave_before(int v, int& total) {
    int sum = v;
#pragma unroll
    for (int d = 1; d < kWave; d *= 2) {
        const int o = __shfl_up(sum, d);
        if (static_cast<int>(lane_id()) >= d) sum += o;
    }
    total = __shfl(sum, kWave - 1);
    return sum - v;
}

__global__ __launch_bounds__(kPlanThreads) void plan_kernel(PlanArgs a) {
    extern __shared__ int32_t next[];  // [waves][E]: where the wave's next pair of e goes; [E]
    __shared__ int32_t wave_total[kPlanWaves];
    const int wave = threadIdx.x / kWave;
    int32_t* const own = next + wave * a.E;
    for (int i = threadIdx.x; i < kPlanWaves * a.E; i += kPlanThreads) next[i] = 0;
    __syncthreads();
    int from, to;
    span_of(a, wave, from, to);
    count_span(a, own, from, to);
    __syncthreads();
    // Each thread has `each` consecutive experts.
    constexpr int kEach = kMaxExperts / kPlanThreads;
    const int each = (a.E + kPlanThreads - 1) / kPlanThreads, e0 = threadIdx.x * each;
    int all[kEach], before[kEach], sum = 0;
#pragma unroll
    for (int j = 0; j < kEach; ++j) {
        all[j] = before[j] = 0;
        const int e = e0 + j;
        if (j >= each || e >= a.E) continue;
        if (a.blocks == 1) {
            for (int w = 0; w < kPlanWaves; ++w) all[j] += next[w * a.E + e];
        } else {
            // (Sixteen loads on their way at a time.)
            for (int b0 = 0; b0 < a.blocks; b0 += 16) {
                int n[16];
#pragma unroll
                for (int i = 0; i < 16; ++i) n[i] = b0 + i < a.blocks ? a.counts[int64_t(b0 + i) * a.E + e] : 0;
#pragma unroll
                for (int i = 0; i < 16; ++i) {
                    before[j] += b0 + i < static_cast<int>(blockIdx.x) ? n[i] : 0;
                    all[j] += n[i];
                }
            }
        }
        sum += all[j];
    }
    int total;
    int at = wave_before(sum, total);
    if (lane_id() == 0) wave_total[wave] = total;
    int32_t* const sizes = next + kPlanWaves * a.E;
#pragma unroll
    for (int j = 0; j < kEach; ++j)
        if (j < each && e0 + j < a.E) sizes[e0 + j] = all[j];
    __syncthreads();
    // The experts by size, the largest first (of equal ones the lower number), a wave
    // for each: its place is the number of those before it.  Of few pairs, which one
    // block counts, they stay in their order.
    for (int e = blockIdx.x * kPlanWaves + wave; e < a.E; e += a.blocks * kPlanWaves) {
        const int mine = sizes[e];
        int rank = a.blocks == 1 ? e : 0;
        if (a.blocks > 1)
            for (int base = 0; base < a.E; base += kWave) {
                const int i = base + static_cast<int>(lane_id()), n = i < a.E ? sizes[i] : -1;
                rank += __popcll(__ballot(n > mine || (n == mine && i < e)));
            }
        if (lane_id() == 0) a.by_size[rank] = e;
    }
    for (int w = 0; w < wave; ++w) at += wave_total[w];
#pragma unroll
    for (int j = 0; j < kEach; ++j) {
        const int e = e0 + j;
        if (j >= each || e >= a.E) continue;
        if (blockIdx.x == 0) a.offsets[e] = at;
        int to_next = at + before[j];
        for (int w = 0; w < kPlanWaves; ++w) {
            const int n = next[w * a.E + e];
            next[w * a.E + e] = to_next;
            to_next += n;
        }
        at += all[j];
        if (blockIdx.x == 0 && e == a.E - 1) a.offsets[a.E] = at;
    }
    __syncthreads();
    int ahead = from + static_cast<int>(lane_id()) < to ? a.experts[from + static_cast<int>(lane_id())] : -1;
    for (int base = from; base < to; base += kWave) {  // (uniform over the wave)
        const int i = base + static_cast<int>(lane_id());
        const int e = ahead;
        ahead = i + kWave < to ? a.experts[i + kWave] : -1;
        const bool is = routed(e, a.E);
        uint64_t same = __ballot(is);
        for (int bit = 1; bit < a.E; bit *= 2) {
            const uint64_t have = __ballot((e & bit) != 0);
            same &= e & bit ? have : ~have;
        }
        const uint64_t lower = same & ((uint64_t(1) << lane_id()) - 1);
        int place = -1;
        if (is) place = own[e] + __popcll(lower);
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        __builtin_amdgcn_wave_barrier();
        if (is && lower == 0) own[e] += __popcll(same);
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        __builtin_amdgcn_wave_barrier();
        if (i < to) a.place[i] = place;
        if (is) a.order[place] = i;
    }
}

int64_t blocks_of(int64_t P) {
    const int64_t want = (P + kPlanPairs - 1) / kPlanPairs;
    return want < 1 ? 1 : want < kMaxPlanBlocks ? want : kMaxPlanBlocks;
}

}  // namespace

int64_t plan_size(int64_t P, int64_t E) {
    const int64_t blocks = blocks_of(P);
    return E + 1 + 2 * P + E + (blocks > 1 ? blocks * E : 0);
}

PlanArgs plan_of(int64_t P, int64_t E, int32_t* plan) {
    PlanArgs a = {};
    a.P = static_cast<int32_t>(P), a.E = static_cast<int32_t>(E);
    a.offsets = plan;
    a.order = plan + E + 1;
    a.place = a.order + P;
    a.by_size = a.place + P;
    a.counts = a.by_size + E;
    const int64_t blocks = blocks_of(P), per = (P + blocks - 1) / blocks;
    a.span = static_cast<int32_t>((per + kPlanThreads - 1) / kPlanThreads * kPlanThreads);
    a.blocks = static_cast<int32_t>(P == 0 ? 1 : (P + a.span - 1) / a.span);
    return a;
}

void launch_plan(const PlanArgs& a, hipStream_t st) {
    if (a.blocks > 1) plan_count_kernel<<<a.blocks, kPlanThreads, a.E * sizeof(int32_t), st>>>(a);
    plan_kernel<<<a.blocks, kPlanThreads, (kPlanWaves + 1) * a.E * sizeof(int32_t), st>>>(a);
}

}  // namespace iabn_impl
