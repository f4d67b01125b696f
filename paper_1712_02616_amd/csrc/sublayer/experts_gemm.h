// The products of routed experts: how those of ffn_gemm.h and ffn_few.h are
// launched over groups of rows.
//
// The number of rows that an expert has is not known on the host, so that a launch
// has as many blocks as the worst division of the pairs needs (for each expert one
// tile that is not full); those past the last tile end at once.
//
// Fetch-bound as much as by the matrix cores (busy in 0.38-0.53 of the cycles): an
// expert's weights serve few rows, so that more of a step's 64 KB comes from HBM.
// With 512 rows of each of 64 experts, up projection (2048 -> 2x1024) bf16, 254 us
// before the fetch was cut in two; 239 without the products, 206 without the fetches, 216
// without the results.  bf16, 8192 tokens, 8 of 64 experts of skewed popularity, 2048
// -> 1024 (fastest and median of 10 passes): dh 400 and 415 us, dW 310 and 710 (down;
// gate and up), 330 and 760, dx 540 and 580: 0.69, 0.89, 0.77, 1.0 PFLOP/s; the
// forward of 4096 tokens 315 and 365 us (up), 213 and 250 (down): 0.87, 0.65.  fp32,
// 333 tokens, 2 of 7 experts, 1000 -> 731: 43 and 22 us, 46 TFLOP/s, one block of four
// waves on a CU.  Few tokens (HBM): one token, 8 of 64 experts, 13.5 and 8.7 us, 5.0
// and 3.9 TB/s; 24 tokens, 4 of 32, 1200 hidden, fp16 57 and 33 us, 5.2 and 4.7.
#pragma once

#include "ffn_few.h"
#include "ffn_gemm.h"

namespace iabn_impl {

// Tiles of `tile` rows for P pairs over E experts, at most.
inline int64_t most_tiles(int64_t P, int64_t E, int64_t tile) { return P / tile + (E < P ? E : P); }

template <int DT, int KIND, int TM, int TN, int WAVES_M, int WAVES_N, bool DMA>
void launch_group_tiles(const GroupArgs& a, int products, hipStream_t st) {
    constexpr int kCols = KindOf<KIND>::kDual ? TN / 2 : TN;
    constexpr bool kDw = KindOf<KIND>::kBase == kGemmDw;
    const int64_t tn = (a.N + kCols - 1) / kCols, tm = kDw ? (a.M + TM - 1) / TM : most_tiles(a.P, a.E, TM);
    const int64_t blocks = kDw ? a.E * tm * tn : tm * tn;
    gemm_kernel<DT, KIND, TM, TN, WAVES_M, WAVES_N, DMA>
        <<<dim3(static_cast<uint32_t>(blocks), 1, products), WAVES_M * WAVES_N * kWave, 0, st>>>(
            a, static_cast<int>(tm), static_cast<int>(tn));
}

template <int DT, int KIND, bool DMA>
void launch_group_planned(const GroupArgs& a, int products, hipStream_t st) {
    switch (plan_grouped(DT, KindOf<KIND>::kBase, DMA, a.P, a.E, a.M, a.N, a.K, products)) {
        case kTile256:
            if constexpr (DMA && DT != IABN_F32) launch_group_tiles<DT, KIND, 256, 256, 2, 4, DMA>(a, products, st);
            break;
        case kTile128:
            if constexpr (DMA) launch_group_tiles<DT, KIND, 128, 128, 2, 2, DMA>(a, products, st);
            break;
        case kTile64: launch_group_tiles<DT, KIND, 64, 128, 2, 2, DMA>(a, products, st); break;
        case kTile32: launch_group_tiles<DT, KIND, 32, 128, 2, 2, DMA>(a, products, st); break;
    }
}

// tokens: rows of the matrix that an operand is gathered from; 0 where it is not.
// A gathered operand's rows have 32-bit offsets, and its last chunk of a row may
// not reach into the next one (the matrix may end there).
template <int DT>
bool group_fetchable(const Operand& o, int64_t row, bool strided, int64_t tokens) {
    constexpr int64_t es = sizeof(typename Elem<DT>::T), E = 16 / es;
    if (!fetchable<DT>(o, row)) return false;
    return tokens == 0 || (tokens * o.ld * es <= 0xfffff000 && (!strided || row % E == 0));
}

template <int DT, int KIND>
void launch_group_kind(const GroupArgs& a, int products, hipStream_t st) {
    using Kind = KindOf<KIND>;
    const int64_t tokens = iabn_divmagic_div(static_cast<uint32_t>(a.P), a.top);
    if (group_fetchable<DT>(a.x, Kind::kXStrided ? a.M : a.K, Kind::kXStrided, Kind::kGatherX ? tokens : 0) &&
        group_fetchable<DT>(a.y, Kind::kYStrided ? a.N : a.K, Kind::kYStrided, Kind::kGatherY ? tokens : 0))
        launch_group_planned<DT, KIND, true>(a, products, st);
    else
        launch_group_planned<DT, KIND, false>(a, products, st);
}

template <int DT>
void launch_grouped(int kind, const GroupArgs& a, int products, hipStream_t st) {
    switch (kind) {
        case kOverGroups + kGemmUp: launch_group_kind<DT, kOverGroups + kGemmUp>(a, products, st); break;
        case kOverGroups + kGemmDown: launch_group_kind<DT, kOverGroups + kGemmDown>(a, products, st); break;
        case kOverGroups + kGemmDh: launch_group_kind<DT, kOverGroups + kGemmDh>(a, products, st); break;
        case kOverGroups + kGemmDx: launch_group_kind<DT, kOverGroups + kGemmDx>(a, products, st); break;
        case kOverGroups + kGemmDw: launch_group_kind<DT, kOverGroups + kGemmDw>(a, products, st); break;
        case kGroupDwTokensY: launch_group_kind<DT, kGroupDwTokensY>(a, products, st); break;
    }
}

template <int DT, int KIND, int MT>
void launch_group_few_tiles(GroupArgs a, hipStream_t st) {
    constexpr bool kUp = KIND == kOverGroups + kGemmUp;
    a.splits = !kUp ? plan_grouped_few(a.P, a.E, a.N, a.K, DT) : 1;
    constexpr int kLine = 128 / sizeof(typename Elem<DT>::T), NW = kUp ? 2 : 1;
    const int64_t blocks = (a.N + 15) / 16 * most_tiles(a.P, a.E, MT * 16), lines = (a.K + kLine - 1) / kLine;
    int waves = MT;
    while (waves < 8 && blocks * a.splits * waves < 2048 && waves * 2 * kFewLines * a.splits <= lines) waves *= 2;
    // In fp32 no wave adds more than 256 terms of up to 2048 (then their share): y of 16
    // tokens, 6 of 84 experts (1512 -> 688), is off by 4.5e-7 in root mean square instead
    // of 1.1e-6, in 164 us instead of 153; of 24 tokens, 8 of 64 (1024 -> 1024), 5.2e-7
    // instead of 1.0e-6, in 142 instead of 153.
    if (DT == IABN_F32)
        while (waves < 8 && waves * 8 * a.splits < lines) waves *= 2;
    const size_t lds = static_cast<size_t>(waves) * NW * MT * kWave * sizeof(f32x4);
    few_kernel<DT, KIND, MT>
        <<<dim3(static_cast<uint32_t>(blocks), a.splits), waves * kWave, lds, st>>>(a);
}

template <int DT, int KIND>
void launch_group_few_kind(const GroupArgs& a, hipStream_t st) {
    // By the rows that an expert has: twice the mean, and no more than there are tokens.
    const int64_t busy = a.E < a.P ? a.E : a.P, tokens = iabn_divmagic_div(static_cast<uint32_t>(a.P), a.top);
    const int64_t twice = 2 * a.P / busy, rows = twice < tokens ? twice : tokens;
    if (rows <= 16) launch_group_few_tiles<DT, KIND, 1>(a, st);
    else if (rows <= 32) launch_group_few_tiles<DT, KIND, 2>(a, st);
    else launch_group_few_tiles<DT, KIND, 4>(a, st);
}

template <int DT>
void launch_grouped_few(int kind, const GroupArgs& a, hipStream_t st) {
    if (kind == kOverGroups + kGemmUp) launch_group_few_kind<DT, kOverGroups + kGemmUp>(a, st);
    else launch_group_few_kind<DT, kOverGroups + kGemmDown>(a, st);
}

}  // namespace iabn_impl
