// The C ABI of the feed-forward sublayer (include/iabn.h): argument
// validation on the host before any launch, how the work is split, and the
// entry points themselves.

#include <cmath>

#include "checks.h"
#include "ffn.h"

namespace iabn_impl {
namespace {

constexpr int64_t kMaxWidth = (int64_t(1) << 31) - 1;
constexpr int64_t kMaxNormWidth = int64_t(kMaxRowWaves) * kWave * 2 * kChunk;
constexpr int64_t kMaxElems = int64_t(1) << 46;

int check_rows(int dtype, int64_t R, int64_t C, int64_t max_width) {
    if (!valid_dtype(dtype)) return fail(IABN_ERR_DTYPE, "unknown dtype %d", dtype);
    if (R < 0 || C < 0)
        return fail(IABN_ERR_SHAPE, "negative size R=%lld C=%lld", (long long)R, (long long)C);
    if (C > max_width)
        return fail(IABN_ERR_SHAPE, "C=%lld exceeds %lld", (long long)C, (long long)max_width);
    if (C != 0 && R > kMaxElems / C) return fail(IABN_ERR_SHAPE, "R*C exceeds 2^46");
    return IABN_OK;
}

int check_dropout(float p, uint64_t seed, uint64_t offset, Dropout* d) {
    if (!(p >= 0.0f && p <= 1.0f)) return fail(IABN_ERR_PARAM, "p=%g is not in [0, 1]", p);
    const uint32_t t = static_cast<uint32_t>(static_cast<double>(p) * 65536.0 + 0.5);
    *d = {t, t < 65536 ? static_cast<float>(65536.0 / (65536.0 - t)) : 0.0f, seed, offset};
    return IABN_OK;
}

int check_norm(const char* what, int kind, const void* weight, const void* bias) {
    if (kind != IABN_NORM_NONE && kind != IABN_NORM_RMS && kind != IABN_NORM_LAYER)
        return fail(IABN_ERR_PARAM, "unknown %s norm %d", what, kind);
    if (kind == IABN_NORM_NONE && (weight || bias))
        return fail(IABN_ERR_PARAM, "a weight or bias of the %s norm without the norm", what);
    return IABN_OK;
}

int check_gate(const void* gate, int64_t groups, int64_t R) {
    if (gate == nullptr || (R == 0 && groups == 0)) return IABN_OK;
    if (groups < 1 || R % groups != 0)
        return fail(IABN_ERR_SHAPE, "%lld rows of the gate do not divide R=%lld", (long long)groups,
                    (long long)R);
    return IABN_OK;
}

// How the backward's rows go over its blocks.  Enough blocks to fill the
// chip, few enough that their columns' sums (4 or 5 vectors of C floats,
// written and read once) stay small against the rows: a block takes at least
// kBwdMinRows of them, or two while there are fewer blocks than CUs ((1031,
// 1501) fp32: 30.6 us with 8, 22.3 with 4, 25.4 with 2; (512, 1024) fp16 14.0,
// 9.1, 7.2).  The kernels' registers let 8 waves run on a CU; unmasked rows of
// 16-bit values in at most 4 waves are held to 12 ((16384, 2048) bf16: 109 us
// with 8, 81 with 12; masked ones spill: (1031, 1501) fp32 20.6, 31.7).
constexpr int64_t kCUs = 256;
constexpr int64_t kBwdMinRows = 4;
// A wave's fp32 sum over its rows, one after the other, has at most so many
// terms: what a chain can lose, 1024 * 2^-24 of its terms, does not grow with the
// rows (the blocks' sums are joined in double).  Past 2^20 blocks' worth of rows
// it does again, which rows of 8 or more elements on one GPU do not reach.
constexpr int64_t kChain = 1024;
constexpr int64_t kMaxBwdBlocks = int64_t(1) << 20;

ResnormSplit split_rows(int64_t R, int64_t C, int64_t groups, int64_t waves_on_cu) {
    if (R == 0) return {1, 0, 0, 0, 0};
    const RowShape shape = row_shape(chunks_of(C), kBwdOneWave);
    // (A block of one-wave rows has four of them.)
    const int64_t on_cu = shape.waves == 1 ? 2 : waves_on_cu / shape.waves;
    const int64_t target = kCUs * (on_cu > 1 ? on_cu : 1);
    int64_t most_rows = kChain * (shape.waves == 1 ? 4 : 1);  // of a block
    if (most_rows < div_up(R, kMaxBwdBlocks)) most_rows = div_up(R, kMaxBwdBlocks);
    ResnormSplit s;
    s.groups = groups > 0 && groups < R ? groups : 1;
    s.group_rows = R / s.groups;
    int64_t per = 1, segs = 1;
    if (s.groups >= target) {
        segs = div_up(s.groups, target);
    } else {
        const int64_t fewest = kCUs / s.groups, two = (s.group_rows + 1) / 2;
        const int64_t most = div_up(s.group_rows, kBwdMinRows);
        per = target / s.groups;
        if (per > most) per = most;
        if (per < fewest) per = fewest < two ? fewest : two;
    }
    if (per < div_up(s.group_rows, most_rows)) per = div_up(s.group_rows, most_rows);
    if (per > 1) segs = 1;
    else if (segs > 1 && segs * s.group_rows > most_rows) segs = most_rows / s.group_rows;
    s.per_group = static_cast<int>(per);
    s.segs = static_cast<int>(segs);
    s.blocks = static_cast<int>(div_up(s.groups * per, segs));
    return s;
}

int64_t waves_on_cu(int dtype, int64_t C) {
    return dtype != IABN_F32 && C % (kWave * kChunk) == 0 && C <= 4 * kWave * kChunk ? 12 : 8;
}

size_t resnorm_workspace(const ResnormSplit& s, int64_t C) {
    return static_cast<size_t>(5) * s.blocks * C * sizeof(float);
}

// ---------------------------------------------------------------- gated feed-forward block

constexpr int64_t kMaxFfnWidth = int64_t(1) << 24;
constexpr int64_t kMaxFfnRows = int64_t(1) << 26;
// Elements of any of its matrices (so that its tiles fit a launch).
constexpr int64_t kMaxFfnElems = int64_t(1) << 37;

int check_ffn(int dtype, int act, float slope, int64_t M, int64_t C, int64_t F) {
    if (!valid_dtype(dtype)) return fail(IABN_ERR_DTYPE, "unknown dtype %d", dtype);
    if (M < 0 || C < 0 || F < 0)
        return fail(IABN_ERR_SHAPE, "negative size M=%lld C=%lld F=%lld", (long long)M, (long long)C,
                    (long long)F);
    if (M > kMaxFfnRows || C > kMaxFfnWidth || F > kMaxFfnWidth)
        return fail(IABN_ERR_SHAPE, "M=%lld, C=%lld or F=%lld is too large", (long long)M,
                    (long long)C, (long long)F);
    if (M * C > kMaxFfnElems || M * F > kMaxFfnElems || C * F > kMaxFfnElems)
        return fail(IABN_ERR_SHAPE, "a matrix of M=%lld, C=%lld, F=%lld exceeds 2^37 elements",
                    (long long)M, (long long)C, (long long)F);
    if (act != IABN_ACT_SILU && act != IABN_ACT_GELU && act != IABN_ACT_LEAKY)
        return fail(IABN_ERR_PARAM, "unknown activation %d", act);
    if (act == IABN_ACT_LEAKY && !(slope >= 0.0f && std::isfinite(slope)))
        return fail(IABN_ERR_PARAM, "slope=%g must be >= 0 and finite", slope);
    return IABN_OK;
}

// h, [M, F], and then the largest of the products' sums.
size_t h_bytes(int64_t M, int64_t F, int dtype) {
    return (static_cast<size_t>(M) * F * elem_bytes(dtype) + 255) / 256 * 256;
}

size_t ffn_workspace(int64_t M, int64_t C, int64_t F, int dtype) {
    size_t part = 0;
    for (size_t p : {part_bytes(dtype, kGemmDown, M, C, F, 1), part_bytes(dtype, kGemmDx, M, C, F, 1),
                     part_bytes(dtype, kGemmDw, C, F, M, 1), part_bytes(dtype, kGemmDw, F, C, M, 2)})
        part = part < p ? p : part;
    return h_bytes(M, F, dtype) + part;
}

// A product of the block, whose split sums go behind h in the workspace.
void gemm(int dtype, GemmKind kind, GemmArgs a, int products, void* workspace, int64_t M, int64_t F,
          hipStream_t st) {
    a.part = reinterpret_cast<float*>(static_cast<char*>(workspace) + h_bytes(M, F, dtype));
    const bool few = few_rows(kind, a.M);
    switch (dtype) {
        case IABN_F32:
            few ? launch_few<IABN_F32>(kind, a, st) : launch_gemm<IABN_F32>(kind, a, products, st);
            break;
        case IABN_F16:
            few ? launch_few<IABN_F16>(kind, a, st) : launch_gemm<IABN_F16>(kind, a, products, st);
            break;
        default:
            few ? launch_few<IABN_BF16>(kind, a, st) : launch_gemm<IABN_BF16>(kind, a, products, st);
            break;
    }
}

bool finite(float v) { return std::isfinite(v); }

}  // namespace
}  // namespace iabn_impl

using namespace iabn_impl;

extern "C" {

int iabn_dropout(const void* x, void* y, int dtype, float p, uint64_t seed, uint64_t offset,
                 int64_t R, int64_t C, void* stream) {
    int rc = check_rows(dtype, R, C, kMaxWidth);
    if (rc) return rc;
    Dropout d;
    if ((rc = check_dropout(p, seed, offset, &d))) return rc;
    if (R == 0 || C == 0) return ok();
    if (!x || !y) return fail(IABN_ERR_NULL, "x or y is NULL");
    launch_dropout(dtype, x, y, R, static_cast<int>(C), d, static_cast<hipStream_t>(stream));
    return launched("dropout");
}

int iabn_resnorm_forward(const void* x, const void* h, void* r, void* u, int dtype,
                         const void* gate, int64_t groups, int post_norm, const float* post_weight,
                         const float* post_bias, int pre_norm, const float* pre_weight,
                         const float* pre_bias, float* post_stats, float* pre_stats, float alpha,
                         float beta, float eps, float p, uint64_t seed, uint64_t offset, int64_t R,
                         int64_t C, void* stream) {
    int rc = check_rows(dtype, R, C, kMaxNormWidth);
    if (rc) return rc;
    if ((rc = check_norm("post", post_norm, post_weight, post_bias))) return rc;
    if ((rc = check_norm("pre", pre_norm, pre_weight, pre_bias))) return rc;
    if ((rc = check_gate(gate, groups, R))) return rc;
    ResnormArgs a = {};
    if ((rc = check_dropout(p, seed, offset, &a.drop))) return rc;
    if (!finite(alpha) || !finite(beta)) return fail(IABN_ERR_PARAM, "alpha or beta is not finite");
    if (!(eps > 0.0f) || !finite(eps)) return fail(IABN_ERR_PARAM, "eps must be positive and finite");
    if (R == 0 || C == 0) return ok();
    if (!x) return fail(IABN_ERR_NULL, "x is NULL");
    if (!h && (post_norm != IABN_NORM_NONE || gate))
        return fail(IABN_ERR_NULL, "a norm or a gate of h, which is NULL");
    if ((u == nullptr) != (pre_norm == IABN_NORM_NONE))
        return fail(u ? IABN_ERR_PARAM : IABN_ERR_NULL, "u and the pre norm go together");
    if (!r && !u) return fail(IABN_ERR_NULL, "r and u are both NULL");
    a.x = x, a.h = h, a.r = r, a.u = u, a.gate = gate;
    a.post_w = post_weight, a.post_b = post_bias, a.pre_w = pre_weight, a.pre_b = pre_bias;
    a.post_stats = post_stats, a.pre_stats = pre_stats;
    a.post = post_norm, a.pre = pre_norm;
    a.alpha = alpha, a.beta = beta, a.eps = eps;
    a.inv_c = static_cast<float>(1.0 / static_cast<double>(C));
    a.R = R;
    a.gate_rows = gate ? R / groups : R;
    a.C = static_cast<int>(C);
    a.chunks = chunks_of(C);
    launch_resnorm_fwd(dtype, a, static_cast<hipStream_t>(stream));
    return launched("resnorm_forward");
}

size_t iabn_resnorm_workspace_size(int64_t R, int64_t C, int64_t groups) {
    if (R < 0 || C < 0 || C > kMaxNormWidth || (C != 0 && R > kMaxElems / C)) return 0;
    // (Enough for every storage type.)
    const size_t a = resnorm_workspace(split_rows(R, C, groups, 8), C);
    const size_t b = resnorm_workspace(split_rows(R, C, groups, 12), C);
    return a > b ? a : b;
}

int iabn_resnorm_backward(const void* dr, const void* du, const void* r, const void* h, void* dx,
                          void* dh, int dtype, const void* gate, int64_t groups, int post_norm,
                          const float* post_weight, const float* post_bias, int pre_norm,
                          const float* pre_weight, const float* post_stats, const float* pre_stats,
                          void* dgate, float* dpost_weight, float* dpost_bias, float* dpre_weight,
                          float* dpre_bias, float alpha, float beta, float p, uint64_t seed,
                          uint64_t offset, int64_t R, int64_t C, void* workspace,
                          size_t workspace_bytes, void* stream) {
    int rc = check_rows(dtype, R, C, kMaxNormWidth);
    if (rc) return rc;
    if ((rc = check_norm("post", post_norm, post_weight, post_bias))) return rc;
    if ((rc = check_norm("pre", pre_norm, pre_weight, nullptr))) return rc;
    if ((rc = check_gate(gate, groups, R))) return rc;
    ResnormBwdArgs a = {};
    if ((rc = check_dropout(p, seed, offset, &a.drop))) return rc;
    if (!finite(alpha) || !finite(beta)) return fail(IABN_ERR_PARAM, "alpha or beta is not finite");
    if (dgate && !gate) return fail(IABN_ERR_PARAM, "a gradient of the gate, which is NULL");
    if ((dpost_weight || dpost_bias) && post_norm == IABN_NORM_NONE)
        return fail(IABN_ERR_PARAM, "gradients of the post norm's vectors without the norm");
    if ((dpre_weight || dpre_bias) && pre_norm == IABN_NORM_NONE)
        return fail(IABN_ERR_PARAM, "gradients of the pre norm's vectors without the norm");
    if (C == 0) return ok();
    const hipStream_t st = static_cast<hipStream_t>(stream);
    const bool pre = pre_norm != IABN_NORM_NONE, post = post_norm != IABN_NORM_NONE;
    if (R > 0) {
        if ((du == nullptr) != !pre)
            return fail(du ? IABN_ERR_PARAM : IABN_ERR_NULL, "du and the pre norm go together");
        if (!dr && !du) return fail(IABN_ERR_NULL, "dr and du are both NULL");
        if (pre && (!r || !pre_stats)) return fail(IABN_ERR_NULL, "r or pre_stats is NULL");
        if (post && !post_stats) return fail(IABN_ERR_NULL, "post_stats is NULL");
        if ((post || dgate) && !h) return fail(IABN_ERR_NULL, "h is NULL");
        if (dh && dh == dx) return fail(IABN_ERR_PARAM, "dx and dh are one buffer");
    }
    a.split = split_rows(R, C, gate ? groups : 0, waves_on_cu(dtype, C));
    if ((rc = check_workspace(workspace, workspace_bytes, resnorm_workspace(a.split, C)))) return rc;
    if (R == 0) {
        float* const vectors[] = {dpost_weight, dpost_bias, dpre_weight, dpre_bias};
        for (float* v : vectors)
            if (v) launch_zero(v, C * 4, st);
        if (dgate) launch_zero(dgate, groups * C * elem_bytes(dtype), st);
        return launched("resnorm_backward");
    }
    a.dr = dr, a.du = du, a.r = r, a.h = h, a.dx = dx, a.dh = dh, a.gate = gate, a.dgate = dgate;
    a.post_w = post_weight, a.post_b = post_bias, a.pre_w = pre_weight;
    a.post_stats = post_stats, a.pre_stats = pre_stats;
    a.dpost_w = dpost_weight, a.dpost_b = dpost_bias, a.dpre_w = dpre_weight, a.dpre_b = dpre_bias;
    a.post = post_norm, a.pre = pre_norm;
    a.alpha = alpha, a.beta = beta;
    a.inv_c = static_cast<float>(1.0 / static_cast<double>(C));
    a.R = R;
    a.gate_rows = gate ? R / groups : R;
    a.gate_each_row = gate && groups == R;
    a.C = static_cast<int>(C);
    a.chunks = chunks_of(C);
    a.part = static_cast<float*>(workspace);
    a.gpart = a.part + static_cast<size_t>(4) * a.split.blocks * C;
    launch_resnorm_bwd(dtype, a, st);
    return launched("resnorm_backward");
}

size_t iabn_ffn_workspace_size(int64_t M, int64_t C, int64_t F, int dtype) {
    if (check_ffn(dtype, IABN_ACT_SILU, 0.0f, M, C, F) != IABN_OK) return 0;
    return ffn_workspace(M, C, F, dtype);
}

int iabn_ffn_forward(const void* x, const void* w_gate, const void* w_up, const void* w_down,
                     void* y, void* g, void* u, int dtype, int act, float slope, int64_t M,
                     int64_t C, int64_t F, void* workspace, size_t workspace_bytes, void* stream) {
    int rc = check_ffn(dtype, act, slope, M, C, F);
    if (rc) return rc;
    if ((g == nullptr) != (u == nullptr)) return fail(IABN_ERR_NULL, "one of g and u is NULL");
    if (M == 0) return ok();
    const hipStream_t st = static_cast<hipStream_t>(stream);
    const int eb = elem_bytes(dtype);
    if (C == 0 || F == 0) {
        if (C > 0 && !y) return fail(IABN_ERR_NULL, "y is NULL");
        launch_zero(y, M * C * eb, st);
        if (g) launch_zero(g, M * F * eb, st);
        if (u) launch_zero(u, M * F * eb, st);
        return launched("ffn_forward");
    }
    if (!x || !w_gate || !w_up || !w_down || !y)
        return fail(IABN_ERR_NULL, "x, y or a weight is NULL");
    if ((rc = check_workspace(workspace, workspace_bytes, ffn_workspace(M, C, F, dtype)))) return rc;
    GemmArgs up = {};
    up.x = {{x, x}, C}, up.y = {{w_gate, w_up}, C};
    up.M = M, up.N = F, up.K = C;
    up.out[0] = workspace, up.dg = g, up.du = u;
    up.act = act, up.slope = slope;
    gemm(dtype, kGemmUp, up, 1, workspace, M, F, st);
    GemmArgs down = {};
    down.x = {{workspace, workspace}, F}, down.y = {{w_down, w_down}, F};
    down.M = M, down.N = C, down.K = F;
    down.out[0] = y;
    gemm(dtype, kGemmDown, down, 1, workspace, M, F, st);
    return launched("ffn_forward");
}

int iabn_ffn_backward(const void* dy, const void* x, const void* g, const void* u,
                      const void* w_gate, const void* w_up, const void* w_down, void* dx, void* dg,
                      void* du, void* dw_gate, void* dw_up, void* dw_down, int dtype, int act,
                      float slope, int64_t M, int64_t C, int64_t F, void* workspace,
                      size_t workspace_bytes, void* stream) {
    int rc = check_ffn(dtype, act, slope, M, C, F);
    if (rc) return rc;
    const hipStream_t st = static_cast<hipStream_t>(stream);
    const int eb = elem_bytes(dtype);
    if (M == 0 || C == 0 || F == 0) {
        // Sums over nothing: no tokens, or no width on one side.
        if ((M * C > 0 && !dx) || (M * F > 0 && (!dg || !du)) ||
            (C * F > 0 && (!dw_gate || !dw_up || !dw_down)))
            return fail(IABN_ERR_NULL, "an output is NULL");
        launch_zero(dx, M * C * eb, st);
        launch_zero(dg, M * F * eb, st);
        launch_zero(du, M * F * eb, st);
        for (void* w : {dw_gate, dw_up, dw_down}) launch_zero(w, C * F * eb, st);
        return launched("ffn_backward");
    }
    if (!dy || !x || !g || !u || !w_gate || !w_up || !w_down)
        return fail(IABN_ERR_NULL, "dy, x, g, u or a weight is NULL");
    if (!dx || !dg || !du || !dw_gate || !dw_up || !dw_down)
        return fail(IABN_ERR_NULL, "an output is NULL");
    if ((rc = check_workspace(workspace, workspace_bytes, ffn_workspace(M, C, F, dtype)))) return rc;
    GemmArgs dh = {};
    dh.x = {{dy, dy}, C}, dh.y = {{w_down, w_down}, F};
    dh.M = M, dh.N = F, dh.K = C;
    dh.out[0] = workspace, dh.g = g, dh.u = u, dh.dg = dg, dh.du = du;
    dh.act = act, dh.slope = slope;
    gemm(dtype, kGemmDh, dh, 1, workspace, M, F, st);
    GemmArgs dwd = {};
    dwd.x = {{dy, dy}, C}, dwd.y = {{workspace, workspace}, F};
    dwd.M = C, dwd.N = F, dwd.K = M;
    dwd.out[0] = dw_down;
    gemm(dtype, kGemmDw, dwd, 1, workspace, M, F, st);
    GemmArgs dwp = {};
    dwp.x = {{dg, du}, F}, dwp.y = {{x, x}, C};
    dwp.M = F, dwp.N = C, dwp.K = M;
    dwp.out[0] = dw_gate, dwp.out[1] = dw_up;
    gemm(dtype, kGemmDw, dwp, 2, workspace, M, F, st);
    GemmArgs dxp = {};
    dxp.x = {{dg, du}, F}, dxp.y = {{w_gate, w_up}, C};
    dxp.M = M, dxp.N = C, dxp.K = F;
    dxp.out[0] = dx;
    gemm(dtype, kGemmDx, dxp, 1, workspace, M, F, st);
    return launched("ffn_backward");
}

}  // extern "C"
