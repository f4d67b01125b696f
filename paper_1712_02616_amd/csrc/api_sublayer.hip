// The C ABI of the feed-forward sublayer (include/iabn.h): argument
// validation on the host before any launch, how the work is split, and the
// entry points themselves.

#include <cmath>

#include "errors.h"
#include "sublayer.h"

namespace iabn_impl {
namespace {

constexpr int64_t kMaxWidth = (int64_t(1) << 31) - 1;
constexpr int64_t kMaxNormWidth = int64_t(kMaxRowWaves) * kWave * 2 * kChunk;
constexpr int64_t kMaxElems = int64_t(1) << 46;

bool valid_dtype(int dtype) { return dtype == IABN_F32 || dtype == IABN_F16 || dtype == IABN_BF16; }

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
    if (gate == nullptr) return IABN_OK;
    if (groups < 1 || R % groups != 0)
        return fail(IABN_ERR_SHAPE, "%lld rows of the gate do not divide R=%lld", (long long)groups,
                    (long long)R);
    return IABN_OK;
}

// How the backward's rows go over its blocks.  Enough blocks to fill the
// chip, few enough that their columns' sums (4 or 5 vectors of C floats,
// written and read once) stay small against the rows: a block takes at least
// kMinRows of them.
constexpr int64_t kBwdWaves = 2048;
constexpr int64_t kBwdMinRows = 8;

ResnormSplit split_rows(int64_t R, int64_t C, int64_t groups) {
    if (R == 0) return {1, 0, 0, 0, 0};
    const RowShape shape = row_shape(static_cast<int>((C + kChunk - 1) / kChunk));
    const int waves = shape.waves == 1 ? 4 : shape.waves;
    int64_t target = kBwdWaves / waves;
    if (target < 1) target = 1;
    ResnormSplit s;
    s.groups = groups > 0 && groups < R ? groups : 1;
    s.group_rows = R / s.groups;
    if (s.groups >= target) {
        s.per_group = 1;
        s.segs = static_cast<int>((s.groups + target - 1) / target);
        s.blocks = static_cast<int>((s.groups + s.segs - 1) / s.segs);
    } else {
        const int64_t most = (s.group_rows + kBwdMinRows - 1) / kBwdMinRows;
        int64_t per = target / s.groups;
        if (per > most) per = most;
        s.per_group = static_cast<int>(per);
        s.segs = 1;
        s.blocks = static_cast<int>(s.groups * per);
    }
    return s;
}

size_t resnorm_workspace(const ResnormSplit& s, int64_t C) {
    return static_cast<size_t>(5) * s.blocks * C * sizeof(float);
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
    a.chunks = static_cast<int>((C + kChunk - 1) / kChunk);
    launch_resnorm_fwd(dtype, a, static_cast<hipStream_t>(stream));
    return launched("resnorm_forward");
}

size_t iabn_resnorm_workspace_size(int64_t R, int64_t C, int64_t groups) {
    if (R < 0 || C < 0 || C > kMaxNormWidth || (C != 0 && R > kMaxElems / C)) return 0;
    return resnorm_workspace(split_rows(R, C, groups), C);
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
    a.split = split_rows(R, C, gate ? groups : 0);
    const size_t need = resnorm_workspace(a.split, C);
    if (need > 0) {
        if (!workspace) return fail(IABN_ERR_NULL, "workspace is NULL");
        if (workspace_bytes < need)
            return fail(IABN_ERR_WORKSPACE, "workspace of %zu bytes, %zu needed", workspace_bytes, need);
        if (reinterpret_cast<uintptr_t>(workspace) % 16 != 0)
            return fail(IABN_ERR_WORKSPACE, "workspace is not 16-byte aligned");
    }
    const int eb = dtype == IABN_F32 ? 4 : 2;
    if (R == 0) {
        float* const vectors[] = {dpost_weight, dpost_bias, dpre_weight, dpre_bias};
        for (float* v : vectors)
            if (v) launch_zero(v, C * 4, st);
        if (dgate) launch_zero(dgate, groups * C * eb, st);
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
    a.chunks = static_cast<int>((C + kChunk - 1) / kChunk);
    a.part = static_cast<float*>(workspace);
    a.gpart = a.part + static_cast<size_t>(4) * a.split.blocks * C;
    launch_resnorm_bwd(dtype, a, st);
    return launched("resnorm_backward");
}

}  // extern "C"
