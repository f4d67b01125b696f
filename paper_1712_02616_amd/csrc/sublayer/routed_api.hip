// The C ABI of the routed experts and of the gradients' clipping
// (include/iabn.h): argument validation on the host before any launch, and the
// entry points themselves.

#include <algorithm>
#include <cmath>
#include <memory>
#include <new>

#include "checks.h"
#include "groups.h"

namespace iabn_impl {
namespace {

constexpr int64_t kMaxRouteRows = int64_t(1) << 25;
constexpr int64_t kMaxPairs = int64_t(1) << 30;
constexpr int64_t kMaxGroups = 64;
// Widths and elements of the products' matrices (so that their tiles fit a launch).
constexpr int64_t kMaxExpertWidth = int64_t(1) << 17;
constexpr int64_t kMaxExpertElems = int64_t(1) << 35;
// (2^30 pairs in tiles of 64 rows, 256 threads each, would be 2^32 threads.)
constexpr int64_t kMaxExpertPairs = int64_t(1) << 29;

int check_pairs(int64_t M, int64_t k, int64_t E) {
    if (M < 0 || M > kMaxRouteRows)
        return fail(IABN_ERR_SHAPE, "M=%lld is not in [0, 2^25]", (long long)M);
    if (E < 1 || E > kMaxExperts)
        return fail(IABN_ERR_SHAPE, "E=%lld is not in [1, %d]", (long long)E, kMaxExperts);
    if (k < 0 || k > kMaxTop)
        return fail(IABN_ERR_SHAPE, "k=%lld is not in [0, %d]", (long long)k, kMaxTop);
    if (M * k > kMaxPairs) return fail(IABN_ERR_SHAPE, "M*k exceeds 2^30");
    return IABN_OK;
}

int check_route(int dtype, int score, float scale, int64_t M, int64_t E, int64_t k) {
    if (!valid_dtype(dtype)) return fail(IABN_ERR_DTYPE, "unknown dtype %d", dtype);
    const int rc = check_pairs(M, k, E);
    if (rc) return rc;
    if (k > E) return fail(IABN_ERR_SHAPE, "k=%lld of E=%lld experts", (long long)k, (long long)E);
    if (score != IABN_SCORE_SOFTMAX && score != IABN_SCORE_SIGMOID)
        return fail(IABN_ERR_PARAM, "unknown score %d", score);
    if (!std::isfinite(scale)) return fail(IABN_ERR_PARAM, "scale is not finite");
    return IABN_OK;
}

int check_experts(int dtype, int act, float slope, int64_t M, int64_t k, int64_t E, int64_t C, int64_t F) {
    if (!valid_dtype(dtype)) return fail(IABN_ERR_DTYPE, "unknown dtype %d", dtype);
    const int rc = check_pairs(M, k, E);
    if (rc) return rc;
    if (C < 0 || F < 0 || C > kMaxExpertWidth || F > kMaxExpertWidth)
        return fail(IABN_ERR_SHAPE, "C=%lld or F=%lld is not in [0, 2^17]", (long long)C, (long long)F);
    if (M * k > kMaxExpertPairs) return fail(IABN_ERR_SHAPE, "M*k exceeds 2^29");
    const int64_t rows = k > 1 ? M * k : M;
    if (rows * C > kMaxExpertElems || rows * F > kMaxExpertElems || E * C * F > kMaxExpertElems)
        return fail(IABN_ERR_SHAPE, "a matrix of M=%lld, k=%lld, E=%lld, C=%lld, F=%lld exceeds 2^35 elements",
                    (long long)M, (long long)k, (long long)E, (long long)C, (long long)F);
    if (act != IABN_ACT_SILU && act != IABN_ACT_GELU && act != IABN_ACT_LEAKY)
        return fail(IABN_ERR_PARAM, "unknown activation %d", act);
    if (act == IABN_ACT_LEAKY && !(slope >= 0.0f && std::isfinite(slope)))
        return fail(IABN_ERR_PARAM, "slope=%g must be >= 0 and finite", slope);
    return IABN_OK;
}

size_t padded(size_t bytes) { return (bytes + 255) / 256 * 256; }

// h (forward and backward), then the pairs' terms, [P][C] as store_terms leaves them
// or of fp32 for few tokens; in the backward the dots, [P][ceil(F/64)], after them.
struct ExpertsSpace {
    size_t h, terms, dots;
    size_t low;  // of the terms, from their begin
    size_t all() const { return h + terms + dots; }
};
ExpertsSpace experts_space(int64_t M, int64_t k, int64_t E, int64_t C, int64_t F, int dtype) {
    const size_t P = static_cast<size_t>(M) * k, eb = elem_bytes(dtype);
    ExpertsSpace s = {padded(P * F * eb), padded(P * C * eb), padded(P * div_up(F, 64) * sizeof(float)), 0};
    s.low = s.terms;
    if (dtype != IABN_F32) s.terms += padded(P * C);
    if (P > 0 && few_pairs(M)) {
        const size_t few = padded(plan_grouped_few(P, E, C, F, dtype) * P * C * sizeof(float));
        s.terms = s.terms < few ? few : s.terms;
    }
    return s;
}

GroupArgs group_args(const PlanArgs& plan, const float* weights, int64_t k, int64_t C, int64_t F, int act,
                     float slope) {
    GroupArgs a = {};
    a.offsets = plan.offsets, a.order = plan.order, a.by_size = plan.by_size, a.weights = weights;
    a.top = iabn_divmagic_make(static_cast<uint32_t>(k));
    a.E = plan.E, a.P = plan.P;
    a.expert_stride = C * F;
    a.act = act, a.slope = slope;
    a.splits = 1;
    return a;
}

void grouped(int dtype, int kind, const GroupArgs& a, int products, hipStream_t st) {
    switch (dtype) {
        case IABN_F32: launch_grouped<IABN_F32>(kind, a, products, st); break;
        case IABN_F16: launch_grouped<IABN_F16>(kind, a, products, st); break;
        default: launch_grouped<IABN_BF16>(kind, a, products, st); break;
    }
}

void grouped_few(int dtype, int kind, const GroupArgs& a, hipStream_t st) {
    switch (dtype) {
        case IABN_F32: launch_grouped_few<IABN_F32>(kind, a, st); break;
        case IABN_F16: launch_grouped_few<IABN_F16>(kind, a, st); break;
        default: launch_grouped_few<IABN_BF16>(kind, a, st); break;
    }
}

// ---------------------------------------------------------------- gradients

// Elements of a piece: enough pieces to fill the chip several times, and few enough
// that their sums are quickly joined.
constexpr int64_t kPieces = 8192, kMinPiece = 4096, kPieceStep = kThreads * kChunk;
constexpr int64_t kMaxGrads = 1 << 20, kMaxGradElems = int64_t(1) << 42;

struct GradList {
    int64_t piece, pieces;
};
int check_grads(const int64_t* sizes, int64_t count, GradList* list) {
    if (count < 0 || count > kMaxGrads)
        return fail(IABN_ERR_SHAPE, "count=%lld is not in [0, 2^20]", (long long)count);
    if (count > 0 && !sizes) return fail(IABN_ERR_NULL, "sizes is NULL");
    int64_t all = 0;
    for (int64_t i = 0; i < count; ++i) {
        if (sizes[i] < 0 || sizes[i] > kMaxGradElems || all + sizes[i] > kMaxGradElems)
            return fail(IABN_ERR_SHAPE, "sizes[%lld]=%lld is negative or too large", (long long)i,
                        (long long)sizes[i]);
        all += sizes[i];
    }
    list->piece = div_up(div_up(all, kPieces), kPieceStep) * kPieceStep;
    if (list->piece < kMinPiece) list->piece = kMinPiece;
    list->pieces = 0;
    for (int64_t i = 0; i < count; ++i) list->pieces += div_up(sizes[i], list->piece);
    return IABN_OK;
}

int check_grad_tensors(const void* const* grads, const void* const* outs, bool with_outs, const int* dtypes,
                       const int64_t* sizes, int64_t count) {
    if (count == 0) return IABN_OK;
    if (!grads || !dtypes || (with_outs && !outs)) return fail(IABN_ERR_NULL, "a list is NULL");
    for (int64_t i = 0; i < count; ++i) {
        if (!valid_dtype(dtypes[i])) return fail(IABN_ERR_DTYPE, "unknown dtype %d", dtypes[i]);
        if (sizes[i] > 0 && (!grads[i] || (with_outs && !outs[i])))
            return fail(IABN_ERR_NULL, "tensor %lld is NULL", (long long)i);
    }
    return IABN_OK;
}

// No two outputs may share an element: which of the two wrote it last would be
// chance, and in place it would be scaled once or twice.  Nor may an output lie over
// what other blocks read: a gradient, but for its own in the same place, or the norm.
int check_apart(const void* const* grads, void* const* outs, const int* dtypes, const int64_t* sizes, int64_t count,
                const float* norm) {
    struct Span {
        uintptr_t begin, end;
    };
    const auto span_at = [](const void* p, size_t bytes) {
        const uintptr_t begin = reinterpret_cast<uintptr_t>(p);
        return Span{begin, begin + bytes};
    };
    Span few[kGradTensors];
    std::unique_ptr<Span[]> many;
    if (count > kGradTensors) {
        many.reset(new (std::nothrow) Span[count]);
        if (!many) return fail(IABN_ERR_SHAPE, "no memory to look through %lld tensors", (long long)count);
    }
    Span* const spans = many ? many.get() : few;
    int64_t n = 0;
    for (int64_t i = 0; i < count; ++i) {
        if (sizes[i] == 0) continue;
        spans[n++] = span_at(outs[i], static_cast<size_t>(sizes[i]) * elem_bytes(dtypes[i]));
    }
    std::sort(spans, spans + n, [](const Span& a, const Span& b) { return a.begin < b.begin; });
    for (int64_t i = 1; i < n; ++i)
        if (spans[i].begin < spans[i - 1].end) return fail(IABN_ERR_PARAM, "two outputs overlap");
    // (Of spans apart, the last one that begins before the end is the one to look at.)
    const auto meets_an_output = [&](const Span& s) {
        const Span* const after = std::lower_bound(spans, spans + n, s.end,
                                                   [](const Span& o, uintptr_t end) { return o.begin < end; });
        return after != spans && after[-1].end > s.begin;
    };
    for (int64_t i = 0; i < count; ++i)
        if (sizes[i] > 0 && grads[i] != outs[i] &&
            meets_an_output(span_at(grads[i], static_cast<size_t>(sizes[i]) * elem_bytes(dtypes[i]))))
            return fail(IABN_ERR_PARAM, "an output overlaps tensor %lld", (long long)i);
    if (meets_an_output(span_at(norm, sizeof(float)))) return fail(IABN_ERR_PARAM, "an output overlaps norm");
    return IABN_OK;
}

// Calls launch(args) for each group of tensors that a launch takes.
template <typename Launch>
void over_grads(const void* const* grads, void* const* outs, const int* dtypes, const int64_t* sizes,
                int64_t count, int64_t piece, Launch launch) {
    GradArgs a = {};
    a.piece = static_cast<int32_t>(piece);
    for (int64_t i = 0; i < count; ++i) {
        if (sizes[i] == 0) continue;
        const int t = a.count++;
        a.in[t] = grads[i], a.out[t] = outs ? outs[i] : nullptr;
        a.n[t] = sizes[i];
        a.dtype[t] = static_cast<uint8_t>(dtypes[i]);
        a.first[a.count] = a.first[t] + static_cast<int32_t>(div_up(sizes[i], piece));
        if (a.count == kGradTensors) {
            launch(a);
            a.count = 0;
        }
    }
    if (a.count > 0) launch(a);
}

}  // namespace
}  // namespace iabn_impl

using namespace iabn_impl;

extern "C" {

int iabn_route_forward(const void* logits, int dtype, const float* bias, int32_t* experts, float* weights,
                       int score, int64_t groups, int64_t groups_kept, int group_top, int renormalise,
                       float scale, int64_t M, int64_t E, int64_t k, void* stream) {
    const int rc = check_route(dtype, score, scale, M, E, k);
    if (rc) return rc;
    if (groups < 1 || groups > kMaxGroups || E % groups != 0)
        return fail(IABN_ERR_SHAPE, "%lld groups of E=%lld experts (at most %lld, dividing E)", (long long)groups,
                    (long long)E, (long long)kMaxGroups);
    if (groups_kept < 1 || groups_kept > groups)
        return fail(IABN_ERR_PARAM, "groups_kept=%lld is not in [1, %lld]", (long long)groups_kept,
                    (long long)groups);
    if (group_top != 1 && group_top != 2) return fail(IABN_ERR_PARAM, "group_top=%d is not 1 or 2", group_top);
    if (M == 0 || k == 0) return ok();
    if (!logits || !experts || !weights) return fail(IABN_ERR_NULL, "logits, experts or weights is NULL");
    RouteArgs a = {};
    a.logits = logits, a.bias = bias, a.experts = experts, a.weights = weights;
    a.M = M, a.E = static_cast<int>(E), a.k = static_cast<int>(k);
    a.groups = static_cast<int>(groups), a.kept = static_cast<int>(groups_kept), a.group_top = group_top;
    a.per = static_cast<int>(E / groups);
    a.per_magic = static_cast<uint32_t>(((int64_t(1) << 20) + a.per - 1) / a.per);
    a.scale = scale;
    a.sigmoid = score == IABN_SCORE_SIGMOID, a.renormalise = renormalise != 0;
    launch_route_fwd(dtype, a, static_cast<hipStream_t>(stream));
    return launched("route_forward");
}

int iabn_route_backward(const float* dweights, const void* logits, const int32_t* experts, void* dlogits,
                        int dtype, int score, int renormalise, float scale, int64_t M, int64_t E, int64_t k,
                        void* stream) {
    const int rc = check_route(dtype, score, scale, M, E, k);
    if (rc) return rc;
    if (M == 0) return ok();
    if (!dlogits) return fail(IABN_ERR_NULL, "dlogits is NULL");
    const hipStream_t st = static_cast<hipStream_t>(stream);
    if (k == 0) {
        launch_zero(dlogits, M * E * elem_bytes(dtype), st);
        return launched("route_backward");
    }
    if (!dweights || !logits || !experts) return fail(IABN_ERR_NULL, "dweights, logits or experts is NULL");
    RouteBwdArgs a = {};
    a.dweights = dweights, a.logits = logits, a.experts = experts, a.dlogits = dlogits;
    a.M = M, a.E = static_cast<int>(E), a.k = static_cast<int>(k);
    a.scale = scale;
    a.sigmoid = score == IABN_SCORE_SIGMOID, a.renormalise = renormalise != 0;
    launch_route_bwd(dtype, a, st);
    return launched("route_backward");
}

int64_t iabn_experts_plan_size(int64_t M, int64_t k, int64_t E) {
    if (check_pairs(M, k, E) != IABN_OK) return 0;
    return plan_size(M * k, E);
}

int iabn_experts_plan(const int32_t* experts, int32_t* plan, int64_t M, int64_t k, int64_t E, void* stream) {
    const int rc = check_pairs(M, k, E);
    if (rc) return rc;
    if (!plan || (M * k > 0 && !experts)) return fail(IABN_ERR_NULL, "experts or plan is NULL");
    PlanArgs a = plan_of(M * k, E, plan);
    a.experts = experts;
    launch_plan(a, static_cast<hipStream_t>(stream));
    return launched("experts_plan");
}

size_t iabn_experts_workspace_size(int64_t M, int64_t k, int64_t E, int64_t C, int64_t F, int dtype) {
    if (check_experts(dtype, IABN_ACT_SILU, 0.0f, M, k, E, C, F) != IABN_OK) return 0;
    if (M == 0 || k == 0 || C == 0 || F == 0) return 0;
    return experts_space(M, k, E, C, F, dtype).all();
}

int iabn_experts_forward(const void* x, const int32_t* plan, const float* weights, const void* w_gate,
                         const void* w_up, const void* w_down, void* y, void* g, void* u, int dtype, int act,
                         float slope, int64_t M, int64_t k, int64_t E, int64_t C, int64_t F, void* workspace,
                         size_t workspace_bytes, void* stream) {
    int rc = check_experts(dtype, act, slope, M, k, E, C, F);
    if (rc) return rc;
    if ((g == nullptr) != (u == nullptr)) return fail(IABN_ERR_NULL, "one of g and u is NULL");
    if (M == 0) return ok();
    const hipStream_t st = static_cast<hipStream_t>(stream);
    const int eb = elem_bytes(dtype);
    const int64_t P = M * k;
    if (k == 0 || C == 0 || F == 0) {
        if (C > 0 && !y) return fail(IABN_ERR_NULL, "y is NULL");
        launch_zero(y, M * C * eb, st);
        if (g) launch_zero(g, P * F * eb, st);
        if (u) launch_zero(u, P * F * eb, st);
        return launched("experts_forward");
    }
    if (!x || !plan || !weights || !w_gate || !w_up || !w_down || !y)
        return fail(IABN_ERR_NULL, "x, plan, weights, y or an expert's weight is NULL");
    const ExpertsSpace space = experts_space(M, k, E, C, F, dtype);
    if ((rc = check_workspace(workspace, workspace_bytes, space.all()))) return rc;
    const PlanArgs sorted = plan_of(P, E, const_cast<int32_t*>(plan));
    void* const terms = static_cast<char*>(workspace) + space.h;
    const bool few = few_pairs(M);
    GroupArgs up = group_args(sorted, weights, k, C, F, act, slope);
    up.x = {{x, x}, C}, up.y = {{w_gate, w_up}, C};
    up.M = P, up.N = F, up.K = C;
    up.out[0] = workspace, up.dg = g, up.du = u;
    few ? grouped_few(dtype, kOverGroups + kGemmUp, up, st) : grouped(dtype, kOverGroups + kGemmUp, up, 1, st);
    GroupArgs down = group_args(sorted, weights, k, C, F, act, slope);
    down.x = {{workspace, workspace}, F}, down.y = {{w_down, w_down}, F};
    down.M = P, down.N = C, down.K = F;
    down.out[0] = terms, down.out[1] = static_cast<char*>(terms) + space.low, down.part = static_cast<float*>(terms);
    few ? grouped_few(dtype, kOverGroups + kGemmDown, down, st) : grouped(dtype, kOverGroups + kGemmDown, down, 1, st);
    CombineArgs join = {};
    join.terms = terms, join.low = down.out[1], join.place = sorted.place, join.weights = few ? weights : nullptr, join.y = y;
    join.M = M, join.C = C, join.k = static_cast<int32_t>(k), join.P = sorted.P;
    join.splits = few ? plan_grouped_few(P, E, C, F, dtype) : 1;
    launch_combine(dtype, join, st);
    return launched("experts_forward");
}

int iabn_experts_backward(const void* dy, const void* x, const int32_t* plan, const float* weights, const void* g,
                          const void* u, const void* w_gate, const void* w_up, const void* w_down, void* dx,
                          float* dweights, void* dg, void* du, void* dw_gate, void* dw_up, void* dw_down,
                          int dtype, int act, float slope, int64_t M, int64_t k, int64_t E, int64_t C, int64_t F,
                          void* workspace, size_t workspace_bytes, void* stream) {
    int rc = check_experts(dtype, act, slope, M, k, E, C, F);
    if (rc) return rc;
    const hipStream_t st = static_cast<hipStream_t>(stream);
    const int eb = elem_bytes(dtype);
    const int64_t P = M * k;
    if (P == 0 || C == 0 || F == 0) {
        // Sums over nothing: no pairs, or no width on one side.
        if ((M * C > 0 && !dx) || (P > 0 && !dweights) || (P * F > 0 && (!dg || !du)) ||
            (C * F > 0 && (!dw_gate || !dw_up || !dw_down)))
            return fail(IABN_ERR_NULL, "an output is NULL");
        launch_zero(dx, M * C * eb, st);
        launch_zero(dweights, P * 4, st);
        launch_zero(dg, P * F * eb, st);
        launch_zero(du, P * F * eb, st);
        for (void* w : {dw_gate, dw_up, dw_down}) launch_zero(w, E * C * F * eb, st);
        return launched("experts_backward");
    }
    if (!dy || !x || !plan || !weights || !g || !u || !w_gate || !w_up || !w_down)
        return fail(IABN_ERR_NULL, "dy, x, plan, weights, g, u or an expert's weight is NULL");
    if (!dx || !dweights || !dg || !du || !dw_gate || !dw_up || !dw_down)
        return fail(IABN_ERR_NULL, "an output is NULL");
    const ExpertsSpace space = experts_space(M, k, E, C, F, dtype);
    if ((rc = check_workspace(workspace, workspace_bytes, space.all()))) return rc;
    const PlanArgs sorted = plan_of(P, E, const_cast<int32_t*>(plan));
    void* const terms = static_cast<char*>(workspace) + space.h;
    float* const dots = reinterpret_cast<float*>(static_cast<char*>(terms) + space.terms);
    const GroupArgs base = group_args(sorted, weights, k, C, F, act, slope);
    GroupArgs dh = base;
    dh.x = {{dy, dy}, C}, dh.y = {{w_down, w_down}, F};
    dh.M = P, dh.N = F, dh.K = C;
    dh.out[0] = workspace, dh.g = g, dh.u = u, dh.dg = dg, dh.du = du;
    dh.dots = dots;
    grouped(dtype, kOverGroups + kGemmDh, dh, 1, st);
    launch_dots(dots, sorted.place, dweights, P, div_up(F, 64), st);
    GroupArgs dwd = base;
    dwd.x = {{dy, dy}, C}, dwd.y = {{workspace, workspace}, F};
    dwd.M = C, dwd.N = F, dwd.K = P;
    dwd.out[0] = dw_down;
    grouped(dtype, kOverGroups + kGemmDw, dwd, 1, st);
    GroupArgs dwp = base;
    dwp.x = {{dg, du}, F}, dwp.y = {{x, x}, C};
    dwp.M = F, dwp.N = C, dwp.K = P;
    dwp.out[0] = dw_gate, dwp.out[1] = dw_up;
    grouped(dtype, kGroupDwTokensY, dwp, 2, st);
    GroupArgs dxp = base;
    dxp.x = {{dg, du}, F}, dxp.y = {{w_gate, w_up}, C};
    dxp.M = P, dxp.N = C, dxp.K = F;
    dxp.out[0] = terms, dxp.out[1] = static_cast<char*>(terms) + space.low;
    grouped(dtype, kOverGroups + kGemmDx, dxp, 1, st);
    CombineArgs join = {};
    join.terms = terms, join.low = dxp.out[1], join.place = sorted.place, join.y = dx;
    join.M = M, join.C = C, join.k = static_cast<int32_t>(k), join.P = sorted.P, join.splits = 1;
    launch_combine(dtype, join, st);
    return launched("experts_backward");
}

size_t iabn_grad_norm_workspace_size(const int64_t* sizes, int64_t count) {
    GradList list;
    if (check_grads(sizes, count, &list) != IABN_OK) return 0;
    return static_cast<size_t>(list.pieces) * sizeof(double);
}

int iabn_grad_norm(const void* const* grads, const int* dtypes, const int64_t* sizes, int64_t count, float* norm,
                   void* workspace, size_t workspace_bytes, void* stream) {
    GradList list;
    int rc = check_grads(sizes, count, &list);
    if (rc) return rc;
    if ((rc = check_grad_tensors(grads, nullptr, false, dtypes, sizes, count))) return rc;
    if (!norm) return fail(IABN_ERR_NULL, "norm is NULL");
    if ((rc = check_workspace(workspace, workspace_bytes, static_cast<size_t>(list.pieces) * sizeof(double))))
        return rc;
    const hipStream_t st = static_cast<hipStream_t>(stream);
    double* part = static_cast<double*>(workspace);
    over_grads(grads, nullptr, dtypes, sizes, count, list.piece, [&](GradArgs& a) {
        a.part = part;
        launch_grad_norm(a, st);
        part += a.first[a.count];
    });
    launch_grad_join(static_cast<double*>(workspace), list.pieces, norm, st);
    return launched("grad_norm");
}

int iabn_grad_clip(const void* const* grads, void* const* outs, const int* dtypes, const int64_t* sizes,
                   int64_t count, const float* norm, float max_norm, void* stream) {
    GradList list;
    int rc = check_grads(sizes, count, &list);
    if (rc) return rc;
    if ((rc = check_grad_tensors(grads, outs, true, dtypes, sizes, count))) return rc;
    if (!(max_norm >= 0.0f)) return fail(IABN_ERR_PARAM, "max_norm=%g must be >= 0", max_norm);
    if (list.pieces == 0) return ok();
    if (!norm) return fail(IABN_ERR_NULL, "norm is NULL");
    if ((rc = check_apart(grads, outs, dtypes, sizes, count, norm))) return rc;
    const hipStream_t st = static_cast<hipStream_t>(stream);
    over_grads(grads, outs, dtypes, sizes, count, list.piece, [&](GradArgs& a) {
        a.norm = norm, a.max_norm = max_norm;
        launch_grad_clip(a, st);
    });
    return launched("grad_clip");
}

}  // extern "C"
