// A feed-forward sublayer of routed experts, and the clipping of a list of
// gradients: what the host side hands to the kernels.
#pragma once

#include "sublayer.h"

namespace iabn_impl {

// ---------------------------------------------------------------- routing

constexpr int kMaxExperts = 1024;
constexpr int kMaxTop = 64;

struct RouteArgs {
    const void* logits;   // [M, E]
    const float* bias;    // [E] or null
    int32_t* experts;     // [M, k]
    float* weights;       // [M, k]
    int64_t M;
    int E, k;
    int groups, kept, group_top, per;  // per = E / groups
    uint32_t per_magic;   // e / per = e*per_magic >> 20 for e < 1024
    float scale;
    bool sigmoid, renormalise;
};

struct RouteBwdArgs {
    const float* dweights;    // [M, k]
    const void* logits;       // [M, E]
    const int32_t* experts;   // [M, k]
    void* dlogits;            // [M, E]
    int64_t M;
    int E, k;
    float scale;
    bool sigmoid, renormalise;
};

bool launch_route_fwd(int dtype, const RouteArgs& a, hipStream_t st);
bool launch_route_bwd(int dtype, const RouteBwdArgs& a, hipStream_t st);

// ---------------------------------------------------------------- the plan

// int32: offsets [E + 1], order [P], place [P], the experts by size [E], and where
// several blocks count, their counts [blocks][E].
struct PlanArgs {
    const int32_t* experts;  // [P]
    int32_t *offsets, *order, *place, *by_size, *counts;
    int32_t P, E;
    int32_t blocks, span;    // pairs of a block
};
PlanArgs plan_of(int64_t P, int64_t E, int32_t* plan);
int64_t plan_size(int64_t P, int64_t E);
void launch_plan(const PlanArgs& a, hipStream_t st);

// ---------------------------------------------------------------- gradients

// A list of tensors is cut into pieces, one a block; a launch takes up to
// kGradTensors tensors of it (its arguments hold fewer than 4096 bytes).
constexpr int kGradTensors = 128;
struct GradArgs {
    const void* in[kGradTensors];
    void* out[kGradTensors];
    int64_t n[kGradTensors];
    int32_t first[kGradTensors + 1];  // of each tensor's pieces
    uint8_t dtype[kGradTensors];
    int32_t count;
    int32_t piece;                    // elements
    double* part;                     // the launch's pieces' sums
    const float* norm;
    float max_norm;
};
static_assert(sizeof(GradArgs) <= 4096, "a launch's arguments");

void launch_grad_norm(const GradArgs& a, hipStream_t st);
void launch_grad_join(const double* part, int64_t n, float* norm, hipStream_t st);
void launch_grad_clip(const GradArgs& a, hipStream_t st);

}  // namespace iabn_impl
