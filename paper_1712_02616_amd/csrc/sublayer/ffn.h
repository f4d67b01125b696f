// The gated feed-forward block's kernels: what the host side hands to them.
//
//   g = x Wg^T, u = x Wu^T, h = act(g)*u, y = h Wd^T       (x [M, C], W* as stored:
//   dh = dy Wd, dg = dh*u*act'(g), du = dh*act(g)           Wg, Wu [F, C], Wd [C, F])
//   dWd = dy^T h, dWg = dg^T x, dWu = du^T x, dx = dg Wg + du Wu
#pragma once

#include "sublayer.h"

namespace iabn_impl {

// out[m][n] = sum over k of X[m][k]*Y[n][k], an operand stored with k
// contiguous (rows m or n of ld elements) or strided (rows k of ld elements).
struct Operand {
    // Two matrices of one shape: the gate's and the up projection's.  See GemmKind.
    const void* p[2];
    int64_t ld;
};

// The products of the block.
enum GemmKind {
    kGemmUp,       // y: Wg and Wu side by side, k contiguous; out h, and g, u where kept
    kGemmDown,     // out y: both k contiguous
    kGemmDh,       // Wd k-strided; out dg, du, h from g, u
    kGemmDx,       // Wg, Wu k-strided; the sum of two products
    kGemmDw,       // both k-strided; two products (blockIdx.z) of x[z] and y[z] or one
};

struct GemmArgs {
    Operand x, y;
    int64_t M, N, K;
    void* out[2];
    // kGemmUp: h -> out[0], g, u (may be null).  kGemmDh: g, u -> dg, du, out[0] = h.
    const void *g, *u;
    void *dg, *du;
    int act;
    float slope;
    // Where the sum over k is split over blocks: their fp32 sums, [splits]
    // [products][M][N], which launch_join adds up in this order.
    // (Set by the launch.)
    float* part;
    int splits;
};

// out[z][m][n] = sum over the splits, rounded once.
void launch_join(int dtype, const GemmArgs& a, int products, hipStream_t st);

// v with its infinities (below: the negative one) as the largest finite values.
__device__ __forceinline__ float from_below(float v) { return fmaxf(v, -__FLT_MAX__); }
__device__ __forceinline__ float finite_part(float v) {
    return __builtin_amdgcn_fmed3f(v, -__FLT_MAX__, __FLT_MAX__);
}

// act(v) and its derivative, for values stored as DT, each to an error relative to
// itself (the tails too, where they are small).  fp32 values: the library's
// functions and a division.  16-bit ones: the hardware's exponential and
// reciprocal (the exponential's argument is rounded, which costs 2^-24 |v| of SiLU
// and 2^-24 v^2 of GELU), and for the GELU
//
//   Phi(-|v|) = t P(t) exp(-v^2/2),  t = 1/(1 + p |v|/sqrt 2),
//
// whose exponential the derivative shares, at a quarter of the work of the
// library's function.  P has degree 7; p and P were fitted here to the least
// largest relative error over all v (iterated weighted least squares on
// Chebyshev nodes in t): 6.8e-7, evaluated in fp32 9.6e-7.
//
// An infinite v (a projection that overflowed when it was stored) gives the limits,
// no inf * 0; a NaN stays one through s, c or the slope.
template <int ACT, int DT>
__device__ __forceinline__ void activate(float slope, float v, float& a, float& da) {
    if constexpr (ACT == IABN_ACT_SILU) {
        float s;
        if constexpr (DT == IABN_F32) s = 1.0f / (1.0f + expf(-v));
        else s = __builtin_amdgcn_rcpf(1.0f + __expf(-v));
        a = from_below(v) * s;
        da = s * (1.0f + finite_part(v) * (1.0f - s));
    } else if constexpr (ACT == IABN_ACT_GELU) {
        float e, c;
        if constexpr (DT == IABN_F32) {
            e = expf(-0.5f * v * v);
            c = 0.5f * erfcf(v * -0.70710678118654752f);
        } else {
            e = __expf(-0.5f * v * v);
            const float t = __builtin_amdgcn_rcpf(fmaf(0.4598f * 0.70710678118654752f, fabsf(v), 1.0f));
            float q = fmaf(0.06771509742f, t, -0.2269875242f);
            q = fmaf(q, t, 0.1701260875f);
            q = fmaf(q, t, 0.05221715356f);
            q = fmaf(q, t, 0.1869866238f);
            q = fmaf(q, t, 0.2310831802f);
            q = fmaf(q, t, 0.2594458275f);
            q = fmaf(q, t, 0.2594141983f);
            q *= 0.5f * t * e;  // Phi(-|v|)
            c = v < 0.0f ? q : 1.0f - q;
        }
        a = from_below(v) * c;
        da = c + finite_part(v) * e * 0.39894228040143268f;
    } else {
        a = v >= 0.0f ? v : slope == 0.0f && v < 0.0f ? 0.0f : slope * v;
        da = v >= 0.0f ? 1.0f : slope;
    }
}

template <int ACT, int DT, int N>
__device__ __forceinline__ void gate_forward_as(float slope, const float (&g)[N], const float (&u)[N],
                                                float (&h)[N]) {
#pragma unroll
    for (int q = 0; q < N; ++q) {
        float v, d;
        activate<ACT, DT>(slope, g[q], v, d);
        h[q] = v * u[q];
    }
}

template <int DT, int N>
__device__ __forceinline__ void gate_forward(int act, float slope, const float (&g)[N],
                                             const float (&u)[N], float (&h)[N]) {
    if (act == IABN_ACT_SILU) gate_forward_as<IABN_ACT_SILU, DT>(slope, g, u, h);
    else if (act == IABN_ACT_GELU) gate_forward_as<IABN_ACT_GELU, DT>(slope, g, u, h);
    else gate_forward_as<IABN_ACT_LEAKY, DT>(slope, g, u, h);
}

template <int ACT, int DT, int N>
__device__ __forceinline__ void gate_backward_as(float slope, const float (&dh)[N], const float (&g)[N],
                                                 const float (&u)[N], float (&dg)[N], float (&du)[N],
                                                 float (&h)[N]) {
#pragma unroll
    for (int q = 0; q < N; ++q) {
        float v, d;
        activate<ACT, DT>(slope, g[q], v, d);
        dg[q] = dh[q] * u[q] * d;
        du[q] = dh[q] * v;
        h[q] = v * u[q];
    }
}

template <int DT, int N>
__device__ __forceinline__ void gate_backward(int act, float slope, const float (&dh)[N],
                                              const float (&g)[N], const float (&u)[N], float (&dg)[N],
                                              float (&du)[N], float (&h)[N]) {
    if (act == IABN_ACT_SILU) gate_backward_as<IABN_ACT_SILU, DT>(slope, dh, g, u, dg, du, h);
    else if (act == IABN_ACT_GELU) gate_backward_as<IABN_ACT_GELU, DT>(slope, dh, g, u, dg, du, h);
    else gate_backward_as<IABN_ACT_LEAKY, DT>(slope, dh, g, u, dg, du, h);
}

// The products kGemmUp and kGemmDown of at most kFewRows tokens (ffn_few.h).
constexpr int kFewRows = 64;
inline bool few_rows(GemmKind kind, int64_t M) {
    return M <= kFewRows && (kind == kGemmUp || kind == kGemmDown);
}
template <int DT>
bool launch_few(GemmKind kind, const GemmArgs& a, hipStream_t st);

extern template bool launch_few<IABN_F32>(GemmKind, const GemmArgs&, hipStream_t);
extern template bool launch_few<IABN_F16>(GemmKind, const GemmArgs&, hipStream_t);
extern template bool launch_few<IABN_BF16>(GemmKind, const GemmArgs&, hipStream_t);

// products: 2 for kGemmDw of both projections, else 1.
template <int DT>
bool launch_gemm(GemmKind kind, const GemmArgs& a, int products, hipStream_t st);

// How a product runs: tiles of 256x256 (kGemmUp: of 128 columns of each
// projection), 128x128, 64x128 or 32x128 outputs, and over how many blocks the
// sum over k is split.  direct: its tiles go straight to LDS.
enum TileSize { kTile256, kTile128, kTile64, kTile32 };
struct GemmPlan {
    TileSize tile;
    int splits;
};
GemmPlan plan_gemm(int dtype, GemmKind kind, bool direct, int64_t M, int64_t N, int64_t K, int products);
int plan_few(int64_t N, int64_t K, int dtype);

// What a product of these sizes can ask of `part`, in bytes.
size_t part_bytes(int dtype, GemmKind kind, int64_t M, int64_t N, int64_t K, int products);

}  // namespace iabn_impl
