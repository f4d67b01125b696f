// Routing: the k experts of every token from its logits, and their weights.
//
//   s = softmax(l) or sigmoid(l),  c = s + bias;  a group's score is the sum of its
//   group_top highest c; the k highest c of the kept groups, then
//   w_j = scale*s_j, or scale*s_j/sum of the chosen s.
//
// A row lies in the registers of L lanes, V consecutive experts each; every
// choice is one maximum over the row and the lowest index that has it.  Scores are
// ordered as unsigned integers (the float's bits, those of negative ones turned
// over), 0 for what may not be chosen, the largest for a NaN.  Without a bias the
// order of the scores is that of the logits, which is exact in 32 bits.  With one
// (or with groups), scores next to each other decide: they are formed in 32 bits
// with a bound of their error, and where two that decide are closer than that, the
// wave forms and compares them in 64 bits.
#include <type_traits>

#include "routed.h"

namespace iabn_impl {
namespace {

constexpr float kInf = __builtin_inff();

// ---------------------------------------------------------------- over the lanes of a row

template <int CTRL>
__device__ __forceinline__ uint32_t dpp_u32(uint32_t v) {
    return static_cast<uint32_t>(
        __builtin_amdgcn_update_dpp(0, static_cast<int>(v), CTRL, 0xF, 0xF, true));
}

// op over L lanes (16 or 64, all of the wave active), in each of them: lane
// pairs, quads, mirrored halves and rows of 16, then the four rows through
// scalar registers.
template <int L, typename Op>
__device__ __forceinline__ uint32_t over_row(uint32_t v, Op op) {
    v = op(v, dpp_u32<0xB1>(v));
    v = op(v, dpp_u32<0x4E>(v));
    v = op(v, dpp_u32<0x141>(v));
    v = op(v, dpp_u32<0x140>(v));
    if constexpr (L == 64) {
        const auto lane = [&](int i) { return static_cast<uint32_t>(__builtin_amdgcn_readlane(static_cast<int>(v), i)); };
        v = op(op(lane(0), lane(16)), op(lane(32), lane(48)));
    }
    return v;
}
template <int L>
__device__ __forceinline__ uint32_t row_max(uint32_t v) {
    return over_row<L>(v, [](uint32_t a, uint32_t b) { return a > b ? a : b; });
}
template <int L>
__device__ __forceinline__ uint32_t row_min(uint32_t v) {
    return over_row<L>(v, [](uint32_t a, uint32_t b) { return a < b ? a : b; });
}
template <int L>
__device__ __forceinline__ float row_maxf(float v) {
    return __builtin_bit_cast(float, over_row<L>(__builtin_bit_cast(uint32_t, v), [](uint32_t a, uint32_t b) {
        return __builtin_bit_cast(uint32_t, fmaxf(__builtin_bit_cast(float, a), __builtin_bit_cast(float, b)));
    }));
}
template <int L>
__device__ __forceinline__ float row_add(float v) {
    return __builtin_bit_cast(float, over_row<L>(__builtin_bit_cast(uint32_t, v), [](uint32_t a, uint32_t b) {
        return __builtin_bit_cast(uint32_t, __builtin_bit_cast(float, a) + __builtin_bit_cast(float, b));
    }));
}
template <int CTRL>
__device__ __forceinline__ double dpp_f64(double v) {
    const uint64_t b = __builtin_bit_cast(uint64_t, v);
    return __builtin_bit_cast(double, uint64_t(dpp_u32<CTRL>(static_cast<uint32_t>(b >> 32))) << 32 |
                                          dpp_u32<CTRL>(static_cast<uint32_t>(b)));
}
template <int L>
__device__ __forceinline__ double row_add64(double v) {
    v += dpp_f64<0xB1>(v);
    v += dpp_f64<0x4E>(v);
    v += dpp_f64<0x141>(v);
    v += dpp_f64<0x140>(v);
    if constexpr (L == 64) {
        v += __shfl_xor(v, 16);
        v += __shfl_xor(v, 32);
    }
    return v;
}

// ---------------------------------------------------------------- scores

// Bits that are ordered as the value (-0 as 0, a NaN above all); 0 is below all.
__device__ __forceinline__ uint32_t order32(float v) {
    if (v != v) return 0xFFFFFFFFu;
    const uint32_t b = __builtin_bit_cast(uint32_t, v + 0.0f);
    return b >> 31 ? ~b : b | 0x80000000u;
}
__device__ __forceinline__ uint64_t order64(double v) {
    if (v != v) return ~uint64_t(0);
    const uint64_t b = __builtin_bit_cast(uint64_t, v + 0.0);
    return b >> 63 ? ~b : b | uint64_t(1) << 63;
}

// exp(v - m), with what the difference loses.
__device__ __forceinline__ float exp_from(float v, float m) {
    const float d = v - m, e = expf(d);
    const float back = d + m;  // (as in a two-sum)
    const float lost = (v - back) + ((back - d) - m);
    return d == d && fabsf(d) < kInf ? fmaf(e, lost, e) : e;
}
// 1/(1 + exp(-v)).
__device__ __forceinline__ float sigmoid(float v) { return 1.0f / (1.0f + expf(-v)); }

// The row's logits, V of each lane; -inf past the last expert.
template <int DT, int V>
__device__ __forceinline__ void load_logits(const void* logits, int64_t row, int E, int first, float (&v)[V]) {
    using T = typename Elem<DT>::T;
    const T* p = static_cast<const T*>(logits) + row * E + first;
    typedef T vec __attribute__((ext_vector_type(V)));
    typedef T mem __attribute__((ext_vector_type(V), aligned(sizeof(T))));
    if (first + V <= E) {
        if constexpr (V == 1) {
            v[0] = static_cast<float>(*p);
        } else {
            const vec r = *reinterpret_cast<const mem*>(p);
#pragma unroll
            for (int j = 0; j < V; ++j) v[j] = static_cast<float>(r[j]);
        }
    } else {
#pragma unroll
        for (int j = 0; j < V; ++j) v[j] = first + j < E ? static_cast<float>(p[j]) : -kInf;
    }
}

// A row's largest logit, and the sum of exp(l - largest) in a given lane's part.
template <int V>
__device__ __forceinline__ float largest(const float (&v)[V]) {
    float m = v[0];
#pragma unroll
    for (int j = 1; j < V; ++j) m = fmaxf(m, v[j]);
    return m;
}

__device__ __forceinline__ void wave_fence() {
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
}

// The groups that a row keeps, a bit each.  t: the scores in LDS, -inf for what
// may not be chosen; gs: a place for the groups' scores.  The scores are off by at
// most `tol`, and sums of two by 2^-22 of themselves besides: `sure` turns false
// where that could change which groups are kept.
template <int L, typename S>
__device__ __forceinline__ uint64_t kept_groups(const RouteArgs& a, const S* t, S* gs, int lane, S tol, bool& sure) {
    // A group belongs to `per_group` lanes, which look through it in turn.
    const int per_group = L / a.groups, g = lane / per_group, part = lane - g * per_group;
    const S none = -kInf;
    S top1 = none, top2 = none;
    const auto larger = [](S x, S y) { return x > y ? x : y; };
    const auto smaller = [](S x, S y) { return x < y ? x : y; };
    if (g < a.groups)
        for (int i = part; i < a.per; i += per_group) {
            S v = t[g * a.per + i];
            if (v != v) v = kInf;
            top2 = larger(top2, smaller(top1, v));
            top1 = larger(top1, v);
        }
    for (int d = 1; d < per_group; d *= 2) {
        const S o1 = __shfl_down(top1, d, L), o2 = __shfl_down(top2, d, L);
        if (part + d < per_group) {
            top2 = larger(smaller(top1, o1), larger(top2, o2));
            top1 = larger(top1, o1);
        }
    }
    if (a.group_top == 2 && top2 > none) top1 += top2;
    if (g < a.groups && part == 0) gs[g] = top1;
    wave_fence();
    bool keep = false, clear = true;
    if (lane < a.groups) {
        const S mine = gs[lane];
        // How many are above, and how many surely are, and may be.
        int above = 0, surely = 0, maybe = 0;
        for (int i = 0; i < a.groups; ++i) {
            const S other = gs[i];
            const bool same = i == lane;
            above += other > mine || (other == mine && i < lane);
            if constexpr (sizeof(S) == 4) {
                const S far = 2.0f * tol + 2.4e-7f * (fabsf(mine) + fabsf(other));
                surely += !same && other - mine > far;
                maybe += !same && other - mine > -far;
            }
        }
        keep = above < a.kept && mine > none;
        if constexpr (sizeof(S) == 4) clear = mine == none || maybe < a.kept || surely >= a.kept;
    }
    sure = sure && __ballot(!clear) == 0;
    const uint64_t all = __ballot(keep);
    if constexpr (L == 64) return all;
    return all >> (lane_id() / L * L) & ((uint64_t(1) << L) - 1);
}

// What a row chose: lane i has the i-th expert (-1: none) and its logit.
struct Choice {
    int expert = -1;
    float logit = 0.0f;
};

// The k highest keys, one after the other (64-bit ones: `low` is their lower half).
// SCORES: the keys are scores, off by tol + 2^-23 of themselves; one choice more is
// looked at, and `sure` turns false where two that follow each other are too close.
// LOGITS: the keys are the logits.
enum KeyKind { kLogitKeys, kScoreKeys, kWideKeys };
template <int L, int V, KeyKind KEYS>
__device__ __forceinline__ Choice choose(uint32_t (&key)[V], uint32_t (&low)[KEYS == kWideKeys ? V : 1], int k, int lane,
                                         float tol, bool& sure) {
    constexpr bool kWide = KEYS == kWideKeys;
    const int first = lane * V;
    Choice c;
    float before = kInf;
    for (int i = 0; i < (KEYS == kScoreKeys ? k + 1 : k); ++i) {
        uint32_t best = key[0], best_low = kWide ? low[0] : 0;
#pragma unroll
        for (int j = 1; j < V; ++j) {
            if constexpr (kWide) {
                const bool more = key[j] > best || (key[j] == best && low[j] > best_low);
                best = more ? key[j] : best;
                best_low = more ? low[j] : best_low;
            } else {
                best = key[j] > best ? key[j] : best;
            }
        }
        const uint32_t top = row_max<L>(best);
        const uint32_t top_low = kWide ? row_max<L>(best == top ? best_low : 0) : 0;
        const float value = __builtin_bit_cast(float, top >> 31 ? top & 0x7FFFFFFFu : ~top);
        if constexpr (KEYS == kScoreKeys) {
            // (A NaN is never far from another.)
            sure = sure && (top == 0 || before - value > 2.0f * tol + 2.4e-7f * fabsf(value));
            before = value;
            if (i == k) break;
        }
        uint32_t at = 0xFFFFFFFFu;
#pragma unroll
        for (int j = V - 1; j >= 0; --j)
            at = key[j] == top && (!kWide || low[j] == top_low) ? first + j : at;
        const uint32_t e = row_min<L>(at);
        const uint32_t mine = e - first;
#pragma unroll
        for (int j = 0; j < V; ++j) key[j] = mine == static_cast<uint32_t>(j) ? 0 : key[j];
        if constexpr (kWide)
#pragma unroll
            for (int j = 0; j < V; ++j) low[j] = mine == static_cast<uint32_t>(j) ? 0 : low[j];
        if (lane == i && top != 0) {
            c.expert = static_cast<int>(e);
            if constexpr (KEYS == kLogitKeys) c.logit = top == 0xFFFFFFFFu ? __builtin_nanf("") : value;
        }
    }
    return c;
}

template <int DT, int L, int V, bool SCORED>
__global__ __launch_bounds__(kThreads) void route_kernel(RouteArgs a) {
    using T = typename Elem<DT>::T;
    const int lane = threadIdx.x % L, first = lane * V;
    const int64_t own = int64_t(blockIdx.x) * (kThreads / L) + threadIdx.x / L;
    const bool there = own < a.M;
    const int64_t row = there ? own : a.M - 1;  // (every lane stays for the maxima)

    float v[V];
    load_logits<DT, V>(a.logits, row, a.E, first, v);
    const float high = a.sigmoid ? 0.0f : row_maxf<L>(largest(v));
    float total = 0.0f;  // of the softmax
    if (!a.sigmoid && !a.renormalise) {
#pragma unroll
        for (int j = 0; j < V; ++j) total += exp_from(v[j], high);
        total = row_add<L>(total);
    }

    Choice c;
    bool sure = true;
    if constexpr (SCORED) {
        extern __shared__ double scores[];  // [rows][E], [rows][groups], of either type
        const bool grouped = a.kept < a.groups;
        float bias[V];
        bool may[V];
#pragma unroll
        for (int j = 0; j < V; ++j) {
            bias[j] = a.bias && first + j < a.E ? a.bias[first + j] : 0.0f;
            may[j] = v[j] != -kInf && bias[j] != -kInf;
        }
        // The keys of scores s, of what may be chosen and is in a kept group.
        const auto in_groups = [&](const auto& s, auto tol) {
            using S = std::remove_cv_t<decltype(tol)>;
            if (!grouped) return ~uint64_t(0);
            // (A row's place is the same for both types: other waves have theirs in use.)
            S* const t = reinterpret_cast<S*>(scores + threadIdx.x / L * a.E);
            S* const gs = reinterpret_cast<S*>(scores + kThreads / L * a.E + threadIdx.x / L * a.groups);
#pragma unroll
            for (int j = 0; j < V; ++j)
                if (first + j < a.E) t[first + j] = may[j] ? s[j] : static_cast<S>(-kInf);
            wave_fence();
            return kept_groups<L, S>(a, t, gs, lane, tol, sure);
        };
        const auto in_kept = [&](uint64_t groups, int j) {
            const int g = static_cast<int>(static_cast<uint32_t>(first + j) * a.per_magic >> 20);
            return may[j] && (!grouped || (groups >> g & 1));
        };
        uint32_t key[V];
        {
            // In 32 bits.  A sigmoid is off by less than 2^-22, a term of the softmax by
            // less than 2^-18 of the largest (its sum by 22 roundings).
            float s[V], sum = 0.0f, tol = 0x1p-21f;
#pragma unroll
            for (int j = 0; j < V; ++j) {
                s[j] = __expf(a.sigmoid ? -v[j] : v[j] - high);
                if (a.sigmoid) s[j] = __builtin_amdgcn_rcpf(1.0f + s[j]);
                sum += s[j];
            }
            if (!a.sigmoid) {
                const float scale = 1.0f / row_add<L>(sum);
                tol = scale * 0x1p-18f;
#pragma unroll
                for (int j = 0; j < V; ++j) s[j] *= scale;
            }
#pragma unroll
            for (int j = 0; j < V; ++j) s[j] += bias[j];
            const uint64_t groups = in_groups(s, tol);
#pragma unroll
            for (int j = 0; j < V; ++j) key[j] = in_kept(groups, j) ? order32(a.bias ? s[j] : v[j]) : 0;
            uint32_t none[1];
            if (a.bias) c = choose<L, V, kScoreKeys>(key, none, a.k, lane, tol, sure);
            else c = choose<L, V, kLogitKeys>(key, none, a.k, lane, tol, sure);
        }
        if (__ballot(!sure) != 0) {
            double s[V], sum = 0.0;
#pragma unroll
            for (int j = 0; j < V; ++j) {
                const double l = v[j];
                s[j] = a.sigmoid ? 1.0 / (1.0 + exp(-l)) : exp(l - static_cast<double>(high));
                sum += s[j];
            }
            if (!a.sigmoid) sum = row_add64<L>(sum);
#pragma unroll
            for (int j = 0; j < V; ++j) s[j] = (a.sigmoid ? s[j] : s[j] / sum) + bias[j];
            wave_fence();
            const uint64_t groups = in_groups(s, 0.0);
            uint32_t low[V];
#pragma unroll
            for (int j = 0; j < V; ++j) {
                const uint64_t o = in_kept(groups, j) ? order64(a.bias ? s[j] : v[j]) : 0;
                key[j] = static_cast<uint32_t>(o >> 32);
                low[j] = static_cast<uint32_t>(o);
            }
            c = choose<L, V, kWideKeys>(key, low, a.k, lane, 0.0f, sure);
        }
        if (c.expert >= 0) c.logit = static_cast<float>(static_cast<const T*>(a.logits)[row * a.E + c.expert]);
    } else {
        uint32_t key[V], none[1];
#pragma unroll
        for (int j = 0; j < V; ++j) key[j] = v[j] == -kInf ? 0 : order32(v[j]);
        c = choose<L, V, kLogitKeys>(key, none, a.k, lane, 0.0f, sure);
    }
    const int mine = c.expert;
    const float logit = c.logit;

    float w = 0.0f;
    if (a.renormalise) {
        // exp(l - m)/sum, and for the sigmoid exp(min(l, 0) - m)/(1 + exp(-|l|)): of
        // any logits, one term is not small.
        const float x = a.sigmoid ? fminf(logit, 0.0f) : logit;
        const float m = row_maxf<L>(mine >= 0 ? x : -kInf);
        w = a.sigmoid ? exp_from(x, m) / (1.0f + expf(-fabsf(logit))) : exp_from(x, m);
        if (logit != logit) w = logit;
        w = mine >= 0 ? w : 0.0f;
        w = w / row_add<L>(w);
    } else {
        w = a.sigmoid ? sigmoid(logit) : exp_from(logit, high) / total;
    }
    if (there && lane < a.k) {
        a.experts[row * a.k + lane] = mine;
        a.weights[row * a.k + lane] = mine >= 0 ? a.scale * w : 0.0f;
    }
}

// ---------------------------------------------------------------- backward
//
//   d_j = scale*dw_j;  softmax: dl = s*(d - sum of s_j d_j), d = 0 for what was not
//   chosen; sigmoid: dl = d*s*(1 - s).  Renormalised, p_j = s_j/sum of the chosen s:
//   q_j = p_j*(d_j - sum p d), dl = q (softmax) or q*(1 - s) (sigmoid), 0 elsewhere.
template <int DT, int L, int V>
__global__ __launch_bounds__(kThreads) void route_bwd_kernel(RouteBwdArgs a) {
    using T = typename Elem<DT>::T;
    const int lane = threadIdx.x % L, first = lane * V;
    const int64_t own = int64_t(blockIdx.x) * (kThreads / L) + threadIdx.x / L;
    const bool there = own < a.M;
    const int64_t row = there ? own : a.M - 1;

    float v[V];
    load_logits<DT, V>(a.logits, row, a.E, first, v);
    // Lane i: the i-th choice.
    int mine = lane < a.k ? a.experts[row * a.k + lane] : -1;
    if (mine < 0 || mine >= a.E) mine = -1;
    float logit = mine >= 0 ? static_cast<float>(static_cast<const T*>(a.logits)[row * a.E + mine]) : -kInf;
    if (logit == -kInf) mine = -1;
    float d = mine >= 0 ? a.scale * a.dweights[row * a.k + lane] : 0.0f;

    float high = 0.0f, total = 1.0f, dot = 0.0f;
    if (a.renormalise) {
        const float x = a.sigmoid ? fminf(logit, 0.0f) : logit;
        const float m = row_maxf<L>(x);
        float p = a.sigmoid ? exp_from(x, m) / (1.0f + expf(-fabsf(logit))) : exp_from(x, m);
        if (logit != logit) p = logit;
        p = mine >= 0 ? p : 0.0f;
        const float sum = row_add<L>(p);
        p = mine >= 0 ? p / sum : 0.0f;
        d = p * (d - row_add<L>(p * d));
        if (a.sigmoid) d *= sigmoid(-logit);
    } else if (!a.sigmoid) {
        high = row_maxf<L>(largest(v));
        total = 0.0f;
#pragma unroll
        for (int j = 0; j < V; ++j) {
            v[j] = v[j] == -kInf ? 0.0f : exp_from(v[j], high);
            total += v[j];
        }
        total = row_add<L>(total);
        dot = row_add<L>(mine >= 0 ? exp_from(logit, high) / total * d : 0.0f);
    }

    float sum[V] = {};
    for (int i = 0; i < a.k; ++i) {
        const int e = __shfl(mine, i, L);
        const float di = __shfl(d, i, L);
#pragma unroll
        for (int j = 0; j < V; ++j) sum[j] += e == first + j ? di : 0.0f;
    }
#pragma unroll
    for (int j = 0; j < V; ++j) {
        if (a.renormalise) v[j] = sum[j];
        else if (a.sigmoid) v[j] = sum[j] == 0.0f ? 0.0f : sum[j] * sigmoid(v[j]) * sigmoid(-v[j]);
        else v[j] = v[j] == 0.0f ? 0.0f : v[j] / total * (sum[j] - dot);
    }
    if (!there) return;
    T* const p = static_cast<T*>(a.dlogits) + row * a.E + first;
    typedef T vec __attribute__((ext_vector_type(V)));
    typedef T mem __attribute__((ext_vector_type(V), aligned(sizeof(T))));
    if (first + V <= a.E) {
        if constexpr (V == 1) {
            *p = static_cast<T>(v[0]);
        } else {
            vec r;
#pragma unroll
            for (int j = 0; j < V; ++j) r[j] = static_cast<T>(v[j]);
            *reinterpret_cast<mem*>(p) = r;
        }
    } else {
#pragma unroll
        for (int j = 0; j < V; ++j)
            if (first + j < a.E) p[j] = static_cast<T>(v[j]);
    }
}

// ---------------------------------------------------------------- launches

// Rows in 16 lanes where they and the choices fit: four rows share every
// instruction of the maxima.
bool narrow_rows(int64_t M, int E, int k, int groups) { return E <= 256 && k <= 16 && groups <= 16 && M > 1024; }

template <int DT, int L, int V>
void launch_fwd_as(const RouteArgs& a, hipStream_t st) {
    const int rows = kThreads / L;
    const dim3 grid(static_cast<uint32_t>((a.M + rows - 1) / rows));
    const bool grouped = a.kept < a.groups;
    const size_t lds = grouped ? static_cast<size_t>(rows) * (a.E + a.groups) * sizeof(double) : 0;
    if (a.bias || grouped) route_kernel<DT, L, V, true><<<grid, kThreads, lds, st>>>(a);
    else route_kernel<DT, L, V, false><<<grid, kThreads, 0, st>>>(a);
}

template <int DT>
void launch_fwd(const RouteArgs& a, hipStream_t st) {
    if (narrow_rows(a.M, a.E, a.k, a.groups)) {
        if (a.E <= 16) launch_fwd_as<DT, 16, 1>(a, st);
        else if (a.E <= 64) launch_fwd_as<DT, 16, 4>(a, st);
        else if (a.E <= 128) launch_fwd_as<DT, 16, 8>(a, st);
        else launch_fwd_as<DT, 16, 16>(a, st);
    } else {
        if (a.E <= 64) launch_fwd_as<DT, 64, 1>(a, st);
        else if (a.E <= 256) launch_fwd_as<DT, 64, 4>(a, st);
        else launch_fwd_as<DT, 64, 16>(a, st);
    }
}

template <int DT, int L, int V>
void launch_bwd_as(const RouteBwdArgs& a, hipStream_t st) {
    const int rows = kThreads / L;
    route_bwd_kernel<DT, L, V><<<dim3(static_cast<uint32_t>((a.M + rows - 1) / rows)), kThreads, 0, st>>>(a);
}

template <int DT>
void launch_bwd(const RouteBwdArgs& a, hipStream_t st) {
    if (narrow_rows(a.M, a.E, a.k, 1)) {
        if (a.E <= 16) launch_bwd_as<DT, 16, 1>(a, st);
        else if (a.E <= 64) launch_bwd_as<DT, 16, 4>(a, st);
        else if (a.E <= 128) launch_bwd_as<DT, 16, 8>(a, st);
        else launch_bwd_as<DT, 16, 16>(a, st);
    } else {
        if (a.E <= 64) launch_bwd_as<DT, 64, 1>(a, st);
        else if (a.E <= 256) launch_bwd_as<DT, 64, 4>(a, st);
        else launch_bwd_as<DT, 64, 16>(a, st);
    }
}

}  // namespace

bool launch_route_fwd(int dtype, const RouteArgs& a, hipStream_t st) {
    switch (dtype) {
        case IABN_F32: launch_fwd<IABN_F32>(a, st); return true;
        case IABN_F16: launch_fwd<IABN_F16>(a, st); return true;
        case IABN_BF16: launch_fwd<IABN_BF16>(a, st); return true;
        default: return false;
    }
}

bool launch_route_bwd(int dtype, const RouteBwdArgs& a, hipStream_t st) {
    switch (dtype) {
        case IABN_F32: launch_bwd<IABN_F32>(a, st); return true;
        case IABN_F16: launch_bwd<IABN_F16>(a, st); return true;
        case IABN_BF16: launch_bwd<IABN_BF16>(a, st); return true;
        default: return false;
    }
}

}  // namespace iabn_impl
