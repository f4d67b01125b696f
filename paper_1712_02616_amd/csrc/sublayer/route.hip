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
// with a bound of their error, and where two that decide are closer than that, those
// few are formed and compared in 64 bits.  (That is what one wave in a hundred does;
// all scores in 64 bits for it (16384, 256) bf16, 8 of 256: 29 us instead of 20.)
//
// Bound by instructions: (16384, 256) bf16, 8 of 256 by sigmoids with a bias in 4 of 8
// groups, 20 us for 9.5 MB, vector units at work in 0.69 of the cycles (17.6 with no
// close scores; 12.5 of them without the groups, 12.2 with one choice).  A choice goes
// through a lane's 16 values three times, a group's sum through LDS twice; the rest of
// the cycles are steps that four waves a SIMD, which go through them once, do not hide.
// Rows in 16 lanes share the instructions of the maxima (in 64 lanes: 27 us, the
// (4099, 61) fp32 case 4.4 instead of 3.7; the backward 9.7 instead of 7.6).  One
// row: 2.6 us, a launch.
#include <limits>
#include <type_traits>
#include <utility>

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

// A value of the row's lane I, in all of its lanes (of 64: the wave's).
constexpr int kRowLanes = 16;
template <int L, int I>
__device__ __forceinline__ uint32_t from_lane(uint32_t v) {
    if constexpr (L == 16) return dpp_u32<0x150 + I>(v);
    else return static_cast<uint32_t>(__builtin_amdgcn_readlane(static_cast<int>(v), I));
}
// fn(i) for the choices i < k, the first 16 of them, i a constant.
template <int L, typename Fn, int... I>
__device__ __forceinline__ void each_choice(int k, Fn fn, std::integer_sequence<int, I...>) {
    ((I < k ? fn(std::integral_constant<int, I>()) : void()), ...);
}
template <int L, typename Fn>
__device__ __forceinline__ void each_choice(int k, Fn fn) {
    each_choice<L>(k, fn, std::make_integer_sequence<int, kRowLanes>());
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

// A row's values of E experts, V of each lane; -inf past the last one.
template <int DT, int V>
__device__ __forceinline__ void load_row(const void* rows, int64_t row, int E, int first, float (&v)[V]) {
    using T = typename Elem<DT>::T;
    const T* p = static_cast<const T*>(rows) + row * E + first;
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
// may not be chosen; gs: a place for the groups' scores.  32-bit scores are off by
// at most `tol` and their own roundings, a group's by twice that: `sure` turns false
// where it could change which groups are kept.  Two scores that cancel in a group's
// keep their roundings, 2^-24 of each: they are bounded by the sum of their sizes,
// which stands behind the groups' scores.  Where that is past fp32's range no
// difference is above it and nothing is sure; a group's score is no less than the
// lowest number, -inf only where the group has nothing.
template <int L, typename S>
__device__ __forceinline__ uint64_t kept_groups(const RouteArgs& a, const S* t, S* gs, int lane, S tol, bool& sure) {
    // A group belongs to `per_group` lanes, which look through it in turn.
    const int per_group = L / a.groups, g = lane / per_group, part = lane - g * per_group;
    const S none = -kInf;
    S top1 = none, top2 = none;
    const auto larger = [](S x, S y) { return x > y ? x : y; };
    const auto smaller = [](S x, S y) { return x < y ? x : y; };
    // (Eight reads on their way at a time; past the group's end, its last one again.)
    constexpr int kReads = 8;
    if (g < a.groups)
        for (int i = part; i < a.per; i += kReads * per_group) {
            S v[kReads];
#pragma unroll
            for (int q = 0; q < kReads; ++q) v[q] = t[g * a.per + min(i + q * per_group, a.per - 1)];
#pragma unroll
            for (int q = 0; q < kReads; ++q) {
                const S x = i + q * per_group >= a.per ? none : v[q] != v[q] ? static_cast<S>(kInf) : v[q];
                top2 = larger(top2, smaller(top1, x));
                top1 = larger(top1, x);
            }
        }
    for (int d = 1; d < per_group; d *= 2) {
        const S o1 = __shfl_down(top1, d, L), o2 = __shfl_down(top2, d, L);
        if (part + d < per_group) {
            top2 = larger(smaller(top1, o1), larger(top2, o2));
            top1 = larger(top1, o1);
        }
    }
    S size = top1 == none ? S(0) : top1 < 0 ? -top1 : top1;
    if (a.group_top == 2 && top2 > none) {
        size += top2 < 0 ? -top2 : top2;
        top1 = larger(top1 + top2, std::numeric_limits<S>::lowest());
    }
    constexpr bool kNarrow = sizeof(S) == 4;  // (half of the place is for the sizes)
    if (g < a.groups && part == 0) {
        gs[g] = top1;
        if constexpr (kNarrow) gs[a.groups + g] = size;
    }
    wave_fence();
    bool keep = false, clear = true;
    if (lane < a.groups) {
        const S mine = gs[lane], my_size = kNarrow ? gs[a.groups + lane] : S(0);
        // How many are above, and how many surely are, and may be.
        int above = 0, surely = 0, maybe = 0;
        for (int i0 = 0; i0 < a.groups; i0 += kReads) {
            S others[kReads], sizes[kReads];
#pragma unroll
            for (int q = 0; q < kReads; ++q) {
                others[q] = gs[min(i0 + q, a.groups - 1)];
                if constexpr (kNarrow) sizes[q] = gs[a.groups + min(i0 + q, a.groups - 1)];
            }
#pragma unroll
            for (int q = 0; q < kReads; ++q) {
                const int i = i0 + q;
                const S other = others[q];
                const bool is = i < a.groups && i != lane;
                above += is && (other > mine || (other == mine && i < lane));
                if constexpr (kNarrow) {
                    const S far = 4.0f * tol + 0x1p-22f * (my_size + sizes[q]);
                    surely += is && other - mine > far;
                    maybe += is && !(mine - other > far);
                }
            }
        }
        keep = above < a.kept && mine > none;
        if constexpr (kNarrow) clear = mine == none || maybe < a.kept || surely >= a.kept;
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
// kScoreKeys: they are scores off by at most tol.  Then more are taken until the
// next one is surely below the k-th, and `close` says how it went: kApart, no two that
// follow each other too close; kClose, the right ones are among the first
// `taken`; kLost, there are more than lanes.  kLogitKeys: the keys are the logits.
enum KeyKind { kLogitKeys, kScoreKeys, kWideKeys };
enum Closeness { kApart, kClose, kLost };
template <int L, int V, KeyKind KEYS>
__device__ __forceinline__ Choice choose(uint32_t (&key)[V], uint32_t (&low)[KEYS == kWideKeys ? V : 1], int k, int lane,
                                         float tol, int& taken, Closeness& close) {
    constexpr bool kWide = KEYS == kWideKeys;
    const int first = lane * V;
    Choice c;
    float before = kInf;
    bool apart = true, closed = false;
    close = kApart;
    for (taken = 0; KEYS == kScoreKeys || taken < k; ++taken) {
        const int i = taken;
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
            // (The scores' own roundings: 2^-24 of them.  A NaN is never far from another.)
            const bool far = top == 0 || before - value > 2.0f * tol + 0x1p-24f * (fabsf(before) + fabsf(value)) || i == 0;
            before = value;
            apart = apart && (far || closed);
            closed = closed || (i >= k && far);
            if (i >= k && __ballot(!closed) == 0) {
                close = __ballot(!apart) == 0 ? kApart : kClose;
                break;
            }
            if (i == L) {
                close = kLost;
                break;
            }
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

// Lane i's choice of `taken`, with its 64-bit key, goes to the lane of its rank.
template <int L>
__device__ __forceinline__ int by_rank(int expert, uint64_t key, int taken, int lane) {
    int rank = 0;
    for (int j = 0; j < taken; ++j) {
        const uint64_t other = uint64_t(__shfl(static_cast<uint32_t>(key >> 32), j, L)) << 32 |
                               __shfl(static_cast<uint32_t>(key), j, L);
        const int e = __shfl(expert, j, L);
        rank += other > key || (other == key && e < expert);
    }
    int out = -1;
    for (int j = 0; j < taken; ++j) {
        const int r = __shfl(rank, j, L), e = __shfl(expert, j, L);
        out = r == lane && e >= 0 ? e : out;
    }
    return out;
}

template <int DT, int L, int V, bool SCORED>
__global__ __launch_bounds__(kThreads) void route_kernel(RouteArgs a) {
    using T = typename Elem<DT>::T;
    const int lane = threadIdx.x % L, first = lane * V;
    const int64_t own = int64_t(blockIdx.x) * (kThreads / L) + threadIdx.x / L;
    const bool there = own < a.M;
    const int64_t row = there ? own : a.M - 1;  // (every lane stays for the maxima)

    float v[V];
    load_row<DT, V>(a.logits, row, a.E, first, v);
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
        extern __shared__ double scores[];  // [rows][V*L], [rows][groups], of either type
        const bool grouped = a.kept < a.groups;
        float bias[V];
        bool may[V];
        if (a.bias) load_row<IABN_F32, V>(a.bias, 0, a.E, first, bias);
#pragma unroll
        for (int j = 0; j < V; ++j) {
            bias[j] = a.bias ? bias[j] : 0.0f;
            may[j] = v[j] != -kInf && bias[j] != -kInf;
        }
        // The keys of scores s, of what may be chosen and is in a kept group.
        const auto in_groups = [&](const auto& s, auto tol) {
            using S = std::remove_cv_t<decltype(tol)>;
            if (!grouped) return ~uint64_t(0);
            // (A row's place is the same for both types: other waves have theirs in use.)
            S* const t = reinterpret_cast<S*>(scores + threadIdx.x / L * (V * L));
            S* const gs = reinterpret_cast<S*>(scores + kThreads * V + threadIdx.x / L * a.groups);
#pragma unroll
            for (int j = 0; j < V; ++j) t[first + j] = may[j] ? s[j] : static_cast<S>(-kInf);
            wave_fence();
            return kept_groups<L, S>(a, t, gs, lane, tol, sure);
        };
        const auto in_kept = [&](uint64_t groups, int j) {
            const int g = static_cast<int>(static_cast<uint32_t>(first + j) * a.per_magic >> 20);
            return may[j] && (!grouped || (groups >> g & 1));
        };
        // In 32 bits.  A sigmoid is off by less than 2^-22, a term of the softmax by less
        // than 2^-18 of the largest (its sum by 22 roundings).
        float s[V], sum = 0.0f, tol = 0x1p-22f;
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
        // And in 64, where they are asked for.
        double sum64 = 0.0;
        const auto score64 = [&](float l) {
            return a.sigmoid ? 1.0 / (1.0 + exp(-static_cast<double>(l)))
                             : exp(static_cast<double>(l) - static_cast<double>(high)) / sum64;
        };
        const auto sum_in_64 = [&]() {
            if (a.sigmoid || sum64 != 0.0) return;
            double t = 0.0;
#pragma unroll
            for (int j = 0; j < V; ++j) t += exp(static_cast<double>(v[j]) - static_cast<double>(high));
            sum64 = row_add64<L>(t);
        };
        const auto all_in_64 = [&](double (&s64)[V]) {
            sum_in_64();
#pragma unroll
            for (int j = 0; j < V; ++j) s64[j] = score64(v[j]) + bias[j];
        };
        uint64_t groups = in_groups(s, tol);
        if (__ballot(!sure) != 0) {
            double s64[V];
            all_in_64(s64);
            wave_fence();
            groups = in_groups(s64, 0.0);
        }
        uint32_t key[V], none[1];
#pragma unroll
        for (int j = 0; j < V; ++j) key[j] = in_kept(groups, j) ? order32(a.bias ? s[j] : v[j]) : 0;
        int taken;
        Closeness close;
        if (a.bias) c = choose<L, V, kScoreKeys>(key, none, a.k, lane, tol, taken, close);
        else c = choose<L, V, kLogitKeys>(key, none, a.k, lane, tol, taken, close);
        if (close == kClose) {
            sum_in_64();
            const bool is = c.expert >= 0;
            const float l = is ? static_cast<float>(static_cast<const T*>(a.logits)[row * a.E + c.expert]) : 0.0f;
            const uint64_t key64 = is ? order64(score64(l) + a.bias[c.expert]) : 0;
            c.expert = by_rank<L>(c.expert, key64, taken, lane);
            if (lane >= a.k) c.expert = -1;
        } else if (close == kLost) {
            double s64[V];
            all_in_64(s64);
            uint32_t low[V];
#pragma unroll
            for (int j = 0; j < V; ++j) {
                const uint64_t o = in_kept(groups, j) ? order64(s64[j]) : 0;
                key[j] = static_cast<uint32_t>(o >> 32);
                low[j] = static_cast<uint32_t>(o);
            }
            c = choose<L, V, kWideKeys>(key, low, a.k, lane, 0.0f, taken, close);
        } else if (lane >= a.k) {
            c.expert = -1;
        }
        if (c.expert >= 0) c.logit = static_cast<float>(static_cast<const T*>(a.logits)[row * a.E + c.expert]);
    } else {
        uint32_t key[V], none[1];
#pragma unroll
        for (int j = 0; j < V; ++j) key[j] = v[j] == -kInf ? 0 : order32(v[j]);
        int taken;
        Closeness close;
        c = choose<L, V, kLogitKeys>(key, none, a.k, lane, 0.0f, taken, close);
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
// (16384, 256) bf16, 8 of 256, not renormalised: 7.6 us for 18 MB, vector arithmetic
// in 0.64 of the busy cycles (a precise exponential for every logit; 11.7 us where
// each lane compared each choice with each of its experts, and with a division); of
// sigmoids 9.5, two for every logit; renormalised 5.0 and 5.1.
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
    load_row<DT, V>(a.logits, row, a.E, first, v);
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

    // The choices' parts to the lanes that have their experts, through LDS; those of
    // an expert that a token has twice are added up by both.
    __shared__ __align__(16) float parts[kThreads * V];
    float* const own_parts = parts + threadIdx.x / L * (L * V);
    float sum[V];
#pragma unroll
    for (int j = 0; j < V; ++j) own_parts[first + j] = 0.0f;
    float mine_sum = 0.0f;
    each_choice<L>(a.k, [&](auto i) {
        const int e = static_cast<int>(from_lane<L, i>(static_cast<uint32_t>(mine)));
        const float di = __builtin_bit_cast(float, from_lane<L, i>(__builtin_bit_cast(uint32_t, d)));
        mine_sum += e == mine ? di : 0.0f;
    });
    if constexpr (L == 64)
        for (int i = kRowLanes; i < a.k; ++i) {
            const int e = __shfl(mine, i);
            const float di = __shfl(d, i);
            mine_sum += e == mine ? di : 0.0f;
        }
    wave_fence();
    if (mine >= 0) own_parts[mine] = mine_sum;
    wave_fence();
#pragma unroll
    for (int j = 0; j < V; ++j) sum[j] = own_parts[first + j];
    const float scale = 1.0f / total;
#pragma unroll
    for (int j = 0; j < V; ++j) {
        if (a.renormalise) v[j] = sum[j];
        else if (a.sigmoid) v[j] = sum[j] == 0.0f ? 0.0f : sum[j] * sigmoid(v[j]) * sigmoid(-v[j]);
        else v[j] = v[j] == 0.0f ? 0.0f : v[j] * scale * (sum[j] - dot);
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

// Rows in 16 lanes where they and the choices fit: four rows share every instruction
// of the maxima, which counts where there are rows for all SIMDs.  (Rows in 16 and in 64
// lanes, bf16, us in a graph, forward and backward, for 1024 / 2048 / 4096 / 16384 rows.
// 2 of 16: 2.1 / 2.1 / 2.1 / 2.6 and 2.3 / 2.4 / 3.0 / 6.2; 2.5 / 2.5 / 2.6 / 3.0 and 2.6 /
// 2.8 / 3.2 / 6.0.  8 of 64: 3.3 / 3.4 / 3.4 / 5.1 and 3.1 / 3.5 / 4.6 / 11.5; 3.1 / 3.1 / 3.1
// / 4.1 and 2.8 / 2.9 / 3.4 / 6.8.  8 of 256: 5.8 / 5.9 / 6.0 / 10.2 and 3.9 / 4.4 / 6.0 /
// 16.2; 4.9 / 5.0 / 5.2 / 7.6 and 3.3 / 3.4 / 4.4 / 9.6.  One limit for all: between it and
// 4096 rows of 256 the other side would take up to 1.9 us less, 2.4 with groups.)
bool narrow_rows(int64_t M, int E, int k, int groups) { return E <= 256 && k <= 16 && groups <= 16 && M > 1024; }

template <int DT, int L, int V>
void launch_fwd_as(const RouteArgs& a, hipStream_t st) {
    const int rows = kThreads / L;
    const dim3 grid(static_cast<uint32_t>((a.M + rows - 1) / rows));
    const bool grouped = a.kept < a.groups;
    const size_t lds = grouped ? static_cast<size_t>(rows) * (V * L + a.groups) * sizeof(double) : 0;
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
