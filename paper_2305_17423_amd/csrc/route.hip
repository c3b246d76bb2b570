// Routing of tokens to experts: keys (a score by softmax or sigmoid, and a bias), groups, the k largest, their weights, and the pairs (token, place) in the
// experts' order.
//
// Reading the logits once bounds it for many tokens, a launch for few.  Sixteen lanes (64 for more than 256 experts, sixteen places or sixteen groups) share a token, each with neighbouring experts in
// registers; k rounds take the largest key, the lowest expert among equal ones.  Which expert is chosen is a whole number, so keys are compared as they are in 64 bits: in float first, and
// again in 64 bits where two keys are closer than float's error explains (65536 tokens of 256 experts, 8 of 4 of 8 groups: 87 us; all in 64 bits 249).  Without a
// bias, and groups by their largest key, the logits are the float keys, and two of them close where their scores may be one number of 64 bits.
// The order of the pairs is that of a counting sort: a wave gives each of its pairs its rank among those of the same expert (ballots of the expert's bits find the lanes that
// share it), the workgroup adds up its waves, and further launches add the workgroups, all in order, so that nothing depends on the run.  Few tokens are one workgroup and one launch.
#include <algorithm>
#include <cmath>
#include "common.h"
#include "route_choice.h"

namespace fise {

struct RouteArgs {
    const void* logits; long long stride; int f32;
    int T, E, k, sigmoid, groups, top_groups, group_top, renorm, lists;
    const float* bias; float scale;
    int* ids; float* weights; int* offsets; int* slots;
    unsigned* pairs; int* hist; int* total;
    int wave_tokens, chunks, bits, wide;
};

// over the L neighbouring lanes of a token; all of them get the result
template <int L> __device__ __forceinline__ int route_max(int v) {
    // rotations within sixteen lanes
    v = max(v, __builtin_amdgcn_update_dpp(0, v, 0x128, 0xf, 0xf, false));
    v = max(v, __builtin_amdgcn_update_dpp(0, v, 0x124, 0xf, 0xf, false));
    v = max(v, __builtin_amdgcn_update_dpp(0, v, 0x122, 0xf, 0xf, false));
    v = max(v, __builtin_amdgcn_update_dpp(0, v, 0x121, 0xf, 0xf, false));
    if constexpr (L == 64) { v = max(v, __shfl_xor(v, 16)); v = max(v, __shfl_xor(v, 32)); }
    return v;
}
template <int L> __device__ __forceinline__ double route_sum(double v) {
#pragma unroll
    for (int o = 1; o < L; o <<= 1) v += __shfl_xor(v, o);
    return v;
}
// the lowest of a token's lanes for which it holds, L if there is none
template <int L> __device__ __forceinline__ int route_lowest(bool holds, int part) {
    const unsigned long long all = __ballot(holds);
    if constexpr (L == 64) return all ? __ffsll(all) - 1 : 64;
    const unsigned mine = (unsigned)(all >> (part * L)) & ((1u << L) - 1);
    return mine ? __ffs((int)mine) - 1 : L;
}
__device__ __forceinline__ float route_logit(const RouteArgs& a, long long t, int e) {
    return a.f32 ? reinterpret_cast<const float*>(a.logits)[t * a.stride + e] : bf2f(reinterpret_cast<const bf16_t*>(a.logits)[t * a.stride + e]);
}
// floats in the order of whole numbers (both zeros are one), and back
__device__ __forceinline__ int route_code(float v) { const int b = __float_as_int(v + 0.f); return b ^ ((b >> 31) & 0x7fffffff); }
__device__ __forceinline__ float route_float(int c) { return __int_as_float(c ^ ((c >> 31) & 0x7fffffff)); }
constexpr int ROUTE_NONE = (int)0x80000000;

// Doubles in the order of whole numbers, and back; the largest of a wave's, and the lowest lane that has it.  (By rotations within sixteen lanes and four scalar reads: shuffles through LDS,
// one behind the other, made a token that comes here take 10 us.)
__device__ __forceinline__ long long route_code64(double v) { const long long b = __double_as_longlong(v + 0.0); return b ^ ((b >> 63) & 0x7fffffffffffffffLL); }
__device__ __forceinline__ double route_double(long long c) { return __longlong_as_double(c ^ ((c >> 63) & 0x7fffffffffffffffLL)); }
constexpr long long ROUTE_NONE64 = (long long)0x8000000000000000ULL;
__device__ __forceinline__ int route_wave_max(int v) {
    v = route_max<16>(v);
    return max(max(__builtin_amdgcn_readlane(v, 0), __builtin_amdgcn_readlane(v, 16)), max(__builtin_amdgcn_readlane(v, 32), __builtin_amdgcn_readlane(v, 48)));
}
__device__ __forceinline__ long long route_first64(long long key, int& lane) {
    const int high = (int)(key >> 32), low = (int)((unsigned)key ^ 0x80000000u), top = route_wave_max(high), then = route_wave_max(high == top ? low : (int)0x80000000);
    lane = __ffsll(__ballot(high == top && low == then)) - 1;
    return (long long)(((unsigned long long)(unsigned)top << 32) | ((unsigned)then ^ 0x80000000u));
}

// One token by a whole wave in 64 bits, as the definition says: lane j gets the expert of place j (-1: none).  `broken`: a key is not a number.
template <int V> __device__ __forceinline__ int route_exact(const RouteArgs& a, long long t, bool& broken) {
    const int lane = threadIdx.x & 63;
    float l[V], top = -INFINITY;
    double score[V], sum = 0.0;
    long long key[V];
#pragma unroll
    for (int i = 0; i < V; ++i) {
        const int e = lane * V + i;
        l[i] = e < a.E ? route_logit(a, t, e) : -INFINITY;
        top = fmaxf(top, l[i]);
        score[i] = (double)l[i];
    }
    top = route_float(route_wave_max(route_code(top)));
#pragma unroll
    for (int i = 0; i < V; ++i) {
        score[i] = l[i] == -INFINITY ? 0.0 : exp(a.sigmoid ? -score[i] : score[i] - (double)top);
        sum += score[i];
    }
    sum = a.sigmoid ? 1.0 : route_sum<64>(sum);
#pragma unroll
    for (int i = 0; i < V; ++i) {
        const int e = lane * V + i;
        score[i] = a.sigmoid ? 1.0 / (1.0 + score[i]) : score[i] / sum;
        if (a.bias && e < a.E) score[i] += (double)a.bias[e];
        broken = broken || (l[i] != -INFINITY && score[i] != score[i]);
    }
#pragma unroll
    for (int i = 0; i < V; ++i) key[i] = l[i] == -INFINITY || score[i] == -INFINITY ? ROUTE_NONE64 : route_code64(score[i]);
    if (a.groups > 1) {
        const int size = a.E / a.groups;
        long long mine = ROUTE_NONE64;                                 // of group `lane`
        for (int g = 0; g < a.groups; ++g) {
            long long m1 = ROUTE_NONE64;
            int at = -1, from;
#pragma unroll
            for (int i = 0; i < V; ++i) {
                const int e = lane * V + i;
                if (e >= g * size && e < (g + 1) * size && key[i] > m1) { m1 = key[i]; at = i; }
            }
            long long best = route_first64(m1, from);
            if (a.group_top > 1 && best != ROUTE_NONE64) {
                long long m2 = ROUTE_NONE64;
#pragma unroll
                for (int i = 0; i < V; ++i) {
                    const int e = lane * V + i;
                    if (e >= g * size && e < (g + 1) * size && key[i] > m2 && !(lane == from && i == at)) m2 = key[i];
                }
                const long long second = route_first64(m2, from);
                if (second != ROUTE_NONE64) best = route_code64(route_double(best) + route_double(second));
            }
            if (lane == g) mine = best;
        }
        unsigned long long kept = 0;
        for (int j = 0; j < a.top_groups; ++j) {
            int g;
            if (route_first64(mine, g) == ROUTE_NONE64) break;
            kept |= 1ull << g;
            if (lane == g) mine = ROUTE_NONE64;
        }
#pragma unroll
        for (int i = 0; i < V; ++i)
            if (!(kept >> (min(lane * V + i, a.E - 1) / size) & 1)) key[i] = ROUTE_NONE64;
    }
    int id = -1;
    for (int j = 0; j < a.k; ++j) {
        long long m = key[0];
        int at = 0, from;
#pragma unroll
        for (int i = 1; i < V; ++i)
            if (key[i] > m) { m = key[i]; at = i; }
        if (route_first64(m, from) == ROUTE_NONE64) break;
        const int e = from * V + __builtin_amdgcn_readlane(at, from);
        if (lane == j) id = e;
#pragma unroll
        for (int i = 0; i < V; ++i)
            if (lane == from && i == at) key[i] = ROUTE_NONE64;
    }
    return id;
}

// Steps of the network: key x and the one D behind it, for all x; then the shorter distances among sorted runs of P keys, and the longer runs.  (Templates, not loops: the compiler
// took the loops' indices for numbers of its run time and searched the keys for each.)
template <int V, int P, int D, int X> __device__ __forceinline__ void route_sort(int (&key)[V]) {
    if constexpr (X >= D % P && (X - D % P) / D % 2 == 0 && X / (2 * P) == (X + D) / (2 * P)) {
        const int high = max(key[X], key[X + D]), low = min(key[X], key[X + D]);
        key[X] = high;
        key[X + D] = low;
    }
    if constexpr (X + 1 < V - D) route_sort<V, P, D, X + 1>(key);
    else if constexpr (D > 1) route_sort<V, P, D / 2, 0>(key);
    else if constexpr (2 * P < V) route_sort<V, 2 * P, 2 * P, 0>(key);
}
// the first key goes, the others move up
template <int V, int X> __device__ __forceinline__ void route_shift(int (&key)[V], bool really) {
    key[X] = really ? (X + 1 < V ? key[X + 1 < V ? X + 1 : X] : ROUTE_NONE) : key[X];
    if constexpr (X + 1 < V) route_shift<V, X + 1>(key, really);
}

// The same by L lanes with keys in float, their order as whole numbers of which the last four bits are the place among a lane's V (the first has the largest).  `close`: two keys of which the
// order matters are no further apart than their errors and those four bits explain, so the token needs route_exact.  ids[j]: the expert of place j, from the lane that has it.
template <int L, int V>
__device__ __forceinline__ void route_fast(const RouteArgs& a, const float* l, float top, const float* bias, bool odd_bias, int sub, int part, volatile int* ids, bool& broken, bool& close) {
    const bool direct = !a.bias && (a.groups == 1 || a.group_top == 1);      // the logits are the keys: larger ones have larger scores, or (close) the same in 64 bits
    float off = 0.f, large = 0.f;
    int key[V];
    if (direct) {
#pragma unroll
        for (int i = 0; i < V; ++i) key[i] = route_code(l[i]);
    } else {
        float v[V];
        if (a.sigmoid) {
#pragma unroll
            for (int i = 0; i < V; ++i) v[i] = __builtin_amdgcn_rcpf(1.f + __expf(-l[i]));
            off = 0x1p-21f;                                            // s (1 - s) (|l| 2^-23 + 2^-21) of the exponential, which is below 2^-22.3, and three roundings of s
        } else {
            double sum = 0.0;
#pragma unroll
            for (int i = 0; i < V; ++i) { v[i] = l[i] == -INFINITY ? 0.f : __expf(l[i] - top); sum += (double)v[i]; }
            const float one = 1.f / (float)route_sum<L>(sum);          // (a token without experts: not used)
#pragma unroll
            for (int i = 0; i < V; ++i) v[i] *= one;
            off = one * 0x1p-19f;                                      // p (|x| 2^-23 + 2^-21) with p = e^-|x|, of the exponential, which is below 2^-20.8; as much of the sum; two roundings
        }
#pragma unroll
        for (int i = 0; i < V; ++i) {
            if (a.bias) v[i] += bias[i];
            large = fmaxf(large, fabsf(v[i]));
            key[i] = l[i] == -INFINITY ? ROUTE_NONE : route_code(v[i]);
        }
        if (odd_bias)
#pragma unroll
            for (int i = 0; i < V; ++i) broken = broken || (l[i] != -INFINITY && v[i] != v[i]);
    }
#pragma unroll
    for (int i = 0; i < V; ++i) key[i] = key[i] <= route_code(-INFINITY) ? ROUTE_NONE : (key[i] & ~15) | (15 - i);
    // Keys as whole numbers without their places, which takes less than 2^-19 off them (bf16 logits: nothing).  Two are in order where they are further apart than that, the errors of both
    // scores and the roundings of their biases.  (For sums of two keys `large` is twice the largest key there is, and their errors are those of two.)
    auto near = [&](int high, int low, float large, float errors) {
        if (low == ROUTE_NONE) return false;
        const float h = route_float(high), w = route_float(low);
        // Logits that are no further apart than this may have one score in 64 bits.  A score moves by (1 - s) dx of itself, with 1 - s >= 1 / (1 + e^x); under softmax by dx, where x - top is a
        // difference in 64 bits.  2^-50 of that is behind every rounding of the score, and a difference of float keys without their places at most 32 times that of the logits.  Below
        // -700 the exponential leaves the normal numbers.
        if (direct) return high == low ? a.f32 != 0 : a.sigmoid ? !(h > -700.f && h - w > 0x1p-45f * (1.f + __expf(h))) : !(h - top > -690.f && h - w > 0x1p-45f * (1.f + (top - h)));
        return !(h - w > errors * off + (0x1p-19f + 0x1p-21f) * fmaxf(large, fmaxf(fabsf(h), fabsf(w))));
    };
    close = false;
    if (a.groups > 1) {                                                // groups of whole lanes, a power of two of them (others take route_exact)
        const int lanes = a.E / a.groups / V;
        int m1 = ROUTE_NONE, m2 = ROUTE_NONE;
#pragma unroll
        for (int i = 0; i < V; ++i) { m2 = max(m2, min(m1, key[i])); m1 = max(m1, key[i]); }
        for (int o = 1; o < lanes; o <<= 1) {
            const int n1 = __shfl_xor(m1, o), n2 = __shfl_xor(m2, o);
            m2 = max(min(m1, n1), max(m2, n2));
            m1 = max(m1, n1);
        }
        m1 &= ~15; m2 &= ~15;
        if (a.group_top > 1 && m2 != ROUTE_NONE) m1 = route_code(route_float(m1) + route_float(m2));
        large = 2.f * __int_as_float(route_max<L>(__float_as_int(large)));
        int mine = sub % lanes == 0 && sub / lanes < a.groups ? m1 : ROUTE_NONE;      // in the group's first lane
        unsigned kept = 0;
        int last = ROUTE_NONE;
        for (int j = 0; j <= a.top_groups && j < a.groups; ++j) {
            const int best = route_max<L>(mine);
            if (j == a.top_groups) {
                close = near(last, best, 2.f * large, 4.f);
                if (direct && __any(best == last)) {                   // equal logits, and a lower one behind them with their score
                    const int lower = route_max<L>(mine < best ? mine : ROUTE_NONE);
                    close = close || (best == last && near(best, lower, 0.f, 0.f));
                }
                break;
            }
            const int from = route_lowest<L>(mine == best, part);
            if (best != ROUTE_NONE && sub / lanes == from / lanes) kept = 1;
            if (sub == from) mine = ROUTE_NONE;
            last = best;
        }
#pragma unroll
        for (int i = 0; i < V; ++i) key[i] = kept ? key[i] : ROUTE_NONE;
    }
    // each lane's keys in descending order (a network of compare-and-exchange steps that merges sorted halves); then the largest of the lanes' first ones, k times
    route_sort<V, 1, 1, 0>(key);
    int taken = ROUTE_NONE, after = ROUTE_NONE;                        // the key of place `sub`, and the first that is not taken
    for (int j = 0; j <= a.k; ++j) {
        const int mine = key[0] & ~15, best = route_max<L>(mine);
        if (j == a.k) after = best;
        if (j == a.k || !__any(best != ROUTE_NONE)) break;
        if (sub == j) taken = best;
        const bool won = sub == route_lowest<L>(mine == best, part) && best != ROUTE_NONE;
        if (won) ids[j] = sub * V + 15 - (key[0] & 15);
        route_shift<V, 0>(key, won);
    }
    // each place against the next
    int next = __shfl_down(taken, 1, L);
    if (sub == a.k - 1) next = after;
    if (sub < a.k && near(taken, next, 0.f, 2.f)) close = true;
    if (direct) {                                                      // the last place's logit once more among those left over, and a lower one behind it with its score
        const bool again = sub == a.k - 1 && taken == after && after != ROUTE_NONE;
        if (__any(again)) {
            int lower = ROUTE_NONE;
#pragma unroll
            for (int i = 0; i < V; ++i) { const int v = key[i] & ~15; lower = max(lower, v < after ? v : ROUTE_NONE); }
            lower = route_max<L>(lower);
            if (again && near(after, lower, 0.f, 0.f)) close = true;
        }
    }
}

template <int L, int V, bool SINGLE>
__global__ __launch_bounds__(SINGLE ? 1024 : 256) void route_kernel(RouteArgs a) {
    extern __shared__ int route_lds[];                                 // [wave][E] counts, [wave][64] ids, then (single) the pairs
    constexpr int WAVES = SINGLE ? ROUTE_SINGLE_WAVES : ROUTE_WAVES, AT_ONCE = 64 / L;
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, sub = lane % L, part = lane / L;
    // lanes read what others of their wave wrote: LDS serves a wave in order, and the compiler keeps that order
    volatile int* const count = route_lds + wave * a.E;
    volatile int* const ids = route_lds + WAVES * a.E + wave * 64 + part * L;
    unsigned* const held = reinterpret_cast<unsigned*>(route_lds + WAVES * (a.E + 64));
    const long long first = ((long long)blockIdx.x * WAVES + wave) * a.wave_tokens;
    if (a.lists)
        for (int e = lane; e < a.E; e += 64) count[e] = 0;
    const int size = a.E / a.groups, lanes = size / V;
    const bool odd_groups = a.groups > 1 && (size % V != 0 || (lanes & (lanes - 1)) != 0);
    float bias[V];
    bool odd_bias = false;                                             // one that is not a number
#pragma unroll
    for (int i = 0; i < V; ++i) { bias[i] = a.bias && sub * V + i < a.E ? a.bias[sub * V + i] : 0.f; odd_bias = odd_bias || bias[i] != bias[i]; }
    odd_bias = __any(odd_bias);
    float ahead[V];                                                    // the next tokens' logits are on their way while these are worked on
    auto fetch = [&](long long t) {
#pragma unroll
        for (int i0 = 0; i0 < V; i0 += 4) {
            const int e = sub * V + i0;
            if (a.wide && t < a.T && e + 4 <= a.E) {
                if (a.f32) {
                    const f32x4_t v = *reinterpret_cast<const f32x4_t*>(reinterpret_cast<const float*>(a.logits) + t * a.stride + e);
#pragma unroll
                    for (int i = 0; i < 4; ++i) ahead[i0 + i] = v[i];
                } else {
                    const u32x2_t v = *reinterpret_cast<const u32x2_t*>(reinterpret_cast<const bf16_t*>(a.logits) + t * a.stride + e);
                    ahead[i0] = lo16(v[0]); ahead[i0 + 1] = hi16(v[0]); ahead[i0 + 2] = lo16(v[1]); ahead[i0 + 3] = hi16(v[1]);
                }
            } else
#pragma unroll
                for (int i = 0; i < 4; ++i) ahead[i0 + i] = t < a.T && e + i < a.E ? route_logit(a, t, e + i) : -INFINITY;
        }
    };
    fetch(first + part);
    for (int r0 = 0; r0 < a.wave_tokens; r0 += AT_ONCE) {
        const long long t = first + r0 + part;
        const bool there = t < a.T;
        if (!__any(there)) break;
        float l[V], top = -INFINITY;
        bool bad = false;
#pragma unroll
        for (int i = 0; i < V; ++i) l[i] = ahead[i];
        if (r0 + AT_ONCE < a.wave_tokens) fetch(t + AT_ONCE);
#pragma unroll
        for (int i = 0; i < V; ++i) {
            bad = bad || l[i] != l[i] || (!a.sigmoid && l[i] == INFINITY);
            top = fmaxf(top, l[i]);
        }
        top = route_float(route_max<L>(route_code(top)));
        bool close = odd_groups;
        ids[sub] = -1;
        if (!odd_groups) route_fast<L, V>(a, l, top, bias, odd_bias, sub, part, ids, bad, close);
        const unsigned long long mask = L == 64 ? ~0ull : ((1ull << L) - 1) << (part * L);
        bad = (__ballot(bad) & mask) != 0;
        int id = ids[sub];
        for (unsigned long long again = __ballot(close && there && !bad); again;) {
            const int p = (__ffsll(again) - 1) / L;
            again &= L == 64 ? 0ull : ~(((1ull << L) - 1) << (p * L));
            bool broken = false;
            const int exact = route_exact<L * V / 64>(a, first + r0 + p, broken);
            broken = __any(broken);
            const int moved = __shfl(exact, sub);
            if (part == p) { id = moved; bad = bad || broken; }
        }
        if (bad) id = -1;
        // the chosen ones' scores in 64 bits, one a lane; a softmax' sum where it does not drop out
        const bool out = there && sub < a.k;
        const double logit = out && id >= 0 ? (double)route_logit(a, t, id) : 0.0;
        double w = 0.0;
        const double p = exp(a.sigmoid ? -logit : logit - (double)top);
        if (out && id >= 0) w = a.sigmoid ? 1.0 / (1.0 + p) : p;
        if (a.renorm || !a.sigmoid) {
            double sum = w;
            if (!a.renorm) {
                // all scores' sum in 64 bits too, the logits read once more: an expert at a time needs no registers for the others (65536 tokens of 256 experts 91 us, 64 with the chosen ones' sum)
                sum = 0.0;
#pragma unroll 2
                for (int e = there ? sub : a.E; e < a.E; e += L) {
                    const float x = route_logit(a, t, e);
                    sum += x == -INFINITY ? 0.0 : exp((double)x - (double)top);
                }
            }
            sum = route_sum<L>(sum);
            w = sum > 0.0 ? w / sum : 0.0;
        }
        if (out) {
            a.ids[t * a.k + sub] = id;
            a.weights[t * a.k + sub] = bad ? NAN : (float)(w * (double)a.scale);
        }
        if (!a.lists) continue;
        // rank among the pairs of this wave with the same expert: pairs ascend with the lanes
        unsigned long long same = __ballot(out && id >= 0);
        for (int b = 0; b < a.bits; ++b) {
            const unsigned long long set = __ballot(id >> b & 1);
            same &= (id >> b & 1) ? set : ~set;
        }
        const bool counted = out && id >= 0;
        const unsigned long long before = same & ((1ull << lane) - 1);
        const int rank = counted ? count[id] + __popcll(before) : 0;
        if (counted && before == 0) count[id] += __popcll(same);       // (LDS is read and written in order within a wave)
        if (out) {
            const unsigned packed = counted ? (unsigned)id << 16 | (unsigned)rank : 0xffffffffu;
            if (SINGLE) held[t * a.k + sub] = packed;
            else a.pairs[t * a.k + sub] = packed;
        }
    }
    if (!a.lists) return;
    __syncthreads();
    // counts become starts: of a wave within the workgroup, and (single) of an expert among all
    if constexpr (SINGLE) {
        int* const sums = reinterpret_cast<int*>(held + a.T * a.k);    // of the 16 waves
        int mine = 0;
        if (tid < a.E)
            for (int w = 0; w < WAVES; ++w) { const int n = route_lds[w * a.E + tid]; route_lds[w * a.E + tid] = mine; mine += n; }
        int up = mine;
#pragma unroll
        for (int o = 1; o < 64; o <<= 1) { const int n = __shfl_up(up, o); if (lane >= o) up += n; }
        if (lane == 63) sums[wave] = up;
        __syncthreads();
        int base = up - mine;
        for (int w = 0; w < wave; ++w) base += sums[w];
        if (tid < a.E) {
            for (int w = 0; w < WAVES; ++w) route_lds[w * a.E + tid] += base;
            a.offsets[tid] = base;
            if (tid == a.E - 1) a.offsets[a.E] = base + mine;
        }
        __syncthreads();
        for (int p = tid; p < a.T * a.k; p += 1024) {
            const unsigned v = held[p];
            if (v == 0xffffffffu) continue;
            const int w = p / a.k / a.wave_tokens;
            a.slots[route_lds[w * a.E + (int)(v >> 16)] + (int)(v & 0xffffu)] = p;
        }
    } else {
        for (int e = tid; e < a.E; e += 256) {
            int sum = 0;
            for (int w = 0; w < WAVES; ++w) { const int n = route_lds[w * a.E + e]; route_lds[w * a.E + e] = sum; sum += n; }
            a.hist[(long long)e * a.chunks + blockIdx.x] = sum;
        }
        __syncthreads();
        const long long t0 = (long long)blockIdx.x * WAVES * a.wave_tokens, p0 = t0 * a.k;
        const int n = (int)min((long long)WAVES * a.wave_tokens, a.T - t0) * a.k;
        for (int i = tid; i < n; i += 256) {                           // (what this workgroup wrote)
            const unsigned v = a.pairs[p0 + i];
            if (v != 0xffffffffu) a.pairs[p0 + i] = v + (unsigned)route_lds[(i / a.k / a.wave_tokens) * a.E + (int)(v >> 16)];
        }
    }
}

// Counts of an expert in all chunks become starts among its pairs: a workgroup an expert, a lane neighbouring chunks.
__global__ __launch_bounds__(256) void route_scan_kernel(int* hist, int* total, int chunks) {
    __shared__ int sums[4];
    int* const h = hist + (long long)blockIdx.x * chunks;
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    int before = 0;
    for (int c0 = 0; c0 < chunks; c0 += 2048) {
        int n[8], mine = 0;
#pragma unroll
        for (int i = 0; i < 8; ++i) { const int c = c0 + tid * 8 + i; n[i] = c < chunks ? h[c] : 0; mine += n[i]; }
        int up = mine;
#pragma unroll
        for (int o = 1; o < 64; o <<= 1) { const int m = __shfl_up(up, o); if (lane >= o) up += m; }
        if (lane == 63) sums[wave] = up;
        __syncthreads();
        int at = before + up - mine;
        for (int w = 0; w < 4; ++w) { if (w < wave) at += sums[w]; before += sums[w]; }
#pragma unroll
        for (int i = 0; i < 8; ++i) { const int c = c0 + tid * 8 + i; if (c < chunks) h[c] = at; at += n[i]; }
        __syncthreads();
    }
    if (tid == 0) total[blockIdx.x] = before;
}

__global__ __launch_bounds__(256) void route_place_kernel(RouteArgs a) {
    __shared__ int base[ROUTE_MAX_EXPERTS];
    __shared__ int sums[4];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    int v[4], mine = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) { const int e = tid * 4 + i; v[i] = e < a.E ? a.total[e] : 0; mine += v[i]; }
    int up = mine;
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) { const int n = __shfl_up(up, o); if (lane >= o) up += n; }
    if (lane == 63) sums[wave] = up;
    __syncthreads();
    int at = up - mine;
    for (int w = 0; w < wave; ++w) at += sums[w];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int e = tid * 4 + i;
        if (e < a.E) {
            base[e] = at;
            if (blockIdx.x == 0) { a.offsets[e] = at; if (e == a.E - 1) a.offsets[a.E] = at + v[i]; }
        }
        at += v[i];
    }
    __syncthreads();
    const int per_chunk = ROUTE_WAVES * a.wave_tokens * a.k;
    const long long pairs = (long long)a.T * a.k, p1 = min(pairs, (long long)(blockIdx.x + 1) * 1024);
    for (long long p = (long long)blockIdx.x * 1024 + tid; p < p1; p += 256) {
        const unsigned w = a.pairs[p];
        if (w == 0xffffffffu) continue;
        const int e = (int)(w >> 16);
        a.slots[base[e] + a.hist[(long long)e * a.chunks + p / per_chunk] + (int)(w & 0xffffu)] = (int)p;
    }
}

template <int L, int V> static int launch_route(const RouteArgs& a, const RouteChoice& c, hipStream_t st) {
    const int lds = (c.waves * (a.E + 64) + (c.single ? a.T * a.k + 16 : 0)) * 4;
    if (c.single) {
        static const hipError_t attr = hipFuncSetAttribute(reinterpret_cast<const void*>(&route_kernel<L, V, true>), hipFuncAttributeMaxDynamicSharedMemorySize,
                                                           (ROUTE_SINGLE_WAVES * (L * V + 64) + ROUTE_SINGLE_PAIRS + 16) * 4);
        if (attr != hipSuccess) return fail(FISE_ERR_HIP, "fise_route_experts: cannot raise the dynamic LDS limit");
        hipLaunchKernelGGL((route_kernel<L, V, true>), dim3(1), dim3(1024), (size_t)lds, st, a);
    } else hipLaunchKernelGGL((route_kernel<L, V, false>), dim3((unsigned)c.chunks), dim3(256), (size_t)lds, st, a);
    FISE_CHECK_LAUNCH("fise_route_experts");
    return FISE_OK;
}

static int route_check(const char* fn, const fise_route_args* g) {
    if (g->E < 1 || g->E > ROUTE_MAX_EXPERTS || g->k < 1 || g->k > g->E || g->k > ROUTE_MAX_K || g->T < 0 || (long long)g->T * g->k > 0x7fffffffLL)
        return fail(FISE_ERR_SHAPE, "%s: T=%d E=%d k=%d", fn, g->T, g->E, g->k);
    if (g->groups < 1 || g->groups > 64 || g->E % g->groups || g->top_groups < 1 || g->top_groups > g->groups || (g->groups > 1 && g->group_top != 1 && g->group_top != 2))
        return fail(FISE_ERR_SHAPE, "%s: %d groups of %d experts, %d of them, by %d", fn, g->groups, g->E, g->top_groups, g->group_top);
    return FISE_OK;
}

}  // namespace fise

using namespace fise;

extern "C" size_t fise_route_experts_workspace_bytes(const fise_route_args* g) {
    if (!g) { fail(FISE_ERR_NULL, "fise_route_experts: null pointer"); return 0; }
    if (route_check("fise_route_experts", g)) return 0;
    return (size_t)route_choose(g->T, g->E, g->k, g->groups, g->offsets || g->slots).bytes;
}

extern "C" int fise_route_experts(const fise_route_args* g, void* workspace, size_t workspace_bytes, void* stream) {
    const char* fn = "fise_route_experts";
    if (!g || !g->logits || !g->ids || !g->weights) return fail(FISE_ERR_NULL, "%s: null pointer", fn);
    if (!g->offsets != !g->slots) return fail(FISE_ERR_NULL, "%s: offsets and slots are given together", fn);
    if (g->dtype != FISE_F32 && g->dtype != FISE_BF16) return fail(FISE_ERR_DTYPE, "%s: dtype %d", fn, g->dtype);
    if (int e = route_check(fn, g)) return e;
    if (g->score != FISE_SCORE_SOFTMAX && g->score != FISE_SCORE_SIGMOID) return fail(FISE_ERR_SHAPE, "%s: score %d", fn, g->score);
    if (g->stride < g->E) return fail(FISE_ERR_SHAPE, "%s: rows of %d logits %lld apart", fn, g->E, (long long)g->stride);
    if ((uintptr_t)g->logits % (g->dtype == FISE_F32 ? 4 : 2) || ((uintptr_t)g->ids | (uintptr_t)g->weights | (uintptr_t)g->offsets | (uintptr_t)g->slots | (uintptr_t)g->bias) & 3)
        return fail(FISE_ERR_ALIGN, "%s: pointers must be aligned to their type", fn);
    const bool lists = g->offsets != nullptr;
    const RouteChoice c = route_choose(g->T, g->E, g->k, g->groups, lists);
    if (c.chunks >= 1 << 24) return fail(FISE_ERR_SHAPE, "%s: T=%d: more tokens than a launch holds", fn, g->T);
    if (c.bytes && (!workspace || workspace_bytes < (size_t)c.bytes)) return fail(FISE_ERR_CAPACITY, "%s: workspace of %zu bytes, %lld needed", fn, workspace ? workspace_bytes : 0, (long long)c.bytes);
    if (c.bytes && ((uintptr_t)workspace & 255)) return fail(FISE_ERR_ALIGN, "%s: workspace must be 256-byte aligned", fn);
    if (g->T == 0) return FISE_OK;
    RouteArgs a{};
    a.logits = g->logits; a.stride = g->stride; a.f32 = g->dtype == FISE_F32;
    a.T = g->T; a.E = g->E; a.k = g->k; a.sigmoid = g->score == FISE_SCORE_SIGMOID; a.groups = g->groups; a.top_groups = g->top_groups; a.group_top = g->group_top;
    a.renorm = g->renormalize != 0; a.lists = lists; a.bias = g->bias; a.scale = g->scale;
    a.ids = g->ids; a.weights = g->weights; a.offsets = g->offsets; a.slots = g->slots;
    a.pairs = (unsigned*)workspace; a.hist = (int*)((unsigned char*)workspace + c.hist_off); a.total = (int*)((unsigned char*)workspace + c.total_off);
    a.wave_tokens = c.wave_tokens; a.chunks = c.chunks;
    while ((1 << a.bits) < a.E) ++a.bits;
    a.wide = g->dtype == FISE_F32 ? aligned16(g->logits) && g->stride % 4 == 0 : (uintptr_t)g->logits % 8 == 0 && g->stride % 4 == 0;
    const hipStream_t st = as_stream(stream);
    if (int e = c.lanes == 64 ? launch_route<64, 16>(a, c, st) : c.values == 4 ? launch_route<16, 4>(a, c, st) : launch_route<16, 16>(a, c, st)) return e;
    if (!lists || c.single) return FISE_OK;
    hipLaunchKernelGGL(route_scan_kernel, dim3((unsigned)a.E), dim3(256), 0, st, a.hist, a.total, a.chunks);
    FISE_CHECK_LAUNCH(fn);
    hipLaunchKernelGGL(route_place_kernel, dim3((unsigned)(((long long)a.T * a.k + 1023) / 1024)), dim3(256), 0, st, a);
    FISE_CHECK_LAUNCH(fn);
    return FISE_OK;
}
