// What stands around the experts' products of a mixture-of-experts layer, on the device:
//   bitcos_route_experts       a router's logits -> the experts of every token and their weights
//   bitcos_group_pairs_slots   the routed pairs sorted by expert (lists of any length), and every pair's place
//   bitcos_combine_pairs       the experts' outputs weighted and added, token by token
#include "bitcos.h"
#include "common.cuh"

#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include <algorithm>
#include <cfloat>
#include <climits>
#include <cmath>

using namespace bitcos_kernels;

namespace {

constexpr uint32_t kFull = 0xFFFFFFFFu;

// ---------------------------------------------------------------------------------------------
// Routing.  One warp per token; a lane holds V consecutive experts (expert = lane * V + v).
//
//   score  s = softmax(z) or 1 / (1 + exp(-z)),   choice c = s + bias
//
// Which expert is taken must not hang on how exp is rounded.  Without a bias (and without sums of scores for the groups)
// the order of the scores is the order of the logits, and that is what is compared.  Otherwise c is formed in 32 bits with
// a bound on its error; where two choices whose order matters lie closer than that allows, the warp does the
// token once more in 64 bits (route_exact).
//
// A warp to a token, so that a place is one reduction over the lanes' first keys and nothing passes through shared memory.  Bound by
// issue slots (1100 warp instructions a token of 256 experts) and, at the end, by the last tokens that need 64 bits (candidates 2 us, a whole
// token 10 us): 16384 tokens of 256 experts in 8 groups, bf16, 30 us, 18.7 without such tokens; of 128 experts without groups, fp32, 11 us; one token
// 2.5 us.  Two or eight warps a block are no faster.  Rows are read 16 bytes a lane only where there are 32 V experts exactly; else value by
// value, with lanes left over, and groups that are no whole runs of lanes are gone through one by one.  16384 tokens, softmax, bf16: 256 experts
// 13 us, 160 14, 384 (V = 16) 34; in groups, sigmoid and bias, 8 of 32 31 us, 8 of 20 51, 8 of 48 82 to 90.
// ---------------------------------------------------------------------------------------------
constexpr int kRouteWarps = 4;
constexpr int kMaxRouteGroups = 32;

struct RouteArgs {
    const void *logits;
    const float *bias;          // NULL: none
    int64_t row_stride;         // elements
    int32_t *expert;            // [tokens][top_k]
    int32_t *xrow;              // [tokens * top_k]
    float *weight;              // [tokens][top_k]
    float scale;
    int tokens, experts, top_k;
    int n_groups, top_groups, group_best, group_size;
    int softmax, renormalise, by_choice;   // by_choice: the order of c, else of the logits
    int vector;                 // rows may be read V values at a time
    int vector_bias;            // four biases at a time
    int segment;                // lanes per group where that is a whole power of two, else 0
};

__device__ __forceinline__ float to_float(float v) { return v; }
__device__ __forceinline__ float to_float(__nv_bfloat16 v) { return __bfloat162float(v); }
__device__ __forceinline__ float to_float(__half v) { return __half2float(v); }

// A value as an unsigned with the same order; 0 stands for "not to be taken" (below every finite value's).
__device__ __forceinline__ uint32_t ordered(float v) {
    const int32_t b = __float_as_int(v);
    return static_cast<uint32_t>(b ^ ((b >> 31) | INT32_MIN));
}
__device__ __forceinline__ float unordered(uint32_t o) { return __uint_as_float(o & 0x80000000u ? o & 0x7FFFFFFFu : ~o); }
__device__ __forceinline__ uint64_t ordered(double v) {
    const int64_t b = __double_as_longlong(v);
    return static_cast<uint64_t>(b ^ ((b >> 63) | INT64_MIN));
}
__device__ __forceinline__ double unordered(uint64_t o) {
    return __longlong_as_double(static_cast<long long>(o >> 63 ? o & ~(1ull << 63) : ~o));
}
__device__ __forceinline__ uint32_t warp_max(uint32_t v) { return __reduce_max_sync(kFull, v); }
__device__ __forceinline__ uint64_t warp_max(uint64_t v) {
    const uint32_t hi = static_cast<uint32_t>(v >> 32), top = __reduce_max_sync(kFull, hi);
    return (static_cast<uint64_t>(top) << 32) | __reduce_max_sync(kFull, hi == top ? static_cast<uint32_t>(v) : 0u);
}

template <typename T>
__device__ __forceinline__ T warp_sum(T v) {
#pragma unroll
    for (int d = 16; d; d >>= 1) v += __shfl_xor_sync(kFull, v, d);
    return v;
}

// A logit as it counts: +inf as the largest finite value, -inf and NaN as masked (-inf), -0 as 0.
__device__ __forceinline__ float clean(float z) {
    if (!(z > -INFINITY)) return -INFINITY;
    return fminf(z, FLT_MAX) + 0.0f;
}

// Lane g < n_groups holds the value of group g: which groups stay, one bit each.
template <typename F>
__device__ __forceinline__ uint32_t kept_groups(const RouteArgs &a, F mine, int lane) {
    int ahead = 0;
    for (int g = 0; g < a.n_groups; ++g) {
        const F other = __shfl_sync(kFull, mine, g);
        ahead += other > mine || (other == mine && g < lane);
    }
    return __ballot_sync(kFull, lane < a.n_groups && ahead < a.top_groups);
}

// Calls f(v, the group of expert lane * V + v).
template <int V, typename Do>
__device__ __forceinline__ void each_group(const RouteArgs &a, int lane, Do f) {
    int at = lane * V / a.group_size, in = lane * V - at * a.group_size;
#pragma unroll
    for (int v = 0; v < V; ++v) {
        f(v, at);
        if (++in == a.group_size) {
            in = 0;
            ++at;
        }
    }
}

// The two largest keys of a set, joined with the two largest of the lane d away.
template <typename K>
__device__ __forceinline__ void add_key(K &one, K &two, K k) {
    two = max(two, min(one, k));
    one = max(one, k);
}
template <typename K>
__device__ __forceinline__ void join_keys(K &one, K &two, int d) {
    const K other = __shfl_xor_sync(kFull, one, d), second = __shfl_xor_sync(kFull, two, d);
    two = max(min(one, other), max(two, second));
    one = max(one, other);
}
// (key 0 has no value; `low`: bits of a key that are not part of it.  In 32 bits a sum below the range counts as the lowest finite value: more
// than that of a group with nothing left, and never apart from its like, which leaves their order to 64 bits.  Above the range it
// is +inf, which is not apart from anything either.)
template <typename K>
__device__ __forceinline__ auto value_of(const RouteArgs &a, K one, K two, K low) {
    decltype(unordered(one)) none = -INFINITY, v = one ? unordered(one & ~low) : none;
    if (a.group_best == 2) {
        v = two ? v + unordered(two & ~low) : none;
        if constexpr (sizeof(K) == 4) v = two ? fmaxf(v, -FLT_MAX) : v;
    }
    return v;
}

// The value of every group (lane g: group g) from the experts' keys.
template <int V>
__device__ __forceinline__ float group_values(const RouteArgs &a, const uint32_t (&key)[V], uint32_t low, int lane) {
    float mine = -INFINITY;
    if (a.segment) {
        // every group is the whole runs of a power of two of lanes
        uint32_t one = 0, two = 0;
#pragma unroll
        for (int v = 0; v < V; ++v) add_key(one, two, key[v]);
        for (int d = 1; d < a.segment; d <<= 1) join_keys(one, two, d);
        mine = __shfl_sync(kFull, value_of(a, one, two, low), lane * a.segment & 31);
    } else {
        for (int g = 0; g < a.n_groups; ++g) {
            uint32_t one = 0, two = 0;
            each_group<V>(a, lane, [&](int v, int at) {
                if (at == g) add_key(one, two, key[v]);
            });
#pragma unroll
            for (int d = 16; d; d >>= 1) join_keys(one, two, d);
            if (lane == g) mine = value_of(a, one, two, low);
        }
    }
    return mine;
}

// The choice of an expert of logit z in 64 bits.  (Few tokens come here, one at a time, and each waits for every instruction to
// be fetched: what follows stays loops and calls; unrolled, a token took 15 us.)
__device__ __noinline__ double exact_choice(const RouteArgs &a, double z, int e, double top, double sum) {
    if (!a.by_choice) return z;
    const double p = exp(a.softmax ? z - top : -z);
    const float b = a.bias ? clean(__ldg(a.bias + e)) : 0.f;
    return (a.softmax ? p : 1.0) / (a.softmax ? sum : 1.0 + p) + static_cast<double>(b) + 0.0;
}

// The sum under the softmax in 64 bits.
template <int V, typename L>
__device__ __noinline__ double exact_sum(const RouteArgs &a, const L *row, int lane, double top) {
    double sum = 0.0;
#pragma unroll 1
    for (int v = 0; v < V; ++v) {
        const int e = lane * V + v;
        if (e < a.experts) sum += exp(static_cast<double>(clean(to_float(row[e]))) - top);
    }
    return warp_sum(sum);
}

// The places of n <= 32 candidates (lane j < n: expert e), among which all that will be taken are: lane j < top_k gets the expert of
// place j.
template <int V, typename L>
__device__ __noinline__ int order_candidates(const RouteArgs &a, const L *row, int lane, float top, int e, int n) {
    const double sum = a.by_choice && a.softmax ? exact_sum<V, L>(a, row, lane, top) : 1.0;
    const bool is = lane < n;
    const double c = is ? exact_choice(a, static_cast<double>(clean(to_float(row[e]))), e, top, sum) : 0.0;
    int place = 0;
#pragma unroll 1
    for (int i = 0; i < n; ++i) {
        const double other = __shfl_sync(kFull, c, i);
        const int index = __shfl_sync(kFull, e, i);
        place += other > c || (other == c && index < e);
    }
    int taken = -1;
#pragma unroll 1
    for (int i = 0; i < n; ++i) {
        const int at = __shfl_sync(kFull, place, i), index = __shfl_sync(kFull, e, i);
        if (lane == at && lane < a.top_k) taken = index;
    }
    return taken;
}

// The whole token in 64 bits: lane j < top_k gets the expert of place j (-1: none is left).
template <int V, typename L>
__device__ __noinline__ int route_exact(const RouteArgs &a, const L *row, int lane, float top) {
    uint64_t key[V];
    const double sum = a.by_choice && a.softmax ? exact_sum<V, L>(a, row, lane, top) : 1.0;
#pragma unroll 1
    for (int v = 0; v < V; ++v) {
        const int e = lane * V + v;
        const float z = e < a.experts ? clean(to_float(row[e])) : -INFINITY;
        const bool there = z > -INFINITY && (!a.by_choice || !a.bias || clean(__ldg(a.bias + e)) > -INFINITY);
        key[v] = there ? ordered(exact_choice(a, z, e, top, sum)) : 0;
    }
    if (a.n_groups > 1) {
        double mine = -INFINITY;
        if (a.segment) {
            uint64_t one = 0, two = 0;
#pragma unroll 1
            for (int v = 0; v < V; ++v) add_key(one, two, key[v]);
#pragma unroll 1
            for (int d = 1; d < a.segment; d <<= 1) join_keys(one, two, d);
            mine = __shfl_sync(kFull, value_of(a, one, two, uint64_t(0)), lane * a.segment & 31);
        } else {
#pragma unroll 1
            for (int g = 0; g < a.n_groups; ++g) {
                uint64_t one = 0, two = 0;
                const int from = max(g * a.group_size - lane * V, 0), to = min((g + 1) * a.group_size - lane * V, V);
#pragma unroll 1
                for (int v = from; v < to; ++v) add_key(one, two, key[v]);
#pragma unroll 1
                for (int d = 16; d; d >>= 1) join_keys(one, two, d);
                if (lane == g) mine = value_of(a, one, two, uint64_t(0));
            }
        }
        const uint32_t kept = kept_groups(a, mine, lane);
        int at = lane * V / a.group_size, in = lane * V - at * a.group_size;
#pragma unroll 1
        for (int v = 0; v < V; ++v) {
            if (at >= a.n_groups || !((kept >> at) & 1u)) key[v] = 0;
            if (++in == a.group_size) {
                in = 0;
                ++at;
            }
        }
    }
    int taken = -1;
    bool look = true;                        // this lane's best is to be found (anew)
    uint64_t best = 0;
    int at = 0;
#pragma unroll 1
    for (int j = 0; j < a.top_k; ++j) {
        if (look) {
            best = 0;
#pragma unroll 1
            for (int v = 0; v < V; ++v)
                if (key[v] > best) {
                    best = key[v];
                    at = v;
                }
        }
        const uint64_t all = warp_max(best);
        if (all == 0) break;
        const int winner = __ffs(__ballot_sync(kFull, best == all)) - 1;      // (lowest lane = lowest expert)
        const int e = __shfl_sync(kFull, lane * V + at, winner);
        look = lane == winner;
        if (look) key[at] = 0;
        if (lane == j) taken = e;
    }
    return taken;
}

// Sorts the keys of a lane, largest first (Batcher's odd-even merge sort).
template <int V>
__device__ __forceinline__ void sort_keys(uint32_t (&key)[V]) {
#pragma unroll
    for (int p = 1; p < V; p *= 2)
#pragma unroll
        for (int k = p; k >= 1; k /= 2)
#pragma unroll
            for (int j = k % p; j + k < V; j += 2 * k)
#pragma unroll
                for (int i = 0; i < k; ++i)
                    if (i + j + k < V && (i + j) / (2 * p) == (i + j + k) / (2 * p)) {
                        const uint32_t hi = max(key[i + j], key[i + j + k]), lo = min(key[i + j], key[i + j + k]);
                        key[i + j] = hi;
                        key[i + j + k] = lo;
                    }
}

template <int V, typename L>
__global__ void __launch_bounds__(kRouteWarps * 32) route_kernel(const __grid_constant__ RouteArgs a) {
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    asm volatile("griddepcontrol.wait;" ::: "memory");
    const int lane = threadIdx.x & 31;
    const int64_t token = static_cast<int64_t>(blockIdx.x) * kRouteWarps + (threadIdx.x >> 5);
    if (token >= a.tokens) return;
    const L *row = static_cast<const L *>(a.logits) + token * a.row_stride;
    float z[V];
    if (a.vector) {
        constexpr int kBytes = V * sizeof(L) < 16 ? V * sizeof(L) : 16;
        constexpr int kPer = kBytes / sizeof(L);
#pragma unroll
        for (int i = 0; i < V / kPer; ++i) {
            alignas(16) L part[kPer];
            const char *src = reinterpret_cast<const char *>(row + lane * V + i * kPer);
            if constexpr (kBytes == 16) *reinterpret_cast<uint4 *>(part) = *reinterpret_cast<const uint4 *>(src);
            else if constexpr (kBytes == 8) *reinterpret_cast<uint2 *>(part) = *reinterpret_cast<const uint2 *>(src);
            else if constexpr (kBytes == 4) *reinterpret_cast<uint32_t *>(part) = *reinterpret_cast<const uint32_t *>(src);
            else *reinterpret_cast<uint16_t *>(part) = *reinterpret_cast<const uint16_t *>(src);
#pragma unroll
            for (int j = 0; j < kPer; ++j) z[i * kPer + j] = clean(to_float(part[j]));
        }
    } else {
#pragma unroll
        for (int v = 0; v < V; ++v) {
            const int e = lane * V + v;
            z[v] = e < a.experts ? clean(to_float(row[e])) : -INFINITY;
        }
    }
    float most = z[0];
#pragma unroll
    for (int v = 1; v < V; ++v) most = fmaxf(most, z[v]);
    const float top = unordered(warp_max(ordered(most)));      // (-inf: nothing is left)
    uint32_t key[V];
    float sum = 1.f;
    if (a.softmax) {
        sum = 0.f;
#pragma unroll
        for (int v = 0; v < V; ++v) {
            const float e = top > -INFINITY ? expf(z[v] - top) : 0.f;          // (a masked one: exp(-inf) = 0)
            key[v] = __float_as_uint(e);
            sum += e;
        }
        sum = warp_sum(sum);
    }
    const auto score = [&](float zz) { return a.softmax ? expf(zz - top) / sum : 1.0f / (1.0f + expf(-zz)); };

    // The low bits of a key say which of its lane's experts it is (V - 1 - v: of equal ones the first is the largest), so that
    // a lane's keys can be sorted with minima and maxima alone.  For 16-bit logits nothing is lost, the bits are not used; otherwise the
    // order is checked below, with what those bits are worth counted as an error.
    constexpr uint32_t kLow = V - 1;
    const auto keyed = [&](float v32, int v) { return (ordered(v32) & ~kLow) | (kLow - v); };
    const bool inexact = a.by_choice || sizeof(L) == 4;
    float unit = 1e-37f;           // no choice is further off than this (a logit: than rel of itself)
    const float rel = a.by_choice ? 0.f : V * 1.1f * 1.1920929e-7f;
    const auto apart = [&](float more, float less, float units) { return more - less > units * unit + rel * (fabsf(more) + fabsf(less)); };
    if (!a.by_choice) {
#pragma unroll
        for (int v = 0; v < V; ++v) {
            const bool there = z[v] > -INFINITY;
            key[v] = there ? keyed(z[v], v) : 0u;
        }
    } else {
        // Only the order hangs on these scores, so the fast exponential and quotient do (2 + 1.2 |z| and 2 units of 2^-23); the
        // weights of the taken ones are formed anew below.  Error of a score, in units of 2^-23 and of the largest score s_max
        // of the token: softmax, s (8 + d) at d = top - z with s = s_max exp(-d), so below 9, and the V + 5 additions of the sum, half a
        // unit each; sigmoid, s (6 + 1.2 |z|), which is largest at the top logit or near z = -1.28, so below 8 + 1.2 |top|.  Then half a
        // unit of |c| for the addition and V for the low bits of the key; scores under the normal range may have been rounded to nothing
        // (1e-37).  All a tenth larger.
        const float inv = 1.0f / sum;
        float bias[V], size = 0.f;
        if (!a.bias) {
#pragma unroll
            for (int v = 0; v < V; ++v) bias[v] = 0.f;
        } else if (V % 4 == 0 && a.vector_bias) {
#pragma unroll
            for (int v = 0; v < V; v += 4) {
                const float4 b = __ldg(reinterpret_cast<const float4 *>(a.bias + lane * V + v));
                bias[v] = b.x, bias[(v + 1) % V] = b.y, bias[(v + 2) % V] = b.z, bias[(v + 3) % V] = b.w;
            }
        } else {
#pragma unroll
            for (int v = 0; v < V; ++v) bias[v] = lane * V + v < a.experts ? __ldg(a.bias + lane * V + v) : 0.f;
        }
#pragma unroll
        for (int v = 0; v < V; ++v) {
            const float s = a.softmax ? __uint_as_float(key[v]) * inv : __fdividef(1.0f, 1.0f + __expf(-z[v]));
            const float c = fminf(s + bias[v], FLT_MAX);          // (fminf makes FLT_MAX of a NaN: the sum is asked)
            const bool there = z[v] > -INFINITY && s + bias[v] > -INFINITY;
            key[v] = there ? keyed(c, v) : 0u;
            if (there) size = fmaxf(size, fabsf(c));
        }
        const float s_max = a.softmax ? inv : 1.0f / (1.0f + expf(-top));
        unit += 1.1f * 1.1920929e-7f * (s_max * (a.softmax ? 12.f + 0.5f * V : 8.f + 1.2f * fminf(fabsf(top), 100.f)) +
                                        __uint_as_float(warp_max(__float_as_uint(size))) * (0.5f + V));
    }

    bool groups_near = false;
    if (a.n_groups > 1) {
        const float mine = group_values<V>(a, key, kLow, lane);
        const uint32_t kept = kept_groups(a, mine, lane);
        if (a.segment) {
            if (!((kept >> (lane / a.segment)) & 1u) || lane / a.segment >= a.n_groups) {
#pragma unroll
                for (int v = 0; v < V; ++v) key[v] = 0u;
            }
        } else {
            each_group<V>(a, lane, [&](int v, int at) {
                if (at >= a.n_groups || !((kept >> at) & 1u)) key[v] = 0u;
            });
        }
        if (inexact && a.top_groups < a.n_groups) {
            // the smallest value of a kept group, the largest of one that is not; a value: two choices and the rounding of their sum
            const bool keep = (kept >> lane) & 1u;
            const float low = unordered(~warp_max(keep ? ~ordered(mine) : 0u));
            const float high = unordered(warp_max(lane < a.n_groups && !keep ? ordered(mine) : ordered(-INFINITY)));
            groups_near = high > -INFINITY && !apart(low, high, 6.f);
        }
    }

    sort_keys<V>(key);
    int taken = -1;                // lane j: the expert of place j
    uint32_t taken_key = 0u;
    // the best of all that are left (0: none), which goes to place j if it is at least `least`
    const auto next = [&](int j, uint32_t least) {
        const uint32_t mine = key[0] & ~kLow, all = warp_max(mine);
        if (all == 0u || all < least) return false;
        const int winner = __ffs(__ballot_sync(kFull, mine == all)) - 1;      // (equal ones: the lowest lane, the lowest expert)
        const uint32_t won = __shfl_sync(kFull, key[0], winner);
        if (lane == winner) {
#pragma unroll
            for (int v = 0; v + 1 < V; ++v) key[v] = key[v + 1];
            key[V - 1] = 0u;
        }
        if (lane == j) {
            taken = winner * V + static_cast<int>(kLow - (won & kLow));
            taken_key = all;
        }
        return true;
    };
    int places = 0;                // how many were found
    while (places < a.top_k && next(places, 0u)) ++places;

    float zt = taken >= 0 ? clean(to_float(row[taken])) : -INFINITY;
    if (inexact) {
        // the taken ones in order, every one above the next by more than both may be off (or the same logit and bias, where
        // the lower index goes first), the last one above all that are left
        const float c = taken >= 0 ? unordered(taken_key) : 0.f;
        const float b = taken >= 0 && a.bias ? clean(__ldg(a.bias + taken)) : 0.f;
        const int e_next = __shfl_down_sync(kFull, taken, 1);
        const float c_next = __shfl_down_sync(kFull, c, 1), z_next = __shfl_down_sync(kFull, zt, 1), b_next = __shfl_down_sync(kFull, b, 1);
        bool close = lane + 1 < places && !apart(c, c_next, 2.f) && !(z_next == zt && b_next == b && taken < e_next);
        if (places == a.top_k) {
            const uint32_t left = warp_max(key[0] & ~kLow);
            close = close || (lane == places - 1 && left != 0u && !apart(c, unordered(left), 2.f));
        }
        const bool some = __any_sync(kFull, close);
        if (groups_near || some) {
            // the candidates: the taken ones and what is left within reach of the last
            int n = places;
            bool whole = groups_near;
            if (!whole && places == a.top_k) {
                const float last = __shfl_sync(kFull, c, places - 1);
                // (a value just under the border may be let in, none over it is left out)
                const uint32_t least = ordered(last - (2.1f * unit + 2.1f * rel * fabsf(last))) & ~kLow;
                while (n < 32 && next(n, least)) ++n;
                const uint32_t more = warp_max(key[0] & ~kLow);
                whole = n == 32 && more != 0u && more >= least;      // (more than a lane each)
            }
            taken = whole ? route_exact<V, L>(a, row, lane, top) : order_candidates<V, L>(a, row, lane, top, taken, n);
            zt = taken >= 0 ? clean(to_float(row[taken])) : -INFINITY;
        }
    }
    float s = taken >= 0 ? score(zt) : 0.f;
    if (a.renormalise) s = s / (warp_sum(s) + 1e-20f);
    if (lane < a.top_k) {
        const int64_t p = token * a.top_k + lane;
        a.expert[p] = taken;
        a.weight[p] = s * a.scale;
        a.xrow[p] = static_cast<int32_t>(token);
    }
}

template <int V, typename L>
int launch_route(const RouteArgs &a, cudaStream_t stream) {
    const unsigned blocks = static_cast<unsigned>((static_cast<int64_t>(a.tokens) + kRouteWarps - 1) / kRouteWarps);
    return launch_pdl(route_kernel<V, L>, dim3(blocks), kRouteWarps * 32, 0, stream, a);
}

template <typename L>
int launch_route_type(RouteArgs a, cudaStream_t stream) {
    int V = 1;
    while (V * 32 < a.experts) V *= 2;
    const size_t chunk = std::min<size_t>(16, V * sizeof(L));
    a.vector = a.experts == V * 32 && reinterpret_cast<uintptr_t>(a.logits) % chunk == 0 && a.row_stride * sizeof(L) % chunk == 0;
    a.vector_bias = a.experts == V * 32 && aligned16(a.bias);
    a.segment = 0;
    if (a.group_size % V == 0 && (a.group_size / V & (a.group_size / V - 1)) == 0) a.segment = a.group_size / V;
    switch (V) {
        case 1: return launch_route<1, L>(a, stream);
        case 2: return launch_route<2, L>(a, stream);
        case 4: return launch_route<4, L>(a, stream);
        case 8: return launch_route<8, L>(a, stream);
        case 16: return launch_route<16, L>(a, stream);
        default: return launch_route<32, L>(a, stream);
    }
}

// ---------------------------------------------------------------------------------------------
// Pairs sorted by expert, lists of any length: a stable counting sort.  The list is cut into one chunk per block, a
// chunk into one run per warp.  With several blocks a first kernel counts every chunk's pairs per expert; then each block
// knows what lies in front of its own (all experts before, the same expert's pairs in earlier chunks), counts its runs, and its
// warps place their runs 32 pairs at a time (match_any: the earlier lanes with the same expert).
// ---------------------------------------------------------------------------------------------
// What bounds it is the chain of passes (count, join, place), each a few dependent reads of memory and shared memory: 11.1 us for
// 262144 pairs of 128 experts, where reading and writing them once takes 0.6 us; 2.3 us for 128 pairs.  Recorded in a graph, with the
// threads that a call gets below:
//   pairs (experts)         1600 (64)  4096 (128)  8192 (128)  32768 (128)  262144 (128)
//   1024 pairs a chunk      6.2        9.2         8.9         10.1         12.8       (one block up to 4096 pairs)
//   256 pairs a chunk       4.9        4.9         5.2          7.8         11.1       (one block up to 512 pairs)
// Past 148 * 256 pairs the chunks grow instead, one block to a multiprocessor.
constexpr int kSortThreads = 1024;
constexpr int kSortWarps = kSortThreads / 32;
constexpr int kSortMaxBlocks = 148;
constexpr int64_t kSortOneBlock = 512;       // up to this many pairs one block does everything
constexpr int64_t kSortChunk = 256;          // above it, pairs per block while there are multiprocessors left

struct SortArgs {
    const int32_t *pair_expert;
    int32_t *group_expert, *group_begin, *xrow, *order, *slot, *n_groups;
    int32_t *counts;            // [blocks][experts], what count_kernel found
    int n_pairs, n_experts, top_k;
    int chunk;                  // pairs per block, a multiple of 32
};

inline int sort_blocks(int64_t n_pairs) {
    return n_pairs <= kSortOneBlock ? 1 : static_cast<int>(std::min<int64_t>(kSortMaxBlocks, (n_pairs + kSortChunk - 1) / kSortChunk));
}

template <typename T>
__device__ __forceinline__ T smaller(T a, T b) {
    return a < b ? a : b;
}

__global__ void __launch_bounds__(kSortThreads) count_kernel(const __grid_constant__ SortArgs a) {
    extern __shared__ int32_t count[];
    for (int e = threadIdx.x; e < a.n_experts; e += blockDim.x) count[e] = 0;
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    asm volatile("griddepcontrol.wait;" ::: "memory");
    __syncthreads();
    const int64_t from = static_cast<int64_t>(blockIdx.x) * a.chunk;
    const int64_t to = smaller<int64_t>(a.n_pairs, from + a.chunk);
    for (int64_t i = from + threadIdx.x; i < to; i += blockDim.x) {
        const int e = __ldg(a.pair_expert + i);
        if (e >= 0 && e < a.n_experts) atomicAdd(count + e, 1);
    }
    __syncthreads();
    for (int e = threadIdx.x; e < a.n_experts; e += blockDim.x) a.counts[static_cast<int64_t>(blockIdx.x) * a.n_experts + e] = count[e];
}

__global__ void __launch_bounds__(kSortThreads) place_kernel(const __grid_constant__ SortArgs a) {
    extern __shared__ int32_t shared[];
    const int E = a.n_experts, warps = blockDim.x >> 5;
    int32_t *run = shared;                       // [warps][E]: pairs of a run per expert, then the run's next free place
    int32_t *start = shared + warps * E;         // [E]: where this block's pairs of an expert go
    int32_t *total = start + E;                  // [E]: all pairs of an expert
    __shared__ int32_t warp_pairs[kSortWarps], warp_groups[kSortWarps];
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    for (int i = tid; i < warps * E; i += blockDim.x) run[i] = 0;
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    asm volatile("griddepcontrol.wait;" ::: "memory");
    __syncthreads();
    // this warp's run: whole rounds of 32 pairs
    const int64_t from = static_cast<int64_t>(blockIdx.x) * a.chunk;
    const int64_t to = smaller<int64_t>(a.n_pairs, from + a.chunk);
    const int rounds = static_cast<int>((to - from + 31) / 32), per = (rounds + warps - 1) / warps;
    const int64_t mine = from + static_cast<int64_t>(warp) * per * 32;
    const int64_t mine_end = smaller<int64_t>(to, mine + static_cast<int64_t>(per) * 32);
    int32_t *next = run + warp * E;
    for (int64_t i = mine + lane; i < mine_end; i += 32) {
        const int e = __ldg(a.pair_expert + i);
        if (e >= 0 && e < E) atomicAdd(next + e, 1);
    }
    __syncthreads();
    // an expert's pairs in this block's earlier runs, and in all if there is no other block
    for (int e = tid; e < E; e += blockDim.x) {
        int sum = 0;
        for (int w = 0; w < warps; ++w) {
            const int n = run[w * E + e];
            run[w * E + e] = sum;
            sum += n;
        }
        start[e] = 0;
        total[e] = gridDim.x > 1 ? 0 : sum;
    }
    __syncthreads();
    if (gridDim.x > 1) {
        // in earlier blocks, and in all: the blocks' counts are shared out over the threads (whole numbers: any order will do)
        const int parts = static_cast<int>(blockDim.x) > E ? static_cast<int>(blockDim.x) / E : 1, blocks = gridDim.x, each = (blocks + parts - 1) / parts;
        for (int i = tid; i < parts * E; i += blockDim.x) {
            const int e = i % E, b0 = i / E * each, b1 = smaller(blocks, b0 + each);
            int before = 0, all = 0;
#pragma unroll 8
            for (int b = b0; b < b1; ++b) {
                const int n = a.counts[static_cast<int64_t>(b) * E + e];
                if (b < static_cast<int>(blockIdx.x)) before += n;
                all += n;
            }
            if (before) atomicAdd(start + e, before);
            if (all) atomicAdd(total + e, all);
        }
        __syncthreads();
    }
    // experts in order: the pairs and the groups in front of each (blockDim.x experts a round)
    int pairs_before = 0, groups_before = 0;
    for (int base = 0; base < E; base += blockDim.x) {
        const int e = base + tid;
        const int n = e < E ? total[e] : 0;
        int p = n, g = n > 0;
#pragma unroll
        for (int d = 1; d < 32; d <<= 1) {
            const int up = __shfl_up_sync(kFull, p, d), ug = __shfl_up_sync(kFull, g, d);
            if (lane >= d) {
                p += up;
                g += ug;
            }
        }
        if (lane == 31) {
            warp_pairs[warp] = p;
            warp_groups[warp] = g;
        }
        __syncthreads();
        int all_pairs = 0, all_groups = 0;
        const int busy = smaller(warps, (E - base + 31) / 32);             // the warps with experts
        for (int w = 0; w < busy; ++w) {
            if (w == warp) {
                p += all_pairs;
                g += all_groups;
            }
            all_pairs += warp_pairs[w];
            all_groups += warp_groups[w];
        }
        if (e < E) {
            const int at = pairs_before + p - n, group = groups_before + g - (n > 0);
            start[e] += at;
            if (n > 0 && blockIdx.x == 0) {
                a.group_expert[group] = e;
                a.group_begin[group] = at;
            }
        }
        pairs_before += all_pairs;
        groups_before += all_groups;
        __syncthreads();
    }
    const int cap = smaller(a.n_pairs, E);
    if (blockIdx.x == 0) {
        for (int g = groups_before + tid; g <= cap; g += blockDim.x) {
            a.group_begin[g] = g == groups_before ? pairs_before : 0;
            if (g < cap) a.group_expert[g] = 0;
        }
        if (tid == 0) *a.n_groups = groups_before;
    }
    for (int64_t i = pairs_before + static_cast<int64_t>(blockIdx.x) * blockDim.x + tid; i < a.n_pairs; i += static_cast<int64_t>(gridDim.x) * blockDim.x) {
        a.xrow[i] = 0;
        a.order[i] = -1;
    }
    for (int64_t base = mine; base < mine_end; base += 32) {
        const int64_t i = base + lane;
        int e = i < mine_end ? __ldg(a.pair_expert + i) : -1;
        if (e < 0 || e >= E) e = -1;
        const uint32_t same = __match_any_sync(kFull, e);
        const int at = e >= 0 ? start[e] + next[e] + __popc(same & ((1u << lane) - 1u)) : -1;
        __syncwarp();
        if (e >= 0 && lane == __ffs(same) - 1) next[e] += __popc(same);
        __syncwarp();
        if (i < mine_end) a.slot[i] = at;
        if (at >= 0) {
            a.order[at] = static_cast<int32_t>(i);
            a.xrow[at] = static_cast<int32_t>(i / a.top_k);
        }
    }
}

// ---------------------------------------------------------------------------------------------
// out[t] = base[t] + sum over j of weight[t][j] * y[slot[t][j]], j ascending, in 32 bits; a thread takes W neighbouring
// columns of one token, reads up to eight experts' values before it adds the first, and rounds once.
// Bound by memory: every y row is read once.  8192 tokens x 8 of 2048 columns, bf16: 52.6 us (5.7 TB/s); what counts is bytes under way, eight
// loads a thread with four blocks a multiprocessor (without the bound on registers 71 us, three blocks 56, six blocks spill).
// ---------------------------------------------------------------------------------------------
struct CombineArgs {
    const void *y;
    const int32_t *slot;
    const float *weight;
    const void *base;           // NULL: none; the output's type
    void *out;
    int64_t chunks;             // tokens * (M / W)
    int64_t M;
    int64_t n_rows;             // rows of y
    int per_row;                // M / W
    int top_k;
};

// W neighbouring values as they lie in memory: words of 32 bits, or one value of 16.
template <typename T, int W>
struct Pack {
    static constexpr int kBytes = sizeof(T) * W, kWords = kBytes < 4 ? 1 : kBytes / 4;
    uint32_t w[kWords];
    __device__ __forceinline__ void load(const T *p) {
        if constexpr (kBytes % 16 == 0) {
#pragma unroll
            for (int i = 0; i < kWords; i += 4) *reinterpret_cast<uint4 *>(w + i) = __ldg(reinterpret_cast<const uint4 *>(p) + i / 4);
        } else if constexpr (kBytes == 8) *reinterpret_cast<uint2 *>(w) = __ldg(reinterpret_cast<const uint2 *>(p));
        else if constexpr (kBytes == 4) w[0] = __ldg(reinterpret_cast<const uint32_t *>(p));
        else w[0] = __ldg(reinterpret_cast<const uint16_t *>(p));
    }
    __device__ __forceinline__ void load_own(const T *p) {            // (of memory that the same thread may write)
        if constexpr (kBytes % 16 == 0) {
#pragma unroll
            for (int i = 0; i < kWords; i += 4) *reinterpret_cast<uint4 *>(w + i) = reinterpret_cast<const uint4 *>(p)[i / 4];
        } else if constexpr (kBytes == 8) *reinterpret_cast<uint2 *>(w) = *reinterpret_cast<const uint2 *>(p);
        else if constexpr (kBytes == 4) w[0] = *reinterpret_cast<const uint32_t *>(p);
        else w[0] = *reinterpret_cast<const uint16_t *>(p);
    }
    __device__ __forceinline__ float get(int i) const {
        if constexpr (sizeof(T) == 4) return __uint_as_float(w[i]);
        else return i & 1 ? bf16_hi(w[i / 2]) : bf16_lo(w[i / 2]);
    }
    __device__ __forceinline__ void put(int i, float v) {
        if constexpr (sizeof(T) == 4) w[i] = __float_as_uint(v);
        else {
            const uint32_t h = __bfloat16_as_ushort(__float2bfloat16_rn(v));
            w[i / 2] = i & 1 ? w[i / 2] | (h << 16) : h;
        }
    }
    __device__ __forceinline__ void store(T *p) const {
        if constexpr (kBytes % 16 == 0) {
#pragma unroll
            for (int i = 0; i < kWords; i += 4) reinterpret_cast<uint4 *>(p)[i / 4] = *reinterpret_cast<const uint4 *>(w + i);
        } else if constexpr (kBytes == 8) *reinterpret_cast<uint2 *>(p) = *reinterpret_cast<const uint2 *>(w);
        else if constexpr (kBytes == 4) *reinterpret_cast<uint32_t *>(p) = w[0];
        else *reinterpret_cast<uint16_t *>(p) = static_cast<uint16_t>(w[0]);
    }
};

constexpr int kCombineBatch = 8;
template <typename Y, typename O, int W>
__global__ void __launch_bounds__(256, 4) combine_kernel(const __grid_constant__ CombineArgs a) {
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    asm volatile("griddepcontrol.wait;" ::: "memory");
    const int64_t chunk = static_cast<int64_t>(blockIdx.x) * blockDim.x + threadIdx.x;
    if (chunk >= a.chunks) return;
    const int64_t token = chunk / a.per_row;
    const int64_t column = (chunk - token * a.per_row) * W;
    float acc[W];
    if (a.base) {
        Pack<O, W> b;
        b.load_own(static_cast<const O *>(a.base) + token * a.M + column);
#pragma unroll
        for (int i = 0; i < W; ++i) acc[i] = b.get(i);
    } else {
#pragma unroll
        for (int i = 0; i < W; ++i) acc[i] = 0.f;
    }
    const int32_t *slot = a.slot + token * a.top_k;
    const float *weight = a.weight + token * a.top_k;
    const Y *y = static_cast<const Y *>(a.y) + column;
    for (int j0 = 0; j0 < a.top_k; j0 += kCombineBatch) {
        Pack<Y, W> part[kCombineBatch];
        float w[kCombineBatch];
        uint32_t there = 0;
#pragma unroll
        for (int j = 0; j < kCombineBatch; ++j) {
            const int r = j0 + j < a.top_k ? __ldg(slot + j0 + j) : -1;
            if (r >= 0 && r < a.n_rows) {
                there |= 1u << j;
                w[j] = __ldg(weight + j0 + j);
                part[j].load(y + r * a.M);
            }
        }
#pragma unroll
        for (int j = 0; j < kCombineBatch; ++j)
            if ((there >> j) & 1u) {
#pragma unroll
                for (int i = 0; i < W; ++i) acc[i] = fmaf(w[j], part[j].get(i), acc[i]);
            }
    }
    Pack<O, W> o;
#pragma unroll
    for (int i = 0; i < W; ++i) o.put(i, acc[i]);
    o.store(static_cast<O *>(a.out) + token * a.M + column);
}

template <typename Y, typename O, int W>
int launch_combine_wide(CombineArgs a, int64_t tokens, cudaStream_t stream) {
    a.per_row = static_cast<int>(a.M / W);
    a.chunks = tokens * a.per_row;
    const int64_t blocks = (a.chunks + 255) / 256;
    if (blocks > INT_MAX) return BITCOS_ERR_SHAPE;
    return launch_pdl(combine_kernel<Y, O, W>, dim3(static_cast<unsigned>(blocks)), 256, 0, stream, a);
}

template <typename Y, typename O>
int launch_combine(const CombineArgs &a, int64_t tokens, cudaStream_t stream) {
    // whole 16-byte loads of y where the rows allow them (rows are M elements apart, all pointers are 16-byte aligned)
    constexpr int kMost = 16 / sizeof(Y);
    if (a.M % kMost == 0) return launch_combine_wide<Y, O, kMost>(a, tokens, stream);
    if (a.M % 2 == 0) return launch_combine_wide<Y, O, 2>(a, tokens, stream);
    return launch_combine_wide<Y, O, 1>(a, tokens, stream);
}

}  // namespace

extern "C" {

int bitcos_route_experts(const void *logits, int logits_type, int64_t row_stride, const float *bias, int n_tokens, int n_experts,
                         int score, int n_groups, int top_groups, int group_best, int top_k, int renormalise, float scale,
                         int32_t *expert, float *weight, int32_t *pair_xrow, void *cuda_stream) {
    if (!logits || !expert || !weight || !pair_xrow) return BITCOS_ERR_NULL;
    if (n_tokens < 0 || n_experts < 1 || n_experts > BITCOS_GROUP_EXPERTS_MAX || row_stride < n_experts) return BITCOS_ERR_SHAPE;
    if (top_k < 1 || top_k > BITCOS_ROUTE_TOP_K_MAX || static_cast<int64_t>(n_tokens) * top_k > INT_MAX) return BITCOS_ERR_SHAPE;
    if (score != BITCOS_SCORE_SOFTMAX && score != BITCOS_SCORE_SIGMOID) return BITCOS_ERR_SHAPE;
    if (n_groups < 1 || n_groups > kMaxRouteGroups || n_experts % n_groups != 0 || top_groups < 1 || top_groups > n_groups)
        return BITCOS_ERR_SHAPE;
    if (group_best < 1 || group_best > 2 || (n_groups > 1 && group_best > n_experts / n_groups)) return BITCOS_ERR_SHAPE;
    if (logits_type != BITCOS_FP32 && logits_type != BITCOS_BF16 && logits_type != BITCOS_FP16) return BITCOS_ERR_SHAPE;
    const size_t size = logits_type == BITCOS_FP32 ? 4 : 2;
    if (reinterpret_cast<uintptr_t>(logits) % size || reinterpret_cast<uintptr_t>(bias) % 4 || reinterpret_cast<uintptr_t>(expert) % 4 ||
        reinterpret_cast<uintptr_t>(weight) % 4 || reinterpret_cast<uintptr_t>(pair_xrow) % 4)
        return BITCOS_ERR_ALIGN;
    if (n_tokens == 0) return BITCOS_OK;
    RouteArgs a{};
    a.logits = logits;
    a.bias = bias;
    a.row_stride = row_stride;
    a.expert = expert;
    a.weight = weight;
    a.xrow = pair_xrow;
    a.scale = scale;
    a.tokens = n_tokens;
    a.experts = n_experts;
    a.top_k = top_k;
    a.n_groups = n_groups;
    a.top_groups = top_groups;
    a.group_best = group_best;
    a.group_size = n_experts / n_groups;
    a.softmax = score == BITCOS_SCORE_SOFTMAX;
    a.renormalise = renormalise != 0;
    a.by_choice = bias != nullptr || (n_groups > 1 && group_best == 2);
    cudaStream_t stream = static_cast<cudaStream_t>(cuda_stream);
    if (logits_type == BITCOS_FP32) return launch_route_type<float>(a, stream);
    if (logits_type == BITCOS_BF16) return launch_route_type<__nv_bfloat16>(a, stream);
    return launch_route_type<__half>(a, stream);
}

size_t bitcos_group_workspace_bytes(int64_t n_pairs, int n_experts) {
    if (n_pairs < 0 || n_pairs > INT_MAX || n_experts < 1 || n_experts > BITCOS_GROUP_EXPERTS_MAX) return 0;
    const int blocks = sort_blocks(n_pairs);
    return blocks == 1 ? 256 : (static_cast<size_t>(blocks) * n_experts * sizeof(int32_t) + 255) / 256 * 256;
}

int bitcos_group_pairs_slots(const int32_t *pair_expert, int64_t n_pairs, int top_k, int n_experts, int32_t *group_expert,
                             int32_t *group_begin, int32_t *pair_xrow_sorted, int32_t *order, int32_t *slot, int32_t *n_groups,
                             void *workspace, size_t workspace_bytes, void *cuda_stream) {
    if (!pair_expert || !group_expert || !group_begin || !pair_xrow_sorted || !order || !slot || !n_groups || !workspace)
        return BITCOS_ERR_NULL;
    if (n_pairs < 1 || n_pairs > INT_MAX || top_k < 1 || n_experts < 1 || n_experts > BITCOS_GROUP_EXPERTS_MAX) return BITCOS_ERR_SHAPE;
    for (const void *p : {static_cast<const void *>(pair_expert), static_cast<const void *>(group_expert), static_cast<const void *>(group_begin),
                          static_cast<const void *>(pair_xrow_sorted), static_cast<const void *>(order), static_cast<const void *>(slot),
                          static_cast<const void *>(n_groups), static_cast<const void *>(workspace)})
        if (reinterpret_cast<uintptr_t>(p) % 4) return BITCOS_ERR_ALIGN;
    if (workspace_bytes < bitcos_group_workspace_bytes(n_pairs, n_experts)) return BITCOS_ERR_CAPACITY;
    cudaStream_t stream = static_cast<cudaStream_t>(cuda_stream);
    SortArgs a{pair_expert, group_expert, group_begin, pair_xrow_sorted, order, slot, n_groups, static_cast<int32_t *>(workspace),
               static_cast<int>(n_pairs), n_experts, top_k, 0};
    const int blocks = sort_blocks(n_pairs);
    a.chunk = static_cast<int>(((n_pairs + blocks - 1) / blocks + 31) / 32 * 32);
    // threads: a warp for every 32 pairs of a chunk, but enough of them for the experts and for the blocks' counts, 32 a thread
    // (32768 pairs of 128 experts: 8.2 us with 512 threads, 12.8 with 256; of 256 experts 10.1 with 1024, 20 with 256)
    const int64_t counts = blocks > 1 ? (static_cast<int64_t>(blocks) * n_experts / 32 + 31) / 32 * 32 : 128;
    int64_t threads = std::max<int64_t>({(n_experts + 31) / 32 * 32, a.chunk, counts});
    threads = std::min<int64_t>(kSortThreads, std::max<int64_t>(threads, 128));
    const size_t smem = (threads / 32 + 2) * static_cast<size_t>(n_experts) * sizeof(int32_t);
    int sms = 0, budget = 0;
    int rc = prepare_kernel<place_kernel>(&sms, &budget);
    if (rc) return rc;
    if (blocks > 1) {
        // (four pairs a thread: 262144 pairs 12.7 us with 256 threads, 13.2 with 1024; a million of 1000 experts 35.3 and 34.3)
        const int counting = static_cast<int>(std::min<int64_t>(kSortThreads, std::max<int64_t>(256, (a.chunk / 4 + 31) / 32 * 32)));
        rc = launch_pdl(count_kernel, dim3(static_cast<unsigned>(blocks)), counting, n_experts * sizeof(int32_t), stream, a);
        if (rc) return rc;
    }
    return launch_pdl(place_kernel, dim3(static_cast<unsigned>(blocks)), static_cast<int>(threads), smem, stream, a);
}

int bitcos_combine_pairs(const void *y, int y_type, int64_t n_rows, const int32_t *slot, const float *weight, int64_t n_tokens, int top_k,
                         int64_t M, const void *base, void *out, int out_type, void *cuda_stream) {
    if (!y || !slot || !weight || !out) return BITCOS_ERR_NULL;
    if (n_rows < 1 || n_tokens < 0 || n_tokens > INT_MAX || top_k < 1 || M < 1 || M > INT_MAX) return BITCOS_ERR_SHAPE;
    if ((y_type != BITCOS_FP32 && y_type != BITCOS_BF16) || (out_type != BITCOS_FP32 && out_type != BITCOS_BF16)) return BITCOS_ERR_SHAPE;
    if (!aligned16(y) || !aligned16(out) || (base && !aligned16(base)) || reinterpret_cast<uintptr_t>(slot) % 4 ||
        reinterpret_cast<uintptr_t>(weight) % 4)
        return BITCOS_ERR_ALIGN;
    if (n_tokens == 0) return BITCOS_OK;
    CombineArgs a{y, slot, weight, base, out, 0, M, n_rows, 0, top_k};
    cudaStream_t stream = static_cast<cudaStream_t>(cuda_stream);
    if (y_type == BITCOS_FP32)
        return out_type == BITCOS_FP32 ? launch_combine<float, float>(a, n_tokens, stream) : launch_combine<float, __nv_bfloat16>(a, n_tokens, stream);
    return out_type == BITCOS_FP32 ? launch_combine<__nv_bfloat16, float>(a, n_tokens, stream)
                                   : launch_combine<__nv_bfloat16, __nv_bfloat16>(a, n_tokens, stream);
}

}  // extern "C"
