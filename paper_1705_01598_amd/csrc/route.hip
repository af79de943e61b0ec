// The router's choice: the largest scores of every token, their softmax, and its gradient.
//
// A group of 16 or 64 lanes to a token, every lane some of its scores in registers as whole numbers that order as the scores
// do.  A round finds the largest number of the group by DPP moves, then the lowest expert that has it, and strikes it out; the
// lane whose turn it is keeps it for the softmax.  Scores are read once; the rounds are what there is to compute.
#include "decode.hpp"
#include "expert_vector.hpp"
#include "plan.hpp"

namespace tperm {

namespace {

constexpr int kRouteThreads = 256;

// Numbers above 0 that order as scores do; 0 for minus infinity, NaN and what is not there.
__device__ __forceinline__ uint32_t key_of(float v) {
    const uint32_t b = __float_as_uint(v + 0.0f);       // one zero
    return v > -__builtin_inff() ? ((int32_t)b < 0 ? ~b : b | 0x80000000u) : 0u;
}
__device__ __forceinline__ float score_of(uint32_t key) { return __uint_as_float((int32_t)key < 0 ? key & 0x7FFFFFFFu : ~key); }

template <int CTRL> __device__ __forceinline__ uint32_t moved(uint32_t v) { return (uint32_t)__builtin_amdgcn_mov_dpp((int)v, CTRL, 0xF, 0xF, true); }
// f over the lanes of a group, in all of them: rotations of a row of 16, then across the rows.
template <int LANES, typename F> __device__ __forceinline__ uint32_t over_group(uint32_t v, F f) {
    v = f(v, moved<0x121>(v));
    v = f(v, moved<0x122>(v));
    v = f(v, moved<0x124>(v));
    v = f(v, moved<0x128>(v));
    if constexpr (LANES == 64) {
        v = f(v, (uint32_t)__shfl_xor((int)v, 16));
        v = f(v, (uint32_t)__shfl_xor((int)v, 32));
    }
    return v;
}
template <int LANES> __device__ __forceinline__ uint32_t largest(uint32_t v) { return over_group<LANES>(v, [](uint32_t a, uint32_t b) { return a > b ? a : b; }); }
template <int LANES> __device__ __forceinline__ uint32_t least(uint32_t v) { return over_group<LANES>(v, [](uint32_t a, uint32_t b) { return a < b ? a : b; }); }
// Sums in an order that is the same for every lane: pairs at a distance, and addition of two does not depend on which is first.
template <int LANES> __device__ __forceinline__ float total(float v) {
    for (int d = 1; d < LANES; d <<= 1) v += __shfl_xor(v, d);
    return v;
}

// exp(score - most), 1 for the largest also where that is infinite.
__device__ __forceinline__ float part_of(float v, float most) { return v == most ? 1.0f : expf(v - most); }

// V scores a lane: expert v * LANES + lane.
template <typename T, int LANES, int V, bool OVER_ALL> __global__ __launch_bounds__(kRouteThreads) void route_kernel(const RouteArgs a) {
    const uint32_t lane = threadIdx.x % LANES;
    const uint64_t t = long_block() * (kRouteThreads / LANES) + threadIdx.x / LANES;
    const uint64_t token = t < a.tokens ? t : a.tokens - 1;
    const T* const row = (const T*)a.scores + (int64_t)token * a.scores_stride;
    uint32_t key[V];
#pragma unroll
    for (int v = 0; v < V; ++v) {
        const uint32_t e = v * LANES + lane;
        key[v] = key_of(e < a.experts ? (float)row[e] : -__builtin_inff());
    }
    uint32_t best = 0, at = 0;
    const auto find = [&] {
        best = key[0], at = 0;
#pragma unroll
        for (int v = 1; v < V; ++v)
            if (key[v] > best) best = key[v], at = v;
    };
    find();
    const uint32_t most_key = largest<LANES>(best);
    const float most = score_of(most_key);
    float all = 0.0f;
    if constexpr (OVER_ALL) {
#pragma unroll
        for (int v = 0; v < V; ++v) all += key[v] != 0 ? part_of(score_of(key[v]), most) : 0.0f;
        all = total<LANES>(all);
    }
    constexpr int kKept = TPERM_SLOTS_MAX / LANES;
    uint32_t kept[kKept] = {};
    int32_t number[kKept];
#pragma unroll
    for (int k = 0; k < kKept; ++k) number[k] = -1;
#pragma unroll
    for (int k = 0; k < kKept; ++k)
        for (uint32_t s = 0; s < LANES && k * LANES + s < a.slots; ++s) {
            const uint32_t top = largest<LANES>(best), mine = at * LANES + lane, e = least<LANES>(best == top ? mine : 0xFFFFFFFFu);
            if (s == lane) kept[k] = top, number[k] = top != 0 ? (int32_t)e : -1;
            if (e == mine && best == top) {
#pragma unroll
                for (int v = 0; v < V; ++v) key[v] = (uint32_t)v == at ? 0u : key[v];
                find();
            }
        }
    float part[kKept];
    float chosen = 0.0f;
#pragma unroll
    for (int k = 0; k < kKept; ++k) {
        part[k] = kept[k] != 0 ? part_of(score_of(kept[k]), most) : 0.0f;
        chosen += part[k];
    }
    const float by = OVER_ALL ? all : total<LANES>(chosen);
    if (t >= a.tokens) return;
#pragma unroll
    for (int k = 0; k < kKept; ++k) {
        const uint32_t s = k * LANES + lane;
        if (s >= a.slots) continue;
        a.expert[token * a.slots + s] = number[k];
        a.weights[token * a.slots + s] = kept[k] != 0 ? part[k] / by : 0.0f;
    }
}

template <typename T, int LANES, int V, bool OVER_ALL> __global__ __launch_bounds__(kRouteThreads) void route_backward_kernel(const RouteArgs a) {
    const uint32_t lane = threadIdx.x % LANES;
    const uint64_t t = long_block() * (kRouteThreads / LANES) + threadIdx.x / LANES;
    const uint64_t token = t < a.tokens ? t : a.tokens - 1;
    constexpr int kKept = TPERM_SLOTS_MAX / LANES;
    int32_t number[kKept];
    float weight[kKept], each[kKept], sum = 0.0f;
#pragma unroll
    for (int k = 0; k < kKept; ++k) {
        const uint32_t s = k * LANES + lane;
        number[k] = s < a.slots ? a.expert[token * a.slots + s] : -1;
        const bool there = (uint32_t)number[k] < a.experts;
        weight[k] = there ? a.weights[token * a.slots + s] : 0.0f;
        each[k] = there ? weight[k] * a.grad_weights[token * a.slots + s] : 0.0f;
        sum += each[k];
    }
    const float mean = total<LANES>(sum);
    float grad[V];
    if constexpr (OVER_ALL) {
        const T* const row = (const T*)a.scores + (int64_t)token * a.scores_stride;
        uint32_t key[V], best = 0;
#pragma unroll
        for (int v = 0; v < V; ++v) {
            const uint32_t e = v * LANES + lane;
            key[v] = key_of(e < a.experts ? (float)row[e] : -__builtin_inff());
            best = key[v] > best ? key[v] : best;
        }
        const float most = score_of(largest<LANES>(best));
        float all = 0.0f;
#pragma unroll
        for (int v = 0; v < V; ++v) {
            grad[v] = key[v] != 0 ? part_of(score_of(key[v]), most) : 0.0f;
            all += grad[v];
        }
        all = total<LANES>(all);
#pragma unroll
        for (int v = 0; v < V; ++v) grad[v] = key[v] != 0 ? grad[v] / all * -mean : 0.0f;
    } else {
#pragma unroll
        for (int v = 0; v < V; ++v) grad[v] = 0.0f;
#pragma unroll
        for (int k = 0; k < kKept; ++k) each[k] -= weight[k] * mean;
    }
#pragma unroll
    for (int k = 0; k < kKept; ++k)
        for (uint32_t s = 0; s < LANES && k * LANES + s < a.slots; ++s) {
            const int32_t e = __shfl(number[k], (int)s, LANES);
            const float d = __shfl(each[k], (int)s, LANES);
#pragma unroll
            for (int v = 0; v < V; ++v) grad[v] += e == (int32_t)(v * LANES + lane) ? d : 0.0f;
        }
    if (t >= a.tokens) return;
    T* const out = (T*)a.grad_scores + (int64_t)token * a.grad_stride;
#pragma unroll
    for (int v = 0; v < V; ++v) {
        const uint32_t e = v * LANES + lane;
        if (e < a.experts) out[e] = (T)grad[v];
    }
}

template <int LANES, typename K> hipError_t go(K kernel, const RouteArgs& a, hipStream_t stream) {
    const uint64_t each = kRouteThreads / LANES;
    hipLaunchKernelGGL(kernel, long_grid((a.tokens + each - 1) / each), dim3(kRouteThreads), 0, stream, a);
    return hipGetLastError();
}
#define TPERM_BY_EXPERTS(KERNEL)                                                                                     \
    (a.experts <= 32    ? go<16>(KERNEL<T, 16, 2, OVER_ALL>, a, stream)                                              \
     : a.experts <= 64  ? go<16>(KERNEL<T, 16, 4, OVER_ALL>, a, stream)                                              \
     : a.experts <= 128 ? go<16>(KERNEL<T, 16, 8, OVER_ALL>, a, stream)                                              \
     : a.experts <= 256 ? go<64>(KERNEL<T, 64, 4, OVER_ALL>, a, stream)                                              \
                        : go<64>(KERNEL<T, 64, 16, OVER_ALL>, a, stream))
template <typename T, bool OVER_ALL> hipError_t route_of(const RouteArgs& a, hipStream_t stream) { return TPERM_BY_EXPERTS(route_kernel); }
template <typename T, bool OVER_ALL> hipError_t backward_of(const RouteArgs& a, hipStream_t stream) { return TPERM_BY_EXPERTS(route_backward_kernel); }

}  // namespace

hipError_t launch_route(const RouteArgs& a, bool over_all, int type, hipStream_t stream) {
    return with_type(type, [&](auto t) { return over_all ? route_of<decltype(t), true>(a, stream) : route_of<decltype(t), false>(a, stream); });
}
hipError_t launch_route_backward(const RouteArgs& a, bool over_all, int type, hipStream_t stream) {
    return with_type(type, [&](auto t) { return over_all ? backward_of<decltype(t), true>(a, stream) : backward_of<decltype(t), false>(a, stream); });
}

}  // namespace tperm
