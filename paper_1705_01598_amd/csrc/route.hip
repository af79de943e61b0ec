// The router's choice: the largest scores of every token, their softmax, and its gradient.
//
// A group of lanes to a token, every lane some of its scores in registers as numbers that order as the scores do.  Up to 8 slots:
// every lane sorts its scores eight (or four) at a time, two sorted lists become the best eight of both by one comparison
// of each with the other in reverse and a bitonic merge, first in a lane, then between lanes by DPP moves.  A score's expert is part of
// its number (the lower, the larger), so that no two are equal and a comparison is one instruction for the larger and one for
// the smaller: whole numbers of 32 bits where scores have 16, doubles where they have 32.  More slots: a round for each finds the
// largest number of the group and strikes it out.
//
// 65536 tokens x 8 of 128 experts: binary32 9.5 us for 38 MB, of which 1.6 is an empty launch, 5.6 the bytes, and the comparisons of doubles, which run at half the
// rate, the longest part (two tokens a lane, the second's scores requested first, 10.4; rounds that strike out, for any number of slots, 19.9); bfloat16 through all 128 9.8.  33 x 4 of 64: 2.2 us.
// Gradient of 16384 x 6 of 101, binary32, through all: 6.6 us for 14 MB; 65536 x 8 of 128 bfloat16 11 us.
#include <type_traits>

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
// f over the lanes of a group, in all of them: lanes 1 and 2 apart, mirrored in 8 and in 16, then across the rows.
template <int LANES, typename F> __device__ __forceinline__ uint32_t over_group(uint32_t v, F f) {
    v = f(v, moved<0xB1>(v));
    v = f(v, moved<0x4E>(v));
    if constexpr (LANES > 4) v = f(v, moved<0x141>(v));
    if constexpr (LANES > 8) v = f(v, moved<0x140>(v));
    if constexpr (LANES == 64) {
        v = f(v, (uint32_t)__shfl_xor((int)v, 16));
        v = f(v, (uint32_t)__shfl_xor((int)v, 32));
    }
    return v;
}
template <int LANES> __device__ __forceinline__ uint32_t largest(uint32_t v) { return over_group<LANES>(v, [](uint32_t a, uint32_t b) { return a > b ? a : b; }); }
template <int LANES> __device__ __forceinline__ uint32_t least(uint32_t v) { return over_group<LANES>(v, [](uint32_t a, uint32_t b) { return a < b ? a : b; }); }
// Sums, the same bits in every lane: who adds does not matter to a sum of two.
template <int LANES> __device__ __forceinline__ float total(float v) {
    const auto add = [&](uint32_t o) { v += __uint_as_float(o); };
    add(moved<0xB1>(__float_as_uint(v)));           // 1 0 3 2
    add(moved<0x4E>(__float_as_uint(v)));           // 2 3 0 1
    if constexpr (LANES > 4) add(moved<0x141>(__float_as_uint(v)));     // mirrored in 8 lanes
    if constexpr (LANES > 8) add(moved<0x140>(__float_as_uint(v)));     // and in 16
    if constexpr (LANES > 16) v += __shfl_xor(v, 16);
    if constexpr (LANES > 32) v += __shfl_xor(v, 32);
    return v;
}

// exp(score - most), 1 for the largest also where that is infinite; 2^x with what x * log2(e) rounds off put right, which leaves
// 2^-23 for exp2 and 2^-24 |x| for the difference.
__device__ __forceinline__ float part_of(float v, float most) {
    constexpr float kLog = 0x1.715476p+0f, kRest = 0x1.4ae0cp-26f;     // log2(e) and what that rounds off
    const float x = v - most, p = x * kLog, rest = __builtin_fmaf(x, kRest, __builtin_fmaf(x, kLog, -p));
    float e = __builtin_amdgcn_exp2f(p);
    e = __builtin_fmaf(e, rest * 0.6931472f, e);
    e = x < -104.0f ? 0.0f : e;         // also where rest is no number
    return v == most ? 1.0f : e;
}

// The same for a sum over all scores, where what the product rounds off, 2^-24 |x| exp(-|x|) at most, is less than what the sum does.
__device__ __forceinline__ float rough_part_of(float v, float most) {
    const float e = __builtin_amdgcn_exp2f((v - most) * 0x1.715476p+0f);
    return v == most ? 1.0f : e;
}

// Numbers that order as the scores of T do, equal ones by expert, none equal to another; minus infinity is barred.  The bits of a score of 16
// as binary32, all but the sign of negative ones complemented: 13 low bits are free for the expert.
template <typename T> struct Ordered {
    typedef int32_t Key;
    static constexpr uint32_t kFree = 0x1FFFu;
    static __device__ __forceinline__ Key key(T v, uint32_t expert) {
        const uint32_t b = __float_as_uint(__builtin_fmaxf((float)v + 0.0f, -__builtin_inff()));      // one zero; NaN as minus infinity
        return (Key)((b ^ ((uint32_t)((int32_t)b >> 31) & (0x7FFFFFFFu & ~kFree))) | (TPERM_EXPERTS_MAX - 1 - expert));
    }
    static __device__ __forceinline__ uint32_t expert(Key k) { return TPERM_EXPERTS_MAX - 1 - ((uint32_t)k & kFree); }
    static __device__ __forceinline__ float score(Key k) {
        const uint32_t b = (uint32_t)k & ~kFree;
        return __uint_as_float(b ^ ((uint32_t)(k >> 31) & (0x7FFFFFFFu & ~kFree)));
    }
    static __device__ __forceinline__ bool barred(Key k) { return score(k) == -__builtin_inff(); }
    static __device__ __forceinline__ Key high(Key a, Key b) { return a > b ? a : b; }
    static __device__ __forceinline__ Key low(Key a, Key b) { return a < b ? a : b; }
};
// The score's bits as the high word of a double, which orders as they do (only a NaN's would make one), and behind them the expert, complemented
// under a negative sign; minus infinity is barred.
template <> struct Ordered<float> {
    typedef double Key;
    static __device__ __forceinline__ Key key(float v, uint32_t expert) {
        const uint32_t b = __float_as_uint(__builtin_fmaxf(v + 0.0f, -__builtin_inff()));      // one zero; NaN as minus infinity
        return __builtin_bit_cast(double, (uint64_t)b << 32 | (uint32_t)((int32_t)b >> 31 ^ (int32_t)(TPERM_EXPERTS_MAX - 1 - expert)));
    }
    static __device__ __forceinline__ uint32_t bits(Key k) { return (uint32_t)(__builtin_bit_cast(uint64_t, k) >> 32); }
    static __device__ __forceinline__ uint32_t expert(Key k) {
        return TPERM_EXPERTS_MAX - 1 - ((uint32_t)__builtin_bit_cast(uint64_t, k) ^ (uint32_t)((int32_t)bits(k) >> 31));
    }
    static __device__ __forceinline__ bool barred(Key k) { return bits(k) == 0xFF800000u; }
    static __device__ __forceinline__ float score(Key k) { return __uint_as_float(bits(k)); }
    static __device__ __forceinline__ Key high(Key a, Key b) { return __builtin_fmax(a, b); }
    static __device__ __forceinline__ Key low(Key a, Key b) { return __builtin_fmin(a, b); }
};
template <int CTRL> __device__ __forceinline__ int32_t from_lane(int32_t v) { return (int32_t)moved<CTRL>((uint32_t)v); }
template <int CTRL> __device__ __forceinline__ double from_lane(double v) {
    const uint64_t b = __builtin_bit_cast(uint64_t, v);
    return __builtin_bit_cast(double, (uint64_t)moved<CTRL>((uint32_t)(b >> 32)) << 32 | moved<CTRL>((uint32_t)b));
}
__device__ __forceinline__ int32_t across(int32_t v, int lanes) { return __shfl_xor(v, lanes); }
__device__ __forceinline__ double across(double v, int lanes) { return __shfl_xor(v, lanes); }

template <typename O, int I, int J, int P> __device__ __forceinline__ void exchange(typename O::Key (&k)[P]) {
    const typename O::Key a = k[I], b = k[J];
    k[I] = O::high(a, b), k[J] = O::low(a, b);
}
// Largest first; networks of 19 and 5 exchanges.
template <typename O> __device__ __forceinline__ void sort(typename O::Key (&k)[8]) {
    exchange<O, 0, 2>(k), exchange<O, 1, 3>(k), exchange<O, 4, 6>(k), exchange<O, 5, 7>(k);
    exchange<O, 0, 4>(k), exchange<O, 1, 5>(k), exchange<O, 2, 6>(k), exchange<O, 3, 7>(k);
    exchange<O, 0, 1>(k), exchange<O, 2, 3>(k), exchange<O, 4, 5>(k), exchange<O, 6, 7>(k);
    exchange<O, 2, 4>(k), exchange<O, 3, 5>(k);
    exchange<O, 1, 4>(k), exchange<O, 3, 6>(k);
    exchange<O, 1, 2>(k), exchange<O, 3, 4>(k), exchange<O, 5, 6>(k);
}
template <typename O> __device__ __forceinline__ void sort(typename O::Key (&k)[4]) {
    exchange<O, 0, 1>(k), exchange<O, 2, 3>(k), exchange<O, 0, 2>(k), exchange<O, 1, 3>(k), exchange<O, 1, 2>(k);
}
// The best P of a sorted list and another one, sorted.
template <typename O, int P, typename F> __device__ __forceinline__ void merge(typename O::Key (&k)[P], F other) {
    typename O::Key both[P];
#pragma unroll
    for (int i = 0; i < P; ++i) both[i] = O::high(k[i], other(P - 1 - i));
#pragma unroll
    for (int i = 0; i < P; ++i) k[i] = both[i];
    if constexpr (P == 8) exchange<O, 0, 4>(k), exchange<O, 1, 5>(k), exchange<O, 2, 6>(k), exchange<O, 3, 7>(k);
    if constexpr (P == 8) exchange<O, 4, 6>(k), exchange<O, 5, 7>(k);
    exchange<O, 0, 2>(k), exchange<O, 1, 3>(k);
    if constexpr (P == 8) exchange<O, 4, 5>(k), exchange<O, 6, 7>(k);
    exchange<O, 0, 1>(k), exchange<O, 2, 3>(k);
}

// Up to P slots, V scores a lane.  ALIGNED: rows of whole 16 bytes, which a lane takes in turn with its neighbours.
template <typename T, int LANES, int V, int P, bool ALIGNED> __global__ __launch_bounds__(kRouteThreads) void route_few_kernel(const RouteArgs a, const bool over_all) {
    typedef Ordered<T> O;
    typedef typename O::Key Key;
    constexpr int C = ALIGNED ? 16 / (int)sizeof(T) : 1;
    static_assert(V % C == 0 && V % P == 0, "whole loads and lists");
    const uint32_t lane = threadIdx.x % LANES;
    const uint64_t t = long_block() * (kRouteThreads / LANES) + threadIdx.x / LANES;
    const uint64_t token = t < a.tokens ? t : a.tokens - 1;
    const T* const row = (const T*)a.scores + (int64_t)token * a.scores_stride;
    const auto expert_of = [&](int v) { return (uint32_t)(v / C * LANES * C + lane * C + v % C); };
    T score[V];
#pragma unroll
    for (int v = 0; v < V; v += C) {
        const uint32_t e = expert_of(v);
        const Vec<T, C> part = load_vec<T, C, ALIGNED>(row + (e < a.experts ? e : 0u));
        for (int c = 0; c < C; ++c) score[v + c] = part[c];
    }
    Key list[V / P][P];
#pragma unroll
    for (int v = 0; v < V; ++v) list[v / P][v % P] = O::key(expert_of(v) < a.experts ? score[v] : (T)-__builtin_inff(), expert_of(v));
#pragma unroll
    for (int l = 0; l < V / P; ++l) sort<O>(list[l]);
#pragma unroll
    for (int l = 1; l < V / P; ++l) merge<O, P>(list[0], [&](int i) { return list[l][i]; });
    Key(&best)[P] = list[0];
    merge<O, P>(best, [&](int i) { return from_lane<0xB1>(best[i]); });                                    // 1 0 3 2
    merge<O, P>(best, [&](int i) { return from_lane<0x4E>(best[i]); });                                    // 2 3 0 1
    if constexpr (LANES > 4) merge<O, P>(best, [&](int i) { return from_lane<0x141>(best[i]); });          // mirrored in 8 lanes
    if constexpr (LANES > 8) merge<O, P>(best, [&](int i) { return from_lane<0x140>(best[i]); });          // and in 16
    if constexpr (LANES > 16) merge<O, P>(best, [&](int i) { return across(best[i], 16); });
    if constexpr (LANES > 32) merge<O, P>(best, [&](int i) { return across(best[i], 32); });
    const float most = O::score(best[0]);
    // lane l holds slots l, l + LANES, ...
    constexpr int kKept = LANES < P ? P / LANES : 1;
    Key kept[kKept];
    float part[kKept], sum = 0.0f;
#pragma unroll
    for (int k = 0; k < kKept; ++k) {
        kept[k] = best[k * LANES];
#pragma unroll
        for (int l = 1; l < LANES && k * LANES + l < P; ++l) kept[k] = lane == (uint32_t)l ? best[k * LANES + l] : kept[k];
        part[k] = k * LANES + lane < a.slots && !O::barred(kept[k]) ? part_of(O::score(kept[k]), most) : 0.0f;
        sum += part[k];
    }
    if (over_all) {
        sum = 0.0f;
#pragma unroll
        for (int v = 0; v < V; ++v) {
            const float s = (float)score[v];
            const float part = rough_part_of(s, most);
            sum += expert_of(v) < a.experts && s > -__builtin_inff() ? part : 0.0f;
        }
    }
    sum = total<LANES>(sum);
    if (t >= a.tokens) return;
#pragma unroll
    for (int k = 0; k < kKept; ++k) {
        const uint32_t s = k * LANES + lane;
        if (s >= a.slots) continue;
        const bool there = s < (uint32_t)P && !O::barred(kept[k]);
        a.expert[token * a.slots + s] = there ? (int32_t)O::expert(kept[k]) : -1;
        a.weights[token * a.slots + s] = there ? part[k] / sum : 0.0f;
    }
}

// Any number of slots, V scores a lane: expert v * LANES + lane.
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
        for (int v = 0; v < V; ++v) all += key[v] != 0 ? rough_part_of(score_of(key[v]), most) : 0.0f;
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

// KEPT: up to that many slots, which every lane loads, or 0: any number, each in a lane and handed round.
// ALIGNED: rows of whole 16 bytes, which a lane takes in turn with its neighbours.
template <typename T, int LANES, int V, int KEPT, bool OVER_ALL, bool ALIGNED> __global__ __launch_bounds__(kRouteThreads) void route_backward_kernel(const RouteArgs a) {
    constexpr int C = ALIGNED ? 16 / (int)sizeof(T) : 1;
    static_assert(V % C == 0, "whole loads");
    const uint32_t lane = threadIdx.x % LANES;
    const uint64_t t = long_block() * (kRouteThreads / LANES) + threadIdx.x / LANES;
    const uint64_t token = t < a.tokens ? t : a.tokens - 1;
    const auto expert_of = [&](int v) { return (uint32_t)(v / C * LANES * C + lane * C + v % C); };
    constexpr int kHere = KEPT != 0 ? KEPT : TPERM_SLOTS_MAX / LANES;
    int32_t number[kHere];
    float weight[kHere], each[kHere], mean = 0.0f;
#pragma unroll
    for (int k = 0; k < kHere; ++k) {
        const uint32_t s = KEPT != 0 ? k : k * LANES + lane, at = s < a.slots ? s : a.slots - 1;
        number[k] = a.expert[token * a.slots + at], weight[k] = a.weights[token * a.slots + at], each[k] = a.grad_weights[token * a.slots + at];
    }
    T score[V];
    if constexpr (OVER_ALL) {
        const T* const row = (const T*)a.scores + (int64_t)token * a.scores_stride;
#pragma unroll
        for (int v = 0; v < V; v += C) {
            const uint32_t e = expert_of(v);
            const Vec<T, C> part = load_vec<T, C, ALIGNED>(row + (e < a.experts ? e : 0u));
            for (int c = 0; c < C; ++c) score[v + c] = part[c];
        }
    }
#pragma unroll
    for (int k = 0; k < kHere; ++k) {
        const bool there = (uint32_t)(KEPT != 0 ? k : k * LANES + lane) < a.slots && (uint32_t)number[k] < a.experts;
        weight[k] = there ? weight[k] : 0.0f, number[k] = there ? number[k] : -1;
        each[k] = there ? weight[k] * each[k] : 0.0f;
        mean += each[k];
    }
    if constexpr (KEPT == 0) mean = total<LANES>(mean);
    float grad[V];
    if constexpr (OVER_ALL) {
        uint32_t best = 0;
#pragma unroll
        for (int v = 0; v < V; ++v) {
            const uint32_t key = key_of(expert_of(v) < a.experts ? (float)score[v] : -__builtin_inff());
            best = key > best ? key : best;
        }
        const float most = score_of(largest<LANES>(best));
        float all = 0.0f;
#pragma unroll
        for (int v = 0; v < V; ++v) {
            const float s = (float)score[v], part = part_of(s, most);
            grad[v] = expert_of(v) < a.experts && s > -__builtin_inff() ? part : 0.0f;
            all += grad[v];
        }
        all = total<LANES>(all);
        const float by = all > 0.0f ? -mean / all : 0.0f;
#pragma unroll
        for (int v = 0; v < V; ++v) grad[v] *= by;
    } else {
#pragma unroll
        for (int v = 0; v < V; ++v) grad[v] = 0.0f;
#pragma unroll
        for (int k = 0; k < kHere; ++k) each[k] -= weight[k] * mean;
    }
    const auto give = [&](int32_t e, float d) {
#pragma unroll
        for (int v = 0; v < V; ++v) grad[v] += e == (int32_t)expert_of(v) ? d : 0.0f;
    };
    if constexpr (KEPT != 0) {
#pragma unroll
        for (int k = 0; k < KEPT; ++k) give(number[k], each[k]);
    } else {
#pragma unroll
        for (int k = 0; k < kHere; ++k)
            for (uint32_t s = 0; s < LANES && k * LANES + s < a.slots; ++s) give(__shfl(number[k], (int)s, LANES), __shfl(each[k], (int)s, LANES));
    }
    if (t >= a.tokens) return;
    T* const out = (T*)a.grad_scores + (int64_t)token * a.grad_stride;
#pragma unroll
    for (int v = 0; v < V; v += C) {
        Vec<T, C> part;
        for (int c = 0; c < C; ++c) part[c] = (T)grad[v + c];
        if (expert_of(v) < a.experts) store_vec<T, C, ALIGNED>(out + expert_of(v), part);
    }
}

template <int LANES, typename K> hipError_t go(K kernel, const RouteArgs& a, hipStream_t stream) {
    const uint64_t each = kRouteThreads / LANES;
    hipLaunchKernelGGL(kernel, long_grid((a.tokens + each - 1) / each), dim3(kRouteThreads), 0, stream, a);
    return hipGetLastError();
}
#define TPERM_BY_EXPERTS(KERNEL, ...)                                                                                \
    (a.experts <= 32    ? go<16>(KERNEL<T, 16, 2, __VA_ARGS__>, a, stream)                                           \
     : a.experts <= 64  ? go<16>(KERNEL<T, 16, 4, __VA_ARGS__>, a, stream)                                           \
     : a.experts <= 128 ? go<16>(KERNEL<T, 16, 8, __VA_ARGS__>, a, stream)                                           \
     : a.experts <= 256 ? go<64>(KERNEL<T, 64, 4, __VA_ARGS__>, a, stream)                                           \
                        : go<64>(KERNEL<T, 64, 16, __VA_ARGS__>, a, stream))
// Few lanes to a token do the fewest operations, more of them answer sooner where there are few tokens.
template <typename T, int P, bool ALIGNED> hipError_t few_slots(const RouteArgs& a, bool over_all, hipStream_t stream) {
    const auto with = [&](auto kernel, uint32_t lanes) {
        const uint64_t each = kRouteThreads / lanes;
        hipLaunchKernelGGL(kernel, long_grid((a.tokens + each - 1) / each), dim3(kRouteThreads), 0, stream, a, over_all);
        return hipGetLastError();
    };
    const bool many = a.tokens >= 8192;
    if (many && a.experts <= 32) return with(route_few_kernel<T, 4, 8, P, ALIGNED>, 4);
    if (many && a.experts <= 64) return with(route_few_kernel<T, 4, 16, P, ALIGNED>, 4);
    if (many && a.experts <= 128) return with(route_few_kernel<T, 4, 32, P, ALIGNED>, 4);
    return a.experts <= 128 ? with(route_few_kernel<T, 16, 8, P, ALIGNED>, 16) : a.experts <= 256 ? with(route_few_kernel<T, 16, 16, P, ALIGNED>, 16)
           : a.experts <= 512 ? with(route_few_kernel<T, 16, 32, P, ALIGNED>, 16) : with(route_few_kernel<T, 64, 16, P, ALIGNED>, 64);
}
template <typename T, bool OVER_ALL> hipError_t route_of(const RouteArgs& a, hipStream_t stream) {
    const bool aligned = ((uintptr_t)a.scores | (uintptr_t)a.scores_stride * sizeof(T)) % 16 == 0 && a.experts * sizeof(T) % 16 == 0;
    if (a.slots <= 4) return aligned ? few_slots<T, 4, true>(a, OVER_ALL, stream) : few_slots<T, 4, false>(a, OVER_ALL, stream);
    if (a.slots <= 8) return aligned ? few_slots<T, 8, true>(a, OVER_ALL, stream) : few_slots<T, 8, false>(a, OVER_ALL, stream);
    return TPERM_BY_EXPERTS(route_kernel, OVER_ALL);
}
#define TPERM_BACKWARD(LANES, V) go<LANES>(route_backward_kernel<T, LANES, V, KEPT, OVER_ALL, ALIGNED>, a, stream)
template <typename T, bool OVER_ALL, int KEPT, bool ALIGNED> hipError_t backward_by_experts(const RouteArgs& a, hipStream_t stream) {
    if constexpr (KEPT != 0) {
        if (a.experts <= 32) return TPERM_BACKWARD(4, 8);
        if (a.experts <= 64) return TPERM_BACKWARD(8, 8);
    }
    return a.experts <= 128 ? TPERM_BACKWARD(16, 8) : a.experts <= 512 ? TPERM_BACKWARD(64, 8) : TPERM_BACKWARD(64, 16);
}
template <typename T, bool OVER_ALL, bool ALIGNED> hipError_t backward_of(const RouteArgs& a, hipStream_t stream) {
    return a.slots <= 4 ? backward_by_experts<T, OVER_ALL, 4, ALIGNED>(a, stream) : a.slots <= 8 ? backward_by_experts<T, OVER_ALL, 8, ALIGNED>(a, stream)
                                                                                                 : backward_by_experts<T, OVER_ALL, 0, ALIGNED>(a, stream);
}
template <typename T, bool OVER_ALL> hipError_t backward_of(const RouteArgs& a, hipStream_t stream) {
    const auto on_16 = [](const void* p, int64_t stride) { return ((uintptr_t)p | (uintptr_t)stride * sizeof(T)) % 16 == 0; };
    const bool aligned = a.experts * sizeof(T) % 16 == 0 && on_16(a.grad_scores, a.grad_stride) && (!OVER_ALL || on_16(a.scores, a.scores_stride));
    return aligned ? backward_of<T, OVER_ALL, true>(a, stream) : backward_of<T, OVER_ALL, false>(a, stream);
}

}  // namespace

hipError_t launch_route(const RouteArgs& a, bool over_all, int type, hipStream_t stream) {
    return with_type(type, [&](auto t) { return over_all ? route_of<decltype(t), true>(a, stream) : route_of<decltype(t), false>(a, stream); });
}
hipError_t launch_route_backward(const RouteArgs& a, bool over_all, int type, hipStream_t stream) {
    return with_type(type, [&](auto t) { return over_all ? backward_of<decltype(t), true>(a, stream) : backward_of<decltype(t), false>(a, stream); });
}

}  // namespace tperm
