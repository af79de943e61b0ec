// Rows gathered to their experts, combined back to their tokens, and the gradients of that.
//
// Pure data movement with a few operations an element: HBM is the bound.  A row is walked by a group of
// lanes, 16 bytes a lane and step; narrow rows take narrow groups, so that a wavefront has as many rows in
// flight as it needs.  Sums are formed in binary32 in the order of the slots.
//
// Results are stored past the caches (rows of 4 KiB: gather of 16384 x 2 50 -> 39 us, combine 39 -> 37, backward of 2048 x 4
// rows of 8 KiB 34 -> 25); rows are read past them too (ONCE) where they fill a third of the memory-side cache (combine and
// backward of 16384 x 2 37 -> 34 and 63 -> 55 us, of 12288 x 2 26 -> 26 and 48 -> 42), while smaller ones may still be
// there from the product that wrote them (6144 x 2 13 -> 14 and 21 -> 24).
// Rows of 4 KiB now: combine of 8192 x 8 50 us, 5.9 TB/s, its backward 105 us, 5.4 TB/s, both near what a copy
// reaches (6.1); gather 74 us, 4.1 TB/s, where a token's row is read eight times, from the memory-side cache.
#include <type_traits>

#include "experts.hpp"
#include "expert_vector.hpp"
#include "plan.hpp"

namespace tperm {

namespace {

constexpr int kRowThreads = 256;

// Which row (or token) a group of LANES lanes works on, and which piece of it: the pieces of a row side by side,
// so that a row is read and written at once (combine, rows of 4 KiB, against all first pieces before all second ones:
// 8192 x 8 67 -> 51 us, 16384 x 2 46 -> 37 us).
template <int LANES> __device__ __forceinline__ uint64_t row_of_group(const RowsArgs& a, uint32_t* piece) {
    const uint64_t at = long_block() * (kRowThreads / LANES) + threadIdx.x / LANES;
    const uint64_t row = a.by_pieces.magic != 0 ? fdiv((uint32_t)at, a.by_pieces) : at / a.pieces;
    *piece = (uint32_t)(at - row * a.pieces);
    return row;
}

// LANES lanes to a piece of a row, STEPS vectors a lane.
template <typename T, int LANES, int STEPS, bool ALIGNED>
__global__ __launch_bounds__(kRowThreads) void gather_kernel(const RowsArgs a) {
    constexpr int V = 16 / sizeof(T);
    uint32_t piece;
    const uint64_t row = row_of_group<LANES>(a, &piece);
    if (row >= a.count) return;
    const uint32_t col = (piece * (LANES * STEPS) + threadIdx.x % LANES) * V;
    const uint32_t from = (uint32_t)a.map[row];
    const bool used = row < (uint32_t)*a.used && from < a.count;
    const T* const x = (const T*)a.in + (int64_t)(used ? from / a.slots : 0u) * a.in_stride;
    T* const out = (T*)a.out + (int64_t)row * a.out_stride;
    Vec<T, V> v[STEPS];
    if (used) {
#pragma unroll
        for (int s = 0; s < STEPS; ++s) {
            const uint32_t c = col + s * LANES * V;
            if (c < a.width) v[s] = load_some<T, V, ALIGNED>(x + c, (int)(a.width - c));
        }
        if (a.weights != nullptr) {
            const float w = a.weights[from];
#pragma unroll
            for (int s = 0; s < STEPS; ++s) v[s] = narrow<T, V>(widen<T, V>(v[s]) * w);
        }
    } else {
#pragma unroll
        for (int s = 0; s < STEPS; ++s) v[s] = Vec<T, V>{};
    }
#pragma unroll
    for (int s = 0; s < STEPS; ++s) {
        const uint32_t c = col + s * LANES * V;
        if (c < a.width) store_once<T, V, ALIGNED>(out + c, v[s], (int)(a.width - c));
    }
}

// Row of a slot, uniform where a whole wavefront works on one token: then its tests are branches of the
// wavefront and its address is a scalar.
template <int LANES> __device__ __forceinline__ uint32_t uniform(uint32_t v) {
    if constexpr (LANES >= 64) return (uint32_t)__builtin_amdgcn_readfirstlane((int)v);
    else return v;
}

// A group of LANES lanes to a token; the rows of SLOTS slots are requested at once.
template <typename T, int LANES, int SLOTS, bool ALIGNED, bool ONCE>
__global__ __launch_bounds__(kRowThreads) void combine_kernel(const RowsArgs a) {
    constexpr int V = 16 / sizeof(T);
    uint32_t piece;
    const uint64_t at = row_of_group<LANES>(a, &piece);
    if (at >= a.tokens) return;
    const uint32_t token = uniform<LANES>((uint32_t)at);
    const uint32_t col = (piece * LANES + threadIdx.x % LANES) * V;
    if (col >= a.width) return;
    const int there = (int)(a.width - col);
    const uint32_t end = (uint32_t)*a.used < a.count ? (uint32_t)*a.used : a.count;
    Vec<float, V> sum = {};
    const uint32_t first = token * a.slots;
    for (uint32_t s0 = 0; s0 < a.slots; s0 += SLOTS) {
        Vec<T, V> v[SLOTS];
        uint32_t row[SLOTS];
        float w[SLOTS];
#pragma unroll
        for (int i = 0; i < SLOTS; ++i) {
            const uint32_t k = first + (s0 + i < a.slots ? s0 + i : a.slots - 1);
            row[i] = (uint32_t)a.map[k];
            w[i] = a.weights != nullptr ? a.weights[k] : 1.0f;
        }
#pragma unroll
        for (int i = 0; i < SLOTS; ++i) {
            row[i] = s0 + i < a.slots ? uniform<LANES>(row[i]) : 0xFFFFFFFFu;
            v[i] = Vec<T, V>{};
            if (row[i] < end) {
                const T* const p = (const T*)a.in + (int64_t)row[i] * a.in_stride + col;
                v[i] = ONCE ? load_once<T, V, ALIGNED>(p, there) : load_some<T, V, ALIGNED>(p, there);
            }
        }
#pragma unroll
        for (int i = 0; i < SLOTS; ++i)
            if (row[i] < end) sum += widen<T, V>(v[i]) * w[i];      // the weight of an unused row may be anything
    }
    store_once<T, V, ALIGNED>((T*)a.out + (int64_t)token * a.out_stride + col, narrow<T, V>(sum), there);
}

// One group of LANES lanes (up to the whole workgroup) to a token: its gradient is read once for SLOTS slots.
template <typename T, int LANES, int SLOTS, bool ALIGNED, bool ONCE>
__global__ __launch_bounds__(kRowThreads) void combine_backward_kernel(const RowsArgs a) {
    constexpr int V = 16 / sizeof(T);
    constexpr int kWaves = LANES > 64 ? LANES / 64 : 1;
    __shared__ float part[kWaves][SLOTS];
    const uint64_t at = long_block() * (kRowThreads / LANES) + threadIdx.x / LANES;
    if (at >= a.tokens) return;      // whole groups of lanes; with LANES > 64 whole workgroups
    const uint32_t token = uniform<LANES>((uint32_t)at);
    const uint32_t lane = threadIdx.x % LANES;
    const uint32_t end = (uint32_t)*a.used < a.count ? (uint32_t)*a.used : a.count;
    const T* const grad = (const T*)a.in + (int64_t)token * a.in_stride;
    for (uint32_t s0 = 0; s0 < a.slots; s0 += SLOTS) {
        uint32_t row[SLOTS];
        float w[SLOTS], dot[SLOTS];
#pragma unroll
        for (int i = 0; i < SLOTS; ++i) {
            const uint32_t k = token * a.slots + (s0 + i < a.slots ? s0 + i : a.slots - 1);
            row[i] = (uint32_t)a.map[k];
            w[i] = a.weights[k];
            dot[i] = 0.0f;
        }
#pragma unroll
        for (int i = 0; i < SLOTS; ++i) row[i] = s0 + i < a.slots ? uniform<LANES>(row[i]) : 0xFFFFFFFFu;
        for (uint32_t c = lane * V; c < a.width; c += LANES * V) {
            const int there = (int)(a.width - c);
            Vec<T, V> v[SLOTS];
            const Vec<T, V> g16 = load_some<T, V, ALIGNED>(grad + c, there);
#pragma unroll
            for (int i = 0; i < SLOTS; ++i) {
                v[i] = Vec<T, V>{};
                if (row[i] < end) {
                    const T* const p = (const T*)a.rows + (int64_t)row[i] * a.rows_stride + c;
                    v[i] = ONCE ? load_once<T, V, ALIGNED>(p, there) : load_some<T, V, ALIGNED>(p, there);
                }
            }
            const Vec<float, V> g = widen<T, V>(g16);
#pragma unroll
            for (int i = 0; i < SLOTS; ++i)
                if (row[i] < a.count) {
                    Vec<float, V> d = {};
                    if (row[i] < end) d = g * w[i];
                    store_once<T, V, ALIGNED>((T*)a.out + (int64_t)row[i] * a.out_stride + c, narrow<T, V>(d), there);
                }
#pragma unroll
            for (int i = 0; i < SLOTS; ++i)
                if (row[i] < end) {
                    const Vec<float, V> r = widen<T, V>(v[i]);
#pragma unroll
                    for (int j = 0; j < V; ++j) dot[i] += g[j] * r[j];
                }
        }
#pragma unroll
        for (int i = 0; i < SLOTS; ++i)
#pragma unroll
            for (int d = 1; d < (LANES < 64 ? LANES : 64); d <<= 1) dot[i] += __shfl_xor(dot[i], d);
        if constexpr (LANES > 64) {
            __syncthreads();
            if (threadIdx.x % 64 == 0)
#pragma unroll
                for (int i = 0; i < SLOTS; ++i) part[threadIdx.x / 64][i] = dot[i];
            __syncthreads();
#pragma unroll
            for (int i = 0; i < SLOTS; ++i) {
                dot[i] = part[0][i];
#pragma unroll
                for (int k = 1; k < kWaves; ++k) dot[i] += part[k][i];
            }
        }
        if (lane == 0)
#pragma unroll
            for (int i = 0; i < SLOTS; ++i)
                if (s0 + i < a.slots) a.grad_weights[token * a.slots + s0 + i] = dot[i];
    }
}

// Rows start on 16 bytes and are whole vectors.
bool on_vectors(size_t elem, uint32_t width, const void* p, int64_t stride) {
    return (width * elem) % 16 == 0 && ((uintptr_t)p | (uintptr_t)stride * elem) % 16 == 0;
}

// Grid for rows in pieces of LANES * steps vectors.
template <int LANES> dim3 grid_of(RowsArgs* a, uint32_t rows, uint32_t vectors, uint32_t steps) {
    constexpr uint32_t kPer = kRowThreads / LANES;
    a->pieces = (vectors + LANES * steps - 1) / (LANES * steps);
    const uint64_t blocks = ((uint64_t)rows * a->pieces + kPer - 1) / kPer;
    a->by_pieces = blocks * kPer < 1ull << 31 ? make_fastdiv(a->pieces) : FastDiv{0, 0};
    return long_grid(blocks);
}

}  // namespace

hipError_t launch_expert_gather(RowsArgs a, int type, hipStream_t stream) {
    return with_type(type, [&](auto t) {
        using T = decltype(t);
        const uint32_t vectors = (a.width * (uint32_t)sizeof(T) + 15) / 16;
        const bool aligned = on_vectors(sizeof(T), a.width, a.in, a.in_stride) && on_vectors(sizeof(T), a.width, a.out, a.out_stride);
        const auto go = [&](auto kernel, dim3 grid) {
            hipLaunchKernelGGL(kernel, grid, dim3(kRowThreads), 0, stream, a);
            return hipGetLastError();
        };
        if (vectors <= 8) return aligned ? go(gather_kernel<T, 4, 2, true>, grid_of<4>(&a, a.count, vectors, 2)) : go(gather_kernel<T, 4, 2, false>, grid_of<4>(&a, a.count, vectors, 2));
        if (vectors <= 64) return aligned ? go(gather_kernel<T, 16, 4, true>, grid_of<16>(&a, a.count, vectors, 4)) : go(gather_kernel<T, 16, 4, false>, grid_of<16>(&a, a.count, vectors, 4));
        return aligned ? go(gather_kernel<T, 64, 4, true>, grid_of<64>(&a, a.count, vectors, 4)) : go(gather_kernel<T, 64, 4, false>, grid_of<64>(&a, a.count, vectors, 4));
    });
}

namespace {

// Calls f with the number of slots whose rows are requested at once.
template <typename F> hipError_t with_slots(uint32_t slots, F f) {
    return slots <= 1 ? f(std::integral_constant<int, 1>()) : slots <= 2 ? f(std::integral_constant<int, 2>()) : slots <= 4 ? f(std::integral_constant<int, 4>())
                                                                                                                    : f(std::integral_constant<int, 8>());
}

// Rows of more than a third of the 256 MiB memory-side cache.
bool read_once(const RowsArgs& a, size_t elem) { return (uint64_t)a.count * a.width * elem * 3 > 256u << 20; }

}  // namespace

hipError_t launch_expert_combine(RowsArgs a, int type, hipStream_t stream) {
    return with_type(type, [&](auto t) {
        // eight slots at once are no faster (51 us either way with 8192 x 8 rows of 4 KiB)
        return with_slots(a.slots < 4 ? a.slots : 4, [&](auto slots) {
            using T = decltype(t);
            constexpr int N = decltype(slots)::value;
            const uint32_t vectors = (a.width * (uint32_t)sizeof(T) + 15) / 16;
            const bool aligned = on_vectors(sizeof(T), a.width, a.in, a.in_stride) && on_vectors(sizeof(T), a.width, a.out, a.out_stride);
            const auto go = [&](auto kernel, dim3 grid) {
                hipLaunchKernelGGL(kernel, grid, dim3(kRowThreads), 0, stream, a);
                return hipGetLastError();
            };
            if (vectors <= 4) return aligned ? go(combine_kernel<T, 4, N, true, false>, grid_of<4>(&a, a.tokens, vectors, 1)) : go(combine_kernel<T, 4, N, false, false>, grid_of<4>(&a, a.tokens, vectors, 1));
            if (vectors <= 32) return aligned ? go(combine_kernel<T, 16, N, true, false>, grid_of<16>(&a, a.tokens, vectors, 1)) : go(combine_kernel<T, 16, N, false, false>, grid_of<16>(&a, a.tokens, vectors, 1));
            const dim3 grid = grid_of<64>(&a, a.tokens, vectors, 1);
            return !aligned ? go(combine_kernel<T, 64, N, false, false>, grid) : read_once(a, sizeof(T)) ? go(combine_kernel<T, 64, N, true, true>, grid) : go(combine_kernel<T, 64, N, true, false>, grid);
        });
    });
}

hipError_t launch_expert_combine_backward(RowsArgs a, int type, hipStream_t stream) {
    return with_type(type, [&](auto t) {
        return with_slots(a.slots, [&](auto slots) {
            using T = decltype(t);
            constexpr int N = decltype(slots)::value;
            const uint32_t vectors = (a.width * (uint32_t)sizeof(T) + 15) / 16;
            const bool aligned = on_vectors(sizeof(T), a.width, a.in, a.in_stride) && on_vectors(sizeof(T), a.width, a.out, a.out_stride) &&
                                 on_vectors(sizeof(T), a.width, a.rows, a.rows_stride);
            const auto go = [&](auto kernel, uint32_t lanes) {
                const uint32_t per = kRowThreads / lanes;
                hipLaunchKernelGGL(kernel, long_grid(((uint64_t)a.tokens + per - 1) / per), dim3(kRowThreads), 0, stream, a);
                return hipGetLastError();
            };
            if (vectors <= 16) return aligned ? go(combine_backward_kernel<T, 16, N, true, false>, 16) : go(combine_backward_kernel<T, 16, N, false, false>, 16);
            // a workgroup to a token where its lanes have work (rows of 4 KiB: 81 -> 63 us with 16384 x 2), else a wavefront
            // (rows of 1.5 KiB: 41 -> 28 us with 9000 x 3)
            if (vectors <= 128) return aligned ? go(combine_backward_kernel<T, 64, N, true, false>, 64) : go(combine_backward_kernel<T, 64, N, false, false>, 64);
            if (aligned && read_once(a, sizeof(T))) return go(combine_backward_kernel<T, 256, N, true, true>, 256);
            return aligned ? go(combine_backward_kernel<T, 256, N, true, false>, 256) : go(combine_backward_kernel<T, 256, N, false, false>, 256);
        });
    });
}

}  // namespace tperm
