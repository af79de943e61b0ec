// Rows gathered to their experts, combined back to their tokens, and the gradients of that.
//
// Pure data movement with a few operations an element: HBM is the bound.  A row is walked by a group of
// lanes, 16 bytes a lane and step; narrow rows take narrow groups, so that a wavefront has as many rows in
// flight as it needs.  Sums are formed in binary32 in the order of the slots.
#include "experts.hpp"
#include "expert_vector.hpp"

namespace tperm {

namespace {

constexpr int kRowThreads = 256;

// LANES lanes to a row, STEPS vectors a lane: a workgroup takes kRowThreads / LANES rows and one piece of
// LANES * STEPS vectors of them.
template <typename T, int LANES, int STEPS, bool ALIGNED>
__global__ __launch_bounds__(kRowThreads) void gather_kernel(const RowsArgs a) {
    constexpr int V = 16 / sizeof(T);
    const uint64_t row = long_block() * (kRowThreads / LANES) + threadIdx.x / LANES;
    if (row >= a.count) return;
    const uint32_t col = (blockIdx.y * (LANES * STEPS) + threadIdx.x % LANES) * V;
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
        if (c < a.width) store_some<T, V, ALIGNED>(out + c, v[s], (int)(a.width - c));
    }
}

template <typename T, int LANES, int STEPS, bool ALIGNED>
__global__ __launch_bounds__(kRowThreads) void combine_kernel(const RowsArgs a) {
    constexpr int V = 16 / sizeof(T);
    const uint64_t at = long_block() * (kRowThreads / LANES) + threadIdx.x / LANES;
    if (at >= a.tokens) return;
    const uint32_t token = (uint32_t)at;
    const uint32_t col = (blockIdx.y * (LANES * STEPS) + threadIdx.x % LANES) * V;
    const uint32_t end = (uint32_t)*a.used < a.count ? (uint32_t)*a.used : a.count;
    Vec<float, V> sum[STEPS] = {};
    const uint32_t first = token * a.slots;
    constexpr int kAhead = 4;       // slots whose rows are requested at once
    for (uint32_t s0 = 0; s0 < a.slots; s0 += kAhead) {
        Vec<T, V> v[kAhead][STEPS];
        float w[kAhead];
        bool used[kAhead];
#pragma unroll
        for (int i = 0; i < kAhead; ++i) {
            used[i] = false;
            if (s0 + i < a.slots) {
                const uint32_t row = (uint32_t)a.map[first + s0 + i];
                used[i] = row < end;
                w[i] = a.weights != nullptr ? a.weights[first + s0 + i] : 1.0f;
                if (used[i]) {
                    const T* const p = (const T*)a.in + (int64_t)row * a.in_stride;
#pragma unroll
                    for (int s = 0; s < STEPS; ++s) {
                        const uint32_t c = col + s * LANES * V;
                        if (c < a.width) v[i][s] = load_some<T, V, ALIGNED>(p + c, (int)(a.width - c));
                    }
                }
            }
        }
#pragma unroll
        for (int i = 0; i < kAhead; ++i)
            if (used[i]) {
#pragma unroll
                for (int s = 0; s < STEPS; ++s) sum[s] += widen<T, V>(v[i][s]) * w[i];
            }
    }
    T* const out = (T*)a.out + (int64_t)token * a.out_stride;
#pragma unroll
    for (int s = 0; s < STEPS; ++s) {
        const uint32_t c = col + s * LANES * V;
        if (c < a.width) store_some<T, V, ALIGNED>(out + c, narrow<T, V>(sum[s]), (int)(a.width - c));
    }
}

// One group of LANES lanes (up to the whole workgroup) to a token: its gradient is read once for a batch of slots.
template <typename T, int LANES, bool ALIGNED>
__global__ __launch_bounds__(kRowThreads) void combine_backward_kernel(const RowsArgs a) {
    constexpr int V = 16 / sizeof(T), kBatch = 8;
    constexpr int kWaves = LANES > 64 ? LANES / 64 : 1;
    __shared__ float part[kWaves][kBatch];
    const uint64_t at = long_block() * (kRowThreads / LANES) + threadIdx.x / LANES;
    if (at >= a.tokens) return;      // whole wavefronts or whole groups of lanes; with LANES > 64 whole workgroups
    const uint32_t token = (uint32_t)at;
    const uint32_t lane = threadIdx.x % LANES;
    const uint32_t end = (uint32_t)*a.used < a.count ? (uint32_t)*a.used : a.count;
    const T* const grad = (const T*)a.in + (int64_t)token * a.in_stride;
    for (uint32_t s0 = 0; s0 < a.slots; s0 += kBatch) {
        uint32_t row[kBatch];
        float w[kBatch], dot[kBatch];
#pragma unroll
        for (int i = 0; i < kBatch; ++i) {
            const uint32_t k = token * a.slots + s0 + i;
            row[i] = s0 + i < a.slots ? (uint32_t)a.map[k] : 0xFFFFFFFFu;
            w[i] = s0 + i < a.slots ? a.weights[k] : 0.0f;
            dot[i] = 0.0f;
        }
        for (uint32_t c = lane * V; c < a.width; c += LANES * V) {
            const int there = (int)(a.width - c);
            Vec<T, V> v[kBatch];
            const Vec<float, V> g = widen<T, V>(load_some<T, V, ALIGNED>(grad + c, there));
#pragma unroll
            for (int i = 0; i < kBatch; ++i)
                if (row[i] < end) v[i] = load_some<T, V, ALIGNED>((const T*)a.rows + (int64_t)row[i] * a.rows_stride + c, there);
#pragma unroll
            for (int i = 0; i < kBatch; ++i) {
                if (row[i] >= a.count) continue;
                Vec<float, V> d = {};
                if (row[i] < end) {
                    const Vec<float, V> r = widen<T, V>(v[i]);
#pragma unroll
                    for (int j = 0; j < V; ++j) dot[i] += g[j] * r[j];
                    d = g * w[i];
                }
                store_some<T, V, ALIGNED>((T*)a.out + (int64_t)row[i] * a.out_stride + c, narrow<T, V>(d), there);
            }
        }
#pragma unroll
        for (int i = 0; i < kBatch; ++i)
#pragma unroll
            for (int d = 1; d < (LANES < 64 ? LANES : 64); d <<= 1) dot[i] += __shfl_xor(dot[i], d);
        if constexpr (LANES > 64) {
            __syncthreads();
            if (threadIdx.x % 64 == 0)
#pragma unroll
                for (int i = 0; i < kBatch; ++i) part[threadIdx.x / 64][i] = dot[i];
            __syncthreads();
#pragma unroll
            for (int i = 0; i < kBatch; ++i) {
                dot[i] = part[0][i];
#pragma unroll
                for (int k = 1; k < kWaves; ++k) dot[i] += part[k][i];
            }
        }
        if (lane == 0)
#pragma unroll
            for (int i = 0; i < kBatch; ++i)
                if (s0 + i < a.slots) a.grad_weights[token * a.slots + s0 + i] = dot[i];
    }
}

// Rows start on 16 bytes and are whole vectors.
bool on_vectors(size_t elem, uint32_t width, const void* p, int64_t stride) {
    return (width * elem) % 16 == 0 && ((uintptr_t)p | (uintptr_t)stride * elem) % 16 == 0;
}

template <int LANES> dim3 grid_of(uint32_t rows, uint32_t vectors, uint32_t steps) {
    const uint32_t per = kRowThreads / LANES;
    return long_grid(((uint64_t)rows + per - 1) / per, (vectors + LANES * steps - 1) / (LANES * steps));
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
        if (vectors <= 8) return aligned ? go(gather_kernel<T, 4, 2, true>, grid_of<4>(a.count, vectors, 2)) : go(gather_kernel<T, 4, 2, false>, grid_of<4>(a.count, vectors, 2));
        if (vectors <= 64) return aligned ? go(gather_kernel<T, 16, 4, true>, grid_of<16>(a.count, vectors, 4)) : go(gather_kernel<T, 16, 4, false>, grid_of<16>(a.count, vectors, 4));
        return aligned ? go(gather_kernel<T, 64, 4, true>, grid_of<64>(a.count, vectors, 4)) : go(gather_kernel<T, 64, 4, false>, grid_of<64>(a.count, vectors, 4));
    });
}

hipError_t launch_expert_combine(RowsArgs a, int type, hipStream_t stream) {
    return with_type(type, [&](auto t) {
        using T = decltype(t);
        const uint32_t vectors = (a.width * (uint32_t)sizeof(T) + 15) / 16;
        const bool aligned = on_vectors(sizeof(T), a.width, a.in, a.in_stride) && on_vectors(sizeof(T), a.width, a.out, a.out_stride);
        const auto go = [&](auto kernel, dim3 grid) {
            hipLaunchKernelGGL(kernel, grid, dim3(kRowThreads), 0, stream, a);
            return hipGetLastError();
        };
        if (vectors <= 4) return aligned ? go(combine_kernel<T, 4, 1, true>, grid_of<4>(a.tokens, vectors, 1)) : go(combine_kernel<T, 4, 1, false>, grid_of<4>(a.tokens, vectors, 1));
        if (vectors <= 32) return aligned ? go(combine_kernel<T, 16, 2, true>, grid_of<16>(a.tokens, vectors, 2)) : go(combine_kernel<T, 16, 2, false>, grid_of<16>(a.tokens, vectors, 2));
        return aligned ? go(combine_kernel<T, 64, 2, true>, grid_of<64>(a.tokens, vectors, 2)) : go(combine_kernel<T, 64, 2, false>, grid_of<64>(a.tokens, vectors, 2));
    });
}

hipError_t launch_expert_combine_backward(RowsArgs a, int type, hipStream_t stream) {
    return with_type(type, [&](auto t) {
        using T = decltype(t);
        const uint32_t vectors = (a.width * (uint32_t)sizeof(T) + 15) / 16;
        const bool aligned = on_vectors(sizeof(T), a.width, a.in, a.in_stride) && on_vectors(sizeof(T), a.width, a.out, a.out_stride) &&
                             on_vectors(sizeof(T), a.width, a.rows, a.rows_stride);
        const auto go = [&](auto kernel, uint32_t lanes) {
            const uint32_t per = kRowThreads / lanes;
            hipLaunchKernelGGL(kernel, long_grid(((uint64_t)a.tokens + per - 1) / per), dim3(kRowThreads), 0, stream, a);
            return hipGetLastError();
        };
        if (vectors <= 16) return aligned ? go(combine_backward_kernel<T, 16, true>, 16) : go(combine_backward_kernel<T, 16, false>, 16);
        if (vectors <= 128) return aligned ? go(combine_backward_kernel<T, 64, true>, 64) : go(combine_backward_kernel<T, 64, false>, 64);
        return aligned ? go(combine_backward_kernel<T, 256, true>, 256) : go(combine_backward_kernel<T, 256, false>, 256);
    });
}

}  // namespace tperm
