// Activations kept in 8 bits, and the gated activation that keeps its input so and takes its gradient from it.
//
// HBM is the bound: every value is read once and every result written once.  A thread takes 8 neighbours, four
// threads side by side a block of 32; the block's largest magnitude goes between them by DPP moves of whole
// bit patterns.  Scales are powers of two, so the division is exact and the only rounding is that of the code.
//
// bfloat16, 32768 rows of 2 x 2048: gated activation 90 us, 541 MB, 6.0 TB/s; its gradient 113 us, 6.0 TB/s, what a copy
// reaches.  Rows of 1170 channels, which start on 4 bytes: 56 and 68 us for 30000 of them, 5.1 TB/s.
#include "experts.hpp"
#include "expert_vector.hpp"
#include "plan.hpp"

namespace tperm {

namespace {

constexpr int kCheckpointThreads = 256;

// Maximum over four neighbouring lanes (DPP quad permutations), in all of them.
__device__ __forceinline__ uint32_t quad_max(uint32_t v) {
    uint32_t o = (uint32_t)__builtin_amdgcn_mov_dpp((int)v, 0xB1, 0xF, 0xF, true);   // 1 0 3 2
    v = v > o ? v : o;
    o = (uint32_t)__builtin_amdgcn_mov_dpp((int)v, 0x4E, 0xF, 0xF, true);            // 2 3 0 1
    return v > o ? v : o;
}

// Scale (biased) of the block that this quad of lanes holds.
__device__ __forceinline__ uint32_t block_scale(Vec<float, 8> x) {
    uint32_t m = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const uint32_t b = finite_magnitude(x[i]);
        m = m > b ? m : b;
    }
    return scale_of(quad_max(m));
}

// Where a thread works: row, first column, and how many of its 8 columns exist (none or fewer at a row's end).
struct Place {
    uint32_t row, col;
    int there;
};
__device__ __forceinline__ Place place_of(const CheckpointArgs& a) {
    const uint32_t rows = a.rows, width = a.width, per_row = (width + 31) / 32 * 4;
    const uint64_t at = long_block() * kCheckpointThreads + threadIdx.x;
    Place p;
    // a 64-bit division takes longer than the rest of a thread's arithmetic
    const uint64_t row = a.per_row.magic != 0 ? fdiv((uint32_t)at, a.per_row) : at / per_row;
    p.row = (uint32_t)row;
    p.col = (uint32_t)(at - row * per_row) * 8;
    p.there = row < rows && p.col < width ? (int)(width - p.col) : 0;
    return p;
}

// Codes and scale of one part of a row; part_scales: where the part's scales start.
template <bool ALIGNED> __device__ __forceinline__ void keep(Vec<float, 8> x, const Place& p, uint8_t* codes, uint8_t* scales) {
    const uint32_t s = block_scale(x);
    const u32x2 c = codes_of(x, s);
    Vec<uint8_t, 8> b;
    __builtin_memcpy(&b, &c, 8);
    if (p.there > 0) {
        store_once<uint8_t, 8, ALIGNED>(codes + p.col, b, p.there);
        if (p.col % 32 == 0) scales[p.col / 32] = (uint8_t)s;
    }
}

// What codes stand for, held to the range of T.
template <typename T, bool ALIGNED> __device__ __forceinline__ Vec<float, 8> kept(const Place& p, const uint8_t* codes, const uint8_t* scales) {
    const Vec<uint8_t, 8> b = load_some<uint8_t, 8, ALIGNED>(codes + p.col, p.there);
    u32x2 c;
    __builtin_memcpy(&c, &b, 8);
    return values_of<T>(c, power_of(scales[p.col / 32]));
}

template <typename T, bool ALIGNED> __global__ __launch_bounds__(kCheckpointThreads) void store_kernel(const CheckpointArgs a) {
    const Place p = place_of(a);
    Vec<float, 8> x = {};
    if (p.there > 0) x = widen<T, 8>(load_some<T, 8, ALIGNED>((const T*)a.in + (int64_t)p.row * a.in_stride + p.col, p.there));
    keep<ALIGNED>(x, p, a.codes + (int64_t)p.row * a.width, a.scales + (int64_t)p.row * ((a.width + 31) / 32));
}

template <typename T, bool ALIGNED> __global__ __launch_bounds__(kCheckpointThreads) void load_kernel(const CheckpointArgs a) {
    const Place p = place_of(a);
    if (p.there <= 0) return;
    const Vec<float, 8> x = kept<T, ALIGNED>(p, a.codes + (int64_t)p.row * a.width, a.scales + (int64_t)p.row * ((a.width + 31) / 32));
    store_once<T, 8, ALIGNED>((T*)a.out + (int64_t)p.row * a.out_stride + p.col, narrow<T, 8>(x), p.there);
}

// The sigmoid of g as p * last, and that of -g.  Below -87 it is no normal number in binary32, though its products with g and with
// larger numbers are, and the hardware's reciprocal, right to 2^-23 like its exp2, gives zero there.
struct Sigmoid {
    float p, last, other;
};
template <typename T> __device__ __forceinline__ Sigmoid sigmoid(float g) {
    constexpr float kHalf = 0x1.715476p-1f, kRest = 0x1.4ae0cp-27f;     // log2(e) / 2 and what that rounds off
    if constexpr (sizeof(T) == 4) {
        // With E = exp(-|g| / 2), r = 1 / (1 + E^2) and for negative g the last E when all else is in a product: no factor
        // leaves the normal numbers before the result does, which is right to 8.25 * 2^-23 whatever g is.
        const float a = __builtin_fminf(__builtin_fabsf(g), 256.0f), x = a * kHalf;       // an infinity would be subtracted from itself
        const float rest = __builtin_fmaf(a, kRest, __builtin_fmaf(a, kHalf, -x)), e0 = __builtin_amdgcn_exp2f(-x), e = __builtin_fmaf(e0, rest * -0.6931472f, e0);
        const float r = __builtin_amdgcn_rcpf(__builtin_fmaf(e, e, 1.0f)), low = g < 0.0f ? e : 1.0f, high = g < 0.0f ? 1.0f : e;
        return {r * low, low, r * high * high};
    } else {
        // The rounding of |g| * log2(e) / 2 adds |g| * 2^-24, and a sigmoid that is no normal number has fewer bits: results of
        // 16 bits show neither.  2^-32 / (2^-32 (1 + exp(-g))) in three operations less; of g and u in 8 bits 91 us
        // against 94 for 32768 rows of 2048 bfloat16 channels.
        const float t = __builtin_amdgcn_exp2f(g * -kHalf), p = __builtin_amdgcn_rcpf(__builtin_fmaf(t * 0x1p-32f, t, 0x1p-32f)) * 0x1p-32f;
        return {p, 1.0f, 1.0f - p};
    }
}

template <typename T, bool ALIGNED> __global__ __launch_bounds__(kCheckpointThreads) void gated_forward_kernel(const CheckpointArgs a) {
    const Place p = place_of(a);
    Vec<float, 8> g = {}, u = {};
    if (p.there > 0) {
        const T* const row = (const T*)a.in + (int64_t)p.row * a.in_stride;
        g = widen<T, 8>(load_some<T, 8, ALIGNED>(row + p.col, p.there));
        u = widen<T, 8>(load_some<T, 8, ALIGNED>(row + a.width + p.col, p.there));
        Vec<float, 8> h;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const Sigmoid s = sigmoid<T>(g[i]);
            h[i] = g[i] * s.p * u[i] * s.last;
        }
        store_once<T, 8, ALIGNED>((T*)a.out + (int64_t)p.row * a.out_stride + p.col, narrow<T, 8>(h), p.there);
    }
    if (a.codes != nullptr) {
        const uint32_t blocks = (a.width + 31) / 32;
        uint8_t* const codes = a.codes + (int64_t)p.row * 2 * a.width;
        uint8_t* const scales = a.scales + (int64_t)p.row * 2 * blocks;
        keep<ALIGNED>(g, p, codes, scales);
        keep<ALIGNED>(u, p, codes + a.width, scales + blocks);
    }
}

template <typename T, bool ALIGNED> __global__ __launch_bounds__(kCheckpointThreads) void gated_backward_kernel(const CheckpointArgs a) {
    const Place p = place_of(a);
    if (p.there <= 0) return;
    const uint32_t blocks = (a.width + 31) / 32;
    const uint8_t* const codes = a.codes + (int64_t)p.row * 2 * a.width;
    const uint8_t* const scales = a.scales + (int64_t)p.row * 2 * blocks;
    const Vec<float, 8> d = widen<T, 8>(load_some<T, 8, ALIGNED>((const T*)a.in + (int64_t)p.row * a.in_stride + p.col, p.there));
    const Vec<float, 8> g = kept<float, ALIGNED>(p, codes, scales), u = kept<float, ALIGNED>(p, codes + a.width, scales + blocks);
    Vec<float, 8> dg, du, h;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const Sigmoid s = sigmoid<T>(g[i]);
        const float silu = g[i] * s.p;
        dg[i] = s.p * (1.0f + g[i] * s.other) * u[i] * d[i] * s.last;
        du[i] = silu * d[i] * s.last;
        h[i] = silu * u[i] * s.last;
    }
    T* const grad = (T*)a.grad_gates + (int64_t)p.row * a.grad_stride + p.col;
    store_once<T, 8, ALIGNED>(grad, narrow<T, 8>(dg), p.there);
    store_once<T, 8, ALIGNED>(grad + a.width, narrow<T, 8>(du), p.there);
    if (a.out != nullptr) store_once<T, 8, ALIGNED>((T*)a.out + (int64_t)p.row * a.out_stride + p.col, narrow<T, 8>(h), p.there);
}

bool on_eight(size_t elem, const void* p, int64_t stride) { return ((uintptr_t)p | (uintptr_t)stride * elem) % (elem * 8 < 16 ? elem * 8 : 16) == 0; }

template <typename K> hipError_t go(K kernel, CheckpointArgs a, hipStream_t stream) {
    const uint32_t per_row = (a.width + 31) / 32 * 4;
    const uint64_t threads = (uint64_t)a.rows * per_row;
    a.per_row = threads < (1ull << 31) - kCheckpointThreads ? make_fastdiv(per_row) : FastDiv{0, 0};
    hipLaunchKernelGGL(kernel, long_grid((threads + kCheckpointThreads - 1) / kCheckpointThreads), dim3(kCheckpointThreads), 0, stream, a);
    return hipGetLastError();
}

}  // namespace

// Rows of whole eights that start on 16 bytes, codes on 8.
hipError_t launch_checkpoint_store(CheckpointArgs a, int type, hipStream_t stream) {
    return with_type(type, [&](auto t) {
        using T = decltype(t);
        const bool aligned = a.width % 8 == 0 && on_eight(sizeof(T), a.in, a.in_stride) && (uintptr_t)a.codes % 8 == 0;
        return aligned ? go(store_kernel<T, true>, a, stream) : go(store_kernel<T, false>, a, stream);
    });
}

hipError_t launch_checkpoint_load(CheckpointArgs a, int type, hipStream_t stream) {
    return with_type(type, [&](auto t) {
        using T = decltype(t);
        const bool aligned = a.width % 8 == 0 && on_eight(sizeof(T), a.out, a.out_stride) && (uintptr_t)a.codes % 8 == 0;
        return aligned ? go(load_kernel<T, true>, a, stream) : go(load_kernel<T, false>, a, stream);
    });
}

hipError_t launch_gated_forward(CheckpointArgs a, int type, hipStream_t stream) {
    return with_type(type, [&](auto t) {
        using T = decltype(t);
        const bool aligned = a.width % 8 == 0 && on_eight(sizeof(T), a.in, a.in_stride) && on_eight(sizeof(T), a.out, a.out_stride) && (uintptr_t)a.codes % 8 == 0;
        return aligned ? go(gated_forward_kernel<T, true>, a, stream) : go(gated_forward_kernel<T, false>, a, stream);
    });
}

hipError_t launch_gated_backward(CheckpointArgs a, int type, hipStream_t stream) {
    return with_type(type, [&](auto t) {
        using T = decltype(t);
        const bool aligned = a.width % 8 == 0 && on_eight(sizeof(T), a.in, a.in_stride) && on_eight(sizeof(T), a.out, a.out_stride) &&
                             on_eight(sizeof(T), a.grad_gates, a.grad_stride) && (uintptr_t)a.codes % 8 == 0;
        return aligned ? go(gated_backward_kernel<T, true>, a, stream) : go(gated_backward_kernel<T, false>, a, stream);
    });
}

}  // namespace tperm
