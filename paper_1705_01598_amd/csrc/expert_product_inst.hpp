// Choice and launch of the experts' product kernels for one element type; included once for each.
#pragma once
#include <atomic>

#include "expert_product.hpp"

namespace tperm {

using SmallTile = TileShape<128, 128, 4, 2>;
using WideTile = TileShape<256, 256, 8, 4>;     // 64 x 128 results to a wavefront: fewer transposing reads than 128 x 64 of a free-fast matrix

template <typename S> constexpr size_t lds_bytes(bool direct) { return (size_t)(S::kFast + S::kSlow) * kStageBytes * (direct ? 2 : 1); }

// Workgroups with more than 64 KiB of LDS have to be allowed it, once on each device.
template <auto KERNEL> hipError_t allow_lds(size_t bytes) {
    static std::atomic<uint64_t> done{0};
    int device = 0;
    hipError_t e = hipGetDevice(&device);
    if (e != hipSuccess) return e;
    const uint64_t bit = 1ull << (device & 63);
    if (done.load(std::memory_order_acquire) & bit) return hipSuccess;
    e = hipFuncSetAttribute((const void*)KERNEL, hipFuncAttributeMaxDynamicSharedMemorySize, (int)bytes);
    if (e == hipSuccess) done.fetch_or(bit, std::memory_order_release);
    return e;
}

template <auto KERNEL, typename S, bool DIRECT, typename A> hipError_t go(uint64_t blocks, const A& a, hipStream_t stream) {
    constexpr size_t kLds = lds_bytes<S>(DIRECT);
    if constexpr (kLds > 64 * 1024) {
        const hipError_t e = allow_lds<KERNEL>(kLds);
        if (e != hipSuccess) return e;
    }
    hipLaunchKernelGGL(KERNEL, long_grid(blocks), dim3(S::kThreads), kLds, stream, a);
    return hipGetLastError();
}

// Rows of whole chunks that start on 16 bytes; offsets inside a tile's rows fit 32 bits.
inline bool on_chunks(size_t elem, const void* p, int64_t stride, uint32_t width) {
    return width * elem % 16 == 0 && ((uintptr_t)p | (uintptr_t)stride * elem) % 16 == 0 && stride < (int64_t)1 << 22;
}

template <typename T, typename S, bool DIRECT> hipError_t product_tiles(const ExpertProductArgs& a, bool w_k_first, hipStream_t stream) {
    const uint64_t tiles = ((uint64_t)a.rows / S::kSlow + a.experts + 1) * ((a.n + S::kFast - 1) / S::kFast);
    const uint64_t blocks = (tiles + kXcds - 1) / kXcds * kXcds;
    return w_k_first ? go<expert_product_kernel<T, kDepthFast, S, DIRECT>, S, DIRECT>(blocks, a, stream)
                     : go<expert_product_kernel<T, kFreeFast, S, DIRECT>, S, DIRECT>(blocks, a, stream);
}

template <typename T> hipError_t product_of(const ExpertProductArgs& a, bool w_k_first, hipStream_t stream) {
    const bool direct = on_chunks(sizeof(T), a.x.p, a.x.stride, a.k) && on_chunks(sizeof(T), a.w, w_k_first ? a.k : a.n, w_k_first ? a.k : a.n);
    if (!direct) return product_tiles<T, SmallTile, false>(a, w_k_first, stream);
    if constexpr (sizeof(T) == 2) {
        if (a.rows >= 128 * a.experts) return product_tiles<T, WideTile, true>(a, w_k_first, stream);
    }
    return product_tiles<T, SmallTile, true>(a, w_k_first, stream);
}

template <typename T, typename S, bool DIRECT> hipError_t gradient_tiles(const WeightGradientArgs& a, hipStream_t stream) {
    const uint64_t tiles = (uint64_t)((a.fast.width + S::kFast - 1) / S::kFast) * ((a.slow.width + S::kSlow - 1) / S::kSlow);
    const uint64_t blocks = (tiles + kXcds - 1) / kXcds * kXcds * a.experts;
    if constexpr (DIRECT) {
        if (a.fast.scales != nullptr) return go<weight_gradient_kernel<T, kCodes, kFreeFast, false, false, S, true>, S, true>(blocks, a, stream);
        if (a.slow.scales != nullptr) return go<weight_gradient_kernel<T, kFreeFast, kCodes, false, false, S, true>, S, true>(blocks, a, stream);
        if (a.fast.source != nullptr) return go<weight_gradient_kernel<T, kFreeFast, kFreeFast, true, false, S, true>, S, true>(blocks, a, stream);
        if (a.slow.source != nullptr) return go<weight_gradient_kernel<T, kFreeFast, kFreeFast, false, true, S, true>, S, true>(blocks, a, stream);
        return go<weight_gradient_kernel<T, kFreeFast, kFreeFast, false, false, S, true>, S, true>(blocks, a, stream);
    } else {
        if (a.fast.scales != nullptr) return go<weight_gradient_kernel<T, kCodes, kFreeFast, false, false, S, false>, S, false>(blocks, a, stream);
        if (a.slow.scales != nullptr) return go<weight_gradient_kernel<T, kFreeFast, kCodes, false, false, S, false>, S, false>(blocks, a, stream);
        return go<weight_gradient_kernel<T, kFreeFast, kFreeFast, false, false, S, false>, S, false>(blocks, a, stream);
    }
}

template <typename T> hipError_t gradient_of(const WeightGradientArgs& a, hipStream_t stream) {
    const auto fits = [](const ProductSide& s) { return s.scales != nullptr ? on_chunks(1, s.p, s.width, s.width) : on_chunks(sizeof(T), s.p, s.stride, s.width); };
    const bool direct = fits(a.fast) && fits(a.slow);
    if (!direct) return gradient_tiles<T, SmallTile, false>(a, stream);
    if constexpr (sizeof(T) == 2) {
        if ((uint64_t)a.fast.width * a.slow.width * a.experts >= 256ull * 256 * 256) return gradient_tiles<T, WideTile, true>(a, stream);
    }
    return gradient_tiles<T, SmallTile, true>(a, stream);
}

}  // namespace tperm
