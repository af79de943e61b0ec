// Choice and launch of the experts' product kernels for one element type; included once for each.
#pragma once
#include <atomic>

#include "expert_product.hpp"

namespace tperm {

// The tiles of Tile.
using TinyTile = TileShape<64, 64, 4, 2, 2>;
using SmallTile = TileShape<128, 128, 4, 2>;
using NarrowTile = TileShape<128, 64, 4, 2>;    // 32-bit elements, which the matrix cores bound: finer rounds of tiles
using WideTile = TileShape<256, 256, 8, 4>;     // 64 x 128 results to a wavefront: fewer transposing reads than 128 x 64 of a free-fast matrix

template <typename S> constexpr bool is(Tile t) { return S::kFast == kTileFast[(int)t] && S::kSlow == kTileSlow[(int)t]; }
static_assert(is<TinyTile>(Tile::kTiny) && is<SmallTile>(Tile::kSmall) && is<NarrowTile>(Tile::kNarrow) && is<WideTile>(Tile::kWide), "as the query says");

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

template <auto KERNEL, typename S, typename A> hipError_t go(uint64_t blocks, const A& a, hipStream_t stream) {
    constexpr size_t kLds = S::kLds;
    if constexpr (kLds > 64 * 1024) {
        const hipError_t e = allow_lds<KERNEL>(kLds);
        if (e != hipSuccess) return e;
    }
    hipLaunchKernelGGL(KERNEL, long_grid(blocks), dim3(S::kAllThreads), kLds, stream, a);
    return hipGetLastError();
}

// Rows of whole chunks that start on 16 bytes; offsets inside a tile's rows fit 32 bits.
inline bool on_chunks(size_t elem, const void* p, int64_t stride, uint32_t width) {
    return width * elem % 16 == 0 && ((uintptr_t)p | (uintptr_t)stride * elem) % 16 == 0 && stride < (int64_t)1 << 22;
}

template <typename T, typename S, bool LOOSE> hipError_t product_tiles(const ExpertProductArgs& a, bool w_k_first, hipStream_t stream) {
    const uint64_t tiles = ((uint64_t)a.rows / S::kSlow + a.experts + 1) * over(a.n, S::kFast), blocks = over(tiles, kXcds) * kXcds;
    return w_k_first ? go<expert_product_kernel<T, kDepthFast, S, LOOSE>, S>(blocks, a, stream) : go<expert_product_kernel<T, kFreeFast, S, LOOSE>, S>(blocks, a, stream);
}

template <typename T, bool LOOSE> hipError_t product_with(const ExpertProductArgs& a, bool w_k_first, hipStream_t stream) {
    const Tile tile = product_tile(sizeof(T), a.rows, a.experts, a.n);
    if constexpr (sizeof(T) == 2) {
        if (tile == Tile::kWide) return product_tiles<T, WideTile, LOOSE>(a, w_k_first, stream);
        if (tile == Tile::kSmall) return product_tiles<T, SmallTile, LOOSE>(a, w_k_first, stream);
    } else {
        if (tile == Tile::kNarrow) return product_tiles<T, NarrowTile, LOOSE>(a, w_k_first, stream);
    }
    return product_tiles<T, TinyTile, LOOSE>(a, w_k_first, stream);
}

template <typename T> hipError_t product_of(const ExpertProductArgs& a, bool w_k_first, hipStream_t stream) {
    const bool whole = on_chunks(sizeof(T), a.x.p, a.x.stride, a.k) && on_chunks(sizeof(T), a.w, w_k_first ? a.k : a.n, w_k_first ? a.k : a.n);
    return whole ? product_with<T, false>(a, w_k_first, stream) : product_with<T, true>(a, w_k_first, stream);
}

template <typename T, typename S, bool LOOSE> hipError_t gradient_tiles(const WeightGradientArgs& a, hipStream_t stream) {
    const uint64_t blocks = over(over(a.fast.width, S::kFast) * over(a.slow.width, S::kSlow), kXcds) * kXcds * a.experts;
    if (a.fast.scales != nullptr)
        return a.fast.source != nullptr ? go<weight_gradient_kernel<T, kCodes, kFreeFast, true, false, S, LOOSE>, S>(blocks, a, stream)
                                        : go<weight_gradient_kernel<T, kCodes, kFreeFast, false, false, S, LOOSE>, S>(blocks, a, stream);
    if (a.slow.scales != nullptr)
        return a.slow.source != nullptr ? go<weight_gradient_kernel<T, kFreeFast, kCodes, false, true, S, LOOSE>, S>(blocks, a, stream)
                                        : go<weight_gradient_kernel<T, kFreeFast, kCodes, false, false, S, LOOSE>, S>(blocks, a, stream);
    if constexpr (!LOOSE) {
        if (a.fast.source != nullptr) return go<weight_gradient_kernel<T, kFreeFast, kFreeFast, true, false, S, false>, S>(blocks, a, stream);
        if (a.slow.source != nullptr) return go<weight_gradient_kernel<T, kFreeFast, kFreeFast, false, true, S, false>, S>(blocks, a, stream);
    }
    return go<weight_gradient_kernel<T, kFreeFast, kFreeFast, false, false, S, LOOSE>, S>(blocks, a, stream);
}

template <typename T, bool LOOSE> hipError_t gradient_with(const WeightGradientArgs& a, hipStream_t stream) {
    const Tile tile = gradient_tile(sizeof(T), a.fast.width, a.slow.width, a.experts);
    if constexpr (sizeof(T) == 2) {
        if (tile == Tile::kWide) return gradient_tiles<T, WideTile, LOOSE>(a, stream);
        if (tile == Tile::kSmall) return gradient_tiles<T, SmallTile, LOOSE>(a, stream);
    } else {
        if (tile == Tile::kNarrow) return gradient_tiles<T, NarrowTile, LOOSE>(a, stream);
    }
    return gradient_tiles<T, TinyTile, LOOSE>(a, stream);
}

template <typename T> hipError_t gradient_of(const WeightGradientArgs& a, hipStream_t stream) {
    const auto fits = [](const ProductSide& s) { return s.scales != nullptr ? on_chunks(1, s.p, s.width, s.width) : on_chunks(sizeof(T), s.p, s.stride, s.width); };
    return fits(a.fast) && fits(a.slow) ? gradient_with<T, false>(a, stream) : gradient_with<T, true>(a, stream);
}

}  // namespace tperm
