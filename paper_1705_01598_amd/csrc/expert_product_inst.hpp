// Choice and launch of the experts' product kernels for one element type; included once for each.
#pragma once
#include "expert_product.hpp"

namespace tperm {

using WideTile = TileShape<128, 128, 2>;

template <typename T> hipError_t product_of(const ExpertProductArgs& a, bool w_k_first, hipStream_t stream) {
    using S = WideTile;
    const uint64_t tiles = ((uint64_t)a.rows / S::kSlow + a.experts + 1) * ((a.n + S::kFast - 1) / S::kFast);
    if (w_k_first) hipLaunchKernelGGL((expert_product_kernel<T, kDepthFast, S>), long_grid(tiles), dim3(S::kThreads), 0, stream, a);
    else hipLaunchKernelGGL((expert_product_kernel<T, kFreeFast, S>), long_grid(tiles), dim3(S::kThreads), 0, stream, a);
    return hipGetLastError();
}

template <typename T> hipError_t gradient_of(const WeightGradientArgs& a, hipStream_t stream) {
    using S = WideTile;
    const uint64_t tiles = (uint64_t)a.experts * ((a.fast.width + S::kFast - 1) / S::kFast) * ((a.slow.width + S::kSlow - 1) / S::kSlow);
    const auto go = [&](auto kernel) {
        hipLaunchKernelGGL(kernel, long_grid(tiles), dim3(S::kThreads), 0, stream, a);
        return hipGetLastError();
    };
    if (a.fast.scales != nullptr) return go(weight_gradient_kernel<T, kCodes, kFreeFast, S>);
    if (a.slow.scales != nullptr) return go(weight_gradient_kernel<T, kFreeFast, kCodes, S>);
    return go(weight_gradient_kernel<T, kFreeFast, kFreeFast, S>);
}

}  // namespace tperm
