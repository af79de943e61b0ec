// Products of few rows with a matrix held in 4 bits.
#include <type_traits>

#include "decode.hpp"
#include "few.hpp"

namespace tperm {

namespace {

constexpr int kTiles = 2;               // of 16 rows of the matrix to a workgroup

template <typename T, bool ALIGNED, int M> __global__ __launch_bounds__(kFewThreads) void four_bit_product_kernel(const FourBitProductArgs a) {
    extern __shared__ f32x4 sums[];
    const uint32_t lane = threadIdx.x & 63u, wave = threadIdx.x >> 6, first = blockIdx.x * kTiles * 16, first_row = blockIdx.y * 64;
    const FourBits w = {a.codes, a.scales, (a.k + 31) / 32};
    uint32_t row[kTiles];
    for (int r = 0; r < kTiles; ++r) {
        const uint32_t j = first + r * 16 + lane % 16;
        row[r] = j < a.n ? j : a.n - 1;
    }
    const T* x[M];
    for (int m = 0; m < M; ++m) {
        const uint32_t c = first_row + m * 16 + lane % 16;
        x[m] = (const T*)a.x + (int64_t)(c < a.rows ? c : a.rows - 1) * a.x_stride;
    }
    const Split<T> cols = {};
    f32x4 sum[kTiles][M] = {};
    rows_by_columns<M == 4 ? 1 : 2, ALIGNED>(w, row, cols, x, 0u, a.k, wave, (uint32_t)kFewWaves, sum);
    for (int r = 0; r < kTiles; ++r)
        for (int m = 0; m < M; ++m) sums[((wave * kTiles + r) * M + m) * 64 + lane] = sum[r][m];
    __syncthreads();
    for (uint32_t tile = wave; tile < kTiles * M; tile += kFewWaves) {
        f32x4 y = {};
        for (uint32_t v = 0; v < kFewWaves; ++v) y += sums[(v * kTiles * M + tile) * 64 + lane];
        const uint32_t c = first_row + tile % M * 16 + lane % 16, j = first + tile / M * 16 + lane / 16 * 4;
        if (c >= a.rows) continue;
        T* const out = (T*)a.out + (int64_t)c * a.out_stride + j;
        store_some<T, 4, false>(out, narrow<T, 4>(y), j < a.n ? (int)(a.n - j) : 0);
    }
}

}  // namespace

hipError_t launch_four_bit_product(const FourBitProductArgs& a, int type, hipStream_t stream) {
    return with_type(type, [&](auto t) {
        using T = decltype(t);
        const bool aligned = ((uintptr_t)a.x | (uintptr_t)a.x_stride * sizeof(T)) % 16 == 0 && a.k % 8 == 0;
        const uint32_t chunks = (a.rows + 63) / 64, m = a.rows <= 16 ? 1 : a.rows <= 32 ? 2 : 4;
        const auto kernel = aligned ? (m == 1 ? four_bit_product_kernel<T, true, 1> : m == 2 ? four_bit_product_kernel<T, true, 2> : four_bit_product_kernel<T, true, 4>)
                                    : (m == 1 ? four_bit_product_kernel<T, false, 1> : m == 2 ? four_bit_product_kernel<T, false, 2> : four_bit_product_kernel<T, false, 4>);
        // a launch has at most 65535 workgroups along the second dimension of its grid here
        FourBitProductArgs part = a;
        for (uint32_t done = 0; done < chunks; done += 65535) {
            const uint32_t now = chunks - done < 65535 ? chunks - done : 65535;
            part.x = (const T*)a.x + (int64_t)done * 64 * a.x_stride, part.out = (T*)a.out + (int64_t)done * 64 * a.out_stride;
            part.rows = a.rows - done * 64 < now * 64 ? a.rows - done * 64 : now * 64;
            hipLaunchKernelGGL(kernel, dim3((a.n + kTiles * 16 - 1) / (kTiles * 16), now), dim3(kFewThreads), (size_t)kFewWaves * kTiles * m * 64 * 16, stream, part);
            const hipError_t e = hipGetLastError();
            if (e != hipSuccess) return e;
        }
        return hipSuccess;
    });
}

}  // namespace tperm
