// Products of few rows with a matrix held in 4 bits.
//
// The matrix is read once for 64 rows, the rows once for every workgroup, whose tiles are as many as leave 256 compute units one each: the rows are
// 4 times the bytes of the matrix for an element, and a compute unit takes in 26 GB/s at most of both together.  bfloat16: one row 2048 x 2048
// 3.3 us (an empty launch takes 1.6); 16 rows 4096 x 32768 20 us, 3.6 TB/s, with tiles of 32 rows of the matrix 34, of 64 21.2;
// one row 8192 x 16384 15.8 us, 4.5 TB/s; 64 rows 4096 x 16384 39 us (tiles of 32 65).
#include <type_traits>

#include "decode.hpp"
#include "few.hpp"
#include "launch.hpp"

namespace tperm {

namespace {

template <typename T, bool ALIGNED, int STEPS, typename S> __global__ __launch_bounds__(kFewThreads) void four_bit_product_kernel(const FourBitProductArgs a) {
    extern __shared__ f32x4 sums[];
    constexpr int R = S::R, M = S::M, kEach = S::kSums * M;
    const uint32_t lane = threadIdx.x & 63u, wave = (uint32_t)__builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6)), first = blockIdx.x * R * 8, first_row = blockIdx.y * 64;
    const FourBits w = {a.codes, a.scales, (a.k + 31) / 32};
    uint32_t row[R];
    for (int r = 0; r < R; ++r) {
        const uint32_t j = first + r * 8 + S::row();
        row[r] = j < a.n ? j : a.n - 1;
    }
    const T* x[M];
    for (int m = 0; m < M; ++m) {
        const uint32_t c = first_row + S::column(m);
        x[m] = (const T*)a.x + (int64_t)(c < a.rows ? c : a.rows - 1) * a.x_stride;
    }
    const Split<T> cols = {odd_of(a.x)};
    f32x4 sum[S::kSums][M] = {};
    rows_by_columns<S, STEPS, ALIGNED>(w, row, cols, x, 0u, a.k, wave, (uint32_t)kFewWaves, sum);
    for (int r = 0; r < S::kSums; ++r)
        for (int m = 0; m < M; ++m) sums[(wave * kEach + r * M + m) * 64 + lane] = sum[r][m];
    __syncthreads();
    // four results of one column to a lane
    for (uint32_t i = threadIdx.x; i < R * M * 2 * S::kColumns; i += kFewThreads) {
        const uint32_t half = i % 2, r = i / 2 % R, column = i / (2 * R), m = column / S::kColumns;
        const uint32_t c = first_row + column, j = first + r * 8 + half * 4;
        if (c >= a.rows || j >= a.n) continue;
        f32x4 y = {};
        for (uint32_t v = 0; v < kFewWaves; ++v) y += sums_at<S>(sums + v * kEach * 64, (int)r, (int)m, half, column % S::kColumns);
        store_some<T, 4, false>((T*)a.out + (int64_t)c * a.out_stride + j, narrow<T, 4>(y), (int)(a.n - j));
    }
}

template <typename T, bool ALIGNED, int STEPS, typename S> hipError_t go(const FourBitProductArgs& a, hipStream_t stream) {
    constexpr auto kKernel = four_bit_product_kernel<T, ALIGNED, STEPS, S>;
    constexpr size_t kLds = (size_t)kFewWaves * S::kSums * S::M * 64 * 16;
    if constexpr (kLds > 64 * 1024) {
        const hipError_t e = allow_lds<kKernel>(kLds);
        if (e != hipSuccess) return e;
    }
    const uint32_t chunks = (a.rows + 63) / 64;
    // a launch has at most 65535 workgroups along the second dimension of its grid here
    FourBitProductArgs part = a;
    for (uint32_t done = 0; done < chunks; done += 65535) {
        const uint32_t now = chunks - done < 65535 ? chunks - done : 65535;
        part.x = (const T*)a.x + (int64_t)done * 64 * a.x_stride, part.out = (T*)a.out + (int64_t)done * 64 * a.out_stride;
        part.rows = a.rows - done * 64 < now * 64 ? a.rows - done * 64 : now * 64;
        hipLaunchKernelGGL(kKernel, dim3((a.n + S::R * 8 - 1) / (S::R * 8), now), dim3(kFewThreads), kLds, stream, part);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    return hipSuccess;
}
template <typename T, bool ALIGNED> hipError_t product_of(const FourBitProductArgs& a, hipStream_t stream) {
    // 256 compute units want a workgroup each
    const uint32_t tiles = (a.n + 7) / 8;
    if (a.rows <= 8) return tiles < 512 ? go<T, ALIGNED, 2, Shape<1, 1, false>>(a, stream) : tiles < 1024 ? go<T, ALIGNED, 2, Shape<2, 1, false>>(a, stream)
                          : tiles < 2048 ? go<T, ALIGNED, 1, Shape<4, 1, false>>(a, stream) : go<T, ALIGNED, 1, Shape<8, 1, false>>(a, stream);
    if (a.rows <= 16) return tiles < 1024 ? go<T, ALIGNED, 1, Shape<2, 1, true>>(a, stream) : tiles < 2048 ? go<T, ALIGNED, 1, Shape<4, 1, true>>(a, stream)
                           : tiles < 4096 ? go<T, ALIGNED, 1, Shape<8, 1, true>>(a, stream) : go<T, ALIGNED, 1, Shape<16, 1, true>>(a, stream);
    if (a.rows <= 32) {
        if constexpr (sizeof(T) == 2)
            if (tiles >= 1024) return go<T, ALIGNED, 1, Shape<8, 2, true>>(a, stream);
        return tiles < 1024 ? go<T, ALIGNED, 1, Shape<2, 2, true>>(a, stream) : go<T, ALIGNED, 1, Shape<4, 2, true>>(a, stream);
    }
    if (a.rows <= 48) {
        if constexpr (sizeof(T) == 2)
            if (tiles >= 1024) return go<T, ALIGNED, 1, Shape<8, 3, true>>(a, stream);
        return tiles < 1024 ? go<T, ALIGNED, 1, Shape<2, 3, true>>(a, stream) : go<T, ALIGNED, 1, Shape<4, 3, true>>(a, stream);
    }
    if constexpr (sizeof(T) == 2)
        if (tiles >= 1024) return go<T, ALIGNED, 1, Shape<8, 4, true>>(a, stream);
    return tiles < 1024 ? go<T, ALIGNED, 1, Shape<2, 4, true>>(a, stream) : go<T, ALIGNED, 1, Shape<4, 4, true>>(a, stream);
}

}  // namespace

hipError_t launch_four_bit_product(const FourBitProductArgs& a, int type, hipStream_t stream) {
    return with_type(type, [&](auto t) {
        using T = decltype(t);
        const bool aligned = ((uintptr_t)a.x | (uintptr_t)a.x_stride * sizeof(T)) % 16 == 0 && a.k % 8 == 0;
        return aligned ? product_of<T, true>(a, stream) : product_of<T, false>(a, stream);
    });
}

}  // namespace tperm
