// Matrices held in 4 bits: rows to codes and scales, and back.
//
// HBM is the bound: every element is read once and every code written once.  A thread takes 8 neighbours, four
// threads side by side a group of 32, whose largest magnitude goes between them by DPP moves.  Scales are powers
// of two, so the division is exact and the only rounding is that of the code, two of which take one conversion.
//
// 65536 x 2048 bfloat16: 61 us to 4 bits, 5.6 TB/s, and 47 back, 7.2 TB/s, as the codes are still in the memory-side cache; 16384 x 8192 binary32
// 103 and 105 us, 5.9 TB/s.
#include <type_traits>

#include "decode.hpp"
#include "expert_vector.hpp"
#include "plan.hpp"

namespace tperm {

namespace {

constexpr int kFourBitThreads = 256;

// Maximum over four neighbouring lanes (DPP quad permutations), in all of them.
__device__ __forceinline__ uint32_t quad_max(uint32_t v) {
    uint32_t o = (uint32_t)__builtin_amdgcn_mov_dpp((int)v, 0xB1, 0xF, 0xF, true);   // 1 0 3 2
    v = v > o ? v : o;
    o = (uint32_t)__builtin_amdgcn_mov_dpp((int)v, 0x4E, 0xF, 0xF, true);            // 2 3 0 1
    return v > o ? v : o;
}

// Biased exponent of a group's scale from the bits of its largest magnitude 1.m * 2^e, the least s for which it is at
// most 6 * 2^s = 1.5 * 2^(s + 2); 255 for an infinity or NaN.
__device__ __forceinline__ uint32_t group_scale(uint32_t magnitude) {
    const int s = (int)(magnitude >> 23) - 2 + ((magnitude & 0x7FFFFFu) > 0x400000u ? 1 : 0);
    return magnitude >= 0x7F800000u ? 255u : (uint32_t)(s < 2 ? 2 : s > 252 ? 252 : s);
}

struct Place {
    uint32_t row, col;
    int there;
};
// V neighbours to a thread.
template <int V> __device__ __forceinline__ Place place_of(const FourBitArgs& a) {
    const uint32_t groups = (a.width + 31) / 32, per_row = groups * (32 / V);
    const uint64_t at = long_block() * kFourBitThreads + threadIdx.x;
    Place p;
    const uint64_t row = a.per_row.magic != 0 ? fdiv((uint32_t)at, a.per_row) : at / per_row;
    p.row = (uint32_t)row;
    const uint32_t part = (uint32_t)(at - row * per_row);
    p.col = part * V;
    p.there = row < a.rows ? (int)a.width - (int)p.col : 0;
    return p;
}

template <typename T, bool ALIGNED> __global__ __launch_bounds__(kFourBitThreads) void four_bit_store_kernel(const FourBitArgs a) {
    const Place p = place_of<8>(a);
    if (p.row >= a.rows) return;        // whole groups of four threads
    Vec<float, 8> x = {};
    // past the caches, where the codes may still be when they are read (65536 x 2048 bfloat16 to 4 bits and back 113 -> 108 us)
    if (p.there > 0) x = widen<T, 8>(load_once<T, 8, ALIGNED>((const T*)a.in + (int64_t)p.row * a.stride + p.col, p.there));
    uint32_t m = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const uint32_t b = __float_as_uint(x[i]) & 0x7FFFFFFFu;
        m = m > b ? m : b;
    }
    const uint32_t s = group_scale(quad_max(m));
    uint32_t c = 0;
    if (s != 255u) {
        const float by = __uint_as_float((254u - s) << 23);     // the division is exact but for values that end as zero
        float q[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) q[i] = __builtin_fminf(__builtin_fmaxf(x[i] * by, -6.0f), 6.0f);
        c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, q[0], q[1], 1.0f, 0);
        c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, q[2], q[3], 1.0f, 1);
        c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, q[4], q[5], 1.0f, 2);
        c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, q[6], q[7], 1.0f, 3);
    }
    const uint64_t groups = (a.width + 31) / 32, group = p.row * groups + p.col / 32;
    ((uint32_t*)a.codes)[group * 4 + p.col % 32 / 8] = c;
    if (p.col % 32 == 0) a.scales[group] = (uint8_t)s;
}

template <typename T> struct Largest;
template <> struct Largest<float> { static constexpr float k = 0x1.fffffep127f; };
template <> struct Largest<__bf16> { static constexpr float k = 0x1.fep127f; };
template <> struct Largest<_Float16> { static constexpr float k = 65504.0f; };

// 16 bytes of results to a thread: stores past the caches that are whole lines (with 32 bytes of binary32, two stores of every other
// 16 bytes, 199 us for 536 MB, now 105).
template <typename T> constexpr int kLoaded = 16 / (int)sizeof(T);
template <typename T, bool ALIGNED> __global__ __launch_bounds__(kFourBitThreads) void four_bit_load_kernel(const FourBitArgs a) {
    constexpr int V = kLoaded<T>;
    typedef std::conditional_t<V == 8, uint32_t, uint16_t> Codes;
    const Place p = place_of<V>(a);
    if (p.there <= 0) return;
    const uint64_t groups = (a.width + 31) / 32, group = p.row * groups + p.col / 32;
    const uint32_t c = ((const Codes*)a.codes)[group * (32 / V) + p.col % 32 / V], s = a.scales[group];
    const float scale = __uint_as_float(s << 23);
    f32x2 v[4] = {__builtin_amdgcn_cvt_scalef32_pk_f32_fp4(c, 1.0f, 0), __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(c, 1.0f, 1)};
    if constexpr (V == 8) v[2] = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(c, 1.0f, 2), v[3] = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(c, 1.0f, 3);
    Vec<float, V> x;
#pragma unroll
    for (int i = 0; i < V; ++i) x[i] = s == 255u ? __builtin_nanf("") : __builtin_fminf(__builtin_fmaxf(v[i / 2][i % 2] * scale, -Largest<T>::k), Largest<T>::k);
    store_once<T, V, ALIGNED>((T*)a.out + (int64_t)p.row * a.stride + p.col, narrow<T, V>(x), p.there);
}

bool on_eight(size_t elem, const void* p, int64_t stride) { return ((uintptr_t)p | (uintptr_t)stride * elem) % 16 == 0; }

template <typename K> hipError_t go(K kernel, FourBitArgs a, int neighbours, hipStream_t stream) {
    const uint32_t per_row = (a.width + 31) / 32 * (32 / neighbours);
    const uint64_t threads = (uint64_t)a.rows * per_row;
    a.per_row = threads < (1ull << 31) - kFourBitThreads ? make_fastdiv(per_row) : FastDiv{0, 0};
    hipLaunchKernelGGL(kernel, long_grid((threads + kFourBitThreads - 1) / kFourBitThreads), dim3(kFourBitThreads), 0, stream, a);
    return hipGetLastError();
}

}  // namespace

hipError_t launch_four_bit_store(FourBitArgs a, int type, hipStream_t stream) {
    return with_type(type, [&](auto t) {
        using T = decltype(t);
        return a.width % 8 == 0 && on_eight(sizeof(T), a.in, a.stride) ? go(four_bit_store_kernel<T, true>, a, 8, stream) : go(four_bit_store_kernel<T, false>, a, 8, stream);
    });
}

hipError_t launch_four_bit_load(FourBitArgs a, int type, hipStream_t stream) {
    return with_type(type, [&](auto t) {
        using T = decltype(t);
        return a.width % 8 == 0 && on_eight(sizeof(T), a.out, a.stride) ? go(four_bit_load_kernel<T, true>, a, kLoaded<T>, stream) : go(four_bit_load_kernel<T, false>, a, kLoaded<T>, stream);
    });
}

}  // namespace tperm
