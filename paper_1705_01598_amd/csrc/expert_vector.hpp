// Vectors of elements, their way from and to memory, and 8-bit codes: what the kernels of the
// mixture-of-experts operators share.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

namespace tperm {

template <typename T, int N> using Vec = T __attribute__((ext_vector_type(N)));
typedef Vec<float, 2> f32x2;
typedef Vec<float, 4> f32x4;
typedef Vec<uint32_t, 2> u32x2;
typedef Vec<uint32_t, 4> u32x4;

// N elements at p.  ALIGNED: p is a multiple of the vector (16 bytes at most); else of the element only,
// which the global memory instructions take as well.
template <typename T, int N, bool ALIGNED> __device__ __forceinline__ Vec<T, N> load_vec(const T* p) {
    Vec<T, N> v;
    constexpr size_t kAlign = sizeof(v) < 16 ? sizeof(v) : 16;
    __builtin_memcpy(&v, ALIGNED ? (const T*)__builtin_assume_aligned(p, kAlign) : p, sizeof(v));
    return v;
}
template <typename T, int N, bool ALIGNED> __device__ __forceinline__ void store_vec(T* p, Vec<T, N> v) {
    constexpr size_t kAlign = sizeof(v) < 16 ? sizeof(v) : 16;
    __builtin_memcpy(ALIGNED ? (T*)__builtin_assume_aligned(p, kAlign) : p, &v, sizeof(v));
}

// The same where only the first `there` elements exist (there >= N: all; ALIGNED: all or none).
template <typename T, int N, bool ALIGNED> __device__ __forceinline__ Vec<T, N> load_some(const T* p, int there) {
    if (there >= N) return load_vec<T, N, ALIGNED>(p);
    Vec<T, N> v = {};
    if constexpr (!ALIGNED)
        for (int i = 0; i < N; ++i)
            if (i < there) v[i] = p[i];
    return v;
}
template <typename T, int N, bool ALIGNED> __device__ __forceinline__ void store_some(T* p, Vec<T, N> v, int there) {
    if (there >= N) return store_vec<T, N, ALIGNED>(p, v);
    if constexpr (!ALIGNED)
        for (int i = 0; i < N; ++i)
            if (i < there) p[i] = v[i];
}

// The same past the caches, for vectors at their alignment (16 bytes at most).
template <typename T, int N, bool ALIGNED> __device__ __forceinline__ Vec<T, N> load_once(const T* p, int there) {
    if constexpr (ALIGNED && sizeof(Vec<T, N>) == 16) return __builtin_bit_cast(Vec<T, N>, __builtin_nontemporal_load((const u32x4*)p));
    else return load_some<T, N, ALIGNED>(p, there);
}
template <typename T, int N, bool ALIGNED> __device__ __forceinline__ void store_once(T* p, Vec<T, N> v, int there) {
    if constexpr (ALIGNED && sizeof(v) == 8) {
        __builtin_nontemporal_store(__builtin_bit_cast(u32x2, v), (u32x2*)p);
    } else if constexpr (ALIGNED && sizeof(v) % 16 == 0) {
        u32x4 w[sizeof(v) / 16];
        __builtin_memcpy(w, &v, sizeof(v));
        for (size_t i = 0; i < sizeof(v) / 16; ++i) __builtin_nontemporal_store(w[i], (u32x4*)p + i);
    } else {
        store_some<T, N, ALIGNED>(p, v, there);
    }
}

// Conversions round to nearest even.
template <typename T, int N> __device__ __forceinline__ Vec<float, N> widen(Vec<T, N> v) { return __builtin_convertvector(v, Vec<float, N>); }
template <typename T, int N> __device__ __forceinline__ Vec<T, N> narrow(Vec<float, N> v) { return __builtin_convertvector(v, Vec<T, N>); }

// Biased exponent (s + 127) of a block's scale from the bits of its largest finite magnitude: with
// magnitude = 1.m * 2^e the least s for which it is at most 448 * 2^s = 1.75 * 2^(s + 8).
__device__ __forceinline__ uint32_t scale_of(uint32_t magnitude) {
    const int s = (int)(magnitude >> 23) - 8 + ((magnitude & 0x7FFFFFu) > 0x600000u ? 1 : 0);
    return (uint32_t)(s < 10 ? 10 : s > 247 ? 247 : s);
}
__device__ __forceinline__ float power_of(uint32_t biased) { return __uint_as_float(biased << 23); }

// Codes of 8 values: x / 2^s is exact but for values that end as zero anyway.
__device__ __forceinline__ u32x2 codes_of(Vec<float, 8> x, uint32_t scale) {
    const float by = power_of(254u - scale);
    u32x2 c;
    for (int h = 0; h < 2; ++h) {
        float q[4];
        for (int i = 0; i < 4; ++i) {
            const float v = x[4 * h + i];
            q[i] = __builtin_isfinite(v) ? v * by : __builtin_nanf("");
        }
        int w = __builtin_amdgcn_cvt_pk_fp8_f32(q[0], q[1], 0, false);
        w = __builtin_amdgcn_cvt_pk_fp8_f32(q[2], q[3], w, true);
        c[h] = (uint32_t)w;
    }
    return c;
}
// What 8 codes stand for, held to the finite range of T: the rounding of 8 bits carries the largest values of a
// type beyond it (binary16's 65504 to 65536, binary32's to 2^128).  Only blocks of the largest scale can
// hold such values; NaN stays.
template <typename T> struct Range;
template <> struct Range<float> { static constexpr float kLargest = 0x1.fffffep127f, kSafe = 0x1p119f; };
template <> struct Range<__bf16> { static constexpr float kLargest = 0x1.fep127f, kSafe = 0x1p119f; };
template <> struct Range<_Float16> { static constexpr float kLargest = 65504.0f, kSafe = 128.0f; };
template <typename T> __device__ __forceinline__ Vec<float, 8> values_of(u32x2 codes, float scale) {
    Vec<float, 8> v;
    for (int h = 0; h < 2; ++h) {
        const f32x2 a = __builtin_amdgcn_cvt_pk_f32_fp8((int)codes[h], false), b = __builtin_amdgcn_cvt_pk_f32_fp8((int)codes[h], true);
        v[4 * h] = a[0] * scale, v[4 * h + 1] = a[1] * scale, v[4 * h + 2] = b[0] * scale, v[4 * h + 3] = b[1] * scale;
    }
    if (scale > Range<T>::kSafe)
        for (int i = 0; i < 8; ++i) v[i] = v[i] > Range<T>::kLargest ? Range<T>::kLargest : v[i] < -Range<T>::kLargest ? -Range<T>::kLargest : v[i];
    return v;
}

// Bits of the magnitude if finite, else 0: finite magnitudes order as their bits do.
__device__ __forceinline__ uint32_t finite_magnitude(float v) {
    const uint32_t b = __float_as_uint(v) & 0x7FFFFFFFu;
    return b < 0x7F800000u ? b : 0u;
}

// A launch has fewer than 2^32 threads along each dimension of its grid: more workgroups than kRow go on along
// the second.
constexpr uint32_t kRow = 1u << 22;
inline dim3 long_grid(uint64_t blocks) {
    return blocks <= kRow ? dim3((uint32_t)blocks) : dim3(kRow, (uint32_t)((blocks + kRow - 1) / kRow));
}
__device__ __forceinline__ uint64_t long_block() { return blockIdx.x + (uint64_t)kRow * blockIdx.y; }

// Calls f with the element type behind a tperm_type_t.
template <typename F> inline auto with_type(int type, F f) {
    return type == 0 ? f(float()) : type == 1 ? f((_Float16)0) : f((__bf16)0);
}

}  // namespace tperm
