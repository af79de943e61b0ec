// Products of a matrix with few rows: device code that the 4-bit products and the layer for a few tokens share.
//
// out[c, j] = sum over i of w[j, i] * x[c, i].  The matrix w is what there is to read, once, straight from memory to the
// registers that the matrix cores take it from.  A wavefront's load takes 16 bytes a lane, 128 of each of 8 rows (a tile):
// whole lines, which come in at 6.7 TB/s where 64 bytes of 16 rows come in at 5.9.  Which elements a lane holds does not matter to
// a product as long as both operands agree, so that such a load is a 16 x 16 product's left operand in one of two ways:
//   - up to 8 columns: the lanes of odd pieces are 8 rows more, and the columns' odd pieces 8 columns more; the product of
//     even pieces and that of odd ones stand on the diagonal, and are added in the end;
//   - more columns, two tiles: odd pieces of the one change places with even pieces of the other, one instruction a word, and
//     16 rows meet 16 columns.
// The matrix cores are idle most of the time either way (1 KB of bfloat16 comes in every 80 clocks a compute unit, and its product takes
// 16 of one SIMD's).  The wavefronts of a workgroup share the sum, piece by piece along i, so that every element of x is read
// once a workgroup too; their sums are joined through LDS in the order of the wavefronts.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "expert_vector.hpp"

namespace tperm {

typedef Vec<__bf16, 2> bf16x2;
typedef Vec<__bf16, 8> bf16x8;
typedef Vec<_Float16, 8> f16x8;

constexpr int kFewWaves = 8, kFewThreads = 64 * kFewWaves;

__device__ __forceinline__ f32x4 multiply(bf16x8 w, bf16x8 x, f32x4 sum) { return __builtin_amdgcn_mfma_f32_16x16x32_bf16(w, x, sum, 0, 0, 0); }
__device__ __forceinline__ f32x4 multiply(f16x8 w, f16x8 x, f32x4 sum) { return __builtin_amdgcn_mfma_f32_16x16x32_f16(w, x, sum, 0, 0, 0); }
__device__ __forceinline__ f32x4 multiply(f32x4 w, f32x4 x, f32x4 sum) {
    for (int i = 0; i < 4; ++i) sum = __builtin_amdgcn_mfma_f32_16x16x4f32(w[i], x[i], sum, 0, 0, 0);
    return sum;
}

// A number as the sum of bfloat16 parts, each what the one before it left: 8 bits to a part, so that two hold a
// binary16 number and three a binary32 one (below 2^-110 what 2^-133 leaves off).  Infinities and NaN are the first part alone.
__device__ __forceinline__ uint32_t first_part(float v, float* rest) {
    uint32_t b = __float_as_uint(v);
    const uint32_t size = b & 0x7FFFFFFFu;
    b |= size > 0x7F800000u ? 0x400000u : 0u;      // a NaN stays one
    b &= 0xFFFF0000u;
    *rest = size < 0x7F800000u ? v - __uint_as_float(b) : 0.0f;
    return b;
}
// P parts of 8 numbers.
template <int P> __device__ __forceinline__ void parts_of(Vec<float, 8> v, bf16x8 (&part)[P]) {
    for (int p = 0; p < P; ++p) {
        u32x4 words;
        for (int i = 0; i < 4; ++i) {
            float rest[2];
            const uint32_t low = first_part(v[2 * i], &rest[0]), high = first_part(v[2 * i + 1], &rest[1]);
            words[i] = low >> 16 | high;
            v[2 * i] = rest[0], v[2 * i + 1] = rest[1];
        }
        part[p] = __builtin_bit_cast(bf16x8, words);
    }
}

// Of 16 lanes, the upper 8 of a change places with the lower 8 of b.
__device__ __forceinline__ void pair_words(uint32_t& a, uint32_t& b) {
    const int p = (int)a, q = (int)b;
    a = (uint32_t)__builtin_amdgcn_update_dpp(p, q, 0x128, 0xF, 0xC, false);       // row_ror:8 into lanes 8 .. 15
    b = (uint32_t)__builtin_amdgcn_update_dpp(q, p, 0x128, 0xF, 0x3, false);       // into lanes 0 .. 7
}
__device__ __forceinline__ void pair_words(u32x4& a, u32x4& b) {
    for (int i = 0; i < 4; ++i) {
        uint32_t p = a[i], q = b[i];
        pair_words(p, q);
        a[i] = p, b[i] = q;
    }
}

// A matrix of elements of T: 16 bytes to a lane and step.
template <typename T> struct Elements {
    static constexpr int kEach = 16 / sizeof(T), kDepth = 8 * kEach, kSub = 1;      // elements of a lane and of a row in a step; products of a step
    typedef Vec<T, kEach> Part;         // what a product takes of a lane
    const T* rows;
    uint32_t stride;                    // bytes from row to row
    struct Step { Part v; };
    template <bool ALIGNED> __device__ __forceinline__ Step load(uint32_t row, uint32_t i) const {
        return {load_vec<T, kEach, ALIGNED>((const T*)((const char*)rows + (row * stride + i * (uint32_t)sizeof(T))))};
    }
    template <bool ALIGNED> __device__ __forceinline__ Step load_some_of(uint32_t row, uint32_t i, int there) const {
        return {load_some<T, kEach, ALIGNED>((const T*)((const char*)rows + (row * stride + (there > 0 ? i : 0u) * (uint32_t)sizeof(T))), there)};
    }
    static __device__ __forceinline__ void open(const Step& s, Part (&part)[kSub]) { part[0] = s.v; }
    static __device__ __forceinline__ void pair(Step& a, Step& b) {
        u32x4 p = __builtin_bit_cast(u32x4, a.v), q = __builtin_bit_cast(u32x4, b.v);
        pair_words(p, q);
        a.v = __builtin_bit_cast(Part, p), b.v = __builtin_bit_cast(Part, q);
    }
};

// A matrix in 4 bits: a group of 32 codes and its scale to a lane and step.  A code times its power of two is exact in bfloat16, and two
// of them take one conversion.
struct FourBits {
    static constexpr int kEach = 32, kDepth = 256, kSub = 4;
    typedef bf16x8 Part;
    const uint8_t *rows, *scales;
    uint32_t groups;                    // of a row
    struct Step { u32x4 codes; uint32_t scale; };
    template <bool ALIGNED> __device__ __forceinline__ Step load(uint32_t row, uint32_t i) const {
        const uint32_t g = row * groups + i / 32;
        return {*(const u32x4*)(rows + (uint64_t)(g * 16u)), scales[g]};
    }
    template <bool ALIGNED> __device__ __forceinline__ Step load_some_of(uint32_t row, uint32_t i, int there) const {
        if (there > 0) return load<ALIGNED>(row, i);
        return {u32x4{}, 127u};
    }
    static __device__ __forceinline__ void open(const Step& s, Part (&part)[kSub]) {
        const float scale = scale_value(s.scale);
        for (int j = 0; j < 4; ++j) {
            const uint32_t w = s.codes[j];
            const bf16x2 a = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, 0), b = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, 1);
            const bf16x2 c = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, 2), d = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, 3);
            part[j] = bf16x8{a[0], a[1], b[0], b[1], c[0], c[1], d[0], d[1]};
        }
    }
    static __device__ __forceinline__ void pair(Step& a, Step& b) {
        pair_words(a.codes, b.codes);
        pair_words(a.scale, b.scale);
    }
    static __device__ __forceinline__ float scale_value(uint32_t biased) { return __uint_as_float(biased == 255u ? 0x7FC00000u : biased << 23); }
};

// Columns that are there as the products take them: kParts arrays of E, `apart` elements from each other.
template <typename E, int P> struct Ready {
    static constexpr int kParts = P, N = 16 / sizeof(E);
    int64_t apart;
    typedef Vec<E, N> Part;
    // sub-product j of a step in which a lane has EACH elements from i on, `there` of which exist
    template <int EACH, bool ALIGNED, bool ALL> __device__ __forceinline__ void get(const E* x, uint32_t i, int there, int j, Part (&part)[P]) const {
        for (int p = 0; p < P; ++p) {
            const E* const at = x + p * apart + i + j * N;
            part[p] = ALL ? load_vec<E, N, ALIGNED>(at) : load_some<E, N, ALIGNED>(there - j * N > 0 ? at : x, there - j * N);
        }
    }
};
// Columns of T that become bfloat16 parts on their way.
template <typename T> struct Split {
    static constexpr int kParts = sizeof(T) == 4 ? 3 : std::is_same_v<T, _Float16> ? 2 : 1;
    typedef bf16x8 Part;
    template <int EACH, bool ALIGNED, bool ALL> __device__ __forceinline__ void get(const T* x, uint32_t i, int there, int j, Part (&part)[kParts]) const {
        const T* const at = x + i + j * 8;
        Vec<T, 8> v;
        if constexpr (ALL) v = load_vec<T, 8, ALIGNED>(at);
        else v = load_some<T, 8, ALIGNED>(there - j * 8 > 0 ? at : x, there - j * 8);
        if constexpr (kParts == 1) part[0] = __builtin_bit_cast(bf16x8, v);
        else parts_of<kParts>(widen<T, 8>(v), part);
    }
};

// How the tiles of a workgroup meet its columns: R tiles of 8 rows, M times 8 or, in pairs of tiles, 16 columns.
template <int R_, int M_, bool PAIRED> struct Shape {
    static constexpr int R = R_, M = M_, kColumns = PAIRED ? 16 : 8, kSums = PAIRED ? R_ / 2 : R_;
    static constexpr bool kPaired = PAIRED;
    static_assert(!PAIRED || R_ % 2 == 0, "pairs");
    // Row of its tile that a lane loads, and the piece of it.
    static __device__ __forceinline__ uint32_t row() { return threadIdx.x % 8; }
    static __device__ __forceinline__ uint32_t piece() { return (threadIdx.x & 63u) / 8; }
    // Column that a lane loads.
    static __device__ __forceinline__ uint32_t column(int m) { return m * kColumns + threadIdx.x % kColumns; }
};

// The sums of a wavefront hold, in the product's layout, at lane 16 * q + c the rows 4 * q + i of column c.  Paired: rows 8 and
// more are those of the second tile.  Else they are the odd pieces, which meet those of columns 8 and more.
// Where 4 rows 4 * half + i of column c of tile `tile` stand: in one lane, or in two that are added.
template <typename S> __device__ __forceinline__ f32x4 sums_at(const f32x4* wave_sums, int tile, int m, uint32_t half, uint32_t c) {
    if constexpr (S::kPaired) return wave_sums[(tile / 2 * S::M + m) * 64 + 16 * (2 * (tile % 2) + half) + c];
    else return wave_sums[(tile * S::M + m) * 64 + 16 * half + c] + wave_sums[(tile * S::M + m) * 64 + 16 * (2 + half) + 8 + c];
}

// STEPS steps of one wavefront from element `i` on: sum += rows row[r] by columns x[m].  ALL: every element of the steps
// exists, else those below `depth`.
template <typename S, int STEPS, bool ALIGNED, bool ALL, typename W, typename X, typename E>
__device__ __forceinline__ void steps(const W& w, const uint32_t (&row)[S::R], const X& cols, const E* const (&x)[S::M], uint32_t i, uint32_t depth,
                                      f32x4 (&sum)[S::kSums][S::M]) {
    constexpr int R = S::R, M = S::M;
    typename W::Step s[STEPS][R];
#pragma unroll
    for (int t = 0; t < STEPS; ++t)
#pragma unroll
        for (int r = 0; r < R; ++r) {
            const uint32_t at = i + t * W::kDepth + S::piece() * W::kEach;
            if constexpr (ALL) s[t][r] = w.template load<ALIGNED>(row[r], at);
            else s[t][r] = w.template load_some_of<ALIGNED>(row[r], at, (int)depth - (int)at);
        }
#pragma unroll
    for (int t = 0; t < STEPS; ++t) {
        if constexpr (S::kPaired)
#pragma unroll
            for (int r = 0; r < R; r += 2) W::pair(s[t][r], s[t][r + 1]);
        // paired: first the even pieces of both tiles, then the odd ones
        constexpr int kTurns = S::kPaired ? 2 : 1;
#pragma unroll
        for (int turn = 0; turn < kTurns; ++turn) {
            const uint32_t at = i + t * W::kDepth + (S::kPaired ? (threadIdx.x & 63u) / 16 * 2 + turn : S::piece()) * W::kEach;
            typename W::Part part[S::kSums][W::kSub];
#pragma unroll
            for (int r = 0; r < S::kSums; ++r) W::open(s[t][S::kPaired ? 2 * r + turn : r], part[r]);
#pragma unroll
            for (int m = 0; m < M; ++m)
#pragma unroll
                for (int j = 0; j < W::kSub; ++j) {
                    typename X::Part c[X::kParts];
                    cols.template get<W::kEach, ALIGNED, ALL>(x[m], at, (int)depth - (int)at, j, c);
#pragma unroll
                    for (int p = 0; p < X::kParts; ++p)
#pragma unroll
                        for (int r = 0; r < S::kSums; ++r) sum[r][m] = multiply(part[r][j], c[p], sum[r][m]);
                }
        }
    }
}

// The piece of the sum from `from` to `to` (a multiple of the steps' depth away, or the row's end) that falls to wavefront `wave`
// of `waves`.
template <typename S, int STEPS, bool ALIGNED, typename W, typename X, typename E>
__device__ __forceinline__ void rows_by_columns(const W& w, const uint32_t (&row)[S::R], const X& cols, const E* const (&x)[S::M], uint32_t from, uint32_t to,
                                                uint32_t wave, uint32_t waves, f32x4 (&sum)[S::kSums][S::M]) {
    constexpr uint32_t kBlock = STEPS * W::kDepth;
    uint32_t i = from + wave * kBlock;
    for (; i + kBlock <= to; i += waves * kBlock) steps<S, STEPS, ALIGNED, true>(w, row, cols, x, i, to, sum);
    for (int t = 0; t < STEPS; ++t, i += W::kDepth)
        if (i < to) steps<S, 1, ALIGNED, false>(w, row, cols, x, i, to, sum);
}

}  // namespace tperm
