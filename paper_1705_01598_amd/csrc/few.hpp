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
#include "few_places.hpp"

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
// Binary32 columns beside a matrix of 16 bits, whose elements are exact in binary32: products of that take the matrix cores 16 times as long.
template <typename T> __device__ __forceinline__ f32x4 multiply(Vec<T, 8> w, Vec<float, 8> x, f32x4 sum) {
    for (int i = 0; i < 8; ++i) sum = __builtin_amdgcn_mfma_f32_16x16x4f32((float)w[i], x[i], sum, 0, 0, 0);
    return sum;
}

// 8 numbers as sums of P bfloat16 parts, each the upper 8 bits of what the one before it left, so that two hold a binary16 number
// and three a binary32 one (below 2^-102 the last of them is no normal number).  Infinities and NaN are the first part alone; with FINITE, which is 44
// instructions for three parts instead of 68, they make the second one NaN.
template <int P, bool FINITE = false> __device__ __forceinline__ void parts_of(Vec<float, 8> v, bf16x8 (&part)[P]) {
    if constexpr (!FINITE)
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = __builtin_canonicalizef(v[i]);      // a NaN with a bit among the upper 16
#pragma unroll
    for (int p = 0; p < P; ++p) {
        u32x4 words;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const uint32_t low = __float_as_uint(v[2 * i]), high = __float_as_uint(v[2 * i + 1]);
            words[i] = __builtin_amdgcn_perm(high, low, 0x07060302u);
        }
        part[p] = __builtin_bit_cast(bf16x8, words);
        if (p + 1 < P)
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const float rest = v[i] - __uint_as_float(__float_as_uint(v[i]) & 0xFFFF0000u);
                v[i] = FINITE || p > 0 || __builtin_isfinite(v[i]) ? rest : 0.0f;
            }
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

// Which of a step's elements exist: all of them; those in front of the row's end; the same where a row is shorter than a lane's load.
enum class Reach { kAll, kEnd, kShort };

// 16 bytes at p, which is a multiple of the element's size.  Of 16-bit elements on an odd one, the 16 bytes from the element in front on and the last
// element: loads that do not start on 4 bytes come in at less than half the rate of all others (2.7 TB/s for 5.9).  odd: 2 where the tensor
// starts on 4 bytes, so that there is an element in front of an odd one, else 0, which loads the bytes as they lie.
__device__ __forceinline__ uint32_t odd_of(const void* tensor) { return (uintptr_t)tensor % 4 == 0 ? 2u : 0u; }
template <typename T, int N> __device__ __forceinline__ Vec<T, N> load_any(const T* p, uint32_t odd) {
    if constexpr (sizeof(T) == 4) {
        return load_vec<T, N, false>(p);
    } else {
        const uint32_t by = (uint32_t)(uintptr_t)p & odd;
        typedef Vec<T, N> Part;
        u32x4 w;
        __builtin_memcpy(&w, (const char*)p - by, 16);
        const uint32_t last = ((const uint16_t*)p)[N - 1];
        for (int k = 0; k < 4; ++k) w[k] = __builtin_amdgcn_alignbit(k < 3 ? w[k + 1] : last, w[k], by * 8);
        return __builtin_bit_cast(Part, w);
    }
}

// N elements of a row of `depth` from element i on, zeros for those behind its end: without a branch around the load, behind which the
// compiler would wait for it.  ALIGNED: depth is a multiple of N, and so is i; else elements that hang over the end are the row's
// last N, moved down.
template <Reach REACH, typename T, int N, bool ALIGNED> __device__ __forceinline__ Vec<T, N> load_reach(const T* row, uint32_t i, uint32_t depth, uint32_t odd) {
    static_assert(N * sizeof(T) == 16, "a lane's load");
    if constexpr (REACH == Reach::kAll) {
        if constexpr (ALIGNED) return load_vec<T, N, true>(row + i);
        else return load_any<T, N>(row + i, odd);
    } else if constexpr (REACH == Reach::kShort) {
        return load_some<T, N, false>(i < depth ? row + i : row, (int)depth - (int)i);
    } else if constexpr (ALIGNED) {
        const Vec<T, N> v = load_vec<T, N, true>(row + start_in(i, depth));
        u32x4 w = __builtin_bit_cast(u32x4, v);
        for (int k = 0; k < 4; ++k) w[k] = i < depth ? w[k] : 0u;
        return __builtin_bit_cast(Vec<T, N>, w);
    } else {
        typedef Vec<uint64_t, 2> Words;
        const uint32_t from = i < depth - N ? i : depth - N, over = i - from;
        const Words v = __builtin_bit_cast(Words, load_any<T, N>(row + from, odd));
        const uint32_t bits = over * 8 * (uint32_t)sizeof(T);
        const uint64_t high = bits < 64 ? v[1] >> bits : 0u;
        const uint64_t low = bits == 0 ? v[0] : bits < 64 ? v[0] >> bits | v[1] << (64 - bits) : bits < 128 ? v[1] >> (bits - 64) : 0u;
        return __builtin_bit_cast(Vec<T, N>, Vec<uint64_t, 2>{low, high});
    }
}

// A matrix of elements of T: 16 bytes to a lane and step.
template <typename T> struct Elements {
    static constexpr int kEach = 16 / sizeof(T), kDepth = 8 * kEach, kSub = 1;      // elements of a lane and of a row in a step; products of a step
    typedef Vec<T, kEach> Part;         // what a product takes of a lane
    const T* rows;
    uint32_t stride;                    // bytes from row to row
    uint32_t odd;
    struct Step { Part v; };
    template <Reach REACH, bool ALIGNED> __device__ __forceinline__ Step load(uint32_t row, uint32_t i, uint32_t depth) const {
        if constexpr (REACH == Reach::kAll) return {load_reach<REACH, T, kEach, ALIGNED>((const T*)((const char*)rows + (row * stride + i * (uint32_t)sizeof(T))), 0, 0, odd)};
        else return {load_reach<REACH, T, kEach, ALIGNED>((const T*)((const char*)rows + row * stride), i, depth, odd)};
    }
    static __device__ __forceinline__ Part open(const Step& s, int) { return s.v; }
    static __device__ __forceinline__ void pair(Step& a, Step& b) {
        u32x4 p = __builtin_bit_cast(u32x4, a.v), q = __builtin_bit_cast(u32x4, b.v);
        pair_words(p, q);
        a.v = __builtin_bit_cast(Part, p), b.v = __builtin_bit_cast(Part, q);
    }
};

// A matrix in 4 bits: a group of 32 codes and its scale to a lane and step.  A code times its power of two is exact in bfloat16, and two
// of them take one conversion.
struct FourBits {
    static constexpr int kEach = 32, kDepth = kFourBitDepth, kSub = 4;
    typedef bf16x8 Part;
    const uint8_t *rows, *scales;
    uint32_t groups;                    // of a row
    struct Step { u32x4 codes; uint32_t scale; };
    template <Reach REACH, bool ALIGNED> __device__ __forceinline__ Step load(uint32_t row, uint32_t i, uint32_t depth) const {
        const bool there = REACH == Reach::kAll || i < depth;
        const uint32_t g = row * groups + (there ? i / 32 : 0u);
        Step s = {*(const u32x4*)(rows + (uint64_t)(g * 16u)), scales[g]};
        for (int k = 0; k < 4; ++k) s.codes[k] = there ? s.codes[k] : 0u;
        s.scale = there ? s.scale : 127u;
        return s;
    }
    static __device__ __forceinline__ Part open(const Step& s, int j) {
        const float scale = scale_value(s.scale);
        const uint32_t w = s.codes[j];
        const bf16x2 a = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, 0), b = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, 1);
        const bf16x2 c = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, 2), d = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, 3);
        return {a[0], a[1], b[0], b[1], c[0], c[1], d[0], d[1]};
    }
    static __device__ __forceinline__ void pair(Step& a, Step& b) {
        pair_words(a.codes, b.codes);
        pair_words(a.scale, b.scale);
    }
    static __device__ __forceinline__ float scale_value(uint32_t biased) { return __uint_as_float(biased == 255u ? 0x7FC00000u : biased << 23); }
};

// Columns that are there as the products take them: kParts arrays of E, `apart` elements from each other.  FILLED: rows start on 16 bytes and are zeros up to
// the end of the step that their last element is in; steps behind that are not looked at, though they may be requested.
template <typename E, int P, bool FILLED = false> struct Ready {
    static constexpr int kParts = P, N = 16 / sizeof(E);
    int64_t apart;
    uint32_t odd;
    typedef Vec<E, N> Part;
    struct Raw { Part part[P]; };
    // sub-product j of the elements that piece `piece` of a step from i on has
    template <typename W, Reach REACH, bool ALIGNED> __device__ __forceinline__ Raw load(const E* x, uint32_t i, uint32_t piece, uint32_t depth, int j) const {
        Raw r;
        constexpr Reach kReach = FILLED && REACH != Reach::kAll ? Reach::kEnd : REACH;
        for (int p = 0; p < P; ++p) r.part[p] = load_reach<kReach, E, N, ALIGNED || FILLED>(x + p * apart, i + piece * W::kEach + j * N, depth, odd);
        return r;
    }
    static __device__ __forceinline__ void open(const Raw& r, Part (&part)[P]) {
        for (int p = 0; p < P; ++p) part[p] = r.part[p];
    }
};
// Columns of T that become bfloat16 parts on their way.
template <typename T> struct Split {
    static constexpr int kParts = sizeof(T) == 4 ? 3 : std::is_same_v<T, _Float16> ? 2 : 1;
    typedef bf16x8 Part;
    typedef Vec<T, 8> Eight;
    static constexpr int kLoads = sizeof(T) / 2, N = 16 / sizeof(T);
    struct Raw { Vec<T, N> v[kLoads]; };
    uint32_t odd;
    template <typename W, Reach REACH, bool ALIGNED> __device__ __forceinline__ Raw load(const T* x, uint32_t i, uint32_t piece, uint32_t depth, int j) const {
        Raw r;
        for (int k = 0; k < kLoads; ++k) r.v[k] = load_reach<REACH, T, N, ALIGNED>(x, i + piece * W::kEach + j * 8 + k * N, depth, odd);
        return r;
    }
    static __device__ __forceinline__ void open(const Raw& r, Part (&part)[kParts]) {
        if constexpr (kParts == 1) part[0] = __builtin_bit_cast(bf16x8, r.v[0]);
        else parts_of<kParts>(widen<T, 8>(__builtin_bit_cast(Eight, r.v)), part);
    }
};
// Columns in binary32, laid out as hidden_place says and zeros to the end of their last step, beside a matrix whose products take PART of a lane: as bfloat16 parts
// (SPLIT; only what is finite, and only beside what is), or as they are.  A binary16 matrix holds neither the range nor the bits of such parts.
template <typename PART, bool SPLIT> struct Held {
    static constexpr bool kSplit = SPLIT && std::is_same_v<PART, bf16x8>;
    static constexpr int kParts = kSplit ? 3 : 1, kNumbers = std::is_same_v<PART, f32x4> ? 4 : 8, kLoads = kNumbers / 4;
    typedef Vec<float, kNumbers> Numbers;
    typedef std::conditional_t<kSplit, bf16x8, Numbers> Part;
    struct Raw { f32x4 v[kLoads]; };
    template <typename W, Reach REACH, bool ALIGNED> __device__ __forceinline__ Raw load(const float* x, uint32_t i, uint32_t piece, uint32_t depth, int j) const {
        const float* const step = x + (REACH == Reach::kAll ? i : start_in(i, depth)) + hidden_piece(piece);
        Raw r;
        for (int k = 0; k < kLoads; ++k) r.v[k] = load_vec<float, 4, true>(step + hidden_quad(j * kLoads + k));
        return r;
    }
    static __device__ __forceinline__ void open(const Raw& r, Part (&part)[kParts]) {
        if constexpr (kSplit) parts_of<kParts, true>(__builtin_bit_cast(Numbers, r.v), part);
        else part[0] = __builtin_bit_cast(Part, r.v);
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

// STEPS steps of one wavefront from element `i` on: sum += rows row[r] by columns x[m], rows of `depth` elements.
template <typename S, int STEPS, bool ALIGNED, Reach REACH, typename W, typename X, typename E>
__device__ __forceinline__ void steps(const W& w, const uint32_t (&row)[S::R], const X& cols, const E* const (&x)[S::M], uint32_t i, uint32_t depth,
                                      f32x4 (&sum)[S::kSums][S::M]) {
    constexpr int R = S::R, M = S::M, kTurns = S::kPaired ? 2 : 1;      // paired: first the even pieces of both tiles, then the odd ones
    const auto there = [&](int t) { return REACH == Reach::kAll || i + t * W::kDepth < depth; };
    typename W::Step s[STEPS][R];
    const auto request = [&] {
#pragma unroll
        for (int t = 0; t < STEPS; ++t)
#pragma unroll
            for (int r = 0; r < R; ++r) s[t][r] = w.template load<REACH, ALIGNED>(row[r], i + t * W::kDepth + S::piece() * W::kEach, depth);
        __builtin_amdgcn_sched_barrier(0);
    };
    const auto columns_of = [&](int t, int turn, int j, int m) {
        const uint32_t piece = S::kPaired ? (threadIdx.x & 63u) / 16 * 2 + turn : S::piece();
        return cols.template load<W, REACH, ALIGNED>(x[m], i + t * W::kDepth, piece, depth, j);
    };
    const auto products = [&](int t, int turn, int j, const typename X::Raw (&raw)[M]) {
        typename X::Part c[M][X::kParts];
#pragma unroll
        for (int m = 0; m < M; ++m) X::open(raw[m], c[m]);
#pragma unroll
        for (int r = 0; r < S::kSums; ++r) {
            const typename W::Part part = W::open(s[t][S::kPaired ? 2 * r + turn : r], j);
#pragma unroll
            for (int m = 0; m < M; ++m)
#pragma unroll
                for (int p = 0; p < X::kParts; ++p) sum[r][m] = multiply(part, c[m][p], sum[r][m]);
        }
    };
    const auto paired = [&](int t) {
        if constexpr (S::kPaired)
#pragma unroll
            for (int r = 0; r < R; r += 2) W::pair(s[t][r], s[t][r + 1]);
    };
    // Loads come back in their order, so the columns, which are near, are requested in front of the matrix, all of them where they fit 32
    // registers, else as many as do.  The fences are for the compiler, which would move the requests down to the products, until a few are
    // under way at a time.
    constexpr int kWords = M * (int)sizeof(typename X::Raw) / 4, kTurnSubs = kTurns * W::kSub;
    constexpr int kHeld = 32 / kWords, kAhead = kHeld >= STEPS * kTurnSubs ? STEPS * kTurnSubs : kHeld >= kTurnSubs ? kTurnSubs : kHeld >= W::kSub ? W::kSub : kHeld >= 2 && W::kSub % 2 == 0 ? 2 : 1;
#pragma unroll
    for (int first = 0; first < STEPS * kTurnSubs; first += kAhead) {
        if (first != 0 && first % kTurnSubs == 0 && !there(first / kTurnSubs)) break;
        typename X::Raw raw[kAhead][M];
#pragma unroll
        for (int u = 0; u < kAhead; ++u)
#pragma unroll
            for (int m = 0; m < M; ++m) raw[u][m] = columns_of((first + u) / kTurnSubs, (first + u) / W::kSub % kTurns, (first + u) % W::kSub, m);
        if (first == 0) request();
#pragma unroll
        for (int u = 0; u < kAhead; ++u) {
            const int t = (first + u) / kTurnSubs, turn = (first + u) / W::kSub % kTurns, j = (first + u) % W::kSub;
            if (u != 0 && (first + u) % kTurnSubs == 0 && !there(t)) break;
            if (turn == 0 && j == 0) paired(t);
            products(t, turn, j, raw[u]);
        }
    }
}

// The piece of the sum from `from` to `to` (a multiple of the steps' depth away, or the row's end) that falls to wavefront `wave`
// of `waves`: blocks of that depth in turn.
template <typename S, int STEPS, bool ALIGNED, typename W, typename X, typename E>
__device__ __forceinline__ void rows_by_columns(const W& w, const uint32_t (&row)[S::R], const X& cols, const E* const (&x)[S::M], uint32_t from, uint32_t to,
                                                uint32_t wave, uint32_t waves, f32x4 (&sum)[S::kSums][S::M]) {
    constexpr uint32_t kBlock = STEPS * W::kDepth;
    uint32_t i = from + wave * kBlock;
    for (; i + kBlock <= to; i += waves * kBlock) steps<S, STEPS, ALIGNED, Reach::kAll>(w, row, cols, x, i, to, sum);
    if (i >= to) return;
    if (!ALIGNED && to < 8) steps<S, 1, ALIGNED, Reach::kShort>(w, row, cols, x, i, to, sum);
    else if (STEPS > 2 && to - i <= W::kDepth) steps<S, 1, ALIGNED, Reach::kEnd>(w, row, cols, x, i, to, sum);
    else steps<S, STEPS, ALIGNED, Reach::kEnd>(w, row, cols, x, i, to, sum);
}

}  // namespace tperm
