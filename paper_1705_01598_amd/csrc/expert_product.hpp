// Products of the experts: rows times their expert's matrix, and the gradient to the matrices.
//
// One tile of the result to a workgroup, summed over the whole depth (the summed index) with MFMA, 128 bytes
// of depth to a stage.  A tile has a fast side, whose index runs along memory in the result, and a slow one.
// The operand of a side lies in memory with the depth running fastest (kDepthFast: rows of activations, a
// matrix with the summed index first) or with the side's own index running fastest (kFreeFast: the other layout of
// a matrix; both operands of the gradient, whose depth are the rows of an expert).  LDS holds each as it
// lies in memory: fragments of the first kind are 16-byte reads, of the second transposing ones.
// Chunks of 16 bytes change places inside their LDS row (swizzle()), so that neither meets bank conflicts.
#pragma once
#include "expert_vector.hpp"
#include "experts.hpp"

namespace tperm {

enum Layout { kDepthFast = 0, kFreeFast = 1, kCodes = 2 };  // kCodes: as kFreeFast, 8-bit codes with scales
constexpr int kStageBytes = 128;                            // depth of a stage in bytes of an element row

#define TPERM_LDS __attribute__((address_space(3)))

// --- fragments ---

template <typename T> struct Matrix;   // the matrix instruction of a type: kDepth summed indices of 16 x 16 results
template <> struct Matrix<__bf16> {
    static constexpr int kDepth = 32;
    static __device__ __forceinline__ f32x4 mul(Vec<__bf16, 8> a, Vec<__bf16, 8> b, f32x4 c) { return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0); }
};
template <> struct Matrix<_Float16> {
    static constexpr int kDepth = 32;
    static __device__ __forceinline__ f32x4 mul(Vec<_Float16, 8> a, Vec<_Float16, 8> b, f32x4 c) { return __builtin_amdgcn_mfma_f32_16x16x32_f16(a, b, c, 0, 0, 0); }
};
template <> struct Matrix<float> {     // four instructions of depth 4; which index goes into which is free
    static constexpr int kDepth = 16;
    static __device__ __forceinline__ f32x4 mul(f32x4 a, f32x4 b, f32x4 c) {
#pragma unroll
        for (int t = 0; t < 4; ++t) c = __builtin_amdgcn_mfma_f32_16x16x4f32(a[t], b[t], c, 0, 0, 0);
        return c;
    }
};
template <typename T> using Frag = Vec<T, 16 / sizeof(T)>;

// Where chunk c (16 bytes) of row `row` lies in an LDS tile of `chunks` chunks a row.  64 banks of 4 bytes: the
// lanes that are served together read 16 rows of one chunk (kDepthFast, two rows of 128 bytes side by side), or
// for a transposing read rows 0-3 and 8-11 of a pair of chunks, for 32-bit elements rows 0, 4, 8, 12 of four.
template <typename T, int LAYOUT> __device__ __forceinline__ uint32_t swizzle(uint32_t row, uint32_t c, uint32_t chunks) {
    if constexpr (LAYOUT == kDepthFast) return c ^ ((row >> 1) & 7u);
    else if constexpr (sizeof(T) == 2) return c ^ ((((row & 3u) | (row >> 1 & 4u)) << 1) & (chunks - 1));
    else return c ^ ((row & 12u) & (chunks - 1));
}

// Fragment of 16 free indices from `free` on, step `kk` of the stage: lane l holds free index l % 16 and the
// depth of its quarter l / 16.
template <typename T, int LAYOUT, int FREE> __device__ __forceinline__ Frag<T> fragment(const char* tile, uint32_t free, uint32_t kk) {
    const uint32_t lane = threadIdx.x & 63u, q = lane >> 4, i = lane & 15u;
    if constexpr (LAYOUT == kDepthFast) {
        const uint32_t f = free + i;
        return *(const Frag<T>*)(tile + f * kStageBytes + swizzle<T, LAYOUT>(f, kk * 4 + q, 8) * 16);
    } else if constexpr (sizeof(T) == 2) {
        // ds_read_tr16: in a quarter, lane 4 j + c names four neighbours of row j; lane 4 c + e gets element e
        // of those from rows 0 .. 3
        typedef short s16x4 __attribute__((ext_vector_type(4)));
        constexpr uint32_t kChunks = FREE * sizeof(T) / 16;
        Vec<short, 8> v;
#pragma unroll
        for (int t = 0; t < 2; ++t) {
            const uint32_t d = kk * 32 + q * 8 + t * 4 + (i >> 2), f = free + 4 * (i & 3u);
            const char* const p = tile + d * (FREE * sizeof(T)) + swizzle<T, LAYOUT>(d, f >> 3, kChunks) * 16 + (f & 7u) * 2;
            const s16x4 h = __builtin_amdgcn_ds_read_tr16_b64_v4i16((TPERM_LDS s16x4*)(TPERM_LDS char*)p);
#pragma unroll
            for (int e = 0; e < 4; ++e) v[4 * t + e] = h[e];
        }
        return __builtin_bit_cast(Frag<T>, v);
    } else {
        constexpr uint32_t kChunks = FREE * sizeof(T) / 16;
        Frag<T> v;
#pragma unroll
        for (int t = 0; t < 4; ++t) {
            const uint32_t d = kk * 16 + q * 4 + t, f = free + i;
            v[t] = *(const T*)(tile + d * (FREE * sizeof(T)) + swizzle<T, LAYOUT>(d, f >> 2, kChunks) * 16 + (f & 3u) * 4);
        }
        return v;
    }
}

// --- from memory to LDS, by way of registers: any size, stride and alignment ---

// The operand of one side: a matrix of memory rows.
struct Operand {
    const void* p;
    const uint8_t* scales;
    const int32_t* source;
    int64_t stride;
    uint32_t slots, rows, width;
    __device__ __forceinline__ explicit Operand(const ProductSide& s) : p(s.p), scales(s.scales), source(s.source), stride(s.stride), slots(s.slots), rows(s.rows), width(s.width) {}
    __device__ __forceinline__ Operand(const void* at, uint32_t r, uint32_t w) : p(at), scales(nullptr), source(nullptr), stride(w), slots(1), rows(r), width(w) {}
    // Memory row behind row r of the order; false: there is none.
    __device__ __forceinline__ bool find(uint32_t r, uint32_t* row) const {
        const uint32_t s = source != nullptr ? (uint32_t)source[r] : r;
        *row = source != nullptr ? s / slots : s;
        return s < 1u << 31 && *row < rows;
    }
};

// A stage of FREE free indices x 128 bytes of depth.  `free_end`, `depth_end`: one behind the last index that
// belongs to the tile; what lies beyond becomes zero.
template <typename T, int LAYOUT, int FREE, int THREADS> struct Stage {
    static constexpr int V = 16 / sizeof(T);                                // elements of a chunk in LDS
    static constexpr int kIn = LAYOUT == kCodes ? 16 : V;                   // elements that a thread fetches at once
    static constexpr int kDepth = kStageBytes / sizeof(T);
    static constexpr int kFetches = FREE * kDepth / kIn / THREADS;
    static constexpr int kAcross = (LAYOUT == kDepthFast ? kDepth : FREE) / kIn;
    static_assert(kFetches * kIn * THREADS == FREE * kDepth, "whole passes");
    u32x4 reg[kFetches];
    float scale[LAYOUT == kCodes ? kFetches : 1];

    __device__ __forceinline__ void fetch(const Operand& m, uint32_t free0, uint32_t free_end, uint32_t depth0, uint32_t depth_end) {
#pragma unroll
        for (int p = 0; p < kFetches; ++p) {
            const uint32_t id = threadIdx.x + p * THREADS, other = id / kAcross, along = id % kAcross * kIn;
            const uint32_t f = free0 + (LAYOUT == kDepthFast ? other : along), d = depth0 + (LAYOUT == kDepthFast ? along : other);
            u32x4 v = {};
            uint32_t row;
            if constexpr (LAYOUT == kCodes) scale[p] = 0.0f;
            if (f < free_end && d < depth_end && m.find(LAYOUT == kDepthFast ? f : d, &row)) {
                const int there = (int)(LAYOUT == kDepthFast ? depth_end - d : free_end - f);
                if constexpr (LAYOUT == kCodes) {
                    v = __builtin_bit_cast(u32x4, load_some<uint8_t, 16, false>((const uint8_t*)m.p + (int64_t)row * m.width + f, there));
                    scale[p] = power_of(m.scales[(int64_t)row * ((m.width + 31) / 32) + f / 32]);
                } else {
                    const T* const at = (const T*)m.p + (int64_t)row * m.stride + (LAYOUT == kDepthFast ? d : f);
                    v = __builtin_bit_cast(u32x4, load_some<T, V, false>(at, there));
                }
            }
            reg[p] = v;
        }
    }
    __device__ __forceinline__ void put(char* tile) const {
#pragma unroll
        for (int p = 0; p < kFetches; ++p) {
            const uint32_t id = threadIdx.x + p * THREADS, row = id / kAcross, c = id % kAcross;
            if constexpr (LAYOUT == kCodes) {
                constexpr uint32_t kChunks = FREE * sizeof(T) / 16;
                char* const at = tile + row * (FREE * sizeof(T));
                Vec<T, 16> v;
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    const Vec<T, 8> w = narrow<T, 8>(values_of<T>(u32x2{reg[p][2 * h], reg[p][2 * h + 1]}, scale[p]));
#pragma unroll
                    for (int e = 0; e < 8; ++e) v[8 * h + e] = w[e];
                }
#pragma unroll
                for (int k = 0; k < 16 / V; ++k) {
                    Frag<T> part;
#pragma unroll
                    for (int e = 0; e < V; ++e) part[e] = v[k * V + e];
                    *(Frag<T>*)(at + swizzle<T, LAYOUT>(row, c * (16 / V) + k, kChunks) * 16) = part;
                }
            } else {
                constexpr uint32_t kPitch = LAYOUT == kDepthFast ? kStageBytes : FREE * sizeof(T);
                *(u32x4*)(tile + row * kPitch + swizzle<T, LAYOUT>(row, c, kPitch / 16) * 16) = reg[p];
            }
        }
    }
};

// A workgroup's tile: FAST x SLOW results, four wavefronts, WF of them along the fast side.
template <int FAST_, int SLOW_, int WF_> struct TileShape {
    static constexpr int kFast = FAST_, kSlow = SLOW_, kThreads = 256;
    static constexpr int kWavesFast = WF_, kWavesSlow = 4 / WF_;
    static constexpr int FI = FAST_ / kWavesFast / 16, SI = SLOW_ / kWavesSlow / 16;   // 16 x 16 blocks of a wavefront
};

// Sum over depth0 .. depth_end into acc: lane l holds fast indices 4 (l / 16) .. + 3 and slow index l % 16 of a block.
template <typename T, int FL, int SL, typename S>
__device__ __forceinline__ void sum_tile(char* lds, const Operand& fast, uint32_t fast0, uint32_t fast_end, const Operand& slow, uint32_t slow0, uint32_t slow_end,
                                         uint32_t depth0, uint32_t depth_end, f32x4 (&acc)[S::SI][S::FI]) {
    constexpr uint32_t kDepth = kStageBytes / sizeof(T);
    const uint32_t wave = threadIdx.x >> 6;
    const uint32_t wf = wave % S::kWavesFast * (S::FI * 16), ws = wave / S::kWavesFast * (S::SI * 16);
    char* const ft = lds;
    char* const st = lds + S::kFast * kStageBytes;
    Stage<T, FL, S::kFast, S::kThreads> fs;
    Stage<T, SL, S::kSlow, S::kThreads> ss;
    if (depth0 < depth_end) {
        fs.fetch(fast, fast0, fast_end, depth0, depth_end);
        ss.fetch(slow, slow0, slow_end, depth0, depth_end);
    }
    for (uint32_t d = depth0; d < depth_end; d += kDepth) {
        __syncthreads();
        fs.put(ft);
        ss.put(st);
        __syncthreads();
        if (d + kDepth < depth_end) {
            fs.fetch(fast, fast0, fast_end, d + kDepth, depth_end);
            ss.fetch(slow, slow0, slow_end, d + kDepth, depth_end);
        }
#pragma unroll
        for (uint32_t kk = 0; kk < kDepth / Matrix<T>::kDepth; ++kk) {
            Frag<T> f[S::FI], s[S::SI];
#pragma unroll
            for (int i = 0; i < S::FI; ++i) f[i] = fragment<T, FL, S::kFast>(ft, wf + i * 16, kk);
#pragma unroll
            for (int i = 0; i < S::SI; ++i) s[i] = fragment<T, SL, S::kSlow>(st, ws + i * 16, kk);
#pragma unroll
            for (int j = 0; j < S::SI; ++j)
#pragma unroll
                for (int i = 0; i < S::FI; ++i) acc[j][i] = Matrix<T>::mul(f[i], s[j], acc[j][i]);
        }
    }
}

// Results of a tile to out (stride: between slow indices): rounded once, after what out holds has been
// added with `accumulate`.
template <typename O, typename S>
__device__ __forceinline__ void store_tile(O* out, int64_t stride, uint32_t fast0, uint32_t fast_end, uint32_t slow0, uint32_t slow_end, bool accumulate,
                                           const f32x4 (&acc)[S::SI][S::FI]) {
    const uint32_t wave = threadIdx.x >> 6, lane = threadIdx.x & 63u;
    const uint32_t f0 = fast0 + wave % S::kWavesFast * (S::FI * 16) + (lane >> 4) * 4;
    const uint32_t s0 = slow0 + wave / S::kWavesFast * (S::SI * 16) + (lane & 15u);
#pragma unroll
    for (int j = 0; j < S::SI; ++j) {
        const uint32_t s = s0 + j * 16;
        if (s >= slow_end) continue;
#pragma unroll
        for (int i = 0; i < S::FI; ++i) {
            const uint32_t f = f0 + i * 16;
            if (f >= fast_end) continue;
            O* const p = out + (int64_t)s * stride + f;
            const int there = (int)(fast_end - f);
            f32x4 v = acc[j][i];
            if (accumulate) v += widen<O, 4>(load_some<O, 4, false>(p, there));
            store_some<O, 4, false>(p, narrow<O, 4>(v), there);
        }
    }
}

// --- which tile ---

// Rows from, end of bin b: expert b, or the unused rows for b == experts.  Held to 0 .. rows whatever offsets says.
__device__ __forceinline__ void rows_of(const int32_t* offsets, uint32_t experts, uint32_t rows, uint32_t b, uint32_t* from, uint32_t* end) {
    const uint32_t o = (uint32_t)offsets[b], p = b < experts ? (uint32_t)offsets[b + 1] : rows;
    *end = p < rows ? p : rows;
    *from = o < *end ? o : *end;
}

// The index-th tile of `height` rows over all bins; false: there are fewer.  Every wavefront looks for itself:
// a lane takes neighbouring bins, a scan over the lanes and a ballot find the lane, the rest is uniform.
__device__ __forceinline__ bool find_rows(const int32_t* offsets, uint32_t experts, uint32_t rows, uint32_t height, uint32_t index, uint32_t* bin, uint32_t* from, uint32_t* end) {
    const uint32_t lane = threadIdx.x & 63u, bins = experts + 1, per = (bins + 63) / 64;
    uint32_t n = 0, o, p;
    for (uint32_t i = 0; i < per; ++i)
        if (lane * per + i < bins) {
            rows_of(offsets, experts, rows, lane * per + i, &o, &p);
            n += (p - o + height - 1) / height;
        }
    uint32_t sum = n;
    for (uint32_t d = 1; d < 64; d <<= 1) {
        const uint32_t before = (uint32_t)__shfl_up((int)sum, d);
        if (lane >= d) sum += before;
    }
    const uint64_t at = __ballot(sum > index);
    if (at == 0) return false;
    const int l = __builtin_ctzll(at);
    uint32_t left = index - (uint32_t)__builtin_amdgcn_readlane((int)(sum - n), l);
    for (uint32_t b = (uint32_t)l * per; b < bins; ++b) {
        rows_of(offsets, experts, rows, b, &o, &p);
        const uint32_t tiles = (p - o + height - 1) / height;
        if (left < tiles) {
            *bin = b;
            *from = o + left * height;
            *end = p - *from < height ? p : *from + height;
            return true;
        }
        left -= tiles;
    }
    return false;
}

// --- kernels ---

template <typename T, int WL, typename S>
__global__ __launch_bounds__(S::kThreads) void expert_product_kernel(const ExpertProductArgs a) {
    __shared__ __attribute__((aligned(16))) char lds[(S::kFast + S::kSlow) * kStageBytes];
    const uint32_t across = (a.n + S::kFast - 1) / S::kFast;
    uint32_t bin, row0, row_end;
    if (!find_rows(a.offsets, a.experts, a.rows, S::kSlow, (uint32_t)long_block() / across, &bin, &row0, &row_end)) return;
    const uint32_t col0 = (uint32_t)long_block() % across * S::kFast, col_end = a.n;
    f32x4 acc[S::SI][S::FI] = {};
    if (bin < a.experts) {
        const T* const w = (const T*)a.w + (int64_t)bin * a.k * a.n;
        const Operand fast = WL == kDepthFast ? Operand(w, a.n, a.k) : Operand(w, a.k, a.n);
        sum_tile<T, WL, kDepthFast, S>(lds, fast, col0, col_end, Operand(a.x), row0, row_end, 0, a.k, acc);
    }
    store_tile<T, S>((T*)a.out, a.out_stride, col0, col_end, row0, row_end, false, acc);
}

template <typename T, int FL, int SL, typename S>
__global__ __launch_bounds__(S::kThreads) void weight_gradient_kernel(const WeightGradientArgs a) {
    __shared__ __attribute__((aligned(16))) char lds[(S::kFast + S::kSlow) * kStageBytes];
    const uint32_t tf = (a.fast.width + S::kFast - 1) / S::kFast, ts = (a.slow.width + S::kSlow - 1) / S::kSlow;
    const uint32_t at_tile = (uint32_t)long_block(), expert = at_tile / (tf * ts), tile = at_tile % (tf * ts);
    if (expert >= a.experts) return;
    const uint32_t f0 = tile % tf * S::kFast, s0 = tile / tf * S::kSlow;
    uint32_t from, end;
    rows_of(a.offsets, a.experts, a.rows, expert, &from, &end);
    f32x4 acc[S::SI][S::FI] = {};
    sum_tile<T, FL, SL, S>(lds, Operand(a.fast), f0, a.fast.width, Operand(a.slow), s0, a.slow.width, from, end, acc);
    const int64_t at = (int64_t)expert * a.fast.width * a.slow.width;
    const bool accumulate = a.accumulate != 0;
    if (a.out_type == TPERM_TYPE_F32) store_tile<float, S>((float*)a.out + at, a.fast.width, f0, a.fast.width, s0, a.slow.width, accumulate, acc);
    else if (a.out_type == TPERM_TYPE_F16) store_tile<_Float16, S>((_Float16*)a.out + at, a.fast.width, f0, a.fast.width, s0, a.slow.width, accumulate, acc);
    else store_tile<__bf16, S>((__bf16*)a.out + at, a.fast.width, f0, a.fast.width, s0, a.slow.width, accumulate, acc);
}

template <typename T> hipError_t product_of(const ExpertProductArgs& a, bool w_k_first, hipStream_t stream);
template <typename T> hipError_t gradient_of(const WeightGradientArgs& a, hipStream_t stream);

}  // namespace tperm
