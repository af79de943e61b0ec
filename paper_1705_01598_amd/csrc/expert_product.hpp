// Products of the experts: rows times their expert's matrix, and the gradient to the matrices.
//
// One tile of the result to a workgroup, summed over the whole depth (the summed index) with MFMA, 128 bytes
// of depth to a stage.  A tile has a fast side, whose index runs along memory in the result, and a slow one.
// The operand of a side lies in memory with the depth running fastest (kDepthFast: rows of activations, a
// matrix with the summed index first) or with the side's own index running fastest (kFreeFast: the other layout of
// a matrix; both operands of the gradient, whose depth are the rows of an expert).  LDS holds each as it
// lies in memory: fragments of the first kind are 16-byte reads, of the second transposing ones.
// Chunks of 16 bytes change places inside their LDS row (swizzle()), which leaves bank conflicts 4 % of the LDS's active
// cycles where fragments are read as they lie and 6 % where they are transposed; writing converted codes makes it 19 %.
//
// Sums are binary32, rounded once where they are stored.  Large products are bound by the matrix cores, whose clock falls
// with their load to about 1.7 GHz: a stage of a 256 x 256 bfloat16 tile takes 1.45 us, 1.5 PFLOP/s with all compute units; requesting the
// first stages and storing the tile takes 9 us more, which a workgroup that fills its compute unit cannot hide.  65536
// rows of 32 experts, 2048 x 4096: 985 us, 1.12 PFLOP/s (the library's 8192^3 product: 1.45); one expert of 16384
// rows, 4096 x 8192: 765 to 825 us, 1.33 to 1.44.  Few rows are bound by the matrices: 32 rows of 64 experts 2048 x 1024: 18 to 20 us, 106 MB.
// Two stages in LDS are enough: a third image leaves 128 x 128 tiles one workgroup a compute unit, and 256 x 256 no room.
#pragma once
#include "expert_vector.hpp"
#include "experts.hpp"

#include <type_traits>

namespace tperm {

enum Layout { kDepthFast = 0, kFreeFast = 1, kCodes = 2 };  // kCodes: as kFreeFast, 8-bit codes with scales
constexpr int kStageBytes = 128;                            // depth of a stage in bytes of an element row

#define TPERM_LDS __attribute__((address_space(3)))

// A value that all lanes have, in a scalar register.  Left in a vector register, where a load may leave it, it makes
// branches of lanes of what follows from it, and buffers that are read in a loop over the lanes.
__device__ __forceinline__ uint32_t uniform(uint32_t v) { return (uint32_t)__builtin_amdgcn_readfirstlane((int)v); }

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

// Fragment of 16 free indices from `free` on, step `kk` of the stage: lane l (`lane`) holds free index l % 16 and the
// depth of its quarter l / 16.
template <typename T, int LAYOUT, int FREE> __device__ __forceinline__ Frag<T> fragment(const char* tile, uint32_t free, uint32_t kk, uint32_t lane) {
    const uint32_t q = lane >> 4, i = lane & 15u;
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

// --- operands ---

// The operand of one side: a matrix of memory rows.
struct Operand {
    const void* p;
    const uint8_t* scales;
    const int32_t* source;
    int64_t stride;
    FastDiv slots;
    uint32_t rows, width;
    __device__ __forceinline__ explicit Operand(const ProductSide& s) : p(s.p), scales(s.scales), source(s.source), stride(s.stride), slots(s.slots), rows(s.rows), width(s.width) {}
    __device__ __forceinline__ Operand(const void* at, uint32_t r, uint32_t w) : p(at), scales(nullptr), source(nullptr), stride(w), slots{}, rows(r), width(w) {}
    // Memory row behind row r of the order; false: there is none.
    __device__ __forceinline__ bool find(uint32_t r, uint32_t* row) const {
        const uint32_t s = source != nullptr ? (uint32_t)source[r] : r;
        *row = source != nullptr ? fdiv(s, slots) : s;      // right for s < 2^31
        return s < 1u << 31 && *row < rows;
    }
};

// A workgroup's tile: FAST x SLOW results, WAVES wavefronts, WF of them along the fast side, two images of a stage in LDS.
// GROUPS such sets of wavefronts and images each take a piece of the depth; their sums are joined in order.
template <int FAST_, int SLOW_, int WAVES, int WF_, int GROUPS = 1> struct TileShape {
    static constexpr int kImage = (FAST_ + SLOW_) * kStageBytes, kGroups = GROUPS, kLds = 2 * GROUPS * kImage;
    static constexpr int kFast = FAST_, kSlow = SLOW_, kThreads = WAVES * 64, kAllThreads = GROUPS * kThreads;     // kThreads: of a group
    static __device__ __forceinline__ uint32_t wave(uint32_t thread) { return thread % kThreads >> 6; }
    static __device__ __forceinline__ uint32_t group() { return uniform(threadIdx.x / kThreads); }
    static constexpr int kWavesFast = WF_, kWavesSlow = WAVES / WF_;
    static constexpr int FI = FAST_ / kWavesFast / 16, SI = SLOW_ / kWavesSlow / 16;   // 16 x 16 blocks of a wavefront
};

// Fragments of one step of a stage, and their products: lane l of a 16 x 16 block of the result holds fast indices
// 4 (l / 16) .. + 3 and slow index l % 16.
constexpr uint32_t kSteps = 2;      // steps of a stage, whatever the type
template <typename T, int FL, int SL, typename S> struct Step {
    static_assert(kStageBytes / sizeof(T) == kSteps * Matrix<T>::kDepth, "two steps");
    Frag<T> f[S::FI], s[S::SI];
    __device__ __forceinline__ void read(uint32_t thread, const char* image, uint32_t kk) {
        const uint32_t wave = S::wave(thread), lane = thread & 63u;
        const uint32_t wf = wave % S::kWavesFast * (S::FI * 16), ws = wave / S::kWavesFast * (S::SI * 16);
#pragma unroll
        for (int i = 0; i < S::SI; ++i) s[i] = fragment<T, SL, S::kSlow>(image + S::kFast * kStageBytes, ws + i * 16, kk, lane);
#pragma unroll
        for (int i = 0; i < S::FI; ++i) f[i] = fragment<T, FL, S::kFast>(image, wf + i * 16, kk, lane);
    }
    __device__ __forceinline__ void multiply(f32x4 (&acc)[S::SI][S::FI]) const {
#pragma unroll
        for (int i = 0; i < S::FI; ++i) multiply(acc, i);
    }
    // The i-th of FI parts of either.
    __device__ __forceinline__ void read(uint32_t thread, const char* image, uint32_t kk, int part) {
        const uint32_t wave = S::wave(thread), lane = thread & 63u;
        const uint32_t wf = wave % S::kWavesFast * (S::FI * 16), ws = wave / S::kWavesFast * (S::SI * 16);
#pragma unroll
        for (int i = 0; i < S::SI; ++i)
            if (i * S::FI / S::SI == part) s[i] = fragment<T, SL, S::kSlow>(image + S::kFast * kStageBytes, ws + i * 16, kk, lane);
        f[part] = fragment<T, FL, S::kFast>(image, wf + part * 16, kk, lane);
    }
    __device__ __forceinline__ void multiply(f32x4 (&acc)[S::SI][S::FI], int i) const {
#pragma unroll
        for (int j = 0; j < S::SI; ++j) acc[j][i] = Matrix<T>::mul(f[i], s[j], acc[j][i]);
    }
};

// --- from memory straight to LDS: rows of whole 16-byte chunks that start on 16 bytes ---

constexpr uint32_t kBeyond = 0xFFFFFF00u;   // lane offset behind every buffer: the access writes zeros to LDS

__device__ __forceinline__ __amdgpu_buffer_rsrc_t buffer_at(const void* p) {
    const uint64_t at = (uint64_t)p, same = (uint64_t)uniform((uint32_t)(at >> 32)) << 32 | uniform((uint32_t)at);
    return __builtin_amdgcn_make_buffer_rsrc((void*)same, 0, (int)kBeyond, 0x00020000);
}

// 16 bytes a lane from base + offset + scalar to 1 KiB of LDS from `to` on.  Written out: behind the builtin the
// compiler lets the next transposing read, of another image, wait for all loads (2.1 us a stage instead of 1.4).  It
// has no result for the compiler to see: arrive() waits for it, and what keeps it behind the reads of the image that it
// overwrites is the "memory" of arrive() alone.  What it reads comes from settled() and scalar arithmetic.
__device__ __forceinline__ void load_to_lds(uint64_t base, uint32_t to, uint32_t offset, uint32_t scalar) {
    const u32x4 buffer = {(uint32_t)base, (uint32_t)(base >> 32) & 0xFFFFu, kBeyond, 0x00020000u};
    asm volatile("s_nop 0\n\tbuffer_load_dwordx4 %1, %2, %3 offen lds" ::"{m0}"(to), "v"(offset), "s"(buffer), "s"(scalar));
}

// Values that all lanes have, in scalar registers that such a load may read: five wait states after a vector instruction wrote
// them at the earliest, and the compiler counts none for instructions that are written out.  Here they pass once for a
// tile; with every load, or every stage, the products lose 1 to 4 % of a call.
__device__ __forceinline__ void settled(uint64_t& base, uint32_t& row_bytes, uint32_t& to) {
    base = (uint64_t)uniform((uint32_t)(base >> 32)) << 32 | uniform((uint32_t)base), row_bytes = uniform(row_bytes), to = uniform(to);
    asm volatile("s_nop 4" : "+s"(base), "+s"(row_bytes), "+s"(to));
}

// Waits until at most LOADS of this wavefront's loads are under way and its LDS accesses are done, then for the other
// wavefronts to do so.
template <int LOADS> __device__ __forceinline__ void arrive() {
    __builtin_amdgcn_sched_barrier(0);
    asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" ::"n"(LOADS) : "memory");
    __builtin_amdgcn_sched_barrier(0);
}

// The operand of one side.  A lane's 16 bytes arrive at a place in LDS that its number fixes, so the swizzle is
// applied to where it reads.  MAPPED: depth rows (kFreeFast) are found through source, one stage ahead.
template <typename T, int LAYOUT, int FREE, int THREADS, bool MAPPED> struct Direct {
    uint32_t me;        // of THREADS
    static constexpr int V = 16 / sizeof(T);
    static constexpr uint32_t kDepth = kStageBytes / sizeof(T);
    static constexpr int kFetches = FREE * kStageBytes / 16 / THREADS;
    static constexpr uint32_t kAcross = LAYOUT == kDepthFast ? 8 : FREE * sizeof(T) / 16;   // chunks of an LDS row
    static constexpr uint32_t kRowsPerFetch = THREADS / kAcross;
    static_assert(kFetches * THREADS * 16 == FREE * kStageBytes && kRowsPerFetch * kAcross == THREADS, "whole passes");
    uint64_t base;
    uint32_t row_bytes, to;             // to: of the wavefront's part of an image
    uint32_t off[kFetches];             // from base (kDepthFast: + depth; kFreeFast: + stage, MAPPED: of the column alone)
    // MAPPED: memory rows that a wavefront's lanes read in each fetch; two are kept in scalar registers (the 16 a
    // stage of narrower tiles take longer than a look-up by every lane: 35 us against 25, 2048 rows of 8 experts)
    static constexpr int kRowsPerWave = 64 / kAcross;
    static constexpr bool kScalar = kRowsPerWave <= 2;
    uint32_t row[MAPPED ? kFetches : 1][MAPPED && kScalar ? kRowsPerWave : 1];
    const int32_t* source;
    FastDiv slots;
    uint32_t rows;

    __device__ __forceinline__ uint32_t lds_row(int p) const { return me / kAcross + (uint32_t)p * kRowsPerFetch; }
    __device__ __forceinline__ uint32_t chunk(int p) const { return swizzle<T, LAYOUT>(lds_row(p), me % kAcross, kAcross); }

    // Depth-fast: rows free0 .. free_end of m, whose row r is m.find(r).
    __device__ __forceinline__ void start(uint32_t thread, const Operand& m, uint32_t free0, uint32_t free_end) {
        me = thread % THREADS;
        row_bytes = (uint32_t)(m.stride * sizeof(T));
        source = m.source, slots = m.slots, rows = m.rows;
        if constexpr (LAYOUT == kDepthFast) {
            base = (uint64_t)m.p + (m.source != nullptr ? 0 : (uint64_t)free0 * row_bytes);
#pragma unroll
            for (int p = 0; p < kFetches; ++p) {
                uint32_t r = free0 + lds_row(p), at;
                off[p] = kBeyond;
                if (r < free_end && m.find(r, &at)) off[p] = (m.source != nullptr ? at : at - free0) * row_bytes + chunk(p) * 16;
            }
        } else {
            base = (uint64_t)m.p;
#pragma unroll
            for (int p = 0; p < kFetches; ++p) {
                const uint32_t f = free0 + chunk(p) * V;
                off[p] = f < free_end ? f * (uint32_t)sizeof(T) + (MAPPED ? 0u : lds_row(p) * row_bytes) : kBeyond;
            }
        }
        to = (me & ~63u) * 16;
        settled(base, row_bytes, to);
    }
    // MAPPED: entries of source for the stage at `depth0`.
    __device__ __forceinline__ void look_up(uint32_t depth0, uint32_t depth_end) {
        if constexpr (MAPPED && !kScalar) {
#pragma unroll
            for (int p = 0; p < kFetches; ++p) {
                const uint32_t d = depth0 + lds_row(p);
                row[p][0] = (uint32_t)source[d < depth_end ? d : depth_end - 1];
            }
        } else if constexpr (MAPPED) {
            typedef const __attribute__((address_space(4))) int32_t* Scalar;
            const uint32_t first = depth0 + uniform(me >> 6) * kRowsPerWave;
#pragma unroll
            for (int p = 0; p < kFetches; ++p)
#pragma unroll
                for (int i = 0; i < kRowsPerWave; ++i) {
                    const uint32_t d = first + p * kRowsPerFetch + i;
                    row[p][i] = (uint32_t)((Scalar)(uintptr_t)source)[d < depth_end ? d : depth_end - 1];
                }
        }
    }
    // Looked-up entries are here from now on.  The compiler does not see load_to_lds(): left to it, the waits for the
    // entries come between a stage's loads and wait for those too (2048 rows of 8 experts 34 us instead of 25).
    __device__ __forceinline__ void looked_up() const {
        if constexpr (MAPPED && !kScalar)
#pragma unroll
            for (int p = 0; p < kFetches; ++p) asm volatile("" ::"v"(row[p][0]));
    }
    __device__ __forceinline__ void issue(char* tile, uint32_t depth0, uint32_t depth_end, int part = 0, int parts = 1) {
        const uint32_t left = depth0 < depth_end ? depth_end - depth0 : 0;      // beyond the end: zeros
        const uint32_t at_lds = (uint32_t)(uintptr_t)(TPERM_LDS char*)tile + to;
        uint64_t from = base;
        uint32_t scalar = 0;
        if constexpr (LAYOUT == kDepthFast) scalar = depth0 * (uint32_t)sizeof(T);
        else if constexpr (!MAPPED) from += (uint64_t)depth0 * row_bytes;
#pragma unroll
        for (int p = 0; p < kFetches; ++p) {
            if (p * parts / kFetches != part) continue;
            uint32_t o = off[p];
            if constexpr (LAYOUT == kDepthFast) {
                if (left < kDepth) o = chunk(p) * V < left ? o : kBeyond;
            } else if constexpr (MAPPED && !kScalar) {
                const uint32_t at = fdiv(row[p][0], slots);
                const bool use = (lds_row(p) < left) & (row[p][0] < 1u << 31) & (at < rows) & (o != kBeyond);     // without branches
                o = use ? at * row_bytes + o : kBeyond;
            } else if constexpr (MAPPED) {
                const uint32_t in_wave = (me & 63u) / kAcross;
                uint32_t start = 0;
#pragma unroll
                for (int i = 0; i < kRowsPerWave; ++i) {
                    const uint32_t at = fdiv(row[p][i], slots);
                    const uint32_t d = uniform(me >> 6) * kRowsPerWave + p * kRowsPerFetch + i;
                    const bool use = (d < left) & (row[p][i] < 1u << 31) & (at < rows);
                    const uint32_t one = use ? at * row_bytes : kBeyond;
                    start = in_wave == (uint32_t)i ? one : start;
                }
                o = __builtin_elementwise_add_sat(start, o);     // kBeyond and more stays behind the buffer
            } else {
                if (left < kDepth) o = lds_row(p) < left ? o : kBeyond;
            }
            load_to_lds(from, at_lds + p * THREADS * 16, o, scalar);
        }
    }
    __device__ __forceinline__ void put(char*) const {}     // it goes there by itself
};

// Up to 16 bytes from q on of a tensor that ends at `end`: `there` elements exist, the others become zero.
template <typename E> __device__ __forceinline__ u32x4 fetch_some(const E* q, int there, const char* end) {
    constexpr int V = 16 / sizeof(E);
    u32x4 v = {};
    if (there > 0) {
        if ((const char*)q + 16 <= end) {
            __builtin_memcpy(&v, q, 16);
            if (there < V) {
#pragma unroll
                for (int w = 0; w < 4; ++w) {
                    const int bits = (there * (int)sizeof(E) - 4 * w) * 8;
                    v[w] = bits >= 32 ? v[w] : bits <= 0 ? 0u : v[w] & ((1u << bits) - 1u);
                }
            }
        } else {
            E e[V] = {};
#pragma unroll
            for (int i = 0; i < V; ++i)
                if (i < there) e[i] = q[i];
            __builtin_memcpy(&v, e, 16);
        }
    }
    return v;
}

// Sides of 64 16-bit elements keep the branches, which leave out rows that are not there (us with and without them: 1001 x 1003,
// 25 rows of an expert 14.7 15.7; gradient of 125 rows, 333 x 555, 17.1 19.0), wider ones do without (gradient of 1024
// rows, 1001 x 1003, 121 78; product of 1024 rows, 2001 x 2003, 208 184).
template <typename T, int FREE> constexpr bool kMoved = FREE * sizeof(T) > 128;

// The same of a row that has 16 bytes at least, without a branch, behind which the compiler would wait for the load: where
// fewer than that are left, the row's last 16 bytes, which straighten() puts right.  left <= 0: any bytes, from `base`.
template <typename E> __device__ __forceinline__ u32x4 fetch_moved(const E* q, int left, const void* base) {
    constexpr int V = 16 / sizeof(E);
    const E* const at = left > 0 ? q - (left < V ? V - left : 0) : (const E*)base;
    u32x4 v;
    __builtin_memcpy(&v, at, 16);
    return v;
}
template <typename E> __device__ __forceinline__ u32x4 straighten(u32x4 v, int left) {
    constexpr int V = 16 / sizeof(E);
    if (left < V) {
        const unsigned __int128 all = __builtin_bit_cast(unsigned __int128, v);
        v = __builtin_bit_cast(u32x4, left > 0 ? all >> ((V - left) * (int)sizeof(E) * 8) : (unsigned __int128)0);
    }
    return v;
}

// The operand of one side, of any size, stride and alignment, by way of registers: requested while the stage before is
// multiplied, put to LDS behind that.
template <typename T, int LAYOUT, int FREE, int THREADS> struct Loose {
    uint32_t me;        // of THREADS
    static constexpr int V = 16 / sizeof(T);
    static constexpr uint32_t kDepth = kStageBytes / sizeof(T);
    static constexpr int kFetches = FREE * kStageBytes / 16 / THREADS;
    static constexpr uint32_t kAcross = LAYOUT == kDepthFast ? 8 : FREE * sizeof(T) / 16;
    static constexpr uint32_t kRowsPerFetch = THREADS / kAcross;
    static_assert(kFetches * THREADS * 16 == FREE * kStageBytes && kRowsPerFetch * kAcross == THREADS, "whole passes");
    const char *base, *end;
    int64_t row_bytes;
    const char* at[LAYOUT == kDepthFast ? kFetches : 1];    // a row's chunk, without the depth; NULL: no such row
    uint32_t row[LAYOUT == kDepthFast ? 1 : kFetches];
    const int32_t* source;
    FastDiv slots;
    uint32_t rows, free, free_end;
    u32x4 reg[kFetches];
    bool moved;         // rows have 16 bytes
    uint32_t left;      // elements of each fetch that exist, a byte each
    static_assert(kFetches <= 4, "a word");

    __device__ __forceinline__ uint32_t lds_row(int p) const { return me / kAcross + (uint32_t)p * kRowsPerFetch; }
    __device__ __forceinline__ void start(uint32_t thread, const Operand& m, uint32_t free0, uint32_t free_end_) {
        me = thread % THREADS;
        base = (const char*)m.p, row_bytes = m.stride * (int64_t)sizeof(T);
        end = base + ((int64_t)m.rows - 1) * row_bytes + (int64_t)m.width * (int64_t)sizeof(T);
        source = m.source, slots = m.slots, rows = m.rows, moved = kMoved<T, FREE> && m.rows > 0 && m.width >= (uint32_t)V;
        if constexpr (LAYOUT == kDepthFast) {
#pragma unroll
            for (int p = 0; p < kFetches; ++p) {
                uint32_t r = free0 + lds_row(p), to;
                at[p] = r < free_end_ && m.find(r, &to) ? base + to * row_bytes + me % kAcross * 16 : nullptr;
            }
        } else {
            free = free0 + me % kAcross * V, free_end = free_end_;
        }
    }
    __device__ __forceinline__ void look_up(uint32_t depth0, uint32_t depth_end) {
        if constexpr (LAYOUT != kDepthFast)
#pragma unroll
            for (int p = 0; p < kFetches; ++p) {
                const uint32_t d = depth0 + lds_row(p);
                row[p] = d >= depth_end ? 0xFFFFFFFFu : source != nullptr ? (uint32_t)source[d] : d;
            }
    }
    __device__ __forceinline__ void looked_up() const {}
    __device__ __forceinline__ void issue(char*, uint32_t depth0, uint32_t depth_end) {
        left = 0;
        const char* q[kFetches];
        int n[kFetches];
#pragma unroll
        for (int p = 0; p < kFetches; ++p) {
            uint32_t exist;
            if constexpr (LAYOUT == kDepthFast) {
                const uint32_t d = depth0 + me % kAcross * V;
                q[p] = at[p] + (uint64_t)depth0 * sizeof(T);
                exist = ((at[p] != nullptr) & (d < depth_end)) ? depth_end - d : 0;
            } else {
                const uint32_t to = source != nullptr ? fdiv(row[p], slots) : row[p];
                q[p] = base + to * row_bytes + (uint64_t)free * sizeof(T);
                exist = ((row[p] < 1u << 31) & (to < rows) & (free < free_end)) ? free_end - free : 0;
            }
            n[p] = (int)(exist < (uint32_t)V ? exist : (uint32_t)V);
            left |= (uint32_t)n[p] << (8 * p);
        }
        if (moved) {
#pragma unroll
            for (int p = 0; p < kFetches; ++p) reg[p] = fetch_moved((const T*)q[p], n[p], base);
        } else {
            left = 0x01010101u * V;
#pragma unroll
            for (int p = 0; p < kFetches; ++p) reg[p] = fetch_some((const T*)q[p], n[p], end);
        }
    }
    __device__ __forceinline__ void put(char* tile) const {
        __builtin_amdgcn_sched_barrier(0);      // not before the products: it would wait for the loads there
        constexpr uint32_t kPitch = LAYOUT == kDepthFast ? kStageBytes : FREE * sizeof(T);
#pragma unroll
        for (int p = 0; p < kFetches; ++p)
            *(u32x4*)(tile + lds_row(p) * kPitch + swizzle<T, LAYOUT>(lds_row(p), me % kAcross, kAcross) * 16) = straighten<T>(reg[p], (int)(left >> (8 * p) & 0xFFu));
    }
};

// 8 codes as elements; `safe`: the scale cannot carry them beyond the type's range.
template <typename T> __device__ __forceinline__ Vec<T, 8> elements_of(u32x2 codes, float scale, bool safe) {
    if constexpr (sizeof(T) == 2) {
        if (safe) {
            Vec<T, 8> v;
#pragma unroll
            for (int h = 0; h < 2; ++h)
#pragma unroll
                for (int k = 0; k < 2; ++k) {
                    Vec<T, 2> e;
                    if constexpr (__is_same(T, __bf16)) e = k ? __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(codes[h], scale, true) : __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(codes[h], scale, false);
                    else e = k ? __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(codes[h], scale, true) : __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(codes[h], scale, false);
                    v[4 * h + 2 * k] = e[0], v[4 * h + 2 * k + 1] = e[1];
                }
            return v;
        }
    }
    return narrow<T, 8>(values_of<T>(codes, scale));
}

// The operand of one side kept in codes: through registers, where codes become elements.  A stage is fetched while the one
// before it is multiplied, its rows looked up one stage before that.  LOOSE: rows of any length and alignment;
// else of whole 16-byte chunks that start on 16 bytes.
template <typename T, int FREE, int THREADS, bool MAPPED, bool LOOSE> struct Coded {
    uint32_t me;        // of THREADS
    static constexpr uint32_t kDepth = kStageBytes / sizeof(T);
    static constexpr uint32_t kAcross = FREE / 16, kRowsPerFetch = THREADS / kAcross;
    // a stage of few 32-bit columns is less than one fetch: the last threads have nothing to do
    static constexpr int kFetches = kRowsPerFetch > kDepth ? 1 : kDepth / kRowsPerFetch;
    static_assert(kFetches * kRowsPerFetch >= kDepth && kRowsPerFetch * kAcross == THREADS, "whole passes");
    const uint8_t *codes, *scales;
    const int32_t* source;
    uint32_t width, blocks, rows, free;
    int free_there;     // elements from `free` to the row's end, 16 at most
    bool moved;         // LOOSE: rows have 16 codes
    uint32_t left;      // LOOSE: codes of each fetch that exist, a byte each
    static_assert(kFetches <= 4, "a word");
    FastDiv slots;
    bool there;
    uint32_t row[MAPPED ? kFetches : 1];
    u32x4 reg[kFetches];
    uint32_t scale[kFetches];

    __device__ __forceinline__ uint32_t lds_row(int p) const { return me / kAcross + (uint32_t)p * kRowsPerFetch; }
    __device__ __forceinline__ void start(uint32_t thread, const Operand& m, uint32_t free0, uint32_t free_end) {
        me = thread % THREADS;
        free = free0 + me % kAcross * 16;
        there = free < free_end && lds_row(0) < kDepth, free_there = free < free_end ? (int)(free_end - free < 16 ? free_end - free : 16) : 0;
        moved = kMoved<T, FREE> && m.rows > 0 && m.width >= 16;
        codes = (const uint8_t*)m.p, scales = m.scales, source = m.source;
        width = m.width, blocks = (m.width + 31) / 32, slots = m.slots, rows = m.rows;
    }
    __device__ __forceinline__ void look_up(uint32_t depth0, uint32_t depth_end) {
        if constexpr (MAPPED)
#pragma unroll
            for (int p = 0; p < kFetches; ++p) row[p] = there && depth0 + lds_row(p) < depth_end ? (uint32_t)source[depth0 + lds_row(p)] : 0xFFFFFFFFu;
    }
    __device__ __forceinline__ void looked_up() const {     // before the other side's loads, as above
        if constexpr (MAPPED)
#pragma unroll
            for (int p = 0; p < kFetches; ++p) asm volatile("" ::"v"(row[p]));
    }
    __device__ __forceinline__ void issue(char*, uint32_t depth0, uint32_t depth_end) {
        // rows that are not looked up are reached from the stage's first one: no limit to the tensor
        const uint64_t from = MAPPED ? 0 : depth0;
        left = 0;
        const __amdgpu_buffer_rsrc_t c = buffer_at(codes + from * width), s = buffer_at(scales + from * blocks);
#pragma unroll
        for (int p = 0; p < kFetches; ++p) {
            const uint32_t at = MAPPED ? fdiv(row[p], slots) : lds_row(p);
            const bool use = there & (MAPPED ? (row[p] < 1u << 31) & (at < rows) : depth0 + at < depth_end);
            const uint32_t code = at * width + free, scale_at = at * blocks + free / 32;
            if constexpr (LOOSE) {
                const uint8_t* const q = codes + (from + at) * width + free;
                const int n = use ? free_there : 0;
                left |= (uint32_t)n << (8 * p);
                reg[p] = moved ? fetch_moved(q, n, codes) : fetch_some(q, n, (const char*)codes + (uint64_t)rows * width);
            } else reg[p] = __builtin_amdgcn_raw_buffer_load_b128(c, (int)(use ? code : kBeyond), 0, 0);
            scale[p] = __builtin_amdgcn_raw_buffer_load_b8(s, (int)(use ? scale_at : kBeyond), 0, 0);
        }
    }
    __device__ __forceinline__ void put(char* tile) const {
        constexpr uint32_t kChunks = FREE * sizeof(T) / 16;
        __builtin_amdgcn_sched_barrier(0);      // not before the products: it would wait for the codes there
#pragma unroll
        for (int p = 0; p < kFetches; ++p) {
            const uint32_t d = lds_row(p), c = me % kAcross;
            if (kRowsPerFetch > kDepth && d >= kDepth) return;
            char* const at = tile + d * (FREE * sizeof(T));
            const float by = power_of(scale[p]);
            const bool safe = __ballot(by > Range<T>::kSafe) == 0;
            const u32x4 code = LOOSE && moved ? straighten<uint8_t>(reg[p], (int)(left >> (8 * p) & 0xFFu)) : reg[p];
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const Vec<T, 8> v = elements_of<T>(u32x2{code[2 * h], code[2 * h + 1]}, by, safe);
                if constexpr (sizeof(T) == 2) {
                    *(Vec<T, 8>*)(at + swizzle<T, kFreeFast>(d, 2 * c + h, kChunks) * 16) = v;
                } else {
#pragma unroll
                    for (int k = 0; k < 2; ++k)
                        *(f32x4*)(at + swizzle<T, kFreeFast>(d, 4 * c + 2 * h + k, kChunks) * 16) = f32x4{(float)v[4 * k], (float)v[4 * k + 1], (float)v[4 * k + 2], (float)v[4 * k + 3]};
                }
            }
        }
    }
};

// Order for the compiler's scheduler, which would move the reads of the next step behind the products of this one to
// save registers: READS LDS reads spread over PRODUCTS matrix instructions.
template <int READS, int PRODUCTS> __device__ __forceinline__ void interleave() {
    constexpr int kEach = PRODUCTS / READS > 0 ? PRODUCTS / READS : 1;
#pragma unroll
    for (int i = 0; i < READS; ++i) {
        __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);
        __builtin_amdgcn_sched_group_barrier(0x8, kEach, 0);
    }
    __builtin_amdgcn_sched_barrier(0);
}

// The sum of a tile, over depth0 .. depth_end.  begin() requests the first stages, multiply() adds up.  While the matrix
// cores work on one step, the fragments of the next one are read; the only barrier of a stage stands between its two
// steps: all wavefronts have read the stage's last fragments then, so its image can receive another stage.
//
// LOOSE: operands of any size and alignment.  Two sets of fragments beside operands in registers (those, and codes) do
// not fit: there the other wavefront of the SIMD multiplies while this one reads.
template <typename T, int LAYOUT, int FREE, int THREADS, bool MAPPED, bool LOOSE>
using Side = std::conditional_t<LAYOUT == kCodes, Coded<T, FREE, THREADS, MAPPED, LOOSE>, std::conditional_t<LOOSE, Loose<T, LAYOUT, FREE, THREADS>, Direct<T, LAYOUT, FREE, THREADS, MAPPED>>>;
template <typename T, int FL, int SL, bool FM, bool SM, typename S, bool LOOSE> struct Sum {
    static constexpr uint32_t kDepth = kStageBytes / sizeof(T), kImage = S::kImage;
    static constexpr bool kRegisters = LOOSE || FL == kCodes || SL == kCodes;      // operands pass through them
    static constexpr bool kOrdered = sizeof(T) == 2;
    static constexpr int kReads = S::FI * (FL == kDepthFast ? 1 : 2) + S::SI * (SL == kDepthFast ? 1 : 2), kProducts = S::FI * S::SI;
    char* lds;
    uint32_t depth0, depth_end, stages, thread;
    Side<T, FL, S::kFast, S::kThreads, FM, LOOSE> fs;
    Side<T, SL, S::kSlow, S::kThreads, SM, LOOSE> ss;

    __device__ __forceinline__ void looked_up() {
        fs.looked_up();
        ss.looked_up();
    }
    __device__ __forceinline__ void issue(uint32_t image, uint32_t d) {
        looked_up();
        fs.issue(lds + image, d, depth_end);
        ss.issue(lds + image + S::kFast * kStageBytes, d, depth_end);
    }
    __device__ __forceinline__ void look_up(uint32_t d) {
        fs.look_up(d, depth_end);
        ss.look_up(d, depth_end);
    }
    __device__ __forceinline__ void put(uint32_t image) {
        fs.put(lds + image);
        ss.put(lds + image + S::kFast * kStageBytes);
    }
    // The images are free: no wavefront reads them any more.
    __device__ __forceinline__ void begin(char* images, const Operand& fast, uint32_t fast0, uint32_t fast_end, const Operand& slow, uint32_t slow0,
                                          uint32_t slow_end, uint32_t from, uint32_t end) {
        lds = images, depth0 = from, depth_end = end, stages = 0, thread = threadIdx.x;
        if (depth0 >= depth_end) return;
        stages = (depth_end - depth0 + kDepth - 1) / kDepth;
        if constexpr (S::kGroups > 1) {
            // every group the same number of stages, since all meet at the barriers: those beyond the end are zeros
            stages = (stages + S::kGroups - 1) / S::kGroups;
            depth0 += S::group() * stages * kDepth;
            depth_end = depth_end - (depth0 < depth_end ? depth0 : depth_end) < stages * kDepth ? depth_end : depth0 + stages * kDepth;
            lds += S::group() * 2 * kImage;
        }
        fs.start(thread, fast, fast0, fast_end);
        if constexpr (kRegisters || SM) ss.start(thread, slow, slow0, slow_end);
        look_up(depth0);
        // the fast side's first stage travels while the slow side's rows are looked up
        fs.issue(lds, depth0, depth_end);
        if constexpr (!kRegisters && !SM) ss.start(thread, slow, slow0, slow_end);
        ss.issue(lds + S::kFast * kStageBytes, depth0, depth_end);
        look_up(depth0 + kDepth);
        if constexpr (!kRegisters) {
            issue(kImage, depth0 + kDepth);
            look_up(depth0 + 2 * kDepth);
        }
    }
    __device__ __forceinline__ void multiply(f32x4 (&acc)[S::SI][S::FI]) {
        if (stages == 0) return;
        if constexpr (kRegisters) {
            put(0);
            for (uint32_t d = depth0, image = 0; stages > 0; --stages, d += kDepth, image ^= kImage) {
                arrive<0>();
                issue(image ^ kImage, d + kDepth);
                look_up(d + 2 * kDepth);
#pragma unroll
                for (uint32_t kk = 0; kk < kSteps; ++kk) {
                    Step<T, FL, SL, S> step;
                    step.read(thread, lds + image, kk);
                    step.multiply(acc);
                }
                put(image ^ kImage);
            }
        } else {
            constexpr int kLoads = decltype(fs)::kFetches + decltype(ss)::kFetches;     // of a stage
            arrive<kLoads>();
            uint32_t image = 0;
            Step<T, FL, SL, S> even, odd;
            even.read(thread, lds, 0);
            for (uint32_t d = depth0; stages > 1; --stages, d += kDepth) {
                odd.read(thread, lds + image, 1);
                even.multiply(acc);
                if constexpr (kOrdered) interleave<kReads, kProducts>();
                arrive<0>();        // the next stage has arrived
                // requests, reads and products in turn: behind each other the requests would hold up the products
                const uint32_t free_image = image;
                looked_up();
                image ^= kImage;
#pragma unroll
                for (int i = 0; i < S::FI; ++i) {
                    fs.issue(lds + free_image, d + 2 * kDepth, depth_end, i, S::FI);
                    ss.issue(lds + free_image + S::kFast * kStageBytes, d + 2 * kDepth, depth_end, i, S::FI);
                    even.read(thread, lds + image, 0, i);
                    odd.multiply(acc, i);
                    __builtin_amdgcn_sched_barrier(0);
                }
                look_up(d + 3 * kDepth);
            }
            odd.read(thread, lds + image, 1);
            even.multiply(acc);
            odd.multiply(acc);
        }
        arrive<0>();            // nothing travels to LDS when it is used again
        if constexpr (S::kGroups > 1) {
            // the sums of the others to the first group, in the groups' order
            f32x4* const sums = (f32x4*)(lds - S::group() * 2 * kImage);
#pragma unroll
            for (int g = 1; g < S::kGroups; ++g) {
                if (S::group() == (uint32_t)g)
#pragma unroll
                    for (int i = 0; i < S::SI * S::FI; ++i) sums[i * S::kThreads + threadIdx.x % S::kThreads] = acc[i / S::FI][i % S::FI];
                __syncthreads();
                if (S::group() == 0)
#pragma unroll
                    for (int i = 0; i < S::SI * S::FI; ++i) acc[i / S::FI][i % S::FI] += sums[i * S::kThreads + threadIdx.x % S::kThreads];
                __syncthreads();
            }
        }
    }
};

// Results of a tile to out (stride: between slow indices): rounded once, after what out holds has been added with
// ACCUMULATE.  A lane's own results are pieces of 4 of 16 rows; every wavefront brings them into rows by way of a
// piece of LDS that it alone uses (L: the type there, O or binary32), whose chunks of 16 bytes change places by their
// row, so that the pieces meet no bank conflicts.  A block of 16 rows is written while the one before is stored.
// WHOLE: rows of out are whole chunks that start on 16 bytes.
template <typename O, typename L, typename S, bool WHOLE, bool ACCUMULATE>
__device__ __forceinline__ void store_rows(char* lds, O* out, int64_t stride, uint32_t fast0, uint32_t fast_end, uint32_t slow0, uint32_t slow_end,
                                           const f32x4 (&acc)[S::SI][S::FI]) {
    constexpr uint32_t V = 16 / sizeof(O), kPitch = S::FI * 16 * sizeof(L), kRowChunks = kPitch / 16, kLane = V * sizeof(L) / 16;
    constexpr uint32_t kAcross = S::FI * 16 / V, kDown = 64 / kAcross;      // lanes to a row, rows at once
    static_assert(S::kThreads / 64 * 16 * kPitch <= (uint32_t)S::kLds && kRowChunks <= 16 && 16 % kDown == 0, "a wavefront's LDS");
    constexpr uint32_t kPiece = 16 * kPitch;
    const uint32_t wave = S::wave(threadIdx.x), lane = threadIdx.x & 63u;
    lds += wave * kPiece;
    fast0 += wave % S::kWavesFast * (S::FI * 16), slow0 += wave / S::kWavesFast * (S::SI * 16);
    const auto chunk = [](uint32_t row, uint32_t c) { return row * kPitch + (c ^ ((row * kRowChunks / 16) & (kRowChunks - 1))) * 16; };
    const uint32_t f = fast0 + lane % kAcross * V, down = lane / kAcross;
    O* p = out + (int64_t)(slow0 + down) * stride + f;
    Vec<L, V> l[16 / kDown];
    const auto store = [&](uint32_t j) {
#pragma unroll
        for (uint32_t t = 0; t < 16 / kDown; ++t, p += kDown * stride) {
            const int there = (int)(fast_end - f);
            if (slow0 + j * 16 + t * kDown + down >= slow_end || f >= fast_end) continue;
            Vec<O, V> v;
            if constexpr (sizeof(L) == 4) {
                if constexpr (ACCUMULATE) l[t] += widen<O, V>(load_some<O, V, WHOLE>(p, there));
                v = narrow<O, V>(l[t]);
            } else {
                v = l[t];
            }
            // past the caches, which hold operands: 2 to 11 % of a call
            if constexpr (WHOLE) __builtin_nontemporal_store(__builtin_bit_cast(u32x4, v), (u32x4*)p);
            else store_some<O, V, false>(p, v, there);
        }
    };
#pragma unroll
    for (int j = 0; j < S::SI; ++j) {
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");      // a wavefront's LDS accesses are done in their order
        __builtin_amdgcn_wave_barrier();
#pragma unroll
        for (int i = 0; i < S::FI; ++i) {
            const uint32_t at = (i * 16 + (lane >> 4) * 4) * (uint32_t)sizeof(L);
            *(Vec<L, 4>*)(lds + chunk(lane & 15u, at / 16) + at % 16) = narrow<L, 4>(acc[j][i]);
        }
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        __builtin_amdgcn_wave_barrier();
        if (j > 0) store(j - 1);
#pragma unroll
        for (uint32_t t = 0; t < 16 / kDown; ++t)
#pragma unroll
            for (uint32_t h = 0; h < kLane; ++h) {
                constexpr int kPart = 16 / sizeof(L);
                const Vec<L, kPart> part = *(const Vec<L, kPart>*)(lds + chunk(t * kDown + down, lane % kAcross * kLane + h));
#pragma unroll
                for (int e = 0; e < kPart; ++e) l[t][h * kPart + e] = part[e];
            }
    }
    store(S::SI - 1);
}

template <typename O, typename L, typename S>
__device__ __forceinline__ void store_tile(char* lds, O* out, int64_t stride, uint32_t fast0, uint32_t fast_end, uint32_t slow0, uint32_t slow_end,
                                           const f32x4 (&acc)[S::SI][S::FI], bool accumulate) {
    if (S::group() != 0) return;
    const bool whole = (fast_end * sizeof(O)) % 16 == 0 && ((uintptr_t)out | (uintptr_t)stride * sizeof(O)) % 16 == 0;
    if constexpr (sizeof(L) == 4) {
        if (accumulate) return whole ? store_rows<O, L, S, true, true>(lds, out, stride, fast0, fast_end, slow0, slow_end, acc)
                                     : store_rows<O, L, S, false, true>(lds, out, stride, fast0, fast_end, slow0, slow_end, acc);
    }
    whole ? store_rows<O, L, S, true, false>(lds, out, stride, fast0, fast_end, slow0, slow_end, acc)
          : store_rows<O, L, S, false, false>(lds, out, stride, fast0, fast_end, slow0, slow_end, acc);
}

// --- which tile ---

// Rows from, end of bin b: expert b, or the unused rows for b == experts.  Held to 0 .. rows whatever offsets says.
__device__ __forceinline__ void rows_of(const int32_t* offsets, uint32_t experts, uint32_t rows, uint32_t b, uint32_t* from, uint32_t* end) {
    const uint32_t o = (uint32_t)offsets[b], next = (uint32_t)offsets[b < experts ? b + 1 : b], p = b < experts ? next : rows;   // both at once
    *end = p < rows ? p : rows;
    *from = o < *end ? o : *end;
}

// Which tile a workgroup takes.  Workgroups go round the 8 XCDs, so numbers that are 8 apart share an L2: each
// XCD takes one run of tiles, and inside an expert runs of kGroup rows of tiles by all columns.
constexpr uint32_t kXcds = 8;
template <uint32_t kGroup> __device__ __forceinline__ void grouped(uint32_t at, uint32_t down, uint32_t across, uint32_t* row, uint32_t* col) {
    const uint32_t g = at / (kGroup * across), in = at - g * kGroup * across;
    const uint32_t high = down - g * kGroup < kGroup ? down - g * kGroup : kGroup;
    *col = in / high;
    *row = g * kGroup + (in - *col * high);
}

// Tiles of `height` rows by `across` columns over all bins; false: this workgroup has none.  Every wavefront looks
// for itself: a lane takes neighbouring bins, a scan over the lanes and a ballot find the lane, the rest is
// uniform.
__device__ __forceinline__ bool find_tile(const int32_t* offsets, uint32_t experts, uint32_t rows, uint32_t height, uint32_t across,
                                          uint32_t* bin, uint32_t* from, uint32_t* end, uint32_t* col) {
    const uint32_t lane = threadIdx.x & 63u, bins = experts + 1, per = (bins + 63) / 64;
    uint32_t n = 0, o = 0, p = 0;
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
    const uint32_t tiles = (uint32_t)__builtin_amdgcn_readlane((int)sum, 63) * across, run = (tiles + kXcds - 1) / kXcds;
    const uint32_t block = (uint32_t)long_block(), index = block % kXcds * run + block / kXcds;
    if (block / kXcds >= run || index >= tiles) return false;
    const uint64_t at = __ballot(sum * across > index);
    if (at == 0) return false;
    const int l = __builtin_ctzll(at);
    uint32_t left = index - (uint32_t)__builtin_amdgcn_readlane((int)(sum - n), l) * across;
    uint32_t b = (uint32_t)l * per, down;
    if (per == 1) {         // the lane has the bin's rows
        o = (uint32_t)__builtin_amdgcn_readlane((int)o, l), p = (uint32_t)__builtin_amdgcn_readlane((int)p, l);
        down = (p - o + height - 1) / height;
    } else {
        for (;; ++b) {
            if (b >= bins) return false;
            rows_of(offsets, experts, rows, b, &o, &p);
            down = (p - o + height - 1) / height;
            if (left < down * across) break;
            left -= down * across;
        }
    }
    uint32_t row;
    grouped<8>(left, down, across, &row, col);
    *bin = uniform(b);
    *from = uniform(o + row * height);
    *end = uniform(p - *from < height ? p : *from + height);
    *col = uniform(*col);
    return true;
}

// --- kernels ---

template <typename T, int WL, typename S, bool LOOSE>
__global__ __launch_bounds__(S::kAllThreads) void expert_product_kernel(const ExpertProductArgs a) {
    extern __shared__ __attribute__((aligned(16))) char lds[];
    const uint32_t across = (a.n + S::kFast - 1) / S::kFast;
    uint32_t bin, row0, row_end, col;
    if (!find_tile(a.offsets, a.experts, a.rows, S::kSlow, across, &bin, &row0, &row_end, &col)) return;
    const uint32_t col0 = col * S::kFast;
    const T* const w = (const T*)a.w + (int64_t)bin * a.k * a.n;
    const Operand fast = WL == kDepthFast ? Operand(w, a.n, a.k) : Operand(w, a.k, a.n);
    f32x4 acc[S::SI][S::FI] = {};
    Sum<T, WL, kDepthFast, false, false, S, LOOSE> sum;
    sum.begin(lds, fast, col0, a.n, Operand(a.x), row0, row_end, 0, bin < a.experts ? a.k : 0);
    sum.multiply(acc);
    store_tile<T, T, S>(lds, (T*)a.out, a.out_stride, col0, a.n, row0, row_end, acc, false);
}

// The i-th expert by number of rows, most first (equal ones in their order), for up to 64 experts: every lane counts how many
// come before its own.  Tiles of large experts that start last would leave the chip idle around them.
__device__ __forceinline__ uint32_t by_size(const int32_t* offsets, uint32_t experts, uint32_t rows, uint32_t i, uint32_t* first, uint32_t* behind) {
    const uint32_t lane = threadIdx.x & 63u;
    uint32_t from = 0, end = 0, rank = 0;
    if (lane < experts) rows_of(offsets, experts, rows, lane, &from, &end);
    const uint32_t size = end - from;
    for (uint32_t e = 0; e < experts; ++e) {
        const uint32_t other = (uint32_t)__builtin_amdgcn_readlane((int)size, (int)e);
        rank += other > size || (other == size && e < lane) ? 1u : 0u;
    }
    const int expert = __builtin_ctzll(__ballot(lane < experts && rank == i));
    *first = (uint32_t)__builtin_amdgcn_readlane((int)from, expert), *behind = (uint32_t)__builtin_amdgcn_readlane((int)end, expert);
    return (uint32_t)expert;
}

// Experts one after the other; every XCD takes a run of an expert's tiles, whichever experts are large.
template <typename T, int FL, int SL, bool FM, bool SM, typename S, bool LOOSE>
__global__ __launch_bounds__(S::kAllThreads) void weight_gradient_kernel(const WeightGradientArgs a) {
    extern __shared__ __attribute__((aligned(16))) char lds[];
    const uint32_t tf = (a.fast.width + S::kFast - 1) / S::kFast, ts = (a.slow.width + S::kSlow - 1) / S::kSlow, run = (tf * ts + kXcds - 1) / kXcds;
    const uint64_t block = long_block();
    const uint32_t i = (uint32_t)(block / kXcds), turn = i / run, tile = ((uint32_t)(block % kXcds) + turn) % kXcds * run + i % run;
    if (turn >= a.experts || tile >= tf * ts) return;
    uint32_t expert = turn, from, end;
    if (a.experts <= 64) expert = by_size(a.offsets, a.experts, a.rows, turn, &from, &end);
    else rows_of(a.offsets, a.experts, a.rows, expert, &from, &end);
    expert = uniform(expert), from = uniform(from), end = uniform(end);
    uint32_t fi, si;
    grouped<4>(tile, ts, tf, &si, &fi);
    const uint32_t f0 = fi * S::kFast, s0 = si * S::kSlow;
    f32x4 acc[S::SI][S::FI] = {};
    Sum<T, FL, SL, FM, SM, S, LOOSE> sum;
    sum.begin(lds, Operand(a.fast), f0, a.fast.width, Operand(a.slow), s0, a.slow.width, from, end);
    sum.multiply(acc);
    const int64_t at = (int64_t)expert * a.fast.width * a.slow.width;
    const auto store = [&](auto o) {
        using O = decltype(o);
        store_tile<O, float, S>(lds, (O*)a.out + at, a.fast.width, f0, a.fast.width, s0, a.slow.width, acc, a.accumulate != 0);
    };
    if (a.out_type == TPERM_TYPE_F32) store(0.0f);
    else if (a.out_type == TPERM_TYPE_F16) store((_Float16)0);
    else store((__bf16)0);
}

template <typename T> hipError_t product_of(const ExpertProductArgs& a, bool w_k_first, hipStream_t stream);
template <typename T> hipError_t gradient_of(const WeightGradientArgs& a, hipStream_t stream);

}  // namespace tperm
