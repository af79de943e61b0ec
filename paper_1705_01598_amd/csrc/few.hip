// A whole mixture-of-experts layer for a few tokens, in two kernels.
//
// The first: a workgroup to 16 hidden channels of one named expert multiplies their g and u rows with the tokens that name
// the expert, applies the gated activation and the token's weight, and stores the hidden row in parts.  Every workgroup finds its
// expert and its tokens from the numbers themselves (at most 64 x 64 of them), so no order has to be made first;
// one workgroup an expert writes down what it found for the second kernel.  The second: a workgroup to 16 channels of the result goes through all
// named experts, its wavefronts share experts and pieces of their sums, and adds up by token in LDS, one
// array for each wavefront, joined in their order: no atomics, and no rows of the experts in memory.
#include <type_traits>

#include "decode.hpp"
#include "few.hpp"
#include "gated.hpp"

namespace tperm {

namespace {

constexpr uint32_t kChannels = 16;      // of a workgroup

// What the second product's columns are: how a hidden row is held between the kernels.
template <typename T, bool FOUR> struct Hidden {
    typedef std::conditional_t<FOUR, __bf16, T> E;
    static constexpr int kParts = !FOUR && sizeof(T) == 4 ? 1 : FOUR && sizeof(T) == 4 ? 3 : 2;
    typedef Ready<E, kParts> Columns;
};
template <typename T, bool FOUR> using Matrix = std::conditional_t<FOUR, FourBits, Elements<T>>;
template <typename T, bool FOUR> using Tokens = std::conditional_t<FOUR, Split<T>, Ready<T, 1>>;

// The rows of expert e's matrix.
template <typename M> __device__ __forceinline__ M matrix_of(const void* p, const uint8_t* scales, uint32_t e, uint32_t rows, uint32_t depth) {
    M m;
    if constexpr (std::is_same_v<M, FourBits>) {
        m.groups = (depth + 31) / 32;
        const uint64_t before = (uint64_t)e * rows * m.groups;
        m.rows = (const uint8_t*)p + before * 16, m.scales = scales + before;
    } else {
        m.stride = depth * (uint32_t)sizeof(*m.rows);
        m.rows = (decltype(m.rows))((const char*)p + (uint64_t)e * rows * m.stride);
    }
    return m;
}

// Bit number `rank` of 1024 in LDS, and how many there are.
__device__ __forceinline__ uint32_t find_bit(const uint32_t* bits, uint32_t rank, uint32_t* total) {
    const uint32_t lane = threadIdx.x & 63u, word = lane < 32 ? bits[lane] : 0u;
    const uint32_t mine = (uint32_t)__builtin_popcount(word);
    uint32_t upto = mine;
    for (uint32_t d = 1; d < 32; d <<= 1) {
        const uint32_t o = (uint32_t)__shfl_up((int)upto, d);
        if (lane >= d) upto += o;
    }
    *total = (uint32_t)__builtin_amdgcn_readlane((int)upto, 31);
    const uint64_t here = __ballot(lane < 32 && rank < upto && rank >= upto - mine);
    if (here == 0) return 0;
    const uint32_t at = (uint32_t)__builtin_ctzll(here);
    uint32_t w = (uint32_t)__builtin_amdgcn_readlane((int)word, at), skip = rank - (uint32_t)__builtin_amdgcn_readlane((int)(upto - mine), at);
    while (skip-- != 0) w &= w - 1;
    return at * 32 + (uint32_t)__builtin_ctz(w);
}

template <typename T, bool FOUR, int STEPS, bool ALIGNED, int M>
__device__ __forceinline__ void hidden_channels(const FewArgs& a, uint32_t pitch, uint32_t e, uint32_t named, const uint32_t* token, const float* weight,
                                                uint32_t first_row, f32x4* sums) {
    typedef Matrix<T, FOUR> W;
    typedef Hidden<T, FOUR> H;
    const uint32_t lane = threadIdx.x & 63u, wave = threadIdx.x >> 6, channel = blockIdx.x * kChannels;
    const W w = matrix_of<W>(a.w_in, a.in_scales, e, 2 * a.hidden, a.width);
    const uint32_t g = channel + lane % 16 < a.hidden ? channel + lane % 16 : a.hidden - 1;
    const uint32_t row[2] = {g, g + a.hidden};
    const T* x[M];
    for (int m = 0; m < M; ++m) {
        const uint32_t c = m * 16 + lane % 16;
        x[m] = (const T*)a.x + (int64_t)token[c < named ? c : 0] * a.x_stride;
    }
    const Tokens<T, FOUR> cols = {};
    f32x4 sum[2][M] = {};
    rows_by_columns<STEPS, ALIGNED>(w, row, cols, x, 0u, a.width, wave, (uint32_t)kFewWaves, sum);
    const uint32_t c = wave * 16 + lane % 16;       // of those who join: one wavefront for 16 columns
    f32x4 gu[2] = {};
#pragma unroll
    for (int r = 0; r < 2; ++r) {
        __syncthreads();        // what was in this place has been read
        for (int m = 0; m < M; ++m) sums[(wave * M + m) * 64 + lane] = sum[r][m];
        __syncthreads();
        if (wave < M)
            for (uint32_t v = 0; v < kFewWaves; ++v) gu[r] += sums[(v * M + wave) * 64 + lane];
    }
    if (wave >= M || c >= named) return;
    f32x4 h;
    for (int i = 0; i < 4; ++i) {
        const Sigmoid s = sigmoid<float>(gu[0][i]);
        h[i] = gu[0][i] * s.p * gu[1][i] * s.last * weight[c];
    }
    const int64_t rows = (int64_t)a.tokens * a.slots;
    typename H::E* const out = (typename H::E*)a.rows + (int64_t)(first_row + c) * pitch + channel + lane / 16 * 4;
    for (int p = 0; p < H::kParts; ++p) {
        const Vec<typename H::E, 4> part = narrow<typename H::E, 4>(h);
        store_vec<typename H::E, 4, true>(out + p * rows * pitch, part);
        const f32x4 back = widen<typename H::E, 4>(part);
        for (int i = 0; i < 4; ++i) h[i] = __builtin_isfinite(back[i]) ? h[i] - back[i] : 0.0f;
    }
}

template <typename T, bool FOUR, bool ALIGNED> __global__ __launch_bounds__(kFewThreads) void few_in_kernel(const FewArgs a, const uint32_t most, const uint32_t pitch) {
    extern __shared__ f32x4 dynamic[];
    __shared__ uint32_t bits[32], token[TPERM_FEW_TOKENS];
    __shared__ float weight[TPERM_FEW_TOKENS];
    const uint32_t lane = threadIdx.x & 63u, wave = threadIdx.x >> 6, count = a.tokens * a.slots;
    int32_t* const number = (int32_t*)dynamic;
    float* const given = (float*)dynamic + count;
    if (threadIdx.x < 32) bits[threadIdx.x] = 0;
    __syncthreads();
    for (uint32_t i = threadIdx.x; i < count; i += kFewThreads) {
        const int32_t e = a.expert[i];
        given[i] = a.weights != nullptr ? a.weights[i] : 1.0f;
        number[i] = e;
        if ((uint32_t)e < a.experts) atomicOr(&bits[(uint32_t)e / 32], 1u << (uint32_t)e % 32);
    }
    __syncthreads();
    uint32_t total;
    const uint32_t rank = blockIdx.y;
    const uint32_t e = find_bit(bits, rank, &total);
    if (blockIdx.x == 0 && rank == 0 && threadIdx.x == 0) a.tables[0] = (int32_t)total;
    if (rank >= total) return;
    // every wavefront: a lane to a token
    uint32_t before = 0;
    float w = 0.0f;
    bool names = false;
    if (lane < a.tokens)
        for (uint32_t s = 0; s < a.slots; ++s) {
            const uint32_t v = (uint32_t)number[lane * a.slots + s];
            before += v < e;
            if (v == e) w += given[lane * a.slots + s], names = true;
        }
    for (uint32_t d = 1; d < 64; d <<= 1) before += (uint32_t)__shfl_xor((int)before, d);
    const uint64_t all = __ballot(names);
    const uint32_t named = (uint32_t)__builtin_popcountll(all), first_row = (uint32_t)__builtin_amdgcn_readfirstlane((int)before);
    if (wave == 0 && names) {
        const uint32_t c = (uint32_t)__builtin_popcountll(all & ((1ull << lane) - 1));
        token[c] = lane, weight[c] = w;
        if (blockIdx.x == 0) a.tables[1 + 2 * most + first_row + c] = (int32_t)lane;
    }
    if (blockIdx.x == 0 && threadIdx.x == 0) a.tables[1 + rank] = (int32_t)(e | named << 16), a.tables[1 + most + rank] = (int32_t)first_row;
    __syncthreads();
    if (named <= 16) hidden_channels<T, FOUR, FOUR ? 2 : 4, ALIGNED, 1>(a, pitch, e, named, token, weight, first_row, dynamic);
    else if (named <= 32) hidden_channels<T, FOUR, 2, ALIGNED, 2>(a, pitch, e, named, token, weight, first_row, dynamic);
    else hidden_channels<T, FOUR, 1, ALIGNED, 4>(a, pitch, e, named, token, weight, first_row, dynamic);
}

template <typename T, bool FOUR, int STEPS, bool ALIGNED, int M>
__device__ __forceinline__ void result_channels(const FewArgs& a, uint32_t pitch, uint32_t e, uint32_t named, const uint8_t* token, uint32_t first_row, uint32_t from,
                                                uint32_t to, float* sums, uint32_t sums_pitch) {
    typedef Matrix<T, FOUR> W;
    typedef Hidden<T, FOUR> H;
    const uint32_t lane = threadIdx.x & 63u, channel = blockIdx.x * kChannels;
    const W w = matrix_of<W>(a.w_out, a.out_scales, e, a.width, a.hidden);
    const uint32_t row[1] = {channel + lane % 16 < a.width ? channel + lane % 16 : a.width - 1};
    const typename H::E* x[M];
    for (int m = 0; m < M; ++m) {
        const uint32_t c = m * 16 + lane % 16;
        x[m] = (const typename H::E*)a.rows + (int64_t)(first_row + (c < named ? c : 0)) * pitch;
    }
    const typename H::Columns cols = {(int64_t)a.tokens * a.slots * pitch};
    f32x4 sum[1][M] = {};
    rows_by_columns<STEPS, ALIGNED>(w, row, cols, x, from, to, 0u, 1u, sum);
    for (int m = 0; m < M; ++m) {
        const uint32_t c = m * 16 + lane % 16;
        if (c < named) {
            f32x4* const at = (f32x4*)(sums + token[first_row + c] * sums_pitch + lane / 16 * 4);
            *at += sum[0][m];
        }
    }
}

template <typename T, bool FOUR, bool ALIGNED> __global__ __launch_bounds__(kFewThreads) void few_out_kernel(const FewArgs a, const uint32_t most, const uint32_t pitch) {
    extern __shared__ f32x4 dynamic[];
    constexpr uint32_t kPitch = kChannels + 4, kSteps = FOUR ? 2 : 4, kBlock = kSteps * Matrix<T, FOUR>::kDepth;
    const uint32_t wave = threadIdx.x >> 6, count = a.tokens * a.slots, words = 1 + 2 * most;
    float* const sums = (float*)dynamic;
    int32_t* const tables = (int32_t*)(sums + kFewWaves * a.tokens * kPitch);
    uint8_t* const token = (uint8_t*)(tables + words);
    for (uint32_t i = threadIdx.x; i < words; i += kFewThreads) tables[i] = a.tables[i];
    for (uint32_t i = threadIdx.x; i < count; i += kFewThreads) token[i] = (uint8_t)a.tables[words + i];
    for (uint32_t i = threadIdx.x; i < kFewWaves * a.tokens * kPitch; i += kFewThreads) sums[i] = 0.0f;
    __syncthreads();
    const uint32_t total = (uint32_t)tables[0];
    float* const mine = sums + wave * a.tokens * kPitch;
    if (total != 0) {
        // an item: an expert and a piece of its sum
        const uint32_t blocks = (a.hidden + kBlock - 1) / kBlock, want = (2 * kFewWaves + total - 1) / total, per = (blocks + want - 1) / want, pieces = (blocks + per - 1) / per;
        for (uint32_t item = (uint32_t)__builtin_amdgcn_readfirstlane((int)wave); item < total * pieces; item += kFewWaves) {
            const uint32_t rank = item / pieces, from = (item - rank * pieces) * per * kBlock, end = from + per * kBlock;
            const uint32_t entry = (uint32_t)__builtin_amdgcn_readfirstlane(tables[1 + rank]), first_row = (uint32_t)__builtin_amdgcn_readfirstlane(tables[1 + most + rank]);
            const uint32_t e = entry & 0xFFFFu, named = entry >> 16, to = end < a.hidden ? end : a.hidden;
            if (named <= 16) result_channels<T, FOUR, kSteps, ALIGNED, 1>(a, pitch, e, named, token, first_row, from, to, mine, kPitch);
            else if (named <= 32) result_channels<T, FOUR, 2, ALIGNED, 2>(a, pitch, e, named, token, first_row, from, to, mine, kPitch);
            else result_channels<T, FOUR, 1, ALIGNED, 4>(a, pitch, e, named, token, first_row, from, to, mine, kPitch);
        }
    }
    __syncthreads();
    for (uint32_t i = threadIdx.x; i < a.tokens * kChannels; i += kFewThreads) {
        const uint32_t t = i / kChannels, c = i % kChannels;
        if (blockIdx.x * kChannels + c >= a.width) continue;
        float y = 0.0f;
        for (uint32_t v = 0; v < kFewWaves; ++v) y += sums[(v * a.tokens + t) * kPitch + c];
        ((T*)a.out)[(int64_t)t * a.out_stride + blockIdx.x * kChannels + c] = (T)y;
    }
}

template <typename T, bool FOUR> hipError_t go(const FewArgs& a, int type, hipStream_t stream) {
    const FewRoom room = few_room(a.tokens, a.slots, a.experts, a.hidden, type, FOUR);
    const uint32_t count = a.tokens * a.slots, columns = a.tokens <= 16 ? 1 : a.tokens <= 32 ? 2 : 4;
    const bool x_aligned = ((uintptr_t)a.x | (uintptr_t)a.x_stride * sizeof(T)) % 16 == 0 && a.width % 8 == 0;
    const bool in_aligned = x_aligned && (FOUR || ((uintptr_t)a.w_in | (uintptr_t)a.width * sizeof(T)) % 16 == 0);
    const bool out_aligned = a.hidden % 8 == 0 && (FOUR || ((uintptr_t)a.w_out | (uintptr_t)a.hidden * sizeof(T)) % 16 == 0);
    const size_t joined = (size_t)kFewWaves * columns * 64 * 16, numbers = (size_t)count * 8;
    const dim3 in_grid((a.hidden + kChannels - 1) / kChannels, room.most);
    const auto in = in_aligned ? few_in_kernel<T, FOUR, true> : few_in_kernel<T, FOUR, false>;
    hipLaunchKernelGGL(in, in_grid, dim3(kFewThreads), joined > numbers ? joined : numbers, stream, a, room.most, room.pitch);
    hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    const size_t sums = (size_t)kFewWaves * a.tokens * (kChannels + 4) * 4;
    const auto out = out_aligned ? few_out_kernel<T, FOUR, true> : few_out_kernel<T, FOUR, false>;
    hipLaunchKernelGGL(out, dim3((a.width + kChannels - 1) / kChannels), dim3(kFewThreads), sums + (size_t)(1 + 2 * room.most) * 4 + count, stream, a, room.most, room.pitch);
    return hipGetLastError();
}

}  // namespace

hipError_t launch_few(const FewArgs& a, int type, hipStream_t stream) {
    return with_type(type, [&](auto t) {
        using T = decltype(t);
        return a.in_scales != nullptr ? go<T, true>(a, type, stream) : go<T, false>(a, type, stream);
    });
}

}  // namespace tperm
