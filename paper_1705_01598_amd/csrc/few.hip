// A whole mixture-of-experts layer for a few tokens, in two kernels.
//
// The first multiplies the g and u rows of 8 hidden channels of a named expert (an item) with the tokens that name it, applies the gated
// activation and the token's weight, and stores the hidden rows in parts; a workgroup goes through every so-many-th
// item.  The second: a workgroup to 8 channels of the result goes through all named experts, its wavefronts share
// experts and pieces of their sums, and add up by token in LDS, one array for each wavefront, joined in their order: no
// atomics on numbers that round, and no rows of the experts in memory.
// Every workgroup of both finds the named experts and their tokens from the numbers themselves (at most 64 x 64 of
// them), so no order has to be made first.
#include <type_traits>

#include "decode.hpp"
#include "few.hpp"
#include "gated.hpp"
#include "launch.hpp"
#include "plan.hpp"

namespace tperm {

namespace {

constexpr uint32_t kChannels = 8;       // of a tile
constexpr uint32_t kInGroups = 512;     // workgroups of the first kernel: two to a compute unit
constexpr uint32_t kColumns = 32;       // tokens of an entry at most
constexpr uint32_t kImages = 2;         // 16 x 16 products of an item of the first kernel at most

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

// What the numbers say, in LDS.  An entry is up to kColumns tokens that name the same expert, in the order of experts: its number and how
// many tokens (<< 16), and their first hidden row; by hidden row there is its token and, for the first kernel, its weight.
struct Named {
    uint32_t* mask;         // two words an expert, a bit to a token
    uint32_t* entry;
    float* weight;
    uint16_t *first, *number, *start;
    uint8_t* token;
    uint32_t total;         // entries
};
constexpr size_t named_bytes(size_t count, size_t experts, size_t most, bool weights) {
    return (experts * 8 + most * 4 + (weights ? count * 4 : 0) + most * 2 + count * 2 + experts * 2 + count + 15) / 16 * 16;
}

// Sums over the lanes up to this one.
__device__ __forceinline__ uint32_t upto(uint32_t v) {
    v += (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x111, 0xF, 0xF, true);      // row_shr 1, 2, 4, 8
    v += (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x112, 0xF, 0xF, true);
    v += (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x114, 0xF, 0xF, true);
    v += (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x118, 0xF, 0xF, true);
    v += (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x142, 0xA, 0xF, false);     // the last lane of a row to the next one
    v += (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x143, 0xC, 0xF, false);     // of the first half to the second
    return v;
}

template <uint32_t THREADS, bool WEIGHTS> __device__ __forceinline__ Named find_named(const FewArgs& a, void* lds, uint32_t most) {
    static_assert(2 * THREADS >= TPERM_EXPERTS_MAX, "two experts to a thread");
    __shared__ uint32_t wave_total[THREADS / 64], twice;
    const uint32_t count = a.tokens * a.slots, wave = threadIdx.x >> 6;
    Named n;
    n.mask = (uint32_t*)lds, n.entry = n.mask + 2 * a.experts, n.weight = (float*)(n.entry + most), n.first = (uint16_t*)(n.weight + (WEIGHTS ? count : 0));
    n.number = n.first + most, n.start = n.number + count, n.token = (uint8_t*)(n.start + a.experts);
    int32_t own = -1;
    float own_weight = 1.0f;
    if (threadIdx.x < count) {
        own = a.expert[threadIdx.x];
        if (WEIGHTS && a.weights != nullptr) own_weight = a.weights[threadIdx.x];
    }
    for (uint32_t i = threadIdx.x; i < 2 * a.experts; i += THREADS) n.mask[i] = 0;
    if (threadIdx.x == 0) twice = 0;
    __syncthreads();
    for (uint32_t i = threadIdx.x; i < count; i += THREADS) {
        const uint32_t e = (uint32_t)(i < THREADS ? own : a.expert[i]), t = fdiv(i, a.by_slots);
        const bool there = e < a.experts;
        n.number[i] = (uint16_t)(there ? e : 0xFFFFu);
        if (there) {
            const uint32_t bit = 1u << t % 32, before = atomicOr(&n.mask[2 * e + t / 32], bit);
            if (WEIGHTS && (before & bit)) twice = 1;
        }
    }
    __syncthreads();
    // entries and rows before each expert: entries in the low half
    const uint32_t each = a.experts <= THREADS ? 1 : 2, e0 = threadIdx.x * each;
    uint32_t names[2] = {};
#pragma unroll
    for (uint32_t k = 0; k < 2; ++k)
        if (k < each && e0 + k < a.experts) names[k] = (uint32_t)__builtin_popcount(n.mask[2 * (e0 + k)]) + (uint32_t)__builtin_popcount(n.mask[2 * (e0 + k) + 1]);
    static_assert(TPERM_FEW_TOKENS <= 2 * kColumns, "two entries an expert at most");
    const auto entries = [](uint32_t tokens) { return (uint32_t)(tokens != 0) + (uint32_t)(tokens > kColumns); };
    const uint32_t mine = (names[0] + names[1]) << 16 | (entries(names[0]) + entries(names[1]));
    const uint32_t up = upto(mine);
    if ((threadIdx.x & 63u) == 63) wave_total[wave] = up;
    __syncthreads();
    uint32_t before = up - mine, all = 0;
#pragma unroll
    for (uint32_t v = 0; v < THREADS / 64; ++v) {
        before += v < wave ? wave_total[v] : 0u;
        all += wave_total[v];
    }
    n.total = (uint32_t)__builtin_amdgcn_readfirstlane((int)(all & 0xFFFFu));
#pragma unroll
    for (uint32_t k = 0; k < 2; ++k)
        if (names[k] != 0) {
            const uint32_t at = before & 0xFFFFu, row = before >> 16, more = names[k] > kColumns ? names[k] - kColumns : 0u;
            n.entry[at] = (e0 + k) | (names[k] - more) << 16;
            n.first[at] = (uint16_t)row;
            if (more != 0) n.entry[at + 1] = (e0 + k) | more << 16, n.first[at + 1] = (uint16_t)(row + kColumns);
            n.start[e0 + k] = (uint16_t)row;
            before += names[k] << 16 | entries(names[k]);
        }
    __syncthreads();
    for (uint32_t i = threadIdx.x; i < count; i += THREADS) {
        const uint32_t e = n.number[i], t = fdiv(i, a.by_slots);
        if (e == 0xFFFFu) continue;
        const uint64_t named = n.mask[2 * e] | (uint64_t)n.mask[2 * e + 1] << 32;
        const uint32_t row = n.start[e] + (uint32_t)__builtin_popcountll(named & ((1ull << t) - 1));
        n.token[row] = (uint8_t)t;
        if constexpr (WEIGHTS) {
            float w = i < THREADS ? own_weight : a.weights != nullptr ? a.weights[i] : 1.0f;
            if (twice) {        // all slots of the token that name this expert write the same sum
                w = 0.0f;
                for (uint32_t s = t * a.slots; s < (t + 1) * a.slots; ++s)
                    if (n.number[s] == e) w += a.weights != nullptr ? a.weights[s] : 1.0f;
            }
            n.weight[row] = w;
        }
    }
    __syncthreads();
    return n;
}

// An item of the first kernel: an entry and 8 hidden channels, of which wavefront `wave` of `waves` adds up its piece.
struct Item {
    uint32_t expert, named, first, channel, wave, waves;
};
template <typename T, bool FOUR, typename S, int STEPS, bool ALIGNED>
__device__ __forceinline__ void hidden_sums(const FewArgs& a, const Named& n, const Item& item, f32x4* sums) {
    typedef Matrix<T, FOUR> W;
    const W w = matrix_of<W>(a.w_in, a.in_scales, item.expert, 2 * a.hidden, a.width);
    const uint32_t g = item.channel + S::row() < a.hidden ? item.channel + S::row() : a.hidden - 1;
    const uint32_t row[2] = {g, g + a.hidden};
    const T* x[S::M];
    for (int m = 0; m < S::M; ++m) x[m] = (const T*)a.x + (int64_t)n.token[item.first + (S::column(m) < item.named ? S::column(m) : 0)] * a.x_stride;
    const Tokens<T, FOUR> cols = {};
    f32x4 sum[S::kSums][S::M] = {};
    rows_by_columns<S, STEPS, ALIGNED>(w, row, cols, x, 0u, a.width, item.wave, item.waves, sum);
    static_assert(S::kSums * S::M <= (int)kImages, "a wavefront's place");
    for (int r = 0; r < S::kSums; ++r)
        for (int m = 0; m < S::M; ++m) sums[(item.wave * kImages + r * S::M + m) * 64 + threadIdx.x % 64] = sum[r][m];
}
// The sums of all wavefronts of an item, the activation, and the hidden rows in parts: four channels of one column to a lane.
template <typename T, bool FOUR, typename S> __device__ __forceinline__ void hidden_rows(const FewArgs& a, uint32_t pitch, const Named& n, const Item& item, const f32x4* sums) {
    typedef Hidden<T, FOUR> H;
    for (uint32_t i = item.wave * 64 + threadIdx.x % 64; i < S::M * 2 * S::kColumns; i += item.waves * 64) {
        const uint32_t m = i / (2 * S::kColumns), half = i / S::kColumns % 2, c = i % S::kColumns, column = m * S::kColumns + c;
        if (column >= item.named) continue;
        f32x4 gu[2] = {};
        for (uint32_t v = 0; v < item.waves; ++v)
            for (int r = 0; r < 2; ++r) gu[r] += sums_at<S>(sums + v * kImages * 64, r, m, half, c);
        const float weight = n.weight[item.first + column];
        f32x4 h;
        for (int k = 0; k < 4; ++k) {
            const Sigmoid s = sigmoid<float>(gu[0][k]);
            h[k] = gu[0][k] * s.p * gu[1][k] * s.last * weight;
        }
        const int64_t rows = (int64_t)a.tokens * a.slots;
        typename H::E* const out = (typename H::E*)a.rows + (int64_t)(item.first + column) * pitch + item.channel + half * 4;
        for (int p = 0; p < H::kParts; ++p) {
            const Vec<typename H::E, 4> part = narrow<typename H::E, 4>(h);
            store_vec<typename H::E, 4, true>(out + p * rows * pitch, part);
            const f32x4 back = widen<typename H::E, 4>(part);
            for (int k = 0; k < 4; ++k) h[k] = __builtin_isfinite(back[k]) ? h[k] - back[k] : 0.0f;
        }
    }
}

template <typename T, bool FOUR, bool ALIGNED> __global__ __launch_bounds__(kFewThreads, 4) void few_in_kernel(const FewArgs a, const uint32_t most, const uint32_t pitch) {
    extern __shared__ f32x4 dynamic[];
    typedef Matrix<T, FOUR> W;
    typedef Shape<2, 1, false> Few;
    typedef Shape<2, 1, true> Some;
    typedef Shape<2, 2, true> Many;
    constexpr uint32_t kPlace = kFewWaves * kImages * 64;      // of all wavefronts' sums; two of them, used in turn
    const Named n = find_named<kFewThreads, true>(a, dynamic + 2 * kPlace, most);
    const uint32_t channels = (a.hidden + kChannels - 1) / kChannels, items = n.total * channels, steps = (a.width + W::kDepth - 1) / W::kDepth;
    // Eight loads in flight a wavefront where there are more than four for each, else one step to each; a workgroup's wavefronts
    // share as many items as that leaves them.
    constexpr int kSteps = 4;
    const bool long_steps = items * steps * 2 > 4 * 2 * kInGroups * kFewWaves;
    const uint32_t pieces = long_steps ? (steps + kSteps - 1) / kSteps : steps, waves = pieces > 4 ? 8 : pieces > 2 ? 4 : pieces, at_once = kFewWaves / waves;
    const uint32_t wave = (uint32_t)__builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6)), group = wave / waves;
    f32x4* place = dynamic + group * waves * kImages * 64;
    for (uint32_t base = blockIdx.x * at_once; base < items; base += gridDim.x * at_once) {
        Item item = {};
        if (base + group < items) {
            const uint32_t rank = (base + group) / channels, entry = (uint32_t)__builtin_amdgcn_readfirstlane((int)n.entry[rank]);
            item = {entry & 0xFFFFu, entry >> 16, (uint32_t)__builtin_amdgcn_readfirstlane((int)n.first[rank]), (base + group - rank * channels) * kChannels, wave % waves, waves};
            if (item.named <= 8 && long_steps) hidden_sums<T, FOUR, Few, kSteps, ALIGNED>(a, n, item, place);
            else if (item.named <= 8) hidden_sums<T, FOUR, Few, 1, ALIGNED>(a, n, item, place);
            else if (item.named <= 16) hidden_sums<T, FOUR, Some, FOUR ? 2 : 4, ALIGNED>(a, n, item, place);
            else hidden_sums<T, FOUR, Many, FOUR ? 1 : 2, ALIGNED>(a, n, item, place);
        }
        __syncthreads();
        if (item.named == 0) {
        } else if (item.named <= 8) hidden_rows<T, FOUR, Few>(a, pitch, n, item, place);
        else if (item.named <= 16) hidden_rows<T, FOUR, Some>(a, pitch, n, item, place);
        else hidden_rows<T, FOUR, Many>(a, pitch, n, item, place);
        place = place < dynamic + kPlace ? place + kPlace : place - kPlace;
    }
}

constexpr uint32_t kOutWaves = 16, kOutThreads = 64 * kOutWaves, kTokenPitch = kChannels;     // kTokenPitch: of a token in a wavefront's array

template <typename T, bool FOUR, int STEPS, bool ALIGNED, int M>
__device__ __forceinline__ void result_channels(const FewArgs& a, uint32_t pitch, uint32_t e, uint32_t named, const uint8_t* token, uint32_t first_row, uint32_t from,
                                                uint32_t to, float* sums) {
    typedef Matrix<T, FOUR> W;
    typedef Hidden<T, FOUR> H;
    typedef Shape<1, M, false> S;
    const uint32_t lane = threadIdx.x & 63u, channel = blockIdx.x * kChannels;
    const W w = matrix_of<W>(a.w_out, a.out_scales, e, a.width, a.hidden);
    const uint32_t row[1] = {channel + S::row() < a.width ? channel + S::row() : a.width - 1};
    const typename H::E* x[M];
    for (int m = 0; m < M; ++m) x[m] = (const typename H::E*)a.rows + (int64_t)(first_row + (S::column(m) < named ? S::column(m) : 0)) * pitch;
    const typename H::Columns cols = {(int64_t)a.tokens * a.slots * pitch};
    f32x4 sum[1][M] = {};
    rows_by_columns<S, STEPS, ALIGNED>(w, row, cols, x, from, to, 0u, 1u, sum);
    // the diagonal: even pieces in lanes 0 .. 7 of the first two sixteens, odd ones 40 lanes on
    for (int m = 0; m < M; ++m) {
        f32x4 y = sum[0][m];
        for (int i = 0; i < 4; ++i) y[i] += __shfl(y[i], (int)(lane + 40));
        if (lane < 32 && lane % 16 < 8 && S::column(m) < named) *(f32x4*)(sums + token[first_row + S::column(m)] * kTokenPitch + lane / 16 * 4) += y;
    }
}

template <typename T, bool FOUR, bool ALIGNED> __global__ __launch_bounds__(kOutThreads) void few_out_kernel(const FewArgs a, const uint32_t most, const uint32_t pitch) {
    extern __shared__ f32x4 dynamic[];
    constexpr uint32_t kSteps = FOUR ? 2 : 8, kBlock = kSteps * Matrix<T, FOUR>::kDepth;
    const uint32_t wave = threadIdx.x >> 6;
    float* const sums = (float*)dynamic;
    for (uint32_t i = threadIdx.x; i < kOutWaves * a.tokens * kTokenPitch; i += kOutThreads) sums[i] = 0.0f;
    const Named n = find_named<kOutThreads, false>(a, sums + kOutWaves * a.tokens * kTokenPitch, most);
    float* const mine = sums + wave * a.tokens * kTokenPitch;
    if (n.total != 0) {
        // an item: an entry and a piece of its sum
        const uint32_t blocks = (a.hidden + kBlock - 1) / kBlock, want = (2 * kOutWaves + n.total - 1) / n.total, per = (blocks + want - 1) / want, pieces = (blocks + per - 1) / per;
        for (uint32_t item = (uint32_t)__builtin_amdgcn_readfirstlane((int)wave); item < n.total * pieces; item += kOutWaves) {
            const uint32_t rank = item / pieces, from = (item - rank * pieces) * per * kBlock, end = from + per * kBlock;
            const uint32_t entry = (uint32_t)__builtin_amdgcn_readfirstlane((int)n.entry[rank]), first_row = (uint32_t)__builtin_amdgcn_readfirstlane((int)n.first[rank]);
            const uint32_t e = entry & 0xFFFFu, named = entry >> 16, to = end < a.hidden ? end : a.hidden;
            if (named <= 8) result_channels<T, FOUR, kSteps, ALIGNED, 1>(a, pitch, e, named, n.token, first_row, from, to, mine);
            else if (named <= 16) result_channels<T, FOUR, FOUR ? 1 : 4, ALIGNED, 2>(a, pitch, e, named, n.token, first_row, from, to, mine);
            else result_channels<T, FOUR, FOUR ? 1 : 2, ALIGNED, 4>(a, pitch, e, named, n.token, first_row, from, to, mine);
        }
    }
    __syncthreads();
    for (uint32_t i = threadIdx.x; i < a.tokens * kChannels; i += kOutThreads) {
        const uint32_t t = i / kChannels, c = i % kChannels;
        if (blockIdx.x * kChannels + c >= a.width) continue;
        float y = 0.0f;
        for (uint32_t v = 0; v < kOutWaves; ++v) y += sums[(v * a.tokens + t) * kTokenPitch + c];
        ((T*)a.out)[(int64_t)t * a.out_stride + blockIdx.x * kChannels + c] = (T)y;
    }
}

template <typename T, bool FOUR> hipError_t go(FewArgs a, int type, hipStream_t stream) {
    const FewRoom room = few_room(a.tokens, a.slots, a.experts, a.hidden, type, FOUR);
    const uint32_t count = a.tokens * a.slots;
    const bool x_aligned = ((uintptr_t)a.x | (uintptr_t)a.x_stride * sizeof(T)) % 16 == 0 && a.width % 8 == 0;
    const bool in_aligned = x_aligned && (FOUR || ((uintptr_t)a.w_in | (uintptr_t)a.width * sizeof(T)) % 16 == 0);
    const bool out_aligned = a.hidden % 8 == 0 && (FOUR || ((uintptr_t)a.w_out | (uintptr_t)a.hidden * sizeof(T)) % 16 == 0);
    a.by_slots = make_fastdiv(a.slots);
    const auto launch_in = [&](auto aligned) {
        constexpr auto kKernel = few_in_kernel<T, FOUR, decltype(aligned)::value>;
        const uint64_t items = (uint64_t)room.most * ((a.hidden + kChannels - 1) / kChannels);
        const size_t lds = (size_t)2 * kFewWaves * kImages * 64 * 16 + named_bytes(count, a.experts, room.most, true);
        const hipError_t e = lds > 64 * 1024 ? allow_lds<kKernel>(80 * 1024) : hipSuccess;
        if (e != hipSuccess) return e;
        hipLaunchKernelGGL(kKernel, dim3((uint32_t)(items < kInGroups ? items : kInGroups)), dim3(kFewThreads), lds, stream, a, room.most, room.pitch);
        return hipGetLastError();
    };
    const auto launch_out = [&](auto aligned) {
        constexpr auto kKernel = few_out_kernel<T, FOUR, decltype(aligned)::value>;
        const size_t lds = (size_t)kOutWaves * a.tokens * kTokenPitch * 4 + named_bytes(count, a.experts, room.most, false);
        hipLaunchKernelGGL(kKernel, dim3((a.width + kChannels - 1) / kChannels), dim3(kOutThreads), lds, stream, a, room.most, room.pitch);
        return hipGetLastError();
    };
    const hipError_t e = in_aligned ? launch_in(std::true_type()) : launch_in(std::false_type());
    return e != hipSuccess ? e : out_aligned ? launch_out(std::true_type()) : launch_out(std::false_type());
}

static_assert(named_bytes(TPERM_FEW_TOKENS * TPERM_SLOTS_MAX, TPERM_EXPERTS_MAX, few_most(TPERM_FEW_TOKENS, TPERM_SLOTS_MAX, TPERM_EXPERTS_MAX), true) <=
                  80 * 1024 - 2 * kFewWaves * kImages * 64 * 16, "LDS of two workgroups");
static_assert(named_bytes(TPERM_FEW_TOKENS * TPERM_SLOTS_MAX, TPERM_EXPERTS_MAX, few_most(TPERM_FEW_TOKENS, TPERM_SLOTS_MAX, TPERM_EXPERTS_MAX), false) <=
                  63 * 1024 - kOutWaves * TPERM_FEW_TOKENS * kTokenPitch * 4, "LDS that needs no leave");

}  // namespace

hipError_t launch_few(const FewArgs& a, int type, hipStream_t stream) {
    return with_type(type, [&](auto t) {
        using T = decltype(t);
        return a.in_scales != nullptr ? go<T, true>(a, type, stream) : go<T, false>(a, type, stream);
    });
}

}  // namespace tperm
