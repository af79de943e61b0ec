// A whole mixture-of-experts layer for a few tokens, in two kernels or three.
//
// The first multiplies the g and u rows of 8 hidden channels of a named expert (an item) with the tokens that name it, applies the gated
// activation and the token's weight, and stores the hidden rows in binary32; a workgroup goes through every so-many-th
// item.  The second: a workgroup to 8 channels of the result goes through all named experts, its wavefronts share
// experts and pieces of their sums, and add up by token in LDS, one array for each wavefront, joined in their order: no
// atomics on numbers that round, and no rows of the experts in memory.  Where there is much to read, several workgroups share the experts of
// their channels, and a third kernel adds up their shares.
// Every workgroup of both finds the named experts and their tokens from the numbers themselves (at most 64 x 64 of
// them; 1.6 us), so no order has to be made first.
//
// The matrices are what bounds it: a compute unit takes in 26 GB/s at most, so both kernels want 256 of them busy.  bfloat16, 2048 -> 2 x 1024 -> 2048,
// kernel times: 64 tokens x 8 of 128 experts, 88 of them named, 142 + 83 + 5 us for 738 + 369 MB, 5.2 and 4.4 TB/s; one token x 4 9.9 + 7.2 us for 33.5 + 16.8 MB, of which 1.6 each is an empty
// launch; a read of so many bytes that does nothing else takes 7.2 and 4.8 us.  8 x 4 of 64 in 4 bits, 20 of them named: 15.6 + 11.6 + 3.8 us for 45 + 22 MB: most of what
// comes in are columns, 64 bytes a lane of tokens and 128 of hidden rows beside 17 of the matrix.
#pragma once
#include <type_traits>

#include "decode.hpp"
#include "few.hpp"
#include "gated.hpp"
#include "launch.hpp"
#include "plan.hpp"

namespace tperm {

namespace {

constexpr uint32_t kChannels = kFewChannels;
constexpr int kShareTiles = kFewShareTiles;
constexpr uint32_t kInGroups = 512;     // workgroups of the first kernel: two to a compute unit, each with many items, so that the tables are made once
                                        // (64 tokens x 8 of 128, a workgroup to every item of 8 channels 212 us, now 142)
constexpr size_t kInLds = 80 * 1024, kOutLds = 112 * 1024;
constexpr uint32_t kColumns = 32;       // tokens of an entry at most

template <typename T, bool FOUR> using Matrix = std::conditional_t<FOUR, FourBits, Elements<T>>;
// What the second product's columns are: hidden rows are held in binary32 between the kernels, and become what the matrix takes on their way.
// Held in two bfloat16 parts, 16 bits, the second kernel takes 85 us for 64 x 8 of 128 instead of 91, and 14.0 for one of 8 x 4 of 64 in 4 bits instead of 14.6;
// in three parts stored by the first kernel 97 and 17.6 (without shares, for 17.0).  In binary16 (64 x 8 of 128: 102) the matrix in two bfloat16
// parts, which meet all three of a hidden value, was no faster than products of binary32.
template <typename T, bool FOUR, bool SPLIT = true> using Hidden = Held<typename Matrix<T, FOUR>::Part, SPLIT>;
// The first product's columns: the tokens as they lie, or, for matrices in 4 bits where all tokens fit it, from LDS, in the parts that such a
// matrix takes and with rows that are filled up with zeros.
template <typename T, bool FOUR, bool STAGED> struct Tokens {
    typedef std::conditional_t<FOUR, Split<T>, Ready<T, 1>> Columns;
    typedef T E;
};
template <typename T> struct Tokens<T, true, true> {
    typedef Ready<__bf16, Split<T>::kParts, true> Columns;
    typedef __bf16 E;
};
template <typename T> constexpr size_t staged_bytes(uint32_t tokens, uint32_t width) { return (size_t)tokens * staged_pitch(width) * 2 * Split<T>::kParts; }
template <typename T, bool ALIGNED> __device__ __forceinline__ void stage(const FewArgs& a, __bf16* rows) {
    constexpr int kParts = Split<T>::kParts;
    const uint32_t pitch = staged_pitch(a.width), eights = pitch / 8 - 1;      // the 16 bytes more are left as they are
    for (uint32_t i = threadIdx.x; i < a.tokens * eights; i += kFewThreads) {
        const uint32_t t = i / eights, at = (i - t * eights) * 8;
        Vec<T, 8> v = {};
        if (at < a.width) v = load_some<T, 8, ALIGNED>((const T*)a.x + (int64_t)t * a.x_stride + at, (int)(a.width - at));
        bf16x8 part[kParts];
        if constexpr (kParts == 1) part[0] = v;
        else parts_of<kParts>(widen<T, 8>(v), part);
        for (int p = 0; p < kParts; ++p) store_vec<__bf16, 8, true>(rows + (p * a.tokens + t) * pitch + at, part[p]);
    }
}

// The rows of expert e's matrix.
template <typename M> __device__ __forceinline__ M matrix_of(const void* p, const uint8_t* scales, uint32_t e, uint32_t rows, uint32_t depth) {
    M m;
    if constexpr (std::is_same_v<M, FourBits>) {
        m.groups = (depth + 31) / 32;
        const uint64_t before = (uint64_t)e * rows * m.groups;
        m.rows = (const uint8_t*)p + before * 16, m.scales = scales + before;
    } else {
        m.stride = depth * (uint32_t)sizeof(*m.rows), m.odd = odd_of(p);
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

template <uint32_t THREADS, bool WEIGHTS> __device__ __forceinline__ Named find_named(const FewArgs& a, void* lds) {
    static_assert(2 * THREADS >= TPERM_EXPERTS_MAX, "two experts to a thread");
    __shared__ uint32_t wave_total[THREADS / 64], twice;
    const uint32_t count = a.tokens * a.slots, wave = threadIdx.x >> 6;
    Named n;
    n.mask = (uint32_t*)lds, n.entry = n.mask + 2 * a.experts, n.weight = (float*)(n.entry + a.room.most), n.first = (uint16_t*)(n.weight + (WEIGHTS ? count : 0));
    n.number = n.first + a.room.most, n.start = n.number + count, n.token = (uint8_t*)(n.start + a.experts);
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

// An item of the first kernel: an entry and R / 2 times 8 hidden channels, of which wavefront `wave` of `waves` adds up its piece.  Tiles 2 b and 2 b + 1 are
// the g and u rows of its b-th 8 channels.
struct Item {
    uint32_t expert, named, first, channel, wave, waves;
};
template <typename T, bool FOUR, bool STAGED, typename S, int STEPS, bool ALIGNED>
__device__ __forceinline__ void hidden_sums(const FewArgs& a, const Named& n, const Item& item, f32x4* sums, const __bf16* staged) {
    typedef Matrix<T, FOUR> W;
    const W w = matrix_of<W>(a.w_in, a.in_scales, item.expert, 2 * a.hidden, a.width);
    uint32_t row[S::R];
    for (int b = 0; b < S::R / 2; ++b) {
        const uint32_t g = item.channel + b * kChannels + S::row();
        row[2 * b] = g < a.hidden ? g : a.hidden - 1, row[2 * b + 1] = row[2 * b] + a.hidden;
    }
    const typename Tokens<T, FOUR, STAGED>::E* x[S::M];
    typename Tokens<T, FOUR, STAGED>::Columns cols = {};
    for (int m = 0; m < S::M; ++m) {
        const uint32_t t = n.token[item.first + (S::column(m) < item.named ? S::column(m) : 0)];
        if constexpr (STAGED) x[m] = staged + t * staged_pitch(a.width);
        else x[m] = (const T*)a.x + (int64_t)t * a.x_stride;
    }
    if constexpr (STAGED) cols.apart = a.tokens * staged_pitch(a.width);
    else cols.odd = odd_of(a.x);
    f32x4 sum[S::kSums][S::M] = {};
    rows_by_columns<S, STEPS, ALIGNED>(w, row, cols, x, 0u, a.width, item.wave, item.waves, sum);
    static_assert(S::kSums * S::M <= S::R, "a wavefront's place");
    for (int r = 0; r < S::kSums; ++r)
        for (int m = 0; m < S::M; ++m) sums[(item.wave * S::R + r * S::M + m) * 64 + threadIdx.x % 64] = sum[r][m];
}
// The sums of all wavefronts of an item, the activation, and the hidden rows: four channels of one column to a lane.
template <uint32_t EACH, typename S> __device__ __forceinline__ void hidden_rows(const FewArgs& a, const Named& n, const Item& item, const f32x4* sums) {
    for (uint32_t i = item.wave * 64 + threadIdx.x % 64; i < S::M * S::R * S::kColumns; i += item.waves * 64) {
        const uint32_t half = i % 2, b = i / 2 % (S::R / 2), column = i / S::R, m = column / S::kColumns, c = column % S::kColumns, channel = item.channel + b * kChannels + half * 4;
        if (column >= item.named) continue;
        f32x4 gu[2] = {};
        for (uint32_t v = 0; v < item.waves; ++v)
            for (int r = 0; r < 2; ++r) gu[r] += sums_at<S>(sums + v * S::R * 64, 2 * b + r, m, half, c);
        const float weight = n.weight[item.first + column];
        f32x4 h;
        for (int k = 0; k < 4; ++k) {
            const Sigmoid s = sigmoid<float>(gu[0][k]);
            h[k] = channel + k < a.hidden ? gu[0][k] * s.p * gu[1][k] * s.last * weight : 0.0f;
        }
        store_vec<float, 4, true>((float*)a.rows + (int64_t)(item.first + column) * a.room.pitch + hidden_place(channel, EACH), h);
    }
    // behind the last channels zeros to the row's end, which whole items reach at most
    const uint32_t end = item.channel + S::R / 2 * kChannels, quads = (a.room.pitch - end) / 4;
    if (end < a.hidden || quads == 0) return;
    for (uint32_t i = item.wave * 64 + threadIdx.x % 64; i < quads * item.named; i += item.waves * 64)
        store_vec<float, 4, true>((float*)a.rows + (int64_t)(item.first + i / quads) * a.room.pitch + hidden_place(end + i % quads * 4, EACH), f32x4{});
}

// All items of a workgroup, with R tiles.
template <typename T, bool FOUR, bool STAGED, bool ALIGNED, int R>
__device__ __forceinline__ void hidden_items(const FewArgs& a, const Named& n, f32x4* places, const __bf16* staged) {
    typedef Matrix<T, FOUR> W;
    typedef Shape<R, 1, false> Few;
    typedef Shape<R, 1, true> Some;
    typedef Shape<R, 2, true> Many;
    constexpr uint32_t kPlace = kFewWaves * R * 64;            // of all wavefronts' sums; two of them, used in turn
    constexpr uint32_t kItem = R / 2 * kChannels;
    // Eight loads in flight a wavefront (four where two conversions follow each) where there are more than four for each, else one step to each;
    // a workgroup's wavefronts share as many items as that leaves them.
    constexpr int kSteps = (FOUR ? 4 : 8) / R;
    const uint32_t channels = (a.hidden + kItem - 1) / kItem, items = n.total * channels, steps = (a.width + W::kDepth - 1) / W::kDepth;
    const bool long_steps = (uint64_t)items * steps * R > 4 * kInGroups * kFewWaves;
    const uint32_t pieces = long_steps ? (steps + kSteps - 1) / kSteps : steps, waves = pieces > 4 ? 8 : pieces > 2 ? 4 : pieces, at_once = kFewWaves / waves;
    const uint32_t wave = (uint32_t)__builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6)), group = wave / waves;
    f32x4* place = places + group * waves * R * 64;
    for (uint32_t base = blockIdx.x * at_once; base < items; base += gridDim.x * at_once) {
        Item item = {};
        if (base + group < items) {
            const uint32_t rank = (base + group) / channels, entry = (uint32_t)__builtin_amdgcn_readfirstlane((int)n.entry[rank]);
            item = {entry & 0xFFFFu, entry >> 16, (uint32_t)__builtin_amdgcn_readfirstlane((int)n.first[rank]), (base + group - rank * channels) * kItem, wave % waves, waves};
            if (item.named <= 8 && long_steps) hidden_sums<T, FOUR, STAGED, Few, kSteps, ALIGNED>(a, n, item, place, staged);
            else if (item.named <= 8) hidden_sums<T, FOUR, STAGED, Few, 1, ALIGNED>(a, n, item, place, staged);
            else if (item.named <= 16) hidden_sums<T, FOUR, STAGED, Some, FOUR ? 1 : kSteps, ALIGNED>(a, n, item, place, staged);
            else hidden_sums<T, FOUR, STAGED, Many, FOUR ? 1 : kSteps / 2, ALIGNED>(a, n, item, place, staged);
        }
        __syncthreads();
        if (item.named == 0) {
        } else if (item.named <= 8) hidden_rows<W::kEach, Few>(a, n, item, place);
        else if (item.named <= 16) hidden_rows<W::kEach, Some>(a, n, item, place);
        else hidden_rows<W::kEach, Many>(a, n, item, place);
        place = place < places + kPlace ? place + kPlace : place - kPlace;
    }
}

template <typename T, bool FOUR, bool STAGED, bool ALIGNED, bool X_ALIGNED, int R>
__global__ __launch_bounds__(kFewThreads, 4) void few_in_kernel(const FewArgs a) {
    extern __shared__ f32x4 dynamic[];
    static_assert(FOUR || !STAGED, "tokens of matrices in 4 bits");
    __bf16* const staged = (__bf16*)(dynamic + 2 * kFewWaves * R * 64);
    if constexpr (STAGED) stage<T, X_ALIGNED>(a, staged);
    const Named n = find_named<kFewThreads, true>(a, (char*)staged + (STAGED ? staged_bytes<T>(a.tokens, a.width) : 0));
    hidden_items<T, FOUR, STAGED, ALIGNED, R>(a, n, dynamic, staged);
}

// What lane l + 40 holds, for the lanes l of the first half whose l % 16 is below 8.
__device__ __forceinline__ float forty_on(float v) {
    const uint32_t w = (uint32_t)__builtin_amdgcn_mov_dpp((int)__float_as_uint(v), 0x128, 0xF, 0xF, true);      // row_ror:8
    return __uint_as_float(__builtin_amdgcn_permlane32_swap(w, w, false, false)[1]);
}

template <typename T, bool FOUR, typename S, int STEPS, bool ALIGNED>
__device__ __forceinline__ void result_sums(const FewArgs& a, uint32_t e, uint32_t named, const uint8_t* token, uint32_t first_row, uint32_t from,
                                            uint32_t to, float* sums) {
    typedef Matrix<T, FOUR> W;
    constexpr int R = S::R, M = S::M;
    const uint32_t lane = threadIdx.x & 63u, channel = blockIdx.x * (R * kChannels);
    const W w = matrix_of<W>(a.w_out, a.out_scales, e, a.width, a.hidden);
    uint32_t row[R];
    for (int r = 0; r < R; ++r) {
        const uint32_t j = channel + r * kChannels + S::row();
        row[r] = j < a.width ? j : a.width - 1;
    }
    const float* x[M];
    for (int m = 0; m < M; ++m) x[m] = (const float*)a.rows + (int64_t)(first_row + (S::column(m) < named ? S::column(m) : 0)) * a.room.pitch;
    f32x4 sum[S::kSums][M] = {};
    rows_by_columns<S, STEPS, ALIGNED>(w, row, Hidden<T, FOUR>{}, x, from, to, 0u, 1u, sum);
    if constexpr (Hidden<T, FOUR>::kSplit) {
        // An infinity has made sums NaN: that of a hidden value all sums of its column, since its second part is none, that of the matrix those where it met a part that is
        // zero.  Such sums are formed again, in products of binary32.
        bool none = false;
        for (int r = 0; r < S::kSums; ++r)
            for (int m = 0; m < M; ++m) none = none || __builtin_isunordered(sum[r][m][0], sum[r][m][1]) || __builtin_isunordered(sum[r][m][2], sum[r][m][3]);
        if (__builtin_amdgcn_ballot_w64(none) != 0) {
            f32x4 again[S::kSums][M] = {};
            rows_by_columns<S, 1, ALIGNED>(w, row, Hidden<T, FOUR, false>{}, x, from, to, 0u, 1u, again);
            for (int r = 0; r < S::kSums; ++r)
                for (int m = 0; m < M; ++m)
                    for (int i = 0; i < 4; ++i) sum[r][m][i] = sum[r][m][i] == sum[r][m][i] ? sum[r][m][i] : again[r][m][i];
        }
    }
    for (int m = 0; m < M; ++m) {
        if constexpr (!S::kPaired)
            for (int r = 0; r < R; ++r)
                for (int i = 0; i < 4; ++i) sum[r][m][i] += forty_on(sum[r][m][i]);
        if ((!S::kPaired && (lane >= 32 || lane % 16 >= 8)) || S::column(m) >= named) continue;
        float* const at = sums + token[first_row + S::column(m)] * (R * kChannels) + lane / 16 * 4;
        for (int r = 0; r < S::kSums; ++r) *(f32x4*)(at + r * (S::kPaired ? 2 : 1) * kChannels) += sum[r][m];
    }
}

// R tiles of 8 channels to a workgroup: columns are read once for them.  64 tokens x 8 of 128 experts, bfloat16: one tile 135 us, as many bytes of hidden rows as of
// the matrix to each workgroup; four, and eight workgroups to share the entries 84.
// With one tile of 8 channels a workgroup goes through all entries, with four through a share of them, and the shares of the same channels are added by the next kernel
// (4.8 us, 1.6 of them the launch).  Adding them in the workgroup that comes to its end last saves a launch, but the others' stores have to be seen across the chip's L2 caches:
// with a release by each workgroup the kernel took 109 us, and with stores past the caches and a wait for them, which no language
// model covers, 91.
template <typename T, bool FOUR, bool ALIGNED, int R>
__global__ __launch_bounds__(kFewThreads, 4) void few_out_kernel(const FewArgs a) {
    extern __shared__ f32x4 dynamic[];
    constexpr uint32_t kWaves = kFewWaves, kThreads = kFewThreads, kSteps = R == 1 ? (FOUR ? 2 : 4) : (FOUR ? 1 : 2), kBlock = kSteps * Matrix<T, FOUR>::kDepth;
    constexpr uint32_t kRows = R * kChannels;
    const uint32_t wave = (uint32_t)__builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6));
    float* const sums = (float*)dynamic;
    for (uint32_t i = threadIdx.x; i < kWaves * a.tokens * kRows; i += kThreads) sums[i] = 0.0f;
    const Named n = find_named<kThreads, false>(a, sums + kWaves * a.tokens * kRows);
    float* const mine = sums + wave * a.tokens * kRows;
    const uint32_t begin = n.total * blockIdx.y / gridDim.y, entries = n.total * (blockIdx.y + 1) / gridDim.y - begin;
    if (entries != 0) {
        // an item: an entry and a piece of its sum
        const uint32_t blocks = (a.hidden + kBlock - 1) / kBlock, want = (2 * kWaves + entries - 1) / entries, per = (blocks + want - 1) / want, pieces = (blocks + per - 1) / per;
        for (uint32_t item = wave; item < entries * pieces; item += kWaves) {
            const uint32_t rank = begin + item / pieces, from = item % pieces * per * kBlock, end = from + per * kBlock;
            const uint32_t entry = (uint32_t)__builtin_amdgcn_readfirstlane((int)n.entry[rank]), first_row = (uint32_t)__builtin_amdgcn_readfirstlane((int)n.first[rank]);
            const uint32_t e = entry & 0xFFFFu, named = entry >> 16, to = end < a.hidden ? end : a.hidden;
            if (named <= 8) result_sums<T, FOUR, Shape<R, 1, false>, kSteps, ALIGNED>(a, e, named, n.token, first_row, from, to, mine);
            else if constexpr (R == 1) {
                if (named <= 16) result_sums<T, FOUR, Shape<R, 2, false>, FOUR ? 1 : 4, ALIGNED>(a, e, named, n.token, first_row, from, to, mine);
                else result_sums<T, FOUR, Shape<R, 4, false>, FOUR ? 1 : 2, ALIGNED>(a, e, named, n.token, first_row, from, to, mine);
            } else {
                if (named <= 16) result_sums<T, FOUR, Shape<R, 1, true>, FOUR ? 1 : 2, ALIGNED>(a, e, named, n.token, first_row, from, to, mine);
                else result_sums<T, FOUR, Shape<R, 2, true>, FOUR ? 1 : 2, ALIGNED>(a, e, named, n.token, first_row, from, to, mine);
            }
        }
    }
    __syncthreads();
    const uint32_t first = blockIdx.x * kRows, channels = a.width - first < kRows ? a.width - first : kRows;
    const auto joined = [&](uint32_t t, uint32_t c) {
        float y = 0.0f;
        for (uint32_t v = 0; v < kWaves; ++v) y += sums[(v * a.tokens + t) * kRows + c];
        return y;
    };
    if (gridDim.y == 1) {
        for (uint32_t i = threadIdx.x; i < a.tokens * kRows; i += kThreads)
            if (i % kRows < channels) ((T*)a.out)[(int64_t)(i / kRows) * a.out_stride + first + i % kRows] = (T)joined(i / kRows, i % kRows);
        return;
    }
    float* const share = a.shares + ((int64_t)blockIdx.x * gridDim.y + blockIdx.y) * a.tokens * kRows;
    for (uint32_t i = threadIdx.x; i < a.tokens * kRows; i += kThreads) share[i] = joined(i / kRows, i % kRows);
}

// Adds up the shares of 4 channels of a token to a thread, in their order, eight of them requested at once.
constexpr uint32_t kJoinThreads = 64;
template <typename T> __global__ __launch_bounds__(kJoinThreads) void few_join_kernel(const FewArgs a) {
    constexpr uint32_t kRows = kShareTiles * kChannels;
    const uint32_t quad = blockIdx.y * kJoinThreads + threadIdx.x, channel = blockIdx.x * kRows + quad % (kRows / 4) * 4;
    if (quad >= a.tokens * (kRows / 4) || channel >= a.width) return;
    const float* const shares = a.shares + (int64_t)blockIdx.x * a.room.shares * a.tokens * kRows + quad * 4;
    f32x4 y = {};
    for (uint32_t first = 0; first < a.room.shares; first += 8) {
        f32x4 part[8];
#pragma unroll
        for (uint32_t v = 0; v < 8; ++v) part[v] = load_vec<float, 4, true>(shares + (int64_t)(first + v < a.room.shares ? first + v : first) * a.tokens * kRows);
#pragma unroll
        for (uint32_t v = 0; v < 8; ++v)
            if (first + v < a.room.shares) y += part[v];
    }
    store_some<T, 4, false>((T*)a.out + (int64_t)(quad / (kRows / 4)) * a.out_stride + channel, narrow<T, 4>(y), (int)(a.width - channel));
}

template <bool B> using Bool = std::integral_constant<bool, B>;
template <int N> using Int = std::integral_constant<int, N>;

template <typename T, bool FOUR> hipError_t layer(FewArgs a, hipStream_t stream) {
    const FewRoom room = a.room;
    a.shares = (float*)((char*)a.rows + room.rows);
    const uint32_t count = a.tokens * a.slots;
    const auto on_eights = [](const void* p, uint64_t stride, uint32_t width) { return ((uintptr_t)p | stride * sizeof(T)) % 16 == 0 && width % 8 == 0; };
    const bool x_aligned = on_eights(a.x, a.x_stride, a.width);
    const bool in_aligned = FOUR || on_eights(a.w_in, a.width, a.width), out_aligned = FOUR ? a.hidden % 8 == 0 : on_eights(a.w_out, a.hidden, a.hidden);
    a.by_slots = make_fastdiv(a.slots);
    const size_t named = named_bytes(count, a.experts, room.most, true), staged = staged_bytes<T>(a.tokens, a.width);
    const auto sums_bytes = [](int tiles) { return (size_t)2 * kFewWaves * tiles * 64 * 16; };
    const auto launch_in = [&](auto from_lds, auto aligned, auto x_is, auto tiles) {
        constexpr bool kStaged = decltype(from_lds)::value;
        constexpr int kTiles = decltype(tiles)::value;
        constexpr auto kKernel = few_in_kernel<T, FOUR, kStaged, decltype(aligned)::value, decltype(x_is)::value, kTiles>;
        const uint64_t items = (uint64_t)room.most * ((a.hidden + kTiles / 2 * kChannels - 1) / (kTiles / 2 * kChannels));
        const size_t lds = sums_bytes(kTiles) + named + (kStaged ? staged : 0);
        const hipError_t e = lds > 64 * 1024 ? allow_lds<kKernel>(kInLds) : hipSuccess;
        if (e != hipSuccess) return e;
        hipLaunchKernelGGL(kKernel, dim3((uint32_t)(items < kInGroups ? items : kInGroups)), dim3(kFewThreads), lds, stream, a);
        return hipGetLastError();
    };
    const auto launch_out = [&](auto aligned, auto tiles) {
        constexpr int kTiles = decltype(tiles)::value;
        constexpr auto kKernel = few_out_kernel<T, FOUR, decltype(aligned)::value, kTiles>;
        const size_t lds = (size_t)kFewWaves * a.tokens * kTiles * kChannels * 4 + named_bytes(count, a.experts, room.most, false);
        const hipError_t e = lds > 64 * 1024 ? allow_lds<kKernel>(kOutLds) : hipSuccess;
        if (e != hipSuccess) return e;
        hipLaunchKernelGGL(kKernel, dim3((a.width + kTiles * kChannels - 1) / (kTiles * kChannels), kTiles == 1 ? 1 : room.shares), dim3(kFewThreads), lds, stream, a);
        return hipGetLastError();
    };
    hipError_t e = hipSuccess;
    // Tokens come from LDS where every workgroup meets them more than four times (8 x 4 of 64 in 4 bits 18.8 -> 15.1 us, while one token's
    // matrices of 16 bits take 11.8 for 10.5).  Four tiles where an expert has several tokens: 64 x 8 of 128 in 4 bits 92 -> 70, bfloat16 154 -> 144.
    const bool many_items = (uint64_t)room.most * over(a.hidden, kChannels) >= 4 * kInGroups;
    if (FOUR && many_items && sums_bytes(2) + named + staged <= kInLds) {
        if constexpr (FOUR) e = x_aligned ? launch_in(Bool<true>(), Bool<true>(), Bool<true>(), Int<2>()) : launch_in(Bool<true>(), Bool<true>(), Bool<false>(), Int<2>());
    } else {
        const bool four_tiles = many_items && count >= (FOUR ? 2 : 3) * room.most && sums_bytes(4) + named <= kInLds, aligned = in_aligned && x_aligned;
        e = four_tiles ? (aligned ? launch_in(Bool<false>(), Bool<true>(), Bool<true>(), Int<4>()) : launch_in(Bool<false>(), Bool<false>(), Bool<false>(), Int<4>()))
                       : (aligned ? launch_in(Bool<false>(), Bool<true>(), Bool<true>(), Int<2>()) : launch_in(Bool<false>(), Bool<false>(), Bool<false>(), Int<2>()));
    }
    if (e != hipSuccess) return e;
    const auto launch_shared = [&](auto aligned) {
        return room.shares == 1 ? launch_out(aligned, Int<1>()) : launch_out(aligned, Int<kShareTiles>());
    };
    e = out_aligned ? launch_shared(Bool<true>()) : launch_shared(Bool<false>());
    if (e != hipSuccess || room.shares == 1) return e;
    constexpr uint32_t kRows = kShareTiles * kChannels;
    hipLaunchKernelGGL(few_join_kernel<T>, dim3((a.width + kRows - 1) / kRows, (a.tokens * (kRows / 4) + kJoinThreads - 1) / kJoinThreads), dim3(kJoinThreads), 0, stream, a);
    return hipGetLastError();
}

static_assert(named_bytes(TPERM_FEW_TOKENS * TPERM_SLOTS_MAX, TPERM_EXPERTS_MAX, few_most(TPERM_FEW_TOKENS, TPERM_SLOTS_MAX, TPERM_EXPERTS_MAX), true) <=
                  kInLds - 2 * kFewWaves * 2 * 64 * 16, "LDS of two workgroups");
static_assert(named_bytes(TPERM_FEW_TOKENS * TPERM_SLOTS_MAX, TPERM_EXPERTS_MAX, few_most(TPERM_FEW_TOKENS, TPERM_SLOTS_MAX, TPERM_EXPERTS_MAX), false) <=
                  kOutLds - 8 * TPERM_FEW_TOKENS * kShareTiles * kChannels * 4, "LDS of a workgroup of the second kernel");

}  // namespace

template <typename T> hipError_t few_of(const FewArgs& a, hipStream_t stream) { return a.in_scales != nullptr ? layer<T, true>(a, stream) : layer<T, false>(a, stream); }

}  // namespace tperm
