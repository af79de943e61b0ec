// Assignments brought into the order of their experts: a stable counting sort.
//
// Up to TPERM_EXPERT_SORT_ONE_BLOCK assignments one workgroup does all of it.  Beyond, every workgroup takes a
// piece of neighbouring assignments; a first kernel counts them by expert, a second one reads all counts (at
// most 128 pieces, from the L2), so that it knows where each expert starts and where its own rows start
// there, and places its piece.  Inside a workgroup every wavefront owns neighbouring assignments: counted by
// LDS atomics (whole numbers, so their order does not matter), scanned over wavefronts, then placed 64 at a time in
// order: a lane's rank among the lanes of its expert comes from one ballot per bit of the expert number.
//
// Latency is the bound: 132 assignments 3.2 us, 524288 of 128 experts 2.7 us for the counts and 14.5 for the placing, with 6 MB
// to move; 3.4 and 16.4 us a call, one behind the other.
#include "experts.hpp"

namespace tperm {

namespace {

constexpr uint32_t kPieces = 128;       // workgroups of a large sort at most: with 256 each reads twice the counts, with 64 it
                                        // places twice the rows (524288 assignments: 16.8 us, 20.0, 18.4)
constexpr uint32_t kLeast = 2048;       // assignments of a piece at least
static_assert(TPERM_EXPERT_SORT_WORKSPACE_BYTES(1 << 20, 7) == kPieces * 8 * 4, "a count for every piece and bin");

// Assignments that name no expert count as one more expert.
__device__ __forceinline__ uint32_t bin_of(int32_t expert, uint32_t experts) { return (uint32_t)expert < experts ? (uint32_t)expert : experts; }

// Exclusive sums of one value per thread over the workgroup.  `sums`: a word per wavefront, free to use.
__device__ __forceinline__ uint32_t exclusive_sum(uint32_t v, uint32_t* sums) {
    const uint32_t lane = threadIdx.x & 63u, wave = threadIdx.x >> 6;
    uint32_t s = v;
    for (uint32_t d = 1; d < 64; d <<= 1) {
        const uint32_t o = (uint32_t)__shfl_up((int)s, d);
        if (lane >= d) s += o;
    }
    if (lane == 63) sums[wave] = s;
    __syncthreads();
    uint32_t before = 0;
    for (uint32_t w = 0; w < wave; ++w) before += sums[w];
    __syncthreads();
    return before + s - v;
}

__global__ __launch_bounds__(1024) void histogram_kernel(const int32_t* __restrict__ expert, uint32_t rows, uint32_t experts,
                                                         uint32_t piece, uint32_t* __restrict__ histograms) {
    __shared__ uint32_t count[TPERM_EXPERTS_MAX + 1];
    for (uint32_t e = threadIdx.x; e <= experts; e += blockDim.x) count[e] = 0;
    __syncthreads();
    const uint32_t from = blockIdx.x * piece, end = rows - from < piece ? rows : from + piece;
    for (uint32_t a = from + threadIdx.x; a < end; a += blockDim.x) atomicAdd(&count[bin_of(expert[a], experts)], 1u);
    __syncthreads();
    for (uint32_t e = threadIdx.x; e <= experts; e += blockDim.x) histograms[blockIdx.x * (experts + 1) + e] = count[e];
}

// `histograms` NULL: this workgroup is alone.  Dynamic LDS: (experts + 1) * (wavefronts + 1) words.
__global__ __launch_bounds__(1024) void place_kernel(const int32_t* __restrict__ expert, uint32_t rows, uint32_t experts, uint32_t piece,
                                                     const uint32_t* __restrict__ histograms, int32_t* __restrict__ offsets,
                                                     int32_t* __restrict__ source, int32_t* __restrict__ place) {
    extern __shared__ uint32_t shared[];
    __shared__ uint32_t sums[16];
    const uint32_t bins = experts + 1, waves = blockDim.x >> 6, wave = threadIdx.x >> 6, lane = threadIdx.x & 63u;
    uint32_t* const total = shared;                    // by bin: all assignments, then the first row
    uint32_t* const next = shared + bins;              // by wavefront and bin: count, then next row
    for (uint32_t i = threadIdx.x; i < bins * (waves + 1); i += blockDim.x) shared[i] = 0;
    __syncthreads();
    const uint32_t from = blockIdx.x * piece, end = rows - from < piece ? rows : from + piece;
    const uint32_t each = ((end - from + waves - 1) / waves + 63u) & ~63u;
    const uint32_t mine = from + wave * each < end ? from + wave * each : end, mine_end = end - mine < each ? end : mine + each;
    for (uint32_t a = mine + lane; a < mine_end; a += 64) atomicAdd(&next[wave * bins + bin_of(expert[a], experts)], 1u);
    // all assignments of a bin, and those of the pieces before this one: threads side by side take
    // neighbouring bins, groups of them every so-many-th piece
    const uint32_t groups = histograms ? blockDim.x / bins : 0;
    uint32_t before[3] = {0, 0, 0};      // 1025 bins and 512 threads: three bins to a thread
    if (histograms != nullptr) {
        const uint32_t pieces = gridDim.x;
        if (groups >= 1) {
            const uint32_t b = threadIdx.x % bins, g = threadIdx.x / bins;
            if (g < groups) {
                uint32_t all = 0, ahead = 0;
#pragma unroll 8
                for (uint32_t p = g; p < pieces; p += groups) {
                    const uint32_t c = histograms[p * bins + b];
                    all += c;
                    if (p < blockIdx.x) ahead += c;
                }
                atomicAdd(&total[b], all);
                before[0] = ahead;
            }
        } else {
            for (uint32_t b = threadIdx.x, i = 0; b < bins; b += blockDim.x, ++i) {
                uint32_t all = 0, ahead = 0;
#pragma unroll 8
                for (uint32_t p = 0; p < pieces; ++p) {
                    const uint32_t c = histograms[p * bins + b];
                    all += c;
                    if (p < blockIdx.x) ahead += c;
                }
                total[b] = all;
                before[i] = ahead;
            }
        }
    }
    __syncthreads();
    if (histograms == nullptr)
        for (uint32_t b = threadIdx.x; b < bins; b += blockDim.x) {
            uint32_t all = 0;
            for (uint32_t w = 0; w < waves; ++w) all += next[w * bins + b];
            total[b] = all;
        }
    __syncthreads();
    // first row of every bin: neighbouring bins to a thread, up to five (1025 bins and 256 threads)
    const uint32_t per = (bins + blockDim.x - 1) / blockDim.x, b0 = threadIdx.x * per;
    uint32_t mine_total = 0;
    for (uint32_t i = 0; i < per; ++i) mine_total += b0 + i < bins ? total[b0 + i] : 0u;
    uint32_t first = exclusive_sum(mine_total, sums);
    for (uint32_t i = 0; i < per; ++i)
        if (b0 + i < bins) {
            const uint32_t n = total[b0 + i];
            total[b0 + i] = first;
            if (blockIdx.x == 0) offsets[b0 + i] = (int32_t)first;
            first += n;
        }
    __syncthreads();
    // + the rows of earlier pieces
    if (histograms != nullptr) {
        if (groups >= 1) {
            if (threadIdx.x / bins < groups) atomicAdd(&total[threadIdx.x % bins], before[0]);
        } else {
            for (uint32_t b = threadIdx.x, i = 0; b < bins; b += blockDim.x, ++i) total[b] += before[i];
        }
        __syncthreads();
    }
    // + those of earlier wavefronts
    for (uint32_t b = threadIdx.x; b < bins; b += blockDim.x) {
        uint32_t row = total[b];
        for (uint32_t w = 0; w < waves; ++w) {
            const uint32_t n = next[w * bins + b];
            next[w * bins + b] = row;
            row += n;
        }
    }
    __syncthreads();
    const uint32_t bits = 32u - (uint32_t)__builtin_clz(experts);
    const uint64_t below = (1ull << lane) - 1ull;
    volatile uint32_t* const rows_of = next + wave * bins;
    for (uint32_t a0 = mine; a0 < mine_end; a0 += 64) {
        const uint32_t a = a0 + lane;
        const bool there = a < mine_end;
        const uint32_t b = there ? bin_of(expert[a], experts) : 0u;
        uint64_t same = __ballot(there);
        for (uint32_t i = 0; i < bits; ++i) {
            const bool one = (b >> i) & 1u;
            const uint64_t m = __ballot(one);
            same &= one ? m : ~m;
        }
        if (there) {
            const uint32_t rank = (uint32_t)__popcll(same & below), row = rows_of[b] + rank;
            place[a] = (int32_t)row;
            source[row] = (int32_t)a;
            // every lane has read; the lane that comes first in its expert moves the counter on
            __builtin_amdgcn_wave_barrier();
            if (rank == 0) rows_of[b] = row + (uint32_t)__popcll(same);
        }
        __builtin_amdgcn_wave_barrier();
    }
}

}  // namespace

hipError_t launch_expert_sort(const int32_t* expert, uint32_t rows, uint32_t experts, int32_t* offsets, int32_t* source,
                              int32_t* place, uint32_t* histograms, hipStream_t stream) {
    // 16 wavefronts, 8 where their counters would pass 64 KiB of LDS
    const auto lds = [&](uint32_t threads) { return (size_t)(experts + 1) * (threads / 64 + 1) * 4; };
    if (rows <= TPERM_EXPERT_SORT_ONE_BLOCK) {
        uint32_t threads = rows <= 256 ? 256 : rows <= 1024 ? 512 : 1024;
        if (lds(threads) > 60 * 1024) threads = 512;
        hipLaunchKernelGGL(place_kernel, dim3(1), dim3(threads), lds(threads), stream, expert, rows, experts, rows ? rows : 1, (const uint32_t*)nullptr, offsets, source, place);
        return hipGetLastError();
    }
    uint32_t piece = (rows + kPieces - 1) / kPieces;
    piece = piece < kLeast ? kLeast : (piece + 63) & ~63u;
    const uint32_t pieces = (rows + piece - 1) / piece, threads = lds(1024) > 60 * 1024 ? 512 : 1024;
    hipLaunchKernelGGL(histogram_kernel, dim3(pieces), dim3(1024), 0, stream, expert, rows, experts, piece, histograms);
    hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    hipLaunchKernelGGL(place_kernel, dim3(pieces), dim3(threads), lds(threads), stream, expert, rows, experts, piece, histograms, offsets, source, place);
    return hipGetLastError();
}

}  // namespace tperm
