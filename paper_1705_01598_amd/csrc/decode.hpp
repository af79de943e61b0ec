// Launch interface between the C-ABI layer and the kernels of tperm_decode.h.  Arguments have been checked: sizes are
// within the limits of the header, strides at least the widths.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "../../include/tperm_decode.h"
#include "experts.hpp"
#include "few_places.hpp"

namespace tperm {

struct RouteArgs {
    const void* scores;
    const float* grad_weights;      // backward
    int32_t* expert;                // backward: read
    float* weights;
    void* grad_scores;
    int64_t scores_stride, grad_stride;
    uint32_t tokens, slots, experts;
};
hipError_t launch_route(const RouteArgs& a, bool over_all, int type, hipStream_t stream);
hipError_t launch_route_backward(const RouteArgs& a, bool over_all, int type, hipStream_t stream);

struct FourBitArgs {
    const void* in;                 // store: x
    void* out;                      // load: out
    uint8_t *codes, *scales;
    int64_t stride;
    uint32_t rows, width;
    FastDiv per_row;                // by the threads of a row, for thread numbers below 2^31 (set by the launcher)
};
hipError_t launch_four_bit_store(FourBitArgs a, int type, hipStream_t stream);
hipError_t launch_four_bit_load(FourBitArgs a, int type, hipStream_t stream);

struct FourBitProductArgs {
    const void* x;
    const uint8_t *codes, *scales;
    void* out;
    int64_t x_stride, out_stride;
    uint32_t rows, k, n;
};
hipError_t launch_four_bit_product(const FourBitProductArgs& a, int type, hipStream_t stream);

constexpr uint32_t kFewChannels = 8;        // of a tile
constexpr uint32_t kFewShareTiles = 4;      // of a workgroup of the second kernel where workgroups share the entries of their channels

// How a few tokens' layer is laid out in its workspace: hidden rows in the order of the experts that are named; the shares of the second kernel's
// workgroups, and a counter to every group of channels that is shared.
constexpr uint32_t few_most(int64_t tokens, int64_t slots, int64_t experts) {
    const int64_t count = tokens * slots;
    return (uint32_t)((experts < count ? experts : count) + count / 33);
}
// Workgroups that share the entries of the same channels, so that there are 512 of them: from 64 MiB of second matrices on (of those of all entries that there
// could be; which experts are named is not known here), and only where columns are much beside the matrix (two tokens to an entry) or 8 channels to a workgroup
// leave compute units idle; in 4 bits, where columns are always much, from 20 MiB on.  Whole calls, without shares and with, in us.  bfloat16: 64 tokens x 8 of 128,
// 2048 -> 2 x 1024, 264 and 227, 64 x 4 of 32 114 and 99, 2 x 1024 from 1024 81 and 56, but 4 x 4 of 64 38 and 43 and 16 x 4 of 32, 2001 -> 2 x 1003, 86 and
// 110.  4 bits: one x 8 of 128, 4096 -> 2 x 4096, 72 and 63, 16 x 4 of 32, 2048 -> 2 x 1024 (32 MiB), 37.9 and 35.4, 8 x 4 of 64 (32 MiB) 30.3 and 29.5,
// 64 x 2 of 8, 2048 -> 2 x 2048 (22 MiB), 66 and 49, but 4 x 4 of 32 (16 MiB) 20.3 and 22.7.
inline uint32_t few_shares(uint64_t width, uint64_t count, uint32_t most, bool four_bits, uint64_t matrix_bytes) {
    if (most * matrix_bytes < (four_bits ? 20 << 20 : 64 << 20) || !(four_bits || count >= 2 * (uint64_t)most || width < 1600)) return 1;
    const uint64_t want = over(512, over(width, kFewShareTiles * kFewChannels));
    return (uint32_t)(want < most ? want : most);
}
struct FewRoom {
    uint32_t most;          // entries at most: one for every 32 tokens that name the same expert
    uint32_t pitch;         // elements of a hidden row
    uint32_t shares;        // workgroups that share the entries of the same channels
    size_t rows, bytes;     // of the hidden rows, and of all
};
inline FewRoom few_room(int64_t tokens, int64_t slots, int64_t experts, int64_t width, int64_t hidden, int type, bool four_bits) {
    FewRoom r;
    const int64_t count = tokens * slots;
    r.most = few_most(tokens, slots, experts);
    r.pitch = hidden_pitch((uint32_t)hidden, four_bits ? 32 : 16 / (uint32_t)type_bytes(type));
    r.rows = (size_t)count * r.pitch * 4;
    const uint64_t blocks = over(width, kFewShareTiles * kFewChannels);
    r.shares = few_shares(width, count, r.most, four_bits, (uint64_t)width * hidden * (four_bits ? 1 : 2 * type_bytes(type)) / 2);
    r.bytes = r.rows + (r.shares == 1 ? 0 : (size_t)r.shares * blocks * tokens * kFewShareTiles * kFewChannels * 4);
    return r;
}

struct FewArgs {
    const void* x;
    const int32_t* expert;
    const float* weights;           // or NULL
    const void *w_in, *w_out;       // elements or codes
    const uint8_t *in_scales, *out_scales;
    void* out;
    int64_t x_stride, out_stride;
    uint32_t tokens, slots, experts, width, hidden;
    FewRoom room;                   // the workspace's layout, by which its size was checked
    void* rows;                     // the workspace: the hidden rows, and behind them (set by the launcher) shares of results
    float* shares;
    FastDiv by_slots;               // set by the launcher
};
hipError_t launch_few(const FewArgs& a, int type, hipStream_t stream);

}  // namespace tperm
