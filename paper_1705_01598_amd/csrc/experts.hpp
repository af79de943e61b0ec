// Launch interface between the C-ABI layer and the kernels of the mixture-of-experts operators.  Arguments
// have been checked: sizes are within the limits of tperm_experts.h, strides at least the widths.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "../../include/tperm_experts.h"
#include "tperm_desc.h"

namespace tperm {

inline size_t type_bytes(int type) { return type == TPERM_TYPE_F32 ? 4 : 2; }

hipError_t launch_expert_sort(const int32_t* expert, uint32_t rows, uint32_t experts, int32_t* offsets, int32_t* source,
                              int32_t* place, uint32_t* histograms, hipStream_t stream);

// One of the row operators' calls: strides in elements.
struct RowsArgs {
    const void* in;             // gather: x; combine: rows; backward: grad
    const void* rows;           // backward: rows
    void* out;                  // gather: out; combine: out; backward: grad_rows
    float* grad_weights;
    const int32_t* map;         // gather: source; the others: place
    const int32_t* used;        // offsets + experts: the number of used rows
    const float* weights;
    int64_t in_stride, rows_stride, out_stride;
    uint32_t tokens, slots, count, width;   // count = tokens * slots
    uint32_t pieces;            // of a row, one to a group of lanes (this and the next set by the launcher)
    FastDiv by_pieces;          // for group numbers below 2^31, else magic 0
};
hipError_t launch_expert_gather(RowsArgs a, int type, hipStream_t stream);
hipError_t launch_expert_combine(RowsArgs a, int type, hipStream_t stream);
hipError_t launch_expert_combine_backward(RowsArgs a, int type, hipStream_t stream);

struct CheckpointArgs {
    const void* in;             // store: x; gated: gates; gated backward: grad
    void* out;                  // load: out; gated: out; gated backward: out
    void* grad_gates;
    uint8_t *codes, *scales;
    int64_t in_stride, out_stride, grad_stride;
    uint32_t rows, width;
    FastDiv per_row;            // by the threads of a row, for thread numbers below 2^31 (set by the launcher)
};
hipError_t launch_checkpoint_store(CheckpointArgs a, int type, hipStream_t stream);
hipError_t launch_checkpoint_load(CheckpointArgs a, int type, hipStream_t stream);
hipError_t launch_gated_forward(CheckpointArgs a, int type, hipStream_t stream);
hipError_t launch_gated_backward(CheckpointArgs a, int type, hipStream_t stream);

// Tile of the result that a workgroup computes: results along memory x across.
enum class Tile { kTiny, kSmall, kNarrow, kWide };      // 64 x 64, 128 x 128, 128 x 64, 256 x 256
constexpr int kTileFast[] = {64, 128, 128, 256}, kTileSlow[] = {64, 128, 64, 256};

inline uint64_t over(uint64_t a, uint64_t b) { return (a + b - 1) / b; }

// Large tiles need fewer bytes an operation, small ones fill the 256 compute units and waste less on experts of
// few rows (bf16, us with tiles of 256, 128, 64; rows of all experts on the average):
//   8 experts 1024 x 1024: 128 rows 26 17 13, 256 rows 26 17 19, 512 rows 27 21 28, 1024 rows 29 35 46
//   8 experts 2048 x 2048: 256 rows 45 36 45, 512 rows 47 59 73;  64 experts: 128 rows 183 171 221, 256 rows 233 243 352
//   64 experts 2048 x 1024: one row 40 26 19, 16 rows 66 61 49
//   f32, 8 experts 1024 x 1024, tiles of 128, 128 x 64, 64: 1024 rows 200 178 182, 4096 rows 554 540 564;
//   701 x 903: 750 rows 123 139 104
inline Tile product_tile(size_t elem, uint64_t all_rows, uint64_t experts, uint64_t n) {
    const uint64_t rows = over(all_rows, experts);
    const auto tiles = [&](uint64_t side) { return over(rows, side) * experts * over(n, side); };
    if (elem == 4) return rows >= 64 && tiles(128) >= 512 ? Tile::kNarrow : Tile::kTiny;
    return rows >= 192 && tiles(256) >= 128 ? Tile::kWide : rows >= 64 && tiles(128) >= 128 ? Tile::kSmall : Tile::kTiny;
}

// As for the products (bf16 in 8 bits, us with tiles of 256, 128, 64): 8 experts 1024 x 1024 (128 tiles of 256) 73 44 56,
// 2048 x 2048 (512) 93 109 207; f32, 8 experts 1024 x 1024 (512 of 128), 128, 128 x 64, 64: 234 152 164
inline Tile gradient_tile(size_t elem, uint64_t fast, uint64_t slow, uint64_t experts) {
    const auto tiles = [&](uint64_t side) { return over(fast, side) * over(slow, side) * experts; };
    if (elem == 4) return tiles(128) >= 512 ? Tile::kNarrow : Tile::kTiny;
    return tiles(256) >= 192 ? Tile::kWide : tiles(128) >= 256 ? Tile::kSmall : Tile::kTiny;
}

// One side of an experts' product.
struct ProductSide {
    const void* p;              // elements, or codes
    const uint8_t* scales;      // of codes
    const int32_t* source;      // row map, or NULL
    int64_t stride;             // elements between rows
    FastDiv slots;              // row(r) = source[r] / slots
    uint32_t rows;              // rows there are
    uint32_t width;             // elements of a row
};
struct ExpertProductArgs {
    ProductSide x;
    const void* w;              // experts' matrices
    void* out;
    const int32_t* offsets;
    int64_t out_stride;
    uint32_t rows, experts, k, n;
};
hipError_t launch_expert_product(const ExpertProductArgs& a, int type, bool w_k_first, hipStream_t stream);

struct WeightGradientArgs {
    ProductSide fast, slow;     // whose index runs fastest in out, and the other; one of them may be codes
    void* out;
    const int32_t* offsets;
    uint32_t rows, experts;
    int out_type;
    int accumulate;
};
hipError_t launch_weight_gradient(const WeightGradientArgs& a, int type, hipStream_t stream);

}  // namespace tperm
