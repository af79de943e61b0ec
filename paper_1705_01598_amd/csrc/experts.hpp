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
