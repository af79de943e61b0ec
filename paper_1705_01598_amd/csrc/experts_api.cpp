// C-ABI entry points declared in include/tperm_experts.h: checks of the arguments, then one launch; and the query
// of their tiles in include/tperm_tuning.h.
#include <hip/hip_runtime.h>

#include "../../include/tperm_tuning.h"
#include "checks.hpp"
#include "experts.hpp"
#include "plan.hpp"

namespace tperm {
template <typename T> hipError_t product_of(const ExpertProductArgs& a, bool w_k_first, hipStream_t stream);
template <typename T> hipError_t gradient_of(const WeightGradientArgs& a, hipStream_t stream);
}  // namespace tperm

using namespace tperm;

namespace tperm {

hipError_t launch_expert_product(const ExpertProductArgs& a, int type, bool w_k_first, hipStream_t stream) {
    return type == TPERM_TYPE_F32 ? product_of<float>(a, w_k_first, stream) : type == TPERM_TYPE_F16 ? product_of<_Float16>(a, w_k_first, stream)
                                                                                                     : product_of<__bf16>(a, w_k_first, stream);
}
hipError_t launch_weight_gradient(const WeightGradientArgs& a, int type, hipStream_t stream) {
    return type == TPERM_TYPE_F32 ? gradient_of<float>(a, stream) : type == TPERM_TYPE_F16 ? gradient_of<_Float16>(a, stream) : gradient_of<__bf16>(a, stream);
}

}  // namespace tperm

extern "C" {

tperm_status_t tperm_expert_sort(const int32_t* expert, int64_t tokens, int64_t slots, int64_t experts, int32_t* offsets, int32_t* source,
                                 int32_t* place, void* workspace, size_t workspace_bytes, void* hip_stream) {
    int64_t rows = 0;
    const tperm_status_t st = count_rows(tokens, slots, experts, &rows);
    if (st != TPERM_OK) return st;
    const size_t need = TPERM_EXPERT_SORT_WORKSPACE_BYTES(rows, experts);
    const Array arrays[] = {{expert, rows * 4, 4, false},
                            {offsets, (experts + 1) * 4, 4, true},
                            {source, rows * 4, 4, true},
                            {place, rows * 4, 4, true},
                            {workspace, (int64_t)need, 4, true}};
    const tperm_status_t bad = check(arrays);
    if (bad != TPERM_OK) return bad;
    if (workspace_bytes < need) return TPERM_ERR_TOO_LARGE;
    return launched(launch_expert_sort(expert, (uint32_t)rows, (uint32_t)experts, offsets, source, place, (uint32_t*)workspace, (hipStream_t)hip_stream));
}

tperm_status_t tperm_expert_gather(const void* x, int64_t x_stride, const int32_t* source, const int32_t* offsets, const float* weights, void* out,
                                   int64_t out_stride, int64_t tokens, int64_t slots, int64_t experts, int64_t width, int type, void* hip_stream) {
    int64_t rows = 0;
    const tperm_status_t st = count_rows(tokens, slots, experts, &rows);
    if (st != TPERM_OK) return st;
    if (!known_width(width) || !known_stride(x_stride, width) || !known_stride(out_stride, width)) return TPERM_ERR_DIMS;
    if (!known_type(type)) return TPERM_ERR_ELEM_SIZE;
    if (rows == 0) return TPERM_OK;
    const size_t elem = type_bytes(type);
    const Array arrays[] = {{x, matrix_bytes(tokens, x_stride, width, elem), elem, false},
                            {source, rows * 4, 4, false},
                            {offsets, (experts + 1) * 4, 4, false},
                            {weights, weights ? rows * 4 : 0, 4, false},
                            {out, matrix_bytes(rows, out_stride, width, elem), elem, true}};
    const tperm_status_t bad = check(arrays);
    if (bad != TPERM_OK) return bad;
    RowsArgs a = {};
    a.in = x, a.out = out, a.map = source, a.used = offsets + experts, a.weights = weights, a.in_stride = x_stride, a.out_stride = out_stride;
    a.tokens = (uint32_t)tokens, a.slots = (uint32_t)slots, a.count = (uint32_t)rows, a.width = (uint32_t)width;
    return launched(launch_expert_gather(a, type, (hipStream_t)hip_stream));
}

tperm_status_t tperm_expert_combine(const void* in, int64_t rows_stride, const int32_t* place, const int32_t* offsets, const float* weights, void* out,
                                    int64_t out_stride, int64_t tokens, int64_t slots, int64_t experts, int64_t width, int type, void* hip_stream) {
    int64_t rows = 0;
    const tperm_status_t st = count_rows(tokens, slots, experts, &rows);
    if (st != TPERM_OK) return st;
    if (!known_width(width) || !known_stride(rows_stride, width) || !known_stride(out_stride, width)) return TPERM_ERR_DIMS;
    if (!known_type(type)) return TPERM_ERR_ELEM_SIZE;
    if (rows == 0) return TPERM_OK;
    const size_t elem = type_bytes(type);
    const Array arrays[] = {{in, matrix_bytes(rows, rows_stride, width, elem), elem, false},
                            {place, rows * 4, 4, false},
                            {offsets, (experts + 1) * 4, 4, false},
                            {weights, weights ? rows * 4 : 0, 4, false},
                            {out, matrix_bytes(tokens, out_stride, width, elem), elem, true}};
    const tperm_status_t bad = check(arrays);
    if (bad != TPERM_OK) return bad;
    RowsArgs a = {};
    a.in = in, a.out = out, a.map = place, a.used = offsets + experts, a.weights = weights, a.in_stride = rows_stride, a.out_stride = out_stride;
    a.tokens = (uint32_t)tokens, a.slots = (uint32_t)slots, a.count = (uint32_t)rows, a.width = (uint32_t)width;
    return launched(launch_expert_combine(a, type, (hipStream_t)hip_stream));
}

tperm_status_t tperm_expert_combine_backward(const void* grad, int64_t grad_stride, const void* in, int64_t rows_stride, const int32_t* place,
                                             const int32_t* offsets, const float* weights, void* grad_rows, int64_t grad_rows_stride, float* grad_weights,
                                             int64_t tokens, int64_t slots, int64_t experts, int64_t width, int type, void* hip_stream) {
    int64_t rows = 0;
    const tperm_status_t st = count_rows(tokens, slots, experts, &rows);
    if (st != TPERM_OK) return st;
    if (!known_width(width) || !known_stride(grad_stride, width) || !known_stride(rows_stride, width) || !known_stride(grad_rows_stride, width)) return TPERM_ERR_DIMS;
    if (!known_type(type)) return TPERM_ERR_ELEM_SIZE;
    if (rows == 0) return TPERM_OK;
    const size_t elem = type_bytes(type);
    const Array arrays[] = {{grad, matrix_bytes(tokens, grad_stride, width, elem), elem, false},
                            {in, matrix_bytes(rows, rows_stride, width, elem), elem, false},
                            {place, rows * 4, 4, false},
                            {offsets, (experts + 1) * 4, 4, false},
                            {weights, rows * 4, 4, false},
                            {grad_rows, matrix_bytes(rows, grad_rows_stride, width, elem), elem, true},
                            {grad_weights, rows * 4, 4, true}};
    const tperm_status_t bad = check(arrays);
    if (bad != TPERM_OK) return bad;
    RowsArgs a = {};
    a.in = grad, a.rows = in, a.out = grad_rows, a.grad_weights = grad_weights, a.map = place, a.used = offsets + experts, a.weights = weights;
    a.in_stride = grad_stride, a.rows_stride = rows_stride, a.out_stride = grad_rows_stride;
    a.tokens = (uint32_t)tokens, a.slots = (uint32_t)slots, a.count = (uint32_t)rows, a.width = (uint32_t)width;
    return launched(launch_expert_combine_backward(a, type, (hipStream_t)hip_stream));
}

tperm_status_t tperm_expert_product(const void* x, int64_t x_stride, int64_t x_rows, const int32_t* source, int64_t slots, const int32_t* offsets,
                                    const void* w, int w_k_first, void* out, int64_t out_stride, int64_t rows, int64_t experts, int64_t k, int64_t n,
                                    int type, void* hip_stream) {
    int64_t assigned = 0;   // without source the rows are x's own
    tperm_status_t st = count_rows(0, source ? slots : 1, experts, &assigned);
    if (st != TPERM_OK) return st;
    if (rows < 0 || x_rows < 0 || !known_width(k) || !known_width(n) || !known_stride(x_stride, k) || !known_stride(out_stride, n)) return TPERM_ERR_DIMS;
    if (source == nullptr && x_rows < rows) return TPERM_ERR_DIMS;
    if (!known_type(type)) return TPERM_ERR_ELEM_SIZE;
    if (rows > kRowsMax || x_rows > kRowsMax) return TPERM_ERR_TOO_LARGE;
    const size_t elem = type_bytes(type);
    if ((source && matrix_bytes(x_rows, x_stride, k, elem) > kOperandBytes) || k * n * (int64_t)elem > kOperandBytes) return TPERM_ERR_TOO_LARGE;
    if (rows == 0) return TPERM_OK;
    const Array arrays[] = {{x, matrix_bytes(x_rows, x_stride, k, elem), elem, false},
                            {source, source ? rows * 4 : 0, 4, false},
                            {offsets, (experts + 1) * 4, 4, false},
                            {w, experts * k * n * (int64_t)elem, elem, false},
                            {out, matrix_bytes(rows, out_stride, n, elem), elem, true}};
    const tperm_status_t bad = check(arrays);
    if (bad != TPERM_OK) return bad;
    ExpertProductArgs a = {};
    a.x.p = x, a.x.source = source, a.x.stride = x_stride, a.x.slots = make_fastdiv(source ? (uint32_t)slots : 1u), a.x.rows = (uint32_t)x_rows, a.x.width = (uint32_t)k;
    a.w = w, a.out = out, a.offsets = offsets, a.out_stride = out_stride;
    a.rows = (uint32_t)rows, a.experts = (uint32_t)experts, a.k = (uint32_t)k, a.n = (uint32_t)n;
    return launched(launch_expert_product(a, type, w_k_first != 0, (hipStream_t)hip_stream));
}

tperm_status_t tperm_expert_weight_gradient(const void* x, int64_t x_stride, const uint8_t* x_scales, int64_t x_rows, const int32_t* source, int64_t slots,
                                            const void* grad, int64_t grad_stride, const int32_t* offsets, void* out, int out_type, int w_k_first,
                                            int accumulate, int64_t rows, int64_t experts, int64_t k, int64_t n, int type, void* hip_stream) {
    int64_t assigned = 0;
    tperm_status_t st = count_rows(0, source ? slots : 1, experts, &assigned);
    if (st != TPERM_OK) return st;
    if (rows < 0 || x_rows < 0 || !known_width(k) || !known_width(n) || !known_stride(grad_stride, n)) return TPERM_ERR_DIMS;
    if (x_scales == nullptr && !known_stride(x_stride, k)) return TPERM_ERR_DIMS;
    if (source == nullptr && x_rows < rows) return TPERM_ERR_DIMS;
    if (!known_type(type) || !known_type(out_type)) return TPERM_ERR_ELEM_SIZE;
    if (rows > kRowsMax || x_rows > kRowsMax) return TPERM_ERR_TOO_LARGE;
    const size_t elem = type_bytes(type), x_elem = x_scales ? 1 : elem;
    if (x_scales != nullptr) x_stride = k;
    const int64_t x_bytes = matrix_bytes(x_rows, x_stride, k, x_elem), grad_bytes = matrix_bytes(rows, grad_stride, n, elem);
    if ((source && x_bytes > kOperandBytes) || k * n * (int64_t)type_bytes(out_type) > kOperandBytes) return TPERM_ERR_TOO_LARGE;
    const Array arrays[] = {{x, rows ? x_bytes : 0, x_elem, false},
                            {x_scales, x_scales && rows ? x_rows * TPERM_CHECKPOINT_BLOCKS(k) : 0, 1, false},
                            {source, source ? rows * 4 : 0, 4, false},
                            {grad, grad_bytes, elem, false},
                            {offsets, (experts + 1) * 4, 4, false},
                            {out, experts * k * n * (int64_t)type_bytes(out_type), type_bytes(out_type), true}};
    const tperm_status_t bad = check(arrays);
    if (bad != TPERM_OK) return bad;
    ProductSide xs = {}, gs = {};
    xs.p = x, xs.scales = x_scales, xs.source = source, xs.stride = x_stride, xs.slots = make_fastdiv(source ? (uint32_t)slots : 1u), xs.rows = (uint32_t)x_rows, xs.width = (uint32_t)k;
    gs.p = grad, gs.stride = grad_stride, gs.slots = make_fastdiv(1u), gs.rows = (uint32_t)rows, gs.width = (uint32_t)n;
    WeightGradientArgs a = {};
    a.fast = w_k_first ? xs : gs, a.slow = w_k_first ? gs : xs;
    a.out = out, a.offsets = offsets, a.rows = (uint32_t)rows, a.experts = (uint32_t)experts, a.out_type = out_type, a.accumulate = accumulate != 0;
    return launched(launch_weight_gradient(a, type, (hipStream_t)hip_stream));
}

tperm_status_t tperm_expert_tile(int gradient, int type, int w_k_first, int64_t rows, int64_t experts, int64_t k, int64_t n, int* along, int* across) {
    int64_t assigned = 0;
    const tperm_status_t st = count_rows(0, 1, experts, &assigned);
    if (st != TPERM_OK) return st;
    if (rows < 0 || !known_width(k) || !known_width(n)) return TPERM_ERR_DIMS;
    if (!known_type(type)) return TPERM_ERR_ELEM_SIZE;
    if (rows > kRowsMax) return TPERM_ERR_TOO_LARGE;
    if (along == nullptr || across == nullptr) return TPERM_ERR_NULL;
    const size_t elem = type_bytes(type);
    const int t = (int)(gradient ? gradient_tile(elem, w_k_first ? k : n, w_k_first ? n : k, experts) : product_tile(elem, rows, experts, n));
    *along = kTileFast[t], *across = kTileSlow[t];
    return TPERM_OK;
}

tperm_status_t tperm_checkpoint_store(const void* x, int64_t x_stride, uint8_t* codes, uint8_t* scales, int64_t rows, int64_t width, int type, void* hip_stream) {
    if (rows < 0 || !known_width(width) || !known_stride(x_stride, width)) return TPERM_ERR_DIMS;
    if (!known_type(type)) return TPERM_ERR_ELEM_SIZE;
    if (rows > kRowsMax) return TPERM_ERR_TOO_LARGE;
    if (rows == 0) return TPERM_OK;
    const size_t elem = type_bytes(type);
    const Array arrays[] = {{x, matrix_bytes(rows, x_stride, width, elem), elem, false},
                            {codes, rows * width, 1, true},
                            {scales, rows * TPERM_CHECKPOINT_BLOCKS(width), 1, true}};
    const tperm_status_t bad = check(arrays);
    if (bad != TPERM_OK) return bad;
    CheckpointArgs a = {};
    a.in = x, a.codes = codes, a.scales = scales, a.in_stride = x_stride, a.rows = (uint32_t)rows, a.width = (uint32_t)width;
    return launched(launch_checkpoint_store(a, type, (hipStream_t)hip_stream));
}

tperm_status_t tperm_checkpoint_load(const uint8_t* codes, const uint8_t* scales, void* out, int64_t out_stride, int64_t rows, int64_t width, int type,
                                     void* hip_stream) {
    if (rows < 0 || !known_width(width) || !known_stride(out_stride, width)) return TPERM_ERR_DIMS;
    if (!known_type(type)) return TPERM_ERR_ELEM_SIZE;
    if (rows > kRowsMax) return TPERM_ERR_TOO_LARGE;
    if (rows == 0) return TPERM_OK;
    const size_t elem = type_bytes(type);
    const Array arrays[] = {{codes, rows * width, 1, false},
                            {scales, rows * TPERM_CHECKPOINT_BLOCKS(width), 1, false},
                            {out, matrix_bytes(rows, out_stride, width, elem), elem, true}};
    const tperm_status_t bad = check(arrays);
    if (bad != TPERM_OK) return bad;
    CheckpointArgs a = {};
    a.out = out, a.codes = const_cast<uint8_t*>(codes), a.scales = const_cast<uint8_t*>(scales), a.out_stride = out_stride, a.rows = (uint32_t)rows, a.width = (uint32_t)width;
    return launched(launch_checkpoint_load(a, type, (hipStream_t)hip_stream));
}

tperm_status_t tperm_gated_forward(const void* gates, int64_t gates_stride, void* out, int64_t out_stride, uint8_t* codes, uint8_t* scales, int64_t rows,
                                   int64_t width, int type, void* hip_stream) {
    if (rows < 0 || !known_width(width) || !known_stride(gates_stride, 2 * width) || !known_stride(out_stride, width)) return TPERM_ERR_DIMS;
    if (!known_type(type)) return TPERM_ERR_ELEM_SIZE;
    if (rows > kRowsMax) return TPERM_ERR_TOO_LARGE;
    if ((codes == nullptr) != (scales == nullptr)) return TPERM_ERR_NULL;
    if (rows == 0) return TPERM_OK;
    const size_t elem = type_bytes(type);
    const Array arrays[] = {{gates, matrix_bytes(rows, gates_stride, 2 * width, elem), elem, false},
                            {out, matrix_bytes(rows, out_stride, width, elem), elem, true},
                            {codes, codes ? rows * 2 * width : 0, 1, true},
                            {scales, scales ? rows * 2 * TPERM_CHECKPOINT_BLOCKS(width) : 0, 1, true}};
    const tperm_status_t bad = check(arrays);
    if (bad != TPERM_OK) return bad;
    CheckpointArgs a = {};
    a.in = gates, a.out = out, a.codes = codes, a.scales = scales, a.in_stride = gates_stride, a.out_stride = out_stride, a.rows = (uint32_t)rows, a.width = (uint32_t)width;
    return launched(launch_gated_forward(a, type, (hipStream_t)hip_stream));
}

tperm_status_t tperm_gated_backward(const void* grad, int64_t grad_stride, const uint8_t* codes, const uint8_t* scales, void* grad_gates,
                                    int64_t grad_gates_stride, void* out, int64_t out_stride, int64_t rows, int64_t width, int type, void* hip_stream) {
    if (rows < 0 || !known_width(width) || !known_stride(grad_stride, width) || !known_stride(grad_gates_stride, 2 * width)) return TPERM_ERR_DIMS;
    if (out != nullptr && !known_stride(out_stride, width)) return TPERM_ERR_DIMS;
    if (!known_type(type)) return TPERM_ERR_ELEM_SIZE;
    if (rows > kRowsMax) return TPERM_ERR_TOO_LARGE;
    if (rows == 0) return TPERM_OK;
    const size_t elem = type_bytes(type);
    const Array arrays[] = {{grad, matrix_bytes(rows, grad_stride, width, elem), elem, false},
                            {codes, rows * 2 * width, 1, false},
                            {scales, rows * 2 * TPERM_CHECKPOINT_BLOCKS(width), 1, false},
                            {grad_gates, matrix_bytes(rows, grad_gates_stride, 2 * width, elem), elem, true},
                            {out, out ? matrix_bytes(rows, out_stride, width, elem) : 0, elem, true}};
    const tperm_status_t bad = check(arrays);
    if (bad != TPERM_OK) return bad;
    CheckpointArgs a = {};
    a.in = grad, a.out = out, a.grad_gates = grad_gates, a.codes = const_cast<uint8_t*>(codes), a.scales = const_cast<uint8_t*>(scales);
    a.in_stride = grad_stride, a.out_stride = out_stride, a.grad_stride = grad_gates_stride, a.rows = (uint32_t)rows, a.width = (uint32_t)width;
    return launched(launch_gated_backward(a, type, (hipStream_t)hip_stream));
}

}  // extern "C"
