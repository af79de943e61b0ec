// C-ABI entry points declared in include/tperm_decode.h: checks of the arguments, then the launches.
#include <hip/hip_runtime.h>

#include "checks.hpp"
#include "decode.hpp"

namespace tperm {
template <typename T> hipError_t few_of(const FewArgs& a, hipStream_t stream);
hipError_t launch_few(const FewArgs& a, int type, hipStream_t stream) {
    return type == TPERM_TYPE_F32 ? few_of<float>(a, stream) : type == TPERM_TYPE_F16 ? few_of<_Float16>(a, stream) : few_of<__bf16>(a, stream);
}
}  // namespace tperm

using namespace tperm;

extern "C" {

tperm_status_t tperm_expert_route(const void* scores, int64_t scores_stride, int32_t* expert, float* weights, int64_t tokens, int64_t slots,
                                  int64_t experts, int over_all, int type, void* hip_stream) {
    int64_t rows = 0;
    const tperm_status_t st = count_rows(tokens, slots, experts, &rows);
    if (st != TPERM_OK) return st;
    if (!known_stride(scores_stride, experts)) return TPERM_ERR_DIMS;
    if (!known_type(type)) return TPERM_ERR_ELEM_SIZE;
    const size_t elem = type_bytes(type);
    const Array arrays[] = {{scores, matrix_bytes(tokens, scores_stride, experts, elem), elem, false}, {expert, rows * 4, 4, true}, {weights, rows * 4, 4, true}};
    const tperm_status_t bad = check(arrays);
    if (bad != TPERM_OK || rows == 0) return bad;
    RouteArgs a = {};
    a.scores = scores, a.expert = expert, a.weights = weights, a.scores_stride = scores_stride;
    a.tokens = (uint32_t)tokens, a.slots = (uint32_t)slots, a.experts = (uint32_t)experts;
    return launched(launch_route(a, over_all != 0, type, (hipStream_t)hip_stream));
}

tperm_status_t tperm_expert_route_backward(const float* grad_weights, const void* scores, int64_t scores_stride, const int32_t* expert,
                                           const float* weights, void* grad_scores, int64_t grad_scores_stride, int64_t tokens, int64_t slots,
                                           int64_t experts, int over_all, int type, void* hip_stream) {
    int64_t rows = 0;
    const tperm_status_t st = count_rows(tokens, slots, experts, &rows);
    if (st != TPERM_OK) return st;
    if ((over_all && !known_stride(scores_stride, experts)) || !known_stride(grad_scores_stride, experts)) return TPERM_ERR_DIMS;
    if (!known_type(type)) return TPERM_ERR_ELEM_SIZE;
    const size_t elem = type_bytes(type);
    const Array arrays[] = {{grad_weights, rows * 4, 4, false},
                            {scores, over_all ? matrix_bytes(tokens, scores_stride, experts, elem) : 0, elem, false},
                            {expert, rows * 4, 4, false},
                            {weights, rows * 4, 4, false},
                            {grad_scores, matrix_bytes(tokens, grad_scores_stride, experts, elem), elem, true}};
    const tperm_status_t bad = check(arrays);
    if (bad != TPERM_OK || rows == 0) return bad;
    RouteArgs a = {};
    a.scores = scores, a.grad_weights = grad_weights, a.expert = const_cast<int32_t*>(expert), a.weights = const_cast<float*>(weights), a.grad_scores = grad_scores;
    a.scores_stride = scores_stride, a.grad_stride = grad_scores_stride;
    a.tokens = (uint32_t)tokens, a.slots = (uint32_t)slots, a.experts = (uint32_t)experts;
    return launched(launch_route_backward(a, over_all != 0, type, (hipStream_t)hip_stream));
}

tperm_status_t tperm_four_bit_store(const void* x, int64_t x_stride, uint8_t* codes, uint8_t* scales, int64_t rows, int64_t width, int type, void* hip_stream) {
    if (rows < 0 || !known_width(width) || !known_stride(x_stride, width)) return TPERM_ERR_DIMS;
    if (!known_type(type)) return TPERM_ERR_ELEM_SIZE;
    if (rows > kRowsMax) return TPERM_ERR_TOO_LARGE;
    const size_t elem = type_bytes(type);
    const int64_t groups = rows * TPERM_FOUR_BIT_GROUPS(width);
    const Array arrays[] = {{x, matrix_bytes(rows, x_stride, width, elem), elem, false}, {codes, groups * 16, 16, true}, {scales, groups, 1, true}};
    const tperm_status_t bad = check(arrays);
    if (bad != TPERM_OK || rows == 0) return bad;
    FourBitArgs a = {};
    a.in = x, a.codes = codes, a.scales = scales, a.stride = x_stride, a.rows = (uint32_t)rows, a.width = (uint32_t)width;
    return launched(launch_four_bit_store(a, type, (hipStream_t)hip_stream));
}

tperm_status_t tperm_four_bit_load(const uint8_t* codes, const uint8_t* scales, void* out, int64_t out_stride, int64_t rows, int64_t width, int type,
                                   void* hip_stream) {
    if (rows < 0 || !known_width(width) || !known_stride(out_stride, width)) return TPERM_ERR_DIMS;
    if (!known_type(type)) return TPERM_ERR_ELEM_SIZE;
    if (rows > kRowsMax) return TPERM_ERR_TOO_LARGE;
    const size_t elem = type_bytes(type);
    const int64_t groups = rows * TPERM_FOUR_BIT_GROUPS(width);
    const Array arrays[] = {{codes, groups * 16, 16, false}, {scales, groups, 1, false}, {out, matrix_bytes(rows, out_stride, width, elem), elem, true}};
    const tperm_status_t bad = check(arrays);
    if (bad != TPERM_OK || rows == 0) return bad;
    FourBitArgs a = {};
    a.out = out, a.codes = const_cast<uint8_t*>(codes), a.scales = const_cast<uint8_t*>(scales), a.stride = out_stride, a.rows = (uint32_t)rows, a.width = (uint32_t)width;
    return launched(launch_four_bit_load(a, type, (hipStream_t)hip_stream));
}

tperm_status_t tperm_four_bit_product(const void* x, int64_t x_stride, const uint8_t* codes, const uint8_t* scales, void* out, int64_t out_stride,
                                      int64_t rows, int64_t k, int64_t n, int type, void* hip_stream) {
    if (rows < 0 || !known_width(k) || !known_width(n) || !known_stride(x_stride, k) || !known_stride(out_stride, n)) return TPERM_ERR_DIMS;
    if (!known_type(type)) return TPERM_ERR_ELEM_SIZE;
    const int64_t groups = n * TPERM_FOUR_BIT_GROUPS(k);
    if (rows > kRowsMax || groups * 16 > kOperandBytes) return TPERM_ERR_TOO_LARGE;
    if (rows == 0) return TPERM_OK;
    const size_t elem = type_bytes(type);
    const Array arrays[] = {{x, matrix_bytes(rows, x_stride, k, elem), elem, false},
                            {codes, groups * 16, 16, false},
                            {scales, groups, 1, false},
                            {out, matrix_bytes(rows, out_stride, n, elem), elem, true}};
    const tperm_status_t bad = check(arrays);
    if (bad != TPERM_OK) return bad;
    FourBitProductArgs a = {};
    a.x = x, a.codes = codes, a.scales = scales, a.out = out, a.x_stride = x_stride, a.out_stride = out_stride;
    a.rows = (uint32_t)rows, a.k = (uint32_t)k, a.n = (uint32_t)n;
    return launched(launch_four_bit_product(a, type, (hipStream_t)hip_stream));
}

static tperm_status_t few_sizes(int64_t tokens, int64_t slots, int64_t experts, int64_t width, int64_t hidden, int type) {
    int64_t rows = 0;
    const tperm_status_t st = count_rows(tokens, slots, experts, &rows);
    if (st != TPERM_OK) return st;
    if (tokens > TPERM_FEW_TOKENS || !known_width(width) || !known_width(hidden) || !known_width(2 * hidden)) return TPERM_ERR_DIMS;
    return known_type(type) ? TPERM_OK : TPERM_ERR_ELEM_SIZE;
}

size_t tperm_expert_few_workspace(int64_t tokens, int64_t slots, int64_t experts, int64_t width, int64_t hidden, int type, int four_bits) {
    if (few_sizes(tokens, slots, experts, width, hidden, type) != TPERM_OK || tokens == 0) return 0;
    return few_room(tokens, slots, experts, width, hidden, type, four_bits != 0).bytes;
}

tperm_status_t tperm_expert_few(const void* x, int64_t x_stride, const int32_t* expert, const float* weights, const void* w_in,
                                const uint8_t* w_in_scales, const void* w_out, const uint8_t* w_out_scales, void* out, int64_t out_stride,
                                void* workspace, size_t workspace_bytes, int64_t tokens, int64_t slots, int64_t experts, int64_t width, int64_t hidden,
                                int type, void* hip_stream) {
    const tperm_status_t st = few_sizes(tokens, slots, experts, width, hidden, type);
    if (st != TPERM_OK) return st;
    if (!known_stride(x_stride, width) || !known_stride(out_stride, width)) return TPERM_ERR_DIMS;
    if ((w_in_scales == nullptr) != (w_out_scales == nullptr)) return TPERM_ERR_NULL;
    const bool four = w_in_scales != nullptr;
    const size_t elem = type_bytes(type), w_align = four ? 16 : elem;
    const int64_t in_groups = 2 * hidden * TPERM_FOUR_BIT_GROUPS(width), out_groups = width * TPERM_FOUR_BIT_GROUPS(hidden);
    const int64_t in_bytes = four ? in_groups * 16 : 2 * hidden * width * (int64_t)elem, out_bytes = four ? out_groups * 16 : hidden * width * (int64_t)elem;
    if (in_bytes > kOperandBytes || out_bytes > kOperandBytes) return TPERM_ERR_TOO_LARGE;
    if (tokens == 0) return TPERM_OK;
    const FewRoom room = few_room(tokens, slots, experts, width, hidden, type, four);
    const Array arrays[] = {{x, matrix_bytes(tokens, x_stride, width, elem), elem, false},
                            {expert, tokens * slots * 4, 4, false},
                            {weights, weights ? tokens * slots * 4 : 0, 4, false},
                            {w_in, experts * in_bytes, w_align, false},
                            {w_in_scales, four ? experts * in_groups : 0, 1, false},
                            {w_out, experts * out_bytes, w_align, false},
                            {w_out_scales, four ? experts * out_groups : 0, 1, false},
                            {out, matrix_bytes(tokens, out_stride, width, elem), elem, true},
                            {workspace, (int64_t)room.bytes, 16, true}};
    const tperm_status_t bad = check(arrays);
    if (bad != TPERM_OK) return bad;
    if (workspace_bytes < room.bytes) return TPERM_ERR_TOO_LARGE;
    FewArgs a = {};
    a.x = x, a.expert = expert, a.weights = weights, a.w_in = w_in, a.w_out = w_out, a.in_scales = w_in_scales, a.out_scales = w_out_scales, a.out = out;
    a.x_stride = x_stride, a.out_stride = out_stride;
    a.tokens = (uint32_t)tokens, a.slots = (uint32_t)slots, a.experts = (uint32_t)experts, a.width = (uint32_t)width, a.hidden = (uint32_t)hidden;
    a.room = room, a.rows = workspace;
    return launched(launch_few(a, type, (hipStream_t)hip_stream));
}

}  // extern "C"
