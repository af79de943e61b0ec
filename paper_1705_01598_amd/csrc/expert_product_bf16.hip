// Experts' products of bf16 elements (one translation unit per type: they compile side by side).
#include "expert_product_inst.hpp"

namespace tperm {
template hipError_t product_of<__bf16>(const ExpertProductArgs&, bool, hipStream_t);
template hipError_t gradient_of<__bf16>(const WeightGradientArgs&, hipStream_t);
}  // namespace tperm
