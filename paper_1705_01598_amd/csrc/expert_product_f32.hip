// Experts' products of f32 elements (one translation unit per type: they compile side by side).
#include "expert_product_inst.hpp"

namespace tperm {
template hipError_t product_of<float>(const ExpertProductArgs&, bool, hipStream_t);
template hipError_t gradient_of<float>(const WeightGradientArgs&, hipStream_t);
}  // namespace tperm
