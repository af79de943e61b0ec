// Experts' products of f16 elements (one translation unit per type: they compile side by side).
#include "expert_product_inst.hpp"

namespace tperm {
template hipError_t product_of<_Float16>(const ExpertProductArgs&, bool, hipStream_t);
template hipError_t gradient_of<_Float16>(const WeightGradientArgs&, hipStream_t);
}  // namespace tperm
