#include "few_layer.hpp"

namespace tperm {

template hipError_t few_of<__bf16>(const FewArgs&, hipStream_t);

}  // namespace tperm
