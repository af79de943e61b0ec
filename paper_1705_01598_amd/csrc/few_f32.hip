#include "few_layer.hpp"

namespace tperm {

template hipError_t few_of<float>(const FewArgs&, hipStream_t);

}  // namespace tperm
