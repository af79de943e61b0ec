#include "few_layer.hpp"

namespace tperm {

template hipError_t few_of<_Float16>(const FewArgs&, hipStream_t);

}  // namespace tperm
