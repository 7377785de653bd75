// Products of rows of type __bf16 with 4-bit weights.
#include "matvec4.h"

namespace lb {

template hipError_t matvec4_of<__bf16>(const Matvec4Args&, hipStream_t);
template size_t matvec4_space<__bf16>(const Packed4&, int64_t);

}  // namespace lb
