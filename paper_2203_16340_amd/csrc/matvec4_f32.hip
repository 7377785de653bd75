// Products of rows of type float with 4-bit weights.
#include "matvec4.h"

namespace lb {

template hipError_t matvec4_of<float>(const Matvec4Args&, hipStream_t);
template size_t matvec4_space<float>(const Packed4&, int64_t);

}  // namespace lb
