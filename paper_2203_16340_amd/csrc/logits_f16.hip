// The losses on rows of logits of type _Float16.
#include "logits_rows.h"

namespace lb {

template hipError_t token_logprob_rows<_Float16>(const LogitsArgs&, const TokenArgs&, SplitRow*, hipStream_t);
template hipError_t token_grad_rows<_Float16>(const LogitsArgs&, const TokenGradArgs&, hipStream_t);
template hipError_t policy_rows<_Float16>(const LogitsArgs&, const PolicyArgs&, float*, SplitRow*, hipStream_t);
template hipError_t distill_rows<_Float16>(const LogitsArgs&, const DistillArgs&, float*, SplitRow*, hipStream_t);

}  // namespace lb
