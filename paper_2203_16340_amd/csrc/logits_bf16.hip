// The losses on rows of logits of type __bf16.
#include "logits_rows.h"

namespace lb {

template hipError_t token_logprob_rows<__bf16>(const LogitsArgs&, const TokenArgs&, SplitRow*, hipStream_t);
template hipError_t token_grad_rows<__bf16>(const LogitsArgs&, const TokenGradArgs&, hipStream_t);
template hipError_t policy_rows<__bf16>(const LogitsArgs&, const PolicyArgs&, float*, SplitRow*, hipStream_t);
template hipError_t distill_rows<__bf16>(const LogitsArgs&, const DistillArgs&, float*, SplitRow*, hipStream_t);

}  // namespace lb
