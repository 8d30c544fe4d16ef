// logprobs_bf16.hip -- bf16 instantiation of logprobs.h.
#include "logprobs.h"

namespace fkm {

hipError_t launch_logprobs_bf16(const LogprobsArgs& a, const LogprobsWs& w, hipStream_t s) {
  return launch_logprobs_dt<DT_BF16>(a, w, s);
}
hipError_t launch_logprobs_grad_bf16(const GradArgs& a, const GradWs& w, hipStream_t s) {
  return launch_grad_dt<DT_BF16>(a, w, s);
}

}  // namespace fkm
