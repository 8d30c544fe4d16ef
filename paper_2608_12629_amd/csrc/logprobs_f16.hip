// logprobs_f16.hip -- f16 instantiation of logprobs.h.
#include "logprobs.h"

namespace fkm {

hipError_t launch_logprobs_f16(const LogprobsArgs& a, const LogprobsWs& w, hipStream_t s) {
  return launch_logprobs_dt<DT_F16>(a, w, s);
}
hipError_t launch_logprobs_grad_f16(const GradArgs& a, const GradWs& w, hipStream_t s) {
  return launch_grad_dt<DT_F16>(a, w, s);
}

}  // namespace fkm
