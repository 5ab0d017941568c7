// The residual join's gradient without a norm of y and without parameters: rows that share a modulation.
#include "join_grad.cuh"

namespace lm {

cudaError_t launch_join_grad_plain(const Ctx& c, const JoinGrad& p, const JoinSums& need, bool whole, const Teams& ranges, bool together) {
  return join_grad_launch<false, true>(c, p, need, whole, ranges, together);
}

}  // namespace lm
