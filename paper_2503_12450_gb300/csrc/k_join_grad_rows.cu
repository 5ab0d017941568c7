// The residual join's gradient where every row has a modulation of its own.
#include "join_grad.cuh"

namespace lm {

cudaError_t launch_join_grad_rowwise(const Ctx& c, const JoinGrad& p, const JoinSums& need, bool whole, const Teams& ranges, bool together) {
  return join_grad_launch<true, false>(c, p, need, whole, ranges, together);
}

}  // namespace lm
