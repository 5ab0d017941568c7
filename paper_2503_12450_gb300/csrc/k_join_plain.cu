// The residual join of many rows without a norm of y and without parameters.
#include "join_ring.cuh"

namespace lm {

cudaError_t launch_join_plain(const Ctx& c, const Join& p, bool whole) { return join_ring_launch<true>(c, p, whole); }

}  // namespace lm
