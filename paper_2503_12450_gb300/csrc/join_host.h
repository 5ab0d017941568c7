// What the residual join's host and device code agree on, apart from CUDA's headers.
#pragma once

#include <cstddef>
#include <cstdint>

namespace lm {

// The gradient's sums over rows lie on boundaries of eight floats, which the kernels read and write at once. A caller's
// workspace starts on a boundary of 16 bytes, so it has room for a step to the next one.
constexpr size_t kSumsAlign = 32;
inline size_t join_sums_bytes(size_t floats) { return floats * sizeof(float) + kSumsAlign - 16; }
inline float* join_sums_at(void* workspace) {
  return reinterpret_cast<float*>((reinterpret_cast<uintptr_t>(workspace) + kSumsAlign - 1) & ~(uintptr_t)(kSumsAlign - 1));
}

}  // namespace lm
