// What the residual join's host and device code agree on, apart from CUDA's headers.
#pragma once

#include <cstddef>
#include <cstdint>

#ifdef __CUDACC__
#define LM_BOTH __host__ __device__ __forceinline__
#else
#define LM_BOTH inline
#endif

namespace lm {

// A tensor of rows of `columns` elements of `e` bytes, `pitch` bytes apart: the end of its last row.
LM_BOTH uintptr_t rows_end(uintptr_t first_row, size_t last_row, size_t pitch, int columns, uint32_t e) {
  return first_row + last_row * pitch + (size_t)(unsigned)columns * e;
}
// Whether a piece of a row (n bytes from p on), copied from the 16-byte boundary before it to the one behind it, reaches
// outside the tensor, whose bytes lie from `lowest` to `end`.
LM_BOTH bool piece_reaches_out(uintptr_t p, uint32_t n, uintptr_t lowest, uintptr_t end) {
  return (p & ~(uintptr_t)15) < lowest || ((p + n + 15) & ~(uintptr_t)15) > end;
}

// The gradient's sums over rows lie on boundaries of eight floats, which the kernels read and write at once. A caller's
// workspace starts on a boundary of 16 bytes, so it has room for a step to the next one.
constexpr size_t kSumsAlign = 32;
inline size_t join_sums_bytes(size_t floats) { return floats * sizeof(float) + kSumsAlign - 16; }
inline float* join_sums_at(void* workspace) {
  return reinterpret_cast<float*>((reinterpret_cast<uintptr_t>(workspace) + kSumsAlign - 1) & ~(uintptr_t)(kSumsAlign - 1));
}

}  // namespace lm
