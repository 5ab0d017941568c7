// The optimizer's operators over a list of tensors (lazymar_params_*).
#pragma once

#include "lazymar_internal.cuh"

namespace lm {

// Tensors are worked on in pieces of kPiece elements (a whole number of them where a list would have more than
// kMostPieces). A piece starts on a boundary of eight elements of the gradient, apart from a tensor's first one, which has
// up to seven elements more in front of it (its head).
constexpr int kPiece = 8192;
constexpr long long kMostPieces = 1 << 20;

// VEC_OUT, VEC_ALL: out, or all of p, m, v, ema and copy, lie on such a boundary where g does.
enum : unsigned { PARAM_G_BF16 = 1u, PARAM_OUT_BF16 = 2u, PARAM_VEC_OUT = 4u, PARAM_VEC_ALL = 8u };

struct Param {
  const void* g;
  void* out;
  float *p, *m, *v, *ema;
  bf16* copy;
  float lr_scale, weight_decay;
  unsigned flags;
};
struct Piece {
  const void* g;
  unsigned tensor;
  unsigned bits;  // elements (24 bits), those of the head (3), whether g is bf16 (1)
  __host__ __device__ int n() const { return (int)(bits & 0xFFFFFFu); }
  __host__ __device__ int head() const { return (int)(bits >> 24 & 7u); }
  __host__ __device__ bool is_bf16() const { return bits >> 27 & 1u; }
};
inline Piece piece_of(const void* g, unsigned tensor, int n, int head, bool is_bf16) {
  return Piece{g, tensor, (unsigned)n | (unsigned)head << 24 | (unsigned)is_bf16 << 27};
}
struct ParamList {
  const Param* params;
  const Piece* pieces;
  double* partial;    // one of each CTA of the norm
  unsigned* arrived;  // its CTAs that are done
  int n_pieces;
};
struct AdamW {
  float lr, eps;
  float more1, more2, more_ema;  // 1 - beta1, 1 - beta2, 1 - ema_decay
  float log1, log2;              // log beta1, log beta2
  const float* lr_device;
  float factor;
  int steps;
};

constexpr int kMostNormCtas = 5;  // on an SM
cudaError_t launch_grad_norm(const Ctx& c, const ParamList& l, double scale, double max_norm, lazymar_step_state* state);
cudaError_t launch_clip_grads(const Ctx& c, const ParamList& l, const lazymar_step_state* state);
cudaError_t launch_adamw(const Ctx& c, const ParamList& l, const AdamW& a, const lazymar_step_state* state);

}  // namespace lm
