// The optimizer's operators over a list of tensors (lazymar_params_*).
#pragma once

#include "lazymar_internal.cuh"

namespace lm {

// Tensors are worked on in pieces of kPiece elements (a whole number of them where a
// list would have more than kMostPieces), in an order that a table in device memory holds.
constexpr int kPiece = 4096;
constexpr long long kMostPieces = 1 << 20;

enum : unsigned { PARAM_G_BF16 = 1u, PARAM_OUT_BF16 = 2u, PARAM_VEC_G = 4u, PARAM_VEC_OUT = 8u, PARAM_VEC_ALL = 16u };

struct Param {
  const void* g;
  void* out;
  float *p, *m, *v, *ema;
  bf16* copy;
  long long n;
  float lr_scale, weight_decay;
  unsigned flags;
};
struct Piece {
  unsigned tensor, index;  // elements index * piece ..
};
struct ParamList {
  const Param* params;
  const Piece* pieces;
  double* partial;  // one of each CTA of the norm
  int n_pieces;
  int piece;        // elements of a piece
};
struct AdamW {
  float lr, eps;
  float more1, more2, more_ema;  // 1 - beta1, 1 - beta2, 1 - ema_decay
  float log1, log2;              // log beta1, log beta2
  const float* lr_device;
  float factor;
  int steps;
};

constexpr int kNormCtasPerSm = 8;
cudaError_t launch_grad_norm(const Ctx& c, const ParamList& l, double scale, double max_norm, lazymar_step_state* state);
cudaError_t launch_clip_grads(const Ctx& c, const ParamList& l, const lazymar_step_state* state);
cudaError_t launch_adamw(const Ctx& c, const ParamList& l, const AdamW& a, const lazymar_step_state* state);

}  // namespace lm
