// The residual join (lazymar_join, lazymar_join_grad): what the kernels take.
#pragma once

#include "block8.cuh"
#include "join_host.h"

namespace lm {

// Rows of fp32, bf16 or 8-bit blocks. vec: rows start on boundaries of eight elements (8-bit ones always do).
struct Rows {
  const void* p;
  const uint8_t* scale;
  int ld, lds, dtype;
  bool vec;
};

struct Join {
  int M, D, group, post, pre;
  float res, eps;
  Rows x, y, gate, scale, shift;
  const float *post_g, *post_b, *pre_g, *pre_b;
  bool params_vec;        // the four on boundaries of eight elements (or NULL)
  MatOut z, h;
  lazymar_block8 h8, z8, y8;
  float *y_mean, *y_rstd, *z_mean, *z_rstd;
};

struct JoinGrad {
  int M, D, group, post, pre;
  float res;
  bool accumulate;
  Rows dh, dz, z, y, gate, scale;
  const float *y_mean, *y_rstd, *z_mean, *z_rstd;
  const float *post_g, *post_b, *pre_g, *pre_b;
  bool params_vec;
  MatOut dx, dy;
  lazymar_block8 dy8;
  MatOut dgate, dscale, dshift;
  float *dpost_g, *dpost_b, *dpre_g, *dpre_b;
  float* ws;  // on a boundary of kSumsAlign bytes
};

cudaError_t launch_join(const Ctx& c, const Join& p);
cudaError_t launch_join_grad(const Ctx& c, const JoinGrad& p);
size_t join_grad_workspace(int M, int D, int group);

}  // namespace lm
