// The end of a training step over a list of tensors: the norm of all gradients,
// their clipping, AdamW. All three are single passes bound by HBM bandwidth: 4 or 2
// bytes an element for the norm, 38 for AdamW with averaged weights and a bf16 copy. A
// CTA takes pieces of 4096 elements in turn, whichever tensors they belong to, so that
// a list of any make-up is one launch.
#include "optim.cuh"
#include "rows.cuh"

namespace lm {

namespace {

constexpr int kThreads = 256;

// The pieces of a CTA, `step` apart; the next piece's entry is on its way while one is worked on.
template <typename F>
__device__ __forceinline__ void for_pieces(const ParamList& l, const F& f) {
  int i = blockIdx.x;
  if (i >= l.n_pieces) return;
  Piece next = l.pieces[i];
  while (true) {
    const Piece now = next;
    const int j = i + gridDim.x;
    if (j < l.n_pieces) next = l.pieces[j];
    const Param& t = l.params[now.tensor];
    const long long first = (long long)now.index * l.piece, n = min((long long)l.piece, t.n - first);
    f(t, first, n);
    if (j >= l.n_pieces) break;
    i = j;
  }
}

// ---------------------------------------------------------------------------
// Norm
// ---------------------------------------------------------------------------
// Squares are summed in fp32 over the 16 elements that a thread holds at once, and those
// sums in fp64. Where a sum says that squares may have left fp32's range (from 2^125 on,
// or below 2^-90 without being a sum of zeros), the 16 elements are squared in fp64.
__device__ __forceinline__ double squares16(const float (&a)[8], const float (&b)[8]) {
  const float s = squares8(a) + squares8(b);
  if (s >= 0x1p-90f && s < 0x1p125f) return (double)s;
  double d = 0.0;
#pragma unroll
  for (int i = 0; i < 8; ++i) d += (double)a[i] * a[i] + (double)b[i] * b[i];
  return d;
}

template <typename T>
__device__ __forceinline__ double squares_of(const T* g, long long n, bool vec) {
  double d = 0.0;
  for (long long k = 0; k < n; k += kPiece) {
    const int m = (int)min((long long)kPiece, n - k);
    float v[2][8];
#pragma unroll
    for (int j = 0; j < 2; ++j) {
      if (vec) {
        const int at = 8 * ((int)threadIdx.x + kThreads * j);
        if (at + 8 <= m) {
          ld8a(g + k + at, v[j]);
        } else {
#pragma unroll
          for (int i = 0; i < 8; ++i) v[j][i] = at + i < m ? to_f(g[k + at + i]) : 0.f;
        }
      } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          const int at = (int)threadIdx.x + kThreads * (8 * j + i);
          v[j][i] = at < m ? to_f(g[k + at]) : 0.f;
        }
      }
    }
    d += squares16(v[0], v[1]);
  }
  return d;
}

// Sum over the CTA, in every thread of the first warp.
__device__ __forceinline__ double cta_sum(double d) {
  __shared__ double red[32];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, warps = blockDim.x >> 5;
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) d += __shfl_xor_sync(0xffffffffu, d, o);
  if (lane == 0) red[warp] = d;
  __syncthreads();
  d = warp == 0 && lane < warps ? red[lane] : 0.0;
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) d += __shfl_xor_sync(0xffffffffu, d, o);
  return d;
}

__device__ __forceinline__ void finish_norm(double squares, double scale, double max_norm, lazymar_step_state* state) {
  const double norm = scale * sqrt(squares);
  const float f = (float)norm;
  state->norm = f;
  if (isfinite(f)) {
    // (never 0, which says that the step is skipped)
    state->factor = fmaxf((float)(norm > max_norm ? scale * (max_norm / norm) : scale), 0x1p-126f);
    state->steps += 1;
  } else {
    state->factor = 0.f;
    state->skipped += 1;
  }
}

// ONE: a single CTA has all pieces.
template <bool ONE>
__global__ void __launch_bounds__(kThreads) grad_norm_kernel(const ParamList l, double scale, double max_norm,
                                                             lazymar_step_state* state) {
  pdl_wait();
  pdl_trigger();
  double d = 0.0;
  for_pieces(l, [&](const Param& t, long long first, long long n) {
    if (t.flags & PARAM_G_BF16) d += squares_of(static_cast<const bf16*>(t.g) + first, n, t.flags & PARAM_VEC_G);
    else d += squares_of(static_cast<const float*>(t.g) + first, n, t.flags & PARAM_VEC_G);
  });
  d = cta_sum(d);
  if (threadIdx.x == 0) {
    if (ONE) finish_norm(d, scale, max_norm, state);
    else l.partial[blockIdx.x] = d;
  }
}

__global__ void __launch_bounds__(kThreads) grad_norm_finish_kernel(const double* partial, int n, double scale,
                                                                    double max_norm, lazymar_step_state* state) {
  pdl_wait();
  pdl_trigger();
  double d = 0.0;
  for (int i = threadIdx.x; i < n; i += kThreads) d += partial[i];
  d = cta_sum(d);
  if (threadIdx.x == 0) finish_norm(d, scale, max_norm, state);
}

// ---------------------------------------------------------------------------
// Clipping
// ---------------------------------------------------------------------------
template <typename T, typename O>
__device__ __forceinline__ void clip_piece(const T* g, O* out, long long n, bool vec, float factor) {
  for (long long k = 0; k < n; k += kPiece) {
    const int m = (int)min((long long)kPiece, n - k);
    if (vec) {
      float v[2][8];
#pragma unroll
      for (int j = 0; j < 2; ++j) {
        const int at = 8 * ((int)threadIdx.x + kThreads * j);
        if (at + 8 <= m) ld8a(g + k + at, v[j]);
      }
#pragma unroll
      for (int j = 0; j < 2; ++j) {
        const int at = 8 * ((int)threadIdx.x + kThreads * j);
        if (at + 8 <= m) {
#pragma unroll
          for (int i = 0; i < 8; ++i) v[j][i] = factor == 0.f ? 0.f : v[j][i] * factor;
          st8a(out + k + at, v[j]);
        } else {
          for (int i = at; i < m; ++i) out[k + i] = from_f<O>(factor == 0.f ? 0.f : to_f(g[k + i]) * factor);
        }
      }
    } else {
      float v[16];
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        const int at = (int)threadIdx.x + kThreads * i;
        v[i] = at < m ? to_f(g[k + at]) : 0.f;
      }
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        const int at = (int)threadIdx.x + kThreads * i;
        if (at < m) out[k + at] = from_f<O>(factor == 0.f ? 0.f : v[i] * factor);
      }
    }
  }
}

__global__ void __launch_bounds__(kThreads) clip_grads_kernel(const ParamList l, const lazymar_step_state* state) {
  pdl_wait();
  pdl_trigger();
  const float factor = state->factor;
  for_pieces(l, [&](const Param& t, long long first, long long n) {
    if (factor == 1.f && t.out == t.g) return;  // (in place: nothing to do)
    const bool vec = t.flags & PARAM_VEC_OUT;
    const float* gf = static_cast<const float*>(t.g) + first;
    const bf16* gb = static_cast<const bf16*>(t.g) + first;
    float* of = static_cast<float*>(t.out) + first;
    bf16* ob = static_cast<bf16*>(t.out) + first;
    switch (t.flags & (PARAM_G_BF16 | PARAM_OUT_BF16)) {
      case 0: clip_piece(gf, of, n, vec, factor); break;
      case PARAM_G_BF16: clip_piece(gb, of, n, vec, factor); break;
      case PARAM_OUT_BF16: clip_piece(gf, ob, n, vec, factor); break;
      default: clip_piece(gb, ob, n, vec, factor);
    }
  });
}

// ---------------------------------------------------------------------------
// AdamW
// ---------------------------------------------------------------------------
struct Step {
  float factor, lr, decay;      // lr: the tensor's, decay: lr weight_decay
  float inv1, inv2;             // 1 / (1 - beta^t)
};

__device__ __forceinline__ void adamw_one(const AdamW& a, const Step& s, float g, float& p, float& m, float& v) {
  g *= s.factor;
  m = fmaf(a.more1, g - m, m);
  v = fmaf(a.more2, fmaf(g, g, -v), v);
  const float step = (m * s.inv1) / (sqrtf(v * s.inv2) + a.eps);
  p = p - fmaf(s.lr, step, s.decay * p);
}

template <typename T>
__device__ __forceinline__ void adamw_piece(const AdamW& a, const Step& s, const Param& t, long long first, long long n) {
  const T* g = static_cast<const T*>(t.g) + first;
  float *p = t.p + first, *m = t.m + first, *v = t.v + first, *ema = t.ema ? t.ema + first : nullptr;
  bf16* copy = t.copy ? t.copy + first : nullptr;
  auto one = [&](long long i) {
    float pp = p[i], mm = m[i], vv = v[i];
    adamw_one(a, s, to_f(g[i]), pp, mm, vv);
    p[i] = pp;
    m[i] = mm;
    v[i] = vv;
    if (ema) ema[i] = fmaf(a.more_ema, pp - ema[i], ema[i]);
    if (copy) copy[i] = from_f<bf16>(pp);
  };
  if (!(t.flags & PARAM_VEC_ALL)) {
    for (long long i = threadIdx.x; i < n; i += kThreads) one(i);
    return;
  }
  for (long long i = 8 * threadIdx.x; i < n; i += 8 * kThreads) {
    if (i + 8 > n) {
      for (; i < n; ++i) one(i);
      break;
    }
    float vg[8], vp[8], vm[8], vv[8], ve[8];
    ld8a(g + i, vg);
    ld8a(p + i, vp);
    ld8a(m + i, vm);
    ld8a(v + i, vv);
    if (ema) ld8a(ema + i, ve);
#pragma unroll
    for (int k = 0; k < 8; ++k) {
      adamw_one(a, s, vg[k], vp[k], vm[k], vv[k]);
      ve[k] = fmaf(a.more_ema, vp[k] - ve[k], ve[k]);
    }
    st8a(p + i, vp);
    st8a(m + i, vm);
    st8a(v + i, vv);
    if (ema) st8a(ema + i, ve);
    if (copy) st8a(copy + i, vp);
  }
}

__global__ void __launch_bounds__(kThreads) adamw_kernel(const ParamList l, const AdamW a,
                                                         const lazymar_step_state* state) {
  pdl_wait();
  pdl_trigger();
  Step s;
  s.factor = state ? state->factor : a.factor;
  if (s.factor == 0.f) return;
  const float t = (float)max(state ? state->steps : a.steps, 1);
  // 1 - beta^t without cancellation
  s.inv1 = 1.f / -expm1f(t * a.log1);
  s.inv2 = 1.f / -expm1f(t * a.log2);
  const float lr = a.lr_device ? *a.lr_device : a.lr;
  for_pieces(l, [&](const Param& q, long long first, long long n) {
    s.lr = lr * q.lr_scale;
    s.decay = s.lr * q.weight_decay;
    if (q.flags & PARAM_G_BF16) adamw_piece<bf16>(a, s, q, first, n);
    else adamw_piece<float>(a, s, q, first, n);
  });
}

unsigned ctas(const Ctx& c, const ParamList& l, int per_sm) {
  const int most = c.num_sms * per_sm;
  return (unsigned)(l.n_pieces < most ? l.n_pieces : most);
}

}  // namespace

cudaError_t launch_grad_norm(const Ctx& c, const ParamList& l, double scale, double max_norm, lazymar_step_state* state) {
  if (l.n_pieces <= 4)
    return launch_pdl(grad_norm_kernel<true>, dim3(1), dim3(kThreads), 0, c.stream, l, scale, max_norm, state);
  const unsigned n = ctas(c, l, kNormCtasPerSm);
  cudaError_t e = launch_pdl(grad_norm_kernel<false>, dim3(n), dim3(kThreads), 0, c.stream, l, scale, max_norm, state);
  if (e != cudaSuccess) return e;
  return launch_pdl(grad_norm_finish_kernel, dim3(1), dim3(kThreads), 0, c.stream, (const double*)l.partial, (int)n, scale,
                    max_norm, state);
}

cudaError_t launch_clip_grads(const Ctx& c, const ParamList& l, const lazymar_step_state* state) {
  if (l.n_pieces == 0) return cudaSuccess;
  return launch_pdl(clip_grads_kernel, dim3(ctas(c, l, 8)), dim3(kThreads), 0, c.stream, l, state);
}

cudaError_t launch_adamw(const Ctx& c, const ParamList& l, const AdamW& a, const lazymar_step_state* state) {
  if (l.n_pieces == 0) return cudaSuccess;
  return launch_pdl(adamw_kernel, dim3(ctas(c, l, 8)), dim3(kThreads), 0, c.stream, l, a, state);
}

}  // namespace lm
