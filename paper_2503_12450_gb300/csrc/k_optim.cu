// The end of a training step over a list of tensors: the norm of all gradients,
// their clipping, AdamW. All three are single passes bound by HBM bandwidth: 4 or 2
// bytes an element for the norm, 38 for AdamW with averaged weights and a bf16 copy. A
// CTA takes pieces of 8192 elements, whichever tensors they belong to, so that a list of any make-up is one
// launch. 403 million weights (floors at the rate of a copy): norm of fp32 gradients 221 us (238), of bf16 118 (119), AdamW 2197
// (2258); clipping 157 million from fp32 to fp32 182 (186).
#include "optim.cuh"
#include "rows.cuh"

#include <algorithm>

namespace lm {

namespace {

constexpr int kThreads = 256;

// The pieces of a CTA, as far apart as there are CTAs, first to last or last to first. The table never changes, so
// its first entry is read before the preceding kernel is waited for, and the next while one is worked on.
template <bool BACKWARD, typename F>
__device__ __forceinline__ void for_pieces(const ParamList& l, const Piece& first, const F& f) {
  Piece next = first;
  for (int i = blockIdx.x; i < l.n_pieces; i += gridDim.x) {
    const Piece now = next;
    const int j = i + gridDim.x;
    if (j < l.n_pieces) next = l.pieces[BACKWARD ? l.n_pieces - 1 - j : j];
    f(now);
  }
}
template <bool BACKWARD>
__device__ __forceinline__ Piece first_piece(const ParamList& l) {
  const int i = (int)blockIdx.x < l.n_pieces ? (int)blockIdx.x : 0;
  return l.pieces[BACKWARD ? l.n_pieces - 1 - i : i];
}
// Where a piece starts in its tensor.
template <typename T>
__device__ __forceinline__ long long offset_of(const Param& t, const Piece& q) {
  return static_cast<const T*>(q.g) - static_cast<const T*>(t.g);
}

// ---------------------------------------------------------------------------
// Norm
// ---------------------------------------------------------------------------
// Squares are summed in fp32 over eight elements, and those sums in two fp32 numbers (the sum and what its roundings
// have lost), because one conversion to fp64 and one addition for every 16 elements already bound the norm of bf16
// gradients (403 million: 292 us, floor 119). Where a sum of eight says that squares may have left fp32's range, or that the
// sum of all could (from 2^96 on, or below 2^-90 without being all zeros), they are squared in fp64.
struct Squares {
  float sum = 0.f, lost = 0.f;
  double rest = 0.0;

  __device__ __forceinline__ void add8(const float (&a)[8]) {
    const float s = squares8(a);
    if (s >= 0x1p-90f && s < 0x1p96f) {
      const float t = sum + s, b = t - sum;
      lost += (sum - (t - b)) + (s - b);
      sum = t;
    } else {
      uint32_t any = 0;  // (gradients that are all zero, as behind a gate of zero, stay cheap)
#pragma unroll
      for (int i = 0; i < 8; ++i) any |= __float_as_uint(a[i]) << 1;
      if (any)
        for (int i = 0; i < 8; ++i) rest += (double)a[i] * a[i];
    }
  }
  __device__ __forceinline__ double total() const { return rest + (double)sum + (double)lost; }
};

// Vectors of eight that a thread of the norm has under way: 64 bytes.
template <typename T>
constexpr int kVecs = sizeof(T) == 4 ? 2 : 4;

template <typename T>
__device__ __forceinline__ void squares_of(Squares& d, const T* g, int n, int head) {
  constexpr int U = kVecs<T>;
  if ((int)threadIdx.x < head) {
    const double x = (double)to_f(g[threadIdx.x]);
    d.rest += x * x;
  }
  g += head;
  n -= head;
  int k = 8 * (int)threadIdx.x;
  for (; k - 8 * (int)threadIdx.x + U * 8 * kThreads <= n; k += U * 8 * kThreads) {
    float v[U][8];
#pragma unroll
    for (int j = 0; j < U; ++j) ld8a(g + k + 8 * kThreads * j, v[j]);
#pragma unroll
    for (int j = 0; j < U; ++j) d.add8(v[j]);
  }
#pragma unroll 1
  for (; k < n; k += 8 * kThreads) {
    float v[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = 0.f;
    if (k + 8 <= n) {
      ld8a(g + k, v);
    } else {
#pragma unroll
      for (int i = 0; i < 8; ++i)
        if (k + i < n) v[i] = to_f(g[k + i]);
    }
    d.add8(v);
  }
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
    // (a subnormal number where gradients are near fp32's end, but never 0, which says that the step is skipped)
    state->factor = fmaxf((float)(norm > max_norm ? scale * (max_norm / norm) : scale), 0x1p-149f);
    state->steps += 1;
  } else {
    state->factor = 0.f;
    state->skipped += 1;
  }
}

// The CTA that is done last adds all CTAs' sums, each of its threads every 256th, in a fixed order.
__global__ void __launch_bounds__(kThreads, kMostNormCtas) grad_norm_kernel(const ParamList l, double scale, double max_norm,
                                                                            lazymar_step_state* state) {
  __shared__ bool last;
  const Piece first = first_piece<false>(l);
  pdl_wait();
  pdl_trigger();
  Squares squares;
  for_pieces<false>(l, first, [&](const Piece& q) {
    if (q.is_bf16()) squares_of(squares, static_cast<const bf16*>(q.g), q.n(), q.head());
    else squares_of(squares, static_cast<const float*>(q.g), q.n(), q.head());
  });
  double d = cta_sum(squares.total());
  if (gridDim.x > 1) {
    if (threadIdx.x == 0) {
      l.partial[blockIdx.x] = d;
      __threadfence();
      last = atomicAdd(l.arrived, 1u) == gridDim.x - 1;
    }
    __syncthreads();
    if (!last) return;
    __threadfence();
    d = 0.0;
    for (int i = threadIdx.x; i < (int)gridDim.x; i += kThreads) d += __ldcg(l.partial + i);
    d = cta_sum(d);
    if (threadIdx.x == 0) *l.arrived = 0u;
  }
  if (threadIdx.x == 0) finish_norm(d, scale, max_norm, state);
}

// ---------------------------------------------------------------------------
// Clipping
// ---------------------------------------------------------------------------
template <typename T, typename O>
__device__ __forceinline__ void clip_piece(const T* g, O* out, int n, int head, bool vec, float factor) {
  const auto clipped = [&](float x) { return factor == 0.f ? 0.f : x * factor; };
  if (vec) {
    if ((int)threadIdx.x < head) out[threadIdx.x] = from_f<O>(clipped(to_f(g[threadIdx.x])));
    g += head;
    out += head;
    n -= head;
    constexpr int U = 4;
    int k = 8 * (int)threadIdx.x;
    for (; k - 8 * (int)threadIdx.x + U * 8 * kThreads <= n; k += U * 8 * kThreads) {
      float v[U][8];
#pragma unroll
      for (int j = 0; j < U; ++j) ld8a(g + k + 8 * kThreads * j, v[j]);
#pragma unroll
      for (int j = 0; j < U; ++j) {
#pragma unroll
        for (int i = 0; i < 8; ++i) v[j][i] = clipped(v[j][i]);
        st8a(out + k + 8 * kThreads * j, v[j]);
      }
    }
#pragma unroll 1
    for (; k < n; k += 8 * kThreads) {
      float v[8];
      if (k + 8 <= n) {
        ld8a(g + k, v);
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = clipped(v[i]);
        st8a(out + k, v);
      } else {
        for (int i = k; i < n; ++i) out[i] = from_f<O>(clipped(to_f(g[i])));
      }
    }
    return;
  }
  for (int k = (int)threadIdx.x; k < n; k += 8 * kThreads) {
    float v[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = k + kThreads * i < n ? to_f(g[k + kThreads * i]) : 0.f;
#pragma unroll
    for (int i = 0; i < 8; ++i)
      if (k + kThreads * i < n) out[k + kThreads * i] = from_f<O>(clipped(v[i]));
  }
}

// Last piece first: what the norm has read last is still in L2.
__global__ void __launch_bounds__(kThreads, 4) clip_grads_kernel(const ParamList l, const lazymar_step_state* state) {
  const Piece first = first_piece<true>(l);
  pdl_wait();
  pdl_trigger();
  const float factor = state->factor;
  for_pieces<true>(l, first, [&](const Piece& q) {
    const Param& t = l.params[q.tensor];
    if (factor == 1.f && t.out == t.g) return;  // (in place: nothing to do)
    const bool vec = t.flags & PARAM_VEC_OUT;
    const long long at = q.is_bf16() ? offset_of<bf16>(t, q) : offset_of<float>(t, q);
    const float* gf = static_cast<const float*>(q.g);
    const bf16* gb = static_cast<const bf16*>(q.g);
    float* of = static_cast<float*>(t.out) + at;
    bf16* ob = static_cast<bf16*>(t.out) + at;
    switch (t.flags & (PARAM_G_BF16 | PARAM_OUT_BF16)) {
      case 0: clip_piece(gf, of, q.n(), q.head(), vec, factor); break;
      case PARAM_G_BF16: clip_piece(gb, of, q.n(), q.head(), vec, factor); break;
      case PARAM_OUT_BF16: clip_piece(gf, ob, q.n(), q.head(), vec, factor); break;
      default: clip_piece(gb, ob, q.n(), q.head(), vec, factor);
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
__device__ __forceinline__ void adamw_piece(const AdamW& a, const Step& s, const Param& t, const Piece& q) {
  const long long first = offset_of<T>(t, q);
  const int n = q.n();
  const T* g = static_cast<const T*>(q.g);
  float *p = t.p + first, *m = t.m + first, *v = t.v + first, *ema = t.ema ? t.ema + first : nullptr;
  bf16* copy = t.copy ? t.copy + first : nullptr;
  auto one = [&](int i) {
    float pp = p[i], mm = m[i], vv = v[i];
    adamw_one(a, s, to_f(g[i]), pp, mm, vv);
    p[i] = pp;
    m[i] = mm;
    v[i] = vv;
    if (ema) ema[i] = fmaf(a.more_ema, pp - ema[i], ema[i]);
    if (copy) copy[i] = from_f<bf16>(pp);
  };
  if (!(t.flags & PARAM_VEC_ALL)) {
    for (int i = threadIdx.x; i < n; i += kThreads) one(i);
    return;
  }
  if ((int)threadIdx.x < q.head()) one(threadIdx.x);
#pragma unroll 1
  for (int i = q.head() + 8 * (int)threadIdx.x; i < n; i += 8 * kThreads) {
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

__global__ void __launch_bounds__(kThreads, 3) adamw_kernel(const ParamList l, const AdamW a,
                                                         const lazymar_step_state* state) {
  const Piece first = first_piece<true>(l);
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
  for_pieces<true>(l, first, [&](const Piece& q) {  // (as above)
    const Param& t = l.params[q.tensor];
    s.lr = lr * t.lr_scale;
    s.decay = s.lr * t.weight_decay;
    if (q.is_bf16()) adamw_piece<bf16>(a, s, t, q);
    else adamw_piece<float>(a, s, t, q);
  });
}

// CTAs of a launch: at most per_sm for each SM, with as many pieces each.
unsigned ctas(const Ctx& c, const ParamList& l, int per_sm) {
  const int most = c.num_sms * per_sm, rounds = (l.n_pieces + most - 1) / most;
  return (unsigned)((l.n_pieces + rounds - 1) / rounds);
}

}  // namespace

cudaError_t launch_grad_norm(const Ctx& c, const ParamList& l, double scale, double max_norm, lazymar_step_state* state) {
  // (Where a CTA has few pieces, more loads under way at first gain more than the same share for each: 8.4 million fp32
  // gradients 12.7 us with all CTAs that live at once, 13.8 with as many pieces each; 403 million in bf16 118.0 and 116.5.)
  const int most = c.num_sms * kMostNormCtas;
  const unsigned n = l.n_pieces == 0 ? 1u : l.n_pieces > 4 * most ? ctas(c, l, kMostNormCtas) : (unsigned)std::min(l.n_pieces, most);
  return launch_pdl(grad_norm_kernel, dim3(n), dim3(kThreads), 0, c.stream, l, scale, max_norm, state);
}

// The passes that write have more CTAs than live at once, so that what is read and written at a time lies together:
// clipping 157 million fp32 gradients 183 us with eight times as many, 195 with the resident ones alone; AdamW of
// 403 million weights 2197 us with a CTA for each piece, 2321 with four times the resident ones, 2404 with these alone.
cudaError_t launch_clip_grads(const Ctx& c, const ParamList& l, const lazymar_step_state* state) {
  if (l.n_pieces == 0) return cudaSuccess;
  return launch_pdl(clip_grads_kernel, dim3(ctas(c, l, 32)), dim3(kThreads), 0, c.stream, l, state);
}

cudaError_t launch_adamw(const Ctx& c, const ParamList& l, const AdamW& a, const lazymar_step_state* state) {
  if (l.n_pieces == 0) return cudaSuccess;
  return launch_pdl(adamw_kernel, dim3((unsigned)l.n_pieces), dim3(kThreads), 0, c.stream, l, a, state);
}

}  // namespace lm
