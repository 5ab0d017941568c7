// Row-wise kernels of block training: LayerNorm's forward pass with statistics
// and 8-bit outputs, its backward pass with the column sums of the gain's and
// shift's gradients, and the passes between fp32/bf16 tensors and the 8-bit
// block format (checkpoint, GELU's gradient from a checkpoint, weights).
//
// All of them are bound by HBM bandwidth. A warp covers a block of 128 columns
// with four consecutive ones a lane: loads and stores are whole 128-byte lines
// in every type, and a block's maximum is one warp reduction.
#include "block8.cuh"

namespace lm {

namespace {

constexpr int kSMs = 152;

// ---------------------------------------------------------------------------
// Four columns of a row
// ---------------------------------------------------------------------------
__device__ __forceinline__ float4 ld4_bf16(const bf16* p) {
  const uint2 u = *reinterpret_cast<const uint2*>(p);
  const float2 a = __bfloat1622float2(*reinterpret_cast<const __nv_bfloat162*>(&u.x));
  const float2 b = __bfloat1622float2(*reinterpret_cast<const __nv_bfloat162*>(&u.y));
  return make_float4(a.x, a.y, b.x, b.y);
}
// Columns col..col+3 of a row; those from D on read as zero. vec: the row
// starts on a boundary of four elements.
template <typename T>
__device__ __forceinline__ float4 ld4(const T* row, int col, int D, bool vec) {
  if (vec && col + 4 <= D) {
    if constexpr (sizeof(T) == 2) return ld4_bf16(row + col);
    else return *reinterpret_cast<const float4*>(row + col);
  }
  float v[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) v[i] = col + i < D ? to_f(row[col + i]) : 0.f;
  return make_float4(v[0], v[1], v[2], v[3]);
}
template <typename T>
__device__ __forceinline__ void st4(T* row, int col, int D, bool vec, float4 v) {
  if (vec && col + 4 <= D) {
    if constexpr (sizeof(T) == 2)
      *reinterpret_cast<uint2*>(row + col) = make_uint2(pack_bf16(v.x, v.y), pack_bf16(v.z, v.w));
    else
      *reinterpret_cast<float4*>(row + col) = v;
    return;
  }
  const float o[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
  for (int i = 0; i < 4; ++i)
    if (col + i < D) row[col + i] = from_f<T>(o[i]);
}
// The same without a boundary: every column exists and rows are aligned.
template <typename T, bool FULL>
__device__ __forceinline__ float4 ld4t(const T* row, int col, int D, bool vec) {
  return FULL ? ld4<T>(row, col, col + 4, true) : ld4<T>(row, col, D, vec);
}
// Four E4M3 bytes of a block8 row. Rows are 16-byte aligned and padded to 16
// bytes, so the word is readable where any of its columns exists; bytes of
// columns that do not are cleared.
__device__ __forceinline__ uint32_t ldq4(const uint8_t* row, int col, int D) {
  if (col >= D) return 0u;
  uint32_t w = *reinterpret_cast<const uint32_t*>(row + col);
  if (col + 4 > D) w &= 0xFFFFFFFFu >> (8 * (col + 4 - D));
  return w;
}
// Columns at and beyond D keep what the padding held.
__device__ __forceinline__ void stq4(uint8_t* row, int col, int D, uint32_t w) {
  if (col + 4 <= D) {
    *reinterpret_cast<uint32_t*>(row + col) = w;
  } else {
    for (int i = 0; col + i < D; ++i) row[col + i] = (uint8_t)(w >> (8 * i));
  }
}
__device__ __forceinline__ float4 mask4(float4 v, int col, int D) {
  return make_float4(col < D ? v.x : 0.f, col + 1 < D ? v.y : 0.f, col + 2 < D ? v.z : 0.f, col + 3 < D ? v.w : 0.f);
}
__device__ __forceinline__ float sum4(float4 v) { return (v.x + v.y) + (v.z + v.w); }

// Sum of v over the WPR warps of a row (`red`: this row's slots in shared
// memory). Every warp of the CTA takes part.
template <int WPR>
__device__ __forceinline__ float row_sum(float v, float* red, int part) {
  v = warp_sum(v);
  if constexpr (WPR > 1) {
    if ((threadIdx.x & 31) == 0) red[part] = v;
    __syncthreads();
    float s = 0.f;
#pragma unroll
    for (int i = 0; i < WPR; ++i) s += red[i];
    v = s;
  }
  return v;
}

// ---------------------------------------------------------------------------
// LayerNorm forward
// ---------------------------------------------------------------------------
// WPR warps a row, NB blocks of 128 columns a warp, the row in registers: one
// read of x, mean and then the squared deviations from it (no cancellation).
// FULL: D = 128 NB WPR and aligned rows, so that no column needs a check.
template <int NB, int WPR, bool FULL>
__global__ void __launch_bounds__(WPR > 8 ? WPR * 32 : 256) ln_forward_kernel(const LnForward p) {
  constexpr int GROUPS = WPR > 8 ? 1 : 8 / WPR;
  __shared__ float red[2][GROUPS][WPR];
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, grp = warp / WPR, part = warp % WPR;
  const int D = p.D, row = blockIdx.x * GROUPS + grp, c0 = part * NB * kBlk + 4 * lane;
  const bool live = row < p.M;
  pdl_wait();
  pdl_trigger();
  float4 v[NB];
  if (live) {
    if (p.x.dtype == LAZYMAR_F32) {
      const float* xr = static_cast<const float*>(p.x.p) + (size_t)row * p.x.ld;
#pragma unroll
      for (int j = 0; j < NB; ++j) v[j] = ld4t<float, FULL>(xr, c0 + j * kBlk, D, p.vec);
    } else {
      const bf16* xr = static_cast<const bf16*>(p.x.p) + (size_t)row * p.x.ld;
#pragma unroll
      for (int j = 0; j < NB; ++j) v[j] = ld4t<bf16, FULL>(xr, c0 + j * kBlk, D, p.vec);
    }
  } else {
#pragma unroll
    for (int j = 0; j < NB; ++j) v[j] = make_float4(0.f, 0.f, 0.f, 0.f);
  }
  float s = 0.f;
#pragma unroll
  for (int j = 0; j < NB; ++j) s += sum4(v[j]);
  const float mean = row_sum<WPR>(s, red[0][grp], part) / (float)D;
  float q = 0.f;
#pragma unroll
  for (int j = 0; j < NB; ++j) {
    float4 d = make_float4(v[j].x - mean, v[j].y - mean, v[j].z - mean, v[j].w - mean);
    if (!FULL) d = mask4(d, c0 + j * kBlk, D);
    q += (d.x * d.x + d.y * d.y) + (d.z * d.z + d.w * d.w);
  }
  const float rstd = rsqrtf(row_sum<WPR>(q, red[1][grp], part) / (float)D + p.eps);
  if (!live) return;
  if (part == 0 && lane == 0) {
    if (p.mean) p.mean[row] = mean;
    if (p.rstd) p.rstd[row] = rstd;
  }
#pragma unroll
  for (int j = 0; j < NB; ++j) {
    const int col = c0 + j * kBlk;
    if (!FULL && col - 4 * lane >= D) break;  // (uniform over the warp)
    if (p.x8.q) {
      uint32_t w;
      const uint32_t byte = block8_quantize(v[j], w);
      uint8_t* qr = static_cast<uint8_t*>(p.x8.q) + (size_t)row * p.x8.ldq;
      if (FULL) *reinterpret_cast<uint32_t*>(qr + col) = w;
      else stq4(qr, col, D, w);
      if (lane == 0) p.x8.scale[(size_t)(part * NB + j) * p.x8.lds + row] = (uint8_t)byte;
    }
    float4 y = make_float4((v[j].x - mean) * rstd, (v[j].y - mean) * rstd, (v[j].z - mean) * rstd,
                           (v[j].w - mean) * rstd);
    if (p.g) {
      const float4 g = FULL ? *reinterpret_cast<const float4*>(p.g + col) : ld4<float>(p.g, col, D, false);
      y = make_float4(y.x * g.x, y.y * g.y, y.z * g.z, y.w * g.w);
    }
    if (p.b) {
      const float4 b = FULL ? *reinterpret_cast<const float4*>(p.b + col) : ld4<float>(p.b, col, D, false);
      y = make_float4(y.x + b.x, y.y + b.y, y.z + b.z, y.w + b.w);
    }
    if (!FULL) y = mask4(y, col, D);
    if (p.y8.q) {
      uint32_t w;
      const uint32_t byte = block8_quantize(y, w);
      uint8_t* qr = static_cast<uint8_t*>(p.y8.q) + (size_t)row * p.y8.ldq;
      if (FULL) *reinterpret_cast<uint32_t*>(qr + col) = w;
      else stq4(qr, col, D, w);
      if (lane == 0) p.y8.scale[(size_t)(part * NB + j) * p.y8.lds + row] = (uint8_t)byte;
    }
    if (p.y.p) {
      if (p.y.dtype == LAZYMAR_F32)
        st4<float>(static_cast<float*>(p.y.p) + (size_t)row * p.y.ld, col, FULL ? col + 4 : D, FULL || p.vec, y);
      else
        st4<bf16>(static_cast<bf16*>(p.y.p) + (size_t)row * p.y.ld, col, FULL ? col + 4 : D, FULL || p.vec, y);
    }
  }
}

template <int NB, int WPR>
cudaError_t ln_forward_run(const Ctx& c, const LnForward& p) {
  constexpr int GROUPS = WPR > 8 ? 1 : 8 / WPR;
  const dim3 grid((unsigned)((p.M + GROUPS - 1) / GROUPS)), block(WPR > 8 ? WPR * 32 : 256);
  const bool aligned = ((reinterpret_cast<uintptr_t>(p.g) | reinterpret_cast<uintptr_t>(p.b)) & 15u) == 0;
  if (p.vec && aligned && p.D == NB * WPR * kBlk)
    return launch_pdl(ln_forward_kernel<NB, WPR, true>, grid, block, 0, c.stream, p);
  return launch_pdl(ln_forward_kernel<NB, WPR, false>, grid, block, 0, c.stream, p);
}

// ---------------------------------------------------------------------------
// Column sums of per-CTA partial rows
// ---------------------------------------------------------------------------
// out[c] (+)= sum over the P rows of part [P, n], in row order within each of
// eight slices and slice order after that: the same result for the same sizes.
// Columns from n1 on belong to out2.
__global__ void __launch_bounds__(256) column_sums_kernel(const float* __restrict__ part, int P, int n, int n1,
                                                          float* __restrict__ out, float* __restrict__ out2,
                                                          bool accumulate) {
  __shared__ float red[8][32];
  const int lane = threadIdx.x & 31, slice = threadIdx.x >> 5, col = blockIdx.x * 32 + lane;
  pdl_wait();
  pdl_trigger();
  float s = 0.f;
  if (col < n) {
    const float* p = part + col;
#pragma unroll 8
    for (int r = slice; r < P; r += 8) s += p[(size_t)r * n];
  }
  red[slice][lane] = s;
  __syncthreads();
  if (slice == 0 && col < n) {
#pragma unroll
    for (int i = 1; i < 8; ++i) s += red[i][lane];
    float* o = col < n1 ? out + col : out2 + (col - n1);
    if (accumulate) s += *o;
    *o = s;
  }
}

cudaError_t column_sums(const Ctx& c, const float* part, int P, int n, int n1, float* out, float* out2,
                        bool accumulate) {
  return launch_pdl(column_sums_kernel, dim3((unsigned)((n + 31) / 32)), dim3(256), 0, c.stream, part, P, n, n1, out,
                    out2, accumulate);
}

// ---------------------------------------------------------------------------
// LayerNorm backward
// ---------------------------------------------------------------------------
// With xh = (x - mean) rstd and a = dy g:
//   dx = rstd (a - mean(a) - xh mean(a xh)) [+ dres],  dg = sum dy xh,  db = sum dy.
// A CTA works through rows of a stride and keeps its share of dg and db in
// registers (a lane owns its columns), so that the column sums cost one pass
// over 2 D floats a CTA instead of one over the data.
template <int NB, int WPR, bool FULL>
__global__ void __launch_bounds__(WPR > 8 ? WPR * 32 : 256) ln_backward_kernel(const LnBackward p) {
  constexpr int GROUPS = WPR > 8 ? 1 : 8 / WPR;
  extern __shared__ float cols[];  // [2][NB WPR 128]
  __shared__ float red[2][2][GROUPS][WPR];
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, grp = warp / WPR, part = warp % WPR;
  const int D = p.D, c0 = part * NB * kBlk + 4 * lane;
  pdl_wait();
  pdl_trigger();
  float4 dg[NB], db[NB];
#pragma unroll
  for (int j = 0; j < NB; ++j) dg[j] = db[j] = make_float4(0.f, 0.f, 0.f, 0.f);
  const int stride = (int)gridDim.x * GROUPS;
  int it = 0;
  // (every warp makes the same number of rounds: row_sum is a CTA-wide step)
  for (int base = (int)blockIdx.x * GROUPS; base < p.M; base += stride, it ^= 1) {
    const int row = base + grp;
    const bool live = row < p.M;
    float4 xh[NB], a[NB];
    if (live) {
      if (p.dy.dtype == LAZYMAR_F32) {
        const float* r = static_cast<const float*>(p.dy.p) + (size_t)row * p.dy.ld;
#pragma unroll
        for (int j = 0; j < NB; ++j) a[j] = ld4t<float, FULL>(r, c0 + j * kBlk, D, p.vec);
      } else {
        const bf16* r = static_cast<const bf16*>(p.dy.p) + (size_t)row * p.dy.ld;
#pragma unroll
        for (int j = 0; j < NB; ++j) a[j] = ld4t<bf16, FULL>(r, c0 + j * kBlk, D, p.vec);
      }
      const float mean = p.mean[row], rstd = p.rstd[row];
      if (!p.x.p) {
        const uint8_t* r = static_cast<const uint8_t*>(p.x8.q) + (size_t)row * p.x8.ldq;
        const int nb = (D + kBlk - 1) / kBlk - part * NB;  // blocks from this warp's first on
        const uint32_t sb = lane < NB && lane < nb ? p.x8.scale[(size_t)(part * NB + lane) * p.x8.lds + row] : 0u;
#pragma unroll
        for (int j = 0; j < NB; ++j) {
          const uint32_t w = FULL ? *reinterpret_cast<const uint32_t*>(r + c0 + j * kBlk) : ldq4(r, c0 + j * kBlk, D);
          xh[j] = e4m3x4_to_f4(w, block8_scale(__shfl_sync(0xffffffffu, sb, j)));
        }
      } else if (p.x.dtype == LAZYMAR_F32) {
        const float* r = static_cast<const float*>(p.x.p) + (size_t)row * p.x.ld;
#pragma unroll
        for (int j = 0; j < NB; ++j) xh[j] = ld4t<float, FULL>(r, c0 + j * kBlk, D, p.vec);
      } else {
        const bf16* r = static_cast<const bf16*>(p.x.p) + (size_t)row * p.x.ld;
#pragma unroll
        for (int j = 0; j < NB; ++j) xh[j] = ld4t<bf16, FULL>(r, c0 + j * kBlk, D, p.vec);
      }
      float s1 = 0.f, s2 = 0.f;
#pragma unroll
      for (int j = 0; j < NB; ++j) {
        const int col = c0 + j * kBlk;
        float4 h = make_float4((xh[j].x - mean) * rstd, (xh[j].y - mean) * rstd, (xh[j].z - mean) * rstd,
                               (xh[j].w - mean) * rstd);
        if (!FULL) h = mask4(h, col, D);
        xh[j] = h;
        const float4 y = a[j];
        dg[j].x = fmaf(y.x, h.x, dg[j].x); dg[j].y = fmaf(y.y, h.y, dg[j].y);
        dg[j].z = fmaf(y.z, h.z, dg[j].z); dg[j].w = fmaf(y.w, h.w, dg[j].w);
        db[j].x += y.x; db[j].y += y.y; db[j].z += y.z; db[j].w += y.w;
        if (p.g) {
          const float4 g = FULL ? *reinterpret_cast<const float4*>(p.g + col) : ld4<float>(p.g, col, D, false);
          a[j] = make_float4(y.x * g.x, y.y * g.y, y.z * g.z, y.w * g.w);
        }
        s1 += sum4(a[j]);
        s2 += (a[j].x * h.x + a[j].y * h.y) + (a[j].z * h.z + a[j].w * h.w);
      }
      s1 = warp_sum(s1);
      s2 = warp_sum(s2);
      if constexpr (WPR > 1) {
        if (lane == 0) {
          red[it][0][grp][part] = s1;
          red[it][1][grp][part] = s2;
        }
      } else {
        red[it][0][grp][0] = s1;  // (its own warp's: read back below)
        red[it][1][grp][0] = s2;
      }
    }
    if constexpr (WPR > 1) __syncthreads();
    else __syncwarp();
    if (live) {
      float s1 = 0.f, s2 = 0.f;
#pragma unroll
      for (int i = 0; i < WPR; ++i) {
        s1 += red[it][0][grp][i];
        s2 += red[it][1][grp][i];
      }
      s1 /= (float)D;
      s2 /= (float)D;
      const float rstd = p.rstd[row];
#pragma unroll
      for (int j = 0; j < NB; ++j) {
        const int col = c0 + j * kBlk;
        float4 o = make_float4(rstd * (a[j].x - s1 - xh[j].x * s2), rstd * (a[j].y - s1 - xh[j].y * s2),
                               rstd * (a[j].z - s1 - xh[j].z * s2), rstd * (a[j].w - s1 - xh[j].w * s2));
        if (p.dres.p) {
          const float4 r = ld4t<float, FULL>(static_cast<const float*>(p.dres.p) + (size_t)row * p.dres.ld, col, D,
                                             p.vec);
          o = make_float4(o.x + r.x, o.y + r.y, o.z + r.z, o.w + r.w);
        }
        if (p.dx.dtype == LAZYMAR_F32)
          st4<float>(static_cast<float*>(p.dx.p) + (size_t)row * p.dx.ld, col, FULL ? col + 4 : D, FULL || p.vec, o);
        else
          st4<bf16>(static_cast<bf16*>(p.dx.p) + (size_t)row * p.dx.ld, col, FULL ? col + 4 : D, FULL || p.vec, o);
      }
    }
  }
  if (!p.dg) return;
  // the CTA's rows' sums: its groups add in turn
  constexpr int W = NB * WPR * kBlk;
  for (int g = 0; g < GROUPS; ++g) {
    if (g == grp) {
#pragma unroll
      for (int j = 0; j < NB; ++j) {
        float4* s = reinterpret_cast<float4*>(cols + c0 + j * kBlk);
        float4* t = reinterpret_cast<float4*>(cols + W + c0 + j * kBlk);
        if (g == 0) {
          *s = dg[j];
          *t = db[j];
        } else {
          const float4 u = *s, w = *t;
          *s = make_float4(u.x + dg[j].x, u.y + dg[j].y, u.z + dg[j].z, u.w + dg[j].w);
          *t = make_float4(w.x + db[j].x, w.y + db[j].y, w.z + db[j].z, w.w + db[j].w);
        }
      }
    }
    __syncthreads();
  }
  float* o = p.ws + (size_t)blockIdx.x * 2 * D;
  for (int i = threadIdx.x; i < 2 * D; i += blockDim.x) o[i] = i < D ? cols[i] : cols[W + i - D];
}

// CTAs of a backward launch: two resident ones for every SM.
int ln_backward_ctas(int M, int groups) {
  const int need = (M + groups - 1) / groups, most = 2 * kSMs;
  return need < most ? need : most;
}

template <int NB, int WPR>
cudaError_t ln_backward_run(const Ctx& c, const LnBackward& p) {
  constexpr int GROUPS = WPR > 8 ? 1 : 8 / WPR;
  const int ctas = ln_backward_ctas(p.M, GROUPS);
  const dim3 grid((unsigned)ctas), block(WPR > 8 ? WPR * 32 : 256);
  constexpr size_t smem = (size_t)2 * NB * WPR * kBlk * sizeof(float);
  const bool full = p.vec && (reinterpret_cast<uintptr_t>(p.g) & 15u) == 0 && p.D == NB * WPR * kBlk;
  cudaError_t e;
  if (full) {
    if (smem > 48 * 1024)
      if ((e = cudaFuncSetAttribute(ln_backward_kernel<NB, WPR, true>, cudaFuncAttributeMaxDynamicSharedMemorySize,
                                    (int)smem)) != cudaSuccess)
        return e;
    e = launch_pdl(ln_backward_kernel<NB, WPR, true>, grid, block, smem, c.stream, p);
  } else {
    if (smem > 48 * 1024)
      if ((e = cudaFuncSetAttribute(ln_backward_kernel<NB, WPR, false>, cudaFuncAttributeMaxDynamicSharedMemorySize,
                                    (int)smem)) != cudaSuccess)
        return e;
    e = launch_pdl(ln_backward_kernel<NB, WPR, false>, grid, block, smem, c.stream, p);
  }
  if (e != cudaSuccess || !p.dg) return e;
  return column_sums(c, p.ws, ctas, 2 * p.D, p.D, p.dg, p.db, p.accumulate);
}

// ---------------------------------------------------------------------------
// The GELU gradient and the checkpoint
// ---------------------------------------------------------------------------
// GELU'(x) = Phi(x) + x phi(x) for the erf form, from a table: a checkpoint's
// values have three mantissa bits, so sign, exponent and those bits name them
// all. Below 2^-26 the gradient is 1/2 to 1.2e-8, from 16 on it is 0 or 1 in fp32,
// which leaves 241 entries a sign. A look-up takes half of the instructions of
// an evaluation and has the error of erfcf and expf (1e-7) instead of a
// polynomial's.
constexpr int kGradLo = (127 - 26) << 3, kGradHi = (127 + 4) << 3, kGradN = kGradHi - kGradLo + 1;

__device__ __forceinline__ void gelu_grad_table(float* tab) {
  for (int i = threadIdx.x; i < 2 * kGradN; i += blockDim.x) {
    const float a = __uint_as_float((uint32_t)(kGradLo + i % kGradN) << 20), x = i < kGradN ? a : -a;
    tab[i] = fmaf(x * 0.39894228040143268f, expf(-0.5f * x * x), 0.5f * erfcf(-0.70710678118654752f * x));
  }
}
__device__ __forceinline__ float gelu_grad_at(const float* tab, float x) {
  const uint32_t b = __float_as_uint(x);
  const int i = min(max((int)((b >> 20) & 0x7FFu), kGradLo), kGradHi) - kGradLo + (((int)b >> 31) & kGradN);
  return fmaf(x, 0.f, tab[i]);  // NaN stays NaN
}

// in [rows, cols] through an optional GELU' of the checkpoint u, to `out`
// and / or block8, with optional column sums. A warp owns a block of 128
// columns and a stride of rows, kRowsU at a time, so that the column sums stay
// in its registers; neighbouring warps take neighbouring blocks of the same
// rows.
constexpr int kRowsU = 4;

template <typename T, bool HAS_U>
__global__ void __launch_bounds__(256) rows8_kernel(const Rows8 p, int nblk, int groups) {
  const int lane = threadIdx.x & 31;
  const int task = (int)blockIdx.x * 8 + (threadIdx.x >> 5);
  const int grp = task / nblk, blk = task - grp * nblk, col = blk * kBlk + 4 * lane, cols = p.cols;
  __shared__ float grad[HAS_U ? 2 * kGradN : 1];
  if (HAS_U) {
    gelu_grad_table(grad);
    __syncthreads();
  }
  pdl_wait();
  pdl_trigger();
  if (grp >= groups) return;
  float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
  const T* in = static_cast<const T*>(p.in.p);
  for (long long r0 = (long long)grp * kRowsU; r0 < p.rows; r0 += (long long)groups * kRowsU) {
    float4 v[kRowsU];
    uint32_t uq[kRowsU], us[kRowsU];
#pragma unroll
    for (int i = 0; i < kRowsU; ++i) {
      const size_t r = (size_t)(r0 + i);
      const bool live = r0 + i < p.rows;
      v[i] = live ? ld4<T>(in + r * p.in.ld, col, cols, p.vec) : make_float4(0.f, 0.f, 0.f, 0.f);
      if (HAS_U) {
        uq[i] = live ? ldq4(static_cast<const uint8_t*>(p.u.q) + r * p.u.ldq, col, cols) : 0u;
        us[i] = live ? p.u.scale[(size_t)blk * p.u.lds + r] : 0u;
      }
    }
#pragma unroll
    for (int i = 0; i < kRowsU; ++i) {
      if (r0 + i >= p.rows) break;
      const size_t r = (size_t)(r0 + i);
      if (HAS_U) {
        const float4 u = e4m3x4_to_f4(uq[i], block8_scale(us[i]));
        v[i].x *= gelu_grad_at(grad, u.x);
        v[i].y *= gelu_grad_at(grad, u.y);
        v[i].z *= gelu_grad_at(grad, u.z);
        v[i].w *= gelu_grad_at(grad, u.w);
      }
      if (p.db) {
        acc.x += v[i].x; acc.y += v[i].y; acc.z += v[i].z; acc.w += v[i].w;
      }
      if (p.out.p) {
        if (p.out.dtype == LAZYMAR_F32)
          st4<float>(static_cast<float*>(p.out.p) + r * p.out.ld, col, cols, p.vec, v[i]);
        else
          st4<bf16>(static_cast<bf16*>(p.out.p) + r * p.out.ld, col, cols, p.vec, v[i]);
      }
      if (p.out8.q) {
        uint32_t w;
        const uint32_t byte = block8_quantize(v[i], w);
        stq4(static_cast<uint8_t*>(p.out8.q) + r * p.out8.ldq, col, cols, w);
        if (lane == 0) p.out8.scale[(size_t)blk * p.out8.lds + r] = (uint8_t)byte;
      }
    }
  }
  if (p.db) st4<float>(p.ws + (size_t)grp * cols, col, cols, false, acc);
}

// Row groups of a launch: about 48 warps for every SM in all.
int rows8_groups(int rows, int nblk) {
  const int want = (kSMs * 48 + nblk - 1) / nblk, most = (rows + kRowsU - 1) / kRowsU;
  return want < most ? want : most;
}

// ---------------------------------------------------------------------------
// Back to fp32 / bf16, and weights
// ---------------------------------------------------------------------------
template <typename T>
__global__ void __launch_bounds__(256) unpack8_kernel(const lazymar_block8 q, T* __restrict__ x, int ld, int rows,
                                                      int cols, int nblk, bool vec) {
  const int lane = threadIdx.x & 31;
  pdl_wait();
  pdl_trigger();
  const long long tasks = (long long)rows * nblk, step = (long long)gridDim.x * 8 * 4;
  for (long long t0 = ((long long)blockIdx.x * 8 + (threadIdx.x >> 5)) * 4; t0 < tasks; t0 += step) {
    uint32_t w[4], s[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const long long t = t0 + i < tasks ? t0 + i : tasks - 1;
      const size_t r = (size_t)(t / nblk);
      const int blk = (int)(t - (long long)r * nblk);
      w[i] = ldq4(static_cast<const uint8_t*>(q.q) + r * q.ldq, blk * kBlk + 4 * lane, cols);
      s[i] = q.scale[(size_t)blk * q.lds + r];
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const long long t = t0 + i;
      if (t >= tasks) break;
      const size_t r = (size_t)(t / nblk);
      const int blk = (int)(t - (long long)r * nblk);
      st4<T>(x + r * ld, blk * kBlk + 4 * lane, cols, vec, e4m3x4_to_f4(w[i], block8_scale(s[i])));
    }
  }
}

// One 128 x 128 block of a weight matrix to E4M3 with one scale, and the same
// bytes transposed. Each warp holds 16 rows; the transpose goes through shared
// memory, 132 bytes a row.
__global__ void __launch_bounds__(256) pack_weight8_kernel(const Mat w, const lazymar_block8 q,
                                                           const lazymar_block8 qt, int N, int K, bool vec) {
  __shared__ uint32_t tile[128][33];
  __shared__ uint32_t mx[8];
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int n0 = (int)blockIdx.y * kBlk, k0 = (int)blockIdx.x * kBlk, col = k0 + 4 * lane;
  pdl_wait();
  pdl_trigger();
  float4 v[16];
  float m = 0.f;
#pragma unroll
  for (int i = 0; i < 16; ++i) {
    const int n = n0 + warp * 16 + i;
    v[i] = make_float4(0.f, 0.f, 0.f, 0.f);
    if (n < N) {
      if (w.dtype == LAZYMAR_F32)
        v[i] = ld4<float>(static_cast<const float*>(w.p) + (size_t)n * w.ld, col, K, vec);
      else
        v[i] = ld4<bf16>(static_cast<const bf16*>(w.p) + (size_t)n * w.ld, col, K, vec);
    }
    const float4 z = f4_nonfinite_to(v[i], 0.f);
    m = fmaxf(m, fmax3(fmaxf(fabsf(z.x), fabsf(z.y)), fabsf(z.z), fabsf(z.w)));
    v[i] = f4_nonfinite_to(v[i], __uint_as_float(0x7FC00000u));
  }
  const uint32_t wm = __reduce_max_sync(0xffffffffu, __float_as_uint(m));
  if (lane == 0) mx[warp] = wm;
  __syncthreads();
  uint32_t amax = mx[0];
#pragma unroll
  for (int i = 1; i < 8; ++i) amax = max(amax, mx[i]);
  const uint32_t byte = block8_exp(amax);
  const float s = block8_inv(byte);
  if (threadIdx.x == 0) {
    if (q.q) q.scale[(size_t)blockIdx.x * q.lds + blockIdx.y] = (uint8_t)byte;
    if (qt.q) qt.scale[(size_t)blockIdx.y * qt.lds + blockIdx.x] = (uint8_t)byte;
  }
#pragma unroll
  for (int i = 0; i < 16; ++i) {
    const int n = n0 + warp * 16 + i;
    const uint32_t b = e4m3x4(v[i].x * s, v[i].y * s, v[i].z * s, v[i].w * s);
    if (q.q && n < N) stq4(static_cast<uint8_t*>(q.q) + (size_t)n * q.ldq, col, K, b);
    tile[warp * 16 + i][lane] = b;
  }
  if (!qt.q) return;
  __syncthreads();
  const uint8_t* tb = reinterpret_cast<const uint8_t*>(&tile[0][0]);
#pragma unroll 4
  for (int i = 0; i < 16; ++i) {
    const int k = warp * 16 + i;
    uint32_t b = 0;
#pragma unroll
    for (int j = 0; j < 4; ++j) b |= (uint32_t)tb[(4 * lane + j) * 132 + k] << (8 * j);
    if (k0 + k < K) stq4(static_cast<uint8_t*>(qt.q) + (size_t)(k0 + k) * qt.ldq, n0 + 4 * lane, N, b);
  }
}

}  // namespace

cudaError_t launch_ln_forward(const Ctx& c, const LnForward& p) {
  if (p.M == 0) return cudaSuccess;
  const int nb = (p.D + kBlk - 1) / kBlk;
  if (nb <= 1) return ln_forward_run<1, 1>(c, p);
  if (nb <= 2) return ln_forward_run<2, 1>(c, p);
  if (nb <= 4) return ln_forward_run<4, 1>(c, p);
  if (nb <= 6) return ln_forward_run<6, 1>(c, p);
  if (nb <= 8) return ln_forward_run<8, 1>(c, p);
  if (nb <= 10) return ln_forward_run<10, 1>(c, p);
  if (nb <= 16) return ln_forward_run<8, 2>(c, p);
  if (nb <= 20) return ln_forward_run<10, 2>(c, p);
  if (nb <= 32) return ln_forward_run<8, 4>(c, p);
  if (nb <= 40) return ln_forward_run<10, 4>(c, p);
  return ln_forward_run<8, 8>(c, p);
}

size_t ln_backward_workspace(int M, int D) {
  return M > 0 && D > 0 ? (size_t)ln_backward_ctas(M, 1) * 2 * D * sizeof(float) : 0;
}

cudaError_t launch_ln_backward(const Ctx& c, const LnBackward& p) {
  if (p.M == 0) {
    if (!p.dg || p.accumulate) return cudaSuccess;
    return column_sums(c, p.ws, 0, 2 * p.D, p.D, p.dg, p.db, false);
  }
  const int nb = (p.D + kBlk - 1) / kBlk;
  if (nb <= 1) return ln_backward_run<1, 1>(c, p);
  if (nb <= 2) return ln_backward_run<2, 1>(c, p);
  if (nb <= 4) return ln_backward_run<4, 1>(c, p);
  if (nb <= 6) return ln_backward_run<3, 2>(c, p);
  if (nb <= 8) return ln_backward_run<4, 2>(c, p);
  if (nb <= 10) return ln_backward_run<5, 2>(c, p);
  if (nb <= 16) return ln_backward_run<4, 4>(c, p);
  if (nb <= 20) return ln_backward_run<5, 4>(c, p);
  if (nb <= 32) return ln_backward_run<4, 8>(c, p);
  if (nb <= 40) return ln_backward_run<5, 8>(c, p);
  return ln_backward_run<4, 16>(c, p);
}

size_t rows8_workspace(int rows, int cols) {
  if (rows < 1 || cols < 1) return 0;
  return (size_t)rows8_groups(rows, (cols + kBlk - 1) / kBlk) * cols * sizeof(float);
}

cudaError_t launch_rows8(const Ctx& c, const Rows8& p) {
  if (p.rows == 0) {
    if (!p.db || p.accumulate) return cudaSuccess;
    return column_sums(c, p.ws, 0, p.cols, p.cols, p.db, nullptr, false);
  }
  const int nblk = (p.cols + kBlk - 1) / kBlk, groups = rows8_groups(p.rows, nblk);
  const dim3 grid((unsigned)(((long long)nblk * groups + 7) / 8)), block(256);
  cudaError_t e;
  if (p.in.dtype == LAZYMAR_F32)
    e = p.u.q ? launch_pdl(rows8_kernel<float, true>, grid, block, 0, c.stream, p, nblk, groups)
              : launch_pdl(rows8_kernel<float, false>, grid, block, 0, c.stream, p, nblk, groups);
  else
    e = p.u.q ? launch_pdl(rows8_kernel<bf16, true>, grid, block, 0, c.stream, p, nblk, groups)
              : launch_pdl(rows8_kernel<bf16, false>, grid, block, 0, c.stream, p, nblk, groups);
  if (e != cudaSuccess || !p.db) return e;
  return column_sums(c, p.ws, groups, p.cols, p.cols, p.db, nullptr, p.accumulate);
}

cudaError_t launch_unpack8(const Ctx& c, const lazymar_block8& q, const MatOut& x, int rows, int cols) {
  if (rows == 0) return cudaSuccess;
  const int nblk = (cols + kBlk - 1) / kBlk;
  const bool vec = x.ld % 4 == 0 && reinterpret_cast<uintptr_t>(x.p) % (x.dtype == LAZYMAR_F32 ? 16 : 8) == 0;
  long long ctas = ((long long)rows * nblk + 31) / 32;
  if (ctas > kSMs * 16) ctas = kSMs * 16;
  if (x.dtype == LAZYMAR_F32)
    return launch_pdl(unpack8_kernel<float>, dim3((unsigned)ctas), dim3(256), 0, c.stream, q, static_cast<float*>(x.p),
                      x.ld, rows, cols, nblk, vec);
  return launch_pdl(unpack8_kernel<bf16>, dim3((unsigned)ctas), dim3(256), 0, c.stream, q, static_cast<bf16*>(x.p),
                    x.ld, rows, cols, nblk, vec);
}

cudaError_t launch_pack_weight8(const Ctx& c, const Mat& w, const lazymar_block8& q, const lazymar_block8& qt, int N,
                                int K) {
  const bool vec = w.ld % 4 == 0 && reinterpret_cast<uintptr_t>(w.p) % (w.dtype == LAZYMAR_F32 ? 16 : 8) == 0;
  const dim3 grid((unsigned)((K + kBlk - 1) / kBlk), (unsigned)((N + kBlk - 1) / kBlk));
  return launch_pdl(pack_weight8_kernel, grid, dim3(256), 0, c.stream, w, q, qt, N, K, vec);
}

}  // namespace lm
