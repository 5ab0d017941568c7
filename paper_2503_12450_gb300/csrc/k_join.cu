// The residual join and its gradient: the norm behind a branch, its gate, the
// residual addition and the modulated norm in front of the next branch, each tensor
// read and written once. Bound by HBM bandwidth (13 bytes an element forward with an fp32
// stream, a bf16 branch and three 8-bit outputs, 17 backward), and next to it by
// instruction issue.
#include "join.cuh"
#include "rows.cuh"

namespace lm {

namespace {

// ---------------------------------------------------------------------------
// Eight columns of rows of any type, first as they are loaded, then widened: so that
// the loads of all tensors are under way before the first is waited for.
// ---------------------------------------------------------------------------
struct Raw {
  uint32_t w[8], s;
};
__device__ __forceinline__ void ld8b(const void* p, uint32_t (&w)[8]) {
  asm volatile("ld.global.v8.b32 {%0, %1, %2, %3, %4, %5, %6, %7}, [%8];"
               : "=r"(w[0]), "=r"(w[1]), "=r"(w[2]), "=r"(w[3]), "=r"(w[4]), "=r"(w[5]), "=r"(w[6]), "=r"(w[7])
               : "l"(p));
}
template <bool FULL>
__device__ __forceinline__ void fetch8(const Rows& m, size_t row, int cc, int D, Raw& r) {
  const int col = cc + 8 * (int)(threadIdx.x & 31);
  if (m.dtype == LAZYMAR_E4M3) {
    const uint2 q = ldq8(static_cast<const uint8_t*>(m.p) + row * m.ld, col, D);
    r.w[0] = q.x;
    r.w[1] = q.y;
    r.s = m.scale[(size_t)(min(col, D - 1) / kBlk) * m.lds + row];
  } else if (!FULL && !m.vec) {
    ld8s(Mat{m.p, m.ld, m.dtype, false}, row, cc, D, r.w);
  } else if (m.dtype == LAZYMAR_F32) {
    const float* p = static_cast<const float*>(m.p) + row * m.ld + col;
    if (FULL || col + 8 <= D) {
      ld8b(p, r.w);
    } else {
#pragma unroll
      for (int i = 0; i < 8; ++i) r.w[i] = col + i < D ? __float_as_uint(p[i]) : 0u;
    }
  } else {
    const bf16* p = static_cast<const bf16*>(m.p) + row * m.ld + col;
    if (FULL || col + 8 <= D) {
      const uint4 u = *reinterpret_cast<const uint4*>(p);
      r.w[0] = u.x;
      r.w[1] = u.y;
      r.w[2] = u.z;
      r.w[3] = u.w;
    } else {
      const uint16_t* h = reinterpret_cast<const uint16_t*>(p);
#pragma unroll
      for (int i = 0; i < 8; i += 2)
        r.w[i / 2] = (col + i < D ? h[i] : 0u) | (col + i + 1 < D ? (uint32_t)h[i + 1] << 16 : 0u);
    }
  }
}
template <bool FULL>
__device__ __forceinline__ void widen8(const Rows& m, const Raw& r, float* sm, float (&v)[8]) {
  if (m.dtype == LAZYMAR_E4M3) {
    block8_values(make_uint2(r.w[0], r.w[1]), block8_scale(r.s), v);
  } else if (!FULL && !m.vec) {
    turn8(sm, r.w, m.dtype == LAZYMAR_F32 ? 0 : 16, v);
  } else if (m.dtype == LAZYMAR_F32) {
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = __uint_as_float(r.w[i]);
  } else {
    bf16x8(make_uint4(r.w[0], r.w[1], r.w[2], r.w[3]), v);
  }
}
// y = v * a (+ b)
__device__ __forceinline__ void fma8(float (&v)[8], const float (&a)[8], const float (&b)[8]) {
#pragma unroll
  for (int i = 0; i < 8; i += 2)
    f32x2_unpack(f32x2_fma(f32x2_pack(v[i], v[i + 1]), f32x2_pack(a[i], a[i + 1]), f32x2_pack(b[i], b[i + 1])), v[i],
                 v[i + 1]);
}

// Waits for the WPR warps of a row.
template <int WPR>
__device__ __forceinline__ void row_barrier(int grp) {
  asm volatile("bar.sync %0, %1;" ::"r"(grp + 1), "n"(WPR * 32) : "memory");
}

// Mean and 1 / deviation of a row whose columns are spread over WPR warps, NC chunks a
// warp, columns that do not exist zero. Each warp takes the squares about its own mean,
// and the warps' sums are joined about the row's: one exchange between the warps, and
// no cancellation. RMS: the mean counts as 0.
template <int NC, int WPR, bool FULL>
__device__ __forceinline__ void moments(const float (&v)[NC][8], bool layer, int D, int c0, float eps, float2* red, int grp,
                                        int part, float& mean, float& rstd) {
  const int lane = threadIdx.x & 31;
  const auto columns = [&](int i) { return (float)min(max(D - i * NC * kChunk, 0), NC * kChunk); };
  const float n = columns(part);
  float m = 0.f, q = 0.f;
  if (layer) {
    float s = 0.f;
#pragma unroll
    for (int c = 0; c < NC; ++c) s += sum8(v[c]);
    m = n > 0.f ? warp_sum(s) / n : 0.f;
  }
#pragma unroll
  for (int c = 0; c < NC; ++c) {
    float d[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) d[i] = v[c][i];
    sub8(d, m);
    mask8<FULL>(d, c0 + c * kChunk + 8 * lane, D);
    q += squares8(d);
  }
  q = warp_sum(q);
  mean = m;
  if constexpr (WPR > 1) {
    if (lane == 0) red[part] = make_float2(m, q);
    row_barrier<WPR>(grp);
    float s = 0.f;
#pragma unroll
    for (int i = 0; i < WPR; ++i) s += red[i].x * columns(i);
    mean = s / (float)D;
    q = 0.f;
#pragma unroll
    for (int i = 0; i < WPR; ++i) {
      const float2 r = red[i];
      const float off = r.x - mean;
      q += r.y + columns(i) * off * off;
    }
  }
  rstd = rsqrtf(q / (float)D + eps);
}

template <int WPR>
constexpr int kWarps = WPR == 5 ? 10 : WPR > 8 ? 16 : 8;

// ---------------------------------------------------------------------------
// Forward
// ---------------------------------------------------------------------------
// WPR warps a row, NC chunks of 256 columns a warp, the row in registers throughout.
// FULL: D = 256 NC WPR and every row on a boundary, so that no column needs a check.
template <int NC, int WPR, bool FULL>
__global__ void __launch_bounds__(kWarps<WPR> * 32, NC == 1 ? 3 : 2) join_kernel(const Join p) {
  constexpr int GROUPS = kWarps<WPR> / WPR;
  __shared__ float2 red[2][GROUPS][WPR];
  __shared__ float stage[FULL ? 1 : kWarps<WPR>][kStage];
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, grp = warp / WPR, part = warp % WPR;
  float* sm = stage[FULL ? 0 : warp];
  const int D = p.D, row = blockIdx.x * GROUPS + grp, c0 = part * NC * kChunk;
  pdl_wait();
  pdl_trigger();
  if (row >= p.M) return;
  const int r = p.group > 0 ? row / p.group : 0;
  Raw rx[NC], ry[NC], rg[NC];
#pragma unroll
  for (int c = 0; c < NC; ++c) {
    fetch8<FULL>(p.x, row, c0 + c * kChunk, D, rx[c]);
    if (p.y.p) fetch8<FULL>(p.y, row, c0 + c * kChunk, D, ry[c]);
    if (p.gate.p) fetch8<FULL>(p.gate, r, c0 + c * kChunk, D, rg[c]);
  }
  float v[NC][8];
  if (p.y.p) {
#pragma unroll
    for (int c = 0; c < NC; ++c) {
      widen8<FULL>(p.y, ry[c], sm, v[c]);
      if (p.y8.q && (FULL || c0 + c * kChunk < D)) put8<FULL>(p.y8, row, c0 + c * kChunk, D, v[c]);
    }
    float mean = 0.f, rstd = 1.f;
    if (p.post != LAZYMAR_NORM_NONE) {
      moments<NC, WPR, FULL>(v, p.post == LAZYMAR_NORM_LAYER, D, c0, p.eps, red[0][grp], grp, part, mean, rstd);
      if (part == 0 && lane == 0) {
        if (p.y_mean) p.y_mean[row] = mean;
        if (p.y_rstd) p.y_rstd[row] = rstd;
      }
    }
#pragma unroll
    for (int c = 0; c < NC; ++c) {
      const int col = c0 + c * kChunk + 8 * lane;
      float t[8];
      if (p.post != LAZYMAR_NORM_NONE) {
        sub8(v[c], mean);
        scale8(v[c], rstd, v[c]);
      }
      if (p.post_g) {
        ld_param<FULL>(p.post_g, p.params_vec, col, D, t);
        mul8(v[c], t);
      }
      if (p.post_b) {
        ld_param<FULL>(p.post_b, p.params_vec, col, D, t);
        add8(v[c], t);
      }
      if (p.gate.p) {
        widen8<FULL>(p.gate, rg[c], sm, t);
        mul8(v[c], t);
      }
      widen8<FULL>(p.x, rx[c], sm, t);
      const float res[8] = {p.res, p.res, p.res, p.res, p.res, p.res, p.res, p.res};
      fma8(t, res, v[c]);
#pragma unroll
      for (int i = 0; i < 8; ++i) v[c][i] = t[i];
      mask8<FULL>(v[c], col, D);
    }
  } else {
#pragma unroll
    for (int c = 0; c < NC; ++c) {
      widen8<FULL>(p.x, rx[c], sm, v[c]);
      scale8(v[c], p.res, v[c]);
    }
  }
  Raw rs[NC], rt[NC];
#pragma unroll
  for (int c = 0; c < NC; ++c) {
    if (p.scale.p) fetch8<FULL>(p.scale, r, c0 + c * kChunk, D, rs[c]);
    if (p.shift.p) fetch8<FULL>(p.shift, r, c0 + c * kChunk, D, rt[c]);
  }
#pragma unroll
  for (int c = 0; c < NC; ++c) {
    const int cc = c0 + c * kChunk;
    if (!FULL && cc >= D) break;  // (uniform over the warp)
    if (p.z.p) st_mat<FULL>(p.z, row, cc, D, sm, v[c]);
    if (p.z8.q) put8<FULL>(p.z8, row, cc, D, v[c]);
  }
  if (p.pre == LAZYMAR_NORM_NONE) return;
  float mean, rstd;
  moments<NC, WPR, FULL>(v, p.pre == LAZYMAR_NORM_LAYER, D, c0, p.eps, red[1][grp], grp, part, mean, rstd);
  if (part == 0 && lane == 0) {
    if (p.z_mean) p.z_mean[row] = mean;
    if (p.z_rstd) p.z_rstd[row] = rstd;
  }
  if (!p.h.p && !p.h8.q) return;
#pragma unroll
  for (int c = 0; c < NC; ++c) {
    const int cc = c0 + c * kChunk, col = cc + 8 * lane;
    if (!FULL && cc >= D) break;
    float t[8];
    sub8(v[c], mean);
    scale8(v[c], rstd, v[c]);
    if (p.pre_g) {
      ld_param<FULL>(p.pre_g, p.params_vec, col, D, t);
      mul8(v[c], t);
    }
    if (p.pre_b) {
      ld_param<FULL>(p.pre_b, p.params_vec, col, D, t);
      add8(v[c], t);
    }
    if (p.scale.p) {
      widen8<FULL>(p.scale, rs[c], sm, t);
#pragma unroll
      for (int i = 0; i < 8; ++i) t[i] += 1.f;
      mul8(v[c], t);
    }
    if (p.shift.p) {
      widen8<FULL>(p.shift, rt[c], sm, t);
      add8(v[c], t);
    }
    mask8<FULL>(v[c], col, D);
    if (p.h.p) st_mat<FULL>(p.h, row, cc, D, sm, v[c]);
    if (p.h8.q) put8<FULL>(p.h8, row, cc, D, v[c]);
  }
}

bool on_eight(const Rows& r) { return !r.p || r.vec; }
bool on_eight(const MatOut& r) { return !r.p || r.vec; }

template <int NC, int WPR>
cudaError_t join_run(const Ctx& c, const Join& p) {
  constexpr int GROUPS = kWarps<WPR> / WPR;
  const dim3 grid((unsigned)((p.M + GROUPS - 1) / GROUPS)), block(kWarps<WPR> * 32);
  if (p.D == NC * WPR * kChunk && on_eight(p.x) && on_eight(p.y) && on_eight(p.gate) && on_eight(p.scale) &&
      on_eight(p.shift) && on_eight(p.z) && on_eight(p.h) && p.params_vec)
    return launch_pdl(join_kernel<NC, WPR, true>, grid, block, 0, c.stream, p);
  return launch_pdl(join_kernel<NC, WPR, false>, grid, block, 0, c.stream, p);
}

// ---------------------------------------------------------------------------
// Gradient
// ---------------------------------------------------------------------------
// A row is worked on by WPR warps (a team), NC chunks of 256 columns a warp. The teams of
// the launch divide the rows into consecutive ranges, so that a group's rows (those with one
// row of modulation) meet in one team or a few neighbouring ones. A lane keeps four sums
// of each of its columns while the group lasts,
//   A = sum dh, B = sum dh n, P = sum Z, Q = sum Z u,
// from which all gradients of modulation and parameters follow. A group that lies in
// one team's range is finished there; the others leave their sums in the workspace, two
// places a team (the group that its range begins in, and the one that it ends in).
// ROWWISE (every row has its own modulation): the modulation's gradients are written with
// the row, and the four sums, weighted, are those of the parameters.
enum { SUM_A = 0, SUM_B = 1, SUM_P = 2, SUM_Q = 3 };

__host__ __device__ __forceinline__ long long team_start(int M, int teams, int t) { return (long long)M * t / teams; }
__host__ __device__ __forceinline__ int team_of(int M, int teams, long long row) {
  return (int)(((row + 1) * teams - 1) / M);
}

template <int NC, int WPR, bool FULL, bool ROWWISE>
__global__ void __launch_bounds__(kWarps<WPR> * 32, NC == 1 && kWarps<WPR> <= 10 ? 2 : 1)
    join_grad_kernel(const JoinGrad p, int teams, bool params) {
  constexpr int GROUPS = kWarps<WPR> / WPR, W = NC * WPR * kChunk;
  extern __shared__ float weighted[];  // [GROUPS][4][W] (params and not ROWWISE)
  __shared__ float red[2][2][GROUPS][WPR][2];
  __shared__ float stage[FULL ? 1 : kWarps<WPR>][kStage];
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, grp = warp / WPR, part = warp % WPR;
  float* sm = stage[FULL ? 0 : warp];
  const int D = p.D, c0 = part * NC * kChunk, team = (int)blockIdx.x * GROUPS + grp;
  pdl_wait();
  pdl_trigger();
  if (team >= teams) return;
  const long long first = team_start(p.M, teams, team), end = team_start(p.M, teams, team + 1);
  const bool pre = p.pre != LAZYMAR_NORM_NONE, post = p.post != LAZYMAR_NORM_NONE;
  const bool pre_layer = p.pre == LAZYMAR_NORM_LAYER, post_layer = p.post == LAZYMAR_NORM_LAYER;
  float* mine = weighted + (size_t)grp * 4 * W + c0 + 8 * lane;  // this lane's columns of its first chunk
  if (!ROWWISE && params) {
#pragma unroll
    for (int k = 0; k < 4; ++k)
#pragma unroll
      for (int c = 0; c < NC; ++c)
#pragma unroll
        for (int i = 0; i < 8; ++i) mine[k * W + c * kChunk + i] = 0.f;
  }

  Raw rdh[NC], rz[NC], rdz[NC], ry[NC], rg[NC], rs[NC];
  float next_ym = 0.f, next_yr = 1.f, next_zm = 0.f, next_zr = 1.f;
  auto modulation = [&](size_t r) {
#pragma unroll
    for (int c = 0; c < NC; ++c) {
      if (p.gate.p) fetch8<FULL>(p.gate, r, c0 + c * kChunk, D, rg[c]);
      if (p.scale.p) fetch8<FULL>(p.scale, r, c0 + c * kChunk, D, rs[c]);
    }
  };
  auto fetch = [&](long long row) {
    if (row >= end) return;
#pragma unroll
    for (int c = 0; c < NC; ++c) {
      const int cc = c0 + c * kChunk;
      if (p.dh.p) fetch8<FULL>(p.dh, row, cc, D, rdh[c]);
      if (pre) fetch8<FULL>(p.z, row, cc, D, rz[c]);
      if (p.dz.p) fetch8<FULL>(p.dz, row, cc, D, rdz[c]);
      if (p.y.p) fetch8<FULL>(p.y, row, cc, D, ry[c]);
    }
    if (pre) {
      if (pre_layer) next_zm = p.z_mean[row];
      next_zr = p.z_rstd[row];
    }
    if (post) {
      if (post_layer) next_ym = p.y_mean[row];
      next_yr = p.y_rstd[row];
    }
    if (ROWWISE) modulation((size_t)row);
  };

  float sums[4][NC][8], gate[NC][8], scale[NC][8];  // scale: 1 + scale
#pragma unroll
  for (int c = 0; c < NC; ++c)
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      sums[0][c][i] = sums[1][c][i] = sums[2][c][i] = sums[3][c][i] = 0.f;
      gate[c][i] = scale[c][i] = 1.f;
    }
  auto widen_modulation = [&] {
#pragma unroll
    for (int c = 0; c < NC; ++c) {
      if (p.gate.p) widen8<FULL>(p.gate, rg[c], sm, gate[c]);
      if (p.scale.p) {
        widen8<FULL>(p.scale, rs[c], sm, scale[c]);
#pragma unroll
        for (int i = 0; i < 8; ++i) scale[c][i] += 1.f;
      }
    }
  };
  // out (+)= v for a row of a modulation's gradient
  auto put = [&](const MatOut& o, size_t r, int c, float (&v)[8]) {
    const int cc = c0 + c * kChunk;
    if (!o.p || (!FULL && cc >= D)) return;
    if (p.accumulate) {
      const int col = cc + 8 * lane;
#pragma unroll
      for (int i = 0; i < 8; ++i)
        if (col + i < D)
          v[i] += o.dtype == LAZYMAR_F32 ? static_cast<const float*>(o.p)[r * o.ld + col + i]
                                         : to_f(static_cast<const bf16*>(o.p)[r * o.ld + col + i]);
    }
    st_mat<FULL>(o, r, cc, D, sm, v);
  };

  // The end of a group, or of its part in this range: rows start .. stop.
  auto flush = [&](long long start, long long stop) {
    const long long q = p.group > 0 ? start / p.group : 0;
    const long long g0 = p.group > 0 ? q * p.group : 0;
    const long long g1 = p.group > 0 ? min(g0 + p.group, (long long)p.M) : p.M;
    const bool whole = start == g0 && stop == g1;
    float* slot = p.ws + ((size_t)team * 2 + (start > first)) * 4 * D;
#pragma unroll
    for (int c = 0; c < NC; ++c) {
      const int col = c0 + c * kChunk + 8 * lane;
      if (params) {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          float* w = mine + c * kChunk + i;
          w[SUM_A * W] += scale[c][i] * sums[SUM_A][c][i];
          w[SUM_B * W] += scale[c][i] * sums[SUM_B][c][i];
          w[SUM_P * W] += gate[c][i] * sums[SUM_P][c][i];
          w[SUM_Q * W] += gate[c][i] * sums[SUM_Q][c][i];
        }
      }
      if (whole) {
        float v[8], t[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = sums[SUM_A][c][i];
        put(p.dshift, q, c, v);
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = sums[SUM_B][c][i];
        if (p.pre_g) {
          ld_param<FULL>(p.pre_g, p.params_vec, col, D, t);
          mul8(v, t);
        }
        if (p.pre_b) {
          ld_param<FULL>(p.pre_b, p.params_vec, col, D, t);
          fma8(t, sums[SUM_A][c], v);
          put(p.dscale, q, c, t);
        } else {
          put(p.dscale, q, c, v);
        }
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = sums[SUM_Q][c][i];
        if (p.post_g) {
          ld_param<FULL>(p.post_g, p.params_vec, col, D, t);
          mul8(v, t);
        }
        if (p.post_b) {
          ld_param<FULL>(p.post_b, p.params_vec, col, D, t);
          fma8(t, sums[SUM_P][c], v);
          put(p.dgate, q, c, t);
        } else {
          put(p.dgate, q, c, v);
        }
      } else if (p.dshift.p || p.dscale.p || p.dgate.p) {
#pragma unroll
        for (int k = 0; k < 4; ++k)
#pragma unroll
          for (int i = 0; i < 8; ++i)
            if (FULL || col + i < D) slot[(size_t)k * D + col + i] = sums[k][c][i];
      }
#pragma unroll
      for (int k = 0; k < 4; ++k)
#pragma unroll
        for (int i = 0; i < 8; ++i) sums[k][c][i] = 0.f;
    }
  };

  int it = 0;
  fetch(first);
  long long start = first, stop = first;  // of the group's part
  for (long long row = first; row < end; ++row, it ^= 1) {
    if (!ROWWISE && row == stop) {
      if (row > first) flush(start, stop);
      start = row;
      stop = p.group > 0 ? min(end, (row / p.group + 1) * p.group) : end;
      modulation(p.group > 0 ? (size_t)(row / p.group) : 0);
      widen_modulation();
    }
    float dh[NC][8], n[NC][8], Z[NC][8], u[NC][8];
    const float ym = next_ym, yr = next_yr, zm = next_zm, zr = next_zr;
#pragma unroll
    for (int c = 0; c < NC; ++c) {
      if (p.dh.p) widen8<FULL>(p.dh, rdh[c], sm, dh[c]);
      if (pre) widen8<FULL>(p.z, rz[c], sm, n[c]);
      if (p.dz.p) widen8<FULL>(p.dz, rdz[c], sm, Z[c]);
      else
#pragma unroll
        for (int i = 0; i < 8; ++i) Z[c][i] = 0.f;
      if (p.y.p) widen8<FULL>(p.y, ry[c], sm, u[c]);
      else
#pragma unroll
        for (int i = 0; i < 8; ++i) u[c][i] = 0.f;
    }
    if (ROWWISE) widen_modulation();
    fetch(row + 1);
    if (pre) {
      float d[NC][8], s1 = 0.f, s2 = 0.f;
#pragma unroll
      for (int c = 0; c < NC; ++c) {
        const int cc = c0 + c * kChunk, col = cc + 8 * lane;
        float t[8];
        sub8(n[c], zm);
        scale8(n[c], zr, n[c]);
        mask8<FULL>(n[c], col, D);
#pragma unroll
        for (int i = 0; i < 8; ++i) d[c][i] = dh[c][i] * scale[c][i];
        if (ROWWISE) {
#pragma unroll
          for (int i = 0; i < 8; ++i) {
            sums[SUM_A][c][i] += d[c][i];
            sums[SUM_B][c][i] = fmaf(d[c][i], n[c][i], sums[SUM_B][c][i]);
          }
          if (p.dscale.p) {
            float v[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) v[i] = n[c][i];
            if (p.pre_g) {
              ld_param<FULL>(p.pre_g, p.params_vec, col, D, t);
              mul8(v, t);
            }
            if (p.pre_b) {
              ld_param<FULL>(p.pre_b, p.params_vec, col, D, t);
              add8(v, t);
            }
            mul8(v, dh[c]);
            put(p.dscale, row, c, v);
          }
          put(p.dshift, row, c, dh[c]);
        } else {
#pragma unroll
          for (int i = 0; i < 8; ++i) {
            sums[SUM_A][c][i] += dh[c][i];
            sums[SUM_B][c][i] = fmaf(dh[c][i], n[c][i], sums[SUM_B][c][i]);
          }
        }
        if (p.pre_g) {
          ld_param<FULL>(p.pre_g, p.params_vec, col, D, t);
          mul8(d[c], t);
        }
        s1 += sum8(d[c]);
#pragma unroll
        for (int i = 0; i < 8; ++i) s2 = fmaf(d[c][i], n[c][i], s2);
      }
      s1 = warp_sum(s1);
      s2 = warp_sum(s2);
      if constexpr (WPR > 1) {
        if (lane == 0) {
          red[it][0][grp][part][0] = s1;
          red[it][0][grp][part][1] = s2;
        }
        row_barrier<WPR>(grp);
        s1 = s2 = 0.f;
#pragma unroll
        for (int i = 0; i < WPR; ++i) {
          s1 += red[it][0][grp][i][0];
          s2 += red[it][0][grp][i][1];
        }
      }
      s1 = pre_layer ? s1 / (float)D : 0.f;
      s2 /= (float)D;
#pragma unroll
      for (int c = 0; c < NC; ++c) {
#pragma unroll
        for (int i = 0; i < 8; ++i) Z[c][i] += zr * (d[c][i] - s1 - n[c][i] * s2);
        mask8<FULL>(Z[c], c0 + c * kChunk + 8 * lane, D);
      }
    }
    float s3 = 0.f, s4 = 0.f;
#pragma unroll
    for (int c = 0; c < NC; ++c) {
      const int cc = c0 + c * kChunk, col = cc + 8 * lane;
      float t[8];
      if (post) {
        sub8(u[c], ym);
        scale8(u[c], yr, u[c]);
        mask8<FULL>(u[c], col, D);
      }
      if (p.dx.p && (FULL || cc < D)) {
        scale8(Z[c], p.res, t);
        st_mat<FULL>(p.dx, row, cc, D, sm, t);
      }
      if (ROWWISE) {
        if (p.dgate.p) {
          float v[8];
#pragma unroll
          for (int i = 0; i < 8; ++i) v[i] = u[c][i];
          if (p.post_g) {
            ld_param<FULL>(p.post_g, p.params_vec, col, D, t);
            mul8(v, t);
          }
          if (p.post_b) {
            ld_param<FULL>(p.post_b, p.params_vec, col, D, t);
            add8(v, t);
          }
          mul8(v, Z[c]);
          put(p.dgate, row, c, v);
        }
        mul8(Z[c], gate[c]);
      }
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        sums[SUM_P][c][i] += Z[c][i];
        sums[SUM_Q][c][i] = fmaf(Z[c][i], u[c][i], sums[SUM_Q][c][i]);
      }
      if (!ROWWISE) mul8(Z[c], gate[c]);
      if (p.post_g) {
        ld_param<FULL>(p.post_g, p.params_vec, col, D, t);
        mul8(Z[c], t);
      }
      s3 += sum8(Z[c]);
#pragma unroll
      for (int i = 0; i < 8; ++i) s4 = fmaf(Z[c][i], u[c][i], s4);
    }
    if (!p.dy.p && !p.dy8.q) continue;
    if (post) {
      s3 = warp_sum(s3);
      s4 = warp_sum(s4);
      if constexpr (WPR > 1) {
        if (lane == 0) {
          red[it][1][grp][part][0] = s3;
          red[it][1][grp][part][1] = s4;
        }
        row_barrier<WPR>(grp);
        s3 = s4 = 0.f;
#pragma unroll
        for (int i = 0; i < WPR; ++i) {
          s3 += red[it][1][grp][i][0];
          s4 += red[it][1][grp][i][1];
        }
      }
      s3 = post_layer ? s3 / (float)D : 0.f;
      s4 /= (float)D;
#pragma unroll
      for (int c = 0; c < NC; ++c) {
#pragma unroll
        for (int i = 0; i < 8; ++i) Z[c][i] = yr * (Z[c][i] - s3 - u[c][i] * s4);
        mask8<FULL>(Z[c], c0 + c * kChunk + 8 * lane, D);
      }
    }
#pragma unroll
    for (int c = 0; c < NC; ++c) {
      const int cc = c0 + c * kChunk;
      if (!FULL && cc >= D) break;
      if (p.dy.p) st_mat<FULL>(p.dy, row, cc, D, sm, Z[c]);
      if (p.dy8.q) put8<FULL>(p.dy8, row, cc, D, Z[c]);
    }
  }
  if (!ROWWISE && end > first) flush(start, stop);
  if (!params) return;
  // the team's sums of the parameters, behind the places of the groups
  float* o = p.ws + (ROWWISE ? 0 : (size_t)teams * 8 * D) + (size_t)team * 4 * D;
#pragma unroll
  for (int k = 0; k < 4; ++k)
#pragma unroll
    for (int c = 0; c < NC; ++c)
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const int col = c0 + c * kChunk + 8 * lane + i;
        if (FULL || col < D) o[(size_t)k * D + col] = ROWWISE ? sums[k][c][i] : mine[k * W + c * kChunk + i];
      }
}

// The sums that several teams have part of. blockIdx.y 0: the parameters' (if there are any),
// then one for each group that may be divided. Each of 32 slices of threads adds every 32nd
// team's, and the slices are added in order.
constexpr int kSlices = 32;

__global__ void __launch_bounds__(32 * kSlices) join_grad_finish_kernel(const JoinGrad p, int teams, int groups, bool rowwise,
                                                                        bool params) {
  __shared__ float red[4][kSlices][32];
  const int lane = threadIdx.x & 31, slice = threadIdx.x >> 5, col = blockIdx.x * 32 + lane, D = p.D;
  int y = (int)blockIdx.y;
  const bool param = params && y == 0;
  if (params) y -= 1;
  pdl_wait();
  pdl_trigger();
  int t0 = 0, t1 = teams - 1;
  long long q = 0, g0 = 0;
  if (!param) {
    if (groups < teams) {
      q = y;
    } else {  // the group that teams y and y + 1 share, if y is the first to have some of it
      const long long b = team_start(p.M, teams, y + 1);
      if (b % p.group == 0) return;
      q = b / p.group;
    }
    g0 = p.group > 0 ? q * p.group : 0;
    t0 = team_of(p.M, teams, g0);
    t1 = team_of(p.M, teams, p.group > 0 ? min(g0 + p.group, (long long)p.M) - 1 : p.M - 1);
    if (t0 == t1 || (groups >= teams && t0 != y)) return;
  }
  float s[4] = {0.f, 0.f, 0.f, 0.f};
  if (col < D) {
    for (int t = t0 + slice; t <= t1; t += kSlices) {
      const float* o = param ? p.ws + (rowwise ? 0 : (size_t)teams * 8 * D) + (size_t)t * 4 * D
                             : p.ws + ((size_t)t * 2 + (g0 > team_start(p.M, teams, t))) * 4 * D;
#pragma unroll
      for (int k = 0; k < 4; ++k) s[k] += o[(size_t)k * D + col];
    }
  }
#pragma unroll
  for (int k = 0; k < 4; ++k) red[k][slice][lane] = s[k];
  __syncthreads();
  if (slice != 0 || col >= D) return;
#pragma unroll
  for (int k = 0; k < 4; ++k)
    for (int i = 1; i < kSlices; ++i) s[k] += red[k][i][lane];
  if (param) {
    float* const out[4] = {p.dpre_b, p.dpre_g, p.dpost_b, p.dpost_g};
#pragma unroll
    for (int k = 0; k < 4; ++k)
      if (out[k]) out[k][col] = p.accumulate ? out[k][col] + s[k] : s[k];
    return;
  }
  auto put = [&](const MatOut& o, float v) {
    if (!o.p) return;
    const size_t at = (size_t)q * o.ld + col;
    if (o.dtype == LAZYMAR_F32) {
      float* d = static_cast<float*>(o.p) + at;
      *d = p.accumulate ? *d + v : v;
    } else {
      bf16* d = static_cast<bf16*>(o.p) + at;
      *d = from_f<bf16>(p.accumulate ? to_f(*d) + v : v);
    }
  };
  put(p.dshift, s[SUM_A]);
  put(p.dscale, (p.pre_g ? p.pre_g[col] : 1.f) * s[SUM_B] + (p.pre_b ? p.pre_b[col] * s[SUM_A] : 0.f));
  put(p.dgate, (p.post_g ? p.post_g[col] : 1.f) * s[SUM_Q] + (p.post_b ? p.post_b[col] * s[SUM_P] : 0.f));
}

__global__ void __launch_bounds__(256) join_grad_empty_kernel(const JoinGrad p) {
  const int col = blockIdx.x * 256 + threadIdx.x;
  pdl_wait();
  pdl_trigger();
  if (col >= p.D) return;
  float* const params[4] = {p.dpre_b, p.dpre_g, p.dpost_b, p.dpost_g};
  for (float* o : params)
    if (o) o[col] = 0.f;
  if (p.group > 0) return;
  const MatOut mods[3] = {p.dgate, p.dscale, p.dshift};
  for (const MatOut& o : mods) {
    if (!o.p) continue;
    if (o.dtype == LAZYMAR_F32) static_cast<float*>(o.p)[col] = 0.f;
    else static_cast<bf16*>(o.p)[col] = from_f<bf16>(0.f);
  }
}

// Warps of a row, and teams of a launch: those that live on every SM at once, as far as there are rows.
int row_warps(int D) {
  const int nc = (D + kChunk - 1) / kChunk;
  return nc <= 1 ? 1 : nc <= 2 ? 2 : nc <= 4 ? 4 : nc <= 5 ? 5 : nc <= 8 ? 8 : 16;
}
int grad_teams(int M, int D) {
  const int wpr = row_warps(D), warps = wpr == 5 ? 10 : wpr > 8 ? 16 : 8;
  const int most = kSMs * (warps <= 10 ? 2 : 1) * (warps / wpr);
  return M < most ? M : most;
}

template <int NC, int WPR>
cudaError_t join_grad_run(const Ctx& c, const JoinGrad& p, int teams, bool params) {
  constexpr int GROUPS = kWarps<WPR> / WPR, W = NC * WPR * kChunk;
  const bool rowwise = p.group == 1;
  const bool full = p.D == W && on_eight(p.dh) && on_eight(p.dz) && on_eight(p.z) && on_eight(p.y) && on_eight(p.gate) &&
                    on_eight(p.scale) && on_eight(p.dx) && on_eight(p.dy) && on_eight(p.dgate) && on_eight(p.dscale) &&
                    on_eight(p.dshift) && p.params_vec;
  const dim3 grid((unsigned)((teams + GROUPS - 1) / GROUPS)), block(kWarps<WPR> * 32);
  constexpr size_t most = (size_t)GROUPS * 4 * W * sizeof(float);
  const auto run = [&](auto kernel, bool sums) {
    if (sums && most > 16 * 1024) {
      const cudaError_t e = cudaFuncSetAttribute(reinterpret_cast<const void*>(kernel),
                                                 cudaFuncAttributeMaxDynamicSharedMemorySize, (int)most);
      if (e != cudaSuccess) return e;
    }
    return launch_pdl(kernel, grid, block, sums ? most : 0, c.stream, p, teams, params);
  };
  if (rowwise)
    return full ? run(join_grad_kernel<NC, WPR, true, true>, false) : run(join_grad_kernel<NC, WPR, false, true>, false);
  return full ? run(join_grad_kernel<NC, WPR, true, false>, params) : run(join_grad_kernel<NC, WPR, false, false>, params);
}

int groups_of(int M, int group) { return group > 0 ? (M - 1) / group + 1 : 1; }

}  // namespace

cudaError_t launch_join(const Ctx& c, const Join& p) {
  const int nc = (p.D + kChunk - 1) / kChunk;
  if (nc <= 1) return join_run<1, 1>(c, p);
  if (nc <= 2) return join_run<2, 1>(c, p);
  if (nc <= 4) return join_run<2, 2>(c, p);
  if (nc <= 5) return join_run<1, 5>(c, p);
  if (nc <= 8) return join_run<2, 4>(c, p);
  if (nc <= 16) return join_run<2, 8>(c, p);
  return join_run<2, 16>(c, p);
}

size_t join_grad_workspace(int M, int D, int group) {
  if (M < 1 || D < 1 || D > kLnMaxWidth || group < 0) return 0;
  return (size_t)grad_teams(M, D) * (group == 1 ? 4 : 12) * D * sizeof(float);
}

cudaError_t launch_join_grad(const Ctx& c, const JoinGrad& p) {
  if (p.M == 0) {  // sums over no rows; of gate, scale and shift only the row that all share is there
    if (p.accumulate) return cudaSuccess;
    return launch_pdl(join_grad_empty_kernel, dim3((unsigned)((p.D + 255) / 256)), dim3(256), 0, c.stream, p);
  }
  const bool params = p.dpost_g || p.dpost_b || p.dpre_g || p.dpre_b, mods = p.dgate.p || p.dscale.p || p.dshift.p;
  const int teams = grad_teams(p.M, p.D), groups = groups_of(p.M, p.group);
  cudaError_t e;
  switch (row_warps(p.D)) {
    case 1: e = join_grad_run<1, 1>(c, p, teams, params); break;
    case 2: e = join_grad_run<1, 2>(c, p, teams, params); break;
    case 4: e = join_grad_run<1, 4>(c, p, teams, params); break;
    case 5: e = join_grad_run<1, 5>(c, p, teams, params); break;
    case 8: e = join_grad_run<1, 8>(c, p, teams, params); break;
    default: e = p.D <= 16 * kChunk ? join_grad_run<1, 16>(c, p, teams, params) : join_grad_run<2, 16>(c, p, teams, params);
  }
  if (e != cudaSuccess) return e;
  const int divided = p.group == 1 || !mods || teams == 1 ? 0 : groups < teams ? groups : teams - 1;
  if (!divided && !params) return cudaSuccess;
  return launch_pdl(join_grad_finish_kernel, dim3((unsigned)((p.D + 31) / 32), (unsigned)(divided + (params ? 1 : 0))),
                    dim3(32 * kSlices), 0, c.stream, p, teams, groups, p.group == 1, params);
}

}  // namespace lm
