// The residual join: the norm behind a branch, its gate, the residual addition and the
// modulated norm in front of the next branch, each tensor read and written once (13 bytes an element with
// an fp32 stream, a bf16 branch and three 8-bit outputs). Here the kernel for few rows, up to two an SM, and for more than
// 4096 columns: the row in the registers of a few warps, all loads under way at once. That of many rows is in
// join_ring.cuh.
#include "join_ring.cuh"

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
// Mean and 1 / deviation of a row whose columns are spread over WPR warps, NC chunks a
// warp, columns that do not exist zero. Each warp takes the squares about its own mean,
// and the warps' sums are joined about the row's: one exchange between the warps, and
// no cancellation. RMS: the mean counts as 0.
template <int NC, int WPR, int GROUPS, bool FULL>
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
    row_barrier<WPR, GROUPS>(grp);
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
  rstd = inv_sqrt(q / (float)D + eps);
}

template <int WPR>
constexpr int kWarps = WPR == 5 ? 10 : WPR > 8 ? 16 : 8;

// ---------------------------------------------------------------------------
// Few rows
// ---------------------------------------------------------------------------
// WPR warps a row, NC chunks of 256 columns a warp, the row in registers throughout.
// FULL: D = 256 NC WPR and every row on a boundary, so that no column needs a check. Bound by latency: 2 x 1024 with a
// modulation for each row 3.1 us, 304 x 1024 with three 8-bit outputs 3.9 (through the rings of the other kernel 4.8), 608 rows
// 4.8 (5.0 there), 1216 rows 7.6 (7.1).
template <int NC, int WPR, bool FULL>
__global__ void __launch_bounds__(kWarps<WPR> * 32, NC == 1 ? 3 : WPR > 8 ? 1 : 2) join_kernel(const Join p) {
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
      moments<NC, WPR, GROUPS, FULL>(v, p.post == LAZYMAR_NORM_LAYER, D, c0, p.eps, red[0][grp], grp, part, mean, rstd);
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
  moments<NC, WPR, GROUPS, FULL>(v, p.pre == LAZYMAR_NORM_LAYER, D, c0, p.eps, red[1][grp], grp, part, mean, rstd);
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

template <int NC, int WPR>
cudaError_t join_run(const Ctx& c, const Join& p) {
  constexpr int GROUPS = kWarps<WPR> / WPR;
  const dim3 grid((unsigned)((p.M + GROUPS - 1) / GROUPS)), block(kWarps<WPR> * 32);
  if (p.D == NC * WPR * kChunk && on_eight(p.x) && on_eight(p.y) && on_eight(p.gate) && on_eight(p.scale) &&
      on_eight(p.shift) && on_eight(p.z) && on_eight(p.h) && p.params_vec)
    return launch_pdl(join_kernel<NC, WPR, true>, grid, block, 0, c.stream, p);
  return launch_pdl(join_kernel<NC, WPR, false>, grid, block, 0, c.stream, p);
}

}  // namespace

cudaError_t launch_join(const Ctx& c, const Join& p) {
  const int nc = (p.D + kChunk - 1) / kChunk;
  if (nc <= 16 && p.M > c.num_sms * 2) {
    const bool whole = p.D % 8 == 0 && on_eight(p.x) && on_eight(p.y) && on_eight(p.gate) && on_eight(p.scale) &&
                       on_eight(p.shift) && on_eight(p.z) && on_eight(p.h) && p.params_vec;
    const bool plain = !p.post && p.pre && !p.post_g && !p.post_b && !p.pre_g && !p.pre_b && p.y.p && p.gate.p && p.scale.p &&
                       p.shift.p;
    return plain ? launch_join_plain(c, p, whole) : join_ring_launch<false>(c, p, whole);
  }
  if (nc <= 1) return join_run<1, 1>(c, p);
  if (nc <= 2) return join_run<1, 2>(c, p);
  if (nc <= 4) return join_run<1, 4>(c, p);
  if (nc <= 5) return join_run<1, 5>(c, p);
  if (nc <= 8) return join_run<1, 8>(c, p);
  if (nc <= 16) return join_run<2, 8>(c, p);
  return join_run<2, 16>(c, p);
}

}  // namespace lm
