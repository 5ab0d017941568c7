// The residual join and its gradient: the norm behind a branch, its gate, the
// residual addition and the modulated norm in front of the next branch, each tensor
// read and written once. Bound by HBM bandwidth (13 bytes an element forward with an fp32
// stream, a bf16 branch and three 8-bit outputs, 17 backward), and next to it by
// instruction issue.
#include "join_rows.cuh"

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
// Forward, many rows
// ---------------------------------------------------------------------------
// A team of WPR warps works through consecutive rows, 256 columns a warp; its rows come by bulk
// copies into the warps' rings, so that the memory system always has the next ones to
// deliver while this one's sums are exchanged. Rows of a group follow each other, so
// the modulation stays in registers while a group lasts; ROWWISE (every row has its own) it
// comes with the row.
template <int WPR>
constexpr int kRingWarps = WPR == 5 ? 10 : WPR > 8 ? 16 : 8;
template <int WPR>
constexpr int kRingCtas = WPR > 8 ? 1 : WPR == 5 ? 2 : 3;

// Mean and 1 / deviation of a row of 256 columns a warp, as above. n: the warp's columns, per_n and per_D: 1 / n, 1 / D.
template <int WPR, bool WHOLE>
__device__ __forceinline__ void ring_moments(const float (&v)[8], bool layer, const Columns<WHOLE>& c, float n, float per_n,
                                             float per_D, float eps, float4* red, int grp, int part, float& mean,
                                             float& rstd) {
  float s = 0.f, q;
  mean = 0.f;
  if (layer) {
    s = warp_sum(sum8(v));
    mean = s * per_n;
    float d[8];
    copy8(d, v);
    sub8(d, mean);
    c.mask(d);
    q = squares8(d);
  } else {
    q = squares8(v);
  }
  q = warp_sum(q);
  if constexpr (WPR > 1) {
    if ((threadIdx.x & 31) == 0) red[part] = make_float4(s, q, mean, n);
    row_barrier<WPR>(grp);
    float4 r[WPR];
    q = s = 0.f;
#pragma unroll
    for (int i = 0; i < WPR; ++i) {
      r[i] = red[i];
      s += r[i].x;
      q += r[i].y;
    }
    if (layer) {
      mean = s * per_D;
#pragma unroll
      for (int i = 0; i < WPR; ++i) {
        const float off = r[i].z - mean;
        q = fmaf(r[i].w * off, off, q);
      }
    }
  }
  rstd = rsqrtf(fmaf(q, per_D, eps));
}

enum { X_STREAM = 0, Y_STREAM = 1 };  // then gate, scale, shift as they are there (ROWWISE)

template <int WPR, bool WHOLE, bool ROWWISE>
__global__ void __launch_bounds__(kRingWarps<WPR> * 32, kRingCtas<WPR>)
    join_ring_kernel(const __grid_constant__ Join p, const __grid_constant__ RingPlan plan, const Teams teams, unsigned* err) {
  constexpr int WARPS = kRingWarps<WPR>, GROUPS = WARPS / WPR;
  extern __shared__ __align__(128) uint8_t ring_smem[];
  __shared__ uint64_t bars[WARPS][kMostStages];
  __shared__ float4 red[2][2][GROUPS][WPR];
  __shared__ int abort_word;
  volatile int* abort_flag = &abort_word;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, grp = warp / WPR, part = warp % WPR;
  const int D = p.D, c0 = part * kChunk, team = (int)blockIdx.x * GROUPS + grp;
  const Columns<WHOLE> cols(c0, D);
  if (threadIdx.x == 0) abort_word = 0;
  RowRing<WHOLE> ring;
  ring.init(ring_smem + (size_t)warp * plan.depth * plan.stage, bars[warp], plan, c0, min(kChunk, D - c0));
  pdl_wait();
  pdl_trigger();
  __syncthreads();
  if (team >= teams.n) return;
  const int first = team_start(teams, team), end = team_start(teams, team + 1);
  for (int s = 0; s < plan.depth; ++s)
    if (first + s < end) ring.fetch(plan, first + s, s, c0, p.M);

  const bool post = p.post != LAZYMAR_NORM_NONE, pre = p.pre != LAZYMAR_NORM_NONE, leads = part == 0 && lane == 0;
  const float n = (float)min(max(D - c0, 0), kChunk), per_n = n > 0.f ? 1.f / n : 0.f, per_D = 1.f / (float)D;
  // scales of the next row's 8-bit y
  uint32_t next_s = 0;
  const uint8_t* scales = nullptr;
  if (p.y.p && p.y.dtype == LAZYMAR_E4M3 && lane < 2 && c0 + kBlk * lane < D)
    scales = p.y.scale + (size_t)(c0 / kBlk + lane) * p.y.lds;
  if (scales) next_s = scales[first];
  float gate[8], scale[8], shift[8];  // scale: 1 + scale
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    gate[i] = scale[i] = 1.f;
    shift[i] = 0.f;
  }
  int stop = first, it = 0;  // stop: the end of the group
  bool dead = false;         // a wait ran out: the rows are not written any more
  for (int row = first; row < end; ++row, it ^= 1) {
    if (!ROWWISE && row == stop) {
      const int r = p.group > 0 ? row / p.group : 0;
      stop = p.group > 0 ? min(end - r * p.group, p.group) + r * p.group : end;
      if (p.gate.p) load_row<WHOLE>(p.gate, r, cols, gate);
      if (p.shift.p) load_row<WHOLE>(p.shift, r, cols, shift);
      if (p.scale.p) {
        load_row<WHOLE>(p.scale, r, cols, scale);
#pragma unroll
        for (int i = 0; i < 8; ++i) scale[i] += 1.f;
      }
    }
    const uint32_t s = next_s;
    if (scales && row + 1 < end) next_s = scales[row + 1];
    const bool ok = dead || ring.wait(abort_flag, err);
    dead |= !__all_sync(0xffffffffu, ok);
    float v[8], x[8];
    const auto from = [&](int i, int dtype, float (&to)[8]) {
      load_stage<WHOLE>(ring.piece(plan, i, row, c0), dtype, 0, 0, cols, to);
    };
    from(X_STREAM, p.x.dtype, x);
    if (p.y.p) {
      uint32_t s0 = 0, s1 = 0;
      if (p.y.dtype == LAZYMAR_E4M3) {
        s0 = __shfl_sync(0xffffffffu, s, 0);
        s1 = __shfl_sync(0xffffffffu, s, 1);
      }
      load_stage<WHOLE>(ring.piece(plan, Y_STREAM, row, c0), p.y.dtype, s0, s1, cols, v);
    }
    if (ROWWISE) {
      int i = p.y.p ? Y_STREAM + 1 : Y_STREAM;
      if (p.gate.p) from(i++, p.gate.dtype, gate);
      if (p.scale.p) {
        from(i++, p.scale.dtype, scale);
#pragma unroll
        for (int k = 0; k < 8; ++k) scale[k] += 1.f;
      }
      if (p.shift.p) from(i++, p.shift.dtype, shift);
    }
    ring.next(plan, row + plan.depth, end, c0, p.M, dead);
    float t[8];
    if (p.y.p) {
      if (p.y8.q && !dead) store_row8<WHOLE>(p.y8, row, cols, v);
      if (post) {
        float mean, rstd;
        ring_moments<WPR, WHOLE>(v, p.post == LAZYMAR_NORM_LAYER, cols, n, per_n, per_D, p.eps, red[it][0][grp], grp, part,
                                 mean, rstd);
        if (leads && !dead) {
          if (p.y_mean) p.y_mean[row] = mean;
          if (p.y_rstd) p.y_rstd[row] = rstd;
        }
        sub8(v, mean);
        scale8(v, rstd, v);
      }
      if (p.post_g) {
        load_param<WHOLE>(p.post_g, cols, t);
        mul8(v, t);
      }
      if (p.post_b) {
        load_param<WHOLE>(p.post_b, cols, t);
        add8(v, t);
      }
      mul8(v, gate);
      const float res[8] = {p.res, p.res, p.res, p.res, p.res, p.res, p.res, p.res};
      acc8(v, x, res);
      cols.mask(v);
    } else {
      scale8(x, p.res, v);
    }
    if (!dead) {
      if (p.z.p) store_row<WHOLE>(p.z, row, cols, v);
      if (p.z8.q) store_row8<WHOLE>(p.z8, row, cols, v);
    }
    if (!pre) continue;
    float mean, rstd;
    ring_moments<WPR, WHOLE>(v, p.pre == LAZYMAR_NORM_LAYER, cols, n, per_n, per_D, p.eps, red[it][1][grp], grp, part, mean,
                             rstd);
    if (leads && !dead) {
      if (p.z_mean) p.z_mean[row] = mean;
      if (p.z_rstd) p.z_rstd[row] = rstd;
    }
    sub8(v, mean);
    scale8(v, rstd, v);
    if (p.pre_g) {
      load_param<WHOLE>(p.pre_g, cols, t);
      mul8(v, t);
    }
    if (p.pre_b) {
      load_param<WHOLE>(p.pre_b, cols, t);
      add8(v, t);
    }
    fma8(v, scale, shift);
    cols.mask(v);
    if (dead) continue;
    if (p.h.p) store_row<WHOLE>(p.h, row, cols, v);
    if (p.h8.q) store_row8<WHOLE>(p.h8, row, cols, v);
  }
}

// The streams of a launch, and stages for as many rows as its shared memory holds.
void add_stream(RingPlan& plan, const Rows& r) {
  if (!r.p) return;
  const uint32_t e = r.dtype == LAZYMAR_F32 ? 4 : r.dtype == LAZYMAR_BF16 ? 2 : 1;
  plan.t[plan.n++] = RowStream{static_cast<const uint8_t*>(r.p), (size_t)r.ld * e, plan.stage, e};
  plan.stage += kChunk * e + 32;
}

template <int WPR>
cudaError_t join_ring_run(const Ctx& c, const Join& p, bool whole) {
  constexpr int WARPS = kRingWarps<WPR>, GROUPS = WARPS / WPR;
  RingPlan plan{};
  add_stream(plan, p.x);
  add_stream(plan, p.y);
  if (p.group == 1) {
    add_stream(plan, p.gate);
    add_stream(plan, p.scale);
    add_stream(plan, p.shift);
  }
  constexpr int kRoom = 200 * 1024 / kRingCtas<WPR>;
  plan.depth = kRoom / (WARPS * (int)plan.stage);
  if (plan.depth > 4) plan.depth = 4;
  const Teams teams = teams_of(p.M, c.num_sms * kRingCtas<WPR> * GROUPS);
  const auto run = [&](auto kernel) {
    const cudaError_t e = cudaFuncSetAttribute(reinterpret_cast<const void*>(kernel),
                                               cudaFuncAttributeMaxDynamicSharedMemorySize, kRoom);
    if (e != cudaSuccess) return e;
    return launch_pdl(kernel, dim3((unsigned)((teams.n + GROUPS - 1) / GROUPS)), dim3(WARPS * 32),
                      (size_t)WARPS * plan.depth * plan.stage, c.stream, p, plan, teams, c.err);
  };
  if (p.group == 1)
    return whole ? run(join_ring_kernel<WPR, true, true>) : run(join_ring_kernel<WPR, false, true>);
  return whole ? run(join_ring_kernel<WPR, true, false>) : run(join_ring_kernel<WPR, false, false>);
}

}  // namespace

cudaError_t launch_join(const Ctx& c, const Join& p) {
  const int nc = (p.D + kChunk - 1) / kChunk;
  if (nc <= 16 && p.M > c.num_sms * 2) {
    const bool whole = p.D % 8 == 0 && on_eight(p.x) && on_eight(p.y) && on_eight(p.gate) && on_eight(p.scale) &&
                       on_eight(p.shift) && on_eight(p.z) && on_eight(p.h) && p.params_vec;
    if (nc <= 1) return join_ring_run<1>(c, p, whole);
    if (nc <= 2) return join_ring_run<2>(c, p, whole);
    if (nc <= 4) return join_ring_run<4>(c, p, whole);
    if (nc <= 5) return join_ring_run<5>(c, p, whole);
    if (nc <= 8) return join_ring_run<8>(c, p, whole);
    return join_ring_run<16>(c, p, whole);
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
