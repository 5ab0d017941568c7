// The residual join of many rows (lazymar_join).
#pragma once

#include "join_rows.cuh"

namespace lm {

namespace {

// ---------------------------------------------------------------------------
// Forward, many rows
// ---------------------------------------------------------------------------
// A team of WPR warps works through consecutive rows, 256 columns a warp; its rows come by bulk
// copies into the warps' rings, so that the memory system always has the next ones to
// deliver while this one's sums are exchanged. Rows of a group follow each other, so
// the modulation stays in registers while a group lasts; STREAMED (every row has its own) it
// comes with the row.
// PLAIN: no norm of y and no parameters (the modulated norm of a block); fewer registers and
// so more warps on an SM.
#ifndef LM_SG
#define LM_SG 16
#endif
#ifndef LM_JW
#define LM_JW 20
#endif
constexpr int join_sm_warps(bool plain) { return plain ? LM_JW : 20; }

// Mean and 1 / deviation of a row of 256 columns a warp, as above. n: the warp's columns, per_n and per_D: 1 / n, 1 / D.
template <int WPR, int GROUPS, bool WHOLE>
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
    row_barrier<WPR, GROUPS>(grp);
    q = s = 0.f;
#pragma unroll
    for (int i = 0; i < WPR; ++i) {
      const float2 r = *reinterpret_cast<const float2*>(&red[i]);
      s += r.x;
      q += r.y;
    }
    if (layer) {
      mean = s * per_D;
#pragma unroll
      for (int i = 0; i < WPR; ++i) {
        const float2 r = *reinterpret_cast<const float2*>(&red[i].z);
        const float off = r.x - mean;
        q = fmaf(r.y * off, off, q);
      }
    }
  }
  rstd = rsqrtf(fmaf(q, per_D, eps));
}

enum { X_STREAM = 0, Y_STREAM = 1 };  // then gate, scale, shift as they are there (STREAMED)

template <int WPR, bool WHOLE, bool STREAMED, bool PLAIN>
__global__ void __launch_bounds__(cta_warps(WPR, join_sm_warps(PLAIN)) * 32, sm_ctas(WPR, join_sm_warps(PLAIN)))
    join_ring_kernel(const __grid_constant__ Join p, const __grid_constant__ RingPlan plan, const Teams teams, unsigned* err) {
  constexpr int WARPS = cta_warps(WPR, join_sm_warps(PLAIN)), GROUPS = WARPS / WPR;
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
  ring.init(ring_smem + (size_t)warp * plan.depth * plan.stage, bars[warp], plan, c0, min(kChunk, D - c0), p.M, D);
  pdl_wait();
  pdl_trigger();
  __syncthreads();
  if (team >= teams.n) return;
  const int first = team_start(teams, team), end = team_start(teams, team + 1);
  for (int s = 0; s < plan.depth; ++s)
    if (first + s < end) ring.fetch(plan, first + s, s, c0);

  const bool post = !PLAIN && p.post != LAZYMAR_NORM_NONE, pre = PLAIN || p.pre != LAZYMAR_NORM_NONE, leads = part == 0 && lane == 0;
  const float n = (float)min(max(D - c0, 0), kChunk), per_n = n > 0.f ? 1.f / n : 0.f, per_D = 1.f / (float)D;
  // scales of the next row's 8-bit y
  uint32_t next_s = 0;
  const uint8_t* const scales = scales_of<WHOLE>(p.y, c0, D);
  if (scales) next_s = scales[first];
  float gate[8], scale[8], shift[8];  // scale: 1 + scale
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    gate[i] = scale[i] = 1.f;
    shift[i] = 0.f;
  }
  int it = 0, stop = first;  // stop: the end of the group
  bool dead = false;  // a wait ran out: the rows are not written any more
  for (int row = first; row < end; ++row, it ^= 1) {
    if (!STREAMED && row == stop) {
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
      load_stage<WHOLE>(ring.piece(plan, i, row, c0), dtype, 0, cols, to);
    };
    from(X_STREAM, p.x.dtype, x);
    if (p.y.p) load_stage<WHOLE>(ring.piece(plan, Y_STREAM, row, c0), p.y.dtype, s, cols, v);
    if (STREAMED) {
      int i = p.y.p ? Y_STREAM + 1 : Y_STREAM;
      if (p.gate.p) from(i++, p.gate.dtype, gate);
      if (p.scale.p) {
        from(i++, p.scale.dtype, scale);
#pragma unroll
        for (int k = 0; k < 8; ++k) scale[k] += 1.f;
      }
      if (p.shift.p) from(i++, p.shift.dtype, shift);
    }
    ring.next(plan, row + plan.depth, end, c0, dead);
    float t[8];
    if (p.y.p) {
      if (p.y8.q && !dead) store_row8<WHOLE>(p.y8, row, cols, v);
      if (post) {
        float mean, rstd;
        ring_moments<WPR, GROUPS, WHOLE>(v, p.post == LAZYMAR_NORM_LAYER, cols, n, per_n, per_D, p.eps, red[it][0][grp], grp, part,
                                 mean, rstd);
        if (leads && !dead) {
          if (p.y_mean) p.y_mean[row] = mean;
          if (p.y_rstd) p.y_rstd[row] = rstd;
        }
        sub8(v, mean);
        scale8(v, rstd, v);
      }
      if (!PLAIN && p.post_g) {
        load_param<WHOLE>(p.post_g, cols, t);
        mul8(v, t);
      }
      if (!PLAIN && p.post_b) {
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
    ring_moments<WPR, GROUPS, WHOLE>(v, p.pre == LAZYMAR_NORM_LAYER, cols, n, per_n, per_D, p.eps, red[it][1][grp], grp, part, mean,
                             rstd);
    if (leads && !dead) {
      if (p.z_mean) p.z_mean[row] = mean;
      if (p.z_rstd) p.z_rstd[row] = rstd;
    }
    sub8(v, mean);
    scale8(v, rstd, v);
    if (!PLAIN && p.pre_g) {
      load_param<WHOLE>(p.pre_g, cols, t);
      mul8(v, t);
    }
    if (!PLAIN && p.pre_b) {
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

template <int WPR, bool PLAIN>
cudaError_t join_ring_run(const Ctx& c, const Join& p, bool whole) {
  constexpr int WARPS = cta_warps(WPR, join_sm_warps(PLAIN)), GROUPS = WARPS / WPR, CTAS = sm_ctas(WPR, join_sm_warps(PLAIN));
  RingPlan plan{};
  for (const Rows* r : {&p.x, &p.y}) add_stream(plan, *r, kChunk);
  const bool streamed = p.group > 0 && p.group < LM_SG && (p.gate.p || p.scale.p || p.shift.p);
  if (streamed)
    for (const Rows* r : {&p.gate, &p.scale, &p.shift}) add_stream(plan, *r, kChunk, p.group);
  constexpr int kRoom = 200 * 1024 / CTAS;
  set_depth(plan, kRoom, WARPS);
  const Teams teams = teams_of(p.M, c.num_sms * CTAS * GROUPS);
  const auto run = [&](auto kernel) {
    const cudaError_t e = cudaFuncSetAttribute(reinterpret_cast<const void*>(kernel),
                                               cudaFuncAttributeMaxDynamicSharedMemorySize, kRoom);
    if (e != cudaSuccess) return e;
    return launch_pdl(kernel, dim3((unsigned)((teams.n + GROUPS - 1) / GROUPS)), dim3(WARPS * 32),
                      (size_t)WARPS * plan.depth * plan.stage, c.stream, p, plan, teams, c.err);
  };
  if (streamed)
    return whole ? run(join_ring_kernel<WPR, true, true, PLAIN>) : run(join_ring_kernel<WPR, false, true, PLAIN>);
  return whole ? run(join_ring_kernel<WPR, true, false, PLAIN>) : run(join_ring_kernel<WPR, false, false, PLAIN>);
}

template <bool PLAIN>
cudaError_t join_ring_launch(const Ctx& c, const Join& p, bool whole) {
  switch (row_warps(p.D)) {
    case 1: return join_ring_run<1, PLAIN>(c, p, whole);
    case 2: return join_ring_run<2, PLAIN>(c, p, whole);
    case 3: return join_ring_run<3, PLAIN>(c, p, whole);
    case 4: return join_ring_run<4, PLAIN>(c, p, whole);
    case 5: return join_ring_run<5, PLAIN>(c, p, whole);
    case 8: return join_ring_run<8, PLAIN>(c, p, whole);
    default: return join_ring_run<16, PLAIN>(c, p, whole);
  }
}

}  // namespace

cudaError_t launch_join_plain(const Ctx& c, const Join& p, bool whole);

}  // namespace lm
