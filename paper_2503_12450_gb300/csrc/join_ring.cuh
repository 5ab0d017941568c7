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
// the modulation stays in shared memory while a group lasts; STREAMED (groups of one or two rows) it
// comes with the row. PLAIN: a modulated
// block's, with y, gate, scale and shift, without a norm of y and parameters.
// 40960 x 1024, fp32 stream, bf16 branch, three 8-bit outputs, 320 rows a group: 94 us, 5.8 TB/s (floor 81);
// instructions bound it next to HBM (450 a warp and row). The row in registers without a ring, 16 warps: 223 us. Both
// norms with parameters, 40000 x 777 in bf16: 104 us (floor 37), elements loaded and stored one by one.
// Warps on an SM, as many as need no spills, which cost more than more warps give. 40960 x 1024 with three 8-bit
// outputs: 28 warps 94 us, 24 101; x 1280 30 warps 114, 28 122; both norms at 40000 x 1024 in bf16 28 warps 88, 24 93, x 1280
// 20 warps 120, 25 (which spill) 143. With a row of modulation for each row, which is at HBM's rate, fewer rows at a
// time are better: 20 warps 121, 24 139.
constexpr int join_sm_warps(int wpr, bool plain, bool streamed) {
  return streamed || (!plain && wpr == 5) ? 20 : plain && wpr >= 3 ? 30 : 28;
}

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
  rstd = inv_sqrt(fmaf(q, per_D, eps));
}

enum { X_STREAM = 0, Y_STREAM = 1 };  // then gate, scale, shift as they are there (STREAMED)

template <int WPR, bool WHOLE, bool STREAMED, bool PLAIN>
__global__ void __launch_bounds__(cta_warps(WPR, join_sm_warps(WPR, PLAIN, STREAMED)) * 32, 1)
    join_ring_kernel(const __grid_constant__ Join p, const __grid_constant__ RingPlan plan, const Teams teams, unsigned* err) {
  constexpr int WARPS = cta_warps(WPR, join_sm_warps(WPR, PLAIN, STREAMED)), GROUPS = WARPS / WPR;
  // the four parameters, each warp's modulation (gate, 1 + scale, shift), the rings
  constexpr int PARAMS = PLAIN ? 0 : 4 * WPR * kLaneChunk, MODS = STREAMED ? 0 : 3 * kLaneChunk;
  extern __shared__ __align__(128) float row_smem[];
  __shared__ uint64_t bars[WARPS][kMostStages];
  __shared__ float4 red[2][2][GROUPS][WPR];
  __shared__ int abort_word;
  volatile int* abort_flag = &abort_word;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, grp = warp / WPR, part = warp % WPR;
  const int D = p.D, c0 = part * kChunk, team = (int)blockIdx.x * GROUPS + grp;
  const Columns<WHOLE> cols(c0, D);
  if (threadIdx.x == 0) abort_word = 0;
  const bool live = team < teams.n;
  const int first = live ? team_start(teams, team) : 0, end = live ? team_start(teams, team + 1) : 0;
  RowRing<WHOLE, STREAMED> ring;
  float* const params = row_smem + part * kLaneChunk;
  float* const mods = row_smem + PARAMS + warp * MODS;
  uint8_t* const rings = reinterpret_cast<uint8_t*>(row_smem + PARAMS + WARPS * MODS);
  ring.init(rings + (size_t)warp * plan.depth * plan.stage, bars[warp], plan, c0, min(kChunk, D - c0), p.M, D, first);
  pdl_wait();
  pdl_trigger();
  if (!PLAIN && grp == 0) {
    const float* const given[4] = {p.post_g, p.post_b, p.pre_g, p.pre_b};
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      if (!given[k]) continue;
      float t[8];
      load_param<WHOLE>(given[k], cols, t);
      lane_put(params + k * WPR * kLaneChunk, t);
    }
  }
  __syncthreads();
  if (!live) return;
  for (int s = 0; s < plan.depth; ++s)
    if (first + s < end) ring.fetch(plan, first + s, s, c0);

  const bool post = !PLAIN && p.post != LAZYMAR_NORM_NONE, pre = PLAIN || p.pre != LAZYMAR_NORM_NONE, leads = part == 0 && lane == 0;
  const bool has_y = PLAIN || p.y.p, has_gate = PLAIN || p.gate.p, has_scale = PLAIN || p.scale.p, has_shift = PLAIN || p.shift.p;
  const float n = (float)min(max(D - c0, 0), kChunk), per_n = n > 0.f ? 1.f / n : 0.f, per_D = 1.f / (float)D;
  // scales of the next row's 8-bit y
  uint32_t next_s = 0;
  const uint8_t* const scales = scales_of<WHOLE>(p.y, c0, D);
  if (scales) next_s = scales[first];
  int it = 0, stop = first;  // stop: the end of the group
  bool dead = false;  // a wait ran out: the rows are not written any more
  for (int row = first; row < end; ++row, it ^= 1) {
    if (!STREAMED && row == stop) {
      const int r = p.group > 0 ? row / p.group : 0;
      stop = p.group > 0 ? min(end - r * p.group, p.group) + r * p.group : end;
      float t[8];
      if (has_gate) {
        load_row<WHOLE>(p.gate, r, cols, t);
        lane_put(mods, t);
      }
      if (has_scale) {
        load_row<WHOLE>(p.scale, r, cols, t);
#pragma unroll
        for (int i = 0; i < 8; ++i) t[i] += 1.f;
        lane_put(mods + kLaneChunk, t);
      }
      if (has_shift) {
        load_row<WHOLE>(p.shift, r, cols, t);
        lane_put(mods + 2 * kLaneChunk, t);
      }
    }
    const uint32_t s = next_s;
    if (scales && row + 1 < end) next_s = scales[row + 1];
    const bool ok = dead || ring.wait(abort_flag, err);
    dead |= !__all_sync(0xffffffffu, ok);
    // each piece is read when it is needed, and the stage given on after the last: fewer registers
    float v[8], t[8];
    const int mod = has_y ? Y_STREAM + 1 : Y_STREAM;  // the first stream of the modulation
    const auto from = [&](int i, int dtype, uint32_t scale, float (&to)[8]) {
      load_stage<WHOLE>(ring.piece(plan, i, row, c0), dtype, scale, cols, to);
    };
    if (has_y) {
      from(Y_STREAM, p.y.dtype, s, v);
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
        lane_get(params, t);
        mul8(v, t);
      }
      if (!PLAIN && p.post_b) {
        lane_get(params + WPR * kLaneChunk, t);
        add8(v, t);
      }
      if (has_gate) {
        if (STREAMED) from(mod, p.gate.dtype, 0, t);
        else lane_get(mods, t);
        mul8(v, t);
      }
      from(X_STREAM, p.x.dtype, 0, t);
      const float res[8] = {p.res, p.res, p.res, p.res, p.res, p.res, p.res, p.res};
      acc8(v, t, res);
      cols.mask(v);
    } else {
      from(X_STREAM, p.x.dtype, 0, t);
      scale8(t, p.res, v);
    }
    if (!STREAMED) ring.next(plan, row + plan.depth, end, c0, dead);
    if (!dead) {
      if (p.z.p) store_row<WHOLE>(p.z, row, cols, v);
      if (p.z8.q) store_row8<WHOLE>(p.z8, row, cols, v);
    }
    if (!pre) {
      if (STREAMED) ring.next(plan, row + plan.depth, end, c0, dead);
      continue;
    }
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
      lane_get(params + 2 * WPR * kLaneChunk, t);
      mul8(v, t);
    }
    if (!PLAIN && p.pre_b) {
      lane_get(params + 3 * WPR * kLaneChunk, t);
      add8(v, t);
    }
    int i = mod + (has_gate ? 1 : 0);
    if (has_scale) {
      if (STREAMED) {
        from(i++, p.scale.dtype, 0, t);
#pragma unroll
        for (int k = 0; k < 8; ++k) t[k] += 1.f;
      } else {
        lane_get(mods + kLaneChunk, t);
      }
      mul8(v, t);
    }
    if (has_shift) {
      if (STREAMED) from(i, p.shift.dtype, 0, t);
      else lane_get(mods + 2 * kLaneChunk, t);
      add8(v, t);
    }
    if (STREAMED) ring.next(plan, row + plan.depth, end, c0, dead);
    cols.mask(v);
    if (dead) continue;
    if (p.h.p) store_row<WHOLE>(p.h, row, cols, v);
    if (p.h8.q) store_row8<WHOLE>(p.h8, row, cols, v);
  }
  if (dead) drain_ring(plan, bars);
}

template <int WPR, bool PLAIN, bool STREAMED>
cudaError_t join_ring_run(const Ctx& c, const Join& p, bool whole) {
  constexpr int WARPS = cta_warps(WPR, join_sm_warps(WPR, PLAIN, STREAMED)), GROUPS = WARPS / WPR;
  constexpr int FIXED = (PLAIN ? 0 : 4 * WPR * kLaneChunk * 4) + (STREAMED ? 0 : WARPS * 3 * kLaneChunk * 4);
  RingPlan plan{};
  for (const Rows* r : {&p.x, &p.y}) add_stream(plan, *r, kChunk);
  if (STREAMED)
    for (const Rows* r : {&p.gate, &p.scale, &p.shift}) add_stream(plan, *r, kChunk, p.group);
  set_depth(plan, kSmemRoom - FIXED, WARPS);
  const Teams teams = teams_of(p.M, c.num_sms * GROUPS);
  const auto run = [&](auto kernel) {
    const cudaError_t e = cudaFuncSetAttribute(reinterpret_cast<const void*>(kernel),
                                               cudaFuncAttributeMaxDynamicSharedMemorySize, kSmemRoom);
    if (e != cudaSuccess) return e;
    return launch_pdl(kernel, dim3((unsigned)((teams.n + GROUPS - 1) / GROUPS)), dim3(WARPS * 32),
                      (size_t)FIXED + (size_t)WARPS * plan.depth * plan.stage, c.stream, p, plan, teams, c.err);
  };
  return whole ? run(join_ring_kernel<WPR, true, STREAMED, PLAIN>) : run(join_ring_kernel<WPR, false, STREAMED, PLAIN>);
}

template <bool PLAIN>
cudaError_t join_ring_launch(const Ctx& c, const Join& p, bool whole) {
  // Fetching the modulation with each row costs more than waiting for it at each group's first, except for very small
  // groups: 40960 x 1024 in groups of 2 120 us with the rows, 131 without, of 3 117 and 117, of 8 117 and 101.
  const bool streamed = p.group > 0 && p.group < 3 && (p.gate.p || p.scale.p || p.shift.p);
#define LM_RUN(wpr) (streamed ? join_ring_run<wpr, PLAIN, true>(c, p, whole) : join_ring_run<wpr, PLAIN, false>(c, p, whole))
  switch (row_warps(p.D)) {
    case 1: return LM_RUN(1);
    case 2: return LM_RUN(2);
    case 3: return LM_RUN(3);
    case 4: return LM_RUN(4);
    case 5: return LM_RUN(5);
    case 8: return LM_RUN(8);
    default: return LM_RUN(16);
  }
#undef LM_RUN
}

}  // namespace

cudaError_t launch_join_plain(const Ctx& c, const Join& p, bool whole);

}  // namespace lm
