// The gradient of the residual join (lazymar_join_grad).
//
// A row is worked on by WPR warps (a team), NC chunks of 256 columns a warp. The rows are divided into consecutive
// ranges, so that a group's rows (those with one row of modulation) meet in one place. A lane keeps four sums
// of each of its columns while the group lasts,
//   A = sum dh, B = sum dh n, P = sum Z, Q = sum Z u,
// from which all gradients of modulation and parameters follow. TOGETHER (groups of kTogether rows or more, or one
// for all): a CTA has a range, its teams take the rows in turn and join their sums in shared memory at a group's
// end; otherwise each team has a range of its own. A group that lies in one range is finished there; the others leave
// their sums in the workspace, two places a range (the group that it begins in, and the one that it ends in), and
// a second kernel adds them in the ranges' order. ROWWISE (every row has its own
// modulation): the modulation's gradients are written with the row, and the four
// sums, weighted, are those of the parameters.
// The rows come by bulk copies into a ring in shared memory (join_rows.cuh); a piece is read when it is needed, which
// keeps a lane's registers to what lets 20 warps live on an SM (24 without sums, 16 with all four).
// 40960 x 1280 from two 8-bit checkpoints, bf16 dh, fp32 dz, modulation of 320 rows a group, dy in bf16 and 8 bits: 141
// us, 5.6 TB/s (floor 116), bound by instruction issue (57 % under ncu) and the latency of a row's exchange. 16384 x 1024
// with a modulation and its gradients for each row: 81 (floor 69). Both norms, 4801 x 777 in bf16: 33 (floor 6.6),
// elements loaded and stored one by one, eight rows a team. Two chunks a warp and half the warps: 178 where one chunk
// took 155; the next row in registers instead of a ring: 574.
#pragma once

#include "join_rows.cuh"

namespace lm {

enum { SUM_A = 0, SUM_B = 1, SUM_P = 2, SUM_Q = 3 };

// What a launch computes besides dx and dy: the sums (bits 1 << SUM_*) that modulation and parameters need.
struct JoinSums {
  unsigned mods, params;
};

// PLAIN: a modulated block's: dh, dz, z, y, gate, scale, dx and dy given, no norm of y, no parameters and none of their gradients.
// Warps on an SM, by what a lane keeps: P is not needed then, and ROWWISE no sum at all.
// (40960 x 1280 with 320 rows a group: 20 warps 141 us, 16 152; x 768 15 warps 96, 18 105. More of them spill.)
constexpr int grad_sm_warps(int wpr, bool plain, bool rowwise) { return plain ? (rowwise ? 24 : wpr == 3 ? 15 : 20) : 16; }
constexpr int kMostGradWarps = 24;
constexpr int kTogether = 192;

namespace {

// Sums of a and b over the warp, both in every lane: the halves of the warp take one each after the first exchange.
__device__ __forceinline__ float2 warp_sum2(float a, float b) {
  const bool upper = threadIdx.x & 16;
  float x = upper ? b : a;
  x += __shfl_xor_sync(0xffffffffu, upper ? a : b, 16);
#pragma unroll
  for (int o = 8; o > 0; o >>= 1) x += __shfl_xor_sync(0xffffffffu, x, o);
  const float y = __shfl_xor_sync(0xffffffffu, x, 16);
  return upper ? make_float2(y, x) : make_float2(x, y);
}
// The same over the row's warps (`red`: one place for each).
template <int WPR, int GROUPS>
__device__ __forceinline__ float2 row_sum2(float a, float b, float2* red, int grp, int part) {
  float2 s = warp_sum2(a, b);
  if constexpr (WPR > 1) {
    if ((threadIdx.x & 31) == 0) red[part] = s;
    row_barrier<WPR, GROUPS>(grp);
    s = make_float2(0.f, 0.f);
#pragma unroll
    for (int i = 0; i < WPR; ++i) {
      s.x += red[i].x;
      s.y += red[i].y;
    }
  }
  return s;
}

template <int NC, int WPR, bool WHOLE, bool ROWWISE, bool PLAIN>
__global__ void __launch_bounds__(cta_warps(WPR, grad_sm_warps(WPR, PLAIN, ROWWISE)) * 32, 1)
    join_grad_kernel(const __grid_constant__ JoinGrad p, const __grid_constant__ RingPlan plan, const Teams ranges, int together,
                     JoinSums need, unsigned* err) {
  constexpr int WARPS = cta_warps(WPR, grad_sm_warps(WPR, PLAIN, ROWWISE)), GROUPS = WARPS / WPR;
  // the four parameters (NC 1; of wider rows they stay where they are), each warp's modulation (gate, 1 + scale), the rings
  constexpr int W = NC * WPR * kChunk, PARAMS = PLAIN || NC > 1 ? 0 : 4 * W, MODS = ROWWISE ? 0 : 2 * NC * kLaneChunk;
  constexpr int JOINED = ROWWISE || GROUPS == 1 ? 0 : 4 * W;
  extern __shared__ __align__(128) float row_smem[];
  __shared__ uint64_t bars[WARPS][kMostStages];
  __shared__ float2 red[2][2][GROUPS][WPR];
  __shared__ int abort_word;
  volatile int* abort_flag = &abort_word;
  const int warp = threadIdx.x >> 5, grp = warp / WPR, part = warp % WPR;
  // together: GROUPS, the steps of a team's rows, otherwise 1
  const int D = p.D, c0 = part * NC * kChunk;
  const int range = together > 1 || GROUPS == 1 ? (int)blockIdx.x : (int)blockIdx.x * GROUPS + grp;
  if (threadIdx.x == 0) abort_word = 0;
  const bool live = range < ranges.n;
  const int begin = live ? team_start(ranges, range) : 0, end = live ? team_start(ranges, range + 1) : 0;
  const int first = begin + (together > 1 ? grp : 0);
  RowRing<WHOLE, false> ring;
  float* const params = row_smem + part * kLaneChunk;
  float* const mods = row_smem + PARAMS + warp * MODS;
  float* const joined = row_smem + PARAMS + WARPS * MODS + part * NC * kLaneChunk;  // sums of a CTA's teams
  uint8_t* const rings = reinterpret_cast<uint8_t*>(row_smem + PARAMS + WARPS * MODS + JOINED);
  ring.init(rings + (size_t)warp * plan.depth * plan.stage, bars[warp], plan, c0, min(NC * kChunk, D - c0), p.M, D, first,
            together);
  pdl_wait();
  pdl_trigger();
  if (PARAMS > 0 && grp == 0) {
    const float* const given[4] = {p.post_g, p.post_b, p.pre_g, p.pre_b};
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      if (!given[k]) continue;
      float t[8];
      load_param<WHOLE>(given[k], Columns<WHOLE>(c0, D), t);
      lane_put(params + k * W, t);
    }
  }
  __syncthreads();
  // parameter k (post_g, post_b, pre_g, pre_b) of chunk c
  const auto parameter = [&](int k, const float* at, int c, float (&t)[8]) {
    if (PARAMS > 0) lane_get(params + k * W, t);
    else load_param<WHOLE>(at, Columns<WHOLE>(c0 + c * kChunk, D), t);
  };
  for (int s = 0; s < plan.depth; ++s)
    if (first + s * together < end) ring.fetch(plan, first + s * together, s, c0);
  const float per_D = 1.f / (float)D;
  const bool pre = PLAIN || p.pre != LAZYMAR_NORM_NONE, post = !PLAIN && p.post != LAZYMAR_NORM_NONE;
  const bool pre_layer = p.pre == LAZYMAR_NORM_LAYER, post_layer = p.post == LAZYMAR_NORM_LAYER;
  const unsigned sums_of = need.mods | need.params;
  const bool ab = !(PLAIN && ROWWISE) && (ROWWISE ? need.params & 3u : sums_of & 3u);
  const bool pq = !(PLAIN && ROWWISE) && (ROWWISE ? need.params >> 2 : sums_of >> 2);

  const bool has_dz = PLAIN || p.dz.p, has_y = PLAIN || p.y.p, has_gate = PLAIN || p.gate.p, has_scale = PLAIN || p.scale.p;
  const bool has_dx = PLAIN || p.dx.p, has_dy = PLAIN || p.dy.p;

  // statistics and 8-bit scales of the next row
  float next_ym = 0.f, next_yr = 1.f, next_zm = 0.f, next_zr = 1.f;
  uint32_t next_zs[NC], next_ys[NC];
  const uint8_t* z_scales[NC];
  const uint8_t* y_scales[NC];
#pragma unroll
  for (int c = 0; c < NC; ++c) {
    next_zs[c] = next_ys[c] = 0;
    z_scales[c] = scales_of<WHOLE>(p.z, c0 + c * kChunk, D);
    y_scales[c] = scales_of<WHOLE>(p.y, c0 + c * kChunk, D);
  }
  auto statistics = [&](int row) {
    if (row >= end) return;
    if (pre) {
      if (pre_layer) next_zm = p.z_mean[row];
      next_zr = p.z_rstd[row];
    }
    if (post) {
      if (post_layer) next_ym = p.y_mean[row];
      next_yr = p.y_rstd[row];
    }
#pragma unroll
    for (int c = 0; c < NC; ++c) {
      if (z_scales[c]) next_zs[c] = z_scales[c][row];
      if (y_scales[c]) next_ys[c] = y_scales[c][row];
    }
  };
  statistics(first);

  float sums[4][NC][8];
#pragma unroll
  for (int c = 0; c < NC; ++c)
#pragma unroll
    for (int i = 0; i < 8; ++i) sums[0][c][i] = sums[1][c][i] = sums[2][c][i] = sums[3][c][i] = 0.f;
  bool dead = false;  // a wait ran out: nothing is written any more
  // out (+)= v for a row of a modulation's gradient
  auto put = [&](const MatOut& o, unsigned r, const Columns<WHOLE>& cc, float (&v)[8]) {
    if (p.accumulate) {
      float t[8];
      load_row<WHOLE>(o.p, o.ld, o.dtype, r, cc, t);
      add8(v, t);
    }
    if (!dead) store_row<WHOLE>(o, r, cc, v);
  };
  auto put_sum = [&](float* o, const Columns<WHOLE>& cc, const float (&v)[8]) {
    if (!dead) store_row<WHOLE>(MatOut{o, 0, LAZYMAR_F32, true}, 0u, cc, v);
  };
  float* const slots = p.ws + (size_t)range * 8 * D;
  float* const param = p.ws + (size_t)ranges.n * 8 * D + (size_t)range * 4 * D;

  // The end of a group, or of its part in this range: rows start .. stop.
  auto flush = [&](int start, int stop) {
    if (together > 1) {
      for (int g = 0; g < GROUPS; ++g) {
        if (g == grp) {
#pragma unroll
          for (int k = 0; k < 4; ++k) {
            if ((PLAIN && k == SUM_P) || !(sums_of >> k & 1u)) continue;
#pragma unroll
            for (int c = 0; c < NC; ++c) {
              float* at = joined + k * W + c * kLaneChunk;
              if (g > 0) {
                float t[8];
                lane_get(at, t);
                add8(sums[k][c], t);
              }
              lane_put(at, sums[k][c]);
            }
          }
        }
        __syncthreads();
      }
#pragma unroll
      for (int k = 0; k < 4; ++k)
#pragma unroll
        for (int c = 0; c < NC; ++c) {
          if (grp == 0 && !(PLAIN && k == SUM_P) && (sums_of >> k & 1u)) {
            lane_get(joined + k * W + c * kLaneChunk, sums[k][c]);
          } else {
#pragma unroll
            for (int i = 0; i < 8; ++i) sums[k][c][i] = 0.f;
          }
        }
      if (grp > 0) return;
    }
    const int q = start / p.group, g0 = q * p.group, g1 = g0 + min(p.group, p.M - g0);
    const bool whole = start == g0 && stop == g1;
    float* slot = slots + (size_t)(start > begin) * 4 * D;
#pragma unroll
    for (int c = 0; c < NC; ++c) {
      const Columns<WHOLE> cc(c0 + c * kChunk, D);
      float v[8], t[8];
      // the parameters' sums go on in the workspace, group by group
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        if (PLAIN || !(need.params >> k & 1u)) continue;
        copy8(v, sums[k][c]);
        if (k < 2 ? has_scale : has_gate) {
          lane_get(mods + (k < 2 ? NC + c : c) * kLaneChunk, t);
          mul8(v, t);
        }
        if (start > begin) {
          load_param<WHOLE>(param + (size_t)k * D, cc, t);
          add8(v, t);
        }
        put_sum(param + (size_t)k * D, cc, v);
      }
      if (whole) {
        if (p.dshift.p) {
          copy8(v, sums[SUM_A][c]);
          put(p.dshift, q, cc, v);
        }
        if (p.dscale.p) {
          copy8(v, sums[SUM_B][c]);
          if (!PLAIN && p.pre_g) {
            parameter(2, p.pre_g, c, t);
            mul8(v, t);
          }
          if (!PLAIN && p.pre_b) {
            parameter(3, p.pre_b, c, t);
            acc8(v, t, sums[SUM_A][c]);
          }
          put(p.dscale, q, cc, v);
        }
        if (p.dgate.p) {
          copy8(v, sums[SUM_Q][c]);
          if (!PLAIN && p.post_g) {
            parameter(0, p.post_g, c, t);
            mul8(v, t);
          }
          if (!PLAIN && p.post_b) {
            parameter(1, p.post_b, c, t);
            acc8(v, t, sums[SUM_P][c]);
          }
          put(p.dgate, q, cc, v);
        }
      } else {
#pragma unroll
        for (int k = 0; k < 4; ++k)
          if (!(PLAIN && k == SUM_P) && (need.mods >> k & 1u)) put_sum(slot + (size_t)k * D, cc, sums[k][c]);
      }
#pragma unroll
      for (int k = 0; k < 4; ++k)
#pragma unroll
        for (int i = 0; i < 8; ++i) sums[k][c][i] = 0.f;
    }
  };

  int it = 0, row = first;
  for (int start = begin, stop; start < end; start = stop) {  // group by group
    stop = end;
    if (!ROWWISE) {
      const int r = p.group > 0 ? start / p.group : 0;
      if (p.group > 0) stop = min(end - r * p.group, p.group) + r * p.group;
#pragma unroll
      for (int c = 0; c < NC; ++c) {
        const Columns<WHOLE> cc(c0 + c * kChunk, D);
        float t[8];
        if (has_gate) {
          load_row<WHOLE>(p.gate, r, cc, t);
          lane_put(mods + c * kLaneChunk, t);
        }
        if (has_scale) {
          load_row<WHOLE>(p.scale, r, cc, t);
#pragma unroll
          for (int i = 0; i < 8; ++i) t[i] += 1.f;
          lane_put(mods + (NC + c) * kLaneChunk, t);
        }
      }
    }
    for (; row < stop; row += together, it ^= 1) {
      const float ym = next_ym, yr = next_yr, zm = next_zm, zr = next_zr;
      uint32_t zs[NC], ys[NC];
#pragma unroll
      for (int c = 0; c < NC; ++c) {
        zs[c] = next_zs[c];
        ys[c] = next_ys[c];
      }
      statistics(row + together);
      const bool ok = dead || ring.wait(abort_flag, err);
      dead |= !__all_sync(0xffffffffu, ok);
      float d[NC][8], n[NC][8], Z[NC][8], u[NC][8];
      int i = 0;
      const auto from = [&](const Rows& m, const uint32_t (&scales)[NC], float (&to)[NC][8]) {
        const uint8_t* st = ring.piece(plan, i, row, c0);
#pragma unroll
        for (int c = 0; c < NC; ++c)
          load_stage<WHOLE>(st + (uint32_t)c * kChunk * plan.t[i].e, m.dtype, scales[c], Columns<WHOLE>(c0 + c * kChunk, D), to[c]);
        ++i;
      };
      const auto none = [&](float (&to)[NC][8]) {
#pragma unroll
        for (int c = 0; c < NC; ++c)
#pragma unroll
          for (int k = 0; k < 8; ++k) to[c][k] = 0.f;
      };
      if (pre) {
        from(p.dh, zs, d);
        from(p.z, zs, n);
      }
      float mod[NC][8];  // ROWWISE: 1 + scale, then gate
      if (ROWWISE && has_scale) {
        i = plan.n - 1;
        from(p.scale, zs, mod);
#pragma unroll
        for (int c = 0; c < NC; ++c)
#pragma unroll
          for (int k = 0; k < 8; ++k) mod[c][k] += 1.f;
        i = pre ? 2 : 0;
      }
      // (dz and y are read when they are needed: fewer registers)
      if (pre) {
        float s1 = 0.f, s2 = 0.f;
#pragma unroll
        for (int c = 0; c < NC; ++c) {
          const Columns<WHOLE> cc(c0 + c * kChunk, D);
          float t[8];
          sub8(n[c], zm);
          scale8(n[c], zr, n[c]);
          cc.mask(n[c]);
          if (ROWWISE) {
            if (p.dscale.p) {
              float v[8];
              copy8(v, n[c]);
              if (!PLAIN && p.pre_g) {
                parameter(2, p.pre_g, c, t);
                mul8(v, t);
              }
              if (!PLAIN && p.pre_b) {
                parameter(3, p.pre_b, c, t);
                add8(v, t);
              }
              mul8(v, d[c]);
              put(p.dscale, row, cc, v);
            }
            if (p.dshift.p) {
              copy8(t, d[c]);
              put(p.dshift, row, cc, t);
            }
            if (has_scale) mul8(d[c], mod[c]);
          }
          if (ab) {
            add8(sums[SUM_A][c], d[c]);
            acc8(sums[SUM_B][c], d[c], n[c]);
          }
          if (!ROWWISE && has_scale) {
            lane_get(mods + (NC + c) * kLaneChunk, t);
            mul8(d[c], t);
          }
          if (!PLAIN && p.pre_g) {
            parameter(2, p.pre_g, c, t);
            mul8(d[c], t);
          }
          s1 += sum8(d[c]);
          s2 += dot8(d[c], n[c]);
        }
        const float2 s = row_sum2<WPR, GROUPS>(s1, s2, red[it][0][grp], grp, part);
        s1 = pre_layer ? s.x * per_D : 0.f;
        s2 = -s.y * per_D;
        if (has_dz) from(p.dz, zs, Z);
        else none(Z);
#pragma unroll
        for (int c = 0; c < NC; ++c) {
          const float m2[8] = {s2, s2, s2, s2, s2, s2, s2, s2}, r[8] = {zr, zr, zr, zr, zr, zr, zr, zr};
          sub8(d[c], s1);
          acc8(d[c], n[c], m2);
          acc8(Z[c], d[c], r);
          Columns<WHOLE>(c0 + c * kChunk, D).mask(Z[c]);
        }
      } else {
        from(p.dz, zs, Z);
      }
      if (has_y) from(p.y, ys, u);
      else none(u);
      if (ROWWISE && has_gate) from(p.gate, zs, mod);
      ring.next(plan, row + plan.depth * together, end, c0, dead);
      float s3 = 0.f, s4 = 0.f;
#pragma unroll
      for (int c = 0; c < NC; ++c) {
        const Columns<WHOLE> cc(c0 + c * kChunk, D);
        float t[8];
        if (has_dx && !dead) {
          scale8(Z[c], p.res, t);
          store_row<WHOLE>(p.dx, row, cc, t);
        }
        if (post) {
          sub8(u[c], ym);
          scale8(u[c], yr, u[c]);
          cc.mask(u[c]);
        }
        if (ROWWISE) {
          if (p.dgate.p) {
            float v[8];
            copy8(v, u[c]);
            if (!PLAIN && p.post_g) {
              parameter(0, p.post_g, c, t);
              mul8(v, t);
            }
            if (!PLAIN && p.post_b) {
              parameter(1, p.post_b, c, t);
              add8(v, t);
            }
            mul8(v, Z[c]);
            put(p.dgate, row, cc, v);
          }
          if (has_gate) mul8(Z[c], mod[c]);
        }
        if (pq) {
          if (!PLAIN) add8(sums[SUM_P][c], Z[c]);
          acc8(sums[SUM_Q][c], Z[c], u[c]);
        }
        if (!ROWWISE && has_gate) {
          lane_get(mods + c * kLaneChunk, t);
          mul8(Z[c], t);
        }
        if (!PLAIN && p.post_g) {
          parameter(0, p.post_g, c, t);
          mul8(Z[c], t);
        }
        if (post) {
          s3 += sum8(Z[c]);
          s4 += dot8(Z[c], u[c]);
        }
      }
      if (!has_dy && !p.dy8.q) continue;
      if (post) {
        const float2 s = row_sum2<WPR, GROUPS>(s3, s4, red[it][1][grp], grp, part);
        s3 = post_layer ? s.x * per_D : 0.f;
        s4 = -s.y * per_D;
#pragma unroll
        for (int c = 0; c < NC; ++c) {
          const float m2[8] = {s4, s4, s4, s4, s4, s4, s4, s4};
          sub8(Z[c], s3);
          acc8(Z[c], u[c], m2);
          scale8(Z[c], yr, Z[c]);
          Columns<WHOLE>(c0 + c * kChunk, D).mask(Z[c]);
        }
      }
      if (dead) continue;
#pragma unroll
      for (int c = 0; c < NC; ++c) {
        const Columns<WHOLE> cc(c0 + c * kChunk, D);
        if (has_dy) store_row<WHOLE>(p.dy, row, cc, Z[c]);
        if (p.dy8.q) store_row8<WHOLE>(p.dy8, row, cc, Z[c]);
      }
    }
    if (!ROWWISE && p.group > 0) flush(start, stop);
  }
  if (dead) drain_ring(plan, bars);
  if (!ROWWISE && p.group > 0) return;
  // One group, or none: the teams' sums in turn, through shared memory, to the CTA's place.
  const unsigned of = ROWWISE ? need.params : need.mods | need.params;
  if ((PLAIN && ROWWISE) || !of) return;
  float* const mem = reinterpret_cast<float*>(rings);  // [4][GROUPS][W]
  __syncthreads();  // (the rings are done with)
#pragma unroll
  for (int k = 0; k < 4; ++k) {
    if ((PLAIN && k == SUM_P) || !(of >> k & 1u)) continue;
#pragma unroll
    for (int c = 0; c < NC; ++c) lane_put(mem + (k * GROUPS + grp) * W + (part * NC + c) * kLaneChunk, sums[k][c]);
  }
  __syncthreads();
  if (*abort_flag) return;
  for (int i = threadIdx.x; i < 4 * W; i += WARPS * 32) {
    const int k = i / W, at = i % W, col = at / kLaneChunk * kChunk + lane_column<WHOLE>(at % kLaneChunk);
    if (col >= D || !(of >> k & 1u)) continue;
    float s = 0.f;
#pragma unroll 4
    for (int j = 0; j < GROUPS; ++j) s += mem[(k * GROUPS + j) * W + at];
    p.ws[((size_t)blockIdx.x * 4 + k) * D + col] = s;
  }
}

template <int NC, int WPR, bool ROWWISE, bool PLAIN>
cudaError_t join_grad_run(const Ctx& c, const JoinGrad& p, const JoinSums& need, bool whole, const Teams& ranges, bool together) {
  constexpr int WARPS = cta_warps(WPR, grad_sm_warps(WPR, PLAIN, ROWWISE)), GROUPS = WARPS / WPR;
  RingPlan plan{};
  if (p.pre != LAZYMAR_NORM_NONE)
    for (const Rows* r : {&p.dh, &p.z}) add_stream(plan, *r, NC * kChunk);
  for (const Rows* r : {&p.dz, &p.y}) add_stream(plan, *r, NC * kChunk);
  if (ROWWISE)
    for (const Rows* r : {&p.gate, &p.scale}) add_stream(plan, *r, NC * kChunk);
  constexpr int W = NC * WPR * kChunk, FIXED = (PLAIN || NC > 1 ? 0 : 16 * W) + (ROWWISE ? 0 : WARPS * 2 * NC * kLaneChunk * 4) +
                  (ROWWISE || GROUPS == 1 ? 0 : 16 * W);
  set_depth(plan, kSmemRoom - FIXED, WARPS);
  const size_t rings = (size_t)WARPS * plan.depth * plan.stage, sums = (size_t)16 * GROUPS * W;
  const size_t smem = FIXED + (rings < sums ? sums : rings);
  const auto run = [&](auto kernel) {
    const cudaError_t e = cudaFuncSetAttribute(reinterpret_cast<const void*>(kernel),
                                               cudaFuncAttributeMaxDynamicSharedMemorySize, kSmemRoom);
    if (e != cudaSuccess) return e;
    return launch_pdl(kernel, dim3((unsigned)(together ? ranges.n : (ranges.n + GROUPS - 1) / GROUPS)), dim3(WARPS * 32),
                      smem, c.stream, p, plan, ranges, together ? GROUPS : 1, need, c.err);
  };
  return whole ? run(join_grad_kernel<NC, WPR, true, ROWWISE, PLAIN>) : run(join_grad_kernel<NC, WPR, false, ROWWISE, PLAIN>);
}

template <bool ROWWISE, bool PLAIN>
cudaError_t join_grad_launch(const Ctx& c, const JoinGrad& p, const JoinSums& need, bool whole, const Teams& ranges, bool together) {
  switch (row_warps(p.D)) {
    case 1: return join_grad_run<1, 1, ROWWISE, PLAIN>(c, p, need, whole, ranges, together);
    case 2: return join_grad_run<1, 2, ROWWISE, PLAIN>(c, p, need, whole, ranges, together);
    case 3: return join_grad_run<1, 3, ROWWISE, PLAIN>(c, p, need, whole, ranges, together);
    case 4: return join_grad_run<1, 4, ROWWISE, PLAIN>(c, p, need, whole, ranges, together);
    case 5: return join_grad_run<1, 5, ROWWISE, PLAIN>(c, p, need, whole, ranges, together);
    case 8: return join_grad_run<1, 8, ROWWISE, PLAIN>(c, p, need, whole, ranges, together);
    default:
      return p.D <= 16 * kChunk ? join_grad_run<1, 16, ROWWISE, PLAIN>(c, p, need, whole, ranges, together)
                                : join_grad_run<2, 16, ROWWISE, PLAIN>(c, p, need, whole, ranges, together);
  }
}

}  // namespace

cudaError_t launch_join_grad_rowwise(const Ctx& c, const JoinGrad& p, const JoinSums& need, bool whole, const Teams& ranges, bool together);
cudaError_t launch_join_grad_plain(const Ctx& c, const JoinGrad& p, const JoinSums& need, bool whole, const Teams& ranges, bool together);
cudaError_t launch_join_grad_plain_rowwise(const Ctx& c, const JoinGrad& p, const JoinSums& need, bool whole,
                                           const Teams& ranges, bool together);

}  // namespace lm
