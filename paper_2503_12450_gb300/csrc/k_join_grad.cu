// The residual join's gradient: the kernel for rows that share a modulation (or have
// none), and what follows both kernels.
#include "join_grad.cuh"

namespace lm {

namespace {

// The sums that several teams have part of: the parameters' (blockIdx.y 0, if there are any),
// and those of each group that may be divided. A warp has 128 columns. `slices` warps share
// a task, each adds every so many teams', and they are added in order: all 32 warps of a
// CTA for the parameters and for groups with many teams, otherwise one, and a CTA has 32 groups.
constexpr int kFinishWarps = 32;

__global__ void __launch_bounds__(32 * kFinishWarps) join_grad_finish_kernel(const __grid_constant__ JoinGrad p, const Teams teams,
                                                                             int groups, int tasks, bool rowwise, JoinSums need,
                                                                             int group_slices) {
  __shared__ float red[4][kFinishWarps][32];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, c0 = blockIdx.x * 128 + lane, D = p.D;
  const bool param = need.params && blockIdx.y == 0;
  const int slices = param ? kFinishWarps : group_slices, slice = warp % slices;
  const int y = param ? 0 : ((int)blockIdx.y - (need.params ? 1 : 0)) * (kFinishWarps / slices) + warp / slices;
  const unsigned sums = param ? need.params : need.mods;
  pdl_wait();
  pdl_trigger();
  int t0 = 0, t1 = teams.n - 1, q = 0, g0 = 0;
  bool live = param || y < tasks;
  if (!param && live) {
    if (groups < teams.n) {
      q = y;
    } else {  // the group that teams y and y + 1 share, if y is the first to have some of it
      const int b = team_start(teams, y + 1);
      live = b % p.group != 0;
      q = b / p.group;
    }
    if (p.group > 0) g0 = q * p.group;
    t0 = team_of(teams, g0);
    t1 = team_of(teams, p.group > 0 ? g0 + min(p.group, p.M - g0) - 1 : p.M - 1);
    live = live && t0 != t1 && (groups < teams.n || t0 == y);
  }
  float s[4][4];
#pragma unroll
  for (int k = 0; k < 4; ++k)
#pragma unroll
    for (int i = 0; i < 4; ++i) s[k][i] = 0.f;
  if (live) {
#pragma unroll 2
    for (int t = t0 + slice; t <= t1; t += slices) {
      const float* o = param ? p.ws + (rowwise ? 0 : (size_t)teams.n * 8 * D) + (size_t)t * 4 * D
                             : p.ws + ((size_t)t * 2 + (g0 > team_start(teams, t))) * 4 * D;
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        if (!(sums >> k & 1u)) continue;
#pragma unroll
        for (int i = 0; i < 4; ++i)
          if (c0 + 32 * i < D) s[k][i] += o[(size_t)k * D + c0 + 32 * i];
      }
    }
  }
  if (slices > 1) {  // (uniform over the CTA)
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      __syncthreads();
#pragma unroll
      for (int k = 0; k < 4; ++k) red[k][warp][lane] = s[k][i];
      __syncthreads();
      if (slice == 0) {
#pragma unroll
        for (int k = 0; k < 4; ++k)
          for (int j = 1; j < slices; ++j) s[k][i] += red[k][j][lane];
      }
    }
    if (slice != 0) return;
  }
  if (!live) return;
  auto put = [&](const MatOut& o, int col, float v) {
    if (!o.p) return;
    const size_t at = row_offset(q, o.ld) + col;
    if (o.dtype == LAZYMAR_F32) {
      float* d = static_cast<float*>(o.p) + at;
      *d = p.accumulate ? *d + v : v;
    } else {
      bf16* d = static_cast<bf16*>(o.p) + at;
      *d = from_f<bf16>(p.accumulate ? to_f(*d) + v : v);
    }
  };
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int col = c0 + 32 * i;
    if (col >= D) continue;
    if (param) {
      float* const out[4] = {p.dpre_b, p.dpre_g, p.dpost_b, p.dpost_g};
#pragma unroll
      for (int k = 0; k < 4; ++k)
        if (out[k]) out[k][col] = p.accumulate ? out[k][col] + s[k][i] : s[k][i];
      continue;
    }
    put(p.dshift, col, s[SUM_A][i]);
    put(p.dscale, col, (p.pre_g ? p.pre_g[col] : 1.f) * s[SUM_B][i] + (p.pre_b ? p.pre_b[col] * s[SUM_A][i] : 0.f));
    put(p.dgate, col, (p.post_g ? p.post_g[col] : 1.f) * s[SUM_Q][i] + (p.post_b ? p.post_b[col] * s[SUM_P][i] : 0.f));
  }
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

bool on_eight(const Rows& r) { return !r.p || r.vec; }
bool on_eight(const MatOut& r) { return !r.p || r.vec; }

// Warps of a row, and teams of a launch: those that live on every SM at once, as far as there are rows.
int row_warps(int D) {
  const int nc = (D + kChunk - 1) / kChunk;
  return nc <= 1 ? 1 : nc <= 2 ? 2 : nc <= 4 ? 4 : nc <= 5 ? 5 : nc <= 8 ? 8 : 16;
}
Teams grad_teams(int M, int D) {
  const int wpr = row_warps(D);
  return teams_of(M, kSMs * (wpr > 8 ? 1 : wpr == 5 ? 3 : 2 * (8 / wpr)));
}

}  // namespace

size_t join_grad_workspace(int M, int D, int group) {
  if (M < 1 || D < 1 || D > kLnMaxWidth || group < 0) return 0;
  return (size_t)grad_teams(M, D).n * (group == 1 ? 4 : 12) * D * sizeof(float);
}

cudaError_t launch_join_grad(const Ctx& c, const JoinGrad& p) {
  if (p.M == 0) {  // sums over no rows; of gate, scale and shift only the row that all share is there
    if (p.accumulate) return cudaSuccess;
    return launch_pdl(join_grad_empty_kernel, dim3((unsigned)((p.D + 255) / 256)), dim3(256), 0, c.stream, p);
  }
  JoinSums need{0, 0};
  if (p.dshift.p || (p.dscale.p && p.pre_b)) need.mods |= 1u << SUM_A;
  if (p.dscale.p) need.mods |= 1u << SUM_B;
  if (p.dgate.p && p.post_b) need.mods |= 1u << SUM_P;
  if (p.dgate.p) need.mods |= 1u << SUM_Q;
  if (p.dpre_b) need.params |= 1u << SUM_A;
  if (p.dpre_g) need.params |= 1u << SUM_B;
  if (p.dpost_b) need.params |= 1u << SUM_P;
  if (p.dpost_g) need.params |= 1u << SUM_Q;
  const int wpr = row_warps(p.D), groups = p.group > 0 ? (p.M - 1) / p.group + 1 : 1;
  const Teams teams = grad_teams(p.M, p.D);
  const bool whole = p.D % 8 == 0 && on_eight(p.dh) && on_eight(p.dz) && on_eight(p.z) && on_eight(p.y) &&
                     on_eight(p.gate) && on_eight(p.scale) && on_eight(p.dx) && on_eight(p.dy) && on_eight(p.dgate) &&
                     on_eight(p.dscale) && on_eight(p.dshift) && p.params_vec;
  const cudaError_t e = p.group == 1 ? launch_join_grad_rowwise(c, p, need, whole, wpr, teams)
                                     : join_grad_launch<false>(c, p, need, whole, wpr, teams);
  if (e != cudaSuccess) return e;
  const int divided = p.group == 1 || !need.mods || teams.n == 1 ? 0 : groups < teams.n ? groups : teams.n - 1;
  if (!divided && !need.params) return cudaSuccess;
  const int slices = teams.n / groups >= 32 ? kFinishWarps : 1, each = kFinishWarps / slices;
  return launch_pdl(join_grad_finish_kernel,
                    dim3((unsigned)((p.D + 127) / 128), (unsigned)((divided + each - 1) / each + (need.params ? 1 : 0))),
                    dim3(32 * kFinishWarps), 0, c.stream, p, teams, groups, divided, p.group == 1, need, slices);
}

}  // namespace lm
