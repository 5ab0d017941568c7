// The residual join's gradient: the kernel for rows that share a modulation (or have
// none), and what follows both kernels.
#include "join_grad.cuh"

namespace lm {

namespace {

// The sums that several teams have part of. blockIdx.y 0: the parameters' (if there are any),
// then one for each group that may be divided. Each slice of 32 threads (up to 32 of them)
// adds every so many teams', and the slices are added in order.
constexpr int kMostSlices = 32;

__global__ void __launch_bounds__(32 * kMostSlices) join_grad_finish_kernel(const __grid_constant__ JoinGrad p, int teams, int groups,
                                                                            bool rowwise, JoinSums need, int group_slices) {
  __shared__ float red[4][kMostSlices][32];
  const int lane = threadIdx.x & 31, slice = threadIdx.x >> 5, col = blockIdx.x * 32 + lane, D = p.D;
  int y = (int)blockIdx.y;
  const bool param = need.params && y == 0;
  const int slices = param ? kMostSlices : group_slices;  // (the same sums whatever else is computed)
  if (need.params) y -= 1;
  const unsigned sums = param ? need.params : need.mods;
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
  if (slice < slices && col < D) {
    for (int t = t0 + slice; t <= t1; t += slices) {
      const float* o = param ? p.ws + (rowwise ? 0 : (size_t)teams * 8 * D) + (size_t)t * 4 * D
                             : p.ws + ((size_t)t * 2 + (g0 > team_start(p.M, teams, t))) * 4 * D;
#pragma unroll
      for (int k = 0; k < 4; ++k)
        if (sums >> k & 1u) s[k] += o[(size_t)k * D + col];
    }
  }
#pragma unroll
  for (int k = 0; k < 4; ++k) red[k][slice][lane] = s[k];
  __syncthreads();
  if (slice != 0 || col >= D) return;
#pragma unroll
  for (int k = 0; k < 4; ++k)
    for (int i = 1; i < slices; ++i) s[k] += red[k][i][lane];
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

bool on_eight(const Rows& r) { return !r.p || r.vec; }
bool on_eight(const MatOut& r) { return !r.p || r.vec; }

// Warps of a row, and teams of a launch: those that live on every SM at once, as far as there are rows.
int row_warps(int D) {
  const int nc = (D + kChunk - 1) / kChunk;
  return nc <= 1 ? 1 : nc <= 2 ? 2 : nc <= 4 ? 4 : nc <= 5 ? 5 : nc <= 8 ? 8 : 16;
}
int grad_teams(int M, int D) {
  const int wpr = row_warps(D);
  const int most = kSMs * (wpr > 8 ? 1 : wpr == 5 ? 3 : 2 * (8 / wpr));
  return M < most ? M : most;
}

}  // namespace

size_t join_grad_workspace(int M, int D, int group) {
  if (M < 1 || D < 1 || D > kLnMaxWidth || group < 0) return 0;
  return (size_t)grad_teams(M, D) * (group == 1 ? 4 : 12) * D * sizeof(float);
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
  const int wpr = row_warps(p.D), teams = grad_teams(p.M, p.D), groups = p.group > 0 ? (p.M - 1) / p.group + 1 : 1;
  const bool whole = p.D % 8 == 0 && on_eight(p.dh) && on_eight(p.dz) && on_eight(p.z) && on_eight(p.y) &&
                     on_eight(p.gate) && on_eight(p.scale) && on_eight(p.dx) && on_eight(p.dy) && on_eight(p.dgate) &&
                     on_eight(p.dscale) && on_eight(p.dshift) && p.params_vec;
  const cudaError_t e = p.group == 1 ? launch_join_grad_rowwise(c, p, need, whole, wpr, teams)
                                     : join_grad_launch<false>(c, p, need, whole, wpr, teams);
  if (e != cudaSuccess) return e;
  const int divided = p.group == 1 || !need.mods || teams == 1 ? 0 : groups < teams ? groups : teams - 1;
  if (!divided && !need.params) return cudaSuccess;
  const int group_slices = teams / groups >= 32 ? kMostSlices : 4;
  return launch_pdl(join_grad_finish_kernel, dim3((unsigned)((p.D + 31) / 32), (unsigned)(divided + (need.params ? 1 : 0))),
                    dim3(32 * (unsigned)(need.params ? kMostSlices : group_slices)), 0, c.stream, p, teams, groups, p.group == 1, need,
                    group_slices);
}

}  // namespace lm
