// The residual join's gradient: the kernel for rows that share a modulation (or have
// none), and what follows both kernels.
#include "join_grad.cuh"

namespace lm {

namespace {

// out (+)= v
__device__ __forceinline__ void put_one(const MatOut& o, unsigned row, int col, float v, bool accumulate) {
  const size_t at = row_offset(row, o.ld) + col;
  if (o.dtype == LAZYMAR_F32) {
    float* d = static_cast<float*>(o.p) + at;
    *d = accumulate ? *d + v : v;
  } else {
    bf16* d = static_cast<bf16*>(o.p) + at;
    *d = from_f<bf16>(accumulate ? to_f(*d) + v : v);
  }
}

// Sums over all partial rows: of the parameters, and of the modulation where all rows share one. Partial rows
// are of the CTAs where all rows share one modulation or none does, otherwise of the ranges. A CTA has 32
// columns of one result (blockIdx.y: 0..3 dpre_b, dpre_g, dpost_b, dpost_g; 4..6 dshift, dscale, dgate); each of 32
// slices adds every 32nd partial row, and the slices are added in order. Short chains of loads: it is all latency.
constexpr int kSlices = 32;

__global__ void __launch_bounds__(32 * kSlices) join_grad_sums_kernel(const __grid_constant__ JoinGrad p, int ranges, int ctas,
                                                                      int first_result) {
  __shared__ float red[2][kSlices][32];
  const int lane = threadIdx.x & 31, slice = threadIdx.x >> 5, col = blockIdx.x * 32 + lane, D = p.D;
  const int result = (int)blockIdx.y + first_result, n = ctas ? ctas : ranges;
  pdl_wait();
  pdl_trigger();
  const bool param = result < 4;
  float* const params[4] = {p.dpre_b, p.dpre_g, p.dpost_b, p.dpost_g};
  MatOut o = result == 4 ? p.dshift : result == 5 ? p.dscale : p.dgate;
  const float* const g = result == 5 ? p.pre_g : result == 6 ? p.post_g : nullptr;
  const float* const b = result == 5 ? p.pre_b : result == 6 ? p.post_b : nullptr;
  if (param) o = MatOut{params[result], 0, LAZYMAR_F32, true};
  if (!o.p) return;
  // sums of the result: k0 and, times the shift b, k1
  const int k0 = param ? result : result == 4 ? SUM_A : result == 5 ? SUM_B : SUM_Q, k1 = k0 - 1;
  float s0 = 0.f, s1 = 0.f;
  if (col < D) {
#pragma unroll 4
    for (int t = slice; t < n; t += kSlices) {
      const float* w = p.ws + ((ctas ? 0 : (size_t)ranges * 8) + (size_t)t * 4) * D;
      s0 += w[(size_t)k0 * D + col];
      if (b) s1 += w[(size_t)k1 * D + col];
    }
  }
  red[0][slice][lane] = s0;
  red[1][slice][lane] = s1;
  __syncthreads();
  if (slice != 0 || col >= D) return;
#pragma unroll
  for (int i = 1; i < kSlices; ++i) {
    s0 += red[0][i][lane];
    s1 += red[1][i][lane];
  }
  if (param && p.group == 0) {  // (the one modulation times the sums without it)
    const Rows& m = result < 2 ? p.scale : p.gate;
    if (m.p) {
      const float v = m.dtype == LAZYMAR_F32 ? static_cast<const float*>(m.p)[col] : to_f(static_cast<const bf16*>(m.p)[col]);
      s0 *= result < 2 ? 1.f + v : v;
    }
  }
  if (g) s0 *= g[col];
  if (b) s0 = fmaf(b[col], s1, s0);
  put_one(o, 0u, col, s0, p.accumulate);
}

// Sums of the groups that several neighbouring ranges share: a warp has 128 columns of one result (dshift, dscale, dgate) of
// one group, and adds every SLICES-th range's: four warps share the ranges of a group where it has four or more on average,
// 16 where it has 32 or more. Groups are counted one by one, or where there are more of them than ranges, by the ranges that begin
// inside one. All loads of a step are under way at once, without branches: 2000 x 1280 with 320 rows a group, where 22 ranges share
// one, 19 us with the gradient's kernel before it; range after range, with a branch for each sum, 49.
template <int SLICES>
__global__ void __launch_bounds__(SLICES == 1 ? 128 : 32 * SLICES)
    join_grad_groups_kernel(const __grid_constant__ JoinGrad p, const Teams teams, int groups) {
  __shared__ float red[2][SLICES][128];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, c0 = blockIdx.x * 128 + lane, D = p.D;
  const int y = SLICES == 1 ? (int)blockIdx.y * 4 + warp : (int)blockIdx.y, slice = SLICES == 1 ? 0 : warp;
  const int group = p.group, result = (int)blockIdx.z;
  pdl_wait();
  pdl_trigger();
  const MatOut o = result == 0 ? p.dshift : result == 1 ? p.dscale : p.dgate;
  const float* const g = result == 1 ? p.pre_g : result == 2 ? p.post_g : nullptr;
  const float* const b = result == 1 ? p.pre_b : result == 2 ? p.post_b : nullptr;
  const int k0 = result == 0 ? SUM_A : result == 1 ? SUM_B : SUM_Q;
  if (!o.p) return;
  int q = y;
  if (groups >= teams.n) {
    if (y + 1 >= teams.n) return;
    const int at = team_start(teams, y + 1);
    if (at % group == 0) return;
    q = at / group;
  }
  if (q >= groups) return;
  const int g0 = q * group, t0 = team_of(teams, g0), t1 = team_of(teams, g0 + min(group, p.M - g0) - 1);
  if (t0 == t1 || (groups >= teams.n && t0 != y)) return;  // done there; another task's
  int col[4];
  float s[2][4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    col[i] = min(c0 + 32 * i, D - 1);
    s[0][i] = s[1][i] = 0.f;
  }
  const auto add = [&](int k, float (&to)[4]) {
#pragma unroll 4
    for (int t = t0 + slice; t <= t1; t += SLICES) {
      // (the second place is the group's that begins inside the range)
      const float* w = p.ws + ((size_t)t * 2 + (t == t0 && g0 > team_start(teams, t0))) * 4 * D + (size_t)k * D;
#pragma unroll
      for (int i = 0; i < 4; ++i) to[i] += w[col[i]];
    }
  };
  add(k0, s[0]);
  if (b) add(k0 - 1, s[1]);
  if (SLICES > 1) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      red[0][slice][32 * i + lane] = s[0][i];
      red[1][slice][32 * i + lane] = s[1][i];
    }
    __syncthreads();
    if (slice > 0) return;
#pragma unroll
    for (int j = 1; j < SLICES; ++j)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        s[0][i] += red[0][j][32 * i + lane];
        s[1][i] += red[1][j][32 * i + lane];
      }
  }
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    if (c0 + 32 * i >= D) continue;
    float v = s[0][i];
    if (g) v *= g[col[i]];
    if (b) v = fmaf(b[col[i]], s[1][i], v);
    put_one(o, q, col[i], v, p.accumulate);
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

// Teams of a CTA, one CTA an SM.
int cta_teams(int D, int sm_warps) { return cta_warps(row_warps(D), sm_warps) / row_warps(D); }

}  // namespace

size_t join_grad_workspace(int M, int D, int group) {
  if (M < 1 || D < 1 || D > kLnMaxWidth || group < 0) return 0;
  const size_t rows = group > 1 ? 12 * (size_t)teams_of(M, kSMs * cta_teams(D, kMostGradWarps)).n : 4 * (size_t)kSMs;
  return join_sums_bytes(rows * D);
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
  const bool rowwise = p.group == 1;
  const bool plain = p.pre && !p.post && !p.post_g && !p.post_b && !p.pre_g && !p.pre_b && !need.params && p.dz.p && p.y.p &&
                     p.gate.p && p.scale.p && p.dx.p && p.dy.p;
  const int each = cta_teams(p.D, grad_sm_warps(row_warps(p.D), plain, rowwise));
  // (Joining the teams' sums costs where groups are short, and gains where few rows are divided among many ranges: 40960
  // x 1280 with 64 rows a group 153 us together, 144 apart; with 320 141 and 142, and of 320 rows 8.5 and 11.8.)
  const bool together = p.group == 0 || p.group >= kTogether;
  const int each_cta = (p.M - 1) / each + 1;  // CTAs of one row a team
  const Teams ranges = teams_of(p.M, together ? (each_cta < kSMs ? each_cta : kSMs) : kSMs * each);
  const int groups = p.group > 0 ? (p.M - 1) / p.group + 1 : 1;
  const bool whole = p.D % 8 == 0 && on_eight(p.dh) && on_eight(p.dz) && on_eight(p.z) && on_eight(p.y) &&
                     on_eight(p.gate) && on_eight(p.scale) && on_eight(p.dx) && on_eight(p.dy) && on_eight(p.dgate) &&
                     on_eight(p.dscale) && on_eight(p.dshift) && p.params_vec;
  cudaError_t e = rowwise ? (plain ? launch_join_grad_plain_rowwise(c, p, need, whole, ranges, together)
                                   : launch_join_grad_rowwise(c, p, need, whole, ranges, together))
                          : (plain ? launch_join_grad_plain(c, p, need, whole, ranges, together)
                                   : join_grad_launch<false, false>(c, p, need, whole, ranges, together));
  if (e != cudaSuccess) return e;
  // partial rows of CTAs (one group or none), otherwise of ranges
  const int ctas = p.group > 1 ? 0 : together ? ranges.n : (ranges.n + each - 1) / each;
  const bool one = p.group == 0 && need.mods;
  if (need.params || one)
    e = launch_pdl(join_grad_sums_kernel, dim3((unsigned)((p.D + 31) / 32), (one ? 7u : 4u) - (need.params ? 0u : 4u)),
                   dim3(32 * kSlices), 0, c.stream, p, ranges.n, ctas, need.params ? 0 : 4);
  if (e != cudaSuccess || ctas || !need.mods || ranges.n == 1) return e;
  const int tasks = groups < ranges.n ? groups : ranges.n - 1, shared = ranges.n / groups;
  const auto run = [&](auto kernel, int slices) {
    const int of_cta = slices == 1 ? 4 : 1;
    return launch_pdl(kernel, dim3((unsigned)((p.D + 127) / 128), (unsigned)((tasks + of_cta - 1) / of_cta), 3),
                      dim3(slices == 1 ? 128 : 32 * slices), 0, c.stream, p, ranges, groups);
  };
  return shared >= 32 ? run(join_grad_groups_kernel<16>, 16)
         : shared >= 4 ? run(join_grad_groups_kernel<4>, 4)
                       : run(join_grad_groups_kernel<1>, 1);
}

}  // namespace lm
