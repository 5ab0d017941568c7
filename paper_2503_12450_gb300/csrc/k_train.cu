// Row-wise kernels of block training: LayerNorm's forward pass with statistics
// and 8-bit outputs, its backward pass with the column sums of the gain's and
// shift's gradients, and the passes between fp32/bf16 tensors and the 8-bit
// block format (checkpoint, GELU's gradient from a checkpoint, weights).
//
// All of them are bound by HBM bandwidth, and next to it by instruction issue:
// at 6 bytes an element the memory delivers four elements a cycle and SM, which
// leaves some 30 instructions for each. So a lane takes eight consecutive columns
// (one 16- or 32-byte access a tensor, 8 bytes of E4M3) and a half warp a block of
// 128, whose maximum is a warp reduction; addresses, scales and reductions are
// spread over eight elements.
#include "block8.cuh"

namespace lm {

namespace {

constexpr int kSMs = 152;
constexpr int kChunk = 256;  // columns of a warp: two blocks
// A chunk in shared memory on its way between lanes: one float more after every 32,
// so that neither every 32nd column a lane nor eight consecutive ones meet in a bank.
constexpr int kStage = kChunk + kChunk / 32;
__device__ __forceinline__ int staged(int i) { return i + (i >> 5); }

// ---------------------------------------------------------------------------
// Eight columns of a row
// ---------------------------------------------------------------------------
// At a boundary of eight elements. (Volatile: not to be moved above the wait for
// the predecessor grid.)
__device__ __forceinline__ void ld8a(const float* p, float (&v)[8]) {
  asm volatile("ld.global.v8.f32 {%0, %1, %2, %3, %4, %5, %6, %7}, [%8];"
               : "=f"(v[0]), "=f"(v[1]), "=f"(v[2]), "=f"(v[3]), "=f"(v[4]), "=f"(v[5]), "=f"(v[6]), "=f"(v[7])
               : "l"(p));
}
__device__ __forceinline__ void bf16x8(uint4 u, float (&v)[8]) {
  const uint32_t w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    v[2 * i] = __uint_as_float(w[i] << 16);
    v[2 * i + 1] = __uint_as_float(w[i] & 0xFFFF0000u);
  }
}
__device__ __forceinline__ void ld8a(const bf16* p, float (&v)[8]) { bf16x8(*reinterpret_cast<const uint4*>(p), v); }
__device__ __forceinline__ void st8a(float* p, const float (&v)[8]) {
  asm volatile("st.global.v8.f32 [%8], {%0, %1, %2, %3, %4, %5, %6, %7};" ::"f"(v[0]), "f"(v[1]), "f"(v[2]), "f"(v[3]),
               "f"(v[4]), "f"(v[5]), "f"(v[6]), "f"(v[7]), "l"(p)
               : "memory");
}
__device__ __forceinline__ void st8a(bf16* p, const float (&v)[8]) {
  *reinterpret_cast<uint4*>(p) =
      make_uint4(pack_bf16(v[0], v[1]), pack_bf16(v[2], v[3]), pack_bf16(v[4], v[5]), pack_bf16(v[6], v[7]));
}
// A warp's 256 columns from c0 on, eight consecutive ones a lane; columns from D on
// read as zero and are not written. Rows off the boundary are loaded with every 32nd
// column a lane (ld8s), so that the accesses of a warp stay contiguous, and turned
// through the warp's kStage floats of shared memory. That is a step of its own
// (turn8), and the elements are widened there, so that all loads are under way
// before the first is waited for. Every lane of the warp takes part.
template <typename T>
__device__ __forceinline__ void ld8(const T* row, int c0, int D, float (&v)[8]) {
  const int col = c0 + 8 * (int)(threadIdx.x & 31);
  if (col + 8 <= D) {
    ld8a(row + col, v);
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = col + i < D ? to_f(row[col + i]) : 0.f;
  }
}
__device__ __forceinline__ void ld8s(const Mat& m, size_t row, int c0, int D, uint32_t (&v)[8]) {
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const int c = c0 + 32 * i + (int)(threadIdx.x & 31);
    v[i] = 0u;
    if (c < D)
      v[i] = m.dtype == LAZYMAR_F32 ? static_cast<const uint32_t*>(m.p)[row * m.ld + c]
                                    : static_cast<const uint16_t*>(m.p)[row * m.ld + c];
  }
}
// Every 32nd column a lane, as loaded, to eight consecutive ones.
__device__ __forceinline__ void turn8(float* sm, const uint32_t (&raw)[8], int shift, float (&v)[8]) {
  const int lane = threadIdx.x & 31;
  __syncwarp();
#pragma unroll
  for (int i = 0; i < 8; ++i) sm[33 * i + lane] = __uint_as_float(raw[i] << shift);
  __syncwarp();
#pragma unroll
  for (int i = 0; i < 8; ++i) v[i] = sm[staged(8 * lane) + i];
}
template <typename T>
__device__ __forceinline__ void st8(T* row, int c0, int D, bool vec, float* sm, const float (&v)[8]) {
  const int lane = threadIdx.x & 31, col = c0 + 8 * lane;
  if (vec) {
    if (col + 8 <= D) {
      st8a(row + col, v);
    } else {
#pragma unroll
      for (int i = 0; i < 8; ++i)
        if (col + i < D) row[col + i] = from_f<T>(v[i]);
    }
    return;
  }
  __syncwarp();
#pragma unroll
  for (int i = 0; i < 8; ++i) sm[staged(8 * lane) + i] = v[i];
  __syncwarp();
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const int c = c0 + 32 * i + lane;
    if (c < D) row[c] = from_f<T>(sm[33 * i + lane]);
  }
}
// FULL: every column exists and the row is on the boundary.
template <bool FULL>
__device__ __forceinline__ void ld_mat(const Mat& m, size_t row, int c0, int D, float (&v)[8]) {
  if (m.dtype == LAZYMAR_F32) {
    const float* r = static_cast<const float*>(m.p) + row * m.ld;
    if (FULL) ld8a(r + c0 + 8 * (threadIdx.x & 31), v);
    else ld8<float>(r, c0, D, v);
  } else {
    const bf16* r = static_cast<const bf16*>(m.p) + row * m.ld;
    if (FULL) ld8a(r + c0 + 8 * (threadIdx.x & 31), v);
    else ld8<bf16>(r, c0, D, v);
  }
}
template <bool FULL>
__device__ __forceinline__ void st_mat(const MatOut& m, size_t row, int c0, int D, float* sm, const float (&v)[8]) {
  if (m.dtype == LAZYMAR_F32) {
    float* r = static_cast<float*>(m.p) + row * m.ld;
    if (FULL) st8a(r + c0 + 8 * (threadIdx.x & 31), v);
    else st8<float>(r, c0, D, m.vec, sm, v);
  } else {
    bf16* r = static_cast<bf16*>(m.p) + row * m.ld;
    if (FULL) st8a(r + c0 + 8 * (threadIdx.x & 31), v);
    else st8<bf16>(r, c0, D, m.vec, sm, v);
  }
}
// fp32 parameters of eight columns; vec: on a boundary of eight. (One access a lane:
// eight scalar ones, 32 bytes from lane to lane, are eight cache lines each, and were
// two thirds of the time at 40000 x 1013 fp32.)
template <bool FULL>
__device__ __forceinline__ void ld_param(const float* p, bool vec, int col, int D, float (&v)[8]) {
  if (FULL || (vec && col + 8 <= D)) {
    ld8a(p + col, v);
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = col + i < D ? p[col + i] : 0.f;
  }
}
// Eight E4M3 bytes of a block8 row. Rows are 16-byte aligned and padded to 16
// bytes, so the bytes are readable where the first of them exists; those of
// columns that do not exist are cleared.
__device__ __forceinline__ uint2 clear_beyond(uint2 w, int n) {  // keeps the first n bytes
  if (n < 4) return make_uint2(n <= 0 ? 0u : w.x & (0xFFFFFFFFu >> (32 - 8 * n)), 0u);
  return make_uint2(w.x, n == 4 ? 0u : n < 8 ? w.y & (0xFFFFFFFFu >> (64 - 8 * n)) : w.y);
}
__device__ __forceinline__ uint2 ldq8(const uint8_t* row, int col, int D) {
  if (col >= D) return make_uint2(0u, 0u);
  const uint2 w = *reinterpret_cast<const uint2*>(row + col);
  return col + 8 <= D ? w : clear_beyond(w, D - col);
}
__device__ __forceinline__ void stq8(uint8_t* row, int col, int D, uint2 w) {
  if (col + 8 <= D) {
    *reinterpret_cast<uint2*>(row + col) = w;
  } else {
    for (int i = 0; col + i < D; ++i) row[col + i] = (uint8_t)((i < 4 ? w.x : w.y) >> (8 * (i & 3)));
  }
}
// A warp's 256 columns (two blocks) of row `row` to block8.
template <bool FULL>
__device__ __forceinline__ void put8(const lazymar_block8& o, size_t row, int c0, int D, const float (&v)[8]) {
  const int lane = threadIdx.x & 31, col = c0 + 8 * lane;
  uint2 w;
  const uint32_t byte = block8_quantize(v, w);
  uint8_t* q = static_cast<uint8_t*>(o.q) + row * o.ldq;
  if (FULL) *reinterpret_cast<uint2*>(q + col) = w;
  else stq8(q, col, D, w);
  if ((lane & 15) == 0 && (FULL || col < D)) o.scale[(size_t)(col / kBlk) * o.lds + row] = (uint8_t)byte;
}
template <bool FULL>
__device__ __forceinline__ void mask8(float (&v)[8], int col, int D) {
  if (FULL || col + 8 <= D) return;
#pragma unroll
  for (int i = 0; i < 8; ++i)
    if (col + i >= D) v[i] = 0.f;
}
__device__ __forceinline__ float sum8(const float (&v)[8]) {
  const unsigned long long s =
      f32x2_add(f32x2_add(f32x2_pack(v[0], v[1]), f32x2_pack(v[2], v[3])), f32x2_add(f32x2_pack(v[4], v[5]), f32x2_pack(v[6], v[7])));
  float a, b;
  f32x2_unpack(s, a, b);
  return a + b;
}

// Eight values with paired fp32 instructions: v - m; v * s; v * a + b; sum of squares.
__device__ __forceinline__ void sub8(float (&v)[8], float m) {
  const unsigned long long mm = f32x2_pack(-m, -m);
#pragma unroll
  for (int i = 0; i < 8; i += 2) f32x2_unpack(f32x2_add(f32x2_pack(v[i], v[i + 1]), mm), v[i], v[i + 1]);
}
__device__ __forceinline__ void scale8(const float (&v)[8], float s, float (&y)[8]) {
  const unsigned long long ss = f32x2_pack(s, s);
#pragma unroll
  for (int i = 0; i < 8; i += 2) f32x2_unpack(f32x2_mul(f32x2_pack(v[i], v[i + 1]), ss), y[i], y[i + 1]);
}
__device__ __forceinline__ void mul8(float (&y)[8], const float (&a)[8]) {
#pragma unroll
  for (int i = 0; i < 8; i += 2)
    f32x2_unpack(f32x2_mul(f32x2_pack(y[i], y[i + 1]), f32x2_pack(a[i], a[i + 1])), y[i], y[i + 1]);
}
__device__ __forceinline__ void add8(float (&y)[8], const float (&a)[8]) {
#pragma unroll
  for (int i = 0; i < 8; i += 2)
    f32x2_unpack(f32x2_add(f32x2_pack(y[i], y[i + 1]), f32x2_pack(a[i], a[i + 1])), y[i], y[i + 1]);
}
__device__ __forceinline__ float squares8(const float (&v)[8]) {
  unsigned long long q = f32x2_mul(f32x2_pack(v[0], v[1]), f32x2_pack(v[0], v[1]));
#pragma unroll
  for (int i = 2; i < 8; i += 2) q = f32x2_fma(f32x2_pack(v[i], v[i + 1]), f32x2_pack(v[i], v[i + 1]), q);
  float a, b;
  f32x2_unpack(q, a, b);
  return a + b;
}

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
// WPR warps a row, NC chunks of 256 columns a warp, the row in registers: one
// read of x, mean and then the squared deviations from it (no cancellation).
// FULL: D = 256 NC WPR and aligned rows, so that no column needs a check.
// 40960 x 1024 fp32 with statistics, 8-bit output and 8-bit copy of the input: 43.7
// us, 5.8 TB/s (floor 37 at 6.8); without paired instructions 47, four columns a lane 67.
// 40000 x 1013, off the boundary: 76 (floor 36); with a wait for each chunk 99.
template <int NC, int WPR, bool FULL>
__global__ void __launch_bounds__(256, 4) ln_forward_kernel(const LnForward p) {
  constexpr int GROUPS = 8 / WPR;
  __shared__ float red[2][GROUPS][WPR];
  __shared__ float stage[FULL ? 1 : 8][kStage];
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, grp = warp / WPR, part = warp % WPR;
  float* sm = stage[FULL ? 0 : warp];
  const int D = p.D, row = blockIdx.x * GROUPS + grp, c0 = part * NC * kChunk;
  const bool live = row < p.M;
  pdl_wait();
  pdl_trigger();
  float v[NC][8];
  float s = 0.f;
  if (live) {
#pragma unroll
    for (int c = 0; c < NC; ++c) {
      if (FULL || p.x.vec) ld_mat<FULL>(p.x, row, c0 + c * kChunk, D, v[c]);
    }
    if (!FULL && !p.x.vec) {
      const int shift = p.x.dtype == LAZYMAR_F32 ? 0 : 16;
      uint32_t raw[NC][8];
#pragma unroll
      for (int c = 0; c < NC; ++c) ld8s(p.x, row, c0 + c * kChunk, D, raw[c]);
#pragma unroll
      for (int c = 0; c < NC; ++c) turn8(sm, raw[c], shift, v[c]);
    }
#pragma unroll
    for (int c = 0; c < NC; ++c) s += sum8(v[c]);
  }
  const float mean = row_sum<WPR>(s, red[0][grp], part) / (float)D;
  float q = 0.f;
  if (live) {
#pragma unroll
    for (int c = 0; c < NC; ++c) {
      if (p.x8.q && (FULL || c0 + c * kChunk < D)) put8<FULL>(p.x8, row, c0 + c * kChunk, D, v[c]);
      sub8(v[c], mean);
      mask8<FULL>(v[c], c0 + c * kChunk + 8 * lane, D);
      q += squares8(v[c]);
    }
  }
  const float rstd = rsqrtf(row_sum<WPR>(q, red[1][grp], part) / (float)D + p.eps);
  if (!live) return;
  if (part == 0 && lane == 0) {
    if (p.mean) p.mean[row] = mean;
    if (p.rstd) p.rstd[row] = rstd;
  }
  if (!p.y.p && !p.y8.q) return;
#pragma unroll
  for (int c = 0; c < NC; ++c) {
    const int cc = c0 + c * kChunk, col = cc + 8 * lane;
    if (!FULL && cc >= D) break;  // (uniform over the warp)
    float y[8], t[8];
    scale8(v[c], rstd, y);
    if (p.g) {
      ld_param<FULL>(p.g, p.params_vec, col, D, t);
      mul8(y, t);
    }
    if (p.b) {
      ld_param<FULL>(p.b, p.params_vec, col, D, t);
      add8(y, t);
    }
    mask8<FULL>(y, col, D);
    if (p.y8.q) put8<FULL>(p.y8, row, cc, D, y);
    if (p.y.p) st_mat<FULL>(p.y, row, cc, D, sm, y);
  }
}

template <int NC, int WPR>
cudaError_t ln_forward_run(const Ctx& c, const LnForward& p) {
  constexpr int GROUPS = 8 / WPR;
  const dim3 grid((unsigned)((p.M + GROUPS - 1) / GROUPS)), block(256);
  if (p.x.vec && p.y.vec && p.params_vec && p.D == NC * WPR * kChunk)
    return launch_pdl(ln_forward_kernel<NC, WPR, true>, grid, block, 0, c.stream, p);
  return launch_pdl(ln_forward_kernel<NC, WPR, false>, grid, block, 0, c.stream, p);
}

// ---------------------------------------------------------------------------
// Column sums of per-CTA partial rows
// ---------------------------------------------------------------------------
// out[c] (+)= sum over the P rows of part [P, n], in row order within each of
// kSlices slices and slice order after that: the same result for the same sizes.
// Columns from n1 on belong to out2. Short chains of loads, because a launch
// over the few hundred partial rows is all latency (304 rows of 1554: 8 slices
// 9.3 us cold).
constexpr int kSlices = 32;

__global__ void __launch_bounds__(32 * kSlices) column_sums_kernel(const float* __restrict__ part, int P, int n, int n1,
                                                          float* __restrict__ out, float* __restrict__ out2,
                                                          bool accumulate) {
  __shared__ float red[kSlices][32];
  const int lane = threadIdx.x & 31, slice = threadIdx.x >> 5, col = blockIdx.x * 32 + lane;
  pdl_wait();
  pdl_trigger();
  float s = 0.f;
  if (col < n) {
    const float* p = part + col;
#pragma unroll 8
    for (int r = slice; r < P; r += kSlices) s += p[(size_t)r * n];
  }
  red[slice][lane] = s;
  __syncthreads();
  if (slice == 0 && col < n) {
#pragma unroll
    for (int i = 1; i < kSlices; ++i) s += red[i][lane];
    float* o = col < n1 ? out + col : out2 + (col - n1);
    if (accumulate) s += *o;
    *o = s;
  }
}

cudaError_t column_sums(const Ctx& c, const float* part, int P, int n, int n1, float* out, float* out2,
                        bool accumulate) {
  return launch_pdl(column_sums_kernel, dim3((unsigned)((n + 31) / 32)), dim3(32 * kSlices), 0, c.stream, part, P, n, n1, out,
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

constexpr int kRing = 4;  // most rows of a warp's ring

// Widths that are a multiple of eight up to 4096 with rows on boundaries: WPR
// warps a row, NB blocks of 128 columns a warp, four consecutive columns of a
// block a lane. The rows of dy, x and dres come by bulk copies into the warp's
// ring in shared memory, so that the next rows are on their way while this one
// is worked on and nothing of them waits in registers. 40960 x 1280 from an 8-bit
// checkpoint, bf16 dy, fp32 residual and dx: 109 us, 5.3 TB/s (floor 85); with the
// row in the registers of two warps and nothing ahead 203 us, one warp a row 158.
template <int NB, int WPR>
__global__ void __launch_bounds__(256, 2) ln_backward_ring_kernel(const LnBackward p, int depth, uint32_t row_bytes,
                                                                  uint32_t x_at, uint32_t r_at, unsigned* err) {
  extern __shared__ __align__(128) uint8_t ring_smem[];  // [warps][depth][row_bytes]
  __shared__ uint64_t bars[8][kRing];
  __shared__ float red[2][8 / WPR][2][WPR];
  __shared__ int abort_word;
  volatile int* abort_flag = &abort_word;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, grp = warp / WPR, part = warp % WPR;
  const int groups = (int)(blockDim.x >> 5) / WPR, D = p.D, c0 = part * NB * kBlk;
  const int mine = max(0, min(NB * kBlk, D - c0));  // columns of this warp; the last ones of eight may have none
  uint8_t* ring = ring_smem + (size_t)warp * depth * row_bytes;
  if (threadIdx.x == 0) abort_word = 0;
  if (lane == 0)
    for (int s = 0; s < depth; ++s) mbar_init(&bars[warp][s], 1);
  fence_mbar_init();
  pdl_wait();
  pdl_trigger();
  __syncthreads();
  const int step = (int)gridDim.x * groups, first = (int)blockIdx.x * groups + grp;
  const size_t dy_e = p.dy.dtype == LAZYMAR_F32 ? 4 : 2, x_e = p.x.dtype == LAZYMAR_F32 ? 4 : 2;
  const uint32_t dy_b = (uint32_t)(mine * dy_e);
  const uint32_t x_b = p.x.p ? (uint32_t)(mine * x_e) : (uint32_t)((mine + 15) & ~15);
  const uint32_t r_b = p.dres.p ? (uint32_t)mine * 4 : 0u;
  auto fetch = [&](long long row, int s) {
    uint8_t* dst = ring + (size_t)s * row_bytes;
    uint64_t* bar = &bars[warp][s];
    mbar_arrive_expect_tx(bar, dy_b + x_b + r_b);
    bulk_load(dst, static_cast<const uint8_t*>(p.dy.p) + ((size_t)row * p.dy.ld + c0) * dy_e, dy_b, bar);
    bulk_load(dst + x_at,
              p.x.p ? static_cast<const uint8_t*>(p.x.p) + ((size_t)row * p.x.ld + c0) * x_e
                    : static_cast<const uint8_t*>(p.x8.q) + (size_t)row * p.x8.ldq + c0,
              x_b, bar);
    if (r_b) bulk_load(dst + r_at, static_cast<const float*>(p.dres.p) + (size_t)row * p.dres.ld + c0, r_b, bar);
  };
  if (lane == 0 && mine > 0)
    for (int s = 0; s < depth; ++s)
      if (first + (long long)s * step < p.M) fetch(first + (long long)s * step, s);
  // mean, rstd and the scales (lane: block) of the next row
  float mean = 0.f, rstd = 0.f;
  uint32_t sb = 0;
  auto statistics = [&](long long row) {
    if (row >= p.M) return;
    mean = p.mean[row];
    rstd = p.rstd[row];
    if (!p.x.p && lane < NB && lane * kBlk < mine) sb = p.x8.scale[(size_t)(part * NB + lane) * p.x8.lds + row];
  };
  statistics(first);
  float g[NB][4], dg[NB][4], db[NB][4];
#pragma unroll
  for (int j = 0; j < NB; ++j)
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int c = j * kBlk + 4 * lane + i;
      g[j][i] = c < mine ? (p.g ? p.g[c0 + c] : 1.f) : 0.f;
      dg[j][i] = db[j][i] = 0.f;
    }
  int slot = 0, it = 0;
  uint32_t phase = 0;
  bool dead = false;  // a wait ran out: the rows are not written any more
  for (long long row = first; row < p.M; row += step, it ^= 1) {
    const float mu = mean, rs = rstd;
    const uint32_t scales = sb;
    statistics(row + step);
    // (once a wait has run out, no more: they would take 64 ms for each row that is left)
    const bool ok = mine == 0 || dead || mbar_wait(&bars[warp][slot], phase, abort_flag, err);
    dead |= !__all_sync(0xffffffffu, ok);
    const uint8_t* src = ring + (size_t)slot * row_bytes;
    float y[NB][4], h[NB][4], s1 = 0.f, s2 = 0.f;
#pragma unroll
    for (int j = 0; j < NB; ++j) {
      const int c = j * kBlk + 4 * lane;
      if (p.dy.dtype == LAZYMAR_F32) {
        const float4 a = *reinterpret_cast<const float4*>(src + 4 * c);
        y[j][0] = a.x; y[j][1] = a.y; y[j][2] = a.z; y[j][3] = a.w;
      } else {
        const uint2 a = *reinterpret_cast<const uint2*>(src + 2 * c);
        y[j][0] = __uint_as_float(a.x << 16); y[j][1] = __uint_as_float(a.x & 0xFFFF0000u);
        y[j][2] = __uint_as_float(a.y << 16); y[j][3] = __uint_as_float(a.y & 0xFFFF0000u);
      }
      if (!p.x.p) {
        const uint32_t w = *reinterpret_cast<const uint32_t*>(src + x_at + c);
        const float s = block8_scale(__shfl_sync(0xffffffffu, scales, j));
        const float2 a = e4m3x2_to_f2(w & 0xFFFFu), b = e4m3x2_to_f2(w >> 16);
        h[j][0] = a.x * s; h[j][1] = a.y * s; h[j][2] = b.x * s; h[j][3] = b.y * s;
      } else if (p.x.dtype == LAZYMAR_F32) {
        const float4 a = *reinterpret_cast<const float4*>(src + x_at + 4 * c);
        h[j][0] = a.x; h[j][1] = a.y; h[j][2] = a.z; h[j][3] = a.w;
      } else {
        const uint2 a = *reinterpret_cast<const uint2*>(src + x_at + 2 * c);
        h[j][0] = __uint_as_float(a.x << 16); h[j][1] = __uint_as_float(a.x & 0xFFFF0000u);
        h[j][2] = __uint_as_float(a.y << 16); h[j][3] = __uint_as_float(a.y & 0xFFFF0000u);
      }
      if (c >= mine) {  // what a shorter row leaves of the ring's last columns
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          y[j][i] = 0.f;
          h[j][i] = mu;
        }
      }
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        h[j][i] = (h[j][i] - mu) * rs;
        dg[j][i] = fmaf(y[j][i], h[j][i], dg[j][i]);
        db[j][i] += y[j][i];
        y[j][i] *= g[j][i];
        s1 += y[j][i];
        s2 = fmaf(y[j][i], h[j][i], s2);
      }
    }
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) {
      s1 += __shfl_xor_sync(0xffffffffu, s1, o);
      s2 += __shfl_xor_sync(0xffffffffu, s2, o);
    }
    if constexpr (WPR > 1) {
      if (lane == 0) {
        red[it][grp][0][part] = s1;
        red[it][grp][1][part] = s2;
      }
      asm volatile("bar.sync %0, %1;" ::"r"(grp + 1), "n"(WPR * 32) : "memory");  // the row's warps
      s1 = s2 = 0.f;
#pragma unroll
      for (int i = 0; i < WPR; ++i) {
        s1 += red[it][grp][0][i];
        s2 += red[it][grp][1][i];
      }
    }
    s1 /= (float)D;
    s2 /= (float)D;
#pragma unroll
    for (int j = 0; j < NB; ++j) {
      const int c = j * kBlk + 4 * lane;
      if (c >= mine) continue;
#pragma unroll
      for (int i = 0; i < 4; ++i) y[j][i] = rs * (y[j][i] - s1 - h[j][i] * s2);
      if (r_b) {
        const float4 r = *reinterpret_cast<const float4*>(src + r_at + 4 * c);
        y[j][0] += r.x; y[j][1] += r.y; y[j][2] += r.z; y[j][3] += r.w;
      }
      if (dead) continue;
      if (p.dx.dtype == LAZYMAR_F32)
        *reinterpret_cast<float4*>(static_cast<float*>(p.dx.p) + (size_t)row * p.dx.ld + c0 + c) =
            make_float4(y[j][0], y[j][1], y[j][2], y[j][3]);
      else
        *reinterpret_cast<uint2*>(static_cast<bf16*>(p.dx.p) + (size_t)row * p.dx.ld + c0 + c) =
            make_uint2(pack_bf16(y[j][0], y[j][1]), pack_bf16(y[j][2], y[j][3]));
    }
    __syncwarp();  // every lane has read the row
    if (lane == 0 && mine > 0 && !dead && row + (long long)depth * step < p.M) {
      fence_proxy_async_smem();
      fetch(row + (long long)depth * step, slot);
    }
    if (++slot == depth) { slot = 0; phase ^= 1u; }
  }
  if (!p.dg) return;
  // the groups' sums in turn, where the ring was, to the CTA's row of the workspace
  constexpr int W = NB * WPR * kBlk;
  float* cols = reinterpret_cast<float*>(ring_smem);
  for (int k = 0; k < groups; ++k) {
    __syncthreads();
    if (k == grp) {
#pragma unroll
      for (int j = 0; j < NB; ++j) {
        float4* s = reinterpret_cast<float4*>(cols + c0 + j * kBlk + 4 * lane);
        float4* t = reinterpret_cast<float4*>(cols + W + c0 + j * kBlk + 4 * lane);
        const float4 u = k ? *s : make_float4(0.f, 0.f, 0.f, 0.f), w = k ? *t : make_float4(0.f, 0.f, 0.f, 0.f);
        *s = make_float4(u.x + dg[j][0], u.y + dg[j][1], u.z + dg[j][2], u.w + dg[j][3]);
        *t = make_float4(w.x + db[j][0], w.y + db[j][1], w.z + db[j][2], w.w + db[j][3]);
      }
    }
  }
  __syncthreads();
  float* o = p.ws + (size_t)blockIdx.x * 2 * D;
  for (int i = threadIdx.x; i < 2 * D; i += blockDim.x) o[i] = i < D ? cols[i] : cols[W + i - D];
}

// Any width, stride and alignment: WPR warps a row, NC chunks of 256 columns a
// warp, every 32nd column of a chunk a lane (so that a warp's accesses are
// contiguous without a boundary), dy and x in registers, the next row's on their
// way. Up to 4096 columns one chunk a warp, so that nothing spills and the gains stay
// in registers. Only a row's own warps wait for each other. Measured (us, in
// brackets with two chunks a warp, all of a CTA waiting, and the residual loaded where it
// is added): 4801 x 777 bf16 13.3 (16.8; floor 3.3), 36071 x 1254 94 (174; floor 67), 20000
// x 777 from 8 bits with residual 45 (188; floor 21), x 1601 the same 87 (183; floor 52), 20000 x
// 1013 fp32 47 (62; floor 36), 5000 x 4001 bf16 44 (54; floor 18).
// (The elements are widened at their use: the next row is under way in registers
// while this one is worked on, and a use would wait for it.)
// Warps of a CTA and CTAs on an SM, so that a thread has 128 registers (ten warps with
// 96 each spill: 185 us at 36071 x 1254 instead of 107).
template <int WPR>
constexpr int kLnWarps = WPR > 8 ? 16 : WPR == 5 ? 5 : 8;
template <int WPR>
constexpr int kLnCtas = WPR > 8 ? 1 : WPR == 5 ? 3 : 2;

template <int NC, int WPR>
__global__ void __launch_bounds__(kLnWarps<WPR> * 32, kLnCtas<WPR>) ln_backward_kernel(const LnBackward p) {
  constexpr int GROUPS = kLnWarps<WPR> / WPR, W = NC * WPR * kChunk;
  extern __shared__ float cols[];  // [2][W]
  __shared__ float red[2][2][GROUPS][WPR];
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, grp = warp / WPR, part = warp % WPR;
  const int D = p.D, c0 = part * NC * kChunk;
  const int dy_shift = p.dy.dtype == LAZYMAR_F32 ? 0 : 16, x_shift = p.x.dtype == LAZYMAR_F32 ? 0 : 16;
  pdl_wait();
  pdl_trigger();
  float dg[NC][8], db[NC][8];
#pragma unroll
  for (int c = 0; c < NC; ++c)
#pragma unroll
    for (int i = 0; i < 8; ++i) dg[c][i] = db[c][i] = 0.f;
  float g[NC == 1 ? 8 : 1];
  if constexpr (NC == 1) {
#pragma unroll
    for (int i = 0; i < 8; ++i) g[i] = p.g && c0 + 32 * i + lane < D ? p.g[c0 + 32 * i + lane] : 1.f;
  }
  const int step = (int)gridDim.x * GROUPS;
  const long long first = (long long)blockIdx.x * GROUPS + grp;
  uint32_t ry[NC][8], rx[NC][8], rs[NC][2];
  float rmean = 0.f, rrstd = 0.f;
  auto fetch = [&](long long row) {
    if (row >= p.M) return;
    rmean = p.mean[row];
    rrstd = p.rstd[row];
#pragma unroll
    for (int c = 0; c < NC; ++c) {
      const int cc = c0 + c * kChunk;
      ld8s(p.dy, (size_t)row, cc, D, ry[c]);
      if (p.x.p) {
        ld8s(p.x, (size_t)row, cc, D, rx[c]);
      } else {
        const uint8_t* q = static_cast<const uint8_t*>(p.x8.q) + (size_t)row * p.x8.ldq;
        const int blk = min(cc, D - 1) / kBlk, more = cc + kBlk < D ? 1 : 0;  // the chunk's blocks
        rs[c][0] = p.x8.scale[(size_t)blk * p.x8.lds + row];
        rs[c][1] = p.x8.scale[(size_t)(blk + more) * p.x8.lds + row];
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          const int k = cc + 32 * i + lane;
          rx[c][i] = k < D ? q[k] : 0u;
        }
      }
    }
  };
  int it = 0;
  fetch(first);
  for (long long row = first; row < p.M; row += step, it ^= 1) {
    float h[NC][8], a[NC][8], s1 = 0.f, s2 = 0.f;
    const float mean = rmean, rstd = rrstd;
#pragma unroll
    for (int c = 0; c < NC; ++c) {
      const float sc[2] = {block8_scale(rs[c][0]), block8_scale(rs[c][1])};
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        a[c][i] = __uint_as_float(ry[c][i] << dy_shift);
        h[c][i] = p.x.p ? __uint_as_float(rx[c][i] << x_shift) : e4m3x2_to_f2(rx[c][i]).x * sc[i >> 2];
      }
    }
    fetch(row + step);
    // the residual's row: all of it under way before the first is added (dx's stores
    // would wait for each), with one chunk a warp already during the sums
    float r[NC][8];
    auto residual = [&] {
#pragma unroll
      for (int c = 0; c < NC; ++c)
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          const int k = c0 + c * kChunk + 32 * i + lane;
          r[c][i] = k < D ? static_cast<const float*>(p.dres.p)[(size_t)row * p.dres.ld + k] : 0.f;
        }
    };
    if (NC == 1 && p.dres.p) residual();
#pragma unroll
    for (int c = 0; c < NC; ++c) {
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const int k = c0 + c * kChunk + 32 * i + lane;
        const float x = k < D ? (h[c][i] - mean) * rstd : 0.f;
        const float gain = NC == 1 ? g[i & (NC == 1 ? 7 : 0)] : p.g && k < D ? p.g[k] : 1.f;
        h[c][i] = x;
        dg[c][i] = fmaf(a[c][i], x, dg[c][i]);
        db[c][i] += a[c][i];
        a[c][i] *= gain;
        s1 += a[c][i];
        s2 = fmaf(a[c][i], x, s2);
      }
    }
    s1 = warp_sum(s1);
    s2 = warp_sum(s2);
    if constexpr (WPR > 1) {
      if (lane == 0) {
        red[it][0][grp][part] = s1;
        red[it][1][grp][part] = s2;
      }
      asm volatile("bar.sync %0, %1;" ::"r"(grp + 1), "n"(WPR * 32) : "memory");  // the row's warps
      s1 = s2 = 0.f;
#pragma unroll
      for (int i = 0; i < WPR; ++i) {
        s1 += red[it][0][grp][i];
        s2 += red[it][1][grp][i];
      }
    }
    s1 /= (float)D;
    s2 /= (float)D;
#pragma unroll
    for (int c = 0; c < NC; ++c)
#pragma unroll
      for (int i = 0; i < 8; ++i) a[c][i] = rstd * (a[c][i] - s1 - h[c][i] * s2);
    if (p.dres.p) {
      if (NC > 1) residual();
#pragma unroll
      for (int c = 0; c < NC; ++c)
#pragma unroll
        for (int i = 0; i < 8; ++i) a[c][i] += r[c][i];
    }
#pragma unroll
    for (int c = 0; c < NC; ++c) {
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const int k = c0 + c * kChunk + 32 * i + lane;
        if (k >= D) continue;
        const float o = a[c][i];
        if (p.dx.dtype == LAZYMAR_F32) static_cast<float*>(p.dx.p)[(size_t)row * p.dx.ld + k] = o;
        else static_cast<bf16*>(p.dx.p)[(size_t)row * p.dx.ld + k] = from_f<bf16>(o);
      }
    }
  }
  if (!p.dg) return;
  // the groups' sums in turn, to the CTA's row of the workspace
  for (int n = 0; n < GROUPS; ++n) {
    __syncthreads();
    if (n == grp) {
#pragma unroll
      for (int c = 0; c < NC; ++c)
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          float* s = cols + c0 + c * kChunk + 32 * i + lane;
          s[0] = n ? s[0] + dg[c][i] : dg[c][i];
          s[W] = n ? s[W] + db[c][i] : db[c][i];
        }
    }
  }
  __syncthreads();
  float* o = p.ws + (size_t)blockIdx.x * 2 * D;
  for (int i = threadIdx.x; i < 2 * D; i += blockDim.x) o[i] = i < D ? cols[i] : cols[W + i - D];
}

// CTAs of a backward launch: the resident ones of every SM (three at most), as far as there are rows.
int ln_backward_ctas(int M, int groups, int per_sm) {
  const int need = (M - 1) / groups + 1, most = per_sm * kSMs;
  return need < most ? need : most;
}

// Lets a kernel have up to `most` bytes of dynamic shared memory, the same at every call.
// (The 48 KB that need no leave count a kernel's static shared memory too.)
cudaError_t big_smem(const void* kernel, size_t most) {
  return most > 32 * 1024 ? cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)most)
                          : cudaSuccess;
}
constexpr int kRingBytes = 220 * 1024;  // most of a CTA

// Rows in shared memory: as many a warp as let two CTAs of eight warps live on
// an SM with two rows a warp at least, otherwise one CTA.
template <int NB, int WPR>
cudaError_t ln_backward_ring_run(const Ctx& c, const LnBackward& p, int* ctas) {
  constexpr uint32_t W = NB * kBlk;
  const uint32_t dy_b = W * (p.dy.dtype == LAZYMAR_F32 ? 4 : 2);
  const uint32_t x_b = W * (p.x.p ? (p.x.dtype == LAZYMAR_F32 ? 4 : 2) : 1);
  const uint32_t r_b = p.dres.p ? W * 4 : 0u, row_b = dy_b + x_b + r_b;
  int warps = 8, per_sm = 2, depth = (int)(110 * 1024 / (warps * row_b));
  if (depth < 2) {
    per_sm = 1;
    depth = (int)(kRingBytes / (warps * row_b));
  }
  if (depth > kRing) depth = kRing;
  size_t smem = (size_t)warps * depth * row_b;
  const size_t sums = (size_t)2 * W * WPR * 4;
  if (smem < sums) smem = sums;
  *ctas = ln_backward_ctas(p.M, warps / WPR, per_sm);
  const auto kernel = ln_backward_ring_kernel<NB, WPR>;
  cudaError_t e = big_smem(reinterpret_cast<const void*>(kernel), kRingBytes);
  if (e != cudaSuccess) return e;
  return launch_pdl(kernel, dim3((unsigned)*ctas), dim3((unsigned)warps * 32), smem, c.stream, p, depth, row_b, dy_b,
                    dy_b + x_b, c.err);
}

template <int NC, int WPR>
cudaError_t ln_backward_run(const Ctx& c, const LnBackward& p, int* ctas) {
  constexpr int WARPS = kLnWarps<WPR>;
  constexpr size_t smem = (size_t)2 * NC * WPR * kChunk * sizeof(float);
  *ctas = ln_backward_ctas(p.M, WARPS / WPR, kLnCtas<WPR>);
  cudaError_t e = big_smem(reinterpret_cast<const void*>(ln_backward_kernel<NC, WPR>), smem);
  if (e != cudaSuccess) return e;
  return launch_pdl(ln_backward_kernel<NC, WPR>, dim3((unsigned)*ctas), dim3(WARPS * 32), smem, c.stream, p);
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
constexpr int kGradLo = (127 - 26) << 3, kGradN = ((127 + 4) << 3) - kGradLo + 1, kGradNeg = 256;
constexpr int kGradSize = kGradNeg + kGradN;

__device__ __forceinline__ void gelu_grad_table(float* tab) {
  for (int i = threadIdx.x; i < kGradSize; i += blockDim.x) {
    const int j = i & (kGradNeg - 1);
    if (j >= kGradN) continue;
    const float a = __uint_as_float((uint32_t)(kGradLo + j) << 20), x = i < kGradNeg ? a : -a;
    tab[i] = fmaf(x * 0.39894228040143268f, expf(-0.5f * x * x), 0.5f * erfcf(-0.70710678118654752f * x));
  }
}
__device__ __forceinline__ float gelu_grad_at(const float* tab, float x) {
  const uint32_t b = __float_as_uint(x);
  // byte offsets: entry (exponent and mantissa bits - kGradLo), clamped, 1024 up for negative x
  const int i = min(max((int)((b >> 18) & 0x1FFCu) - 4 * kGradLo, 0), 4 * (kGradN - 1));
  const uint32_t at = ((b >> 21) & (4u * kGradNeg)) | (uint32_t)i;
  return fmaf(x, 0.f, *reinterpret_cast<const float*>(reinterpret_cast<const char*>(tab) + at));  // NaN stays NaN
}

// in [rows, cols] through an optional GELU' of the checkpoint u, to `out`
// and / or block8, with optional column sums. A warp owns 256 columns and a
// stride of rows, U at a time (bytes in flight), so that the column sums stay in its registers;
// neighbouring warps take neighbouring columns of the same rows.
// VEC: rows on boundaries and cols a multiple of eight, so that a lane's columns
// all exist or none does; otherwise every 32nd column a lane, turned in shared
// memory (20480 x 4001 bf16 to 8 bits 63 us; with one row in flight 94).
// 40960 x 4096, bf16 in and out, 8-bit out, bias gradient: 168 us, 6.0 TB/s (floor
// 148); four columns a lane and a polynomial for the gradient took 499.
template <typename T, bool HAS_U, bool VEC>
__global__ void __launch_bounds__(256, HAS_U ? 3 : 4) rows8_kernel(const Rows8 p, int nchunk, int groups) {
  constexpr int U = sizeof(T) == 4 ? 2 : 4;  // rows in flight, as registers allow
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int task = (int)blockIdx.x * 8 + warp;
  const int grp = task / nchunk, c0 = (task - grp * nchunk) * kChunk, col = c0 + 8 * lane, cols = p.cols;
  __shared__ float grad[HAS_U ? kGradSize : 1];
  __shared__ float stage[VEC ? 1 : 8][kStage];
  float* sm = stage[VEC ? 0 : warp];
  if (HAS_U) {
    gelu_grad_table(grad);
    __syncthreads();
  }
  pdl_wait();
  pdl_trigger();
  if (grp >= groups) return;
  float acc[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) acc[i] = 0.f;
  const bool on = col < cols;
  const int at = on ? col : 0;
  const T* in = static_cast<const T*>(p.in.p);
  const uint8_t* us = HAS_U ? p.u.scale + (size_t)(at / kBlk) * p.u.lds : nullptr;
  for (int r0 = grp * U; r0 < p.rows; r0 += groups * U) {
    constexpr int W = sizeof(T) / 2;
    uint4 raw[VEC ? U : 1][W];
    uint32_t one[VEC ? 1 : U][8];  // every 32nd column
    uint2 uq[U];
    uint32_t ub[U];
#pragma unroll
    for (int j = 0; j < U; ++j) {
      const size_t r = (size_t)min(r0 + j, p.rows - 1);
      if (VEC) {
        const uint4* src = reinterpret_cast<const uint4*>(in + r * p.in.ld + at);
#pragma unroll
        for (int k = 0; k < W; ++k) raw[j][k] = src[k];
      } else {
        ld8s(Mat{p.in.p, p.in.ld, W == 1 ? LAZYMAR_BF16 : LAZYMAR_F32, false}, r, c0, cols, one[j]);
      }
      if (HAS_U) {
        const uint8_t* q = static_cast<const uint8_t*>(p.u.q) + r * p.u.ldq;
        uq[j] = VEC ? *reinterpret_cast<const uint2*>(q + at) : ldq8(q, col, cols);
        ub[j] = us[r];
      }
    }
#pragma unroll
    for (int j = 0; j < U; ++j) {
      if (r0 + j >= p.rows) break;
      const size_t r = (size_t)(r0 + j);
      float v[8];
      if constexpr (!VEC) {
        turn8(sm, one[j], W == 1 ? 16 : 0, v);
      } else if constexpr (W == 1) {
        bf16x8(raw[j][0], v);
      } else {
        const uint32_t w[8] = {raw[j][0].x, raw[j][0].y, raw[j][0].z, raw[j][0].w,
                               raw[j][W - 1].x, raw[j][W - 1].y, raw[j][W - 1].z, raw[j][W - 1].w};
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = __uint_as_float(w[i]);
      }
      if (HAS_U) {
        float u[8];
        block8_values(uq[j], block8_scale(ub[j]), u);
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] *= gelu_grad_at(grad, u[i]);
      }
      if (VEC && !on) {
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = 0.f;
      }
      if (p.db) {
#pragma unroll
        for (int i = 0; i < 8; ++i) acc[i] += v[i];
      }
      if (VEC) {
        if (p.out.p && on) {
          if (p.out.dtype == LAZYMAR_F32) st8a(static_cast<float*>(p.out.p) + r * p.out.ld + col, v);
          else st8a(static_cast<bf16*>(p.out.p) + r * p.out.ld + col, v);
        }
        if (p.out8.q) {
          uint2 w;
          const uint32_t byte = block8_quantize(v, w);
          if (on) {
            *reinterpret_cast<uint2*>(static_cast<uint8_t*>(p.out8.q) + r * p.out8.ldq + col) = w;
            if ((lane & 15) == 0) p.out8.scale[(size_t)(col / kBlk) * p.out8.lds + r] = (uint8_t)byte;
          }
        }
      } else {
        if (p.out.p) st_mat<false>(p.out, r, c0, cols, sm, v);
        if (p.out8.q) put8<false>(p.out8, r, c0, cols, v);
      }
    }
  }
  if (p.db) {
    float* o = p.ws + (size_t)grp * cols + col;
#pragma unroll
    for (int i = 0; i < 8; ++i)
      if (col + i < cols) o[i] = acc[i];
  }
}

// Row groups of a launch: the warps that fit on every SM, once: 24 with four rows
// in flight each for GELU's gradient (40960 x 4096: 171 us then; 32 with two 180), 32
// without it (pack of 20480 x 4096: 41 us; 24 warps 47).
int rows8_groups(int rows, int nchunk, bool has_u) {
  const int want = kSMs * (has_u ? 24 : 32) / nchunk, most = (rows + 1) / 2;
  return want < 1 ? 1 : want < most ? want : most;
}

// ---------------------------------------------------------------------------
// Back to fp32 / bf16, and weights
// ---------------------------------------------------------------------------
template <typename T>
__global__ void __launch_bounds__(256, 4) unpack8_kernel(const lazymar_block8 q, T* __restrict__ x, int ld, int rows,
                                                         int cols, int nchunk, bool vec) {
  __shared__ float stage[8][kStage];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  pdl_wait();
  pdl_trigger();
  const long long tasks = (long long)rows * nchunk, step = (long long)gridDim.x * 8 * 4;
  for (long long t0 = ((long long)blockIdx.x * 8 + warp) * 4; t0 < tasks; t0 += step) {
    uint2 w[4];
    uint32_t s[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const long long t = t0 + i < tasks ? t0 + i : tasks - 1;
      const long long r = t / nchunk;
      const int col = (int)(t - r * nchunk) * kChunk + 8 * lane;
      w[i] = ldq8(static_cast<const uint8_t*>(q.q) + (size_t)r * q.ldq, col, cols);
      s[i] = q.scale[(size_t)(min(col, cols - 1) / kBlk) * q.lds + r];
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const long long t = t0 + i;
      if (t >= tasks) break;
      const long long r = t / nchunk;
      float v[8];
      block8_values(w[i], block8_scale(s[i]), v);
      st8<T>(x + (size_t)r * ld, (int)(t - r * nchunk) * kChunk, cols, vec, stage[warp], v);
    }
  }
}

// Columns col..col+3 of a weight's row; those from K on read as zero.
template <typename T>
__device__ __forceinline__ float4 ld4(const T* row, int col, int K, bool vec) {
  if (vec && col + 4 <= K) {
    if constexpr (sizeof(T) == 2) {
      const uint2 u = *reinterpret_cast<const uint2*>(row + col);
      return make_float4(__uint_as_float(u.x << 16), __uint_as_float(u.x & 0xFFFF0000u), __uint_as_float(u.y << 16),
                         __uint_as_float(u.y & 0xFFFF0000u));
    } else {
      return *reinterpret_cast<const float4*>(row + col);
    }
  }
  float v[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) v[i] = col + i < K ? to_f(row[col + i]) : 0.f;
  return make_float4(v[0], v[1], v[2], v[3]);
}
__device__ __forceinline__ void stq4(uint8_t* row, int col, int K, uint32_t w) {
  if (col + 4 <= K) {
    *reinterpret_cast<uint32_t*>(row + col) = w;
  } else {
    for (int i = 0; col + i < K; ++i) row[col + i] = (uint8_t)(w >> (8 * i));
  }
}
__device__ __forceinline__ float4 f4_nonfinite_to(float4 v, float to) {
  return make_float4(nonfinite_to(v.x, to), nonfinite_to(v.y, to), nonfinite_to(v.z, to), nonfinite_to(v.w, to));
}

// One 128 x 128 block of a weight matrix to E4M3 with one scale, and the same
// bytes transposed. Each warp holds 16 rows; the transpose goes through shared
// memory, 132 bytes a row.
__global__ void __launch_bounds__(256) pack_weight8_kernel(const Mat w, const lazymar_block8 q,
                                                           const lazymar_block8 qt, int N, int K) {
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
      v[i] = w.dtype == LAZYMAR_F32 ? ld4<float>(static_cast<const float*>(w.p) + (size_t)n * w.ld, col, K, w.vec)
                                    : ld4<bf16>(static_cast<const bf16*>(w.p) + (size_t)n * w.ld, col, K, w.vec);
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
  const int nc = (p.D + kChunk - 1) / kChunk;
  if (nc <= 1) return ln_forward_run<1, 1>(c, p);
  if (nc <= 2) return ln_forward_run<2, 1>(c, p);
  if (nc <= 3) return ln_forward_run<3, 1>(c, p);
  if (nc <= 4) return ln_forward_run<4, 1>(c, p);
  if (nc <= 5) return ln_forward_run<5, 1>(c, p);
  if (nc <= 8) return ln_forward_run<4, 2>(c, p);
  if (nc <= 10) return ln_forward_run<5, 2>(c, p);
  if (nc <= 16) return ln_forward_run<4, 4>(c, p);
  if (nc <= 20) return ln_forward_run<5, 4>(c, p);
  return ln_forward_run<4, 8>(c, p);
}

size_t ln_backward_workspace(int M, int D) {
  return M > 0 && D > 0 ? (size_t)ln_backward_ctas(M, 1, 3) * 2 * D * sizeof(float) : 0;
}

cudaError_t launch_ln_backward(const Ctx& c, const LnBackward& p) {
  if (p.M == 0) {
    if (!p.dg || p.accumulate) return cudaSuccess;
    return column_sums(c, p.ws, 0, 2 * p.D, p.D, p.dg, p.db, false);
  }
  const int nc = (p.D + kChunk - 1) / kChunk;
  int ctas = 0;
  cudaError_t e;
  if (p.D <= 4096 && p.D % 8 == 0 && p.dy.vec && p.x.vec && p.dres.vec && p.dx.vec) {
    const int nb = (p.D + kBlk - 1) / kBlk;
    e = nb <= 1   ? ln_backward_ring_run<1, 1>(c, p, &ctas)
        : nb <= 2 ? ln_backward_ring_run<2, 1>(c, p, &ctas)
        : nb <= 4 ? ln_backward_ring_run<2, 2>(c, p, &ctas)
        : nb <= 6 ? ln_backward_ring_run<3, 2>(c, p, &ctas)
        : nb <= 8 ? ln_backward_ring_run<4, 2>(c, p, &ctas)
        : nb <= 10 ? ln_backward_ring_run<5, 2>(c, p, &ctas)
        : nb <= 12 ? ln_backward_ring_run<3, 4>(c, p, &ctas)
        : nb <= 16 ? ln_backward_ring_run<4, 4>(c, p, &ctas)
                   : ln_backward_ring_run<4, 8>(c, p, &ctas);
  } else {
    e = nc <= 1    ? ln_backward_run<1, 1>(c, p, &ctas)
        : nc <= 2  ? ln_backward_run<1, 2>(c, p, &ctas)
        : nc <= 4  ? ln_backward_run<1, 4>(c, p, &ctas)
        : nc <= 5  ? ln_backward_run<1, 5>(c, p, &ctas)
        : nc <= 8  ? ln_backward_run<1, 8>(c, p, &ctas)
        : nc <= 16 ? ln_backward_run<1, 16>(c, p, &ctas)
                   : ln_backward_run<2, 16>(c, p, &ctas);
  }
  if (e != cudaSuccess || !p.dg) return e;
  return column_sums(c, p.ws, ctas, 2 * p.D, p.D, p.dg, p.db, p.accumulate);
}

size_t rows8_workspace(int rows, int cols) {
  if (rows < 1 || cols < 1) return 0;
  return (size_t)rows8_groups(rows, (cols + kChunk - 1) / kChunk, false) * cols * sizeof(float);  // (the larger number)
}

cudaError_t launch_rows8(const Ctx& c, const Rows8& p) {
  if (p.rows == 0) {
    if (!p.db || p.accumulate) return cudaSuccess;
    return column_sums(c, p.ws, 0, p.cols, p.cols, p.db, nullptr, false);
  }
  const int nchunk = (p.cols + kChunk - 1) / kChunk, groups = rows8_groups(p.rows, nchunk, p.u.q != nullptr);
  const dim3 grid((unsigned)(((long long)nchunk * groups + 7) / 8)), block(256);
  const bool vec = p.in.vec && p.out.vec && p.cols % 8 == 0;
#define LM_ROWS8(T, HAS_U)                                                                                \
  (vec ? launch_pdl(rows8_kernel<T, HAS_U, true>, grid, block, 0, c.stream, p, nchunk, groups)             \
       : launch_pdl(rows8_kernel<T, HAS_U, false>, grid, block, 0, c.stream, p, nchunk, groups))
  const cudaError_t e = p.in.dtype == LAZYMAR_F32 ? (p.u.q ? LM_ROWS8(float, true) : LM_ROWS8(float, false))
                                                  : (p.u.q ? LM_ROWS8(bf16, true) : LM_ROWS8(bf16, false));
#undef LM_ROWS8
  if (e != cudaSuccess || !p.db) return e;
  return column_sums(c, p.ws, groups, p.cols, p.cols, p.db, nullptr, p.accumulate);
}

cudaError_t launch_unpack8(const Ctx& c, const lazymar_block8& q, const MatOut& x, int rows, int cols) {
  if (rows == 0) return cudaSuccess;
  const int nchunk = (cols + kChunk - 1) / kChunk;
  long long ctas = ((long long)rows * nchunk + 31) / 32;
  if (ctas > kSMs * 8) ctas = kSMs * 8;
  if (x.dtype == LAZYMAR_F32)
    return launch_pdl(unpack8_kernel<float>, dim3((unsigned)ctas), dim3(256), 0, c.stream, q, static_cast<float*>(x.p),
                      x.ld, rows, cols, nchunk, x.vec);
  return launch_pdl(unpack8_kernel<bf16>, dim3((unsigned)ctas), dim3(256), 0, c.stream, q, static_cast<bf16*>(x.p),
                    x.ld, rows, cols, nchunk, x.vec);
}

cudaError_t launch_pack_weight8(const Ctx& c, const Mat& w, const lazymar_block8& q, const lazymar_block8& qt, int N,
                                int K) {
  const dim3 grid((unsigned)((K + kBlk - 1) / kBlk), (unsigned)((N + kBlk - 1) / kBlk));
  return launch_pdl(pack_weight8_kernel, grid, dim3(256), 0, c.stream, w, q, qt, N, K);
}

}  // namespace lm
