// The block-scaled 8-bit product for a few rows of a (serving: single tokens up
// to 32): bound by reading the weights and, at a few MB of them, by latency. A
// tcgen05 tile of 128 rows would leave most SMs without a tile and pay for
// descriptors, tensor memory and a pipeline; here a CTA of eight warps takes 16 rows
// of w, the warps take its K blocks in turn, and all loads of a warp's block are in
// flight at once. Measured (us, against the tcgen05 kernel on single CTAs): 2 x 4096
// x 1024 3.1 : 9.2 (the weights' 4 MB: 0.6), 8 x 1024 x 4096 5.1 : 17.4, 32 x 1024 x 4096
// 8.5 : 18.5 (and 7.4 with K in parts: the limit of 32 rows is not the best at every K),
// 32 x 4096 x 1024 4.8 : 9.6.
//
// E4M3 is exact in fp16, so the products run as fp16 warp MMAs (m16n8k16, w as the
// 16-row operand, tokens as the 8 columns) with fp32 sums; a block's sum is scaled
// by 2^(ea + ew) and added in fp32. The order of k inside a block is free as long
// as both operands agree: every lane takes 16 consecutive bytes of its row of w and
// of its token, and the four lanes of a row 64 of the block's 128.
//
// 8-bit outputs need a token's maximum over 128 columns: eight CTAs form a
// cluster and exchange their 16 columns' maxima through distributed shared
// memory.
#include "block8.cuh"

namespace lm {

namespace {

constexpr int kWarps = 8, kCols = 16;

struct RowsParams {
  const uint8_t *a, *w, *a_scale, *w_scale;
  int lda, ldw, lds_a, lds_w;
  int epilogue, M, N, K;
  const float* bias;
  const float* residual;
  int ldr;
  void* out;
  int ldo, out_dtype;
  uint8_t *out8, *out8_scale, *u8, *u8_scale;
  int ldout8, lds_out8, ldu8, lds_u8;
};

__device__ __forceinline__ uint32_t e4m3x2_to_h2(uint32_t two) {
  const __half2_raw h = __nv_cvt_fp8x2_to_halfraw2((__nv_fp8x2_storage_t)two, __NV_E4M3);
  return (uint32_t)h.x | ((uint32_t)h.y << 16);
}
__device__ __forceinline__ void mma_f16(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0,
                                        uint32_t b1) {
  asm volatile(
      "mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, "
      "{%0, %1, %2, %3};"
      : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
      : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
// 16 bytes of a row from column k on; those from K on are zero.
__device__ __forceinline__ uint4 row16(const uint8_t* row, int k, int K) {
  if (k >= K) return make_uint4(0u, 0u, 0u, 0u);
  uint4 v = *reinterpret_cast<const uint4*>(row + k);
  if (k + 16 > K) {
    uint32_t* w = reinterpret_cast<uint32_t*>(&v);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int n = K - k - 4 * i;  // bytes of this word
      if (n < 4) w[i] = n <= 0 ? 0u : w[i] & (0xFFFFFFFFu >> (32 - 8 * n));
    }
  }
  return v;
}
__device__ __forceinline__ uint32_t ld_cluster_u32(uint32_t addr) {
  uint32_t v;
  asm volatile("ld.shared::cluster.u32 %0, [%1];" : "=r"(v) : "r"(addr) : "memory");
  return v;
}

// TILES of eight tokens. BLOCK8: 8-bit outputs, in clusters of eight CTAs.
template <int TILES, bool BLOCK8>
__global__ void __launch_bounds__(kWarps * 32) linear8_rows_kernel(const RowsParams p) {
  constexpr int TOK = 8 * TILES;
  __shared__ float part[kWarps][TOK][kCols + 1];
  __shared__ uint32_t most[2][TOK];  // bits of the largest finite magnitudes: of u, of the output
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
  const int n0 = (int)blockIdx.x * kCols, KB = (p.K + kBlk - 1) / kBlk;
  pdl_wait();
  pdl_trigger();
  float sum[TILES][4];
#pragma unroll
  for (int j = 0; j < TILES; ++j)
#pragma unroll
    for (int i = 0; i < 4; ++i) sum[j][i] = 0.f;
  if (n0 < p.N) {
    const uint8_t* w0 = p.w + (size_t)(n0 + g) * p.ldw;
    const uint8_t* w1 = w0 + (size_t)8 * p.ldw;
    const bool has0 = n0 + g < p.N, has1 = n0 + g + 8 < p.N;
    for (int kb = warp; kb < KB; kb += kWarps) {
      uint4 va[2][2], vb[TILES][2];
      uint32_t sa[TILES][2];
      const uint32_t sw = p.w_scale[(size_t)kb * p.lds_w + n0 / kBlk];
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const int k = kb * kBlk + 64 * h + 16 * t;
        va[0][h] = row16(w0, has0 ? k : p.K, p.K);
        va[1][h] = row16(w1, has1 ? k : p.K, p.K);
#pragma unroll
        for (int j = 0; j < TILES; ++j)
          vb[j][h] = row16(p.a + (size_t)(8 * j + g) * p.lda, 8 * j + g < p.M ? k : p.K, p.K);
      }
#pragma unroll
      for (int j = 0; j < TILES; ++j)
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          const int m = 8 * j + 2 * t + i;
          sa[j][i] = m < p.M ? p.a_scale[(size_t)kb * p.lds_a + m] : 127u;
        }
      float d[TILES][4];
#pragma unroll
      for (int j = 0; j < TILES; ++j)
#pragma unroll
        for (int i = 0; i < 4; ++i) d[j][i] = 0.f;
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const uint32_t a0[4] = {va[0][h].x, va[0][h].y, va[0][h].z, va[0][h].w};
        const uint32_t a1[4] = {va[1][h].x, va[1][h].y, va[1][h].z, va[1][h].w};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const uint32_t x0 = e4m3x2_to_h2(a0[i] & 0xFFFFu), x1 = e4m3x2_to_h2(a1[i] & 0xFFFFu);
          const uint32_t x2 = e4m3x2_to_h2(a0[i] >> 16), x3 = e4m3x2_to_h2(a1[i] >> 16);
#pragma unroll
          for (int j = 0; j < TILES; ++j) {
            const uint32_t b[4] = {vb[j][h].x, vb[j][h].y, vb[j][h].z, vb[j][h].w};
            mma_f16(d[j], x0, x1, x2, x3, e4m3x2_to_h2(b[i] & 0xFFFFu), e4m3x2_to_h2(b[i] >> 16));
          }
        }
      }
      // One factor after the other (their product may leave fp32's range where the sum does
      // not), the smaller one first: d is a multiple of 2^-18 below 2^25, so d times a factor
      // below one is exact and finite, and if both are one or more, a step that overflows
      // only does what the result does.
      const float ws = block8_scale(sw);
#pragma unroll
      for (int j = 0; j < TILES; ++j) {  // accumulator: rows g and g + 8 of w, tokens 2 t and 2 t + 1
        const float s0 = block8_scale(sa[j][0]), s1 = block8_scale(sa[j][1]);
        const float l0 = fminf(s0, ws), l1 = fminf(s1, ws), h0 = fmaxf(s0, ws), h1 = fmaxf(s1, ws);
        sum[j][0] = fmaf(d[j][0] * l0, h0, sum[j][0]);
        sum[j][1] = fmaf(d[j][1] * l1, h1, sum[j][1]);
        sum[j][2] = fmaf(d[j][2] * l0, h0, sum[j][2]);
        sum[j][3] = fmaf(d[j][3] * l1, h1, sum[j][3]);
      }
    }
  }
#pragma unroll
  for (int j = 0; j < TILES; ++j)
#pragma unroll
    for (int i = 0; i < 4; ++i) part[warp][8 * j + 2 * t + (i & 1)][g + 8 * (i >> 1)] = sum[j][i];
  __syncthreads();
  // element (token, column) by thread: 16 lanes a token
  constexpr int EACH = (TOK * kCols + kWarps * 32 - 1) / (kWarps * 32);
  float u[EACH], y[EACH];
#pragma unroll
  for (int e = 0; e < EACH; ++e) {
    const int i = (int)threadIdx.x + e * kWarps * 32, m = i / kCols, c = i % kCols, n = n0 + c;
    u[e] = y[e] = 0.f;
    const bool here = m < p.M && n < p.N && m < TOK;
    if (here) {
      float s = 0.f;
#pragma unroll
      for (int k = 0; k < kWarps; ++k) s += part[k][m][c];
      if (p.bias) s += p.bias[n];
      u[e] = s;
      y[e] = s;
      if (p.epilogue == LAZYMAR_EPI_GELU) {
        float other = s;
        gelu_erf6_x2(y[e], other);
      } else if (p.epilogue == LAZYMAR_EPI_RESIDUAL) {
        y[e] += p.residual[(size_t)m * p.ldr + n];
      }
      if (p.out) {
        if (p.out_dtype == LAZYMAR_F32) static_cast<float*>(p.out)[(size_t)m * p.ldo + n] = y[e];
        else static_cast<bf16*>(p.out)[(size_t)m * p.ldo + n] = from_f<bf16>(y[e]);
      }
    }
    if (BLOCK8) {
      auto finite = [](float x) {
        const uint32_t b = __float_as_uint(x) & 0x7FFFFFFFu;
        return b < 0x7F800000u ? b : 0u;
      };
      uint32_t mu = finite(u[e]), my = finite(y[e]);
#pragma unroll
      for (int o = 8; o > 0; o >>= 1) {
        mu = max(mu, __shfl_xor_sync(0xffffffffu, mu, o));
        my = max(my, __shfl_xor_sync(0xffffffffu, my, o));
      }
      if (c == 0 && m < TOK) {
        most[0][m] = mu;
        most[1][m] = my;
      }
    }
  }
  if constexpr (BLOCK8) {
    cluster_sync();
    const uint32_t ranks = cluster_nctarank();
#pragma unroll
    for (int e = 0; e < EACH; ++e) {
      const int i = (int)threadIdx.x + e * kWarps * 32, m = i / kCols, c = i % kCols, n = n0 + c;
      if (m >= p.M || m >= TOK || n >= p.N) continue;
      auto put = [&](int which, float x, uint8_t* q, int ldq, uint8_t* scale, int lds) {
        uint32_t amax = 0;
        for (uint32_t r = 0; r < ranks; ++r) amax = max(amax, ld_cluster_u32(cluster_map(smem_u32(&most[which][m]), r)));
        const uint32_t byte = block8_exp(amax);
        const float v = nonfinite_to(x, __uint_as_float(0x7FC00000u)) * block8_inv(byte);
        q[(size_t)m * ldq + n] = (uint8_t)__nv_cvt_float_to_fp8(v, __NV_SATFINITE, __NV_E4M3);
        if (n % kBlk == 0) scale[(size_t)(n / kBlk) * lds + m] = (uint8_t)byte;
      };
      if (p.u8) put(0, u[e], p.u8, p.ldu8, p.u8_scale, p.lds_u8);
      if (p.out8) put(1, y[e], p.out8, p.ldout8, p.out8_scale, p.lds_out8);
    }
    cluster_sync();  // no CTA leaves while another may read its maxima
  }
}

template <int TILES>
cudaError_t run_rows(const Ctx& c, const RowsParams& p) {
  if (p.out8 || p.u8) {
    const unsigned grid = (unsigned)((p.N + kBlk - 1) / kBlk) * (kBlk / kCols);
    return launch_pdl_cluster(linear8_rows_kernel<TILES, true>, dim3(grid), dim3(kWarps * 32), 0, kBlk / kCols, c.stream, p);
  }
  return launch_pdl(linear8_rows_kernel<TILES, false>, dim3((unsigned)((p.N + kCols - 1) / kCols)), dim3(kWarps * 32), 0,
                    c.stream, p);
}

}  // namespace

cudaError_t launch_linear8_rows(const Ctx& c, const Linear8& x) {
  RowsParams p{};
  p.a = static_cast<const uint8_t*>(x.a.q);
  p.w = static_cast<const uint8_t*>(x.w.q);
  p.a_scale = x.a.scale;
  p.w_scale = x.w.scale;
  p.lda = x.a.ldq;
  p.ldw = x.w.ldq;
  p.lds_a = x.a.lds;
  p.lds_w = x.w.lds;
  p.epilogue = x.epilogue;
  p.M = x.M;
  p.N = x.N;
  p.K = x.K;
  p.bias = x.bias;
  p.residual = static_cast<const float*>(x.residual.p);
  p.ldr = x.residual.ld;
  p.out = x.out.p;
  p.ldo = x.out.ld;
  p.out_dtype = x.out.dtype;
  p.out8 = static_cast<uint8_t*>(x.out8.q);
  p.out8_scale = x.out8.scale;
  p.ldout8 = x.out8.ldq;
  p.lds_out8 = x.out8.lds;
  p.u8 = static_cast<uint8_t*>(x.u8.q);
  p.u8_scale = x.u8.scale;
  p.ldu8 = x.u8.ldq;
  p.lds_u8 = x.u8.lds;
  if (x.M <= 8) return run_rows<1>(c, p);
  if (x.M <= 16) return run_rows<2>(c, p);
  return run_rows<4>(c, p);
}

}  // namespace lm
