// The 8-bit block format ("block8") of activations kept for the backward pass
// and of the 8-bit matrix products' operands: E4M3 bytes with one power-of-two
// scale, held as its biased exponent, for each row and 128 columns (weights:
// for each 128 x 128 block).
//
// Why powers of two. A scale max / 448 would use E4M3's range to the last bit;
// rounding it up to a power of two gives at most one binade of E4M3's 17 away
// and leaves the relative precision (2^-4) as it is, because E4M3 is itself
// floating. In return x 2^-e is exact (one rounding, to E4M3), q 2^e is exact
// in bf16 from 2^-130 on (the weight gradient's product takes the checkpoint
// without another rounding; below, bf16 has only multiples of 2^-133), a scale is a
// byte, and the tensor cores apply it themselves.
#pragma once

#include <cuda_fp8.h>

#include "lazymar_internal.cuh"

namespace lm {

constexpr int kBlk = 128;  // columns that share a scale

// Biased exponent of the scale of a block whose largest finite magnitude has
// the bits `amax`: the smallest e >= -126 with amax <= 448 2^e, 448 = 1.75 2^8.
// Adding 0x1FFFFF carries into the exponent exactly for mantissas above 1.75.
__device__ __forceinline__ uint32_t block8_exp(uint32_t amax) {
  const uint32_t k = (amax + 0x1FFFFFu) >> 23;
  return k > 9u ? k - 8u : 1u;
}
// 2^e and 2^-e of a scale byte (1..247, so both are normal numbers).
__device__ __forceinline__ float block8_scale(uint32_t byte) { return __uint_as_float(byte << 23); }
__device__ __forceinline__ float block8_inv(uint32_t byte) { return __uint_as_float((254u - byte) << 23); }

// Four values to four E4M3 bytes, nearest even; NaN stays NaN.
__device__ __forceinline__ uint32_t e4m3x4(float a, float b, float c, float d) {
  const uint32_t lo = __nv_cvt_float2_to_fp8x2(make_float2(a, b), __NV_SATFINITE, __NV_E4M3);
  const uint32_t hi = __nv_cvt_float2_to_fp8x2(make_float2(c, d), __NV_SATFINITE, __NV_E4M3);
  return lo | (hi << 16);
}
__device__ __forceinline__ float2 e4m3x2_to_f2(uint32_t two) {
  const __half2_raw h = __nv_cvt_fp8x2_to_halfraw2((__nv_fp8x2_storage_t)two, __NV_E4M3);
  return __half22float2(*reinterpret_cast<const __half2*>(&h));
}

// Two blocks of 128 columns in a warp, one in each half, eight consecutive
// columns a lane, to E4M3: the scale byte of the lane's block and the lane's
// eight bytes. The scale is that of the finite values; infinities and NaN become
// NaN, so an overflow stays visible and does not disturb its neighbours.
__device__ __forceinline__ uint32_t block8_amax(const float (&v)[8]) {
  // (plain fmaxf: the compiler folds the magnitudes into three-input maxima)
  float m = fmaxf(fabsf(v[0]), fabsf(v[1]));
#pragma unroll
  for (int i = 2; i < 8; i += 2) m = fmaxf(fmaxf(m, fabsf(v[i])), fabsf(v[i + 1]));
  return __float_as_uint(m);
}
__device__ __forceinline__ float nonfinite_to(float x, float to) {
  return (__float_as_uint(x) & 0x7F800000u) == 0x7F800000u ? to : x;
}
__device__ __forceinline__ uint32_t half_warp_max(uint32_t m, bool upper, uint32_t& both) {
  const uint32_t lo = __reduce_max_sync(0xffffffffu, upper ? 0u : m);
  const uint32_t hi = __reduce_max_sync(0xffffffffu, upper ? m : 0u);
  both = max(lo, hi);
  return upper ? hi : lo;
}
__device__ __forceinline__ uint32_t block8_quantize(const float (&v)[8], uint2& q) {
  const bool upper = threadIdx.x & 16;
  auto scaled = [&](const float (&x)[8], uint32_t amax) {
    const uint32_t byte = block8_exp(amax);
    const float s = block8_inv(byte);
    const unsigned long long ss = f32x2_pack(s, s);
    float w[8];
#pragma unroll
    for (int i = 0; i < 8; i += 2) f32x2_unpack(f32x2_mul(f32x2_pack(x[i], x[i + 1]), ss), w[i], w[i + 1]);
    q = make_uint2(e4m3x4(w[0], w[1], w[2], w[3]), e4m3x4(w[4], w[5], w[6], w[7]));
    return byte;
  };
  uint32_t both;
  const uint32_t amax = half_warp_max(block8_amax(v), upper, both);
  if (both < 0x7F800000u) return scaled(v, amax);
  float z[8], n[8];  // an infinity
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    z[i] = nonfinite_to(v[i], 0.f);
    n[i] = nonfinite_to(v[i], __uint_as_float(0x7FC00000u));
  }
  return scaled(n, half_warp_max(block8_amax(z), upper, both));
}
// Eight E4M3 bytes times a scale.
__device__ __forceinline__ void block8_values(uint2 q, float s, float (&v)[8]) {
  const float2 a = e4m3x2_to_f2(q.x & 0xFFFFu), b = e4m3x2_to_f2(q.x >> 16);
  const float2 c = e4m3x2_to_f2(q.y & 0xFFFFu), d = e4m3x2_to_f2(q.y >> 16);
  const unsigned long long ss = f32x2_pack(s, s);
  f32x2_unpack(f32x2_mul(f32x2_pack(a.x, a.y), ss), v[0], v[1]);
  f32x2_unpack(f32x2_mul(f32x2_pack(b.x, b.y), ss), v[2], v[3]);
  f32x2_unpack(f32x2_mul(f32x2_pack(c.x, c.y), ss), v[4], v[5]);
  f32x2_unpack(f32x2_mul(f32x2_pack(d.x, d.y), ss), v[6], v[7]);
}

// GELU in the erf form for the 8-bit product's epilogues: gelu_erf of
// lazymar_internal.cuh with a tail polynomial of degree 6 (csrc/gen_gelu_poly.py),
// within 1.1e-7 max(1, |x|) instead of 2.8e-7 (and 4e-8 for exp2_approx), which moves
// fewer values over an E4M3 rounding boundary, for one more paired instruction. The
// bound is absolute: relative to GELU itself 4e-6 above -2, 1e-3 at -4, 3 % at -6,
// and below -6 the result stays at -5.8e-9.
__device__ __forceinline__ void gelu_erf6_x2(float& x0, float& x1) {
  constexpr float kGelu6P0 = -9.999947548e-01f;
  constexpr float kGelu6P1 = -1.151182413e+00f;
  constexpr float kGelu6P2 = -4.588403106e-01f;
  constexpr float kGelu6P3 = -5.330511183e-02f;
  constexpr float kGelu6P4 = 8.002257906e-03f;
  constexpr float kGelu6P5 = -7.424726500e-04f;
  constexpr float kGelu6P6 = 2.970655623e-05f;
  // in v = -min(|x|, 6): the odd coefficients change sign
  const float v0 = fmaxf(-fabsf(x0), -6.0f), v1 = fmaxf(-fabsf(x1), -6.0f);
  const unsigned long long v = f32x2_pack(v0, v1);
  unsigned long long p = f32x2_fma(f32x2_pack(kGelu6P6, kGelu6P6), v, f32x2_pack(-kGelu6P5, -kGelu6P5));
  p = f32x2_fma(p, v, f32x2_pack(kGelu6P4, kGelu6P4));
  p = f32x2_fma(p, v, f32x2_pack(-kGelu6P3, -kGelu6P3));
  p = f32x2_fma(p, v, f32x2_pack(kGelu6P2, kGelu6P2));
  p = f32x2_fma(p, v, f32x2_pack(-kGelu6P1, -kGelu6P1));
  p = f32x2_fma(p, v, f32x2_pack(kGelu6P0, kGelu6P0));
  float p0, p1;
  f32x2_unpack(p, p0, p1);
  const unsigned long long h = f32x2_pack(exp2_approx(p0), exp2_approx(p1));
  const unsigned long long half = f32x2_mul(f32x2_add(f32x2_pack(x0, x1), f32x2_pack(fabsf(x0), fabsf(x1))),
                                            f32x2_pack(0.5f, 0.5f));
  f32x2_unpack(f32x2_fma(v, h, half), x0, x1);
}

// Arrives on a barrier of a CTA pair's even CTA for what this warp has written to,
// or read from, its own CTA's shared or tensor memory (and fenced for the
// asynchronous proxy or tcgen05). The MMA that the even CTA then issues touches it
// through this SM's half alone, never through the other CTA's threads, so the
// release need not reach beyond this CTA; one that does (release.cluster) waits
// for every write of the warp that is under way, and held the weight gradient's
// stages up by 0.3 us each.
__device__ __forceinline__ void arrive_even(uint64_t* bar) {
  asm volatile("mbarrier.arrive.release.cta.shared::cluster.b64 _, [%0];" ::"r"(cluster_map(smem_u32(bar), 0)) : "memory");
}

// Tensors as the kernels take them. dtype LAZYMAR_F32 or LAZYMAR_BF16; vec:
// rows start on boundaries of eight elements.
struct Mat {
  const void* p;
  int ld, dtype;
  bool vec;
};
struct MatOut {
  void* p;
  int ld, dtype;
  bool vec;
};

struct LnForward {
  Mat x;
  const float *g, *b;
  bool params_vec;         // g and b on boundaries of eight elements (or NULL)
  MatOut y;                // p may be NULL
  lazymar_block8 y8, x8;   // q may be NULL
  float *mean, *rstd;      // may be NULL
  int M, D;
  float eps;
};
struct LnBackward {
  Mat dy, x;          // x.p NULL: x8
  lazymar_block8 x8;
  const float *mean, *rstd, *g;
  Mat dres;           // fp32, p may be NULL
  MatOut dx;
  float *dg, *db;     // may be NULL (both)
  bool accumulate;
  int M, D;
  float* ws;
};
// The row-wise pass over [rows, cols] behind pack and the GELU gradient.
struct Rows8 {
  Mat in;
  lazymar_block8 u;    // q NULL: no activation
  MatOut out;          // p may be NULL
  lazymar_block8 out8; // q may be NULL
  float* db;           // may be NULL
  bool accumulate;
  int rows, cols;
  float* ws;
};

constexpr int kLnMaxWidth = 8192;

cudaError_t launch_ln_forward(const Ctx& c, const LnForward& p);
cudaError_t launch_ln_backward(const Ctx& c, const LnBackward& p);
size_t ln_backward_workspace(int M, int D);
cudaError_t launch_rows8(const Ctx& c, const Rows8& p);
size_t rows8_workspace(int rows, int cols);
cudaError_t launch_unpack8(const Ctx& c, const lazymar_block8& q, const MatOut& x, int rows, int cols);
cudaError_t launch_pack_weight8(const Ctx& c, const Mat& w, const lazymar_block8& q, const lazymar_block8& qt, int N,
                                int K);

// The 8-bit product (lazymar_block8_linear).
struct Linear8 {
  int epilogue;
  lazymar_block8 a, w;
  const float* bias;
  Mat residual;
  MatOut out;          // p may be NULL
  lazymar_block8 out8, u8;
  int M, N, K;
};
cudaError_t launch_linear8(const Ctx& c, const Linear8& p);
// The same for at most kLinear8FewRows rows of a.
constexpr int kLinear8FewRows = 32;
cudaError_t launch_linear8_rows(const Ctx& c, const Linear8& p);

// The weight gradient (lazymar_block8_wgrad).
struct Wgrad8 {
  const void* dy;
  int lddy;
  lazymar_block8 x;
  float* dw;
  int lddw;
  bool accumulate;
  int M, N, K;
  float* ws;
};
cudaError_t launch_wgrad8(const Ctx& c, const Wgrad8& p);
size_t wgrad8_workspace(int M, int N, int K);

}  // namespace lm
