// The 8-bit block format ("block8") of activations kept for the backward pass
// and of the 8-bit matrix products' operands: E4M3 bytes with one power-of-two
// scale, held as its biased exponent, for each row and 128 columns (weights:
// for each 128 x 128 block).
//
// Why powers of two. A scale max / 448 would use E4M3's range to the last bit;
// rounding it up to a power of two gives at most one binade of E4M3's 17 away
// and leaves the relative precision (2^-4) as it is, because E4M3 is itself
// floating. In return x 2^-e is exact (one rounding, to E4M3), q 2^e is exact
// in bf16 (the weight gradient's product takes the checkpoint without another
// rounding), a scale is a byte, and the tensor cores apply it themselves.
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
__device__ __forceinline__ float4 e4m3x4_to_f4(uint32_t four, float s) {
  const float2 a = e4m3x2_to_f2(four & 0xFFFFu), b = e4m3x2_to_f2(four >> 16);
  return make_float4(a.x * s, a.y * s, b.x * s, b.y * s);
}

__device__ __forceinline__ float4 f4_nonfinite_to(float4 v, float to) {
  auto f = [&](float x) { return (__float_as_uint(x) & 0x7F800000u) == 0x7F800000u ? to : x; };
  return make_float4(f(v.x), f(v.y), f(v.z), f(v.w));
}

// A warp's block of 128 columns, four consecutive ones a lane, to E4M3: the
// scale byte (the same in every lane) and this lane's four bytes. The scale is
// that of the finite values; infinities and NaN become NaN, so an overflow
// stays visible and does not disturb its neighbours.
__device__ __forceinline__ uint32_t block8_quantize(float4 v, uint32_t& q) {
  const float m = fmax3(fmaxf(fabsf(v.x), fabsf(v.y)), fabsf(v.z), fabsf(v.w));
  uint32_t amax = __reduce_max_sync(0xffffffffu, __float_as_uint(m));
  if (amax >= 0x7F800000u) {  // an infinity, or a lane of NaN alone
    const float4 z = f4_nonfinite_to(v, 0.f);
    const float mz = fmax3(fmaxf(fabsf(z.x), fabsf(z.y)), fabsf(z.z), fabsf(z.w));
    amax = __reduce_max_sync(0xffffffffu, __float_as_uint(mz));
    v = f4_nonfinite_to(v, __uint_as_float(0x7FC00000u));
  }
  const uint32_t byte = block8_exp(amax);
  const float s = block8_inv(byte);
  q = e4m3x4(v.x * s, v.y * s, v.z * s, v.w * s);
  return byte;
}

// Tensors as the kernels take them. dtype LAZYMAR_F32 or LAZYMAR_BF16.
struct Mat {
  const void* p;
  int ld, dtype;
};
struct MatOut {
  void* p;
  int ld, dtype;
};

struct LnForward {
  Mat x;
  const float *g, *b;
  MatOut y;                // p may be NULL
  lazymar_block8 y8, x8;   // q may be NULL
  float *mean, *rstd;      // may be NULL
  int M, D;
  float eps;
  bool vec;  // rows of x and y start on 4-element boundaries
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
  bool vec;
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
  bool vec;
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
