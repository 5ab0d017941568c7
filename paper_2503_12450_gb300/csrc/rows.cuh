// Rows of fp32, bf16 and 8-bit tensors as the row-wise kernels take them: a warp's
// 256 columns, eight consecutive ones a lane; and sums over a row's warps.
#pragma once

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

}  // namespace

}  // namespace lm
