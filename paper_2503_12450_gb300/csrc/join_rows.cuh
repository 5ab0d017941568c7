// What the residual join's kernels share: rows that stream through shared memory, a
// lane's columns of them, and the sums over a row's warps.
#pragma once

#include "join.cuh"
#include "rows.cuh"

namespace lm {

// The tensors whose rows a warp's ring holds, as the host lays them out.
struct RowStream {
  const uint8_t* p;
  size_t pitch;   // bytes from row to row
  uint32_t at;    // place in a stage
  uint32_t e;     // bytes of an element
};
constexpr int kMostStreams = 6;
constexpr int kMostStages = 8;
struct RingPlan {
  RowStream t[kMostStreams];
  int n;
  int depth;        // stages of a warp's ring
  uint32_t stage;   // bytes of a stage
};

namespace {

// Waits for the WPR warps of a row.
template <int WPR>
__device__ __forceinline__ void row_barrier(int grp) {
  asm volatile("bar.sync %0, %1;" ::"r"(grp + 1), "n"(WPR * 32) : "memory");
}

// ---------------------------------------------------------------------------
// A lane's eight columns of a chunk of 256
// ---------------------------------------------------------------------------
// Whole rows (WHOLE: on boundaries of eight elements, D a multiple of eight): four
// consecutive columns of each of the chunk's two blocks, accesses of four elements that
// are contiguous over the warp and free of bank conflicts. Other rows: every 32nd column.
// Either way values 0..3 are of the first block, 4..7 of the second.
template <bool WHOLE>
__device__ __forceinline__ int column(int k) {
  const int lane = threadIdx.x & 31;
  return WHOLE ? kBlk * (k >> 2) + 4 * lane + (k & 3) : 32 * k + lane;
}
template <bool WHOLE>
__device__ __forceinline__ void mask_columns(float (&v)[8], int c0, int D) {
  if (c0 + kChunk <= D) return;
#pragma unroll
  for (int k = 0; k < 8; ++k)
    if (c0 + column<WHOLE>(k) >= D) v[k] = 0.f;
}
__device__ __forceinline__ void widen4(uint2 u, float* v) {
  v[0] = __uint_as_float(u.x << 16);
  v[1] = __uint_as_float(u.x & 0xFFFF0000u);
  v[2] = __uint_as_float(u.y << 16);
  v[3] = __uint_as_float(u.y & 0xFFFF0000u);
}
__device__ __forceinline__ void put4(float4 a, float* v) {
  v[0] = a.x; v[1] = a.y; v[2] = a.z; v[3] = a.w;
}
// From global memory: row `row` of m (fp32 or bf16), columns from c0 on; those from D on read as zero.
template <bool WHOLE>
__device__ __forceinline__ void load_row(const Rows& m, size_t row, int c0, int D, float (&v)[8]) {
#pragma unroll
  for (int k = 0; k < 8; ++k) v[k] = 0.f;
  if (WHOLE) {
#pragma unroll
    for (int j = 0; j < 2; ++j) {
      const int col = c0 + column<true>(4 * j);
      if (col >= D) continue;
      if (m.dtype == LAZYMAR_F32)
        put4(*reinterpret_cast<const float4*>(static_cast<const float*>(m.p) + row * m.ld + col), v + 4 * j);
      else
        widen4(*reinterpret_cast<const uint2*>(static_cast<const bf16*>(m.p) + row * m.ld + col), v + 4 * j);
    }
  } else {
#pragma unroll
    for (int k = 0; k < 8; ++k) {
      const int col = c0 + column<false>(k);
      if (col >= D) continue;
      v[k] = m.dtype == LAZYMAR_F32 ? static_cast<const float*>(m.p)[row * m.ld + col]
                                    : to_f(static_cast<const bf16*>(m.p)[row * m.ld + col]);
    }
  }
}
template <bool WHOLE>
__device__ __forceinline__ void load_param(const float* p, int c0, int D, float (&v)[8]) {
  load_row<WHOLE>(Rows{p, nullptr, 0, 0, LAZYMAR_F32, true}, 0, c0, D, v);
}
// From a warp's stage. `shift`: the row's first byte in it (rows that are not whole).
template <bool WHOLE>
__device__ __forceinline__ void load_stage(const uint8_t* st, int dtype, uint32_t shift, uint32_t s0, uint32_t s1,
                                           float (&v)[8]) {
  const int lane = threadIdx.x & 31;
  if (dtype == LAZYMAR_E4M3) {
    const float s[2] = {block8_scale(s0), block8_scale(s1)};
#pragma unroll
    for (int j = 0; j < 2; ++j) {
      uint32_t w;
      if (WHOLE) {
        w = *reinterpret_cast<const uint32_t*>(st + kBlk * j + 4 * lane);
      } else {
        w = 0;
#pragma unroll
        for (int i = 0; i < 4; ++i) w |= (uint32_t)st[kBlk * j + 32 * i + lane] << (8 * i);
      }
      const float2 a = e4m3x2_to_f2(w & 0xFFFFu), b = e4m3x2_to_f2(w >> 16);
      v[4 * j] = a.x * s[j]; v[4 * j + 1] = a.y * s[j]; v[4 * j + 2] = b.x * s[j]; v[4 * j + 3] = b.y * s[j];
    }
  } else if (WHOLE) {
#pragma unroll
    for (int j = 0; j < 2; ++j) {
      if (dtype == LAZYMAR_F32) put4(*reinterpret_cast<const float4*>(st + 4 * (kBlk * j + 4 * lane)), v + 4 * j);
      else widen4(*reinterpret_cast<const uint2*>(st + 2 * (kBlk * j + 4 * lane)), v + 4 * j);
    }
  } else {
#pragma unroll
    for (int k = 0; k < 8; ++k)
      v[k] = dtype == LAZYMAR_F32 ? *reinterpret_cast<const float*>(st + shift + 4 * (32 * k + lane))
                                  : __uint_as_float((uint32_t)*reinterpret_cast<const uint16_t*>(st + shift + 2 * (32 * k + lane)) << 16);
  }
}
template <bool WHOLE>
__device__ __forceinline__ void store_row(const MatOut& m, size_t row, int c0, int D, const float (&v)[8]) {
  if (WHOLE) {
#pragma unroll
    for (int j = 0; j < 2; ++j) {
      const int col = c0 + column<true>(4 * j);
      if (col >= D) continue;
      if (m.dtype == LAZYMAR_F32)
        *reinterpret_cast<float4*>(static_cast<float*>(m.p) + row * m.ld + col) =
            make_float4(v[4 * j], v[4 * j + 1], v[4 * j + 2], v[4 * j + 3]);
      else
        *reinterpret_cast<uint2*>(static_cast<bf16*>(m.p) + row * m.ld + col) =
            make_uint2(pack_bf16(v[4 * j], v[4 * j + 1]), pack_bf16(v[4 * j + 2], v[4 * j + 3]));
    }
  } else {
#pragma unroll
    for (int k = 0; k < 8; ++k) {
      const int col = c0 + column<false>(k);
      if (col >= D) continue;
      if (m.dtype == LAZYMAR_F32) static_cast<float*>(m.p)[row * m.ld + col] = v[k];
      else static_cast<bf16*>(m.p)[row * m.ld + col] = from_f<bf16>(v[k]);
    }
  }
}
// To block8: a block is four values of each lane of the warp. Columns from D on hold zero.
template <bool WHOLE>
__device__ __forceinline__ void store_row8(const lazymar_block8& o, size_t row, int c0, int D, const float (&v)[8]) {
  const int lane = threadIdx.x & 31;
  uint8_t* q = static_cast<uint8_t*>(o.q) + row * o.ldq;
#pragma unroll
  for (int j = 0; j < 2; ++j) {
    if (c0 + kBlk * j >= D) break;  // (uniform over the warp)
    float w[4] = {v[4 * j], v[4 * j + 1], v[4 * j + 2], v[4 * j + 3]};
    uint32_t amax = __float_as_uint(fmaxf(fmaxf(fabsf(w[0]), fabsf(w[1])), fmaxf(fabsf(w[2]), fabsf(w[3]))));
    amax = __reduce_max_sync(0xffffffffu, amax);
    if (amax >= 0x7F800000u) {  // an infinity: the finite values' maximum
      float m = 0.f;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        m = fmaxf(m, fabsf(nonfinite_to(w[i], 0.f)));
        w[i] = nonfinite_to(w[i], __uint_as_float(0x7FC00000u));
      }
      amax = __reduce_max_sync(0xffffffffu, __float_as_uint(m));
    }
    const uint32_t byte = block8_exp(amax);
    const float s = block8_inv(byte);
    const unsigned long long ss = f32x2_pack(s, s);
    f32x2_unpack(f32x2_mul(f32x2_pack(w[0], w[1]), ss), w[0], w[1]);
    f32x2_unpack(f32x2_mul(f32x2_pack(w[2], w[3]), ss), w[2], w[3]);
    const uint32_t b = e4m3x4(w[0], w[1], w[2], w[3]);
    if (WHOLE) {
      const int col = c0 + column<true>(4 * j);
      if (col < D) *reinterpret_cast<uint32_t*>(q + col) = b;
    } else {
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int col = c0 + column<false>(4 * j + i);
        if (col < D) q[col] = (uint8_t)(b >> (8 * i));
      }
    }
    if (lane == 0) o.scale[(size_t)((c0 + kBlk * j) / kBlk) * o.lds + row] = (uint8_t)byte;
  }
}

// y = v a + b; paired
__device__ __forceinline__ void fma8(float (&v)[8], const float (&a)[8], const float (&b)[8]) {
#pragma unroll
  for (int i = 0; i < 8; i += 2)
    f32x2_unpack(f32x2_fma(f32x2_pack(v[i], v[i + 1]), f32x2_pack(a[i], a[i + 1]), f32x2_pack(b[i], b[i + 1])), v[i],
                 v[i + 1]);
}
// s += v a; paired
__device__ __forceinline__ void acc8(float (&s)[8], const float (&v)[8], const float (&a)[8]) {
#pragma unroll
  for (int i = 0; i < 8; i += 2)
    f32x2_unpack(f32x2_fma(f32x2_pack(v[i], v[i + 1]), f32x2_pack(a[i], a[i + 1]), f32x2_pack(s[i], s[i + 1])), s[i],
                 s[i + 1]);
}
__device__ __forceinline__ float dot8(const float (&v)[8], const float (&a)[8]) {
  unsigned long long q = f32x2_mul(f32x2_pack(v[0], v[1]), f32x2_pack(a[0], a[1]));
#pragma unroll
  for (int i = 2; i < 8; i += 2) q = f32x2_fma(f32x2_pack(v[i], v[i + 1]), f32x2_pack(a[i], a[i + 1]), q);
  float x, y;
  f32x2_unpack(q, x, y);
  return x + y;
}
__device__ __forceinline__ void copy8(float (&y)[8], const float (&v)[8]) {
#pragma unroll
  for (int i = 0; i < 8; ++i) y[i] = v[i];
}

// ---------------------------------------------------------------------------
// A warp's ring of row pieces: its columns of every tensor, `depth` rows ahead, by bulk
// copies. Rows that are not on a 16-byte boundary are copied from the boundary before
// to the one behind, which are the row's neighbours' bytes; the first and the last row, whose
// neighbours are not the tensor's, come element by element.
// ---------------------------------------------------------------------------
template <bool WHOLE>
struct RowRing {
  uint8_t* base;
  uint64_t* bars;
  int depth, mine, c0, slot;
  uint32_t stage, phase;

  __device__ __forceinline__ void init(uint8_t* smem, uint64_t* b, const RingPlan& plan, int first_column, int columns) {
    base = smem;
    bars = b;
    depth = plan.depth;
    stage = plan.stage;
    c0 = first_column;
    mine = columns;
    slot = 0;
    phase = 0;
    if ((threadIdx.x & 31) == 0)
      for (int s = 0; s < depth; ++s) mbar_init(&bars[s], 1);
    fence_mbar_init();
  }
  __device__ __forceinline__ static uint32_t shift(const RowStream& t, size_t row, int c0) {
    return WHOLE ? 0u : (uint32_t)(reinterpret_cast<uintptr_t>(t.p) + row * t.pitch + (size_t)c0 * t.e) & 15u;
  }
  // Row `row` into stage s. All lanes call it.
  __device__ __forceinline__ void fetch(const RingPlan& plan, long long row, int s, int M) {
    if (mine <= 0) return;
    const int lane = threadIdx.x & 31;
    uint8_t* dst = base + (size_t)s * stage;
    if (!WHOLE && (row == 0 || row == M - 1)) {
      for (int i = 0; i < plan.n; ++i) {
        const RowStream& t = plan.t[i];
        const uint8_t* src = t.p + (size_t)row * t.pitch + (size_t)c0 * t.e;
        uint8_t* to = dst + t.at + shift(t, (size_t)row, c0);
        for (int c = lane; c < mine; c += 32) {
          if (t.e == 4) reinterpret_cast<float*>(to)[c] = reinterpret_cast<const float*>(src)[c];
          else if (t.e == 2) reinterpret_cast<uint16_t*>(to)[c] = reinterpret_cast<const uint16_t*>(src)[c];
          else to[c] = src[c];
        }
      }
      __syncwarp();
      if (lane == 0) mbar_arrive(&bars[s]);
      return;
    }
    if (lane != 0) return;
    uint32_t total = 0;
    for (int i = 0; i < plan.n; ++i) {
      const RowStream& t = plan.t[i];
      total += (shift(t, (size_t)row, c0) + (uint32_t)mine * t.e + 15u) & ~15u;
    }
    mbar_arrive_expect_tx(&bars[s], total);
    for (int i = 0; i < plan.n; ++i) {
      const RowStream& t = plan.t[i];
      const uint32_t sh = shift(t, (size_t)row, c0);
      bulk_load(dst + t.at, t.p + (size_t)row * t.pitch + (size_t)c0 * t.e - sh, (sh + (uint32_t)mine * t.e + 15u) & ~15u,
                &bars[s]);
    }
  }
  __device__ __forceinline__ bool wait(volatile int* abort_flag, unsigned* err) {
    return mine <= 0 || mbar_wait(&bars[slot], phase, abort_flag, err);
  }
  __device__ __forceinline__ const uint8_t* row() const { return base + (size_t)slot * stage; }
  // The row has been read by every lane: its stage takes the row `ahead`, if there is one.
  __device__ __forceinline__ void next(const RingPlan& plan, long long ahead, long long end, int M, bool dead) {
    __syncwarp();
    if (!dead && ahead < end) {
      fence_proxy_async_smem();
      fetch(plan, ahead, slot, M);
    }
    if (++slot == depth) {
      slot = 0;
      phase ^= 1u;
    }
  }
};

}  // namespace

// Ranges of consecutive rows, one for each team (the warps that work on a row together).
__host__ __device__ __forceinline__ long long team_start(int M, int teams, int t) { return (long long)M * t / teams; }
__host__ __device__ __forceinline__ int team_of(int M, int teams, long long row) {
  return (int)(((row + 1) * teams - 1) / M);
}

}  // namespace lm
