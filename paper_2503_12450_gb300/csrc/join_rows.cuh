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
struct Columns {
  int c0;     // first column of the chunk
  int left;   // columns that the chunk has from the lane's first one on
  bool full;  // all 256

  __device__ __forceinline__ Columns(int chunk, int D)
      : c0(chunk), left(D - chunk - (WHOLE ? 4 : 1) * (int)(threadIdx.x & 31)), full(chunk + kChunk <= D) {}
  __device__ __forceinline__ int first() const { return c0 + (WHOLE ? 4 : 1) * (int)(threadIdx.x & 31); }
  // From the lane's first column to its k-th.
  __device__ __forceinline__ static constexpr int offset(int k) { return WHOLE ? kBlk * (k >> 2) + (k & 3) : 32 * k; }
  __device__ __forceinline__ bool on(int k) const { return offset(k) < left; }
  __device__ __forceinline__ void mask(float (&v)[8]) const {
    if (full) return;  // (uniform over the warp)
#pragma unroll
    for (int k = 0; k < 8; ++k)
      if (!on(k)) v[k] = 0.f;
  }
};
__device__ __forceinline__ void widen4(uint2 u, float* v) {
  v[0] = __uint_as_float(u.x << 16);
  v[1] = __uint_as_float(u.x & 0xFFFF0000u);
  v[2] = __uint_as_float(u.y << 16);
  v[3] = __uint_as_float(u.y & 0xFFFF0000u);
}
__device__ __forceinline__ void put4(float4 a, float* v) {
  v[0] = a.x; v[1] = a.y; v[2] = a.z; v[3] = a.w;
}
__device__ __forceinline__ size_t row_offset(unsigned row, int ld) { return (size_t)row * (unsigned)ld; }

// From global memory: a row of fp32 or bf16; columns from D on read as zero.
template <bool WHOLE>
__device__ __forceinline__ void load_row(const void* base, int ld, int dtype, unsigned row, const Columns<WHOLE>& c,
                                         float (&v)[8]) {
  const size_t at = row_offset(row, ld) + c.first();
#pragma unroll
  for (int k = 0; k < 8; ++k) v[k] = 0.f;
  if (dtype == LAZYMAR_F32) {
    const float* p = static_cast<const float*>(base) + at;
    if (WHOLE) {
      if (c.on(0)) put4(*reinterpret_cast<const float4*>(p), v);
      if (c.on(4)) put4(*reinterpret_cast<const float4*>(p + kBlk), v + 4);
    } else {
#pragma unroll
      for (int k = 0; k < 8; ++k)
        if (c.on(k)) v[k] = p[32 * k];
    }
  } else {
    const bf16* p = static_cast<const bf16*>(base) + at;
    if (WHOLE) {
      if (c.on(0)) widen4(*reinterpret_cast<const uint2*>(p), v);
      if (c.on(4)) widen4(*reinterpret_cast<const uint2*>(p + kBlk), v + 4);
    } else {
#pragma unroll
      for (int k = 0; k < 8; ++k)
        if (c.on(k)) v[k] = to_f(p[32 * k]);
    }
  }
}
template <bool WHOLE>
__device__ __forceinline__ void load_row(const Rows& m, unsigned row, const Columns<WHOLE>& c, float (&v)[8]) {
  load_row<WHOLE>(m.p, m.ld, m.dtype, row, c, v);
}
template <bool WHOLE>
__device__ __forceinline__ void load_param(const float* p, const Columns<WHOLE>& c, float (&v)[8]) {
  load_row<WHOLE>(p, 0, LAZYMAR_F32, 0u, c, v);
}
template <bool WHOLE>
__device__ __forceinline__ void store_row(const MatOut& m, unsigned row, const Columns<WHOLE>& c, const float (&v)[8]) {
  const size_t at = row_offset(row, m.ld) + c.first();
  if (m.dtype == LAZYMAR_F32) {
    float* p = static_cast<float*>(m.p) + at;
    if (WHOLE) {
      if (c.on(0)) *reinterpret_cast<float4*>(p) = make_float4(v[0], v[1], v[2], v[3]);
      if (c.on(4)) *reinterpret_cast<float4*>(p + kBlk) = make_float4(v[4], v[5], v[6], v[7]);
    } else {
#pragma unroll
      for (int k = 0; k < 8; ++k)
        if (c.on(k)) p[32 * k] = v[k];
    }
  } else {
    bf16* p = static_cast<bf16*>(m.p) + at;
    if (WHOLE) {
      if (c.on(0)) *reinterpret_cast<uint2*>(p) = make_uint2(pack_bf16(v[0], v[1]), pack_bf16(v[2], v[3]));
      if (c.on(4)) *reinterpret_cast<uint2*>(p + kBlk) = make_uint2(pack_bf16(v[4], v[5]), pack_bf16(v[6], v[7]));
    } else {
#pragma unroll
      for (int k = 0; k < 8; k += 2) {
        const uint32_t two = pack_bf16(v[k], v[k + 1]);
        uint16_t* q = reinterpret_cast<uint16_t*>(p);
        if (c.on(k)) q[32 * k] = (uint16_t)two;
        if (c.on(k + 1)) q[32 * (k + 1)] = (uint16_t)(two >> 16);
      }
    }
  }
}
__device__ __forceinline__ void copy8(float (&y)[8], const float (&v)[8]) {
#pragma unroll
  for (int i = 0; i < 8; ++i) y[i] = v[i];
}
// To block8: a block is four values of each lane of the warp. Columns from D on hold zero.
template <bool WHOLE>
__device__ __forceinline__ void store_row8(const lazymar_block8& o, unsigned row, const Columns<WHOLE>& c, const float (&v)[8]) {
  const int lane = threadIdx.x & 31;
  uint8_t* q = static_cast<uint8_t*>(o.q) + row_offset(row, o.ldq) + c.first();
  uint32_t amax[2];
#pragma unroll
  for (int j = 0; j < 2; ++j)
    amax[j] = __reduce_max_sync(0xffffffffu, __float_as_uint(fmaxf(fmaxf(fabsf(v[4 * j]), fabsf(v[4 * j + 1])),
                                                                   fmaxf(fabsf(v[4 * j + 2]), fabsf(v[4 * j + 3])))));
  float w[8];
  copy8(w, v);
  if (max(amax[0], amax[1]) >= 0x7F800000u) {  // an infinity: the finite values' maxima
#pragma unroll
    for (int j = 0; j < 2; ++j) {
      float m = 0.f;
#pragma unroll
      for (int i = 4 * j; i < 4 * j + 4; ++i) {
        m = fmaxf(m, fabsf(nonfinite_to(w[i], 0.f)));
        w[i] = nonfinite_to(w[i], __uint_as_float(0x7FC00000u));
      }
      amax[j] = __reduce_max_sync(0xffffffffu, __float_as_uint(m));
    }
  }
#pragma unroll
  for (int j = 0; j < 2; ++j) {
    const float s = block8_inv(block8_exp(amax[j]));
    const unsigned long long ss = f32x2_pack(s, s);
    f32x2_unpack(f32x2_mul(f32x2_pack(w[4 * j], w[4 * j + 1]), ss), w[4 * j], w[4 * j + 1]);
    f32x2_unpack(f32x2_mul(f32x2_pack(w[4 * j + 2], w[4 * j + 3]), ss), w[4 * j + 2], w[4 * j + 3]);
    const uint32_t b = e4m3x4(w[4 * j], w[4 * j + 1], w[4 * j + 2], w[4 * j + 3]);
    if (WHOLE) {
      if (c.on(4 * j)) *reinterpret_cast<uint32_t*>(q + kBlk * j) = b;
    } else {
#pragma unroll
      for (int i = 0; i < 4; ++i)
        if (c.on(4 * j + i)) q[32 * (4 * j + i)] = (uint8_t)(b >> (8 * i));
    }
  }
  // (lane 0 the first block's scale, lane 1 the second's)
  const uint32_t byte = block8_exp(lane == 0 ? amax[0] : amax[1]);
  if (lane < 2 && c.c0 + kBlk * lane < c.left + c.first()) o.scale[(size_t)(unsigned)(c.c0 / kBlk + lane) * (unsigned)o.lds + row] = (uint8_t)byte;
}
// From a warp's stage. `st`: the row's chunk in it; s0, s1: the scales of an 8-bit row.
template <bool WHOLE>
__device__ __forceinline__ void load_stage(const uint8_t* st, int dtype, uint32_t s0, uint32_t s1, const Columns<WHOLE>& c,
                                           float (&v)[8]) {
  const int lane = threadIdx.x & 31;
  if (dtype == LAZYMAR_F32) {
    if (WHOLE) {
      const float4* p = reinterpret_cast<const float4*>(st) + lane;
      put4(p[0], v);
      put4(p[32], v + 4);
    } else {
      const float* p = reinterpret_cast<const float*>(st) + lane;
#pragma unroll
      for (int k = 0; k < 8; ++k) v[k] = p[32 * k];
    }
  } else if (dtype == LAZYMAR_BF16) {
    if (WHOLE) {
      const uint2* p = reinterpret_cast<const uint2*>(st) + lane;
      widen4(p[0], v);
      widen4(p[32], v + 4);
    } else {
      const uint16_t* p = reinterpret_cast<const uint16_t*>(st) + lane;
#pragma unroll
      for (int k = 0; k < 8; ++k) v[k] = __uint_as_float((uint32_t)p[32 * k] << 16);
    }
  } else {
    const float s[2] = {block8_scale(s0), block8_scale(s1)};
#pragma unroll
    for (int j = 0; j < 2; ++j) {
      uint32_t w;
      if (WHOLE) {
        w = reinterpret_cast<const uint32_t*>(st)[32 * j + lane];
      } else {
        w = 0;
#pragma unroll
        for (int i = 0; i < 4; ++i) w |= (uint32_t)st[kBlk * j + 32 * i + lane] << (8 * i);
      }
      const float2 a = e4m3x2_to_f2(w & 0xFFFFu), b = e4m3x2_to_f2(w >> 16);
      const unsigned long long ss = f32x2_pack(s[j], s[j]);
      f32x2_unpack(f32x2_mul(f32x2_pack(a.x, a.y), ss), v[4 * j], v[4 * j + 1]);
      f32x2_unpack(f32x2_mul(f32x2_pack(b.x, b.y), ss), v[4 * j + 2], v[4 * j + 3]);
    }
  }
  c.mask(v);
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

// ---------------------------------------------------------------------------
// A warp's ring of row pieces: its columns of every tensor, `depth` rows ahead, by bulk
// copies, one lane a tensor. Rows that are not on a 16-byte boundary are copied from the
// boundary before to the one behind, which are the row's neighbours' bytes; the first and the
// last row, whose neighbours are not the tensor's, come element by element.
// ---------------------------------------------------------------------------
template <bool WHOLE>
struct RowRing {
  uint8_t* base;
  uint64_t* bars;
  int depth, mine, slot, streams;
  uint32_t stage, phase;
  // this lane's tensor: the piece of row 0, bytes from row to row and of a row, its place in a stage
  uintptr_t src;
  size_t pitch;
  uint32_t bytes, at, total;

  __device__ __forceinline__ void init(uint8_t* smem, uint64_t* b, const RingPlan& plan, int first_column, int columns) {
    const int lane = threadIdx.x & 31;
    base = smem;
    bars = b;
    depth = plan.depth;
    stage = plan.stage;
    mine = columns;
    slot = 0;
    phase = 0;
    streams = plan.n;
    bytes = 0;
    if (lane < streams) {
      const RowStream& t = plan.t[lane];
      src = reinterpret_cast<uintptr_t>(t.p) + (size_t)first_column * t.e;
      pitch = t.pitch;
      bytes = (uint32_t)max(mine, 0) * t.e;
      at = t.at;
    }
    if (WHOLE) {
      bytes = (bytes + 15u) & ~15u;
      total = __reduce_add_sync(0xffffffffu, bytes);
    }
    if (lane == 0)
      for (int s = 0; s < depth; ++s) mbar_init(&bars[s], 1);
    fence_mbar_init();
  }
  // Row `row` into stage s. All lanes call it.
  __device__ __forceinline__ void fetch(const RingPlan& plan, int row, int s, int first_column, int M) {
    if (mine <= 0) return;
    const int lane = threadIdx.x & 31;
    uint8_t* dst = base + (uint32_t)s * stage;
    if (!WHOLE && (row == 0 || row == M - 1)) {
      for (int i = 0; i < plan.n; ++i) {
        const RowStream& t = plan.t[i];
        const uint8_t* from = t.p + (size_t)row * t.pitch + (size_t)first_column * t.e;
        uint8_t* to = dst + t.at + (reinterpret_cast<uintptr_t>(from) & 15u);
        for (int c = lane; c < mine; c += 32) {
          if (t.e == 4) reinterpret_cast<float*>(to)[c] = reinterpret_cast<const float*>(from)[c];
          else if (t.e == 2) reinterpret_cast<uint16_t*>(to)[c] = reinterpret_cast<const uint16_t*>(from)[c];
          else to[c] = from[c];
        }
      }
      __syncwarp();
      if (lane == 0) mbar_arrive(&bars[s]);
      return;
    }
    uintptr_t p = src + (size_t)(unsigned)row * pitch;
    uint32_t n = bytes, sum = total;
    if (!WHOLE) {
      n = lane < streams ? (((uint32_t)p & 15u) + bytes + 15u) & ~15u : 0u;
      p &= ~(uintptr_t)15;
      sum = __reduce_add_sync(0xffffffffu, n);
    }
    if (lane == 0) mbar_arrive_expect_tx(&bars[s], sum);
    __syncwarp();
    if (lane < streams) bulk_load(dst + at, reinterpret_cast<const void*>(p), n, &bars[s]);
  }
  __device__ __forceinline__ bool wait(volatile int* abort_flag, unsigned* err) {
    return mine <= 0 || mbar_wait(&bars[slot], phase, abort_flag, err);
  }
  // Tensor i's piece of the row that has come.
  __device__ __forceinline__ const uint8_t* piece(const RingPlan& plan, int i, int row, int first_column) const {
    const RowStream& t = plan.t[i];
    const uint8_t* st = base + (uint32_t)slot * stage + t.at;
    if (WHOLE) return st;
    return st + (((uint32_t)reinterpret_cast<uintptr_t>(t.p) + (uint32_t)first_column * t.e + (uint32_t)row * (uint32_t)t.pitch) & 15u);
  }
  // The row has been read by every lane: its stage takes row `ahead`, if there is one.
  __device__ __forceinline__ void next(const RingPlan& plan, int ahead, int end, int first_column, int M, bool dead) {
    __syncwarp();
    if (!dead && ahead < end) {
      fence_proxy_async_smem();
      fetch(plan, ahead, slot, first_column, M);
    }
    if (++slot == depth) {
      slot = 0;
      phase ^= 1u;
    }
  }
};

}  // namespace

inline bool on_eight(const Rows& r) { return !r.p || r.vec; }
inline bool on_eight(const MatOut& r) { return !r.p || r.vec; }

// The streams of a launch; stages for as many rows as `room` bytes hold for a CTA's warps, four at most.
inline void add_stream(RingPlan& plan, const Rows& r, int columns) {
  if (!r.p) return;
  const uint32_t e = r.dtype == LAZYMAR_F32 ? 4 : r.dtype == LAZYMAR_BF16 ? 2 : 1;
  plan.t[plan.n++] = RowStream{static_cast<const uint8_t*>(r.p), (size_t)r.ld * e, plan.stage, e};
  plan.stage += (uint32_t)columns * e + 32;
}
inline void set_depth(RingPlan& plan, int room, int warps) {
  plan.depth = room / (warps * (int)plan.stage);
  if (plan.depth > 4) plan.depth = 4;
}

// Warps of a row of D columns, warps of a CTA (whole teams, and a multiple of four, so that the SM's four
// schedulers have as many each: with CTAs of five warps 40960 x 1280 took 200 us instead of 154), and CTAs
// on an SM for about `warps` warps there.
inline int row_warps(int D) {
  const int nc = (D + kChunk - 1) / kChunk;
  return nc <= 5 ? nc : nc <= 8 ? 8 : 16;
}
constexpr int cta_warps(int wpr) { return wpr <= 2 ? 4 : wpr % 4 ? 4 * wpr : wpr; }
constexpr int sm_ctas(int wpr, int warps) { return warps / cta_warps(wpr) > 0 ? warps / cta_warps(wpr) : 1; }

// Ranges of consecutive rows, one for each team (the warps that work on a row together).
struct Teams {
  int n, rows, more;  // the first `more` teams have one row more
};
inline Teams teams_of(int M, int most) {
  const int n = M < most ? M : most;
  return Teams{n, M / n, M % n};
}
__host__ __device__ __forceinline__ int team_start(const Teams& t, int i) { return i * t.rows + (i < t.more ? i : t.more); }
__host__ __device__ __forceinline__ int team_of(const Teams& t, int row) {
  const int edge = t.more * (t.rows + 1);
  return row < edge ? row / (t.rows + 1) : t.more + (row - edge) / t.rows;
}

}  // namespace lm
