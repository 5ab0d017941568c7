// What the residual join's kernels share: rows that stream through shared memory, a
// lane's columns of them, and the sums over a row's warps.
#pragma once

#include "join.cuh"
#include "rows.cuh"

namespace lm {

// The tensors whose rows a warp's ring holds, as the host lays them out.
// Row r of the call is row r / group of the tensor, for 0 <= r < 2^31 the upper bits of r * magic: with
// 2^(l-1) < group <= 2^l and magic = floor(2^(31+l) / group) + 1 < 2^32, r * magic / 2^(31+l) exceeds r / group by
// less than r / 2^(31+l) < 1 / group.
struct RowStream {
  const uint8_t* p;
  size_t pitch;    // bytes from row to row
  uint32_t at;     // place in a stage
  uint32_t e;      // bytes of an element
  uint32_t magic, shift;
};
__device__ __forceinline__ unsigned stream_row(uint32_t magic, uint32_t shift, int row) {
  return (unsigned)(((unsigned long long)(unsigned)row * magic) >> shift);
}
constexpr int kMostStreams = 6;
constexpr int kMostStages = 8;
struct RingPlan {
  RowStream t[kMostStreams];
  int n;
  int depth;        // stages of a warp's ring
  uint32_t stage;   // bytes of a stage
};

namespace {

// Waits for the WPR warps of a row, one of GROUPS teams of the CTA: barriers 1 .. 15, because 0 is __syncthreads's,
// with another number of threads. (With a number known at run time a CTA would be given all 16
// barriers, and an SM's 64 would limit it to four CTAs.)
template <int WPR, int GROUPS>
__device__ __forceinline__ void row_barrier(int grp) {
  static_assert(WPR == 1 || GROUPS <= 15, "a barrier for each team");
#define LM_BAR(i) case i: asm volatile("bar.sync %0, %1;" ::"n"(i < GROUPS ? i + 1 : 1), "n"(WPR * 32) : "memory"); break;
  switch (GROUPS == 1 ? 0 : grp) {
    LM_BAR(0) LM_BAR(1) LM_BAR(2) LM_BAR(3) LM_BAR(4) LM_BAR(5) LM_BAR(6) LM_BAR(7)
    LM_BAR(8) LM_BAR(9) LM_BAR(10) LM_BAR(11) LM_BAR(12) LM_BAR(13) LM_BAR(14)
  }
#undef LM_BAR
}

// ---------------------------------------------------------------------------
// A lane's eight columns of a chunk of 256
// ---------------------------------------------------------------------------
// Whole rows (WHOLE: on boundaries of eight elements, D a multiple of eight): eight
// consecutive columns, all there or none, half a warp a block of 128: one access a tensor (fp32 from
// shared memory two, with two-way bank conflicts) and one block's scale a lane. With four columns of each of
// two blocks a lane, 40960 x 1024 with three 8-bit outputs took 539 instructions a warp and row. Other rows:
// every 32nd column, values 0..3 of the first block, 4..7 of the second.
template <bool WHOLE>
struct Columns {
  int c0;     // first column of the chunk
  int left;   // columns that the chunk has from the lane's first one on
  bool full;  // all 256

  __device__ __forceinline__ Columns(int chunk, int D)
      : c0(chunk), left(D - chunk - (WHOLE ? 8 : 1) * (int)(threadIdx.x & 31)), full(chunk + kChunk <= D) {}
  __device__ __forceinline__ int first() const { return c0 + (WHOLE ? 8 : 1) * (int)(threadIdx.x & 31); }
  __device__ __forceinline__ bool on(int k) const { return (WHOLE ? 0 : 32 * k) < left; }
  __device__ __forceinline__ void mask(float (&v)[8]) const {
    if (full) return;  // (uniform over the warp)
#pragma unroll
    for (int k = 0; k < 8; ++k)
      if (!on(k)) v[k] = 0.f;
  }
};
__device__ __forceinline__ size_t row_offset(unsigned row, int ld) { return (size_t)row * (unsigned)ld; }

// A chunk that a lane keeps its eight values of in shared memory: two accesses without bank conflicts.
constexpr int kLaneChunk = kChunk;  // floats
__device__ __forceinline__ void lane_put(float* m, const float (&v)[8]) {
  float4* p = reinterpret_cast<float4*>(m) + (threadIdx.x & 31);
  p[0] = make_float4(v[0], v[1], v[2], v[3]);
  p[32] = make_float4(v[4], v[5], v[6], v[7]);
}
__device__ __forceinline__ void lane_get(const float* m, float (&v)[8]) {
  const float4* p = reinterpret_cast<const float4*>(m) + (threadIdx.x & 31);
  const float4 a = p[0], b = p[32];
  v[0] = a.x; v[1] = a.y; v[2] = a.z; v[3] = a.w;
  v[4] = b.x; v[5] = b.y; v[6] = b.z; v[7] = b.w;
}
// The column, from the chunk's first one, that place i of such a chunk is of.
template <bool WHOLE>
__device__ __forceinline__ int lane_column(int i) {
  const int lane = (i & 127) >> 2, k = (i >> 7) * 4 + (i & 3);
  return WHOLE ? 8 * lane + k : 32 * k + lane;
}

// From global memory: a row of fp32 or bf16; columns from D on read as zero.
template <bool WHOLE, typename T>
__device__ __forceinline__ void load_columns(const T* p, const Columns<WHOLE>& c, float (&v)[8]) {
#pragma unroll
  for (int k = 0; k < 8; ++k) v[k] = 0.f;
  if (WHOLE) {
    if (c.on(0)) ld8a(p, v);
  } else if (c.full) {
#pragma unroll
    for (int k = 0; k < 8; ++k) v[k] = to_f(p[32 * k]);
  } else {
#pragma unroll
    for (int k = 0; k < 8; ++k)
      if (c.on(k)) v[k] = to_f(p[32 * k]);
  }
}
template <bool WHOLE>
__device__ __forceinline__ void load_row(const void* base, int ld, int dtype, unsigned row, const Columns<WHOLE>& c,
                                         float (&v)[8]) {
  const size_t at = row_offset(row, ld) + c.first();
  if (dtype == LAZYMAR_F32) load_columns<WHOLE>(static_cast<const float*>(base) + at, c, v);
  else load_columns<WHOLE>(static_cast<const bf16*>(base) + at, c, v);
}
template <bool WHOLE>
__device__ __forceinline__ void load_row(const Rows& m, unsigned row, const Columns<WHOLE>& c, float (&v)[8]) {
  load_row<WHOLE>(m.p, m.ld, m.dtype, row, c, v);
}
template <bool WHOLE>
__device__ __forceinline__ void load_param(const float* p, const Columns<WHOLE>& c, float (&v)[8]) {
  load_columns<WHOLE>(p + c.first(), c, v);
}
template <bool WHOLE>
__device__ __forceinline__ void store_row(const MatOut& m, unsigned row, const Columns<WHOLE>& c, const float (&v)[8]) {
  const size_t at = row_offset(row, m.ld) + c.first();
  if (m.dtype == LAZYMAR_F32) {
    float* p = static_cast<float*>(m.p) + at;
    if (WHOLE) {
      if (c.on(0)) st8a(p, v);
    } else if (c.full) {
#pragma unroll
      for (int k = 0; k < 8; ++k) p[32 * k] = v[k];
    } else {
#pragma unroll
      for (int k = 0; k < 8; ++k)
        if (c.on(k)) p[32 * k] = v[k];
    }
  } else {
    bf16* p = static_cast<bf16*>(m.p) + at;
    if (WHOLE) {
      if (c.on(0)) st8a(p, v);
    } else {
      uint16_t* q = reinterpret_cast<uint16_t*>(p);
      if (c.full) {
#pragma unroll
        for (int k = 0; k < 8; k += 2) {
          const uint32_t two = pack_bf16(v[k], v[k + 1]);
          q[32 * k] = (uint16_t)two;
          q[32 * (k + 1)] = (uint16_t)(two >> 16);
        }
      } else {
#pragma unroll
        for (int k = 0; k < 8; k += 2) {
          const uint32_t two = pack_bf16(v[k], v[k + 1]);
          if (c.on(k)) q[32 * k] = (uint16_t)two;
          if (c.on(k + 1)) q[32 * (k + 1)] = (uint16_t)(two >> 16);
        }
      }
    }
  }
}
__device__ __forceinline__ void copy8(float (&y)[8], const float (&v)[8]) {
#pragma unroll
  for (int i = 0; i < 8; ++i) y[i] = v[i];
}
// To block8. Columns from D on hold zero.
template <bool WHOLE>
__device__ __forceinline__ void store_row8(const lazymar_block8& o, unsigned row, const Columns<WHOLE>& c, const float (&v)[8]) {
  const int lane = threadIdx.x & 31;
  uint8_t* q = static_cast<uint8_t*>(o.q) + row_offset(row, o.ldq) + c.first();
  if constexpr (WHOLE) {
    uint2 w;
    const uint32_t byte = block8_quantize(v, w);
    if (c.on(0)) {
      *reinterpret_cast<uint2*>(q) = w;
      if ((lane & 15) == 0) o.scale[row_offset((unsigned)(c.c0 / kBlk + (lane >> 4)), o.lds) + row] = (uint8_t)byte;
    }
    return;
  }
  // a block is four values of each lane of the warp
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
    const uint32_t b = e4m3x4(w[4 * j] * s, w[4 * j + 1] * s, w[4 * j + 2] * s, w[4 * j + 3] * s);
#pragma unroll
    for (int i = 0; i < 4; ++i)
      if (c.on(4 * j + i)) q[32 * (4 * j + i)] = (uint8_t)(b >> (8 * i));
  }
  // (lane 0 the first block's scale, lane 1 the second's)
  const uint32_t byte = block8_exp(lane == 0 ? amax[0] : amax[1]);
  if (lane < 2 && kBlk * lane - lane < c.left) o.scale[row_offset((unsigned)(c.c0 / kBlk + lane), o.lds) + row] = (uint8_t)byte;
}
// From a warp's stage. `st`: the row's chunk in it. An 8-bit row's scales: `s`, the lane's own block's where
// rows are whole, otherwise lane 0 has the first block's and lane 1 the second's.
template <bool WHOLE>
__device__ __forceinline__ void load_stage(const uint8_t* st, int dtype, uint32_t s, const Columns<WHOLE>& c, float (&v)[8]) {
  const int lane = threadIdx.x & 31;
  if (dtype == LAZYMAR_F32) {
    if (WHOLE) {
      const float4* p = reinterpret_cast<const float4*>(st) + 2 * lane;
      const float4 a = p[0], b = p[1];
      v[0] = a.x; v[1] = a.y; v[2] = a.z; v[3] = a.w;
      v[4] = b.x; v[5] = b.y; v[6] = b.z; v[7] = b.w;
    } else {
      const float* p = reinterpret_cast<const float*>(st) + lane;
#pragma unroll
      for (int k = 0; k < 8; ++k) v[k] = p[32 * k];
    }
  } else if (dtype == LAZYMAR_BF16) {
    if (WHOLE) {
      bf16x8(reinterpret_cast<const uint4*>(st)[lane], v);
    } else {
      const uint16_t* p = reinterpret_cast<const uint16_t*>(st) + lane;
#pragma unroll
      for (int k = 0; k < 8; ++k) v[k] = __uint_as_float((uint32_t)p[32 * k] << 16);
    }
  } else if (WHOLE) {
    block8_values(reinterpret_cast<const uint2*>(st)[lane], block8_scale(s), v);
  } else {
#pragma unroll
    for (int j = 0; j < 2; ++j) {
      const float t = block8_scale(__shfl_sync(0xffffffffu, s, j));
      uint32_t w = 0;
#pragma unroll
      for (int i = 0; i < 4; ++i) w |= (uint32_t)st[kBlk * j + 32 * i + lane] << (8 * i);
      const float2 a = e4m3x2_to_f2(w & 0xFFFFu), b = e4m3x2_to_f2(w >> 16);
      v[4 * j] = a.x * t; v[4 * j + 1] = a.y * t; v[4 * j + 2] = b.x * t; v[4 * j + 3] = b.y * t;
    }
  }
  c.mask(v);
}
// Where a lane finds the scales of its chunk of an 8-bit tensor (row by row), as load_stage takes them.
template <bool WHOLE>
__device__ __forceinline__ const uint8_t* scales_of(const Rows& m, int c0, int D) {
  const int lane = threadIdx.x & 31, j = WHOLE ? lane >> 4 : lane;
  if (!m.p || m.dtype != LAZYMAR_E4M3 || j > 1 || c0 + kBlk * j >= D) return nullptr;
  return m.scale + row_offset((unsigned)(c0 / kBlk + j), m.lds);
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

// 1 / sqrt(a) with a Newton step, r += r (1 - a r^2) / 2, which takes rsqrtf's error (up to two steps of fp32) out of a normed
// row: three instructions. Over 40960 x 1024 normed and modulated values the relative error fell from 6.5e-8 to 6.2e-8.
__device__ __forceinline__ float inv_sqrt(float a) {
  const float r = rsqrtf(a);
  return r > 0.f ? fmaf(0.5f * r, fmaf(-a * r, r, 1.f), r) : r;  // (squares that have left fp32's range give 0)
}

// ---------------------------------------------------------------------------
// A warp's ring of row pieces: its columns of every tensor, `depth` rows ahead, by bulk
// copies, one lane a tensor. Pieces that are not on 16-byte boundaries are copied from the
// boundary before to the one behind, which are the row's neighbours' bytes; where those are not the
// tensor's (before its first element, behind its last: rows of a few bytes have several such, and so has a row whose last
// piece is of a few bytes), the piece comes element by element.
// ---------------------------------------------------------------------------
// DIVIDED: some tensors have a row for each group of rows; otherwise a lane's pointer moves on by a row each time.
template <bool WHOLE, bool DIVIDED>
struct RowRing {
  uint8_t* base;
  uint64_t* bars;
  int mine, slot;
  uint32_t phase;
  // this lane's tensor: the piece of row 0 or of the row to be fetched next, bytes from row to row
  // and of a row, those of all tensors
  uintptr_t src;
  size_t pitch;
  uint32_t bytes, total, magic, shift;
  uintptr_t lowest, tensor_end;  // where the tensor's first row starts, and where its last one ends

  // first: the first row that will be fetched; step: from one to the next
  __device__ __forceinline__ void init(uint8_t* smem, uint64_t* b, const RingPlan& plan, int first_column, int columns, int M, int D,
                                       int first, int step = 1) {
    const int lane = threadIdx.x & 31;
    base = smem;
    bars = b;
    mine = columns;
    slot = 0;
    phase = 0;
    bytes = 0;
    if (lane < plan.n) {
      const RowStream& t = plan.t[lane];
      src = reinterpret_cast<uintptr_t>(t.p) + (size_t)first_column * t.e;
      pitch = t.pitch;
      magic = t.magic;
      shift = t.shift;
      bytes = (uint32_t)max(mine, 0) * t.e;
      lowest = reinterpret_cast<uintptr_t>(t.p);
      tensor_end = rows_end(lowest, stream_row(magic, shift, M - 1), pitch, D, t.e);
      if (!DIVIDED) {
        src += (size_t)(unsigned)first * pitch;
        pitch *= (unsigned)step;
      }
    }
    if (WHOLE) {
      bytes = (bytes + 15u) & ~15u;
      total = __reduce_add_sync(0xffffffffu, bytes);
    }
    if (lane == 0)
      for (int s = 0; s < plan.depth; ++s) mbar_init(&bars[s], 1);
    fence_mbar_init();
  }
  // Row `row` into stage s. All lanes call it.
  __device__ __forceinline__ void fetch(const RingPlan& plan, int row, int s, int first_column) {
    if (mine <= 0) return;
    const int lane = threadIdx.x & 31;
    uint8_t* dst = base + (uint32_t)s * plan.stage;
    uintptr_t p = src;
    if (DIVIDED) p += (size_t)stream_row(magic, shift, row) * pitch;
    else src += pitch;
    uint32_t n = bytes, sum = total;
    bool copies = lane < plan.n;
    if (!WHOLE) {
      const bool outside = copies && piece_reaches_out(p, bytes, lowest, tensor_end);
      for (unsigned them = __ballot_sync(0xffffffffu, outside); them; them &= them - 1) {
        const RowStream& t = plan.t[__ffs((int)them) - 1];
        const uint8_t* from = t.p + (size_t)stream_row(t.magic, t.shift, row) * t.pitch + (size_t)first_column * t.e;
        uint8_t* to = dst + t.at + (reinterpret_cast<uintptr_t>(from) & 15u);
        for (int c = lane; c < mine; c += 32) {
          if (t.e == 4) reinterpret_cast<float*>(to)[c] = reinterpret_cast<const float*>(from)[c];
          else if (t.e == 2) reinterpret_cast<uint16_t*>(to)[c] = reinterpret_cast<const uint16_t*>(from)[c];
          else to[c] = from[c];
        }
      }
      copies = copies && !outside;
      n = copies ? (((uint32_t)p & 15u) + bytes + 15u) & ~15u : 0u;
      p &= ~(uintptr_t)15;
      sum = __reduce_add_sync(0xffffffffu, n);
      __syncwarp();
    }
    if (lane == 0) mbar_arrive_expect_tx(&bars[s], sum);
    __syncwarp();
    if (copies) bulk_load(dst + plan.t[lane].at, reinterpret_cast<const void*>(p), n, &bars[s]);
  }
  __device__ __forceinline__ bool wait(volatile int* abort_flag, unsigned* err) {
    return mine <= 0 || mbar_wait(&bars[slot], phase, abort_flag, err);
  }
  // Tensor i's piece of the row that has come.
  __device__ __forceinline__ const uint8_t* piece(const RingPlan& plan, int i, int row, int first_column) const {
    const RowStream& t = plan.t[i];
    const uint8_t* st = base + (uint32_t)slot * plan.stage + t.at;
    if (WHOLE) return st;
    return st + (((uint32_t)reinterpret_cast<uintptr_t>(t.p) + (uint32_t)first_column * t.e +
                  (DIVIDED ? stream_row(t.magic, t.shift, row) : (uint32_t)row) * (uint32_t)t.pitch) & 15u);
  }
  // The row has been read by every lane: its stage takes row `ahead`, if there is one.
  __device__ __forceinline__ void next(const RingPlan& plan, int ahead, int end, int first_column, bool dead) {
    __syncwarp();
    if (!dead && ahead < end) {
      fence_proxy_async_smem();
      fetch(plan, ahead, slot, first_column);
    }
    if (++slot == plan.depth) {
      slot = 0;
      phase ^= 1u;
    }
  }
};

// After a wait that ran out: waits, with a limit (500 tries of a millisecond a stage), for the warp's copies that are under way, so
// that none of them writes to shared memory that is another's by then. A stage's phase that has not ended is that of
// such a copy, or of none: then the limit runs out. (The loop over the rows keeps no account of it, not even its place among
// the CTA's rings, `all`: one register more there spilled, and took the gradient of 40960 x 1280 from 142 to 151 us.)
__device__ __forceinline__ void drain_ring(const RingPlan& plan, uint64_t (*all)[kMostStages]) {
  uint32_t thread;
  asm volatile("mov.u32 %0, %%tid.x;" : "=r"(thread));
  uint64_t* const bars = all[thread >> 5];
  for (int s = 0; s < plan.depth; ++s) {
    const uint32_t now = mbar_try_wait<false>(&bars[s], 0u) ? 1u : 0u;  // (a phase of parity 0 has ended: this one's is 1)
    for (int i = 0; i < 500 && !mbar_try_wait(&bars[s], now); ++i) {}
  }
}

}  // namespace

inline bool on_eight(const Rows& r) { return !r.p || r.vec; }
inline bool on_eight(const MatOut& r) { return !r.p || r.vec; }

// The streams of a launch; stages for as many rows as `room` bytes hold for a CTA's warps, four at most.
inline void add_stream(RingPlan& plan, const Rows& r, int columns, int group = 1) {
  if (!r.p) return;
  const uint32_t e = r.dtype == LAZYMAR_F32 ? 4 : r.dtype == LAZYMAR_BF16 ? 2 : 1;
  int l = 0;
  while (l < 31 && (1u << l) < (unsigned)group) ++l;
  plan.t[plan.n++] = RowStream{static_cast<const uint8_t*>(r.p), (size_t)r.ld * e, plan.stage, e,
                               (uint32_t)((1ull << (31 + l)) / (unsigned)group + 1), (uint32_t)(31 + l)};
  plan.stage += (uint32_t)columns * e + 32;
}
inline void set_depth(RingPlan& plan, int room, int warps) {
  plan.depth = room / (warps * (int)plan.stage);
  if (plan.depth > 4) plan.depth = 4;
}

// Warps of a row of D columns, and of a CTA: whole teams, one CTA an SM, so that parameters are in
// shared memory once, and that the SM's four schedulers have as many warps each (with CTAs of one team of
// five warps 40960 x 1280 took 200 us where this took 154).
inline int row_warps(int D) {
  const int nc = (D + kChunk - 1) / kChunk;
  return nc <= 5 ? nc : nc <= 8 ? 8 : 16;
}
constexpr int cta_warps(int wpr, int warps) { return warps < wpr ? wpr : warps / wpr * wpr; }
constexpr int kSmemRoom = 215 * 1024;  // of a CTA

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
