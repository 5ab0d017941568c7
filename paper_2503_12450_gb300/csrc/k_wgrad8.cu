// The weight gradient from an 8-bit checkpoint (lazymar_block8_wgrad):
//   dw[n, k] (+)= sum_m dy[m, n] x[m, k],  dy bf16, x block8.
//
// The sum runs over tokens, and a checkpoint's scales differ from token to
// token, so the 8-bit tensor cores cannot apply them. But E4M3 times a power of
// two is exact in bf16 (from 2^-130 on; subnormals count): converter warps turn
// the checkpoint's bytes into the bf16 operand in shared memory, and the product
// runs at the bf16 rate without the activation ever being written out in 16 bits.
//
// Both operands are "MN-major" (the reduced axis is the rows of the tensors):
// an operand tile is 64-column pieces of 128-byte rows, one row a token, in the
// 128-byte swizzle, as TMA writes dy and the converters write x.
//
// The tensor cores' fp32 accumulation truncates, which over thousands of tokens
// costs digits (measured 1.0e-6 of the result at 1024 tokens, 1.9e-5 at 16384). So
// every 512 tokens the accumulator is added to fp32 registers of the epilogue
// warps, rounding to nearest, while the next 512 run into the other half of
// tensor memory (2.2e-7 at 20480 tokens; an fp32 library product 8.5e-7).
//
// Measured: 20480 tokens x 4096 x 1024 130 us, 1320 TFLOP/s on 64 of 76 CTA pairs
// (a library's bf16 product at its best: 1901 on all), 135 in long runs. Bound by the converters: 8 warps need 0.29 us for
// a stage's 64 x 128 bytes, the MMAs 0.2 to 0.25.
#include <cuda.h>

#include <cstring>

#include "block8.cuh"

namespace lm {

// k_gemm.cu
bool make_tmap_bf16(CUtensorMap* m, const void* base, uint64_t inner, uint64_t outer, uint64_t pitch_bytes,
                    uint32_t box_inner, uint32_t box_outer, CUtensorMapSwizzle swz);
bool make_tmap_u8(CUtensorMap* m, const void* base, uint64_t inner, uint64_t outer, uint64_t pitch_bytes,
                  uint32_t box_inner, uint32_t box_outer, CUtensorMapSwizzle swz);

namespace w8 {

constexpr int TOK = 64;               // tokens of a pipeline stage
constexpr int STAGES = 4;
constexpr uint32_t PIECE = TOK * 128; // 64 columns of a stage, in bytes
constexpr uint32_t OP_BYTES = 2 * PIECE;  // 128 columns of an operand
// The checkpoint's bytes have a ring of their own, deeper than the operands':
// they are loaded long before the converters get to them, so that an operand
// stage that falls free waits for dy and the conversion at the same time, not for
// a load and then the conversion.
constexpr uint32_t Q_BYTES = TOK * 128;
constexpr int Q_STAGES = 6;
constexpr uint32_t STAGE_BYTES = 2 * OP_BYTES;
constexpr int CHUNK = 8;              // stages between two additions in registers
constexpr int EPI_WARPS = 8, CONV_WARPS = 8, CONV_GROUP = 4;
constexpr uint32_t STG_BYTES = 32 * 128;
constexpr size_t SMEM =
    1024 + STAGES * STAGE_BYTES + Q_STAGES * Q_BYTES + EPI_WARPS * STG_BYTES + Q_STAGES * TOK * 4 + 512;
constexpr int THREADS = 128 + 32 * (EPI_WARPS + CONV_WARPS);  // warps 0 TMA of dy, 1 MMA, 2 scales, 3 TMA of x, 4-11 converters, 12-19 epilogue
// Registers: 640 threads launch with 96.
constexpr int REGS_LAUNCH = 96, REGS_EPI = 168, REGS_CONV = 56, REGS_REST = 32;
static_assert(REGS_EPI * 256 + REGS_CONV * 256 + REGS_REST * 128 <= REGS_LAUNCH * THREADS,
              "the register split must fit what the launch holds");

struct Params {
  const uint8_t* scale;
  int lds;
  float* out;          // dw, or the partial sums [split, N, K]
  long long out_split; // distance between the partial sums of two splits
  int ldo;
  bool accumulate, vec;
  int M, N, K, split, per;  // per: tokens of a split, a multiple of TOK
};

// kind::f16 with bf16 operands, both MN-major (bits 15 and 16).
constexpr uint32_t idesc(int m, int n) {
  return (1u << 4) | (1u << 7) | (1u << 10) | (1u << 15) | (1u << 16) | ((uint32_t)(n >> 3) << 17) |
         ((uint32_t)(m >> 4) << 24);
}
// MN-major tile in the 128-byte swizzle: 64-column pieces PIECE bytes apart
// (leading byte offset), groups of eight token rows 1024 bytes apart (stride
// byte offset).
__device__ __forceinline__ uint64_t desc(uint32_t saddr) {
  return (uint64_t)((saddr >> 4) & 0x3FFFu) | ((uint64_t)(PIECE >> 4) << 16) | ((uint64_t)(1024 >> 4) << 32) |
         ((uint64_t)1 << 46) | ((uint64_t)2 << 61);
}

}  // namespace w8

// PAIR: two CTAs share a tile of 256 rows (n) by 256 columns (k) of dw: each its
// own 128 rows, and each converts 128 of the columns. Otherwise 128 x 128 tiles.
template <bool PAIR>
__global__ void __launch_bounds__(w8::THREADS, 1)
    wgrad8_kernel(const __grid_constant__ CUtensorMap tmY, const __grid_constant__ CUtensorMap tmX, const w8::Params p,
                  unsigned* err) {
  using namespace w8;
  extern __shared__ uint8_t smem_raw[];
  uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
  uint8_t* sA = smem;
  uint8_t* sB = smem + STAGES * OP_BYTES;
  uint8_t* sQ = smem + STAGES * 2 * OP_BYTES;
  uint8_t* sStg = sQ + Q_STAGES * Q_BYTES;
  float* sScale = reinterpret_cast<float*>(sStg + EPI_WARPS * STG_BYTES);
  uint64_t* full = reinterpret_cast<uint64_t*>(sScale + Q_STAGES * TOK);  // dy has come and x is converted
  uint64_t* empty = full + STAGES;
  uint64_t* full_q = empty + STAGES;
  uint64_t* empty_q = full_q + Q_STAGES;
  uint64_t* acc_full = empty_q + Q_STAGES;
  uint64_t* acc_empty = acc_full + 2;
  uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(acc_empty + 2);
  volatile int* abort_flag = reinterpret_cast<volatile int*>(tmem_slot + 1);

  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  constexpr int TM = PAIR ? 256 : 128, TN = PAIR ? 256 : 128;
  const int num_k = (p.K + TN - 1) / TN, tiles = ((p.N + TM - 1) / TM) * num_k, items = tiles * p.split;
  const int rank = PAIR ? (int)cluster_ctarank() : 0;
  const int first = PAIR ? (int)blockIdx.x / 2 : (int)blockIdx.x, step = PAIR ? (int)gridDim.x / 2 : (int)gridDim.x;
  struct Item {
    int n, k, m, stages;  // first row and column of dw, first token, stages of TOK tokens
    int split;
  };
  auto item_at = [&](int i) {
    const int s = i / tiles, t = i - s * tiles;
    const int m = s * p.per, rows = min(p.per, p.M - m);
    return Item{(t / num_k) * TM, (t % num_k) * TN, m, (rows + TOK - 1) / TOK, s};
  };

  if (threadIdx.x == 0) {
    for (int s = 0; s < STAGES; ++s) {
      mbar_init(&full[s], 1 + (PAIR ? 2 * CONV_GROUP : CONV_GROUP));
      mbar_init(&empty[s], 1);
    }
    for (int s = 0; s < Q_STAGES; ++s) {
      mbar_init(&full_q[s], 2);  // the bytes and the scales
      mbar_init(&empty_q[s], CONV_GROUP);
    }
    for (int b = 0; b < 2; ++b) {
      mbar_init(&acc_full[b], 1);
      mbar_init(&acc_empty[b], PAIR ? 2 * EPI_WARPS : EPI_WARPS);
    }
    *abort_flag = 0;
    fence_mbar_init();
    prefetch_tmap(&tmY);
    prefetch_tmap(&tmX);
  }
  if (warp == 1) {
    if (PAIR) {
      tmem_alloc_pair(tmem_slot, 512);
      tmem_relinquish_pair();
    } else {
      tmem_alloc(tmem_slot, 512);
      tmem_relinquish();
    }
  }
  tc_fence_before();
  __syncthreads();
  if (PAIR) cluster_sync();
  tc_fence_after();
  const uint32_t tmem_base = *tmem_slot;
  pdl_wait();
  pdl_trigger();

  if (warp < 4) {
    asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(REGS_REST));
    if (warp == 0 && lane == 0) {
      // ---------------- TMA producer: dy ----------------
      int stage = 0;
      uint32_t phase = 0;
      bool ok = true;
      for (int i = first; i < items && ok; i += step) {
        const Item t = item_at(i);
        for (int s = 0; s < t.stages; ++s) {
          if (!mbar_wait(&empty[stage], phase ^ 1u, abort_flag, err)) { ok = false; break; }
          uint8_t* dst = sA + stage * OP_BYTES;
          const int n = t.n + rank * 128, m = t.m + s * TOK;
          if (PAIR) {
            if (rank == 0) mbar_arrive_expect_tx(&full[stage], 2 * OP_BYTES);
            const uint32_t bar = cluster_map(smem_u32(&full[stage]), 0);
            tma_load_2d_pair(&tmY, bar, dst, n, m);
            tma_load_2d_pair(&tmY, bar, dst + PIECE, n + 64, m);
          } else {
            mbar_arrive_expect_tx(&full[stage], OP_BYTES);
            tma_load_2d(&tmY, &full[stage], dst, n, m);
            tma_load_2d(&tmY, &full[stage], dst + PIECE, n + 64, m);
          }
          if (++stage == STAGES) { stage = 0; phase ^= 1u; }
        }
      }
    } else if (warp == 2) {
      // ---------------- scales of a stage's tokens, as numbers ----------------
      int stage = 0;
      uint32_t phase = 0;
      bool ok = true;
      for (int i = first; i < items && ok; i += step) {
        const Item t = item_at(i);
        const uint8_t* sc = p.scale + (size_t)min((t.k + rank * 128) / kBlk, (p.K - 1) / kBlk) * p.lds;
        uint32_t b0 = sc[min(t.m + lane, p.M - 1)], b1 = sc[min(t.m + 32 + lane, p.M - 1)];
        for (int s = 0; s < t.stages; ++s) {
          const uint32_t c0 = b0, c1 = b1;
          const int next = t.m + (s + 1) * TOK + lane;
          b0 = sc[min(next, p.M - 1)];
          b1 = sc[min(next + 32, p.M - 1)];
          const bool done = mbar_wait(&empty_q[stage], phase ^ 1u, abort_flag, err);
          if (!__all_sync(0xffffffffu, done)) { ok = false; break; }
          sScale[stage * TOK + lane] = block8_scale(c0);
          sScale[stage * TOK + 32 + lane] = block8_scale(c1);
          __syncwarp();
          if (lane == 0) mbar_arrive(&full_q[stage]);
          if (++stage == Q_STAGES) { stage = 0; phase ^= 1u; }
        }
      }
    } else if (warp == 3 && lane == 0) {
      // ---------------- TMA producer: the checkpoint's bytes ----------------
      int stage = 0;
      uint32_t phase = 0;
      bool ok = true;
      for (int i = first; i < items && ok; i += step) {
        const Item t = item_at(i);
        for (int s = 0; s < t.stages; ++s) {
          if (!mbar_wait(&empty_q[stage], phase ^ 1u, abort_flag, err)) { ok = false; break; }
          mbar_arrive_expect_tx(&full_q[stage], Q_BYTES);
          tma_load_2d(&tmX, &full_q[stage], sQ + stage * Q_BYTES, t.k + rank * 128, t.m + s * TOK);
          if (++stage == Q_STAGES) { stage = 0; phase ^= 1u; }
        }
      }
    } else if (warp == 1 && rank == 0) {
      // ---------------- MMA issuer (of a pair: the even CTA's) ----------------
      const bool lead = elect_one();
      auto all = [&](bool ok) { return (bool)__all_sync(0xffffffffu, ok); };
      int stage = 0, buf = 0;
      uint32_t phase = 0, use = 0;
      bool ok = true;
      for (int i = first; i < items && ok; i += step) {
        const int stages = item_at(i).stages;
        for (int s = 0; s < stages; ++s) {
          const bool fresh = s % CHUNK == 0, last = s % CHUNK == CHUNK - 1 || s == stages - 1;
          if (fresh && !(ok = all(mbar_wait(&acc_empty[buf], use ^ 1u, abort_flag, err)))) break;
          if (!(ok = all(mbar_wait(&full[stage], phase, abort_flag, err)))) break;
          tc_fence_after();
          if (lead) {
            const uint64_t a0 = desc(smem_u32(sA + stage * OP_BYTES)), b0 = desc(smem_u32(sB + stage * OP_BYTES));
            const uint32_t d = tmem_base + (uint32_t)(buf * 256);
#pragma unroll
            for (int k = 0; k < TOK / 16; ++k) {  // 16 tokens: 16 rows of 128 bytes
              const uint64_t o = (uint64_t)(k * 16 * 128 >> 4);
              const uint32_t acc = fresh && k == 0 ? 0u : 1u;
              if (PAIR) umma_bf16_pair(d, a0 + o, b0 + o, idesc(TM, TN), acc);
              else umma_bf16(d, a0 + o, b0 + o, idesc(TM, TN), acc);
            }
            if (PAIR) umma_commit_pair(&empty[stage]);
            else umma_commit(&empty[stage]);
            if (last) {
              if (PAIR) umma_commit_pair(&acc_full[buf]);
              else umma_commit(&acc_full[buf]);
            }
          }
          __syncwarp();
          if (last) {
            buf ^= 1;
            if (buf == 0) use ^= 1u;
          }
          if (++stage == STAGES) { stage = 0; phase ^= 1u; }
        }
      }
    }
    __syncwarp();
  } else if (warp < 4 + CONV_WARPS) {
    // ---------------- converters: the checkpoint's bytes to bf16 ----------------
    // Two groups of four warps take the stages in turn, so that one group's
    // waits and fences pass while the other converts. A lane takes eight columns
    // of a token (16 lanes a token of 128 columns), eight tokens a stage. What
    // lies beyond M or K has come as zero bytes.
    asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(REGS_CONV));
    const int cw = (warp - 4) & (CONV_GROUP - 1), group = (warp - 4) / CONV_GROUP;
    const int col = 8 * (lane & 15), t0 = 2 * cw + (lane >> 4);  // tokens t0 + 8 j
    int stage = 0, qstage = 0, turn = 0;
    uint32_t phase = 0, qphase = 0;
    bool ok = true;
    for (int i = first; i < items && ok; i += step) {
      const int stages = item_at(i).stages;
      for (int s = 0; s < stages; ++s, turn ^= 1) {
        if (turn == group) {
          bool done = mbar_wait(&full_q[qstage], qphase, abort_flag, err);
          done = done && mbar_wait(&empty[stage], phase ^ 1u, abort_flag, err);
          if (!__all_sync(0xffffffffu, done)) { ok = false; break; }
          const uint8_t* src = sQ + qstage * Q_BYTES + col;
          const float* sc = sScale + qstage * TOK;
          // row (token) r, 16-byte piece c of its 64 columns at piece c ^ (r & 7)
          uint8_t* dst = sB + stage * OP_BYTES + (col >> 6) * PIECE;
          const int c = ((col >> 3) & 7) ^ (t0 & 7);  // (the same for all of the lane's tokens)
          uint2 w[8];
          float f[8];
#pragma unroll
          for (int j = 0; j < 8; ++j) {
            w[j] = *reinterpret_cast<const uint2*>(src + (t0 + 8 * j) * 128);
            f[j] = sc[t0 + 8 * j];
          }
#pragma unroll
          for (int j = 0; j < 8; ++j) {
            float v[8];
            block8_values(w[j], f[j], v);
            *reinterpret_cast<uint4*>(dst + (t0 + 8 * j) * 128 + (c << 4)) =
                make_uint4(pack_bf16(v[0], v[1]), pack_bf16(v[2], v[3]), pack_bf16(v[4], v[5]), pack_bf16(v[6], v[7]));
          }
          fence_proxy_async_smem();
          __syncwarp();
          if (lane == 0) {
            if (PAIR) arrive_even(&full[stage]);
            else mbar_arrive(&full[stage]);
            mbar_arrive(&empty_q[qstage]);
          }
        }
        if (++stage == STAGES) { stage = 0; phase ^= 1u; }
        if (++qstage == Q_STAGES) { qstage = 0; qphase ^= 1u; }
      }
    }
    __syncwarp();
  } else {
    // ---------------- epilogue ----------------
    asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(REGS_EPI));
    constexpr int COLS = TN / 2;  // columns of a warp: two warps share a lane quarter's rows
    const int quarter = warp & 3, half = (warp - 4 - CONV_WARPS) >> 2;
    uint8_t* stg = sStg + (warp - 4 - CONV_WARPS) * STG_BYTES;
    int buf = 0;
    uint32_t use = 0;
    bool ok = true;
    for (int i = first; i < items && ok; i += step) {
      const Item t = item_at(i);
      float acc[COLS];
#pragma unroll
      for (int c = 0; c < COLS; ++c) acc[c] = 0.f;
      for (int s = 0; s < t.stages; s += CHUNK) {
        const bool done = mbar_wait(&acc_full[buf], use, abort_flag, err);
        if (!__all_sync(0xffffffffu, done)) { ok = false; break; }
        tc_fence_after();
        const uint32_t a = tmem_base + ((uint32_t)(quarter * 32) << 16) + (uint32_t)(buf * 256 + half * COLS);
#pragma unroll
        for (int c = 0; c < COLS; c += 16) {
          uint32_t r[16];
          tmem_ld16(a + c, r);
          tmem_wait_ld_regs(r);
#pragma unroll
          for (int j = 0; j < 16; ++j) acc[c + j] += __uint_as_float(r[j]);
        }
        tc_fence_before();
        __syncwarp();
        if (lane == 0) {
          if (PAIR) arrive_even(&acc_empty[buf]);
          else mbar_arrive(&acc_empty[buf]);
        }
        buf ^= 1;
        if (buf == 0) use ^= 1u;
      }
      if (!ok) break;
      const int n0 = t.n + rank * 128 + quarter * 32, lr0 = lane >> 3, cq = lane & 7;
      float* out = p.out + (size_t)t.split * p.out_split;
#pragma unroll
      for (int c = 0; c < COLS; c += 32) {
        const int k0 = t.k + half * COLS + c, col = k0 + 4 * cq;
        if (k0 >= p.K || n0 >= p.N) break;
        __syncwarp();
#pragma unroll
        for (int j = 0; j < 8; ++j)
          *reinterpret_cast<float4*>(stg + lane * 128 + ((j ^ (lane & 7)) << 4)) =
              make_float4(acc[c + 4 * j], acc[c + 4 * j + 1], acc[c + 4 * j + 2], acc[c + 4 * j + 3]);
        __syncwarp();
#pragma unroll
        for (int q = 0; q < 8; ++q) {
          const int lr = 4 * q + lr0, n = n0 + lr;
          float4 o = *reinterpret_cast<const float4*>(stg + lr * 128 + ((cq ^ (lr & 7)) << 4));
          if (n >= p.N || col >= p.K) continue;
          float* y = out + (size_t)n * p.ldo + col;
          if (p.vec && col + 4 <= p.K) {
            if (p.accumulate) {
              const float4 z = *reinterpret_cast<const float4*>(y);
              o = make_float4(o.x + z.x, o.y + z.y, o.z + z.z, o.w + z.w);
            }
            *reinterpret_cast<float4*>(y) = o;
          } else {
            const float e[4] = {o.x, o.y, o.z, o.w};
#pragma unroll
            for (int j = 0; j < 4; ++j)
              if (col + j < p.K) y[j] = p.accumulate ? y[j] + e[j] : e[j];
          }
        }
      }
    }
  }
  __syncthreads();
  if (PAIR) cluster_sync();
  if (warp == 1) {
    tc_fence_after();
    if (PAIR) tmem_dealloc_pair(tmem_base, 512);
    else tmem_dealloc(tmem_base, 512);
  }
}

// dw (+)= sum of the splits' partial sums [split, N, K], in split order. Threads
// along a row, VEC columns each, and rows by CTA.
template <int VEC>
__global__ void __launch_bounds__(256) wgrad8_sum_kernel(const float* __restrict__ part, int split, float* dw, int lddw,
                                                         int N, int K, bool accumulate) {
  const int col = ((int)blockIdx.x * 256 + (int)threadIdx.x) * VEC;
  const size_t n = (size_t)N * K;
  pdl_wait();
  pdl_trigger();
  if (col >= K) return;
  for (int row = (int)blockIdx.y; row < N; row += (int)gridDim.y) {
    const float* p = part + (size_t)row * K + col;
    float* o = dw + (size_t)row * lddw + col;
    float s[VEC];
#pragma unroll
    for (int i = 0; i < VEC; ++i) s[i] = 0.f;
#pragma unroll 4
    for (int j = 0; j < split; ++j) {
      if constexpr (VEC == 4) {
        const float4 v = *reinterpret_cast<const float4*>(p + (size_t)j * n);
        s[0] += v.x; s[1] += v.y; s[2] += v.z; s[3] += v.w;
      } else {
        s[0] += p[(size_t)j * n];
      }
    }
#pragma unroll
    for (int i = 0; i < VEC; ++i) o[i] = accumulate ? o[i] + s[i] : s[i];
  }
}

cudaError_t wgrad8_sum(const Ctx& c, const float* part, int split, float* dw, int lddw, int N, int K, bool accumulate) {
  const bool vec = K % 4 == 0;
  const unsigned x = (unsigned)((K + 256 * (vec ? 4 : 1) - 1) / (256 * (vec ? 4 : 1))), y = (unsigned)(N < 4096 ? N : 4096);
  return launch_pdl(vec ? wgrad8_sum_kernel<4> : wgrad8_sum_kernel<1>, dim3(x, y), dim3(256), 0, c.stream, part, split, dw,
                    lddw, N, K, accumulate);
}

namespace {

constexpr int kSMs = 152;

// Tiles of 256 x 256 on pairs or 128 x 128 on single CTAs, and in how many parts
// the tokens are summed, by the time that was measured: a stage of 64 tokens 0.39
// us on a pair and 0.36 on a single CTA (a quarter of the work: its
// short MMAs do not hide the stage's hand-over), 6 and 4 us for a launch, 1 us a
// tile, and, if there are parts, 1 us and 0.35 us a MB of partial sums and result. (us
// measured, pairs : single CTAs: 20480 x 4096 x 1024 130 : 238, 3211 x 1000 x 776 in 1, 2
// and 4 parts 27, 20, 17 : 23, 17, 19, 640 x 1024 x 256 11.1 : 7.9, 20480 x 1280 x 1280 in 1 and 3
// parts 128, 56 : 121, 91, 5000 x 5120 x 1280 70 : 94.)
struct Plan {
  bool pair;
  int split, per;
};
Plan plan_wgrad8(int M, int N, int K) {
  Plan best{false, 1, 0};
  double least = 0;
  const long long stages = ((long long)M + w8::TOK - 1) / w8::TOK;
  for (int pair = 0; pair < 2; ++pair) {
    const int t = pair ? 256 : 128, slots = pair ? kSMs / 2 : kSMs;
    const long long tiles = (long long)((N + t - 1) / t) * ((K + t - 1) / t);
    for (int split = 1; split <= 32 && split <= (stages > 0 ? stages : 1); ++split) {
      const long long per = (stages + split - 1) / split;
      if (split > 1 && (split - 1) * per >= stages) continue;  // an empty split
      const double rounds = (double)((tiles * split + slots - 1) / slots);
      const double us = (pair ? 6.0 : 4.0) + rounds * (per * (pair ? 0.39 : 0.36) + 1.0) +
                        (split > 1 ? 1.0 + 0.35e-6 * 4.0 * (split + 1) * N * K : 0.0);
      if (least == 0 || us < least) {
        least = us;
        best = Plan{pair != 0, split, (int)(per * w8::TOK)};
      }
    }
  }
  return best;
}

template <bool PAIR>
cudaError_t prepare_wgrad8() {
  static int ready[64] = {};
  int dev = 0;
  cudaError_t e = cudaGetDevice(&dev);
  if (e != cudaSuccess) return e;
  if (dev >= 0 && dev < 64 && ready[dev]) return cudaSuccess;
  cudaFuncAttributes a;
  if ((e = cudaFuncGetAttributes(&a, wgrad8_kernel<PAIR>)) != cudaSuccess) return e;
  if (a.numRegs < w8::REGS_LAUNCH) return cudaErrorInvalidConfiguration;
  e = cudaFuncSetAttribute(wgrad8_kernel<PAIR>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)w8::SMEM);
  if (e == cudaSuccess && dev >= 0 && dev < 64) ready[dev] = 1;
  return e;
}

}  // namespace

size_t wgrad8_workspace(int M, int N, int K) {
  if (M < 1 || N < 1 || K < 1) return 0;
  const Plan pl = plan_wgrad8(M, N, K);
  return pl.split > 1 ? (size_t)pl.split * N * K * sizeof(float) : 0;
}

cudaError_t launch_wgrad8(const Ctx& c, const Wgrad8& x) {
  using namespace w8;
  const size_t n = (size_t)x.N * x.K;
  if (x.M == 0) {
    if (x.accumulate) return cudaSuccess;
    return wgrad8_sum(c, nullptr, 0, x.dw, x.lddw, x.N, x.K, false);
  }
  const Plan pl = plan_wgrad8(x.M, x.N, x.K);
  CUtensorMap ty, tx;
  if (!make_tmap_bf16(&ty, x.dy, x.N, x.M, (uint64_t)x.lddy * 2, 64, TOK, CU_TENSOR_MAP_SWIZZLE_128B) ||
      !make_tmap_u8(&tx, x.x.q, x.K, x.M, x.x.ldq, 128, TOK, CU_TENSOR_MAP_SWIZZLE_NONE))
    return cudaErrorInvalidValue;
  Params p{};
  p.scale = x.x.scale;
  p.lds = x.x.lds;
  p.M = x.M;
  p.N = x.N;
  p.K = x.K;
  p.split = pl.split;
  p.per = pl.per;
  if (pl.split > 1) {
    p.out = x.ws;
    p.out_split = (long long)n;
    p.ldo = x.K;
    p.vec = x.K % 4 == 0;
  } else {
    p.out = x.dw;
    p.ldo = x.lddw;
    p.accumulate = x.accumulate;
    p.vec = x.lddw % 4 == 0 && (reinterpret_cast<uintptr_t>(x.dw) & 15u) == 0;
  }
  const int t = pl.pair ? 256 : 128, slots = pl.pair ? kSMs / 2 : kSMs;
  const long long items = (long long)((x.N + t - 1) / t) * ((x.K + t - 1) / t) * pl.split;
  const unsigned grid = (unsigned)(items < slots ? items : slots);
  cudaError_t e;
  if (pl.pair) {
    if ((e = prepare_wgrad8<true>()) != cudaSuccess) return e;
    e = launch_pdl_cluster(wgrad8_kernel<true>, dim3(2 * grid), dim3(THREADS), SMEM, 2, c.stream, ty, tx, p, c.err);
  } else {
    if ((e = prepare_wgrad8<false>()) != cudaSuccess) return e;
    e = launch_pdl(wgrad8_kernel<false>, dim3(grid), dim3(THREADS), SMEM, c.stream, ty, tx, p, c.err);
  }
  if (e != cudaSuccess || pl.split == 1) return e;
  return wgrad8_sum(c, x.ws, pl.split, x.dw, x.lddw, x.N, x.K, x.accumulate);
}

}  // namespace lm
