// The block-scaled 8-bit product (lazymar_block8_linear):
//   y[m, n] = sum_k a[m, k] 2^ea[m, k/128] w[n, k] 2^ew[n/128, k/128] + bias[n]
// with E4M3 a and w, fp32 accumulation, and bias, GELU or an fp32 residual,
// fp32, bf16 and / or 8-bit outputs in the epilogue.
//
// The scales are powers of two, so the tensor cores apply them themselves:
// kind::mxf8f6f4 takes one exponent byte per row and 32 columns of K from tensor
// memory, and a block of 128 is four equal ones. A 32-bit column of tensor
// memory holds four bytes a row; here they are the scales of four K blocks of
// 128, and the instruction descriptor names the byte. So the scales of 512
// columns of K are four tensor-memory columns for the 128 rows of a (lane =
// row % 32, column = row / 32, the same in each quarter of the lanes) and eight for
// 256 rows of w, written by tcgen05.st straight from the scale bytes.
//
// Measured: 20480 x 5120 x 1280 with GELU and two 8-bit outputs 111 us (2410 TFLOP/s) in
// short runs and 124 in long ones, 40960 x 1024 x 4096 with fp32 residual and output
// 131 (2620) and 151; without any output 97 and 100 us or so. What bounds it: in a long
// run the 1400 W limit (sw_power_cap active, SM clock 1755 and 1462 MHz of 2070); in a
// short one the MMAs of a stage, 690 cycles alone (512 nominal; the difference is not
// explained) and 900 next to the loads of the next stages and the epilogue, which
// share shared and tensor memory with them.
//
// Accuracy: the accumulator of the tensor cores is fp32 and truncates, so a sum comes
// out too small in magnitude by 6.9e-8 of itself at K = 1280, 3.3e-7 at 5120 and 4e-6
// at 65536 (fp32 additions to nearest: no bias, 6.2e-8 to 6.5e-7 of noise). k_wgrad8.cu
// adds its accumulator to registers every 512 terms; here that would be one more pass
// over tensor memory for each step of an epilogue that the MMAs already wait for, for
// operands that were rounded at 2^-4.
#include <cuda.h>

#include <cstring>

#include "block8.cuh"
#include "linear8_shape.h"

namespace lm {

// k_gemm.cu
bool make_tmap_u8(CUtensorMap* m, const void* base, uint64_t inner, uint64_t outer, uint64_t pitch_bytes,
                  uint32_t box_inner, uint32_t box_outer, CUtensorMapSwizzle swz);

namespace l8 {

constexpr int BM = 128;               // rows of a CTA's tile
constexpr int KB_BYTES = 128;         // K of a pipeline stage: one scale block, one swizzle atom
constexpr uint32_t A_BYTES = BM * KB_BYTES;
constexpr uint32_t B_BYTES = 128 * KB_BYTES;  // rows of w in a CTA's shared memory: the tile's, or a pair's half
constexpr uint32_t STAGE_BYTES = A_BYTES + B_BYTES;
constexpr int EPI_WARPS = 8;
constexpr uint32_t STG_BYTES = 32 * 128;      // one of a warp's two staging buffers: 32 rows of 128 bytes
constexpr uint32_t SCALE_BYTES = 2 * 132 * 4;   // two groups' scales on their way between the scale warps
constexpr uint32_t BIAS_BYTES = EPI_WARPS * 128 * 4;
// Pipeline stages and a warp's staging buffers: 8-bit outputs leave from two
// buffers in turn, the others from one, which makes room for a stage.
constexpr int stages(int out) { return out == 2 ? 4 : 5; }
constexpr int buffers(int out) { return out == 2 ? 2 : 1; }
constexpr size_t smem_bytes(int out) {
  return 1024 + stages(out) * STAGE_BYTES + EPI_WARPS * buffers(out) * STG_BYTES + BIAS_BYTES + SCALE_BYTES + 512;
}
constexpr int THREADS = 512;  // warps 0 TMA, 1 MMA, 4-7 scales, 8-15 epilogue
// Registers: 512 threads launch with 128; the epilogue holds a row's 128 values.
constexpr int REGS_EPI = 208, REGS_REST = 48;
static_assert((REGS_EPI + REGS_REST) * 256 <= 128 * THREADS, "the register split must fit what the launch holds");
// Kinds of output: fp32 or bf16; the same with a residual; 8-bit tensors (and
// fp32 or bf16 next to them).
enum { OUT_PLAIN = 0, OUT_RESIDUAL = 1, OUT_BLOCK8 = 2 };
// Tensor memory: a pair's tile takes 256 columns, and two of them would leave
// none for the scales. So they overlap by 32 columns: tile i starts at column 0
// or 224 in turn, and its MMAs wait for the epilogue of tile i - 1 to have read
// those 32 columns, which it reads first. Single tiles take 128 columns each.
constexpr uint32_t ACC_SECOND = 224;
constexpr int SF_SLOTS = 2;           // scale slots of 16 columns: 4 of a, 8 of w
constexpr uint32_t SF_BASE = 480;     // behind the accumulators
static_assert(ACC_SECOND + 256 <= SF_BASE && SF_BASE + 16 * SF_SLOTS <= 512, "tensor memory has 512 columns");

struct Params {
  const uint8_t *a_scale, *w_scale;
  int lds_a, lds_w;
  int epilogue, M, N, K;
  const float* bias;
  const float* residual;
  int ldr;
  void* out;
  int ldo, out_dtype;
  uint8_t *out8, *u8;  // may be NULL
  int ldout8, ldu8;
  uint8_t *out8_scale, *u8_scale;
  int lds_out8, lds_u8;
  bool bias_vec;
  bool rows_vec;  // rows of out and residual on boundaries of four elements
};

// Instruction descriptor of kind::mxf8f6f4: E4M3 operands (format 0), K-major,
// N / 8 at bit 17, UE8M0 scales (bit 23), M / 16 at bit 24; the byte of the scale
// columns at bit 29 (a) and 4 (w).
__device__ __forceinline__ constexpr uint32_t idesc(int m, int n, uint32_t sf) {
  return (sf << 4) | ((uint32_t)(n >> 3) << 17) | (1u << 23) | ((uint32_t)(m >> 4) << 24) | (sf << 29);
}
template <bool PAIR>
__device__ __forceinline__ void mma(uint32_t d, uint64_t ad, uint64_t bd, uint32_t id, uint32_t sfa, uint32_t sfb,
                                    uint32_t accumulate) {
  if (PAIR)
    asm volatile(
        "{\n\t.reg .pred p;\n\t"
        "setp.ne.b32 p, %6, 0;\n\t"
        "tcgen05.mma.cta_group::2.kind::mxf8f6f4.block_scale.scale_vec::1X [%0], %1, %2, %3, [%4], [%5], p;\n\t}" ::"r"(
            d),
        "l"(ad), "l"(bd), "r"(id), "r"(sfa), "r"(sfb), "r"(accumulate)
        : "memory");
  else
    asm volatile(
        "{\n\t.reg .pred p;\n\t"
        "setp.ne.b32 p, %6, 0;\n\t"
        "tcgen05.mma.cta_group::1.kind::mxf8f6f4.block_scale.scale_vec::1X [%0], %1, %2, %3, [%4], [%5], p;\n\t}" ::"r"(
            d),
        "l"(ad), "l"(bd), "r"(id), "r"(sfa), "r"(sfb), "r"(accumulate)
        : "memory");
}
__device__ __forceinline__ uint64_t sw128_desc(uint32_t saddr) {
  return (uint64_t)((saddr >> 4) & 0x3FFFu) | ((uint64_t)1 << 16) | ((uint64_t)(1024 >> 4) << 32) |
         ((uint64_t)1 << 46) | ((uint64_t)2 << 61);
}
__device__ __forceinline__ void tmem_st4(uint32_t taddr, const uint32_t (&r)[4]) {
  asm volatile("tcgen05.st.sync.aligned.32x32b.x4.b32 [%0], {%1, %2, %3, %4};" ::"r"(taddr), "r"(r[0]), "r"(r[1]),
               "r"(r[2]), "r"(r[3])
               : "memory");
}

// A row's 128 values to E4M3 words and the scale byte. The scale is that of the
// finite values; infinities become NaN (with NaN, apart from the fast path).
__device__ __forceinline__ uint32_t quantize_row(const float (&v)[128], uint32_t (&w)[32]) {
  float m[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
  for (int i = 0; i < 128; i += 8)
#pragma unroll
    for (int j = 0; j < 4; ++j) m[j] = fmaxf(fmaxf(m[j], fabsf(v[i + 2 * j])), fabsf(v[i + 2 * j + 1]));
  uint32_t amax = __float_as_uint(fmaxf(fmaxf(m[0], m[1]), fmaxf(m[2], m[3])));
  const bool special = amax >= 0x7F800000u;
  if (special) {
    amax = 0;
#pragma unroll
    for (int i = 0; i < 128; ++i) {
      const uint32_t b = __float_as_uint(v[i]) & 0x7FFFFFFFu;
      amax = max(amax, b < 0x7F800000u ? b : 0u);
    }
  }
  const uint32_t byte = block8_exp(amax);
  const float s = block8_inv(byte);
  const unsigned long long ss = f32x2_pack(s, s);
#pragma unroll
  for (int i = 0; i < 32; ++i) {
    float a, b, c, d;
    f32x2_unpack(f32x2_mul(f32x2_pack(v[4 * i], v[4 * i + 1]), ss), a, b);
    f32x2_unpack(f32x2_mul(f32x2_pack(v[4 * i + 2], v[4 * i + 3]), ss), c, d);
    w[i] = e4m3x4(a, b, c, d);
  }
  if (special) {  // (saturated to 448 above)
#pragma unroll
    for (int i = 0; i < 128; ++i)
      if ((__float_as_uint(v[i]) & 0x7F800000u) == 0x7F800000u) w[i / 4] |= 0x7Fu << (8 * (i % 4));
  }
  return byte;
}

__device__ __forceinline__ float4 ld_cluster_f4(uint32_t addr) {
  float4 v;
  asm volatile("ld.shared::cluster.v4.f32 {%0, %1, %2, %3}, [%4];"
               : "=f"(v.x), "=f"(v.y), "=f"(v.z), "=f"(v.w)
               : "r"(addr)
               : "memory");
  return v;
}
// A row's block of 128 columns, four a lane of the warp (those from N on are not
// there), to E4M3 and its scale byte.
__device__ __forceinline__ void put_row8(const float (&u)[4], uint8_t* q, uint8_t* scale, int col, int N) {
  float x[4];
  uint32_t m = 0;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    x[i] = col + i < N ? u[i] : 0.f;
    const uint32_t b = __float_as_uint(x[i]) & 0x7FFFFFFFu;
    m = max(m, b < 0x7F800000u ? b : 0u);
    x[i] = nonfinite_to(x[i], __uint_as_float(0x7FC00000u));
  }
  const uint32_t byte = block8_exp(__reduce_max_sync(0xffffffffu, m));
  const float s = block8_inv(byte);
  const uint32_t w = e4m3x4(x[0] * s, x[1] * s, x[2] * s, x[3] * s);
  if (col + 4 <= N) {
    *reinterpret_cast<uint32_t*>(q + col) = w;
  } else {
    for (int i = 0; col + i < N; ++i) q[col + i] = (uint8_t)(w >> (8 * i));
  }
  if ((threadIdx.x & 31) == 0) *scale = (uint8_t)byte;
}

}  // namespace l8

// PAIR: two CTAs (a cluster of two) share a tile of 256 x 256, each its own 128
// rows of a and half of the tile's rows of w; the even CTA issues the MMAs for
// both. Otherwise tiles of 128 x 128 on single CTAs.
// The epilogue warps (two for each lane quarter, one for each 128 columns) take
// a row's 128 columns into registers and hand the accumulator back at once.
// OUT: what the epilogue writes, so that each kind has the registers it needs.
// SPLIT (single CTAs): the CTAs of a cluster share a tile, each with a part of K.
// They leave their partial sums in the shared memory that the operands have used,
// and each finishes its share of the tile's rows, a row a warp: the sum over the
// cluster through distributed shared memory, then every kind of output.
template <bool PAIR, int OUT, bool SPLIT>
__global__ void __launch_bounds__(l8::THREADS, 1)
    linear8_kernel(const __grid_constant__ CUtensorMap tmA, const __grid_constant__ CUtensorMap tmB,
                   const __grid_constant__ CUtensorMap tmO8, const __grid_constant__ CUtensorMap tmU8,
                   const l8::Params p, unsigned* err) {
  using namespace l8;
  extern __shared__ uint8_t smem_raw[];
  uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
  constexpr int STAGES = stages(OUT), BUFFERS = buffers(OUT);
  uint8_t* sA = smem;
  uint8_t* sB = smem + STAGES * A_BYTES;
  uint8_t* sStg = smem + STAGES * STAGE_BYTES;
  uint8_t* sBias = sStg + EPI_WARPS * BUFFERS * STG_BYTES;
  uint8_t* sScale = sBias + BIAS_BYTES;
  uint64_t* full = reinterpret_cast<uint64_t*>(sScale + SCALE_BYTES);
  uint64_t* empty = full + STAGES;
  uint64_t* sf_full = empty + STAGES;
  uint64_t* sf_empty = sf_full + SF_SLOTS;
  uint64_t* acc_full = sf_empty + SF_SLOTS;
  uint64_t* acc_empty = acc_full + 2;
  uint64_t* lap = acc_empty + 2;  // the columns shared with the next tile are read (pairs)
  uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(lap + 1);
  volatile int* abort_flag = reinterpret_cast<volatile int*>(tmem_slot + 1);

  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  constexpr int TM = PAIR ? 2 * BM : BM, TN = PAIR ? 256 : 128;
  const int num_n = (p.N + TN - 1) / TN, tiles = ((p.M + TM - 1) / TM) * num_n;
  const int all_kb = (p.K + KB_BYTES - 1) / KB_BYTES;
  const int rank = PAIR ? (int)cluster_ctarank() : 0;
  // CTAs that share a tile, this one's part of K: KB blocks from kb_first on
  const int parts = SPLIT ? (int)cluster_nctarank() : 1, part = SPLIT ? (int)cluster_ctarank() : 0;
  const int kb_first = SPLIT ? part * all_kb / parts : 0, KB = SPLIT ? (part + 1) * all_kb / parts - kb_first : all_kb;
  const int ways = PAIR ? 2 : parts, first = (int)blockIdx.x / ways, step = (int)gridDim.x / ways;

  if (threadIdx.x == 0) {
    for (int s = 0; s < STAGES; ++s) {
      mbar_init(&full[s], 1);
      mbar_init(&empty[s], 1);
    }
    for (int s = 0; s < SF_SLOTS; ++s) {
      mbar_init(&sf_full[s], PAIR ? 8 : 4);
      mbar_init(&sf_empty[s], 1);
    }
    for (int b = 0; b < 2; ++b) {
      mbar_init(&acc_full[b], 1);
      mbar_init(&acc_empty[b], PAIR ? 2 * EPI_WARPS : EPI_WARPS / 2);
    }
    mbar_init(lap, EPI_WARPS);
    *abort_flag = 0;
    fence_mbar_init();
    prefetch_tmap(&tmA);
    prefetch_tmap(&tmB);
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

  if (warp < 8) {
    asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(REGS_REST));
    if (warp == 0 && lane == 0) {
      // ---------------- TMA producer ----------------
      int stage = 0;
      uint32_t phase = 0;
      bool ok = true;
      for (int tile = first; tile < tiles && ok; tile += step) {
        const int m0 = (tile / num_n) * TM + rank * BM, n0 = (tile % num_n) * TN + rank * 128;
        for (int kb = 0; kb < KB; ++kb) {
          if (!mbar_wait(&empty[stage], phase ^ 1u, abort_flag, err)) { ok = false; break; }
          uint8_t *da = sA + stage * A_BYTES, *db = sB + stage * B_BYTES;
          if (PAIR) {
            if (rank == 0) mbar_arrive_expect_tx(&full[stage], 2 * STAGE_BYTES);
            const uint32_t bar = cluster_map(smem_u32(&full[stage]), 0);
            tma_load_2d_pair(&tmA, bar, da, kb * KB_BYTES, m0);
            tma_load_2d_pair(&tmB, bar, db, kb * KB_BYTES, n0);
          } else {
            mbar_arrive_expect_tx(&full[stage], STAGE_BYTES);
            tma_load_2d(&tmA, &full[stage], da, (kb_first + kb) * KB_BYTES, m0);
            tma_load_2d(&tmB, &full[stage], db, (kb_first + kb) * KB_BYTES, n0);
          }
          if (++stage == STAGES) { stage = 0; phase ^= 1u; }
        }
      }
    } else if (warp == 1 && rank == 0) {
      // ---------------- MMA issuer (of a pair: the even CTA's) ----------------
      const bool lead = elect_one();
      auto wait = [&](uint64_t* bar, uint32_t parity) {
        const bool done = mbar_wait(bar, parity, abort_flag, err);
        return (bool)__all_sync(0xffffffffu, done);
      };
      int stage = 0, slot = 0, it = 0;
      uint32_t phase = 0, sf_phase = 0;
      bool ok = true;
      for (int tile = first; tile < tiles && ok; tile += step, ++it) {
        const int buf = it & 1;
        const uint32_t use = (uint32_t)(it >> 1) & 1u;
        if (!wait(&acc_empty[buf], use ^ 1u)) break;
        if (PAIR && it > 0 && !wait(lap, (uint32_t)(it - 1) & 1u)) break;
        tc_fence_after();
        const uint32_t d = tmem_base + (uint32_t)buf * (PAIR ? ACC_SECOND : 128u);
        for (int kb = 0; kb < KB; ++kb) {
          if ((kb & 3) == 0 && !(ok = wait(&sf_full[slot], sf_phase))) break;
          if (!(ok = wait(&full[stage], phase))) break;
          tc_fence_after();
          const uint64_t a0 = sw128_desc(smem_u32(sA + stage * A_BYTES));
          const uint64_t b0 = sw128_desc(smem_u32(sB + stage * B_BYTES));
          const uint32_t sf = tmem_base + SF_BASE + (uint32_t)(slot * 16);
          const uint32_t id = idesc(TM, TN, (uint32_t)(kb & 3));
          if (lead) {
#pragma unroll
            for (int k = 0; k < 4; ++k)
              mma<PAIR>(d, a0 + 2 * k, b0 + 2 * k, id, sf, sf + 4, (kb | k) != 0 ? 1u : 0u);
            if (PAIR) umma_commit_pair(&empty[stage]);
            else umma_commit(&empty[stage]);
            if ((kb & 3) == 3 || kb == KB - 1) {
              if (PAIR) umma_commit_pair(&sf_empty[slot]);
              else umma_commit(&sf_empty[slot]);
            }
          }
          __syncwarp();
          if ((kb & 3) == 3 || kb == KB - 1)
            if (++slot == SF_SLOTS) { slot = 0; sf_phase ^= 1u; }
          if (++stage == STAGES) { stage = 0; phase ^= 1u; }
        }
        if (ok && lead) {
          if (PAIR) umma_commit_pair(&acc_full[buf]);
          else umma_commit(&acc_full[buf]);
        }
        __syncwarp();
      }
    } else if (warp >= 4) {
      // ---------------- scales: global memory to tensor memory ----------------
      // Each warp writes its own quarter of the lanes, and each quarter takes all
      // of a group's scales (128 rows, four K blocks). So a warp fetches one K
      // block, and they exchange them through shared memory, a 32-bit word a row.
      // The bytes come from L2 or DRAM, and a group is due every four stages: they
      // are fetched AHEAD groups early (fetched when due, the MMAs waited for
      // scales a third of the time).
      constexpr int AHEAD = 3, HALVES = TN / kBlk;
      const int sw = warp & 3, nblk = (p.N + kBlk - 1) / kBlk, per_tile = (KB + 3) / 4;
      const uint32_t lane_quarter = (uint32_t)(sw * 32) << 16;
      uint8_t* const words = reinterpret_cast<uint8_t*>(sScale);  // [2][128 rows + HALVES][4]
      uint32_t fa[AHEAD][4], fb[AHEAD];
      int ftile = first, fgroup = 0;  // the next group to fetch
      auto fetch = [&](uint32_t (&wa)[4], uint32_t& wb) {
        if (ftile < tiles) {
          const int kb = kb_first + min(4 * fgroup + sw, KB - 1);
          const int m0 = (ftile / num_n) * TM + rank * BM, b0 = (ftile % num_n) * HALVES;
          const uint8_t* sa = p.a_scale + (size_t)kb * p.lds_a;
#pragma unroll
          for (int c = 0; c < 4; ++c) wa[c] = sa[min(m0 + 32 * c + lane, p.M - 1)];
          if (lane < HALVES) wb = p.w_scale[(size_t)kb * p.lds_w + min(b0 + lane, nblk - 1)];
          if (++fgroup == per_tile) {
            fgroup = 0;
            ftile += step;
          }
        }
      };
#pragma unroll
      for (int i = 0; i < AHEAD; ++i) {
#pragma unroll
        for (int c = 0; c < 4; ++c) fa[i][c] = 127u;
        fb[i] = 127u;
        fetch(fa[i], fb[i]);
      }
      int slot = 0, half = 0;
      uint32_t sf_phase = 0;
      bool dead = false;  // a wait ran out: no more waits and writes, but the barrier below is kept
      auto group = [&](uint32_t (&wa)[4], uint32_t& wb) {
        uint8_t* const w = words + half * (128 + HALVES) * 4;
#pragma unroll
        for (int c = 0; c < 4; ++c) w[(32 * c + lane) * 4 + sw] = (uint8_t)wa[c];
        if (lane < HALVES) w[(128 + lane) * 4 + sw] = (uint8_t)wb;
        fetch(wa, wb);
        asm volatile("bar.sync 1, 128;" ::: "memory");  // the four scale warps
        const uint32_t* r = reinterpret_cast<const uint32_t*>(w);
        const uint32_t va[4] = {r[lane], r[32 + lane], r[64 + lane], r[96 + lane]};
        half ^= 1;
        if (!dead) dead = !__all_sync(0xffffffffu, mbar_wait(&sf_empty[slot], sf_phase ^ 1u, abort_flag, err));
        if (!dead) {
          const uint32_t t = tmem_base + lane_quarter + SF_BASE + (uint32_t)(slot * 16);
          tc_fence_after();
          tmem_st4(t, va);
#pragma unroll
          for (int h = 0; h < HALVES; ++h) {
            const uint32_t v = r[128 + h], w4[4] = {v, v, v, v};
            tmem_st4(t + 4 + 4 * h, w4);
          }
          tmem_wait_st();
          tc_fence_before();
          __syncwarp();
          if (lane == 0) {
            if (PAIR) arrive_even(&sf_full[slot]);
            else mbar_arrive(&sf_full[slot]);
          }
        }
        if (++slot == SF_SLOTS) { slot = 0; sf_phase ^= 1u; }
      };
      const int mine = first < tiles ? (tiles - first + step - 1) / step : 0;
      const int groups = mine * per_tile;
      for (int i = 0; i < groups; i += AHEAD) {
#pragma unroll
        for (int j = 0; j < AHEAD; ++j)
          if (i + j < groups) group(fa[j], fb[j]);
      }
    }
    __syncwarp();
    if constexpr (SPLIT) {  // the epilogue's two meetings of the cluster
      cluster_sync();
      cluster_sync();
    }
  } else if constexpr (SPLIT) {
    // ---------------- partial sums to shared memory ----------------
    asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(REGS_EPI));
    const int quarter = warp & 3, half = (warp - 8) >> 2;  // lane quarter, 64 of the tile's 128 columns
    const bool done = mbar_wait(&acc_full[0], 0, abort_flag, err);
    if (__all_sync(0xffffffffu, done)) {
      tc_fence_after();
      uint32_t r[2][32];
      const uint32_t t = tmem_base + ((uint32_t)(quarter * 32) << 16) + (uint32_t)(half * 64);
      tmem_ld32(t, r[0]);
      tmem_ld32(t + 32, r[1]);
      tmem_wait_ld_regs(r[0]);
      tmem_wait_ld_regs(r[1]);
      // (every load into the ring has been consumed) row of 512 bytes, 16-byte piece j at j ^ (row & 31)
      uint8_t* row = smem + (quarter * 32 + lane) * 512;
#pragma unroll
      for (int j = 0; j < 16; ++j)
        *reinterpret_cast<uint4*>(row + (((16 * half + j) ^ lane) << 4)) =
            make_uint4(r[j / 8][4 * (j % 8)], r[j / 8][4 * (j % 8) + 1], r[j / 8][4 * (j % 8) + 2], r[j / 8][4 * (j % 8) + 3]);
    }
    __syncwarp();
    // ---------------- this CTA's share of the rows ----------------
    cluster_sync();
    const int m0 = (first / num_n) * TM, n0 = (first % num_n) * TN, col = n0 + 4 * lane, each = BM / parts;
#pragma unroll 2
    for (int r0 = warp - 8; r0 < each; r0 += EPI_WARPS) {
      const int lr = part * each + r0, row = m0 + lr;
      if (row >= p.M) continue;
      const uint32_t at = smem_u32(smem + lr * 512 + ((lane ^ (lr & 31)) << 4));
      float4 x[8], v = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
      for (int k = 0; k < 8; ++k)  // (all on their way before the first is used)
        if (k < parts) x[k] = ld_cluster_f4(cluster_map(at, (uint32_t)k));
#pragma unroll
      for (int k = 0; k < 8; ++k)
        if (k < parts) v = make_float4(v.x + x[k].x, v.y + x[k].y, v.z + x[k].z, v.w + x[k].w);
      float u[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
      for (int i = 0; i < 4; ++i)
        if (col + i < p.N && p.bias) u[i] += p.bias[col + i];
      if (p.u8) put_row8(u, p.u8 + (size_t)row * p.ldu8, p.u8_scale + (size_t)(n0 / kBlk) * p.lds_u8 + row, col, p.N);
      if (p.epilogue == LAZYMAR_EPI_GELU) {
        gelu_erf6_x2(u[0], u[1]);
        gelu_erf6_x2(u[2], u[3]);
      }
      if (p.epilogue == LAZYMAR_EPI_RESIDUAL) {
#pragma unroll
        for (int i = 0; i < 4; ++i)
          if (col + i < p.N) u[i] += p.residual[(size_t)row * p.ldr + col + i];
      }
      if (p.out8)
        put_row8(u, p.out8 + (size_t)row * p.ldout8, p.out8_scale + (size_t)(n0 / kBlk) * p.lds_out8 + row, col, p.N);
      if (p.out && col < p.N) {
        if (p.out_dtype == LAZYMAR_F32) {
          float* y = static_cast<float*>(p.out) + (size_t)row * p.ldo + col;
          if (p.rows_vec && col + 4 <= p.N) {
            *reinterpret_cast<float4*>(y) = make_float4(u[0], u[1], u[2], u[3]);
          } else {
#pragma unroll
            for (int i = 0; i < 4; ++i)
              if (col + i < p.N) y[i] = u[i];
          }
        } else {
          bf16* y = static_cast<bf16*>(p.out) + (size_t)row * p.ldo + col;
          if (p.rows_vec && col + 4 <= p.N) {
            *reinterpret_cast<uint2*>(y) = make_uint2(pack_bf16(u[0], u[1]), pack_bf16(u[2], u[3]));
          } else {
#pragma unroll
            for (int i = 0; i < 4; ++i)
              if (col + i < p.N) y[i] = from_f<bf16>(u[i]);
          }
        }
      }
    }
    __syncwarp();
    cluster_sync();  // no CTA leaves while another may read its partial sums
  } else {
    // ---------------- epilogue ----------------
    asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(REGS_EPI));
    const int quarter = warp & 3, unit = (warp - 8) >> 2;  // lane quarter, 128 columns of the accumulator
    // A row's 128 values are taken 32 columns at a time from the rot-th 32 on, so
    // that the columns that the next tile of a pair waits for come first: the last
    // ones of the first tile, the first ones of the second.
    const int rot = PAIR && unit == 1 ? 3 : 0;
    uint8_t* const stg2 = sStg + (warp - 8) * BUFFERS * STG_BYTES;
    float4* const bias = reinterpret_cast<float4*>(sBias) + (warp - 8) * 32;  // of the tile's 128 columns
    int flip = 0, it = 0;
    for (int tile = first; tile < tiles; tile += step, ++it) {
      // single CTAs: the tiles alternate between the two units
      if (!PAIR && (it & 1) != unit) continue;
      const int buf = it & 1;
      const uint32_t use = (uint32_t)(it >> 1) & 1u;
      const int rbase = (tile / num_n) * TM + rank * BM + quarter * 32;
      const int n0 = (tile % num_n) * TN + (PAIR ? unit * 128 : 0);
      const int lr0 = lane >> 3, cq = lane & 7;  // row of four and 16-byte piece in the output passes
      // the residual of 32 columns, eight passes of four rows; the first ones'
      // before the accumulator is ready
      float4 res[8];
      // (rows off the boundary: a row an access, lane = column, so that the accesses
      // stay contiguous; row r is the r % 4th of res[r / 4])
      auto load_res = [&](int c) {
        if (!p.rows_vec) {
          const int col = n0 + 32 * ((c + rot) & 3) + lane;
          auto at = [&](int r) { return col < p.N && rbase + r < p.M ? p.residual[(size_t)(rbase + r) * p.ldr + col] : 0.f; };
#pragma unroll
          for (int q = 0; q < 8; ++q) res[q] = make_float4(at(4 * q), at(4 * q + 1), at(4 * q + 2), at(4 * q + 3));
          return;
        }
        const int col = n0 + 32 * ((c + rot) & 3) + 4 * cq;
#pragma unroll
        for (int q = 0; q < 8; ++q) {
          const int r = rbase + 4 * q + lr0;
          res[q] = make_float4(0.f, 0.f, 0.f, 0.f);
          if (r >= p.M || col >= p.N) continue;
          const float* x = p.residual + (size_t)r * p.ldr + col;
          if (col + 4 <= p.N) {
            res[q] = *reinterpret_cast<const float4*>(x);
          } else {
            res[q].x = x[0];
            if (col + 1 < p.N) res[q].y = x[1];
            if (col + 2 < p.N) res[q].z = x[2];
            if (col + 3 < p.N) res[q].w = x[3];
          }
        }
      };
      if (OUT == OUT_RESIDUAL) load_res(0);
      if (p.bias) {
        float4 b = make_float4(0.f, 0.f, 0.f, 0.f);
        const int col = n0 + 4 * lane;
        if (p.bias_vec && col + 4 <= p.N) {
          b = *reinterpret_cast<const float4*>(p.bias + col);
        } else {
          if (col < p.N) b.x = p.bias[col];
          if (col + 1 < p.N) b.y = p.bias[col + 1];
          if (col + 2 < p.N) b.z = p.bias[col + 2];
          if (col + 3 < p.N) b.w = p.bias[col + 3];
        }
        __syncwarp();
        bias[lane] = b;
        __syncwarp();
      }
      const bool done = mbar_wait(&acc_full[buf], use, abort_flag, err);
      if (!__all_sync(0xffffffffu, done)) break;
      tc_fence_after();
      float v[128];
      {
        const uint32_t t = tmem_base + ((uint32_t)(quarter * 32) << 16) +
                           (PAIR ? (uint32_t)buf * ACC_SECOND + (uint32_t)unit * 128u : (uint32_t)buf * 128u);
        uint32_t r[4][32];
        tmem_ld32(t + 32 * rot, r[0]);
        tmem_wait_ld_regs(r[0]);
        if (PAIR && unit != buf) {
          tc_fence_before();
          __syncwarp();
          if (lane == 0) arrive_even(lap);
        }
#pragma unroll
        for (int c = 1; c < 4; ++c) tmem_ld32(t + 32 * ((c + rot) & 3), r[c]);
#pragma unroll
        for (int c = 1; c < 4; ++c) tmem_wait_ld_regs(r[c]);
#pragma unroll
        for (int c = 0; c < 4; ++c)
#pragma unroll
          for (int i = 0; i < 32; ++i) v[32 * c + i] = __uint_as_float(r[c][i]);
      }
      tc_fence_before();
      __syncwarp();
      if (lane == 0) {
        if (PAIR) arrive_even(&acc_empty[buf]);
        else mbar_arrive(&acc_empty[buf]);
      }
      if (n0 >= p.N || rbase >= p.M) continue;
      const int row = rbase + lane;
      if (p.bias) {
#pragma unroll
        for (int i = 0; i < 32; ++i) {
          const float4 b = bias[(i + 8 * rot) & 31];
          f32x2_unpack(f32x2_add(f32x2_pack(v[4 * i], v[4 * i + 1]), f32x2_pack(b.x, b.y)), v[4 * i], v[4 * i + 1]);
          f32x2_unpack(f32x2_add(f32x2_pack(v[4 * i + 2], v[4 * i + 3]), f32x2_pack(b.z, b.w)), v[4 * i + 2],
                       v[4 * i + 3]);
        }
      }
      // a row's 128 E4M3 bytes: staged with the TMA's 128-byte swizzle, one store
      // of 32 rows. TMA writes whole 16-byte pieces, so a last piece that the
      // tensor does not fill leaves by plain stores.
      auto put8 = [&](const CUtensorMap* tm, uint8_t* q, int ldq, uint8_t* scale, int lds) {
        uint32_t w[32];
        const uint32_t byte = quantize_row(v, w);
        if (row < p.M) scale[(size_t)(n0 / kBlk) * lds + row] = (uint8_t)byte;
        uint8_t* stg = stg2 + flip * STG_BYTES;
        flip ^= 1;
        const bool tma = (p.N & 15) == 0 || n0 + 128 <= p.N;
        if (lane == 0) {  // what this buffer held has been stored
          if (tma) bulk_wait_read_but_one();
          else bulk_wait_read();
        }
        __syncwarp();
#pragma unroll
        for (int j = 0; j < 8; ++j)
          *reinterpret_cast<uint4*>(stg + lane * 128 + ((((j + 2 * rot) & 7) ^ (lane & 7)) << 4)) =
              make_uint4(w[4 * j], w[4 * j + 1], w[4 * j + 2], w[4 * j + 3]);
        if (tma) {
          fence_proxy_async_smem();
          __syncwarp();
          if (lane == 0) {
            tma_store_2d(tm, stg, n0, rbase);
            bulk_commit();
          }
          return;
        }
        __syncwarp();
        const int piece = lane & 7, here = min(16, p.N - n0 - 16 * piece);
#pragma unroll 1
        for (int i = 0; i < 8; ++i) {
          const int lr = 4 * i + (lane >> 3), r = rbase + lr;
          if (r >= p.M || here <= 0) continue;
          const uint8_t* src = stg + lr * 128 + ((piece ^ (lr & 7)) << 4);
          uint8_t* dst = q + (size_t)r * ldq + n0 + 16 * piece;
          if (here == 16) *reinterpret_cast<uint4*>(dst) = *reinterpret_cast<const uint4*>(src);
          else
            for (int j = 0; j < here; ++j) dst[j] = src[j];
        }
        __syncwarp();
      };
      if (OUT == OUT_BLOCK8 && p.u8) put8(&tmU8, p.u8, p.ldu8, p.u8_scale, p.lds_u8);
      if (OUT != OUT_RESIDUAL && p.epilogue == LAZYMAR_EPI_GELU) {
#pragma unroll
        for (int i = 0; i < 64; ++i) gelu_erf6_x2(v[2 * i], v[2 * i + 1]);
      }
      if (OUT == OUT_BLOCK8 && p.out8) put8(&tmO8, p.out8, p.ldout8, p.out8_scale, p.lds_out8);
      if (p.out) {
        // 32 columns at a time through the staging buffer, so that stores and
        // residual loads cover whole rows of it
        if (lane == 0) bulk_wait_read();
        __syncwarp();
#pragma unroll
        for (int c = 0; c < 4; ++c) {
          const int col = n0 + 32 * ((c + rot) & 3) + 4 * cq;
          uint8_t* stg = stg2 + (c % BUFFERS) * STG_BYTES;
          if (BUFFERS == 1) __syncwarp();  // the columns before have been read
#pragma unroll
          for (int j = 0; j < 8; ++j)
            *reinterpret_cast<float4*>(stg + lane * 128 + ((j ^ (lane & 7)) << 4)) =
                make_float4(v[32 * c + 4 * j], v[32 * c + 4 * j + 1], v[32 * c + 4 * j + 2], v[32 * c + 4 * j + 3]);
          __syncwarp();
          if (!p.rows_vec) {
            // a row an access, lane = column: four scalars a lane would touch four times
            // the sectors (37823 x 699 x 768, bf16 and a checkpoint: 85 us)
            const int one = n0 + 32 * ((c + rot) & 3) + lane;
            float e[32];
#pragma unroll
            for (int r = 0; r < 32; ++r)
              e[r] = *reinterpret_cast<const float*>(stg + r * 128 + (((lane >> 2) ^ (r & 7)) << 4) + ((lane & 3) << 2));
            if (OUT == OUT_RESIDUAL) {
#pragma unroll
              for (int q = 0; q < 8; ++q) {
                e[4 * q] += res[q].x;
                e[4 * q + 1] += res[q].y;
                e[4 * q + 2] += res[q].z;
                e[4 * q + 3] += res[q].w;
              }
              if (c < 3) load_res(c + 1);
            }
            if (one < p.N) {
              const size_t first_at = (size_t)rbase * p.ldo + one;
#pragma unroll
              for (int r = 0; r < 32; ++r) {
                if (rbase + r >= p.M) break;
                if (p.out_dtype == LAZYMAR_F32) static_cast<float*>(p.out)[first_at + (size_t)r * p.ldo] = e[r];
                else static_cast<bf16*>(p.out)[first_at + (size_t)r * p.ldo] = from_f<bf16>(e[r]);
              }
            }
            continue;
          }
          float4 o[8];
#pragma unroll
          for (int q = 0; q < 8; ++q) {
            const int lr = 4 * q + lr0;
            o[q] = *reinterpret_cast<const float4*>(stg + lr * 128 + ((cq ^ (lr & 7)) << 4));
          }
          if (OUT == OUT_RESIDUAL) {
#pragma unroll
            for (int q = 0; q < 8; ++q)
              o[q] = make_float4(o[q].x + res[q].x, o[q].y + res[q].y, o[q].z + res[q].z, o[q].w + res[q].w);
            // (other columns than those stored below, so in place is fine)
            if (c < 3) load_res(c + 1);
          }
#pragma unroll
          for (int q = 0; q < 8; ++q) {
            const int r = rbase + 4 * q + lr0;
            if (r >= p.M || col >= p.N) continue;
            if (p.out_dtype == LAZYMAR_F32) {
              float* y = static_cast<float*>(p.out) + (size_t)r * p.ldo + col;
              if (col + 4 <= p.N) {
                *reinterpret_cast<float4*>(y) = o[q];
              } else {
                y[0] = o[q].x;
                if (col + 1 < p.N) y[1] = o[q].y;
                if (col + 2 < p.N) y[2] = o[q].z;
                if (col + 3 < p.N) y[3] = o[q].w;
              }
            } else {
              bf16* y = static_cast<bf16*>(p.out) + (size_t)r * p.ldo + col;
              if (col + 4 <= p.N) {
                *reinterpret_cast<uint2*>(y) = make_uint2(pack_bf16(o[q].x, o[q].y), pack_bf16(o[q].z, o[q].w));
              } else {
                y[0] = from_f<bf16>(o[q].x);
                if (col + 1 < p.N) y[1] = from_f<bf16>(o[q].y);
                if (col + 2 < p.N) y[2] = from_f<bf16>(o[q].z);
                if (col + 3 < p.N) y[3] = from_f<bf16>(o[q].w);
              }
            }
          }
        }
        __syncwarp();
      }
    }
    if (lane == 0) bulk_wait_all();
    __syncwarp();
  }
  __syncthreads();
  if (PAIR) cluster_sync();
  if (warp == 1) {
    tc_fence_after();
    if (PAIR) tmem_dealloc_pair(tmem_base, 512);
    else tmem_dealloc(tmem_base, 512);
  }
}

namespace {

// Once for each device: the shared-memory size, and the check that the launch
// holds the registers that the kernel's warps share out.
template <bool PAIR, int OUT, bool SPLIT>
cudaError_t run_linear8(const Ctx& c, const CUtensorMap& ta, const CUtensorMap& tb, const CUtensorMap& to,
                        const CUtensorMap& tu, const l8::Params& p, long long tiles, int cluster) {
  using namespace l8;
  const auto kernel = linear8_kernel<PAIR, OUT, SPLIT>;
  constexpr size_t smem = smem_bytes(OUT);
  static int ready[64] = {};
  int dev = 0;
  cudaError_t e = cudaGetDevice(&dev);
  if (e != cudaSuccess) return e;
  if (dev < 0 || dev >= 64 || !ready[dev]) {
    cudaFuncAttributes a;
    if ((e = cudaFuncGetAttributes(&a, kernel)) != cudaSuccess) return e;
    if (a.numRegs * THREADS < (REGS_EPI + REGS_REST) * 256) return cudaErrorInvalidConfiguration;
    if ((e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem)) != cudaSuccess) return e;
    if (dev >= 0 && dev < 64) ready[dev] = 1;
  }
  // (with K in parts a cluster takes one tile, so there are as many of them)
  const int slots = c.num_sms / cluster;
  const unsigned grid = (unsigned)((SPLIT || tiles < slots ? tiles : slots) * cluster);
  if (cluster > 1)
    return launch_pdl_cluster(kernel, dim3(grid), dim3(THREADS), smem, cluster, c.stream, ta, tb, to, tu, p, c.err);
  return launch_pdl(kernel, dim3(grid), dim3(THREADS), smem, c.stream, ta, tb, to, tu, p, c.err);
}

template <bool PAIR>
cudaError_t run_linear8(const Ctx& c, const CUtensorMap& ta, const CUtensorMap& tb, const CUtensorMap& to,
                        const CUtensorMap& tu, const l8::Params& p, long long tiles) {
  constexpr int CTAS = PAIR ? 2 : 1;
  if (p.out8 || p.u8) return run_linear8<PAIR, l8::OUT_BLOCK8, false>(c, ta, tb, to, tu, p, tiles, CTAS);
  if (p.epilogue == LAZYMAR_EPI_RESIDUAL)
    return run_linear8<PAIR, l8::OUT_RESIDUAL, false>(c, ta, tb, to, tu, p, tiles, CTAS);
  return run_linear8<PAIR, l8::OUT_PLAIN, false>(c, ta, tb, to, tu, p, tiles, CTAS);
}

}  // namespace

cudaError_t launch_linear8(const Ctx& c, const Linear8& x) {
  using namespace l8;
  if (x.M <= kLinear8FewRows) return launch_linear8_rows(c, x);
  CUtensorMap ta, tb, to, tu;
  std::memset(&to, 0, sizeof to);
  std::memset(&tu, 0, sizeof tu);
  const auto sw = CU_TENSOR_MAP_SWIZZLE_128B;
  if (!make_tmap_u8(&ta, x.a.q, x.K, x.M, x.a.ldq, KB_BYTES, BM, sw) ||
      !make_tmap_u8(&tb, x.w.q, x.K, x.N, x.w.ldq, KB_BYTES, 128, sw) ||
      (x.out8.q && !make_tmap_u8(&to, x.out8.q, x.N, x.M, x.out8.ldq, 128, 32, sw)) ||
      (x.u8.q && !make_tmap_u8(&tu, x.u8.q, x.N, x.M, x.u8.ldq, 128, 32, sw)))
    return cudaErrorInvalidValue;
  Params p{};
  p.a_scale = x.a.scale;
  p.w_scale = x.w.scale;
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
  p.out8_scale = x.out8.scale;
  p.u8_scale = x.u8.scale;
  p.lds_out8 = x.out8.lds;
  p.lds_u8 = x.u8.lds;
  p.out8 = static_cast<uint8_t*>(x.out8.q);
  p.u8 = static_cast<uint8_t*>(x.u8.q);
  p.ldout8 = x.out8.ldq;
  p.ldu8 = x.u8.ldq;
  p.bias_vec = reinterpret_cast<uintptr_t>(x.bias) % 16 == 0;
  p.rows_vec = rows_on_four(x.out.p, x.out.ld, x.out.dtype == LAZYMAR_F32 ? 4 : 2) &&
               rows_on_four(x.residual.p, x.residual.ld, 4);
  const Shape shape = choose(c.num_sms, x.M, x.N, x.K);
  if (shape.pair) return run_linear8<true>(c, ta, tb, to, tu, p, shape.tiles);
  if (shape.parts > 1) return run_linear8<false, OUT_PLAIN, true>(c, ta, tb, to, tu, p, shape.tiles, shape.parts);
  return run_linear8<false>(c, ta, tb, to, tu, p, shape.tiles);
}

}  // namespace lm
