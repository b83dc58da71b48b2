// The LM head in 8-bit floating point: C[m, n] = sum_j sa[m, j] sb[n / 128, j] sum_{k in block j} A[m, k] B[n, k], e4m3
// operands with a float32 scale for each 128 columns (and each 128 rows of B), and the quantiser of such operands.
//
// The scales change along K, so a sum over a block of 128 is all that the tensor cores can form by themselves: four
// tcgen05.mma of kind::f8f6f4 (K = 32 each) into one of two (or eight) accumulators in tensor memory, which the epilogue warps
// read back, multiply by the block's scales and add to float32 accumulators in registers while the next block is
// multiplied.  That also keeps every sum in the tensor core, which cuts off what does not fit its accumulator, to 128 terms.
//
//   many tokens   pairs of blocks on 256 x 256 tiles, as the 16-bit contraction has them; bound by the tensor cores
//   few tokens    (M <= 64) operands swapped: 128 rows of B are the M of the instruction, the tokens its N; one block streams
//                 its rows of B through a deep ring of TMA loads; bound by HBM
#include <cmath>

#include "dvp_common.cuh"
#include "dvp_fp8.cuh"
#include "dvp_tensor.cuh"

namespace dvp {
namespace fp8 {

using namespace gemm;

constexpr int kBlock = 128;  // K of a scale: one slice of the ring, 128 bytes a row
constexpr int kUmmaK8 = 32;
constexpr long long kMost = 0x7fffff00LL;

struct Params8 {
  void *C;
  long long ldc, ld_sa, ld_sb;
  const float *sa, *sb;
  int *status;
  int M, N, K;
  int vec;        // C takes 32-byte stores
  int tile_rows;  // few tokens: rows of B a tile
};

__device__ __forceinline__ uint32_t instr_desc8(int m, int n) {
  return (1u << 4) | ((uint32_t)(n >> 3) << 17) | ((uint32_t)(m >> 4) << 24);  // e4m3 x e4m3, float32 accumulators
}
__device__ __forceinline__ void umma8_pair(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, uint32_t accumulate) {
  asm volatile(
      "{\n\t.reg .pred p;\n\t"
      "setp.ne.b32 p, %4, 0;\n\t"
      "tcgen05.mma.cta_group::2.kind::f8f6f4 [%0], %1, %2, %3, p;\n\t}" ::"r"(d),
      "l"(a), "l"(b), "r"(idesc), "r"(accumulate)
      : "memory");
}
__device__ __forceinline__ void umma8(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, uint32_t accumulate) {
  asm volatile(
      "{\n\t.reg .pred p;\n\t"
      "setp.ne.b32 p, %4, 0;\n\t"
      "tcgen05.mma.cta_group::1.kind::f8f6f4 [%0], %1, %2, %3, p;\n\t}" ::"r"(d),
      "l"(a), "l"(b), "r"(idesc), "r"(accumulate)
      : "memory");
}
// The 16 columns of a warp's rows, read and waited for; for whole warps.
__device__ __forceinline__ void tmem_ld16_wait(uint32_t taddr, uint32_t (&r)[16]) {
  __syncwarp();
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15}, [%16];"
      : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]),
        "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15])
      : "r"(taddr));
  __syncwarp();
  asm volatile("tcgen05.wait::ld.sync.aligned;"
               : "+r"(r[0]), "+r"(r[1]), "+r"(r[2]), "+r"(r[3]), "+r"(r[4]), "+r"(r[5]), "+r"(r[6]), "+r"(r[7]), "+r"(r[8]),
                 "+r"(r[9]), "+r"(r[10]), "+r"(r[11]), "+r"(r[12]), "+r"(r[13]), "+r"(r[14]), "+r"(r[15])
               :
               : "memory");
}

// Sixteen neighbouring values of a row of C, the first `n` of which exist.
template <typename TC>
__device__ __forceinline__ void store16(TC *c, const float *v, int n, bool vec) {
  if (vec && n >= 16) {
    uint32_t w[8];
    if constexpr (sizeof(TC) == 4) {
#pragma unroll
      for (int h = 0; h < 2; ++h) {
#pragma unroll
        for (int j = 0; j < 8; ++j) w[j] = __float_as_uint(v[8 * h + j]);
        st_stream32(c + 8 * h, w);
      }
    } else {
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const TC lo = Storage<TC>::narrow(v[2 * j]), hi = Storage<TC>::narrow(v[2 * j + 1]);
        w[j] = (uint32_t) * reinterpret_cast<const uint16_t *>(&lo) | (uint32_t) * reinterpret_cast<const uint16_t *>(&hi) << 16;
      }
      st_stream32(c, w);
    }
  } else {
#pragma unroll
    for (int j = 0; j < 16; ++j)
      if (j < n) c[j] = Storage<TC>::narrow(v[j]);
  }
}

// ---- many tokens ---------------------------------------------------------------------------------------------------------
// Block 2 i + r of pair i keeps 128 rows of A, 128 of the 256 rows of B and the 128 x 256 sums of its own rows.  Warp 0: TMA,
// warp 1: MMA (of the leader, for both), warps 4 to 11: the epilogue, a quarter of the rows and half of the columns each, so that a
// thread holds 128 sums.  A slice's MMAs take some 512 clocks of an SM, its 128 multiply-adds a thread, two warps a
// scheduler, 256, and tensor memory is read beside them: the next 32 columns while 32 are added.  For that the epilogue's warps
// take over registers of the others: 168 a thread at launch, 56 and 224 then, which is the same sum.
//
// Bound by the waits of the reading back: tensor cores busy 44 % of the cycles, tensor memory 55 % (18,944 rows of B).  4,096 x 4,096 x 151,936 to bfloat16: 2,740 us by itself
// (1,860 TFLOP/s), some 3,150 in a row of calls, where the board's power lowers the clock.  Slower were packed multiply-adds
// (3,008 us), four accumulators of 128 columns (3,316), sixteen epilogue warps (3,037), one lane that waits for its warp (2,759).
constexpr int kThreads8 = 384;
constexpr int kEpilogueWarps = 8;
constexpr int kRegsLaunch = 168, kRegsFew = 56, kRegsMany = 224;
static_assert(kRegsFew + 2 * kRegsMany <= 3 * kRegsLaunch, "setmaxnreg waits for registers that the block does not have");
constexpr uint32_t kBytesA8 = 128 * kBlock, kStageBytes8 = 2 * kBytesA8;
constexpr int kStages8 = 6;
constexpr int kTurnLd = 33;  // 32 x 32 values of a warp, turned so that lanes store neighbouring columns
constexpr size_t kTurnBytes = (size_t)kEpilogueWarps * 32 * kTurnLd * 4;
constexpr size_t kSmemBytes8 = 1024 + (size_t)kStages8 * kStageBytes8 + 256 + kTurnBytes;
static_assert(kSmemBytes8 <= 227 * 1024, "shared memory of a block");

struct Shared8 {
  uint64_t full[kStages8], empty[kStages8], tmem_full[2], tmem_empty[2];
  uint32_t tmem_base;
  int abort_flag;
};

__device__ __forceinline__ void give_up(volatile int *abort_flag, int *status, int code) {
  if (!*abort_flag) {
    *abort_flag = 1;
    atomicExch(status, code);
  }
}

// The producer's last act: waits until the products of the last stages have handed them back, so that no arrival is on its way to a
// barrier of a block that has ended.  `n` stages were filled, one hand-over each.
template <int kStages>
__device__ __forceinline__ void wait_for_last(const uint64_t (&empty)[kStages], uint32_t n, volatile int *abort_flag, int *status) {
  for (uint32_t it = n > kStages ? n - kStages : 0; it < n && !*abort_flag; ++it)
    if (!mbar_wait(smem_u32(&empty[it % kStages]), (it / kStages) & 1, abort_flag)) give_up(abort_flag, status, kErrProducerWait);
}

template <typename TC>
__global__ void __launch_bounds__(kThreads8, 1)
gemm_fp8_pair_kernel(const __grid_constant__ CUtensorMap map_a, const __grid_constant__ CUtensorMap map_b, const Params8 p) {
  extern __shared__ uint8_t smem_raw[];
  const uint32_t base = (smem_u32(smem_raw) + 1023u) & ~1023u;
  Shared8 *sh = reinterpret_cast<Shared8 *>(smem_raw + (base - smem_u32(smem_raw)) + (size_t)kStages8 * kStageBytes8);
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const uint32_t rank = cluster_ctarank();
  const int pair = blockIdx.x >> 1, n_pairs = gridDim.x >> 1;
  const int tiles_m = (p.M + 255) / 256, tiles_n = (p.N + 255) / 256, n_tiles = tiles_m * tiles_n;
  const int slices = (p.K + kBlock - 1) / kBlock;
  const bool m_fastest = tiles_m <= tiles_n;

  if (threadIdx.x == 0) {
    for (int s = 0; s < kStages8; ++s) {
      mbar_init(smem_u32(&sh->full[s]), 1);   // the leader's producer, plus the bytes of both blocks
      mbar_init(smem_u32(&sh->empty[s]), 1);  // one commit
    }
    for (int b = 0; b < 2; ++b) {
      mbar_init(smem_u32(&sh->tmem_full[b]), 1);
      mbar_init(smem_u32(&sh->tmem_empty[b]), 2 * kEpilogueWarps);  // of both blocks
    }
    sh->abort_flag = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    if (blockIdx.x == 0) *p.status = 0;  // a wait gives up after seconds
  }
  if (warp == 1) {
    asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(&sh->tmem_base)),
                 "r"(kTmemCols)
                 : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;" ::: "memory");
  }
  tc_fence_before();
  cluster_barrier();  // barriers of both blocks are initialised before anyone signals them
  tc_fence_after();
  const uint32_t tmem_base = sh->tmem_base;
  volatile int *abort_flag = &sh->abort_flag;

  __syncwarp();
  if (warp < 4) {
    asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(kRegsFew));
    if (warp == 0 && lane == 0) {
      uint32_t it = 0;
      for (int tile = pair; tile < n_tiles && !*abort_flag; tile += n_pairs) {
        const int tm = m_fastest ? tile % tiles_m : tile / tiles_n, tn = m_fastest ? tile / tiles_m : tile % tiles_n;
        for (int ks = 0; ks < slices; ++ks, ++it) {
          const uint32_t s = it % kStages8, round = it / kStages8;
          if (round > 0 && !mbar_wait(smem_u32(&sh->empty[s]), (round - 1) & 1, abort_flag)) {
            give_up(abort_flag, p.status, kErrProducerWait);
            break;
          }
          const uint32_t bar_local = smem_u32(&sh->full[s]);
          if (rank == 0) mbar_expect_tx(bar_local, 2 * kStageBytes8);
          const uint32_t bar = map_to_rank(bar_local, 0), dst = base + s * kStageBytes8;
          tma_load_2d_pair(dst, &map_a, bar, ks * kBlock, tm * 256 + (int)rank * 128);
          tma_load_2d_pair(dst + kBytesA8, &map_b, bar, ks * kBlock, tn * 256 + (int)rank * 128);
        }
      }
      wait_for_last(sh->empty, it, abort_flag, p.status);
    } else if (warp == 1 && lane == 0 && rank == 0) {
      const uint32_t idesc = instr_desc8(256, 256);
      uint32_t it = 0;
      for (int tile = pair; tile < n_tiles && !*abort_flag; tile += n_pairs) {
        bool ok = true;
        for (int ks = 0; ks < slices; ++ks, ++it) {  // every slice has an accumulator of its own
          const uint32_t s = it % kStages8, round = it / kStages8, buf = it & 1, use = it >> 1;
          if (use > 0 && !mbar_wait(smem_u32(&sh->tmem_empty[buf]), (use - 1) & 1, abort_flag)) {
            give_up(abort_flag, p.status, kErrMmaWaitTmem);
            ok = false;
            break;
          }
          if (!mbar_wait(smem_u32(&sh->full[s]), round & 1, abort_flag)) {
            give_up(abort_flag, p.status, kErrMmaWaitFull);
            ok = false;
            break;
          }
          tc_fence_after();
          const uint32_t a_addr = base + s * kStageBytes8;
          const uint64_t adesc = smem_desc_sw128(a_addr), bdesc = smem_desc_sw128(a_addr + kBytesA8);
#pragma unroll
          for (int k = 0; k < kBlock / kUmmaK8; ++k)
            umma8_pair(tmem_base + buf * 256, adesc + k * (kUmmaK8 >> 4), bdesc + k * (kUmmaK8 >> 4), idesc, k > 0 ? 1u : 0u);
          umma_commit_pair(smem_u32(&sh->empty[s]));
          umma_commit_pair(smem_u32(&sh->tmem_full[buf]));
        }
        if (!ok) break;
      }
    }
  } else {
    asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(kRegsMany));
    const int quarter = warp & 3, half = (warp - 4) >> 2;
    float *turn = reinterpret_cast<float *>(reinterpret_cast<uint8_t *>(sh) + 256) + (warp - 4) * 32 * kTurnLd;
    uint32_t it = 0;
    bool ok = true;
    for (int tile = pair; tile < n_tiles && ok; tile += n_pairs) {
      const int tm = m_fastest ? tile % tiles_m : tile / tiles_n, tn = m_fastest ? tile / tiles_m : tile % tiles_n;
      const int row = tm * 256 + (int)rank * 128 + quarter * 32 + lane, col0 = tn * 256 + half * 128;
      const float *sa = p.sa + (long long)(row < p.M ? row : 0) * p.ld_sa;
      const float *sb = p.sb + (long long)(col0 < p.N ? col0 / kBlock : 0) * p.ld_sb;
      float acc[128];
#pragma unroll
      for (int j = 0; j < 128; ++j) acc[j] = 0.f;
      float scale = __ldg(sa) * __ldg(sb);
      for (int ks = 0; ks < slices; ++ks, ++it) {
        const uint32_t buf = it & 1, use = it >> 1;
        // the next slice's scales are fetched while this one's sums are waited for
        const int next = ks + 1 < slices ? ks + 1 : ks;
        const float sa_next = __ldg(sa + next), sb_next = __ldg(sb + next);
        // the whole warp goes on or none of it
        if (!__all_sync(0xffffffffu, !*abort_flag && mbar_wait(smem_u32(&sh->tmem_full[buf]), use & 1, abort_flag))) {
          give_up(abort_flag, p.status, kErrEpilogueWait);
          ok = false;
          break;
        }
        tc_fence_after();
        const uint32_t at = tmem_base + ((uint32_t)(quarter * 32) << 16) + buf * 256 + half * 128;
        uint32_t ra[32], rb[32];
        tmem_ld32(at, ra);
        tmem_wait_ld(ra);
        tmem_ld32(at + 32, rb);
#pragma unroll
        for (int j = 0; j < 32; ++j) acc[0 + j] = fmaf(__uint_as_float(ra[j]), scale, acc[0 + j]);
        tmem_wait_ld(rb);
        tmem_ld32(at + 64, ra);
#pragma unroll
        for (int j = 0; j < 32; ++j) acc[32 + j] = fmaf(__uint_as_float(rb[j]), scale, acc[32 + j]);
        tmem_wait_ld(ra);
        tmem_ld32(at + 96, rb);
#pragma unroll
        for (int j = 0; j < 32; ++j) acc[64 + j] = fmaf(__uint_as_float(ra[j]), scale, acc[64 + j]);
        tmem_wait_ld(rb);
        tc_fence_before();  // all has been read
        __syncwarp();
        if (lane == 0) mbar_arrive_remote(map_to_rank(smem_u32(&sh->tmem_empty[buf]), 0));
#pragma unroll
        for (int j = 0; j < 32; ++j) acc[96 + j] = fmaf(__uint_as_float(rb[j]), scale, acc[96 + j]);
        scale = sa_next * sb_next;
      }
      if (ok && p.vec) {
        TC *c = static_cast<TC *>(p.C) + (long long)row * p.ldc + col0;
        if (row < p.M) {
#pragma unroll
          for (int j = 0; j < 8; ++j)
            if (col0 + 16 * j < p.N) store16(c + 16 * j, acc + 16 * j, p.N - (col0 + 16 * j), true);
        }
      } else if (ok) {
        // Rows that lie anyhow: a thread's own row value by value touched a sector for each (163 x 45,277 float32, K = 416: 72 us a call)
        const int row0 = row - lane;
#pragma unroll
        for (int q = 0; q < 4; ++q) {
          if (col0 + 32 * q >= p.N) break;
          __syncwarp();
#pragma unroll
          for (int j = 0; j < 32; ++j) turn[lane * kTurnLd + j] = acc[32 * q + j];
          __syncwarp();
          const int col = col0 + 32 * q + lane, rows = min(32, p.M - row0);
          TC *c = static_cast<TC *>(p.C) + (long long)row0 * p.ldc + col;
          if (col < p.N) {
#pragma unroll 8
            for (int r = 0; r < rows; ++r) c[(long long)r * p.ldc] = Storage<TC>::narrow(turn[r * kTurnLd + lane]);
          }
        }
      }
    }
  }

  tc_fence_before();
  __syncthreads();
  if (*abort_flag && threadIdx.x == 0) {
    // give this block's copies in flight time to land before the memory is released
    for (int i = 0; i < 2000; ++i) __nanosleep(500);
  }
  cluster_barrier();  // nobody frees tensor memory the pair still uses
  if (warp == 1) {
    tc_fence_after();
    asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" ::"r"(tmem_base), "r"(kTmemCols) : "memory");
  }
}

// ---- few tokens ------------------------------------------------------------------------------------------------------------
// A tile is `tile_rows` <= 128 rows of B, so many that all blocks have the same number of tiles (152 thousand rows in tiles of
// 128 were 1,187 tiles for 148 blocks, nine for some and eight for most); rows of the instruction behind them compute on
// what the ring held before, and nobody reads their sums.
// Warp 0: TMA, warp 1: MMA, the others: epilogue, a row of B and up to 32 tokens a thread.
// Bound by HBM: 16 x 4,096 x 151,936 takes 110 to 118 us, 627 MB at 5.3 to 5.7 TB/s.  64 tokens 135 to 144 us, floor 98: a stage of four
// slices is 98 KB then, so that the ring has two.
constexpr int kSlicesPerStage = 4;  // a row of B is asked for in so many times 128 bytes (16 x 4,096 x 151,936: 111 us, with two 117)

template <int NT>
struct Few {
  static constexpr int kParts = NT <= 32 ? 1 : NT / 32, kTokens = NT / kParts;  // the epilogue's parts of the tokens
  static constexpr int kThreads = 64 + 128 * kParts;
  static constexpr uint32_t kBytesB = 128 * kBlock, kBytesX = NT * kBlock, kSlice = kBytesB + kBytesX,
                            kStage = kSlicesPerStage * kSlice;
  static constexpr int kAccs = 8;
  static constexpr uint32_t kCols = NT * kAccs;
  static constexpr int kStages = (int)(220 * 1024 / kStage);
  struct Shared {
    uint64_t full[kStages], empty[kStages], tmem_full[kAccs], tmem_empty[kAccs];
    uint32_t tmem_base;
    int abort_flag;
    alignas(16) float scale[4 * kParts][2][kTokens];  // read four at a time; an epilogue warp's token scales of a slice
  };
  static constexpr size_t kSmem = 1024 + (size_t)kStages * kStage + sizeof(Shared);
  static_assert(kSmem <= 227 * 1024 && kCols <= kTmemCols, "a block's room");
};

template <typename TC, int NT>
__global__ void __launch_bounds__(Few<NT>::kThreads, 1)
gemm_fp8_few_kernel(const __grid_constant__ CUtensorMap map_x, const __grid_constant__ CUtensorMap map_b, const Params8 p) {
  using F = Few<NT>;
  extern __shared__ uint8_t smem_raw[];
  const uint32_t base = (smem_u32(smem_raw) + 1023u) & ~1023u;
  typename F::Shared *sh =
      reinterpret_cast<typename F::Shared *>(smem_raw + (base - smem_u32(smem_raw)) + (size_t)F::kStages * F::kStage);
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int tiles = (p.N + p.tile_rows - 1) / p.tile_rows, slices = (p.K + kBlock - 1) / kBlock;

  if (threadIdx.x == 0) {
    for (int s = 0; s < F::kStages; ++s) {
      mbar_init(smem_u32(&sh->full[s]), 1);
      mbar_init(smem_u32(&sh->empty[s]), 1);
    }
    for (int b = 0; b < F::kAccs; ++b) {
      mbar_init(smem_u32(&sh->tmem_full[b]), 1);
      mbar_init(smem_u32(&sh->tmem_empty[b]), 4 * F::kParts);
    }
    sh->abort_flag = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    if (blockIdx.x == 0) *p.status = 0;
  }
  if (warp == 1) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(&sh->tmem_base)),
                 "r"(F::kCols)
                 : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem_base = sh->tmem_base;
  volatile int *abort_flag = &sh->abort_flag;

  if (warp == 0) {
    if (lane == 0) {
      uint32_t it = 0;
      for (int tile = blockIdx.x; tile < tiles && !*abort_flag; tile += gridDim.x)
        for (int ks = 0; ks < slices; ks += kSlicesPerStage, ++it) {
          const uint32_t s = it % F::kStages, round = it / F::kStages;
          if (round > 0 && !mbar_wait(smem_u32(&sh->empty[s]), (round - 1) & 1, abort_flag)) {
            give_up(abort_flag, p.status, kErrProducerWait);
            break;
          }
          const uint32_t bar = smem_u32(&sh->full[s]), dst = base + s * F::kStage;
          const int n = min(kSlicesPerStage, slices - ks);
          mbar_expect_tx(bar, (uint32_t)(p.tile_rows + NT) * kBlock * n);
          for (int h = 0; h < n; ++h) tma_load_2d(dst + h * F::kSlice, &map_b, bar, (ks + h) * kBlock, tile * p.tile_rows);
          for (int h = 0; h < n; ++h) tma_load_2d(dst + h * F::kSlice + F::kBytesB, &map_x, bar, (ks + h) * kBlock, 0);
        }
      wait_for_last(sh->empty, it, abort_flag, p.status);
    }
  } else if (warp == 1) {
    if (lane == 0) {
      const uint32_t idesc = instr_desc8(128, NT);
      uint32_t it = 0, sums = 0;
      bool ok = true;
      for (int tile = blockIdx.x; tile < tiles && ok; tile += gridDim.x)
        for (int ks = 0; ks < slices && ok; ks += kSlicesPerStage, ++it) {
          const uint32_t s = it % F::kStages, round = it / F::kStages;
          if (!mbar_wait(smem_u32(&sh->full[s]), round & 1, abort_flag)) {
            give_up(abort_flag, p.status, kErrMmaWaitFull);
            ok = false;
            break;
          }
          const int n = min(kSlicesPerStage, slices - ks);
          for (int h = 0; h < n; ++h, ++sums) {  // every slice has an accumulator of its own
            const uint32_t buf = sums % F::kAccs, use = sums / F::kAccs;
            if (use > 0 && !mbar_wait(smem_u32(&sh->tmem_empty[buf]), (use - 1) & 1, abort_flag)) {
              give_up(abort_flag, p.status, kErrMmaWaitTmem);
              ok = false;
              break;
            }
            tc_fence_after();
            const uint32_t b_addr = base + s * F::kStage + h * F::kSlice;
            const uint64_t bdesc = smem_desc_sw128(b_addr), xdesc = smem_desc_sw128(b_addr + F::kBytesB);
#pragma unroll
            for (int k = 0; k < kBlock / kUmmaK8; ++k)
              umma8(tmem_base + buf * NT, bdesc + k * (kUmmaK8 >> 4), xdesc + k * (kUmmaK8 >> 4), idesc, k > 0 ? 1u : 0u);
            umma_commit(smem_u32(&sh->tmem_full[buf]));
          }
          if (ok) umma_commit(smem_u32(&sh->empty[s]));
        }
    }
  } else {
    const int quarter = warp & 3, part = (warp - 2) >> 2, first = part * F::kTokens;
    float (*mine)[F::kTokens] = sh->scale[warp - 2];
    uint32_t it = 0;
    bool ok = true;
    for (int tile = blockIdx.x; tile < tiles && ok; tile += gridDim.x) {
      const int in_tile = quarter * 32 + lane, row = tile * p.tile_rows + in_tile;
      const bool live = in_tile < p.tile_rows && row < p.N;
      const float *sb = p.sb + (long long)(live ? row / kBlock : 0) * p.ld_sb;
      const bool token = lane < F::kTokens && first + lane < p.M;  // whose scales this lane fetches
      const float *sa = p.sa + (long long)(token ? first + lane : 0) * p.ld_sa;
      float acc[F::kTokens];
#pragma unroll
      for (int j = 0; j < F::kTokens; ++j) acc[j] = 0.f;
      for (int ks = 0; ks < slices; ++ks, ++it) {
        const uint32_t buf = it % F::kAccs, use = it / F::kAccs;
        const float s = __ldg(sb + ks);
        // two sets: the slice before may still be read by a lane that is behind
        float *scale = mine[it & 1];
        if (lane < F::kTokens) scale[lane] = token ? __ldg(sa + ks) : 0.f;
        if (!__all_sync(0xffffffffu, !*abort_flag && mbar_wait(smem_u32(&sh->tmem_full[buf]), use & 1, abort_flag))) {
          give_up(abort_flag, p.status, kErrEpilogueWait);
          ok = false;
          break;
        }
        tc_fence_after();
        const uint32_t at = tmem_base + ((uint32_t)(quarter * 32) << 16) + buf * NT + first;
        uint32_t r[F::kTokens];
        if constexpr (F::kTokens == 16) {
          tmem_ld16_wait(at, r);
        } else {
          tmem_ld32(at, r);
          tmem_wait_ld(r);
        }
        tc_fence_before();  // all has been read
        __syncwarp();
        if (lane == 0) mbar_arrive(smem_u32(&sh->tmem_empty[buf]));
#pragma unroll
        for (int j = 0; j < F::kTokens; j += 4) {
          const float4 t = *reinterpret_cast<const float4 *>(scale + j);
          acc[j] = fmaf(__uint_as_float(r[j]), t.x * s, acc[j]);
          acc[j + 1] = fmaf(__uint_as_float(r[j + 1]), t.y * s, acc[j + 1]);
          acc[j + 2] = fmaf(__uint_as_float(r[j + 2]), t.z * s, acc[j + 2]);
          acc[j + 3] = fmaf(__uint_as_float(r[j + 3]), t.w * s, acc[j + 3]);
        }
      }
      if (ok && live) {
        TC *c = static_cast<TC *>(p.C) + (long long)first * p.ldc + row;
#pragma unroll
        for (int j = 0; j < F::kTokens; ++j)
          if (first + j < p.M) c[(long long)j * p.ldc] = Storage<TC>::narrow(acc[j]);
      }
    }
  }

  tc_fence_before();
  __syncthreads();
  if (*abort_flag && threadIdx.x == 0) {
    for (int i = 0; i < 2000; ++i) __nanosleep(500);
  }
  __syncthreads();
  if (warp == 1) {
    tc_fence_after();
    asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem_base), "r"(F::kCols) : "memory");
  }
}

// ---- the quantiser -----------------------------------------------------------------------------------------------------
// q = e4m3(x / c), c = max(max |x|, 2^-96) / 448 over a block.  A block of threads takes 128 rows x 128 columns, a warp 16 of the
// rows, a lane four neighbouring columns, all of it in registers, so that the matrix is read once; kRowScale: every row has a
// scale of its own.  151,936 x 4,096 bfloat16: 1,526 us, 1.2 TB/s (floor 284), by rows 1,888; one block of 256 threads loads, then
// computes, then stores its 128 x 128, and at 128 registers a thread two of them share an SM.
template <typename T, bool kRowScale>
__global__ void __launch_bounds__(256) quantize_kernel(const T *x, long long ld_x, uint8_t *out, long long ld_out, float *scale,
                                                       long long ld_scale, long long rows, long long cols, int vec) {
  __shared__ float part[8];
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const long long row_blocks = (rows + 127) / 128;
  const long long rb = blockIdx.x % row_blocks, cb = blockIdx.x / row_blocks;
  const long long c = cb * kBlock + lane * 4, r0 = rb * 128 + warp * 16;
  const bool whole = vec && c + 4 <= cols;
  float v[16][4], amax = kLeastAmax;
#pragma unroll
  for (int i = 0; i < 16; ++i) {
#pragma unroll
    for (int j = 0; j < 4; ++j) v[i][j] = 0.f;
    const long long r = r0 + i;
    if (r >= rows) continue;
    const T *p = x + r * ld_x + c;
    if (whole) {
      if constexpr (sizeof(T) == 4) {
        const float4 q = *reinterpret_cast<const float4 *>(p);  // not by __ldg, which may be executed ahead of its checks
        v[i][0] = q.x, v[i][1] = q.y, v[i][2] = q.z, v[i][3] = q.w;
      } else {
        const uint2 q = *reinterpret_cast<const uint2 *>(p);
        const T *e = reinterpret_cast<const T *>(&q);
#pragma unroll
        for (int j = 0; j < 4; ++j) v[i][j] = Storage<T>::widen(e[j]);
      }
    } else {
#pragma unroll
      for (int j = 0; j < 4; ++j)
        if (c + j < cols) v[i][j] = Storage<T>::widen(p[j]);
    }
  }
  const auto warp_max = [](float a) {
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) a = fmaxf(a, __shfl_xor_sync(0xffffffffu, a, o));
    return a;
  };
  if constexpr (!kRowScale) {
#pragma unroll
    for (int i = 0; i < 16; ++i)
#pragma unroll
      for (int j = 0; j < 4; ++j) amax = fmaxf(amax, fabsf(v[i][j]));
    amax = warp_max(amax);
    if (lane == 0) part[warp] = amax;
    __syncthreads();
#pragma unroll
    for (int i = 0; i < 8; ++i) amax = fmaxf(amax, part[i]);
    if (threadIdx.x == 0) scale[rb * ld_scale + cb] = scale_of(amax);
  }
#pragma unroll
  for (int i = 0; i < 16; ++i) {
    const long long r = r0 + i;
    if (r >= rows) break;
    if constexpr (kRowScale) {
      amax = warp_max(fmaxf(fmaxf(fmaxf(fabsf(v[i][0]), fabsf(v[i][1])), fmaxf(fabsf(v[i][2]), fabsf(v[i][3]))), kLeastAmax));
      if (lane == 0) scale[r * ld_scale + cb] = scale_of(amax);
    }
    uint32_t q[1];
    quotients<4>(v[i], scale_of(amax), q);
    uint8_t *o = out + r * ld_out + c;
    if (whole) {
      *reinterpret_cast<uint32_t *>(o) = q[0];
    } else {
#pragma unroll
      for (int j = 0; j < 4; ++j)
        if (c + j < cols) o[j] = (uint8_t)(q[0] >> (8 * j));
    }
  }
}

// ---- host --------------------------------------------------------------------------------------------------------------

// Tensor map of a row-major [rows, k] matrix of bytes for boxes of box_rows x 128 with the 128-byte swizzle; reads past the
// extents return zeros.
bool make_map8(CUtensorMap *map, const void *base, long long rows, long long k, long long ld, int box_rows) {
  EncodeTiledFn fn = encode_fn();
  if (!fn) return false;
  cuuint64_t dims[2] = {(cuuint64_t)k, (cuuint64_t)rows};
  cuuint64_t strides[1] = {(cuuint64_t)ld};
  cuuint32_t box[2] = {(cuuint32_t)kBlock, (cuuint32_t)box_rows};
  cuuint32_t estr[2] = {1, 1};
  return fn(map, CU_TENSOR_MAP_DATA_TYPE_UINT8, 2, const_cast<void *>(base), dims, strides, box, estr,
            CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
            CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

template <typename TC>
cudaError_t launch_pair(const dvp_gemm_fp8_args *a, const Params8 &p, int sms, cudaStream_t stream) {
  CUtensorMap map_a, map_b;
  if (!make_map8(&map_a, a->a, a->M, a->K, a->lda, 128) || !make_map8(&map_b, a->b, a->N, a->K, a->ldb, 128))
    return cudaErrorInvalidValue;
  auto kernel = gemm_fp8_pair_kernel<TC>;
  // the split of the registers is good for a block that has as many as it was compiled for
  static const bool as_compiled = [&] {
    cudaFuncAttributes f;
    return cudaFuncGetAttributes(&f, kernel) == cudaSuccess && f.numRegs >= kRegsLaunch;
  }();
  if (!as_compiled) return cudaErrorLaunchOutOfResources;
  cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)kSmemBytes8);
  if (e != cudaSuccess) return e;
  const long long tiles = ((a->M + 255) / 256) * ((a->N + 255) / 256);
  const long long pairs = tiles < sms / 2 ? tiles : sms / 2;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)(2 * pairs), 1, 1);
  cfg.blockDim = dim3(kThreads8, 1, 1);
  cfg.dynamicSmemBytes = kSmemBytes8;
  cfg.stream = stream;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeClusterDimension;
  attr[0].val.clusterDim.x = 2;
  attr[0].val.clusterDim.y = 1;
  attr[0].val.clusterDim.z = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  return cudaLaunchKernelEx(&cfg, kernel, map_a, map_b, p);
}

template <typename TC, int NT>
cudaError_t launch_few(const dvp_gemm_fp8_args *a, Params8 p, int sms, cudaStream_t stream) {
  // the same number of tiles for every block, each of at least 8 rows
  const long long per_block = (a->N + 128LL * sms - 1) / (128LL * sms);
  long long rows = (a->N + per_block * sms - 1) / (per_block * sms);
  if (rows < 8) rows = 8;
  p.tile_rows = (int)rows;
  CUtensorMap map_x, map_b;
  if (!make_map8(&map_x, a->a, a->M, a->K, a->lda, NT) || !make_map8(&map_b, a->b, a->N, a->K, a->ldb, p.tile_rows))
    return cudaErrorInvalidValue;
  auto kernel = gemm_fp8_few_kernel<TC, NT>;
  cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)Few<NT>::kSmem);
  if (e != cudaSuccess) return e;
  const long long tiles = (a->N + rows - 1) / rows;
  kernel<<<(unsigned)(tiles < sms ? tiles : sms), Few<NT>::kThreads, Few<NT>::kSmem, stream>>>(map_x, map_b, p);
  return cudaGetLastError();
}

// By the tokens: B is read once either way, but of pair tiles a few tokens fill only a part (64 x 4,096 x 151,936: 135 to 144 us, by
// pairs 198 to 204, which is what 128 tokens take; 128 tokens with swapped operands were 284).
template <typename TC>
cudaError_t launch(const dvp_gemm_fp8_args *a, const Params8 &p, int sms, cudaStream_t stream) {
  if (a->M > 64 || a->launch_hint == 1) return launch_pair<TC>(a, p, sms, stream);
  if (a->M <= 16) return launch_few<TC, 16>(a, p, sms, stream);
  if (a->M <= 32) return launch_few<TC, 32>(a, p, sms, stream);
  return launch_few<TC, 64>(a, p, sms, stream);
}

template <typename T>
cudaError_t quantize(const dvp_quantize_fp8_args *a, cudaStream_t stream) {
  const long long blocks = ((a->rows + 127) / 128) * ((a->cols + kBlock - 1) / kBlock);
  const int vec = (uintptr_t)a->x % (4 * sizeof(T)) == 0 && a->ld_x % 4 == 0 && (uintptr_t)a->out % 4 == 0 && a->ld_out % 4 == 0;
  auto kernel = a->block_rows == 1 ? quantize_kernel<T, true> : quantize_kernel<T, false>;
  kernel<<<(unsigned)blocks, 256, 0, stream>>>(static_cast<const T *>(a->x), a->ld_x, static_cast<uint8_t *>(a->out), a->ld_out,
                                               a->scale, a->ld_scale, a->rows, a->cols, vec);
  return cudaGetLastError();
}

}  // namespace fp8
}  // namespace dvp

extern "C" {

int dvp_gemm_fp8(const dvp_gemm_fp8_args *a) {
  using namespace dvp::fp8;
  if (!a || a->struct_size != sizeof(dvp_gemm_fp8_args)) return DVP_ERR_INVALID_ARG;
  if (a->c_dtype != DVP_F32 && a->c_dtype != DVP_BF16 && a->c_dtype != DVP_F16) return DVP_ERR_UNSUPPORTED;
  if (a->M < 0 || a->N < 0 || a->K < 1 || a->launch_hint > 2) return DVP_ERR_INVALID_ARG;
  if (a->M > kMost || a->N > kMost || a->K > kMost) return DVP_ERR_UNSUPPORTED;
  if (((a->M + 255) / 256) * ((a->N + 255) / 256) > kMost) return DVP_ERR_UNSUPPORTED;  // tiles are counted in 32 bits
  if (a->launch_hint == 2 && a->M > 64) return DVP_ERR_INVALID_ARG;
  if (a->M == 0 || a->N == 0) return DVP_OK;
  if (!a->a || !a->b || !a->a_scale || !a->b_scale || !a->c || !a->status) return DVP_ERR_INVALID_ARG;
  const int64_t blocks = (a->K + kBlock - 1) / kBlock;
  if (a->lda < a->K || a->ldb < a->K || a->ldc < a->N || a->ld_a_scale < blocks || a->ld_b_scale < blocks)
    return DVP_ERR_INVALID_ARG;
  if (a->lda % 16 || a->ldb % 16 || (uintptr_t)a->a % 16 || (uintptr_t)a->b % 16) return DVP_ERR_UNSUPPORTED;
  int dev = 0, sms = 0;
  if (cudaGetDevice(&dev) != cudaSuccess || cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev) != cudaSuccess)
    return DVP_ERR_CUDA;
  const int size = a->c_dtype == DVP_F32 ? 4 : 2;
  Params8 p{a->c, a->ldc, a->ld_a_scale, a->ld_b_scale, a->a_scale, a->b_scale, a->status, (int)a->M, (int)a->N, (int)a->K,
            (uintptr_t)a->c % 32 == 0 && a->ldc * size % 32 == 0, 0};
  const cudaStream_t stream = static_cast<cudaStream_t>(a->stream);
  const cudaError_t e = a->c_dtype == DVP_F32    ? launch<float>(a, p, sms, stream)
                        : a->c_dtype == DVP_BF16 ? launch<__nv_bfloat16>(a, p, sms, stream)
                                                 : launch<__half>(a, p, sms, stream);
  if (e == cudaErrorInvalidValue) return DVP_ERR_UNSUPPORTED;
  return e == cudaSuccess ? DVP_OK : DVP_ERR_CUDA;
}

int dvp_quantize_fp8(const dvp_quantize_fp8_args *a) {
  using namespace dvp::fp8;
  if (!a || a->struct_size != sizeof(dvp_quantize_fp8_args)) return DVP_ERR_INVALID_ARG;
  if (a->x_dtype != DVP_F32 && a->x_dtype != DVP_BF16 && a->x_dtype != DVP_F16) return DVP_ERR_UNSUPPORTED;
  if (a->rows < 0 || a->cols < 1 || (a->block_rows != 1 && a->block_rows != 128)) return DVP_ERR_INVALID_ARG;
  if (a->rows > kMost || a->cols > kMost || ((a->rows + 127) / 128) * ((a->cols + 127) / 128) > kMost) return DVP_ERR_UNSUPPORTED;
  if (a->rows == 0) return DVP_OK;
  if (!a->x || !a->out || !a->scale || a->ld_x < a->cols || a->ld_out < a->cols || a->ld_scale < (a->cols + kBlock - 1) / kBlock)
    return DVP_ERR_INVALID_ARG;
  const cudaStream_t stream = static_cast<cudaStream_t>(a->stream);
  const cudaError_t e = a->x_dtype == DVP_F32    ? quantize<float>(a, stream)
                        : a->x_dtype == DVP_BF16 ? quantize<__nv_bfloat16>(a, stream)
                                                 : quantize<__half>(a, stream);
  return e == cudaSuccess ? DVP_OK : DVP_ERR_CUDA;
}

}  // extern "C"
