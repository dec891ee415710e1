// Matrix product of 8-bit floating-point codes with an fp32 scale for each block of 128 along the reduction axis.
//
//   y[m][n] = sum_b sa[m][b] sb[n / 128][b] S_b[m][n],   S_b[m][n] = sum_{k in block b} a[m][k] b[n][k]
//
// The scales are arbitrary fp32 numbers, so the tensor cores can add up one block of 128 only; S_b goes from tensor
// memory to registers, where the running sum is kept in fp32: one fma per output and block, 1/128 of the MMA's
// multiply-adds on pipes of 1/64 of its rate.  sa sb is rounded to fp32 before it meets S_b, by a warp of its own (a second multiplication in the
// sums would double their arithmetic): below 2^-126 that costs bits, and a product that is infinite is reported (PSB_ERR_RANGE).
//
// Many rows (gemm_fp8_kernel): one persistent CTA an SM, or a pair of SMs on one tile (cta_group::2).  Warps of their own copy a, copy
// b, issue the MMAs and multiply the scales; eight warps add up a block of 128 or 256 columns out of one TMEM buffer while the
// MMAs of the next block fill the other, and hand finished tiles to the copy engine.  8192^3: 597 us in a long stream of
// calls (1.84 PFLOP/s; the clocks sink to 1.65 GHz under the power cap), 500 in the first calls on a cool chip (as the times below
// were taken).  A block of 256 x 256 x 128 takes about 950 clocks, 512 of them the MMAs'; in an earlier state, with one of four MMAs and neither
// fmas nor output, it took 650: the wait for the MMAs, the loads from TMEM and the hand-over follow one another, and two buffers are all
// that TMEM holds.  Measured and dropped: sixteen summing warps
// (as fast), halves of the columns handed over one by one (604 us against 576), two warps that issue MMAs (no change), 128 x 256 on
// single SMs (600), a block's first columns fetched before the last arithmetic of the block before it (575 against 560), polls
// that read a clock, more code anywhere in the summing warps (154 KB of it cost 5400 clocks a tile).
// Few rows (stream_fp8_kernel): the other way round, see there.

#include "psb_mma.cuh"

#include <cuda_bf16.h>
#include <cuda_fp16.h>

namespace psb {

namespace {

constexpr uint32_t kBlockK = 128;              // bytes of a row in a stage: one block of scales
constexpr uint32_t kRowsCta = 128;             // rows of a an SM works on
constexpr uint32_t kFirstSumWarp = 4;          // before it: copies of a, MMA, copies of b, scales
constexpr uint32_t kSumWarps = 8;              // warp & 3: quarter of the rows (of the TMEM lanes); upper four: second half of the columns
constexpr uint32_t kGemmThreads = 32 * (kFirstSumWarp + kSumWarps);

constexpr uint32_t kSlotBytes = 2048;          // 32 rows x 64 bytes of output, on their way from an epilogue warp to memory
constexpr uint32_t kBandTiles = 8;             // row tiles that are walked together, so that filter tiles are met again in L2
constexpr uint32_t kMaxRing = 8;
constexpr uint32_t kScaleBlocks = 8;           // blocks of scales that are handed over together, twice buffered
constexpr uint32_t kScaleRow = kRowsCta + 4;   // floats between blocks: eight lanes that write one row's blocks meet eight banks

struct GemmMaps {
  CUtensorMap a, b, out;     // out: boxes of a slot (where its rows start at multiples of 16 bytes)
};

struct GemmParams {
  Fp8GemmArgs g;
  uint32_t k_blocks, n_tiles, stages, idesc;
  uint32_t parts;            // few rows: CTAs of a cluster that share a tile's reduction axis
  uint32_t wide_out;         // output rows start at multiples of 16 bytes
  uint32_t* err;
  uint32_t polls;            // bound of every wait
};

struct GemmCtl {
  unsigned long long full[kMaxRing];
  unsigned long long done[kMaxRing];             // the MMAs on a stage: it may be filled again, its sums may be read
  unsigned long long acc_empty[4];
  unsigned long long scale_full[2], scale_empty[2];
  uint32_t tmem_base;
  uint32_t tiles;            // in all
};

// Waits.  Their bound is counted in polls, without a clock: what reads the clock and the give-up flag of the CTA costs registers
// and code beside 128 accumulators (8192^3 at the time: 541 us like this, 585 with it, 635 where it spilled).  A poll takes from 20 clocks
// to the microseconds for which the hardware suspends it.  A whole warp leaves its wait in one piece, as the tcgen05
// instructions behind it want; a warp that is ahead of the others sleeps between polls and leaves them the issue slots.
__device__ __forceinline__ bool wait_warp(uint32_t bar, uint32_t parity, uint32_t polls) {
#pragma unroll 1
  for (uint32_t i = 0; i < polls; ++i)
    if (__all_sync(0xFFFFFFFFu, mbar_try_wait(bar, parity))) return true;
  return false;
}
template <int kSleep>
__device__ __forceinline__ bool wait_asleep(uint32_t bar, uint32_t parity, uint32_t polls) {
#pragma unroll 1
  for (uint32_t i = 0; i < polls; ++i) {
    if (mbar_try_wait(bar, parity)) return true;
    if (kSleep) __nanosleep(kSleep);
  }
  return false;
}

// A tile: output rows [row, row_end) of one filter, columns from n0 on.
struct GemmTile {
  uint32_t expert, row, row_end, n0;
};

// The experts' runs, as checked: offsets cut to the rows that there are; where they decrease there are no runs at all (runs that share rows could be
// more tiles than 32 bits count).  By the whole block.
template <uint32_t TM>
__device__ __forceinline__ void find_runs(const GemmParams& p, uint32_t* offsets, uint32_t* first, uint32_t* tiles) {
  const uint32_t lane = threadIdx.x & 31u;
  for (uint32_t e = threadIdx.x; e <= p.g.experts; e += blockDim.x) {
    const int o = __ldcg(p.g.offsets + e);
    if (o < 0 || (uint32_t)o > p.g.rows) atomicOr(p.err, kDevErrRange);
    offsets[e] = o < 0 ? 0u : min((uint32_t)o, p.g.rows);
  }
  __syncthreads();
  if (threadIdx.x < 32u) {
    uint32_t carry = 0;
    bool falls = false;
    for (uint32_t e0 = 0; e0 < p.g.experts; e0 += 32u) {
      const uint32_t e = e0 + lane;
      uint32_t mine = 0;
      if (e < p.g.experts) {
        if (offsets[e + 1u] < offsets[e]) falls = true;
        else mine = (offsets[e + 1u] - offsets[e] + TM - 1u) / TM * p.n_tiles;
      }
      uint32_t up = mine;
#pragma unroll
      for (int d = 1; d < 32; d <<= 1) {
        const uint32_t o = __shfl_up_sync(0xFFFFFFFFu, up, d);
        if (lane >= (uint32_t)d) up += o;
      }
      if (e < p.g.experts) first[e] = carry + up - mine;
      carry += __shfl_sync(0xFFFFFFFFu, up, 31);
    }
    if (__any_sync(0xFFFFFFFFu, falls)) {
      carry = 0;
      if (lane == 0) atomicOr(p.err, kDevErrRange);
    }
    if (lane == 0) first[p.g.experts] = *tiles = carry;
  }
}

// first[e] = tiles of the experts before e, offsets as checked (both [experts + 1], shared memory).
template <uint32_t TM, uint32_t BN>
__device__ __forceinline__ GemmTile tile_at(const GemmParams& p, uint32_t t, const uint32_t* first, const uint32_t* offsets) {
  GemmTile tile;
  uint32_t base = 0, rows = p.g.m;
  tile.expert = 0;
  if (p.g.experts) {
    uint32_t lo = 0, hi = p.g.experts;          // first[lo] <= t < first[hi]
    while (hi - lo > 1u) {
      const uint32_t mid = (lo + hi) >> 1;
      if (first[mid] <= t) lo = mid;
      else hi = mid;
    }
    tile.expert = lo;
    base = offsets[lo];
    rows = offsets[lo + 1u] - base;
    t -= first[lo];
  }
  const uint32_t m_tiles = (rows + TM - 1u) / TM;
  const uint32_t band = t / (kBandTiles * p.n_tiles), in = t - band * kBandTiles * p.n_tiles;
  const uint32_t wide = min(kBandTiles, m_tiles - band * kBandTiles);
  const uint32_t nt = in / wide;
  tile.row = base + (band * kBandTiles + in - nt * wide) * TM;
  tile.row_end = base + rows;
  tile.n0 = nt * BN;
  return tile;
}

__device__ __forceinline__ uint32_t cluster_rank() {
  uint32_t r;
  asm volatile("mov.u32 %0, %%cluster_ctarank;" : "=r"(r));
  return r;
}
__device__ __forceinline__ void cluster_sync() {
  __syncwarp();
  asm volatile("barrier.cluster.arrive.aligned;\n\tbarrier.cluster.wait.aligned;" ::: "memory");
}
// The same shared-memory address in another CTA of the cluster.
__device__ __forceinline__ uint32_t in_cta(uint32_t addr, uint32_t rank) {
  uint32_t r;
  asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(r) : "r"(addr), "r"(rank));
  return r;
}

template <int PAIR>
__device__ __forceinline__ void load_a(uint32_t dst, const CUtensorMap* map, uint32_t bar, int x, int y) {
  if (PAIR == 2)
    asm volatile("cp.async.bulk.tensor.2d.cta_group::2.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4}], [%2];"
                 ::"r"(dst), "l"(map), "r"(bar), "r"(x), "r"(y) : "memory");
  else
    tma_load_2d(dst, map, bar, x, y);
}
template <int PAIR>
__device__ __forceinline__ void load_b(uint32_t dst, const CUtensorMap* map, uint32_t bar, int x, int y, int z) {
  if (PAIR == 2)
    asm volatile("cp.async.bulk.tensor.3d.cta_group::2.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4, %5}], [%2];"
                 ::"r"(dst), "l"(map), "r"(bar), "r"(x), "r"(y), "r"(z) : "memory");
  else
    asm volatile("cp.async.bulk.tensor.3d.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4, %5}], [%2];"
                 ::"r"(dst), "l"(map), "r"(bar), "r"(x), "r"(y), "r"(z) : "memory");
}
template <int PAIR>
__device__ __forceinline__ void commit(uint32_t bar) {
  if (PAIR == 2)
    asm volatile("tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.multicast::cluster.b64 [%0], %1;"
                 ::"r"(bar), "h"((uint16_t)3) : "memory");
  else
    tc_commit(bar);
}
template <int PAIR>
__device__ __forceinline__ void mma_f8(uint32_t d_tmem, uint32_t a_lo, uint32_t b_lo, uint32_t desc_hi, uint32_t idesc, uint32_t acc) {
  if (PAIR == 2)
    asm volatile(
        "{\n\t.reg .pred p;\n\t.reg .b64 da, db;\n\t"
        "setp.ne.b32 p, %5, 0;\n\t"
        "mov.b64 da, {%1, %3};\n\t"
        "mov.b64 db, {%2, %3};\n\t"
        "tcgen05.mma.cta_group::2.kind::f8f6f4 [%0], da, db, %4, p;\n\t}"
        ::"r"(d_tmem), "r"(a_lo), "r"(b_lo), "r"(desc_hi), "r"(idesc), "r"(acc));
  else
    asm volatile(
        "{\n\t.reg .pred p;\n\t.reg .b64 da, db;\n\t"
        "setp.ne.b32 p, %5, 0;\n\t"
        "mov.b64 da, {%1, %3};\n\t"
        "mov.b64 db, {%2, %3};\n\t"
        "tcgen05.mma.cta_group::1.kind::f8f6f4 [%0], da, db, %4, p;\n\t}"
        ::"r"(d_tmem), "r"(a_lo), "r"(b_lo), "r"(desc_hi), "r"(idesc), "r"(acc));
}

// Two sums at once, each as fmaf (8192^3 551 us, 565 one by one).
__device__ __forceinline__ void fma_pair(float& x, float& y, uint32_t u, uint32_t v, float s) {
  asm("{\n\t.reg .b64 a, b, c;\n\t"
      "mov.b64 a, {%0, %1};\n\tmov.b64 b, {%2, %3};\n\tmov.b64 c, {%4, %4};\n\t"
      "fma.rn.f32x2 a, b, c, a;\n\t"
      "mov.b64 {%0, %1}, a;\n\t}"
      : "+f"(x), "+f"(y) : "r"(u), "r"(v), "f"(s));
}

template <typename T> __device__ __forceinline__ T round_to(float v);
template <> __device__ __forceinline__ __nv_bfloat16 round_to<__nv_bfloat16>(float v) { return __float2bfloat16_rn(v); }
template <> __device__ __forceinline__ __half round_to<__half>(float v) { return __float2half_rn(v); }

// NaN stays NaN.
__device__ __forceinline__ float relu_of(float y) {
  float r;
  asm("max.NaN.f32 %0, %1, 0f00000000;" : "=f"(r) : "f"(y));
  return r;
}
__device__ __forceinline__ float finish(float y, const float* bias, uint32_t relu) {
  if (bias) y += __ldca(bias);
  return relu ? relu_of(y) : y;
}
__device__ __forceinline__ uint32_t pack_halves(float lo, float hi, bool bf16) {
  uint32_t b, h;
  asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(b) : "f"(hi), "f"(lo));
  asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(h) : "f"(hi), "f"(lo));
  return bf16 ? b : h;
}

// Slots of 32 rows x 64 bytes on their way to memory, columns of `size` bytes from c0 on.  Whole boxes are taken by the copy engine (its 64-byte
// swizzle is the order that keeps the lanes' 16-byte pieces in different banks), so that the warp is back at its sums while
// they drain: all SMs store at the same time.
template <uint32_t kSlots>
__device__ __forceinline__ void send_slots(const GemmMaps& maps, const GemmParams& p, uint8_t* slots, uint32_t size, uint64_t row0, uint32_t rows,
                                           uint32_t col0, uint32_t c0, uint32_t cols, uint32_t lane) {
  const uint32_t per = 64u / size;
  asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
  __syncwarp();
#pragma unroll 1
  for (uint32_t i = 0; i < kSlots; ++i, c0 += per) {
    if (c0 >= cols) break;
    const uint8_t* slot = slots + i * kSlotBytes;
    // (the engine cuts a box at the end of a row to pieces of 16 bytes, not to elements)
    if (p.wide_out && rows == 32u && c0 + per <= cols) {
      if (lane == 0) tma_store_2d(&maps.out, smem_u32(slot), (int)(col0 + c0), (int)row0);
    } else {
      // a lane a column, so that a warp stores what is contiguous (5789 x 4411 x 260: 181 us with a lane storing the 16 bytes it
      // holds value by value)
      const uint32_t c = c0 + lane % per, at = lane % per * size;
      if (c < cols) {
#pragma unroll 4
        for (uint32_t r = lane / per; r < rows; r += 32u / per) {
          const uint8_t* from = slot + r * 64u + (((at >> 4) ^ ((r >> 1) & 3u)) << 4) + (at & 15u);
          const uint64_t to = (row0 + r) * p.g.out_stride + col0 + c;
          if (size == 4u) ((uint32_t*)p.g.out)[to] = *reinterpret_cast<const uint32_t*>(from);
          else ((uint16_t*)p.g.out)[to] = *reinterpret_cast<const uint16_t*>(from);
        }
      }
      __syncwarp();
    }
  }
  if (lane == 0) asm volatile("cp.async.bulk.commit_group;" ::: "memory");
  __syncwarp();
}

__device__ __forceinline__ void put_row(uint8_t* slot, uint32_t lane, const uint32_t (&w)[16]) {
#pragma unroll
  for (uint32_t q = 0; q < 4u; ++q)
    *reinterpret_cast<uint4*>(slot + lane * 64u + ((q ^ ((lane >> 1) & 3u)) << 4)) = make_uint4(w[4 * q], w[4 * q + 1], w[4 * q + 2], w[4 * q + 3]);
}

// A warp's 32 rows (a row a lane) of NC columns: bias, ReLU, rounding, output.  `rows`: rows of these 32 that exist; `cols`: columns that
// exist from the first one on.  The code is kept small: it is run once a tile, and the warps meet it cold (a copy of all of it for every
// type and every 64 bytes of a row made 154 KB, and took 5400 clocks a tile).
template <int NC, uint32_t kSlots>
__device__ __forceinline__ void store_rows(const GemmMaps& maps, const GemmParams& p, float (&acc)[NC], uint8_t* slots, uint64_t row0, uint32_t rows,
                                           uint32_t col0, uint32_t cols, const float* bias, uint32_t lane) {
  if (bias) {
    float mine[NC / 32];          // a lane's columns; the others' come from their lanes
#pragma unroll
    for (int i = 0; i < NC / 32; ++i) mine[i] = 32u * i + lane < cols ? __ldca(bias + 32u * i + lane) : 0.0f;
#pragma unroll
    for (int c = 0; c < NC; ++c) acc[c] += __shfl_sync(0xFFFFFFFFu, mine[c / 32], c % 32);
  }
  if (p.g.relu) {
#pragma unroll
    for (int c = 0; c < NC; ++c) acc[c] = relu_of(acc[c]);
  }
  if (p.g.out_dtype == PSB_DT_F32) {
#pragma unroll
    for (uint32_t c0 = 0; c0 < (uint32_t)NC; c0 += 16u * kSlots) {
      if (lane == 0) asm volatile("cp.async.bulk.wait_group.read 0;" ::: "memory");      // the slots' last boxes have been read
      __syncwarp();
#pragma unroll
      for (uint32_t i = 0; i < kSlots; ++i) {
        uint32_t w[16];
#pragma unroll
        for (uint32_t c = 0; c < 16u; ++c) w[c] = __float_as_uint(acc[c0 + 16u * i + c]);
        put_row(slots + i * kSlotBytes, lane, w);
      }
      send_slots<kSlots>(maps, p, slots, 4u, row0, rows, col0, c0, cols, lane);
    }
  } else {
    static_assert(NC == 32 * kSlots, "a tile's columns in 16 bits fill the slots");
    if (lane == 0) asm volatile("cp.async.bulk.wait_group.read 0;" ::: "memory");
    __syncwarp();
    const bool bf16 = p.g.out_dtype == PSB_DT_BF16;
#pragma unroll
    for (uint32_t i = 0; i < kSlots; ++i) {
      uint32_t w[16];
#pragma unroll
      for (uint32_t c = 0; c < 16u; ++c) w[c] = pack_halves(acc[32u * i + 2u * c], acc[32u * i + 2u * c + 1u], bf16);
      put_row(slots + i * kSlotBytes, lane, w);
    }
    send_slots<kSlots>(maps, p, slots, 2u, row0, rows, col0, 0u, cols, lane);
  }
}

template <int PAIR, int BN>
constexpr uint32_t kGemmStageBytes = (kRowsCta + (uint32_t)BN / PAIR) * kBlockK;
// Output slots of a warp: its columns of a tile in 16 bits.
template <int BN>
constexpr uint32_t kOutSlots = BN / 64;
template <int BN>
constexpr uint32_t kOutBytes = kSumWarps * kOutSlots<BN> * kSlotBytes;
// Products of the scales of a row and of 128 columns, [2][BN / 128][kScaleBlocks][kScaleRow].
template <int BN>
constexpr uint32_t kScaleBytes = 2u * (BN / 128) * kScaleBlocks * kScaleRow * 4u;

// PAIR 2: two SMs work on one tile of 256 rows (cta_group::2): each holds its 128 rows of a and half of the filter's columns,
// and reads the other half through the pair's MMA.
template <int PAIR, int BN>
__global__ void __launch_bounds__(kGemmThreads, 1) gemm_fp8_kernel(const __grid_constant__ GemmMaps maps, const __grid_constant__ GemmParams p) {
  constexpr uint32_t TM = kRowsCta * PAIR;
  constexpr uint32_t kStage = kGemmStageBytes<PAIR, BN>;
  constexpr uint32_t kBufs = 512 / BN;        // accumulators of one block each
  extern __shared__ uint8_t gemm_raw[];
  uint8_t* smem = (uint8_t*)(((uintptr_t)gemm_raw + 1023) & ~(uintptr_t)1023);
  uint8_t* out_stage = smem + p.stages * kStage;
  float* scales = reinterpret_cast<float*>(out_stage + kOutBytes<BN>);
  GemmCtl* ctl = reinterpret_cast<GemmCtl*>(out_stage + kOutBytes<BN> + kScaleBytes<BN>);
  uint32_t* offsets = reinterpret_cast<uint32_t*>(ctl + 1);
  uint32_t* first = offsets + p.g.experts + 1u;
  const uint32_t warp = threadIdx.x >> 5, lane = threadIdx.x & 31u;
  const uint32_t rank = PAIR == 2 ? cluster_rank() : 0u;

  if (threadIdx.x == 0) {
    for (uint32_t s = 0; s < p.stages; ++s) {
      mbar_init(smem_u32(&ctl->full[s]), 1);
      mbar_init(smem_u32(&ctl->done[s]), 1);
    }
    for (uint32_t b = 0; b < kBufs; ++b) mbar_init(smem_u32(&ctl->acc_empty[b]), kSumWarps * PAIR);
    for (uint32_t b = 0; b < 2u; ++b) {
      mbar_init(smem_u32(&ctl->scale_full[b]), 1);
      mbar_init(smem_u32(&ctl->scale_empty[b]), kSumWarps);
    }
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  if (warp == 2) {
    if (PAIR == 2) {
      asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(&ctl->tmem_base)), "r"(kTmemCols) : "memory");
      asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;" ::: "memory");
    } else {
      asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(&ctl->tmem_base)), "r"(kTmemCols) : "memory");
      asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
    }
  }
  pdl_prologue();
  if (p.g.experts) {
    find_runs<TM>(p, offsets, first, &ctl->tiles);
  } else if (threadIdx.x == 0) {
    ctl->tiles = (p.g.m + TM - 1u) / TM * p.n_tiles;
  }
  tc_fence_before();
  if (PAIR == 2) cluster_sync();
  else __syncthreads();
  tc_fence_after();
  const uint32_t tmem_base = ctl->tmem_base, tiles = ctl->tiles;
  const uint32_t step = gridDim.x / PAIR, t0 = blockIdx.x / PAIR;
  bool failed = false;

  if (warp < kFirstSumWarp) {
    if (BN == 256) asm volatile("setmaxnreg.dec.sync.aligned.u32 104;");
    if (warp == 0 || warp == 2) {
      // ------------------------------------------------------------ copies: of a, and of b by a warp of their own
      // (a copy instruction holds its thread for a few hundred clocks)
      if (lane == 0) {
        uint32_t s = 0, ph = 0;
#pragma unroll 1
        for (uint32_t t = t0; t < tiles && !failed; t += step) {
          const GemmTile tile = tile_at<TM, BN>(p, t, first, offsets);
#pragma unroll 1
          for (uint32_t kb = 0; kb < p.k_blocks; ++kb) {
            const uint32_t bar = PAIR == 2 ? in_cta(smem_u32(&ctl->full[s]), 0u) : smem_u32(&ctl->full[s]);
            const uint32_t dst = smem_u32(smem) + s * kStage;
            if (!wait_asleep<20>(smem_u32(&ctl->done[s]), ph ^ 1u, p.polls)) { failed = true; break; }
            if (warp == 0) {
              if (rank == 0u) mbar_expect_tx(smem_u32(&ctl->full[s]), kStage * PAIR);
              load_a<PAIR>(dst, &maps.a, bar, (int)(kb * kBlockK), (int)(tile.row + rank * kRowsCta));
            } else {
              load_b<PAIR>(dst + kRowsCta * kBlockK, &maps.b, bar, (int)(kb * kBlockK), (int)(tile.n0 + rank * (BN / PAIR)), (int)tile.expert);
            }
            if (++s == p.stages) { s = 0; ph ^= 1u; }
          }
        }
      }
      __syncwarp();
    } else if (warp == 1) {
      // ------------------------------------------------------------ MMA
      if (rank == 0u) {
        uint32_t s = 0, ph = 0, buf = 0, bph = 0;
        const uint32_t desc_hi = smem_desc_hi(kBlockK);
#pragma unroll 1
        for (uint32_t t = t0; t < tiles && !failed; t += step) {
#pragma unroll 1
          for (uint32_t kb = 0; kb < p.k_blocks; ++kb) {
            if (!wait_warp(smem_u32(&ctl->full[s]), ph, p.polls) || !wait_warp(smem_u32(&ctl->acc_empty[buf]), bph ^ 1u, p.polls)) {
              failed = true;
              break;
            }
            tc_fence_after();
            const uint32_t a_lo = smem_desc_lo(smem_u32(smem) + s * kStage), b_lo = a_lo + (kRowsCta * kBlockK >> 4);
            if (elect_one()) {
#pragma unroll
              for (uint32_t ks = 0; ks < kBlockK / 32u; ++ks)
                mma_f8<PAIR>(tmem_base + buf * BN, a_lo + ks * 2u, b_lo + ks * 2u, desc_hi, p.idesc, ks);
              commit<PAIR>(smem_u32(&ctl->done[s]));
            }
            __syncwarp();
            if (++s == p.stages) { s = 0; ph ^= 1u; }
            if (++buf == kBufs) { buf = 0; bph ^= 1u; }
          }
        }
      }
    } else {
      // ------------------------------------------------------------ scales
      // Eight lanes read eight blocks of a row (a sector), and leave the products where a warp of the sums finds a block of
      // its 32 rows side by side.
      constexpr uint32_t kHalves = BN / 128, kAtOnce = BN == 128 ? 32 : 16;
      const uint32_t kb_off = lane & 7u, r_off = lane >> 3;
      uint32_t cb = 0, cph = 0;
      float most = 0.0f;          // the largest product (a NaN does not count)
#pragma unroll 1
      for (uint32_t t = t0; t < tiles && !failed; t += step) {
        const GemmTile tile = tile_at<TM, BN>(p, t, first, offsets);
        const uint32_t row = tile.row + rank * kRowsCta + r_off, last = min(tile.row_end, p.g.m) - 1u;
        const float* sb = p.g.b_scale + tile.expert * p.g.b_scale_expert_stride + (uint64_t)(tile.n0 / 128u) * p.g.b_scale_stride;
        const bool second = kHalves == 2u && tile.n0 + 128u < p.g.n;
#pragma unroll 1
        for (uint32_t k0 = 0; k0 < p.k_blocks; k0 += kScaleBlocks) {
          const uint32_t kb = min(k0 + kb_off, p.k_blocks - 1u);
          const float b0 = __ldcg(sb + kb), b1 = second ? __ldcg(sb + p.g.b_scale_stride + kb) : 0.0f;
          if (!wait_asleep<200>(smem_u32(&ctl->scale_empty[cb]), cph ^ 1u, p.polls)) { failed = true; break; }
          float* to = scales + cb * kHalves * kScaleBlocks * kScaleRow + kb_off * kScaleRow + r_off;
#pragma unroll 1
          for (uint32_t r0 = 0; r0 < kRowsCta; r0 += 4u * kAtOnce) {
            float v[kAtOnce];
#pragma unroll
            for (uint32_t i = 0; i < kAtOnce; ++i) v[i] = __ldcg(p.g.a_scale + (uint64_t)min(row + r0 + 4u * i, last) * p.g.a_scale_stride + kb);
#pragma unroll
            for (uint32_t i = 0; i < kAtOnce; ++i) {
              const float q = v[i] * b0;
              to[r0 + 4u * i] = q;
              most = fmaxf(most, fabsf(q));
              if (kHalves == 2u) {
                const float q1 = v[i] * b1;
                to[kScaleBlocks * kScaleRow + r0 + 4u * i] = q1;
                most = fmaxf(most, fabsf(q1));
              }
            }
          }
          __syncwarp();
          if (lane == 0) mbar_arrive(smem_u32(&ctl->scale_full[cb]));
          if (++cb == 2u) { cb = 0; cph ^= 1u; }
        }
      }
      if (most == INFINITY) atomicOr(p.err, kDevErrRange);
    }
  } else {
    // -------------------------------------------------------------- scaled sums and output
    if (BN == 256) asm volatile("setmaxnreg.inc.sync.aligned.u32 200;");
    constexpr int NC = BN / 2;                 // columns of a warp
    const uint32_t quarter = warp & 3u, part = (warp - kFirstSumWarp) >> 2;
    uint8_t* slots = out_stage + (warp - kFirstSumWarp) * (kOutSlots<BN> * kSlotBytes);
    uint32_t s = 0, ph = 0, buf = 0, cb = 0, cph = 0;
#pragma unroll 1
    for (uint32_t t = t0; t < tiles && !failed; t += step) {
      float acc[NC];
#pragma unroll
      for (int i = 0; i < NC; ++i) acc[i] = 0.0f;
      const uint32_t taddr = tmem_base + part * NC + ((quarter * 32u) << 16);
      const float* sc_of = scales + (part * NC / 128u) * kScaleBlocks * kScaleRow + quarter * 32u + lane;
#pragma unroll 1
      for (uint32_t kb = 0; kb < p.k_blocks; ++kb) {
        if (kb % kScaleBlocks == 0u && !wait_warp(smem_u32(&ctl->scale_full[cb]), cph, p.polls)) { failed = true; break; }
        const float sc = sc_of[(cb * (BN / 128) * kScaleBlocks + kb % kScaleBlocks) * kScaleRow];
        if (!wait_warp(smem_u32(&ctl->done[s]), ph, p.polls)) { failed = true; break; }
        tc_fence_after();
        auto handed_back = [&]() {
          tc_fence_before();
          __syncwarp();
          if (lane == 0) {
            if (PAIR == 2)
              asm volatile("mbarrier.arrive.shared::cluster.b64 _, [%0];" ::"r"(in_cta(smem_u32(&ctl->acc_empty[buf]), 0u)) : "memory");
            else
              mbar_arrive(smem_u32(&ctl->acc_empty[buf]));
          }
          __syncwarp();
        };
        // (one load at a time: the other warp of the scheduler computes meanwhile; a second one in flight took 8192^3 from 505 us to 560)
#pragma unroll
        for (int c = 0; c < NC / 16; ++c) {
          uint32_t v[16];
          tc_ld16(taddr + buf * BN + c * 16, v);
          tc_wait_ld();
          if (c + 1 == NC / 16) handed_back();
#pragma unroll
          for (int i = 0; i < 16; i += 2) fma_pair(acc[c * 16 + i], acc[c * 16 + i + 1], v[i], v[i + 1], sc);
        }
        if (++s == p.stages) { s = 0; ph ^= 1u; }
        if (++buf == kBufs) buf = 0;
        if (kb % kScaleBlocks == kScaleBlocks - 1u || kb == p.k_blocks - 1u) {
          __syncwarp();
          if (lane == 0) mbar_arrive(smem_u32(&ctl->scale_empty[cb]));
          __syncwarp();
          if (++cb == 2u) { cb = 0; cph ^= 1u; }
        }
      }
      if (failed) break;
      // (found again: what the output needs takes no registers during the sums)
      const GemmTile tile = tile_at<TM, BN>(p, t, first, offsets);
      const uint32_t row0 = tile.row + rank * kRowsCta + quarter * 32u, col0 = tile.n0 + part * NC;
      const uint32_t rows = row0 < tile.row_end ? min(32u, tile.row_end - row0) : 0u;
      const uint32_t cols = col0 < p.g.n ? min((uint32_t)NC, p.g.n - col0) : 0u;
      const float* bias = p.g.bias ? p.g.bias + (uint64_t)tile.expert * p.g.n + col0 : nullptr;
      store_rows<NC, kOutSlots<BN>>(maps, p, acc, slots, row0, rows, col0, cols, bias, lane);
    }
    if (lane == 0) asm volatile("cp.async.bulk.wait_group 0;" ::: "memory");
  }

  // ---------------------------------------------------------------- common exit
  if (failed) {
    if (lane == 0) atomicOr(p.err, kDevErrTimeout);
    // give copies and MMAs already in flight time to land before the CTA retires
    for (int i = 0; i < 64; ++i) __nanosleep(2000);
  }
  __syncwarp();
  tc_fence_before();
  if (PAIR == 2) cluster_sync();
  else __syncthreads();
  if (warp == 2) {
    tc_fence_after();
    if (PAIR == 2)
      asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" ::"r"(tmem_base), "r"(kTmemCols) : "memory");
    else
      asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem_base), "r"(kTmemCols) : "memory");
  }
}

// ---- few rows ------------------------------------------------------------------------------------------------------------
// The filter's rows take the MMA's 128 rows and BT rows of a its columns, so that an SM does little but stream the filter, and the
// reduction axis is cut among the `parts` CTAs of a cluster where the tiles leave SMs idle.  Two groups of four warps
// take the blocks in turns (a block costs a warp about 500 clocks of waiting and hand-over; 16 KB of the filter come in
// 700); their sums, and those of the cluster's CTAs, are added in a fixed order through shared memory.
constexpr uint32_t kStreamGroups = 2;
constexpr uint32_t kStreamBufs = 4;            // accumulators; even, as the stages, so that a group meets its own ones only
constexpr uint32_t kStreamMaxRing = 12;
constexpr uint32_t kMaxParts = 8;

struct StreamCtl {
  unsigned long long full[kStreamMaxRing], done[kStreamMaxRing];
  unsigned long long acc_empty[kStreamBufs];
  unsigned long long scale_full[2], scale_empty[2];
  uint32_t tmem_base, tiles;
  volatile uint32_t gave_up;   // a warp of the sums did: all of them stop at the next barrier
};
template <int BT> constexpr uint32_t kStreamStageBytes = (kRowsCta + BT) * kBlockK;
template <int BT> constexpr uint32_t kStreamPartBytes = kStreamGroups * BT * kRowsCta * 4u;
template <int BT> constexpr uint32_t kStreamScaleBytes = 2u * kScaleBlocks * BT * 4u;

__device__ __forceinline__ float ld_cluster(uint32_t addr) {
  float v;
  asm volatile("ld.shared::cluster.f32 %0, [%1];" : "=f"(v) : "r"(addr) : "memory");
  return v;
}
__device__ __forceinline__ void store_one(const GemmParams& p, uint64_t at, float y) {
  if (p.g.out_dtype == PSB_DT_F32) ((float*)p.g.out)[at] = y;
  else if (p.g.out_dtype == PSB_DT_BF16) ((__nv_bfloat16*)p.g.out)[at] = round_to<__nv_bfloat16>(y);
  else ((__half*)p.g.out)[at] = round_to<__half>(y);
}

template <int BT>
__global__ void __launch_bounds__(kGemmThreads, 1) stream_fp8_kernel(const __grid_constant__ GemmMaps maps, const __grid_constant__ GemmParams p) {
  constexpr uint32_t kStage = kStreamStageBytes<BT>;
  constexpr uint32_t BN = kRowsCta;           // columns of out, rows of the MMA
  extern __shared__ uint8_t gemm_raw[];
  uint8_t* smem = (uint8_t*)(((uintptr_t)gemm_raw + 1023) & ~(uintptr_t)1023);
  float* part = reinterpret_cast<float*>(smem + p.stages * kStage);             // [group][BT][128]
  float* scales = part + kStreamPartBytes<BT> / 4u;                              // [2][kScaleBlocks][BT]
  StreamCtl* ctl = reinterpret_cast<StreamCtl*>(scales + kStreamScaleBytes<BT> / 4u);
  uint32_t* offsets = reinterpret_cast<uint32_t*>(ctl + 1);
  uint32_t* first = offsets + p.g.experts + 1u;
  const uint32_t warp = threadIdx.x >> 5, lane = threadIdx.x & 31u;
  const uint32_t parts = p.parts, rank = parts > 1u ? cluster_rank() : 0u;

  if (threadIdx.x == 0) {
    for (uint32_t s = 0; s < p.stages; ++s) {
      mbar_init(smem_u32(&ctl->full[s]), 1);
      mbar_init(smem_u32(&ctl->done[s]), 1);
    }
    for (uint32_t b = 0; b < kStreamBufs; ++b) mbar_init(smem_u32(&ctl->acc_empty[b]), kSumWarps / kStreamGroups);
    for (uint32_t b = 0; b < 2u; ++b) {
      mbar_init(smem_u32(&ctl->scale_full[b]), 1);
      mbar_init(smem_u32(&ctl->scale_empty[b]), kSumWarps);
    }
    ctl->gave_up = 0u;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  if (warp == 1) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(&ctl->tmem_base)), "r"(kTmemCols) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
  }
  pdl_prologue();
  if (p.g.experts) {
    find_runs<BT>(p, offsets, first, &ctl->tiles);
  } else if (threadIdx.x == 0) {
    ctl->tiles = (p.g.m + BT - 1u) / BT * p.n_tiles;
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem_base = ctl->tmem_base, tiles = ctl->tiles;
  const uint32_t step = gridDim.x / parts, t0 = blockIdx.x / parts;
  const uint32_t k_lo = p.k_blocks * rank / parts, k_hi = p.k_blocks * (rank + 1u) / parts;
  bool failed = false;

  if (warp == 0 || warp == 2) {
    // -------------------------------------------------------------- copies: of the filter (warp 0), of a (warp 2)
    if (lane == 0) {
      uint32_t s = 0, ph = 0;
#pragma unroll 1
      for (uint32_t t = t0; t < tiles && !failed; t += step) {
        const GemmTile tile = tile_at<BT, BN>(p, t, first, offsets);
#pragma unroll 1
        for (uint32_t kb = k_lo; kb < k_hi; ++kb) {
          const uint32_t bar = smem_u32(&ctl->full[s]), dst = smem_u32(smem) + s * kStage;
          if (!wait_asleep<20>(smem_u32(&ctl->done[s]), ph ^ 1u, p.polls)) { failed = true; break; }
          if (warp == 0) {
            mbar_expect_tx(bar, kStage);
            load_b<1>(dst, &maps.b, bar, (int)(kb * kBlockK), (int)tile.n0, (int)tile.expert);
          } else {
            load_a<1>(dst + kRowsCta * kBlockK, &maps.a, bar, (int)(kb * kBlockK), (int)tile.row);
          }
          if (++s == p.stages) { s = 0; ph ^= 1u; }
        }
      }
    }
    __syncwarp();
  } else if (warp == 1) {
    // -------------------------------------------------------------- MMA
    uint32_t s = 0, ph = 0, buf = 0, bph = 0;
    const uint32_t desc_hi = smem_desc_hi(kBlockK);
#pragma unroll 1
    for (uint32_t t = t0; t < tiles && !failed; t += step) {
#pragma unroll 1
      for (uint32_t kb = k_lo; kb < k_hi; ++kb) {
        if (!wait_warp(smem_u32(&ctl->full[s]), ph, p.polls) || !wait_warp(smem_u32(&ctl->acc_empty[buf]), bph ^ 1u, p.polls)) {
          failed = true;
          break;
        }
        tc_fence_after();
        const uint32_t a_lo = smem_desc_lo(smem_u32(smem) + s * kStage), b_lo = a_lo + (kRowsCta * kBlockK >> 4);
        if (elect_one()) {
#pragma unroll
          for (uint32_t ks = 0; ks < kBlockK / 32u; ++ks)
            mma_f8<1>(tmem_base + buf * BT, a_lo + ks * 2u, b_lo + ks * 2u, desc_hi, p.idesc, ks);
          commit<1>(smem_u32(&ctl->done[s]));
        }
        __syncwarp();
        if (++s == p.stages) { s = 0; ph ^= 1u; }
        if (++buf == kStreamBufs) { buf = 0; bph ^= 1u; }
      }
    }
  } else if (warp == 3) {
    // -------------------------------------------------------------- scales: products for the rows of a, eight blocks at a time
    const uint32_t kb_off = lane & 7u, r_off = lane >> 3;
    uint32_t cb = 0, cph = 0;
    float most = 0.0f;            // the largest product (a NaN does not count)
#pragma unroll 1
    for (uint32_t t = t0; t < tiles && !failed; t += step) {
      const GemmTile tile = tile_at<BT, BN>(p, t, first, offsets);
      const uint32_t row = tile.row + r_off, last = min(tile.row_end, p.g.m) - 1u;
      const float* sb = p.g.b_scale + tile.expert * p.g.b_scale_expert_stride + (uint64_t)(tile.n0 / 128u) * p.g.b_scale_stride;
#pragma unroll 1
      for (uint32_t k0 = k_lo; k0 < k_hi; k0 += kScaleBlocks) {
        const uint32_t kb = min(k0 + kb_off, k_hi - 1u);
        const float b0 = __ldcg(sb + kb);
        float v[BT / 4];
#pragma unroll
        for (uint32_t i = 0; i < BT / 4u; ++i) v[i] = __ldcg(p.g.a_scale + (uint64_t)min(row + 4u * i, last) * p.g.a_scale_stride + kb);
        if (!wait_warp(smem_u32(&ctl->scale_empty[cb]), cph ^ 1u, p.polls)) { failed = true; break; }
        float* to = scales + (cb * kScaleBlocks + kb_off) * BT + r_off;
#pragma unroll
        for (uint32_t i = 0; i < BT / 4u; ++i) {
          const float q = v[i] * b0;
          to[4u * i] = q;
          most = fmaxf(most, fabsf(q));
        }
        __syncwarp();
        if (lane == 0) mbar_arrive(smem_u32(&ctl->scale_full[cb]));
        if (++cb == 2u) { cb = 0; cph ^= 1u; }
      }
    }
    if (most == INFINITY) atomicOr(p.err, kDevErrRange);
  } else {
    // -------------------------------------------------------------- scaled sums: a lane a column of out, a register a row
    const uint32_t quarter = warp & 3u, group = (warp - kFirstSumWarp) >> 2, col = quarter * 32u + lane;
    uint32_t s = 0, ph = 0, buf = 0, cb = 0, cph = 0, turn = 0;
#pragma unroll 1
    for (uint32_t t = t0; t < tiles && !failed; t += step) {
      float acc[BT];
#pragma unroll
      for (int i = 0; i < BT; ++i) acc[i] = 0.0f;
#pragma unroll 1
      for (uint32_t k0 = k_lo; k0 < k_hi && !failed; k0 += kScaleBlocks) {
        if (!wait_warp(smem_u32(&ctl->scale_full[cb]), cph, p.polls)) { failed = true; break; }
#pragma unroll 1
        for (uint32_t kb = k0; kb < min(k0 + kScaleBlocks, k_hi); ++kb) {
          if ((turn++ & 1u) == group) {
            if (!wait_warp(smem_u32(&ctl->done[s]), ph, p.polls)) { failed = true; break; }
            tc_fence_after();
            const float4* sc = reinterpret_cast<const float4*>(scales + (cb * kScaleBlocks + kb - k0) * BT);
#pragma unroll
            for (int c = 0; c < BT / 16; ++c) {
              uint32_t v[16];
              tc_ld16(tmem_base + buf * BT + c * 16 + ((quarter * 32u) << 16), v);
              tc_wait_ld();
#pragma unroll
              for (int i = 0; i < 4; ++i) {
                const float4 q = sc[c * 4 + i];
                acc[c * 16 + 4 * i] = __fmaf_rn(__uint_as_float(v[4 * i]), q.x, acc[c * 16 + 4 * i]);
                acc[c * 16 + 4 * i + 1] = __fmaf_rn(__uint_as_float(v[4 * i + 1]), q.y, acc[c * 16 + 4 * i + 1]);
                acc[c * 16 + 4 * i + 2] = __fmaf_rn(__uint_as_float(v[4 * i + 2]), q.z, acc[c * 16 + 4 * i + 2]);
                acc[c * 16 + 4 * i + 3] = __fmaf_rn(__uint_as_float(v[4 * i + 3]), q.w, acc[c * 16 + 4 * i + 3]);
              }
            }
            tc_fence_before();
            __syncwarp();
            if (lane == 0) mbar_arrive(smem_u32(&ctl->acc_empty[buf]));
            __syncwarp();
          }
          if (++s == p.stages) { s = 0; ph ^= 1u; }
          if (++buf == kStreamBufs) buf = 0;
        }
        __syncwarp();
        if (lane == 0) mbar_arrive(smem_u32(&ctl->scale_empty[cb]));
        __syncwarp();
        if (++cb == 2u) { cb = 0; cph ^= 1u; }
      }
#pragma unroll
      for (int i = 0; i < BT; ++i) part[(group * BT + i) * kRowsCta + col] = acc[i];
      if (parts == 1u) {
        if (failed) ctl->gave_up = 1u;
        asm volatile("bar.sync 1, %0;" ::"n"(kSumWarps * 32) : "memory");
        failed = ctl->gave_up != 0u;
        const GemmTile tile = tile_at<BT, BN>(p, t, first, offsets);
        const uint32_t n = tile.n0 + col, rows = min((uint32_t)BT, tile.row_end - tile.row);
        if (n < p.g.n && !failed) {
          const float* bias = p.g.bias ? p.g.bias + (uint64_t)tile.expert * p.g.n + n : nullptr;
          for (uint32_t r = group; r < rows; r += kStreamGroups)
            store_one(p, (uint64_t)(tile.row + r) * p.g.out_stride + n,
                      finish(part[r * kRowsCta + col] + part[(BT + r) * kRowsCta + col], bias, p.g.relu));
        }
        asm volatile("bar.sync 1, %0;" ::"n"(kSumWarps * 32) : "memory");
      }
    }
  }

  if (parts > 1u) {
    // one tile a cluster: each CTA adds up and stores its share of the rows
    cluster_sync();
    if (t0 < tiles) {
      const GemmTile tile = tile_at<BT, BN>(p, t0, first, offsets);
      const uint32_t share = BT / parts, rows = min((uint32_t)BT, tile.row_end - tile.row);
      uint32_t from[kMaxParts];
#pragma unroll
      for (uint32_t q = 0; q < kMaxParts; ++q) from[q] = in_cta(smem_u32(part), q < parts ? q : 0u);
      for (uint32_t i = threadIdx.x; i < share * kRowsCta; i += kGemmThreads) {
        const uint32_t r = rank * share + i / kRowsCta, col = i % kRowsCta, n = tile.n0 + col;
        if (r >= rows || n >= p.g.n) continue;
        float y = 0.0f;
#pragma unroll
        for (uint32_t q = 0; q < kMaxParts; ++q)
          if (q < parts) y += ld_cluster(from[q] + (r * kRowsCta + col) * 4u) + ld_cluster(from[q] + ((BT + r) * kRowsCta + col) * 4u);
        store_one(p, (uint64_t)(tile.row + r) * p.g.out_stride + n,
                  finish(y, p.g.bias ? p.g.bias + (uint64_t)tile.expert * p.g.n + n : nullptr, p.g.relu));
      }
    }
  }

  // ---------------------------------------------------------------- common exit
  if (failed) {
    if (lane == 0) atomicOr(p.err, kDevErrTimeout);
    // give copies and MMAs already in flight time to land before the CTA retires
    for (int i = 0; i < 64; ++i) __nanosleep(2000);
  }
  __syncwarp();
  tc_fence_before();
  if (parts > 1u) cluster_sync();
  else __syncthreads();
  if (warp == 1) {
    tc_fence_after();
    asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem_base), "r"(kTmemCols) : "memory");
  }
}

// ---- rows in the order of the experts -----------------------------------------------------------------------------------------
// Row r of the copy is row order[r] of a, with its scales: 16 bytes a thread.  (The copy engine's gather of four rows an
// instruction inside the product took 1400 us where rows in order take 390, 16384 rows of 4096 over 8 experts; this copy takes 25.)
struct GatherArgs {
  const uint8_t* a;
  const float* scale;
  const int32_t *order, *last;
  uint8_t* to;
  float* scale_to;
  uint32_t m, rows, k, k_blocks, pieces;      // pieces of 16 bytes in a row of `to`
  uint64_t a_stride, scale_stride;
  uint32_t* err;
};

__global__ void __launch_bounds__(256) gather_rows_kernel(const GatherArgs g) {
  pdl_prologue();
  const int used = __ldcg(g.last);
  const uint32_t rows = used < 0 ? 0u : min((uint32_t)used, g.rows);
  // pieces of codes, then one of scales per block of 128 pieces' row
  const uint32_t per_row = g.pieces + (g.k_blocks + 3u) / 4u;
  const uint32_t i0 = blockIdx.x * blockDim.x + threadIdx.x, stride = gridDim.x * blockDim.x;
  const uint32_t step_r = stride / per_row, step_c = stride - step_r * per_row;
  uint32_t r = i0 / per_row, c = i0 - r * per_row;
  for (; r < rows; r += step_r) {
    const int o = __ldcg(g.order + r);
    if (c == 0u && (o < 0 || (uint32_t)o >= g.m)) atomicOr(g.err, kDevErrRange);
    const uint64_t from = o < 0 ? 0u : min((uint32_t)o, g.m - 1u);
    if (c < g.pieces) {
      const uint8_t* src = g.a + from * g.a_stride + c * 16u;
      uint8_t* dst = g.to + (uint64_t)r * g.pieces * 16u + c * 16u;
      if (c * 16u + 16u <= g.k) *reinterpret_cast<uint4*>(dst) = *reinterpret_cast<const uint4*>(src);
      else
        for (uint32_t b = 0; c * 16u + b < g.k; ++b) dst[b] = src[b];
    } else {
      for (uint32_t b = (c - g.pieces) * 4u; b < min((c - g.pieces) * 4u + 4u, g.k_blocks); ++b)
        g.scale_to[(uint64_t)r * g.k_blocks + b] = g.scale[from * g.scale_stride + b];
    }
    c += step_c;
    if (c >= per_row) { c -= per_row; ++r; }
  }
}

typedef CUresult (*EncodeTiled)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*, const cuuint64_t*,
                                const cuuint32_t*, const cuuint32_t*, CUtensorMapInterleave, CUtensorMapSwizzle,
                                CUtensorMapL2promotion, CUtensorMapFloatOOBfill);

// Codes [depth][rows][k], boxes of 128 bytes x box_rows.
bool encode_codes(void* encode, CUtensorMap* map, const uint8_t* codes, uint32_t rank, uint64_t k, uint64_t rows, uint64_t depth,
                  uint64_t stride, uint64_t depth_stride, uint32_t box_rows) {
  cuuint64_t dims[3] = {k, rows, depth};
  cuuint64_t strides[2] = {stride, depth_stride};
  cuuint32_t box[3] = {kBlockK, box_rows, 1};
  cuuint32_t estr[3] = {1, 1, 1};
  return ((EncodeTiled)encode)(map, CU_TENSOR_MAP_DATA_TYPE_UINT8, rank, const_cast<uint8_t*>(codes), dims, strides, box, estr,
                               CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
                               CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

// What both launches share.
psb_status fill_params(psb_ctx* ctx, const Fp8GemmArgs& a, uint32_t bn, uint32_t box_a, uint32_t box_b, GemmMaps& maps, GemmParams& p) {
  p.g = a;
  p.k_blocks = (a.k + kBlockK - 1u) / kBlockK;
  p.n_tiles = (a.n + bn - 1u) / bn;
  p.parts = 1;
  p.err = ctx->err_dev;
  p.polls = (uint32_t)(ctx->wait_limit_cycles / 256u < 0x7FFFFFFFu ? ctx->wait_limit_cycles / 256u + 1u : 0x7FFFFFFFu);
  const uint64_t size = a.out_dtype == PSB_DT_F32 ? 4u : 2u;
  p.wide_out = (((uintptr_t)a.out | a.out_stride * size) & 15u) == 0u;
  if (!encode_codes(ctx->encode_tiled, &maps.a, a.a, 2, a.k, a.m, 1, a.a_stride, 0, box_a) ||
      !encode_codes(ctx->encode_tiled, &maps.b, a.b, 3, a.k, a.n, a.experts ? a.experts : 1u, a.b_stride,
                    a.experts ? a.b_expert_stride : a.b_stride * a.n, box_b))
    return PSB_ERR_CUDA;
  return PSB_OK;
}

// fp32 accumulators; formats of the operands; columns / 8; rows / 16
uint32_t instruction(uint32_t rows_dtype, uint32_t cols_dtype, uint32_t rows, uint32_t cols) {
  return (1u << 4) | ((rows_dtype == PSB_DT_E5M2 ? 1u : 0u) << 7) | ((cols_dtype == PSB_DT_E5M2 ? 1u : 0u) << 10) | ((cols >> 3) << 17) |
         ((rows >> 4) << 24);
}

// Upper bound of the tiles of `height` rows: every expert has one that is not full.
uint64_t row_tiles(const Fp8GemmArgs& a, uint32_t height) {
  return a.experts ? (uint64_t)a.rows / height + (a.experts < a.rows ? a.experts : a.rows) : ((uint64_t)a.m + height - 1u) / height;
}

template <typename K>
psb_status launch_gemm(K kernel, uint32_t grid, uint32_t cluster, size_t smem, const GemmMaps& maps, const GemmParams& p, cudaStream_t s) {
  const cudaError_t limit = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)kSmemBudget);
  cudaLaunchAttribute attr[2];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  attr[1].id = cudaLaunchAttributeClusterDimension;
  attr[1].val.clusterDim.x = cluster;
  attr[1].val.clusterDim.y = attr[1].val.clusterDim.z = 1;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(grid);
  cfg.blockDim = dim3(kGemmThreads);
  cfg.dynamicSmemBytes = smem;
  cfg.stream = s;
  cfg.attrs = attr;
  cfg.numAttrs = cluster > 1u ? 2 : 1;
  return launched(limit == cudaSuccess ? cudaLaunchKernelEx(&cfg, kernel, maps, p) : limit) == cudaSuccess ? PSB_OK : PSB_ERR_CUDA;
}

uint32_t runs_bytes(const Fp8GemmArgs& a) { return a.experts ? (a.experts + 1u) * 8u : 0u; }

template <int PAIR, int BN>
psb_status launch_tiles(psb_ctx* ctx, const Fp8GemmArgs& a, cudaStream_t s) {
  GemmMaps maps;
  GemmParams p;
  const psb_status st = fill_params(ctx, a, BN, kRowsCta, BN / PAIR, maps, p);
  if (st != PSB_OK) return st;
  p.idesc = instruction(a.a_dtype, a.b_dtype, kRowsCta * PAIR, BN);
  if (p.wide_out) {
    const bool wide = a.out_dtype == PSB_DT_F32;
    cuuint64_t dims[2] = {a.n, a.rows}, strides[1] = {a.out_stride * (wide ? 4u : 2u)};
    cuuint32_t box[2] = {wide ? 16u : 32u, 32u}, estr[2] = {1, 1};
    if (((EncodeTiled)ctx->encode_tiled)(&maps.out, wide ? CU_TENSOR_MAP_DATA_TYPE_FLOAT32 : CU_TENSOR_MAP_DATA_TYPE_UINT16, 2, a.out, dims, strides, box,
                                         estr, CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_64B, CU_TENSOR_MAP_L2_PROMOTION_NONE,
                                         CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) != CUDA_SUCCESS)
      return PSB_ERR_CUDA;
  }
  const uint32_t rest = kOutBytes<BN> + kScaleBytes<BN> + sizeof(GemmCtl) + runs_bytes(a) + 1024u;
  p.stages = (uint32_t)((kSmemBudget - rest) / kGemmStageBytes<PAIR, BN>);
  if (p.stages > kMaxRing) p.stages = kMaxRing;
  const uint64_t tiles = row_tiles(a, kRowsCta * PAIR) * p.n_tiles;
  const uint32_t most = (uint32_t)ctx->sm_count / PAIR;
  return launch_gemm(gemm_fp8_kernel<PAIR, BN>, (uint32_t)(tiles < most ? tiles : most) * PAIR, PAIR,
                     p.stages * kGemmStageBytes<PAIR, BN> + rest, maps, p, s);
}

template <int BT>
psb_status launch_stream(psb_ctx* ctx, const Fp8GemmArgs& a, cudaStream_t s) {
  GemmMaps maps;
  GemmParams p;
  const psb_status st = fill_params(ctx, a, kRowsCta, BT, kRowsCta, maps, p);
  if (st != PSB_OK) return st;
  p.idesc = instruction(a.b_dtype, a.a_dtype, kRowsCta, BT);
  const uint32_t rest = kStreamPartBytes<BT> + kStreamScaleBytes<BT> + sizeof(StreamCtl) + runs_bytes(a) + 1024u;
  p.stages = (uint32_t)((kSmemBudget - rest) / kStreamStageBytes<BT>) & ~1u;
  if (p.stages > kStreamMaxRing) p.stages = kStreamMaxRing;
  const uint64_t tiles = row_tiles(a, BT) * p.n_tiles;
  while (p.parts < kMaxParts && tiles * p.parts * 2u <= (uint32_t)ctx->sm_count && p.k_blocks >= p.parts * 4u) p.parts *= 2u;
  const uint32_t grid = p.parts > 1u ? (uint32_t)tiles * p.parts : (uint32_t)(tiles < (uint32_t)ctx->sm_count ? tiles : (uint32_t)ctx->sm_count);
  return launch_gemm(stream_fp8_kernel<BT>, grid, p.parts, p.stages * kStreamStageBytes<BT> + rest, maps, p, s);
}

}  // namespace

size_t gemm_fp8_scratch_bytes(const Fp8GemmArgs& a) {
  return a.order ? (size_t)a.rows * (round_up(a.k, 16u) + (a.k + kBlockK - 1u) / kBlockK * 4u) : 0u;
}

psb_status launch_gemm_fp8(psb_ctx* ctx, const Fp8GemmArgs& given, void* scratch, cudaStream_t s) {
  if (!ctx->encode_tiled) return PSB_ERR_UNSUPPORTED;
  Fp8GemmArgs a = given;
  if (a.order) {
    GatherArgs g;
    g.a = a.a;
    g.scale = a.a_scale;
    g.order = a.order;
    g.last = a.offsets + a.experts;
    g.to = (uint8_t*)scratch;
    g.m = a.m;
    g.rows = a.rows;
    g.k = a.k;
    g.k_blocks = (a.k + kBlockK - 1u) / kBlockK;
    g.pieces = round_up(a.k, 16u) / 16u;
    g.scale_to = (float*)(g.to + (size_t)a.rows * g.pieces * 16u);
    g.a_stride = a.a_stride;
    g.scale_stride = a.a_scale_stride;
    g.err = ctx->err_dev;
    const uint64_t want = ((uint64_t)a.rows * (g.pieces + (g.k_blocks + 3u) / 4u) + 255u) / 256u;
    if (launched(launch_pdl(gather_rows_kernel, (uint32_t)(want < kSms * 16u ? want : kSms * 16u), 256, 0, s, g)) != cudaSuccess)
      return PSB_ERR_CUDA;      // (there are no rows for the product to read)
    a.a = g.to;
    a.a_scale = g.scale_to;
    a.a_stride = (uint64_t)g.pieces * 16u;
    a.a_scale_stride = g.k_blocks;
    a.m = a.rows;
    a.order = nullptr;
  }
  // Few rows (on average, where they are dealt out to experts) stream the filter; us, streamed with 16 / 32 / 64 rows a tile against
  // tiles of 128 x 128: 4096 x 4096 with 17 rows 10.6 / 10.5 / 11.3 / 17.4, 64 rows 13.7 / 11.4 / 11.1 / 17.7, 128 rows 22.9 / 16.9 /
  // 15.6 / 16.6, 192 rows - / 26.5 / 18.1 / 15.8; 64 experts of 2048 x 2048 with 4 rows each 44.1 / 46.5 / 52.4 / 64.7, with 16 rows
  // 66.4 / 58.1 / 60.5 / 70.6, with 32 rows - / 77 / 72 / 65.
  const uint32_t each = a.experts ? (a.rows + a.experts - 1u) / a.experts : a.m;
  if (each <= (a.experts ? 8u : 16u)) return launch_stream<16>(ctx, a, s);
  if (each <= (a.experts ? 24u : 32u)) return launch_stream<32>(ctx, a, s);
  if (!a.experts && each <= 128u) return launch_stream<64>(ctx, a, s);
  // More rows too, where tiles leave most SMs idle and the reduction axis is long enough to be cut; us, streamed with 64 rows against tiles of
  // 128 x 128: 214 x 1885 x 5071 15.1 and 21.9, 145 x 554 x 2774 8.6 and 12.6, 1024 x 512 x 8192 18.1 and 23.9, 256 x 1000 x 2048 8.9 and 9.7,
  // 512 x 1000 x 2048 10.8 and 9.9.
  const uint64_t streamed = (uint64_t)((each + 63u) / 64u) * ((a.n + 127u) / 128u), blocks = (a.k + kBlockK - 1u) / kBlockK;
  if (!a.experts && ((streamed * 2u <= (uint64_t)ctx->sm_count && blocks >= 24u) || (streamed * 4u <= (uint64_t)ctx->sm_count && blocks >= 8u)))
    return launch_stream<64>(ctx, a, s);
  // Tiles of 256 x 256 by pairs of SMs read half of the bytes per product that single SMs' 128 x 128 do, and take 1.65 times as long a
  // block for twice an SM's work; what counts is the number of rounds of tiles (in halves: a run of an expert ends in the middle of a
  // tile).  us in a stream of calls of a second, pairs against singles: 8192^3 597 and 741, 4096^3 86 and 96, 1500 x 1000 x 2048 16.2 and 10.6,
  // 3000 x 2500 x 1000 24.0 and 25.8, 512 x 4096 x 4096 21.7 and 14.6; 16384 rows over 8 experts of 4096 x 4096 386 and 433, over 64 of
  // 2048 x 2048 190 and 177, 1884 over 18 of 2048 x 3344 70 and 57.
  const uint64_t sms = (uint64_t)ctx->sm_count, of = a.experts ? a.experts : 1u;
  auto rounds = [&](uint32_t tile, uint64_t at_once) {
    const uint64_t part = 2u * (uint64_t)each / tile + 1u, halves = !a.experts ? 2u * ((each + tile - 1u) / tile) : part < 2u ? 2u : part;
    return (of * halves * ((a.n + tile - 1u) / tile) + 2u * at_once - 1u) / (2u * at_once);
  };
  if (rounds(256, sms / 2u) * 33u < rounds(128, sms) * 20u) return launch_tiles<2, 256>(ctx, a, s);
  return launch_tiles<1, 128>(ctx, a, s);
}

}  // namespace psb
