// Matrix product of 8-bit floating-point codes with an fp32 scale for each block of 128 along the reduction axis.
//
//   y[m][n] = sum_b sa[m][b] sb[n / 128][b] S_b[m][n],   S_b[m][n] = sum_{k in block b} a[m][k] b[n][k]
//
// The scales are arbitrary fp32 numbers, so the tensor cores can add up one block of 128 only; S_b goes from tensor
// memory to registers, where the running sum is kept in fp32: one fma per output and block.  That is 1/128 of the MMA's
// multiply-adds, on pipes that do 1/64 of its rate, so the epilogue warps keep up as long as they do little else.
#include "psb_mma.cuh"

#include <cuda_bf16.h>
#include <cuda_fp16.h>

namespace psb {

namespace {

constexpr uint32_t kBlockK = 128;              // bytes of a row in a stage: one block of scales
constexpr uint32_t kRowsCta = 128;             // rows of a an SM works on
constexpr uint32_t kGemmThreads = 32 * 12;     // copies, MMA, two spare, eight epilogue warps
constexpr uint32_t kFirstSumWarp = 4;
constexpr uint32_t kSumWarps = 8;
constexpr uint32_t kStageOutBytes = 2048;      // per epilogue warp: 32 rows x 64 bytes of output
constexpr uint32_t kBandTiles = 8;             // row tiles that are walked together, so that filter tiles are met again in L2
constexpr uint32_t kMaxRing = 8;

struct GemmMaps {
  CUtensorMap a, b;
};

struct GemmParams {
  Fp8GemmArgs g;
  uint32_t k_blocks, n_tiles, stages, idesc;
  uint32_t wide_out;         // output rows start at multiples of 16 bytes
  uint32_t* err;
  unsigned long long wait_limit;
};

struct GemmCtl {
  unsigned long long full[kMaxRing], empty[kMaxRing];
  unsigned long long acc_full[4], acc_empty[4];
  uint32_t tmem_base;
  uint32_t tiles;            // in all
  WaitCtl wait;
};

// A tile: output rows [row, row_end) of one filter, columns from n0 on.
struct GemmTile {
  uint32_t expert, row, row_end, n0;
};

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
// Four rows by their numbers (the map's box is one row high).
template <int PAIR>
__device__ __forceinline__ void load_rows4(uint32_t dst, const CUtensorMap* map, uint32_t bar, int x, const int (&r)[4]) {
  if (PAIR == 2)
    asm volatile("cp.async.bulk.tensor.2d.cta_group::2.shared::cluster.global.tile::gather4.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4, %5, %6, %7}], [%2];"
                 ::"r"(dst), "l"(map), "r"(bar), "r"(x), "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]) : "memory");
  else
    asm volatile("cp.async.bulk.tensor.2d.shared::cluster.global.tile::gather4.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4, %5, %6, %7}], [%2];"
                 ::"r"(dst), "l"(map), "r"(bar), "r"(x), "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]) : "memory");
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

__device__ __forceinline__ void tc_ld32(uint32_t taddr, uint32_t (&v)[32]) {
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x32.b32 "
      "{%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, "
      "%16, %17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31}, [%32];"
      : "=r"(v[0]), "=r"(v[1]), "=r"(v[2]), "=r"(v[3]), "=r"(v[4]), "=r"(v[5]), "=r"(v[6]), "=r"(v[7]), "=r"(v[8]), "=r"(v[9]),
        "=r"(v[10]), "=r"(v[11]), "=r"(v[12]), "=r"(v[13]), "=r"(v[14]), "=r"(v[15]), "=r"(v[16]), "=r"(v[17]), "=r"(v[18]),
        "=r"(v[19]), "=r"(v[20]), "=r"(v[21]), "=r"(v[22]), "=r"(v[23]), "=r"(v[24]), "=r"(v[25]), "=r"(v[26]), "=r"(v[27]),
        "=r"(v[28]), "=r"(v[29]), "=r"(v[30]), "=r"(v[31])
      : "r"(taddr)
      : "memory");
}

// Two fp32 numbers in a register pair: a third of the instructions of two fma each.
__device__ __forceinline__ unsigned long long pair_of(uint32_t lo, uint32_t hi) {
  unsigned long long r;
  asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "r"(lo), "r"(hi));
  return r;
}
__device__ __forceinline__ void fma_pair(unsigned long long& acc, unsigned long long v, unsigned long long s) {
  asm("fma.rn.f32x2 %0, %1, %2, %0;" : "+l"(acc) : "l"(v), "l"(s));
}
__device__ __forceinline__ float low_of(unsigned long long p) { return __uint_as_float((uint32_t)p); }
__device__ __forceinline__ float high_of(unsigned long long p) { return __uint_as_float((uint32_t)(p >> 32)); }

template <typename T> __device__ __forceinline__ T round_to(float v);
template <> __device__ __forceinline__ float round_to<float>(float v) { return v; }
template <> __device__ __forceinline__ __nv_bfloat16 round_to<__nv_bfloat16>(float v) { return __float2bfloat16_rn(v); }
template <> __device__ __forceinline__ __half round_to<__half>(float v) { return __float2half_rn(v); }

__device__ __forceinline__ float finish(float y, const float* bias, uint32_t relu) {
  if (bias) y += __ldcg(bias);
  return relu && y < 0.0f ? 0.0f : y;
}

// A warp's 32 rows (a row a lane) of NC columns leave through shared memory, 64 bytes of a row at a time: four lanes then
// store what is contiguous.  `rows`: rows of these 32 that exist; `cols`: columns that exist from the first one on.
template <typename T, int NC>
__device__ __forceinline__ void store_rows(const GemmParams& p, const unsigned long long (&acc)[NC / 2], uint8_t* stage, uint64_t row0,
                                           uint32_t rows, uint32_t col0, uint32_t cols, const float* bias, uint32_t lane) {
  constexpr uint32_t kCols = 64 / sizeof(T), kPer = 16 / sizeof(T);
  T* out = (T*)p.g.out;
#pragma unroll
  for (uint32_t c0 = 0; c0 < (uint32_t)NC; c0 += kCols) {
    if (c0 < cols) {               // (the same for the whole warp)
      alignas(16) T v[kCols];
#pragma unroll
      for (uint32_t c = 0; c < kCols; ++c) {
        const unsigned long long pr = acc[(c0 + c) / 2];
        v[c] = round_to<T>(finish((c & 1u) ? high_of(pr) : low_of(pr), bias && c0 + c < cols ? bias + c0 + c : nullptr, p.g.relu));
      }
#pragma unroll
      for (uint32_t q = 0; q < 4u; ++q)
        *reinterpret_cast<uint4*>(stage + lane * 64u + ((q ^ ((lane >> 1) & 3u)) << 4)) = reinterpret_cast<const uint4*>(v)[q];
      __syncwarp();
#pragma unroll
      for (uint32_t i = 0; i < 4u; ++i) {
        const uint32_t r = i * 8u + (lane >> 2), q = lane & 3u, c = c0 + q * kPer;
        const uint4 w = *reinterpret_cast<const uint4*>(stage + r * 64u + ((q ^ ((r >> 1) & 3u)) << 4));
        if (r < rows) {
          T* to = out + (row0 + r) * p.g.out_stride + col0 + c;
          if (p.wide_out && c + kPer <= cols) {
            *reinterpret_cast<uint4*>(to) = w;
          } else {
            const T* parts = reinterpret_cast<const T*>(&w);
            for (uint32_t e = 0; e < kPer; ++e)
              if (c + e < cols) to[e] = parts[e];
          }
        }
      }
      __syncwarp();
    }
  }
}

template <int PAIR, int BN>
constexpr uint32_t kGemmStageBytes = (kRowsCta + (uint32_t)BN / PAIR) * kBlockK;

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
  GemmCtl* ctl = reinterpret_cast<GemmCtl*>(out_stage + kSumWarps * kStageOutBytes);
  uint32_t* offsets = reinterpret_cast<uint32_t*>(ctl + 1);
  uint32_t* first = offsets + p.g.experts + 1u;
  const uint32_t warp = threadIdx.x >> 5, lane = threadIdx.x & 31u;
  const uint32_t rank = PAIR == 2 ? cluster_rank() : 0u;

  if (threadIdx.x == 0) {
    for (uint32_t s = 0; s < p.stages; ++s) {
      mbar_init(smem_u32(&ctl->full[s]), 1);
      mbar_init(smem_u32(&ctl->empty[s]), 1);
    }
    for (uint32_t b = 0; b < kBufs; ++b) {
      mbar_init(smem_u32(&ctl->acc_full[b]), 1);
      mbar_init(smem_u32(&ctl->acc_empty[b]), kSumWarps * PAIR);
    }
    ctl->wait.abort = 0;
    ctl->wait.limit = p.wait_limit;
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
    // offsets, cut to what out has; a run that is none counts as empty
    for (uint32_t e = threadIdx.x; e <= p.g.experts; e += kGemmThreads) {
      const int o = __ldcg(p.g.offsets + e);
      if (o < 0 || (uint32_t)o > p.g.rows) atomicOr(p.err, kDevErrRange);
      offsets[e] = o < 0 ? 0u : min((uint32_t)o, p.g.rows);
    }
    __syncthreads();
    if (warp == 0) {
      uint32_t carry = 0;
      for (uint32_t e0 = 0; e0 < p.g.experts; e0 += 32u) {
        const uint32_t e = e0 + lane;
        uint32_t mine = 0;
        if (e < p.g.experts) {
          if (offsets[e + 1u] < offsets[e]) atomicOr(p.err, kDevErrRange);
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
      if (lane == 0) first[p.g.experts] = ctl->tiles = carry;
    }
  } else if (threadIdx.x == 0) {
    ctl->tiles = (p.g.m + TM - 1u) / TM * p.n_tiles;
  }
  tc_fence_before();
  if (PAIR == 2) cluster_sync();
  else __syncthreads();
  tc_fence_after();
  const uint32_t tmem_base = ctl->tmem_base, tiles = ctl->tiles;
  const uint32_t step = gridDim.x / PAIR, t0 = blockIdx.x / PAIR;
  WaitCtl* wc = &ctl->wait;
  bool failed = false;

  if (warp < kFirstSumWarp) {
    if (BN == 256) asm volatile("setmaxnreg.dec.sync.aligned.u32 72;");
    if (warp == 0) {
      // ------------------------------------------------------------ copies
      uint32_t s = 0, ph = 0;
      for (uint32_t t = t0; t < tiles && !failed; t += step) {
        const GemmTile tile = tile_at<TM, BN>(p, t, first, offsets);
        const uint32_t row = tile.row + rank * kRowsCta;
        int rows4[4];
        if (p.g.order) {
#pragma unroll
          for (uint32_t i = 0; i < 4u; ++i) {
            // rows behind the run's end repeat its first one
            const uint32_t r = row + 4u * lane + i;
            const int o = __ldcg(p.g.order + (r < tile.row_end ? r : tile.row));
            if (o < 0 || (uint32_t)o >= p.g.m) atomicOr(p.err, kDevErrRange);
            rows4[i] = o < 0 ? 0 : (int)min((uint32_t)o, p.g.m - 1u);
          }
        }
        for (uint32_t kb = 0; kb < p.k_blocks; ++kb) {
          const uint32_t bar = PAIR == 2 ? in_cta(smem_u32(&ctl->full[s]), 0u) : smem_u32(&ctl->full[s]);
          const uint32_t dst = smem_u32(smem) + s * kStage;
          bool ok = true;
          if (lane == 0) ok = mbar_wait(smem_u32(&ctl->empty[s]), ph ^ 1u, wc);
          if (__any_sync(0xFFFFFFFFu, !ok)) { failed = true; break; }
          if (lane == 0) {
            if (rank == 0u) mbar_expect_tx(smem_u32(&ctl->full[s]), kStage * PAIR);
            if (!p.g.order) load_a<PAIR>(dst, &maps.a, bar, (int)(kb * kBlockK), (int)row);
            load_b<PAIR>(dst + kRowsCta * kBlockK, &maps.b, bar, (int)(kb * kBlockK), (int)(tile.n0 + rank * (BN / PAIR)), (int)tile.expert);
          }
          if (p.g.order) {
            __syncwarp();
            load_rows4<PAIR>(dst + lane * 4u * kBlockK, &maps.a, bar, (int)(kb * kBlockK), rows4);
          }
          if (++s == p.stages) { s = 0; ph ^= 1u; }
        }
      }
    } else if (warp == 1 && rank == 0u) {
      // ------------------------------------------------------------ MMA
      uint32_t s = 0, ph = 0, buf = 0, bph = 0;
      const uint32_t desc_hi = smem_desc_hi(kBlockK);
      for (uint32_t t = t0; t < tiles && !failed; t += step) {
        for (uint32_t kb = 0; kb < p.k_blocks; ++kb) {
          if (!mbar_wait(smem_u32(&ctl->acc_empty[buf]), bph ^ 1u, wc, kNoSleep) || !mbar_wait(smem_u32(&ctl->full[s]), ph, wc, kNoSleep)) {
            failed = true;
            break;
          }
          tc_fence_after();
          const uint32_t a_lo = smem_desc_lo(smem_u32(smem) + s * kStage), b_lo = a_lo + (kRowsCta * kBlockK >> 4);
          if (elect_one()) {
#pragma unroll
            for (uint32_t ks = 0; ks < kBlockK / 32u; ++ks)
              mma_f8<PAIR>(tmem_base + buf * BN, a_lo + ks * 2u, b_lo + ks * 2u, desc_hi, p.idesc, ks);
            commit<PAIR>(smem_u32(&ctl->empty[s]));
            commit<PAIR>(smem_u32(&ctl->acc_full[buf]));
          }
          __syncwarp();
          if (++s == p.stages) { s = 0; ph ^= 1u; }
          if (++buf == kBufs) { buf = 0; bph ^= 1u; }
        }
      }
    }
  } else {
    // -------------------------------------------------------------- scaled sums and output
    if (BN == 256) asm volatile("setmaxnreg.inc.sync.aligned.u32 216;");
    constexpr int NC = BN / 2;                 // columns of a warp
    const uint32_t quarter = warp & 3u, half = (warp - kFirstSumWarp) >> 2;
    uint8_t* stage = out_stage + (warp - kFirstSumWarp) * kStageOutBytes;
    uint32_t buf = 0, bph = 0;
    for (uint32_t t = t0; t < tiles && !failed; t += step) {
      const GemmTile tile = tile_at<TM, BN>(p, t, first, offsets);
      const uint32_t row0 = tile.row + rank * kRowsCta + quarter * 32u, col0 = tile.n0 + half * NC;
      const uint32_t rows = row0 < tile.row_end ? min(32u, tile.row_end - row0) : 0u;
      const uint32_t cols = col0 < p.g.n ? min((uint32_t)NC, p.g.n - col0) : 0u;
      uint32_t from = row0 + min(lane, rows ? rows - 1u : 0u);
      if (!rows) from = tile.row;
      if (p.g.order) {
        const int o = __ldcg(p.g.order + from);
        from = o < 0 ? 0u : min((uint32_t)o, p.g.m - 1u);
      } else {
        from = min(from, p.g.m - 1u);
      }
      const float* sa = p.g.a_scale + (uint64_t)from * p.g.a_scale_stride;
      const float* sb = p.g.b_scale + tile.expert * p.g.b_scale_expert_stride + (uint64_t)(min(col0, p.g.n - 1u) / 128u) * p.g.b_scale_stride;
      unsigned long long acc[NC / 2];
#pragma unroll
      for (int i = 0; i < NC / 2; ++i) acc[i] = 0ull;
      // scales two blocks ahead
      float sc = __ldca(sa) * __ldca(sb);
      const uint32_t last = p.k_blocks - 1u;
      float sc1 = __ldca(sa + min(1u, last)) * __ldca(sb + min(1u, last));
      for (uint32_t kb = 0; kb < p.k_blocks; ++kb) {
        const float na = __ldca(sa + min(kb + 2u, last)), nb = __ldca(sb + min(kb + 2u, last));
        if (!mbar_wait(smem_u32(&ctl->acc_full[buf]), bph, wc, kNoSleep)) { failed = true; break; }
        tc_fence_after();
        const uint32_t taddr = tmem_base + buf * BN + half * NC + ((quarter * 32u) << 16);
        const unsigned long long s2 = pair_of(__float_as_uint(sc), __float_as_uint(sc));
        uint32_t v[2][32];
        tc_ld32(taddr, v[0]);
#pragma unroll
        for (int c = 0; c < NC / 32; ++c) {
          tc_wait_ld();
          if (c + 1 < NC / 32) {
            tc_ld32(taddr + (c + 1) * 32, v[(c + 1) & 1]);
          } else {
            tc_fence_before();
            __syncwarp();
            if (lane == 0) {
              if (PAIR == 2)
                asm volatile("mbarrier.arrive.shared::cluster.b64 _, [%0];" ::"r"(in_cta(smem_u32(&ctl->acc_empty[buf]), 0u)) : "memory");
              else
                mbar_arrive(smem_u32(&ctl->acc_empty[buf]));
            }
          }
#pragma unroll
          for (int i = 0; i < 16; ++i) fma_pair(acc[c * 16 + i], pair_of(v[c & 1][2 * i], v[c & 1][2 * i + 1]), s2);
        }
        sc = sc1;
        sc1 = na * nb;
        if (++buf == kBufs) { buf = 0; bph ^= 1u; }
      }
      if (failed) break;
      const float* bias = p.g.bias ? p.g.bias + (uint64_t)tile.expert * p.g.n + col0 : nullptr;
      if (p.g.out_dtype == PSB_DT_F32) store_rows<float, NC>(p, acc, stage, row0, rows, col0, cols, bias, lane);
      else if (p.g.out_dtype == PSB_DT_BF16) store_rows<__nv_bfloat16, NC>(p, acc, stage, row0, rows, col0, cols, bias, lane);
      else store_rows<__half, NC>(p, acc, stage, row0, rows, col0, cols, bias, lane);
    }
  }

  // ---------------------------------------------------------------- common exit
  if (failed) {
    if (lane == 0) {
      wc->abort = 1u;
      atomicOr(p.err, kDevErrTimeout);
    }
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

template <int PAIR, int BN>
psb_status launch_tiles(psb_ctx* ctx, const Fp8GemmArgs& a, cudaStream_t s) {
  GemmMaps maps;
  GemmParams p;
  p.g = a;
  p.k_blocks = (a.k + kBlockK - 1u) / kBlockK;
  p.n_tiles = (a.n + BN - 1u) / BN;
  p.err = ctx->err_dev;
  p.wait_limit = ctx->wait_limit_cycles;
  const uint64_t size = a.out_dtype == PSB_DT_F32 ? 4u : 2u;
  p.wide_out = (((uintptr_t)a.out | a.out_stride * size) & 15u) == 0u;
  // fp32 accumulators; formats of a and b; columns / 8; rows / 16
  p.idesc = (1u << 4) | ((a.a_dtype == PSB_DT_E5M2 ? 1u : 0u) << 7) | ((a.b_dtype == PSB_DT_E5M2 ? 1u : 0u) << 10) |
            (((uint32_t)BN >> 3) << 17) | ((kRowsCta * PAIR >> 4) << 24);
  const uint32_t ctl_bytes = kSumWarps * kStageOutBytes + sizeof(GemmCtl) + (a.experts ? (a.experts + 1u) * 8u : 0u) + 1024u;
  p.stages = (uint32_t)((kSmemBudget - ctl_bytes) / kGemmStageBytes<PAIR, BN>);
  if (p.stages > kMaxRing) p.stages = kMaxRing;
  if (!encode_codes(ctx->encode_tiled, &maps.a, a.a, 2, a.k, a.m, 1, a.a_stride, 0, a.order ? 1u : kRowsCta) ||
      !encode_codes(ctx->encode_tiled, &maps.b, a.b, 3, a.k, a.n, a.experts ? a.experts : 1u, a.b_stride,
                    a.experts ? a.b_expert_stride : a.b_stride * a.n, BN / PAIR))
    return PSB_ERR_CUDA;
  const size_t smem = p.stages * kGemmStageBytes<PAIR, BN> + ctl_bytes;
  auto kernel = gemm_fp8_kernel<PAIR, BN>;
  if (cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)kSmemBudget) != cudaSuccess) return PSB_ERR_CUDA;
  const uint32_t TM = kRowsCta * PAIR;
  // at most: every expert has one tile that is not full
  const uint64_t m_tiles = a.experts ? (uint64_t)a.rows / TM + (a.experts < a.rows ? a.experts : a.rows) : (a.m + TM - 1u) / TM;
  const uint64_t tiles = m_tiles * p.n_tiles;
  const uint32_t most = (uint32_t)ctx->sm_count / PAIR;
  cudaLaunchAttribute attr[2];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  attr[1].id = cudaLaunchAttributeClusterDimension;
  attr[1].val.clusterDim.x = PAIR;
  attr[1].val.clusterDim.y = attr[1].val.clusterDim.z = 1;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((uint32_t)(tiles < most ? tiles : most) * PAIR);
  cfg.blockDim = dim3(kGemmThreads);
  cfg.dynamicSmemBytes = smem;
  cfg.stream = s;
  cfg.attrs = attr;
  cfg.numAttrs = PAIR == 2 ? 2 : 1;
  const cudaError_t e = cudaLaunchKernelEx(&cfg, kernel, maps, p);
  note_launch();
  if (e != cudaSuccess || cudaGetLastError() != cudaSuccess) return PSB_ERR_CUDA;
  return PSB_OK;
}

}  // namespace

psb_status launch_gemm_fp8(psb_ctx* ctx, const Fp8GemmArgs& a, cudaStream_t s) {
  if (!ctx->encode_tiled) return PSB_ERR_UNSUPPORTED;
  return launch_tiles<1, 128>(ctx, a, s);
}

}  // namespace psb
