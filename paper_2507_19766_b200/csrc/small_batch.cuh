// Logits of a small batch: a[t, v] = hidden[t] . W[v] for at most 64 tokens, bf16 operands, float32 out.
//
// A decoding step reads the whole of W for a handful of tokens and is bound by that stream (151936 x 2048: 622 MB, 96 us
// at 6458 GB/s).  The sweep kernels put tokens on the 256 rows of the MMA: with one token they execute 256 rows of
// work, as long as the stream itself, and load a hidden tile of zeros beside every tile of W.  Here the roles are
// swapped: 128 vocabulary rows are the MMA's M side and the tokens its N (16, 32 or 64), so that contractions are an
// eighth or less of the stream and nearly every byte that arrives is W.  Every SM takes the same number of
// vocabulary rows (a multiple of 16; its last tile is loaded with a shorter box), which the 256-row tiles of the sweep
// cannot give: 594 tiles on 74 CTA pairs are 9 rounds for 8.03 tiles.
// Measured for one token: 104 us, 6.0 TB/s of W (93 % of the copy rate); the whole call 119 us, through the sweep 237.
// The logits go to global memory -- 4 bytes a vocabulary entry and token beside the 2 H bytes of its row of W -- and
// the row kernel does the rest.
#pragma once

#include "common.cuh"
#include "ptx_sm100.cuh"
#include "umma_gemm.cuh"

namespace ulorl {

constexpr int kSmallMaxTokens = 64;
constexpr int kSmallThreads = 192;

struct SmallArgs {
  int T, V, K;
  int rows_per_cta;         // multiple of 16
  float* logits;            // [T][ld]
  size_t ld;
  int* status;
};

template <int kN>
struct SmallConfig {
  static constexpr uint32_t b_bytes = kN * kBK * 2;
  static constexpr uint32_t stage_bytes = kABytes + b_bytes;
  static constexpr int stages = (int)(204800u / stage_bytes) > 12 ? 12 : (int)(204800u / stage_bytes);
  static constexpr size_t smem_bytes = (size_t)stages * stage_bytes + 1024;
  static constexpr int tmem_cols = 2 * kN < 32 ? 32 : 2 * kN;      // two accumulators
};

// map_w: boxes of 128 rows, map_last: boxes of the last tile's rows, map_h: boxes of kN tokens; 64 columns each.
template <int kN>
__global__ void __launch_bounds__(kSmallThreads, 1)
small_logits_kernel(const __grid_constant__ CUtensorMap map_w, const __grid_constant__ CUtensorMap map_last,
                    const __grid_constant__ CUtensorMap map_h, const SmallArgs args) {
  using namespace ptx;
  using Cfg = SmallConfig<kN>;
  constexpr int kStages = Cfg::stages;
  extern __shared__ uint8_t smem_raw[];
  __shared__ __align__(8) uint64_t bar_full[kStages];
  __shared__ __align__(8) uint64_t bar_empty[kStages];
  __shared__ __align__(8) uint64_t bar_tmem_full[2];
  __shared__ __align__(8) uint64_t bar_tmem_empty[2];
  __shared__ uint32_t tmem_base_slot;
  __shared__ int abort_flag;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const uint32_t smem_base = (smem_u32(smem_raw) + 1023u) & ~1023u;
  volatile int* abort_p = &abort_flag;
  const int row_begin = blockIdx.x * args.rows_per_cta;
  const int row_end = min(args.V, row_begin + args.rows_per_cta);
  const int n_tiles = row_begin < row_end ? (args.rows_per_cta + kBM - 1) / kBM : 0;
  const int last_rows = args.rows_per_cta - (n_tiles - 1) * kBM;
  const int k_blocks = (args.K + kBK - 1) / kBK;

  if (threadIdx.x == 0) {
    abort_flag = 0;
    for (int s = 0; s < kStages; ++s) {
      mbar_init(smem_u32(&bar_full[s]), 1);
      mbar_init(smem_u32(&bar_empty[s]), 1);
    }
    for (int b = 0; b < 2; ++b) {
      mbar_init(smem_u32(&bar_tmem_full[b]), 1);
      mbar_init(smem_u32(&bar_tmem_empty[b]), 4);
    }
    mbar_fence_init();
    fence_async_proxy();
  }
  if (warp == 1) {
    tmem_alloc(smem_u32(&tmem_base_slot), Cfg::tmem_cols);
    tmem_relinquish();
  }
  tc_fence_before_sync();
  __syncthreads();
  tc_fence_after_sync();
  const uint32_t tmem_base = tmem_base_slot;

  if (warp == 0) {
    if (lane == 0) {
      uint32_t stage = 0, phase = 0, issued = 0;
      for (int tile = 0; tile < n_tiles; ++tile) {
        const bool last = tile == n_tiles - 1;
        const int row = row_begin + tile * kBM;
        for (int kb = 0; kb < k_blocks; ++kb) {
          if (!mbar_wait_bounded(smem_u32(&bar_empty[stage]), phase ^ 1u, abort_p, kWaitLimitCycles)) goto producer_drain;
          const uint32_t full = smem_u32(&bar_full[stage]);
          mbar_arrive_expect_tx(full, (last ? (uint32_t)last_rows * kBK * 2 : kABytes) + Cfg::b_bytes);
          const uint32_t sa = smem_base + stage * Cfg::stage_bytes;
          tma_load_2d(sa, last ? &map_last : &map_w, full, kb * kBK, row);
          tma_load_2d(sa + kABytes, &map_h, full, kb * kBK, 0);
          ++issued;
          if (++stage == kStages) { stage = 0; phase ^= 1u; }
        }
      }
      // every slot that was filled has been read: no copy and no release is in flight when the block ends
      {
        const uint32_t n_tail = issued < (uint32_t)kStages ? issued : (uint32_t)kStages;
        if (issued < (uint32_t)kStages) { stage = 0; phase = 1u; }
        for (uint32_t b = 0; b < n_tail; ++b) {
          if (!mbar_wait_bounded(smem_u32(&bar_empty[stage]), phase ^ 1u, abort_p, kWaitLimitCycles)) goto producer_drain;
          if (++stage == kStages) { stage = 0; phase ^= 1u; }
        }
      }
    producer_drain:
      if (*abort_p) {
        // give the copies still in flight a bounded time to land before the block goes away
        const long long t0 = clock64();
        while (clock64() - t0 < 20000000LL) {
        }
      }
    }
    __syncwarp();
  } else if (warp == 1) {
    if (lane == 0) {
      constexpr uint32_t idesc = make_idesc_bf16(kBM, kN, 0, 0);
      constexpr uint64_t k_step = (kUmmaK * 2) >> 4;
      uint32_t stage = 0, phase = 0;
      for (int tile = 0; tile < n_tiles; ++tile) {
        const uint32_t buf = tile & 1u, buf_phase = (tile >> 1) & 1u;
        if (!mbar_wait_bounded(smem_u32(&bar_tmem_empty[buf]), buf_phase ^ 1u, abort_p, kWaitLimitCycles)) goto mma_done;
        for (int kb = 0; kb < k_blocks; ++kb) {
          if (!mbar_wait_bounded(smem_u32(&bar_full[stage]), phase, abort_p, kWaitLimitCycles)) goto mma_done;
          tc_fence_after_sync();
          const uint32_t sa = smem_base + stage * Cfg::stage_bytes;
          const uint64_t da = make_smem_desc(sa, 16, 1024), db = make_smem_desc(sa + kABytes, 16, 1024);
#pragma unroll
          for (int k = 0; k < kBK / kUmmaK; ++k)
            umma_bf16(tmem_base + buf * kN, da + k * k_step, db + k * k_step, idesc, (kb > 0 || k > 0) ? 1u : 0u);
          umma_commit(smem_u32(&bar_empty[stage]));
          if (kb == k_blocks - 1) umma_commit(smem_u32(&bar_tmem_full[buf]));
          if (++stage == kStages) { stage = 0; phase ^= 1u; }
        }
      }
    mma_done:;
    }
    __syncwarp();
  } else {
    const int quarter = warp & 3;
    for (int tile = 0; tile < n_tiles; ++tile) {
      const uint32_t buf = tile & 1u, buf_phase = (tile >> 1) & 1u;
      const bool ok = mbar_wait_bounded<true>(smem_u32(&bar_tmem_full[buf]), buf_phase, abort_p, kWaitLimitCycles);
      if (!__all_sync(0xffffffffu, ok)) break;
      tc_fence_after_sync();
      const int in_tile = quarter * 32 + lane, v = row_begin + tile * kBM + in_tile;
      const bool v_ok = v < row_end && (tile < n_tiles - 1 || in_tile < last_rows);
      const uint32_t taddr = tmem_base + buf * kN + ((uint32_t)(quarter * 32) << 16);
#pragma unroll
      for (int c = 0; c < kN; c += 16) {
        if (c >= args.T) break;                         // the same in all lanes
        uint32_t r[16];
        tmem_ld_32x16(taddr + c, r);
        tmem_ld_wait();
#pragma unroll
        for (int j = 0; j < 16; ++j)
          if (v_ok && c + j < args.T) args.logits[(size_t)(c + j) * args.ld + v] = __uint_as_float(r[j]);
        __syncwarp();
      }
      tc_fence_before_sync();
      __syncwarp();
      if (lane == 0) mbar_arrive(smem_u32(&bar_tmem_empty[buf]));
    }
  }
  if (*abort_p && lane == 0) atomicOr(args.status, kStatusTimeout);
  tc_fence_before_sync();
  __syncthreads();
  if (warp == 1) {
    tc_fence_after_sync();
    tmem_dealloc(tmem_base, Cfg::tmem_cols);
  }
}

}  // namespace ulorl
