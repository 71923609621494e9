// Kernels of token scoring and of distillation from a teacher's top logits, around the contractions:
// logits_rows_kernel   softmax statistics, log-prob, entropy and the k largest entries of rows of logits
// merge_scores_kernel  the same from the partials of the LM-head sweep
// distill_*_kernel     teacher lists: sorting, the loss of a row, its gradient on the list, the batch loss
// row_params_kernel    what the dz pass of a row needs
//
// A row's softmax is kept as (m, r): m the maximum of the raw logits a, r the sum of e^(kappa (a - m)) over all
// entries but one that equals m, so that 1 - p and the entropy keep their relative precision in sharply peaked rows;
// ln s = log1p(r), lse = kappa m + ln s.  Ids are chosen by (value falling, id rising).
#pragma once

#include <cooperative_groups.h>
#include <cuda_fp16.h>
#include <limits.h>

#include "common.cuh"
#include "simt.cuh"
#include "umma_gemm.cuh"

namespace ulorl {

constexpr int kMaxTop = 32;            // alternatives a scoring call returns
constexpr int kMaxList = 128;          // entries of a teacher's list
constexpr int kMaxRowLists = 160;      // partial results of a row that the merge takes
constexpr float kLog2e = 1.4426950408889634f;
constexpr float kLn2 = 0.6931471805599453f;

__device__ __forceinline__ float fast_ex2(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
// max that keeps a NaN
__device__ __forceinline__ float max_nan(float a, float b) {
  float y;
  asm("max.NaN.f32 %0, %1, %2;" : "=f"(y) : "f"(a), "f"(b));
  return y;
}

// Unsigned keys in the order of the values: -inf < ... < -0 = +0 < ... < +inf, NaN below them all (0).
__device__ __forceinline__ uint32_t order_key(float x) {
  if (x != x) return 0u;
  const uint32_t b = __float_as_uint(x + 0.f);
  return (b & 0x80000000u) ? ~b : (b | 0x80000000u);
}
__device__ __forceinline__ float key_value(uint32_t k) {
  if (k == 0u) return __uint_as_float(0x7FC00000u);
  return __uint_as_float((k & 0x80000000u) ? (k & 0x7FFFFFFFu) : ~k);
}
constexpr uint32_t kKeyNegInf = 0x007FFFFFu;

__device__ __forceinline__ unsigned long long pack_entry(uint32_t key, int id) {
  return ((unsigned long long)key << 32) | (uint32_t)~id;          // larger = better: value, then the lower id
}

// What the row kernel needs of a type: 16-byte vectors of per_vec entries, the bits of an order key that its values
// use, the largest entry of a vector (NaN aside), and its entries as float32 pairs, nothing below kFloor (see fold).
constexpr float kFloor = -1e30f;
template <typename T> struct RowType;
template <> struct RowType<float> {
  static constexpr int per_vec = 4, key_bits = 32;
  static constexpr uint32_t neg_inf = 0xFF800000u;
  static __device__ __forceinline__ float top(const uint4& v) {
    return fmaxf(fmaxf(__uint_as_float(v.x), __uint_as_float(v.y)), fmaxf(__uint_as_float(v.z), __uint_as_float(v.w)));
  }
  static __device__ __forceinline__ void entries(const uint4& v, float (&x)[4]) {
    x[0] = __uint_as_float(v.x); x[1] = __uint_as_float(v.y); x[2] = __uint_as_float(v.z); x[3] = __uint_as_float(v.w);
  }
  static __device__ __forceinline__ void floored(const uint4& v, float (&x)[4]) {
    entries(v, x);
#pragma unroll
    for (int j = 0; j < 4; ++j) x[j] = max_nan(x[j], kFloor);
  }
};
template <> struct RowType<__nv_bfloat16> {
  static constexpr int per_vec = 8, key_bits = 16;
  static constexpr uint32_t neg_inf = 0xFF80FF80u;
  static __device__ __forceinline__ __nv_bfloat162 pair(uint32_t w) { return *reinterpret_cast<const __nv_bfloat162*>(&w); }
  static __device__ __forceinline__ float top(const uint4& v) {
    const __nv_bfloat162 m = __hmax2(__hmax2(pair(v.x), pair(v.y)), __hmax2(pair(v.z), pair(v.w)));
    return fmaxf(__low2float(m), __high2float(m));
  }
  static __device__ __forceinline__ void entries(const uint4& v, float (&x)[8]) {
    const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      x[2 * i] = __uint_as_float(w[i] << 16);
      x[2 * i + 1] = __uint_as_float(w[i] & 0xFFFF0000u);
    }
  }
  static __device__ __forceinline__ void floored(const uint4& v, float (&x)[8]) {
    const __nv_bfloat162 low = __float2bfloat162_rn(kFloor);
    const __nv_bfloat162 q[4] = {__hmax2_nan(pair(v.x), low), __hmax2_nan(pair(v.y), low), __hmax2_nan(pair(v.z), low),
                                 __hmax2_nan(pair(v.w), low)};
    entries(*reinterpret_cast<const uint4*>(q), x);
  }
};
template <> struct RowType<__half> {
  static constexpr int per_vec = 8, key_bits = 19;                  // sign, 8 exponent and 10 mantissa bits of the float32
  static constexpr uint32_t neg_inf = 0xFC00FC00u;
  static __device__ __forceinline__ __half2 pair(uint32_t w) { return *reinterpret_cast<const __half2*>(&w); }
  static __device__ __forceinline__ float top(const uint4& v) {
    const __half2 m = __hmax2(__hmax2(pair(v.x), pair(v.y)), __hmax2(pair(v.z), pair(v.w)));
    return fmaxf(__low2float(m), __high2float(m));
  }
  static __device__ __forceinline__ void entries(const uint4& v, float (&x)[8]) {
    const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const float2 f = __half22float2(pair(w[i]));
      x[2 * i] = f.x;
      x[2 * i + 1] = f.y;
    }
  }
  static __device__ __forceinline__ void floored(const uint4& v, float (&x)[8]) {
    entries(v, x);
#pragma unroll
    for (int j = 0; j < 8; ++j) x[j] = max_nan(x[j], kFloor);
  }
};
__device__ __forceinline__ float row_value(float x) { return x; }
__device__ __forceinline__ float row_value(__nv_bfloat16 x) { return __bfloat162float(x); }
__device__ __forceinline__ float row_value(__half x) { return __half2float(x); }

struct RowsArgs {
  const void* logits;       // [T][ld], V valid columns
  size_t ld;
  int T, V, k;
  float kappa;
  const int* targets;       // may be NULL
  float *logp, *entropy, *lse;
  float2* norm;             // (m, ln s)
  int* top_ids;             // [T][k]
  float* top_logp;          // [T][k]
  float4* partials;         // (m, r, -, -) for a merge that follows
  int* status;              // timeouts and targets out of range; NULL: their results are NaN, nothing is reported
  long long wait_limit;     // kHeld only
};

constexpr int kRowThreads = 256;
constexpr int kRowUnroll = 4;          // 16-byte vectors of a thread in a batch
constexpr int kRowBatch = kRowUnroll * kRowThreads;       // vectors: 16 KB
constexpr int kRowStages = 3;          // batches on their way or waiting in shared memory
constexpr size_t kRowSmem = (size_t)kRowStages * kRowBatch * 16 + 128;
constexpr int kRowCandidates = 512;
constexpr int kRowMaxCluster = 16;

// Running statistics of a row in one lane: m is the warp's maximum, s and u are the lane's sums of 2^t and 2^t t, t =
// c2 x - ref, over its entries but one that equals m where own = 1.  ref is c2 m rounded, so that an exponent is one
// fused multiply-add, and delta what the rounding took off.  Entries of -inf are raised to kFloor, where 2^t and
// 2^t t are zero; that and the product c2 m hold for maxima between -1e29 and 1e30, and a warp whose maximum lies
// outside (a row of the type's lowest value) takes differences to it instead.
struct RowState {
  float m = -INFINITY, ref = 0.f, delta = 0.f, s = 0.f, u = 0.f, own = 0.f;
  float lane_max = NAN;                                             // no entry yet

  __device__ __forceinline__ bool plain() const { return m >= -1e29f && m <= 1e30f; }
  __device__ __forceinline__ float one() const { return residue_ex2(delta); }

  // folds in n entries: cmax is the largest of them, x their values, not below kFloor; `any`: the lane has some.  All lanes
  // of a warp together.  `exact` gives entry j as it is.
  template <int n, typename Exact>
  __device__ __forceinline__ void fold(float (&x)[n], float cmax, float c2, bool any, Exact exact) {
    if (any) lane_max = fmaxf(lane_max, cmax);
    const int ci = __float_as_int(cmax);
    const int wi = __reduce_max_sync(0xffffffffu, ci ^ ((ci >> 31) & 0x7FFFFFFF));    // ordered as integers
    const float wmax = __int_as_float(wi ^ ((wi >> 31) & 0x7FFFFFFF));
    const bool risen = wmax > m;                                    // the same in all lanes
    if (risen) {
      const float ref_new = fminf(fmaxf(c2 * wmax, -1e37f), 1e37f);
      if (m > -INFINITY) {
        const float d = fmaxf(ref - ref_new, -1000.f), sc = fast_ex2(d), mine = own * one();
        u = sc * (fmaf(d, s + mine, u) + mine * delta);
        s = (s + mine) * sc;
        own = 0.f;
      }
      m = wmax;
      ref = ref_new;
      delta = plain() ? fmaf(c2, m, -ref) : 0.f;
    }
    float ls = 0.f, lu = 0.f;
    if (plain() || m == -INFINITY) {
      if (risen) {
        // the maximum itself is left out before the sums (a peaked row's 1 - p is what the others add up to); of
        // several equal ones the others count
        float equal = 0.f;
#pragma unroll
        for (int j = 0; j < n; ++j) {
          const bool top = x[j] == m;
          equal += top ? 1.f : 0.f;
          x[j] = top ? kFloor : x[j];
        }
        if (equal > 0.f) {
          own = 1.f;
          ls = (equal - 1.f) * one();
          lu = ls * delta;
        }
      }
      constexpr int kChains = n >= 8 ? 4 : 1;
      float a[kChains] = {}, b[kChains] = {};
#pragma unroll
      for (int j = 0; j < n; ++j) {
        const float t = fmaf(x[j], c2, -ref), e = fast_ex2(t);
        a[j % kChains] += e;
        b[j % kChains] = fmaf(e, t, b[j % kChains]);
      }
#pragma unroll
      for (int q = 0; q < kChains; ++q) { ls += a[q]; lu += b[q]; }
    } else {
      float ties = 0.f;
#pragma unroll 1
      for (int j = 0; j < n; ++j) {
        const float v = exact(j);
        const float t = max_nan((v - m) * c2, -1000.f), e = fast_ex2(t);
        const bool top = risen && v == m;
        ties += top ? 1.f : 0.f;
        ls += top ? 0.f : e;
        lu = fmaf(e, t, lu);
      }
      if (ties > 0.f) { own = 1.f; ls += ties - 1.f; }
    }
    s += ls;
    u += lu;
  }
};

// What the blocks of one row tell each other: maximum, sums relative to it (the maximum's own 1 not in r if owners > 0),
// and the slice's largest entries in falling order, 0 behind the last.
struct RowSlice {
  float m, r, u;
  int owners;
  unsigned long long top[kMaxTop];
};

// The statistics that the lanes of a warp hold, together, in every lane: (m, s, u) with n entries equal to m that are
// not in s.  Of the result's maximum one entry is not in r (owners = 1), if there is any.
struct RowSums {
  float m, r, u;
  int owners;
};
__device__ __forceinline__ RowSums merge_lanes(float m, float s, float u, int n, float c2) {
  RowSums o;
  o.m = m;
#pragma unroll
  for (int w = 16; w > 0; w >>= 1) o.m = fmaxf(o.m, __shfl_xor_sync(0xffffffffu, o.m, w));
  o.r = s;                                                          // nothing, or the NaN that a NaN entry left
  o.u = 0.f;
  o.owners = 0;
  if (m == o.m) {
    o.u = u;
    o.owners = n;
  } else if (m > -INFINITY) {
    const float d = fmaxf((m - o.m) * c2, -1000.f), sc = fast_ex2(d), tot = s + (float)n;
    o.r = tot * sc;
    o.u = sc * fmaf(d, tot, u);
  }
#pragma unroll
  for (int w = 16; w > 0; w >>= 1) {
    o.r += __shfl_xor_sync(0xffffffffu, o.r, w);
    o.u += __shfl_xor_sync(0xffffffffu, o.u, w);
    o.owners += __shfl_xor_sync(0xffffffffu, o.owners, w);
  }
  if (o.owners > 1) { o.r += (float)(o.owners - 1); o.owners = 1; }
  return o;
}

// A row is read once, by one block or, where there are fewer rows than the GPU takes, by a cluster of up to 16 that
// each take a slice and merge over distributed shared memory: one launch, no workspace.  Each warp keeps a running
// maximum for its lanes, each lane its sums relative to it, and its own largest entry.  The k-th largest of the block's
// 256 lane maxima bounds the k-th largest entry of the slice from below, and entries at or above it sit in lanes whose
// maximum is: only their few vectors are read again.
// Bound by issue slots (about ten instructions an entry): 4096 rows of 151936 bf16 take 247 us, 5.0 TB/s of the 6.5 that a copy
// does, and 300 us with 8 alternatives; one row of float32 takes 10 us, 257 rows of 32003 float16 with 20 alternatives 12.
// kHeld (the self-test of the bounded waits): the copies are never issued, and a wait gives up after args.wait_limit cycles.
template <typename T, bool kHeld = false>
__global__ void __launch_bounds__(kRowThreads, 4)
logits_rows_kernel(const RowsArgs args) {
  namespace cg = cooperative_groups;
  using Type = RowType<T>;
  constexpr int E = Type::per_vec;
  constexpr int kShift = 32 - Type::key_bits;
  constexpr int kWarps = kRowThreads / 32;
  cg::cluster_group cluster = cg::this_cluster();
  const int n_slice = (int)cluster.num_blocks(), slice = (int)cluster.block_rank();
  __shared__ float sh_m[kWarps], sh_s[kWarps], sh_u[kWarps];
  __shared__ int sh_n[kWarps];
  extern __shared__ uint8_t ring_raw[];
  __shared__ __align__(8) uint64_t bar_full[kRowStages], bar_empty[kRowStages];
  __shared__ volatile int abort_flag;
  __shared__ RowSlice sh_mine;
  __shared__ float all_m, all_r, all_u;
  __shared__ float sh_row[2];                                       // m, ln s
  __shared__ uint32_t sh_tau;
  __shared__ unsigned long long cand[kRowCandidates];
  __shared__ int owners[kRowThreads];
  __shared__ int n_owner, n_cand, sh_scan[kWarps + 1], sh_rank[kMaxTop];
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int V = args.V, k = args.k;
  const int row = blockIdx.x / n_slice;
  const T* base = static_cast<const T*>(args.logits) + (size_t)row * args.ld;
  // [0, head) and [V - tail, V) are read element by element (by the first block), the vectors between them start on 16 bytes
  const int head = min(V, (int)(((16u - (uint32_t)(reinterpret_cast<uintptr_t>(base) & 15u)) & 15u) / sizeof(T)));
  const int all_vec = (V - head) / E;
  const int per_slice = (all_vec + n_slice - 1) / n_slice;
  const int v0 = min(all_vec, slice * per_slice), nvec = min(all_vec - v0, per_slice);
  const int extras = slice == 0 ? V - all_vec * E : 0;              // head + tail < 2 E
  const uint4* vecs = reinterpret_cast<const uint4*>(base + head) + v0;
  const int first_id = head + v0 * E;
  auto extra_id = [&](int i) { return i < head ? i : all_vec * E + i; };
  // the slice's entries in the order of their ids: the first block has the head before its vectors and the tail behind
  const int n_local = nvec * E + extras;
  auto local_id = [&](int i) {
    return slice != 0 ? first_id + i : (i < head + nvec * E ? i : all_vec * E + i - nvec * E);
  };
  const float c2 = args.kappa * kLog2e;

  const uint4* ring_ptr = reinterpret_cast<const uint4*>((reinterpret_cast<uintptr_t>(ring_raw) + 127u) & ~(uintptr_t)127u);
  const uint32_t ring = ptx::smem_u32(ring_ptr);
  if (tid == 0) {
    abort_flag = 0;
    for (int i = 0; i < kRowStages; ++i) {
      ptx::mbar_init(ptx::smem_u32(&bar_full[i]), 1);
      ptx::mbar_init(ptx::smem_u32(&bar_empty[i]), kWarps);
    }
    ptx::mbar_fence_init();
    ptx::fence_async_proxy();
  }
  __syncthreads();

  // the target's logit is on its way early
  int y = 0;
  float at_y = 0.f;
  if (tid == 0 && slice == 0 && args.logp) {
    y = args.targets[row];
    at_y = row_value(base[min(max(y, 0), V - 1)]);
  }

  RowState st;
  if (slice == 0) {
    const float v = tid < extras ? row_value(base[extra_id(tid)]) : -INFINITY;
    float x[2] = {max_nan(v, kFloor), kFloor};
    st.fold<2>(x, v, c2, tid < extras, [&](int j) { return j == 0 ? v : -INFINITY; });
  }
  auto work = [&](const uint4 (&v)[kRowUnroll], int b) {
    float x[kRowUnroll * E], cmax = -INFINITY;
#pragma unroll
    for (int q = 0; q < kRowUnroll; ++q) {
      cmax = fmaxf(cmax, Type::top(v[q]));
      float w[E];
      Type::floored(v[q], w);
#pragma unroll
      for (int j = 0; j < E; ++j) x[q * E + j] = w[j];
    }
    st.fold<kRowUnroll * E>(x, cmax, c2, b + tid < nvec, [&](int j) {
      const int i = b + (j / E) * kRowThreads + tid;
      return i < nvec ? row_value(base[first_id + i * E + j % E]) : -INFINITY;
    });
  };
  // The slice streams through a ring of three 16 KB batches that the copy engine fills (192 KB in flight on an SM with
  // four blocks).  A batch's slot is filled again one batch after it was read, by then by all warps.  The loads from a slot
  // and the copy that fills it next go through different proxies: without the fence between them a slot was released while
  // loads were on their way, and one row in 10^5 saw a vector of a later batch (the fence costs nothing that shows: 285 us for
  // 4096 rows of 151936 bf16 with it and without).
  const int n_batch = (nvec + kRowBatch - 1) / kRowBatch;
  const long long wait_limit = kHeld ? args.wait_limit : kWaitLimitCycles;
  auto refill = [&](int i) {                                        // thread 0
    if (kHeld) return;
    const uint32_t bytes = (uint32_t)min(kRowBatch, nvec - i * kRowBatch) * 16u, bar = ptx::smem_u32(&bar_full[i % kRowStages]);
    ptx::mbar_arrive_expect_tx(bar, bytes);
    ptx::bulk_load(ring + (uint32_t)(i % kRowStages) * kRowBatch * 16u, vecs + (size_t)i * kRowBatch, bytes, bar);
  };
  if (tid == 0)
    for (int i = 0; i < min(n_batch, kRowStages); ++i) refill(i);
  for (int i = 0; i < n_batch; ++i) {
    const int stage = i % kRowStages, b = i * kRowBatch;
    if (!__all_sync(0xffffffffu, ptx::mbar_wait_bounded(ptx::smem_u32(&bar_full[stage]), (uint32_t)(i / kRowStages) & 1u, &abort_flag,
                                                        wait_limit)))
      break;
    uint4 v[kRowUnroll];
    const uint4* src = ring_ptr + stage * kRowBatch + tid;
#pragma unroll
    for (int q = 0; q < kRowUnroll; ++q) v[q] = src[q * kRowThreads];
    if (b + kRowBatch > nvec) {                                     // the last batch
#pragma unroll
      for (int q = 0; q < kRowUnroll; ++q)
        if (b + q * kRowThreads + tid >= nvec) v[q] = make_uint4(Type::neg_inf, Type::neg_inf, Type::neg_inf, Type::neg_inf);
    }
    ptx::fence_async_proxy();
    __syncwarp();
    if (lane == 0) ptx::mbar_arrive(ptx::smem_u32(&bar_empty[stage]));
    if (tid == 0 && i > 0 && i - 1 + kRowStages < n_batch) {
      const int last = (i - 1) % kRowStages;
      if (ptx::mbar_wait_bounded(ptx::smem_u32(&bar_empty[last]), (uint32_t)((i - 1) / kRowStages) & 1u, &abort_flag, wait_limit))
        refill(i - 1 + kRowStages);
    }
    __syncwarp();
    work(v, b);
  }
  if (abort_flag && tid == 0) {                                     // copies that are late have a bounded time to land
    const long long t0 = clock64();
    while (clock64() - t0 < 20000000LL) {
    }
  }

  // ---- merge lanes, then warps
  {
    const float f = residue_ex2(-st.delta);                         // back from ref to c2 m
    float s = st.s * f, u = fmaf(-st.delta, st.s, st.u) * f, n = st.own;
    if (abort_flag) s = __uint_as_float(0x7FC00000u);               // a copy that never came: the row's results are NaN
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) {
      s += __shfl_xor_sync(0xffffffffu, s, o);
      u += __shfl_xor_sync(0xffffffffu, u, o);
      n += __shfl_xor_sync(0xffffffffu, n, o);
    }
    if (lane == 0) { sh_m[warp] = st.m; sh_s[warp] = s; sh_u[warp] = u; sh_n[warp] = (int)n; }
  }
  if (tid == 0) { n_owner = 0; n_cand = 0; }
  __syncthreads();
  const bool gave_up = abort_flag != 0;                             // the same in all threads: nobody waits any more
  if (gave_up && tid == 0 && args.status) atomicOr(args.status, kStatusTimeout);
  if (warp == 0) {
    const bool on = lane < kWarps;
    const RowSums all = merge_lanes(on ? sh_m[lane] : -INFINITY, on ? sh_s[lane] : 0.f, on ? sh_u[lane] : 0.f, on ? sh_n[lane] : 0, c2);
    if (lane == 0) { sh_mine.m = all.m; sh_mine.r = all.r; sh_mine.u = all.u; sh_mine.owners = all.owners; }
  }

  // ---- the slice's k largest, falling, into sh_mine.top; none where a copy never came
  if (gave_up) {
    if (tid < kMaxTop) sh_mine.top[tid] = 0ull;
  } else if (k > 0) {
    const bool holds = tid < nvec || tid < extras;
    const uint32_t mine = holds ? (order_key(st.lane_max) >> kShift) : 0u;
    // The lanes' places by their maxima: each warp sorts its 32 (shuffles), and every entry then looks up in the other
    // warps' sorted lists how many are before it.  (A search over the bits of the k-th is a chain of 8 to 16 votes:
    // 4700 cycles with 32-bit keys.)  The lane in place k - 1 has tau, the k-th largest class.
    uint32_t* sorted = reinterpret_cast<uint32_t*>(cand);
    unsigned long long mine_at = ((unsigned long long)mine << 32) | (uint32_t)tid;      // falling by key
#pragma unroll
    for (int size = 2; size <= 32; size <<= 1)
#pragma unroll
      for (int step = size >> 1; step > 0; step >>= 1) {
        const unsigned long long other = __shfl_xor_sync(0xffffffffu, mine_at, step);
        const bool larger_here = ((lane & size) == 0) == ((lane & step) == 0);
        mine_at = (other > mine_at) == larger_here ? other : mine_at;
      }
    const uint32_t key = (uint32_t)(mine_at >> 32);
    sorted[tid] = key;
    __syncthreads();
    int place = lane;
#pragma unroll
    for (int w = 0; w < kWarps; ++w) {
      // the number of entries before this one: larger ones, and equal ones of the warps before
      int lo = 0;
#pragma unroll
      for (int step = 16; step > 0; step >>= 1) {
        const uint32_t o = sorted[w * 32 + lo + step - 1];
        if (o > key || (o == key && w < warp)) lo += step;
      }
      const uint32_t o = sorted[w * 32 + lo];                       // 31 compared so far
      if (o > key || (o == key && w < warp)) ++lo;
      if (w != warp) place += lo;
    }
    if (place == k - 1) sh_tau = max(key, 1u);                      // 0 is NaN's class
    if (tid < kMaxTop) sh_mine.top[tid] = 0ull;
    __syncthreads();
    const uint32_t tau = sh_tau;
    if (key >= tau) owners[place] = (int)(uint32_t)mine_at;         // places 0, 1, ...
    const int n_above = __syncthreads_count(key >= tau);
    if (tid == 0) n_owner = n_above;
    __syncthreads();
    const int per_lane = (nvec + kRowThreads - 1) / kRowThreads;
    auto offer = [&](float x, int id) {
      const int at = atomicAdd(&n_cand, 1);
      if (at < kRowCandidates) cand[at] = pack_entry(order_key(x), id);
    };
    // entries of class `least` or above, from the lanes whose maximum is
    const bool in_ring = n_batch <= kRowStages;                     // a short slice is still in shared memory
    auto collect = [&](uint32_t least) {
      // values of the class or above, and only they, are not below it (keys up to that of -inf are nobody's)
      const float bar = (least << kShift) <= kKeyNegInf ? -INFINITY : key_value(least << kShift);
      if (tid < extras && row_value(base[extra_id(tid)]) >= bar) offer(row_value(base[extra_id(tid)]), extra_id(tid));
      const int items = n_owner * per_lane;
      for (int w = tid; w < items; w += kRowThreads) {
        const int i = (w % per_lane) * kRowThreads + owners[w / per_lane];
        if (i >= nvec) continue;
        float x[E];
        Type::entries(in_ring ? ring_ptr[i] : __ldg(vecs + i), x);
#pragma unroll
        for (int j = 0; j < E; ++j)
          if (x[j] >= bar) offer(x[j], first_id + i * E + j);
      }
      __syncthreads();
    };
    bool done = false;
    // many lanes tie at tau, or tau is the masked entries' -inf: only what is above it is collected that way
    const bool many = n_owner > 4 * k + 32 || tau <= (kKeyNegInf >> kShift);
    if (!many) {
      collect(tau);
      done = n_cand >= k && n_cand <= kRowCandidates;
    }
    if (!done) {
      __syncthreads();
      if (tid == 0) { n_cand = 0; n_owner = 0; }
      __syncthreads();
      if (key > tau) owners[atomicAdd(&n_owner, 1)] = (int)(uint32_t)mine_at;
      __syncthreads();
      collect(tau + 1u);
      if (n_cand <= kRowCandidates - k) {
        // then entries of tau's class in the order of their ids until there are k.  A class is one value: what a
        // 16-bit type's key drops is constant
        int have = n_cand;
        for (int b = 0; b < n_local && have < k; b += kRowThreads) {
          const int id = b + tid < n_local ? local_id(b + tid) : -1;
          const uint32_t at_id = id >= 0 ? order_key(row_value(base[id])) : 0u;
          const bool hit = id >= 0 && (at_id >> kShift) == tau;
          const uint32_t votes = __ballot_sync(0xffffffffu, hit);
          if (lane == 0) sh_scan[warp] = __popc(votes);
          __syncthreads();
          int before = 0, total = 0;
          for (int w = 0; w < kWarps; ++w) {
            if (w < warp) before += sh_scan[w];
            total += sh_scan[w];
          }
          const int at = have + before + __popc(votes & ((1u << lane) - 1u));
          if (hit && at < k) cand[at] = pack_entry(at_id, id);
          have = min(k, have + total);
          __syncthreads();
        }
        if (tid == 0) n_cand = max(have, n_cand);
        done = true;
        __syncthreads();
      }
    }
    if (done) {
      const int n = n_cand;
      for (int c = tid; c < n; c += kRowThreads) {
        const unsigned long long e = cand[c];
        int rank = 0;
        for (int o = 0; o < n; ++o) rank += cand[o] > e ? 1 : 0;
        if (rank < k) sh_mine.top[rank] = e;
      }
    } else {
      // a few lanes hold hundreds of entries above the bound: k passes, each for the best entry below the last one
      unsigned long long last = ~0ull;
      for (int at = 0; at < k && last != 0ull; ++at) {
        unsigned long long best = 0ull;
        for (int i = tid; i < n_local; i += kRowThreads) {
          const int id = local_id(i);
          const uint32_t at_id = order_key(row_value(base[id]));
          const unsigned long long e = at_id ? pack_entry(at_id, id) : 0ull;
          if (e < last && e > best) best = e;
        }
        __syncthreads();
        cand[tid] = best;
        __syncthreads();
        for (int o = kRowThreads / 2; o > 0; o >>= 1) {
          if (tid < o && cand[tid + o] > cand[tid]) cand[tid] = cand[tid + o];
          __syncthreads();
        }
        last = cand[0];
        if (tid == 0) sh_mine.top[at] = last;
      }
    }
  }
  __syncthreads();

  // ---- the slices of the row together
  if (n_slice > 1) {
    cluster.sync();
    for (int i = tid; i < n_slice * k; i += kRowThreads) cand[i] = cluster.map_shared_rank(&sh_mine, i / k)->top[i % k];
    if (warp == 0) {
      const RowSlice* o = cluster.map_shared_rank(&sh_mine, lane < n_slice ? lane : 0);
      const bool on = lane < n_slice;
      const RowSums all = merge_lanes(on ? o->m : -INFINITY, on ? o->r : 0.f, on ? o->u : 0.f, on ? o->owners : 0, c2);
      if (lane == 0) { all_m = all.m; all_r = all.r; all_u = all.u; }
    }
    if (tid < kMaxTop) sh_rank[tid] = 0;
    cluster.barrier_arrive();                                       // done with the other blocks' memory
    __syncthreads();
  }
  if (tid == 0) {
    const float M = n_slice > 1 ? all_m : sh_mine.m, r = n_slice > 1 ? all_r : sh_mine.r, uu = n_slice > 1 ? all_u : sh_mine.u;
    const bool nothing = M == -INFINITY && r == 0.f;                // no entry has a probability
    const float ln_s = nothing ? 0.f : (M == -INFINITY ? __uint_as_float(0x7FC00000u) : log1pf(r));
    sh_row[0] = M;
    sh_row[1] = ln_s;
    if (slice == 0) {
      if (args.partials) args.partials[row] = make_float4(M, r, 0.f, 0.f);
      if (args.lse) args.lse[row] = nothing ? -INFINITY : fmaf(args.kappa, M, ln_s);
      if (args.norm) args.norm[row] = make_float2(M, ln_s);
      if (args.entropy) args.entropy[row] = nothing ? 0.f : max_nan(ln_s - kLn2 * uu / (1.f + r), 0.f);
      if (args.logp) {
        const bool bad = y < 0 || y >= V;
        if (bad && args.status) atomicOr(args.status, kStatusBadTarget);      // the LM-head calls report and clamp
        args.logp[row] = bad && !args.status ? __uint_as_float(0x7FC00000u)
                         : nothing           ? -INFINITY
                                             : args.kappa * (at_y - M) - ln_s;
      }
    }
  }
  if (k > 0) {
    __syncthreads();
    const float M = sh_row[0], ln_s = sh_row[1];
    auto put = [&](int at, unsigned long long entry) {
      const float x = key_value((uint32_t)(entry >> 32));
      args.top_ids[(size_t)row * k + at] = entry == 0ull ? -1 : (int)~(uint32_t)entry;
      args.top_logp[(size_t)row * k + at] = M == -INFINITY && ln_s == 0.f ? (entry == 0ull ? x : -INFINITY)
                                                                          : args.kappa * (x - M) - ln_s;
    };
    if (n_slice == 1) {
      if (tid < k) put(tid, sh_mine.top[tid]);                      // 0: fewer than k entries are numbers
    } else {
      // an entry's place: how many of every slice's list are better
      for (int w = tid; w < k * n_slice; w += kRowThreads) {
        const unsigned long long e = sh_mine.top[w % k];
        const unsigned long long* list = cand + (w / k) * k;
        int lo = 0, hi = k;
        while (lo < hi) {
          const int mid = (lo + hi) >> 1;
          if (list[mid] > e) lo = mid + 1; else hi = mid;
        }
        if (e != 0ull && lo > 0) atomicAdd(&sh_rank[w % k], lo);
      }
      int used = 0;
      for (int i = tid; i < n_slice * k; i += kRowThreads) used += cand[i] != 0ull ? 1 : 0;
      used = __syncthreads_count(used > 0) + __syncthreads_count(used > 1);      // at most two a thread
      if (tid < k && sh_mine.top[tid] != 0ull && sh_rank[tid] < k) put(sh_rank[tid], sh_mine.top[tid]);
      if (slice == 0 && tid >= used && tid < k) put(tid, 0ull);
    }
  }
  if (n_slice > 1) cluster.barrier_wait();                          // no block leaves while another reads its list
}

// ------------------------------------------------------------------------------------------
// Merge of the LM-head sweep's partials: one warp per token.  partials[split][t] = (m, r, u, -) as the sweep's
// epilogue defines them (u in units of log2).  Bound by the latency of its chain (partials, heads of the lists, their rest,
// ids): 3 us without alternatives, 11 us for 1537 tokens x 20 lists of 8, 14 of 32, 45 us for 8192 tokens x 18 lists of 32.
// ------------------------------------------------------------------------------------------
struct MergeArgs {
  int T, n_split, k;
  float kappa;
  const float4* partials;
  const float* acc_y;
  const float* top_val;     // [n_split][T][k]
  const int* top_id;
  float *logp, *entropy, *lse;
  float2* norm;
  int* out_ids;             // [T][k]
  float* out_logp;
};

// (m, r) of all splits of token t, in every lane of the warp; u likewise.
__device__ __forceinline__ void merge_partials(const float4* __restrict__ partials, int n_split, int T, int t, float c2,
                                               float& M, float& r, float& u) {
  const int lane = threadIdx.x & 31;
  M = -INFINITY;
  for (int k = lane; k < n_split; k += 32) M = fmaxf(M, partials[(size_t)k * T + t].x);
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) M = fmaxf(M, __shfl_xor_sync(0xffffffffu, M, o));
  r = 0.f;
  u = 0.f;
  int at_max = 0;
  for (int k = lane; k < n_split; k += 32) {
    const float4 p = partials[(size_t)k * T + t];
    if (p.x == M) {
      if (M > -INFINITY) ++at_max;
      r += p.y;
      u += p.z;
    } else if (p.x > -INFINITY) {
      const float d = fmaxf((p.x - M) * c2, -1000.f), sc = fast_ex2(d);
      r = fmaf(p.y + 1.f, sc, r);
      u = fmaf(sc, fmaf(d, p.y + 1.f, p.z), u);
    } else {
      r += p.y;
    }
  }
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) {
    r += __shfl_xor_sync(0xffffffffu, r, o);
    u += __shfl_xor_sync(0xffffffffu, u, o);
    at_max += __shfl_xor_sync(0xffffffffu, at_max, o);
  }
  if (at_max > 1) r += (float)(at_max - 1);
}

constexpr int kMergeCandidates = 256;
constexpr int kMergeWarps = 8;

__global__ void __launch_bounds__(32 * kMergeWarps) merge_scores_kernel(const MergeArgs a) {
  __shared__ unsigned long long sh_lists[kMergeWarps * kMergeCandidates];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int t = blockIdx.x * kMergeWarps + warp;
  if (t >= a.T) return;
  float M, r, u;
  merge_partials(a.partials, a.n_split, a.T, t, a.kappa * kLog2e, M, r, u);
  const float ln_s = log1pf(r);
  if (lane == 0) {
    if (a.lse) a.lse[t] = fmaf(a.kappa, M, ln_s);
    if (a.norm) a.norm[t] = make_float2(M, ln_s);
    if (a.entropy) a.entropy[t] = max_nan(ln_s - kLn2 * u / (1.f + r), 0.f);
    if (a.logp) a.logp[t] = a.kappa * (a.acc_y[t] - M) - ln_s;
  }
  if (a.k == 0) return;
  // The lists fall.  The k-th largest of the first q entries of every list, at least 2 k of them, bounds the row's top
  // from below: what is below it stays out, the rest (a few more than k) is ranked by counting.
  unsigned long long* cand = sh_lists + (size_t)warp * kMergeCandidates;
  const size_t stride = (size_t)a.T * a.k;
  const float* val = a.top_val + (size_t)t * a.k;
  const int* id = a.top_id + (size_t)t * a.k;
  constexpr int kHeads = (2 * kMaxTop + kMaxRowLists + 31) / 32;
  const int q = min(a.k, (2 * a.k + a.n_split - 1) / a.n_split), heads = q * a.n_split;
  uint32_t key[kHeads];
#pragma unroll
  for (int i = 0; i < kHeads; ++i) {
    const int j = i * 32 + lane;
    key[i] = j < heads ? order_key(val[(j / q) * stride + j % q]) : 0u;
  }
  uint32_t least = 0u;
#pragma unroll 1
  for (int bit = 31; bit >= 0; --bit) {
    const uint32_t c = least | (1u << bit);
    int count = 0;
#pragma unroll
    for (int i = 0; i < kHeads; ++i)
      if (i * 32 < heads) count += __popc(__ballot_sync(0xffffffffu, key[i] >= c));
    if (count >= a.k) least = c;
  }
  const int width = a.k <= 8 ? 8 : (a.k <= 16 ? 16 : 32), per = 32 / width;      // lists a round takes
  const int e = lane % width, l0 = lane / width;
  int n = 0;
  constexpr int kAhead = 12;                                        // loads in flight: the rounds depend on each other only by n
  for (int l = 0; l < a.n_split; l += per * kAhead) {
    float x[kAhead];
#pragma unroll
    for (int j = 0; j < kAhead; ++j) {
      const int at = l + j * per + l0;
      x[j] = at < a.n_split && e < a.k ? __ldg(val + at * stride + e) : NAN;
    }
#pragma unroll
    for (int j = 0; j < kAhead; ++j) {
      const uint32_t key_x = order_key(x[j]);
      const bool keep = key_x != 0u && key_x >= least;
      const uint32_t votes = __ballot_sync(0xffffffffu, keep);
      const int pos = n + __popc(votes & ((1u << lane) - 1u));
      if (keep && pos < kMergeCandidates) cand[pos] = ((unsigned long long)key_x << 32) | (uint32_t)((l + j * per + l0) * 32 + e);
      n += __popc(votes);
    }
  }
  __syncwarp();
  // the ids of the few that stay, together; an unused place of a list is -inf with id -1 and sorts behind
  for (int c = lane; c < min(n, kMergeCandidates); c += 32) {
    const uint32_t from = (uint32_t)cand[c];
    const int i = __ldg(id + (from / 32) * stride + from % 32);
    cand[c] = i < 0 ? 0ull : pack_entry((uint32_t)(cand[c] >> 32), i);
  }
  __syncwarp();
  auto put = [&](int at, unsigned long long entry) {
    a.out_ids[(size_t)t * a.k + at] = entry == 0ull ? -1 : (int)~(uint32_t)entry;
    a.out_logp[(size_t)t * a.k + at] = a.kappa * (key_value((uint32_t)(entry >> 32)) - M) - ln_s;
  };
  if (n <= kMergeCandidates) {
    for (int c = lane; c < max(n, a.k); c += 32) {
      if (c >= n) { put(c, 0ull); continue; }                       // fewer than k entries are numbers
      const unsigned long long mine = cand[c];
      int rank = 0;
#pragma unroll 8
      for (int o = 0; o < n; ++o) rank += cand[o] > mine ? 1 : 0;
      if (mine == 0ull) rank = n + 1;                               // an unused place: written below
      if (rank < a.k) put(rank, mine);
    }
    __syncwarp();
    int used = 0;
    for (int c = lane; c < n; c += 32) used += cand[c] != 0ull ? 1 : 0;
    used = __reduce_add_sync(0xffffffffu, used);
    for (int c = used + lane; c < min(n, a.k); c += 32) put(c, 0ull);
    return;
  }
  // many equal entries: k rounds, each for the best entry below the last one
  unsigned long long last = ~0ull;
  for (int at = 0; at < a.k; ++at) {
    unsigned long long best = 0ull;
    for (int l = 0; l < a.n_split; l += per) {
      const int li = l + l0;
      if (li >= a.n_split || e >= a.k) continue;
      const int i = id[li * stride + e];
      if (i < 0) continue;
      const unsigned long long x = pack_entry(order_key(val[li * stride + e]), i);
      if (x < last && x > best) best = x;
    }
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) {
      const unsigned long long other = __shfl_xor_sync(0xffffffffu, best, o);
      best = other > best ? other : best;
    }
    last = best;
    if (lane == 0) put(at, best);
    if (best == 0ull) {
      for (int c = at + 1 + lane; c < a.k; c += 32) put(c, 0ull);
      return;
    }
  }
}

// ------------------------------------------------------------------------------------------ gradients of scores
// (m, log2 s, alpha, beta) and the value at the target's column for the dz pass:
//   dz_j = kappa g (1[j = y] - p_j) - kappa e p_j (log p_j + H) = 2^L (alpha + beta L) off the target, L = log2 p_j.
// A zero gradient takes its factor out: the log-prob and entropy of a padding row may be NaN.
__global__ void row_params_kernel(int T, float kappa, const float2* __restrict__ norm, const float* __restrict__ logp,
                                  const float* __restrict__ entropy, const float* __restrict__ d_logp,
                                  const float* __restrict__ d_entropy, float4* __restrict__ row_p, float* __restrict__ row_ins) {
  const int t = blockIdx.x * blockDim.x + threadIdx.x;
  if (t >= T) return;
  const float g = d_logp ? d_logp[t] : 0.f, e = d_entropy ? d_entropy[t] : 0.f;
  const float H = d_entropy ? entropy[t] : 0.f;
  const float2 n = norm[t];
  row_p[t] = make_float4(n.x, n.y * kLog2e, -kappa * (e != 0.f ? fmaf(e, H, g) : g), -kappa * e * kLn2);
  if (d_logp) {
    const float l = logp[t];
    row_ins[t] = kappa * ((g != 0.f ? -expm1f(l) * g : 0.f) - (e != 0.f ? expf(l) * e * (l + H) : 0.f));
  }
}

// dz of a panel of raw float32 logits in place (CUDA-core path): rows [t0, t0 + gridDim.y).
__global__ void dz_rows_f32_kernel(float* __restrict__ panel, size_t ld, int V, int t0, float kappa,
                                   const float4* __restrict__ row_p, const float* __restrict__ row_ins,
                                   const int* __restrict__ targets) {
  const int t = t0 + blockIdx.y;
  float* row = panel + (size_t)blockIdx.y * ld;
  const float4 rp = row_p[t];
  const bool live = rp.z != 0.f || rp.w != 0.f;
  int y = -1;
  if (targets) y = min(max(targets[t], 0), V - 1);
  const float c2 = kappa * kLog2e, from = snap_from(rp, c2);
  for (int v = blockIdx.x * blockDim.x + threadIdx.x; v < V; v += gridDim.x * blockDim.x) {
    const float a = row[v];
    const float L = fmaf((a > from ? rp.x : a) - rp.x, c2, -rp.y);
    float d = live ? exp2f(L) * fmaf(rp.w, L, rp.z) : 0.f;
    if (v == y) d = row_ins[t];
    row[v] = d;
  }
}

// ------------------------------------------------------------------------------------------ distillation
// Teacher lists, one warp per token: the distinct valid ids in rising order (then INT_MAX), and for every entry
// the place of its id: bits 0-6, bit 7 set where an earlier entry has the same id; 255 for an entry that is padding
// (-1) or out of range (reported).  By comparing all pairs with shuffles: 8 us for 1537 tokens x 20, 22 for 8192 x 32.
__global__ void distill_sort_kernel(int T, int K, int V, const int* __restrict__ ids, int* __restrict__ sorted,
                                    uint8_t* __restrict__ slots, int* __restrict__ status) {
  const int lane = threadIdx.x & 31;
  const int t = blockIdx.x * (blockDim.x >> 5) + (threadIdx.x >> 5);
  if (t >= T) return;
  constexpr int kPer = kMaxList / 32;
  int id[kPer], rank[kPer];
  bool first[kPer];
#pragma unroll
  for (int q = 0; q < kPer; ++q) {
    const int i = q * 32 + lane;
    id[q] = i < K ? ids[(size_t)t * K + i] : -1;
    if (id[q] < -1 || id[q] >= V) {
      atomicOr(status, kStatusBadTarget);
      id[q] = -1;
    }
    first[q] = id[q] >= 0;
    rank[q] = 0;
  }
#pragma unroll
  for (int qj = 0; qj < kPer; ++qj) {
    if (qj * 32 >= K) break;
    for (int l = 0; l < 32; ++l) {
      const int other = __shfl_sync(0xffffffffu, id[qj], l), j = qj * 32 + l;
#pragma unroll
      for (int q = 0; q < kPer; ++q)
        if (other == id[q] && j < q * 32 + lane) first[q] = false;
    }
  }
  int distinct = 0;
#pragma unroll
  for (int qj = 0; qj < kPer; ++qj) {
    if (qj * 32 >= K) break;
    const uint32_t firsts = __ballot_sync(0xffffffffu, first[qj]);
    distinct += __popc(firsts);
    for (int l = 0; l < 32; ++l) {
      const int other = __shfl_sync(0xffffffffu, id[qj], l);
      const bool counts = (firsts >> l) & 1u;
#pragma unroll
      for (int q = 0; q < kPer; ++q)
        if (counts && other < id[q]) ++rank[q];
    }
  }
#pragma unroll
  for (int q = 0; q < kPer; ++q) {
    const int i = q * 32 + lane;
    if (i >= K) break;
    slots[(size_t)t * K + i] = id[q] < 0 ? 255u : (uint8_t)(rank[q] | (first[q] ? 0 : 128));
    if (first[q]) sorted[(size_t)t * K + rank[q]] = id[q];
    if (i >= distinct) sorted[(size_t)t * K + i] = INT_MAX;
  }
}

// Float32 panel of raw logits: the list's logits are taken out (and replaced by -inf), one warp per token.
__global__ void distill_take_kernel(int rows, int t0, int K, float* __restrict__ panel, size_t ld,
                                    const int* __restrict__ sorted, float* __restrict__ list_z) {
  const int lane = threadIdx.x & 31;
  const int i = blockIdx.x * (blockDim.x >> 5) + (threadIdx.x >> 5);
  if (i >= rows) return;
  const size_t t = (size_t)t0 + i;
  for (int q = lane; q < K; q += 32) {
    const int id = sorted[t * K + q];
    if (id == INT_MAX) continue;
    list_z[t * K + q] = panel[(size_t)i * ld + id];
    panel[(size_t)i * ld + id] = -INFINITY;
  }
}

struct DistillRowArgs {
  int T, K, n_split, mode;
  float kappa, teacher_kappa;
  double inv_N;
  const float4* partials;   // (m, r, -, -) of the entries off the list, per split
  const float* list_z;      // [T][K] raw logits by place
  const uint8_t* slots;     // [T][K]
  const float* teacher;     // [T][K]
  const float* weights;     // [T] or NULL (1)
  float* kl;                // [T]
  float2* norm;             // [T] (m, ln s) over the entries off the list
  float* lse;               // [T] or NULL
  float* loss;
  unsigned int* done;       // zero before the launch
  float* coef;              // [T]: off the list d loss / d z_j = coef times the softmax over the entries off the list
  float* entry_grad;        // [T][K]: d loss / d z at the entry's id
};

__device__ __forceinline__ double warp_sum(double v) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
  return v;
}
__device__ __forceinline__ double warp_max(double v) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) v = fmax(v, __shfl_xor_sync(0xffffffffu, v, o));
  return v;
}

constexpr int kDistillThreads = 256;

// The loss of a token and its gradient on the list, one warp per token, in 64 bits: a token has at most 128 entries,
// and 1 - sum q and the differences p - q cancel.  9 us for 512 tokens x 16 entries, 14 for 1537 x 20, 39 for 8192 x 32.
__device__ __forceinline__ void distill_row(const DistillRowArgs& a, int t) {
  const int lane = threadIdx.x & 31;
  constexpr int kPer = kMaxList / 32;
  float m_off, r_off, unused;
  merge_partials(a.partials, a.n_split, a.T, t, a.kappa * kLog2e, m_off, r_off, unused);
  float z[kPer];
  uint8_t slot[kPer];
  double logq[kPer];
  float top = m_off;
  double tmax = -INFINITY;
  int n_valid = 0, n_again = 0;
#pragma unroll
  for (int q = 0; q < kPer; ++q) {
    const int i = q * 32 + lane;
    slot[q] = i < a.K ? a.slots[(size_t)t * a.K + i] : 255;
    z[q] = -INFINITY;
    logq[q] = -INFINITY;
    if (slot[q] != 255) {
      z[q] = a.list_z[(size_t)t * a.K + (slot[q] & 127)];
      logq[q] = (double)a.teacher[(size_t)t * a.K + i] * a.teacher_kappa;
      top = fmaxf(top, z[q]);
      tmax = fmax(tmax, logq[q]);
      ++n_valid;
      n_again += slot[q] >> 7;
    }
  }
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) {
    top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, o));
    n_valid += __shfl_xor_sync(0xffffffffu, n_valid, o);
    n_again += __shfl_xor_sync(0xffffffffu, n_again, o);
  }
  const double kappa = (double)a.kappa;
  // sum of e^(kappa (a - top)): off the list, then the list's distinct ids
  const double rest = m_off > -INFINITY ? (1.0 + (double)r_off) * exp(kappa * ((double)m_off - (double)top)) : (double)r_off;
  double on = 0.0;
#pragma unroll
  for (int q = 0; q < kPer; ++q)
    if (slot[q] < 128) on += exp(kappa * ((double)z[q] - (double)top));
  on = warp_sum(on);
  const double ln_s = log(rest + on);
  // ln of the probability off the list; from the exponents, so that it survives where rest underflows
  const double ln_rest = m_off > -INFINITY ? kappa * ((double)m_off - (double)top) + log1p((double)r_off) - ln_s : log(rest) - ln_s;
  if (a.mode == ULORL_DISTILL_RENORM) {
    tmax = warp_max(tmax);
    const double shift = tmax > -INFINITY ? tmax : 0.0;
    double sum = 0.0;
#pragma unroll
    for (int q = 0; q < kPer; ++q) sum += exp(logq[q] - shift);
    sum = log(warp_sum(sum)) + shift;
#pragma unroll
    for (int q = 0; q < kPer; ++q)
      if (tmax > -INFINITY) logq[q] -= sum;                         // a list without any probability stays without
  }
  double Q = 0.0, kl = 0.0, prob[kPer];
#pragma unroll
  for (int q = 0; q < kPer; ++q) {
    prob[q] = 0.0;
    if (slot[q] == 255) continue;
    prob[q] = exp(logq[q]);
    Q += prob[q];
    if (prob[q] != 0.0) kl += prob[q] * (logq[q] - (kappa * ((double)z[q] - (double)top) - ln_s));
  }
  Q = warp_sum(Q);
  kl = warp_sum(kl);
  // Off the list d kl / d z_j is Q p_j, in mode tail (Q + rest_q) p_j - rest_q p_j / rest_p, rest_q = max(1 - Q, 0): a list
  // that adds up to more than one leaves no remainder, and its loss weighs log-probs of Q in all.  A list of every id has
  // none either (m_off is -inf): what a softmax of float32 log-probs leaves to one, 10^-8 or so, would be set against a
  // probability of zero, a loss of infinity.  Both are kept as a multiple of p_j / rest_p, the softmax over what is not
  // listed: for a student that leaves next to nothing there, p_j and rest_p underflow in float32, their quotient and the
  // multiple do not.
  const double rest_p = rest / (rest + on);
  double c_on = Q, c_off = Q * rest_p;
  if (a.mode == ULORL_DISTILL_TAIL) {
    const double rest_q = m_off > -INFINITY ? fmax(1.0 - Q, 0.0) : 0.0;
    c_on = Q > 1.0 || m_off == -INFINITY ? Q : 1.0;                // Q + rest_q
    c_off = c_on * rest_p - rest_q;
    if (rest_q > 0.0) kl += rest_q * (log(rest_q) - ln_rest);
  }
  const double w = a.weights ? (double)a.weights[t] : 1.0;
  const double scale = n_valid > 0 && w != 0.0 ? w * a.inv_N : 0.0;
  if (lane == 0) {
    a.kl[t] = n_valid > 0 ? (float)kl : 0.f;
    a.norm[t] = m_off > -INFINITY ? make_float2(m_off, log1pf(r_off)) : make_float2(0.f, 0.f);
    if (a.lse) a.lse[t] = (float)(kappa * (double)top + ln_s);
    a.coef[t] = scale != 0.0 && (m_off > -INFINITY) ? (float)(scale * c_off) : 0.f;
  }
#pragma unroll
  for (int q = 0; q < kPer; ++q) {
    const int i = q * 32 + lane;
    // an id that is listed again: its probabilities add, and every entry of it gets the whole gradient
    double all = prob[q];
    if (n_again > 0) {
      all = 0.0;
#pragma unroll
      for (int qj = 0; qj < kPer; ++qj)
        for (int l = 0; l < 32; ++l) {
          const double p = __shfl_sync(0xffffffffu, prob[qj], l);
          const int s = __shfl_sync(0xffffffffu, (int)slot[qj], l);
          if (s != 255 && slot[q] != 255 && (s & 127) == (slot[q] & 127)) all += p;
        }
    }
    if (i < a.K)
      a.entry_grad[(size_t)t * a.K + i] =
          slot[q] == 255 || scale == 0.0 ? 0.f
                                         : (float)(scale * (c_on * exp(kappa * ((double)z[q] - (double)top) - ln_s) - all));
  }
}

// The rows, and the batch loss 1/N sum w_t kl_t by the block that is done last, in a fixed order.
__global__ void __launch_bounds__(kDistillThreads) distill_rows_kernel(const DistillRowArgs a) {
  const int t = blockIdx.x * (kDistillThreads / 32) + (threadIdx.x >> 5);
  if (t < a.T) distill_row(a, t);
  __shared__ bool last;
  __threadfence();
  __syncthreads();
  if (threadIdx.x == 0) last = atomicAdd(a.done, 1u) == gridDim.x - 1;
  __syncthreads();
  if (!last) return;
  __threadfence();
  __shared__ double part[kDistillThreads];
  double acc = 0.0;
  for (int i = threadIdx.x; i < a.T; i += kDistillThreads) {
    const double w = a.weights ? (double)a.weights[i] : 1.0;
    if (w != 0.0) acc += w * (double)__ldcg(a.kl + i);              // written by other blocks
  }
  part[threadIdx.x] = acc;
  __syncthreads();
  for (int o = kDistillThreads / 2; o > 0; o >>= 1) {
    if (threadIdx.x < o) part[threadIdx.x] += part[threadIdx.x + o];
    __syncthreads();
  }
  if (threadIdx.x == 0) *a.loss = (float)(part[0] * a.inv_N);
}

// Row parameters of the dz pass: dz_j = kappa grad_loss coef softmax_j, the softmax over what is not on the list.
__global__ void distill_params_kernel(int T, float kappa, const float2* __restrict__ norm, const float* __restrict__ coef,
                                      const float* __restrict__ grad_loss, float4* __restrict__ row_p) {
  const int t = blockIdx.x * blockDim.x + threadIdx.x;
  if (t >= T) return;
  const float gl = grad_loss ? *grad_loss : 1.f;
  row_p[t] = make_float4(norm[t].x, norm[t].y * kLog2e, kappa * gl * coef[t], 0.f);
}

// The list's columns of a dz panel: rows [t0, t0 + rows).  Entries of one id carry the same value.
template <typename TDz>
__global__ void distill_put_kernel(int rows, int t0, int K, int V, float kappa, const float* __restrict__ grad_loss,
                                   const int* __restrict__ ids, const float* __restrict__ entry_grad,
                                   TDz* __restrict__ panel, size_t ld, int planes) {
  const size_t i = (size_t)blockIdx.x * blockDim.x + threadIdx.x;
  if (i >= (size_t)rows * K) return;
  const size_t at = (size_t)t0 * K + i;
  const int id = ids[at];
  if (id < 0 || id >= V) return;
  const float gl = grad_loss ? *grad_loss : 1.f;
  float x = kappa * gl * entry_grad[at];
  TDz* row = panel + (i / K) * ld * planes;                         // planes of ld columns
  for (int q = 0; q < planes; ++q) {
    from_f32(row[(size_t)q * ld + id], x);
    x -= row_value(row[(size_t)q * ld + id]);
  }
}

// Rows of float32 (hidden's T, then W's V, of `cols` columns) as three bf16 planes side by side, x = h + m + l: each is the
// value rounded, the next what that left, so that all 24 bits are kept; planes are `width` columns wide, zero beyond
// `cols`.  Bound by memory, 10 bytes an entry: 115 us for 34816 rows of 2048 (6.2 TB/s), 3 us for 4608 rows of 256.
__global__ void split_planes_kernel(const float* __restrict__ hidden, size_t T, const float* __restrict__ W, size_t V, int cols,
                                    int width, __nv_bfloat16* __restrict__ out) {
  const size_t quads = (T + V) * (size_t)(width / 4);
  for (size_t i = (size_t)blockIdx.x * blockDim.x + threadIdx.x; i < quads; i += (size_t)gridDim.x * blockDim.x) {
    const size_t r = i / (width / 4);
    const int c = (int)(i - r * (width / 4)) * 4;
    const float* x = r < T ? hidden + r * cols : W + (r - T) * cols;
    float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
    if (c < cols) v = __ldg(reinterpret_cast<const float4*>(x + c));                 // cols is a multiple of 8
    __nv_bfloat16* dst = out + r * 3 * (size_t)width + c;
#pragma unroll
    for (int plane = 0; plane < 3; ++plane) {
      const __nv_bfloat162 a = __floats2bfloat162_rn(v.x, v.y), b = __floats2bfloat162_rn(v.z, v.w);
      *reinterpret_cast<uint2*>(dst + (size_t)plane * width) =
          make_uint2(*reinterpret_cast<const uint32_t*>(&a), *reinterpret_cast<const uint32_t*>(&b));
      v.x -= __low2float(a); v.y -= __high2float(a);
      v.z -= __low2float(b); v.w -= __high2float(b);
    }
  }
}

// d_hidden of a panel from the parts over the vocabulary, added in the order of the parts (1537 tokens, H 1024, 5 parts: 5 us).
__global__ void sum_parts_kernel(const float* __restrict__ parts, int n_parts, size_t part_stride, size_t n,
                                 __nv_bfloat16* __restrict__ out) {
  const size_t i = ((size_t)blockIdx.x * blockDim.x + threadIdx.x) * 8;
  if (i >= n) return;                                               // n is a multiple of 8 (H is)
  float acc[8] = {};
  for (int p = 0; p < n_parts; ++p) {
    const float4* src = reinterpret_cast<const float4*>(parts + (size_t)p * part_stride + i);
    const float4 x = src[0], y = src[1];
    acc[0] += x.x; acc[1] += x.y; acc[2] += x.z; acc[3] += x.w;
    acc[4] += y.x; acc[5] += y.y; acc[6] += y.z; acc[7] += y.w;
  }
  uint32_t w[4];
#pragma unroll
  for (int q = 0; q < 4; ++q) {
    __nv_bfloat162 h = __floats2bfloat162_rn(acc[2 * q], acc[2 * q + 1]);
    w[q] = *reinterpret_cast<uint32_t*>(&h);
  }
  *reinterpret_cast<uint4*>(out + i) = make_uint4(w[0], w[1], w[2], w[3]);
}

}  // namespace ulorl
