// Tensor-core kernels (tcgen05 / tensor memory / TMA) for the four dense contractions of the
// token-loss path, bf16 inputs and float32 accumulation:
//
//   kModeStats   a = hidden . W^T per (token tile, vocabulary tile); the epilogue reduces the tile to
//                online-softmax statistics per token (Eq. 6, Eq. 10) -- logits never leave the SM
//   kModeDz      same contraction, epilogue writes dz = coef * (onehot - softmax) as bf16 to a token panel
//   kModeDHidden d_hidden[t, :] = sum_v dz[t, v] W[v, :]
//   kModeDW      d_W[v, :] (+)= sum_t dz[t, v] hidden[t, :]
//
// and the variants of these that token scoring and distillation use:
//
//   kModeScores, kModeScoresTop8, kModeScoresTop32
//                statistics as (max, sum without the maximum's own 1), with the 0, 8 or 32 largest logits of a
//                row kept beside them in registers
//   kModeDistill statistics of the entries that are not on the token's list; the logits of those that are go out
//   kModeDzRow   dz = softmax * (alpha + beta log2 softmax) with per-row alpha and beta, one column overwritten
//   kModeDHiddenPart  d_hidden over a part of the vocabulary, float32 (few token tiles: the parts fill the GPU)
//   kModeDWBf16  d_W rounded to bf16 in the epilogue (all tokens in one launch)
//   kModeDzRow3  kModeDzRow with dz written as three bf16 planes
//
// Of bf16 operands two things are held in fewer bits than a float32 form would, by choice.  dz leaves its kernel as bf16,
// what the two gradient contractions take (as two planes they would cost twice as much): d_hidden and d_W are 2.4e-3 of the
// whole off where rounding them alone gives 1.7e-3 (CUDA-core path: dz in float32).  And a logit is one float32 sum over H that
// the tensor core cuts off rather than rounds: entropy and kl at H 2048 are 2e-6 off where a float32 product is 0.5e-6 off.
//
// Float32 operands of scoring and distillation come as three bf16 planes x = h + m + l (24 bits, see split_planes_kernel)
// side by side in the rows of a matrix, and a contraction runs over six products of planes: what is left out, m l and
// smaller, is 2^-24 of the whole.  hh comes last, so that the accumulator is small while the small products are added.
// 2048 tokens x 32768, H 2048: 1.2 ms a contraction, 1.34 PFLOP/s of bf16 or 220 TFLOP/s of float32, where the CUDA cores
// take 6.9; log-probs 1e-7 and gradients 1e-6 off (relative to the whole).
//
// One kernel template umma_kernel<mode, CTAs per MMA, accumulators per unit>, persistent, one CTA per
// SM: one thread of warp 0 feeds a shared-memory ring with TMA tile loads (128-byte swizzle), one
// thread of warp 1 issues tcgen05.mma into tensor memory, warps 2-5 drain accumulators with
// tcgen05.ld (one output row per thread) and run the mode's epilogue.  192 threads; 320, with
// epilogue warps 2-9, for kModeScores*, kModeDistill, kModeDzRow* and kModeDWBf16.
//   <m, 2, 1>  CTA pair, one 256 x 256 MMA tile over both CTAs, two 256-column accumulator buffers: the
//              epilogue of tile i overlaps the contraction of tile i + 1 (statistics, dz)
//   <m, 2, 2>  CTA pair, 256 x 512 unit = two accumulators fed from the same A stage, tensor memory as
//              one buffer (d_hidden, d_W: long reductions, light epilogues)
//   <m, 1, 1>  single CTA, 128 x 256 tile, two accumulator buffers (cross-check variant)
// Operands whose contraction index is not the contiguous one in memory (W and hidden in the two
// gradient contractions, dz in the d_W one) are loaded as MN-major tiles; nothing is transposed in
// global memory.  No TMA multicast is used.  Every mbarrier wait is bounded.
#pragma once

#include <limits.h>

#include "common.cuh"
#include "ptx_sm100.cuh"

namespace ulorl {

constexpr int kBM = 128;           // accumulator rows (tensor-memory lanes)
constexpr int kBN = 256;           // accumulator columns
constexpr int kBK = 64;            // contraction elements per pipeline stage (128 bytes of bf16)
constexpr int kUmmaK = 16;         // contraction elements per tcgen05.mma
constexpr int kTmemCols = 512;     // two accumulators of kBN columns
constexpr uint32_t kABytes = kBM * kBK * 2;
constexpr uint32_t kBBytes = kBN * kBK * 2;
constexpr uint32_t kChunkBytes = 64 * kBK * 2;   // one MN-major box: 64 k-rows of 64 contiguous elements

// Shared-memory ring per CTA.  One CTA alone loads the whole 256-row B tile (48 KB a stage, 4 stages);
// in a CTA pair each CTA loads its 128 rows of A and half of B (32 KB a stage, 6 stages), and one
// tcgen05.mma over the pair covers 256 x 256 outputs: a third less L2 traffic per flop.  With two
// accumulators per unit (kAcc = 2) a pair covers 256 x 512 outputs per k-block: A is loaded once
// for both column blocks (48 KB a stage, 4 stages), eight MMAs are queued per barrier round trip,
// and tensor memory is used as one 512-column buffer, so the epilogue does not overlap the next
// unit -- right for the gradient contractions, whose reduction runs over 10^4..10^5 elements.

// Two staging tiles (128 rows x 128 bytes each, 128-byte swizzle) through which the d_W epilogue
// hands 32-column chunks of the accumulator to TMA store / reduce-add.
constexpr uint32_t kOutStageBytes = kBM * 128;

// A stage holds kKA "atoms" of 64 contraction elements (one 128-byte swizzle span each); the two
// logits kernels use two atoms a stage, so that eight MMAs are queued per barrier round trip there too.
enum UmmaMode { kModeStats = 0, kModeDz = 1, kModeDHidden = 2, kModeDW = 3,
                kModeScores = 4, kModeScoresTop8 = 5, kModeScoresTop32 = 6, kModeDistill = 7,
                kModeDzRow = 8, kModeDHiddenPart = 9, kModeDWBf16 = 10, kModeDzRow3 = 11 };

// Planes of A and of B in the six products (h 0, m 1, l 2), two bits each: l h, h l, m m, h m, m h, h h.
constexpr uint32_t kProducts = 6, kProductA = 0x118, kProductB = 0x052;

template <int kMode>
struct ModeTraits {
  static constexpr bool scores = (kMode >= kModeScores && kMode <= kModeScoresTop32);
  static constexpr bool sweep = (kMode == kModeStats || scores || kMode == kModeDistill);   // units of vocabulary splits
  static constexpr bool dz_row = (kMode == kModeDzRow || kMode == kModeDzRow3);
  static constexpr bool dz = (kMode == kModeDz || dz_row);
  static constexpr bool dh = (kMode == kModeDHidden || kMode == kModeDHiddenPart);
  static constexpr bool dw = (kMode == kModeDW || kMode == kModeDWBf16);
  static constexpr bool out_bf16 = dz || kMode == kModeDWBf16;        // 64-column bf16 tiles through staging
  static constexpr bool out_f32 = (kMode == kModeDW || kMode == kModeDHiddenPart);   // 32-column float tiles
  static constexpr int top = kMode == kModeScoresTop8 ? 8 : (kMode == kModeScoresTop32 ? 32 : 0);
  static constexpr bool a_mn = dw;
  static constexpr bool b_mn = dh || dw;
  static constexpr bool wide = scores || kMode == kModeDistill;       // eight epilogue warps
  static constexpr bool two_groups = (dz_row || kMode == kModeDWBf16);   // two groups of four, 64 columns in turn
  static constexpr int epi_warps = wide || two_groups ? 8 : 4;
  static constexpr int threads = 64 + 32 * epi_warps;
  static constexpr int out_planes = kMode == kModeDzRow3 ? 3 : 1;
  static constexpr bool may_split = wide || kMode == kModeDzRow3 || kMode == kModeDHiddenPart || dw;   // float32 operands
  static constexpr int timing_kind = sweep ? 0 : (dz ? 1 : (dh ? 2 : 3));
};

template <int kMode, int kCta, int kAcc>
struct KAtoms { static constexpr int value = (kCta == 2 && kAcc == 1) ? 2 : 1; };

template <int kCta, int kAcc, int kKA>
struct PipeConfig {
  static constexpr uint32_t atom_bytes = kABytes + kAcc * kBBytes / kCta;
  static constexpr uint32_t stage_bytes = kKA * atom_bytes;
  static constexpr int stages = (int)(196608u / stage_bytes);
  static constexpr size_t smem_bytes = (size_t)stages * stage_bytes + 1024 + 2 * kOutStageBytes;
};
constexpr long long kWaitLimitCycles = 4000000000LL;   // about two seconds at the maximum SM clock

struct UmmaArgs {
  int M, N, K;              // extents of the contraction handled by this launch (valid elements)
  int m_tiles, n_tiles;     // ceil(M / rows per unit), ceil(N / columns per unit)
  int n_split;              // kModeStats: vocabulary splits; a unit is (token tile, split)
  int tiles_per_split;
  // kModeStats: split s owns the vocabulary tiles [s * split_stride, (s + 1) * split_stride); a launch sweeps the
  // tiles_per_split tiles of each split that start at offset tile_base inside it.  A whole sweep has tile_base = 0
  // and tiles_per_split = split_stride; a sweep cut into several launches (W still arriving) sets `resume` on
  // all but the first, and a row's running (max, sum, sum) then continues from `partials` exactly where the
  // launch before left it, so the cut does not change a bit of the result.
  int split_stride, tile_base, resume;
  int group_m;              // other modes: token tiles per raster group (tiles of a group run m-fastest)
  int a_mn0, a_k0;          // coordinate offsets of operand A in its tensor map (MN index, K index)
  int b_mn0, b_k0;
  int row0;                 // global token (or vocabulary row) index of accumulator row 0 of tile 0
  float kappa;
  const int* targets;
  const float* lse;
  const float* grad_coef;
  const float* grad_loss;
  float4* partials;         // kModeStats: [n_split][T_total]
  float* acc_y;             // kModeStats: raw accumulator at the target column, [T_total]
  int T_total;
  int dz_cols;              // kModeDz: columns of the panel written per row (>= N, zero beyond N); the panel
                            // itself is reached through the kernel's third tensor map
  __nv_bfloat16* d_hidden;  // kModeDHidden: [T][out_ld]
  float* d_W;               // kModeDW: [V][out_ld]
  size_t out_ld;
  int accumulate;
  int* status;
  int l2_a, l2_b;           // ptx::L2Hint of the loads of A and of B (CTA-pair kernels)
  const int* dyn_rows;      // optional device count of rows of the whole (compacted) batch: the launch then
  int dyn_base;             // covers rows [dyn_base, min(dyn_base + capacity, *dyn_rows)) of it (M, or K for d_W)
  // kModeScores*, kModeDistill: partials hold (m, r, u, -), m the maximum of the raw accumulators a, r = sum
  // 2^(c2 (a - m)) without the maximum's own 1, u = sum 2^(c2 (a - m)) c2 (a - m); two of them per split, of the left and
  // of the right halves of its tiles.  kModeScores*: targets may be NULL
  int top_k;                // entries of a row's list that are written
  float* top_val;           // [2 n_split][T_total][top_k] raw accumulators, falling; -inf where there are fewer
  int* top_id;              // [2 n_split][T_total][top_k]; -1 where there are fewer
  uint32_t* top_pub;        // [min(2 n_split, 32)][T_total], zero before the launch
  // kModeDistill
  int list_k;               // slots of a row's list
  const int* list_ids;      // [T_total][list_k] distinct ids in rising order, then INT_MAX
  float* list_z;            // [T_total][list_k] raw accumulators at those ids
  // kModeDzRow
  const float4* row_p;      // (m, log2 s, alpha, beta): L = c2 (a - m) - log2 s, dz = 2^L (alpha + beta L)
  const float* row_ins;     // dz at column targets[t]; read when targets is not NULL
  int row_flat;             // beta is zero in every row
  // float32 operands as planes: n_products is kProducts (else 0), plane q starts q * a_plane (b_plane, out_plane) columns
  // into a row (0 with one plane); K counts one plane
  int n_products;
  int a_plane, b_plane, out_plane;
  // kModeDHiddenPart: part s covers the k-blocks [s * part_blocks, (s + 1) * part_blocks) and writes rows
  // [s * part_rows, ...) of the output map; n_split parts
  int part_blocks, part_rows;
};

// Raster of the (m, n) output tiles for the modes without vocabulary splits: groups of `group_m`
// row tiles, m fastest inside a group, so that the CTAs running at one time share a few B tiles and
// keep the group's A tiles resident in L2 instead of streaming all of B once per row tile.
__device__ __forceinline__ void unit_to_tile(int unit, const UmmaArgs& args, int& m_tile, int& n_tile) {
  const int per_group = args.group_m * args.n_tiles;
  const int group = unit / per_group;
  const int first_m = group * args.group_m;
  const int rows = min(args.group_m, args.m_tiles - first_m);
  const int local = unit - group * per_group;
  m_tile = first_m + local % rows;
  n_tile = local / rows;
}

// Vocabulary tiles [n_begin, n_end) that this launch sweeps for split `split` (kModeStats); may be empty.
__device__ __forceinline__ void stats_tile_range(const UmmaArgs& args, int split, int& n_begin, int& n_end) {
  const int first = split * args.split_stride;
  n_begin = first + args.tile_base;
  n_end = min(min(n_begin + args.tiles_per_split, first + args.split_stride), args.n_tiles);
  if (n_end < n_begin) n_end = n_begin;
}

__device__ __forceinline__ float ex2f(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}

// raw[idx] for an index only known at run time, as a chain of predicated moves over registers.  Written
// as a plain select loop the compiler turns it into an indexed read, which puts the whole chunk in
// local memory: every accumulator then goes through a store and a load (128 bytes of stack per
// thread), and the statistics kernel loses a sixth of its rate.
__device__ __forceinline__ float pick_column(const uint32_t (&raw)[32], int idx) {
  uint32_t v = 0u;
#pragma unroll
  for (int j = 0; j < 32; ++j)
    asm volatile("{\n\t.reg .pred p;\n\tsetp.eq.s32 p, %1, %2;\n\t@p mov.b32 %0, %3;\n\t}"
                 : "+r"(v) : "r"(idx), "r"(j), "r"(raw[j]));
  return __uint_as_float(v);
}

// One 32-column chunk of a row folded into the running (m, s, u) with m the max of the raw
// accumulators a, s = sum 2^(c2 (a - m)) and u = sum 2^(c2 (a - m)) (a - m).  Keeping u relative to the
// max makes the entropy ln s - kappa u / s free of cancellation for sharply peaked rows, and the
// chunk's terms are summed among themselves before they meet the running totals, so 10^5 tiny
// terms are not lost one by one against a total near one.
template <bool kFull>
__device__ __forceinline__ void stats_chunk(const uint32_t (&raw)[32], int nvalid, float c2, float& run_m,
                                            float& run_s, float& run_u) {
  float cmax = -INFINITY;
#pragma unroll
  for (int j = 0; j < 32; ++j)
    if (kFull || j < nvalid) cmax = fmaxf(cmax, __uint_as_float(raw[j]));
  const float m_new = fmaxf(run_m, cmax);
  if (run_s > 0.f) {                                  // move the running sums to the new max
    const float d = run_m - m_new;                    // <= 0
    const float sc = ex2f(d * c2);
    run_u = sc * fmaf(d, run_s, run_u);
    run_s *= sc;
  }
  run_m = m_new;
  float s0 = 0.f, s1 = 0.f, u0 = 0.f, u1 = 0.f;       // two chains for instruction-level parallelism
#pragma unroll
  for (int j = 0; j < 32; j += 2) {
    if (kFull || j < nvalid) {
      const float t = __uint_as_float(raw[j]) - m_new;
      const float e = ex2f(t * c2);
      s0 += e;
      u0 = fmaf(e, t, u0);
    }
    if (kFull || j + 1 < nvalid) {
      const float t = __uint_as_float(raw[j + 1]) - m_new;
      const float e = ex2f(t * c2);
      s1 += e;
      u1 = fmaf(e, t, u1);
    }
  }
  run_s += s0 + s1;
  run_u += u0 + u1;
}

// The same by five levels of selects on the bits of idx: 31 instructions in five dependent steps instead of a
// chain of 32 (the chain needs no predicate registers beyond one, which the code around it may need).
__device__ __forceinline__ float pick_by_bits(const uint32_t (&raw)[32], int idx) {
  uint32_t a[16], b[8], c[4], d[2];
  const bool p4 = idx & 16, p3 = idx & 8, p2 = idx & 4, p1 = idx & 2, p0 = idx & 1;
#pragma unroll
  for (int j = 0; j < 16; ++j) a[j] = p4 ? raw[j + 16] : raw[j];
#pragma unroll
  for (int j = 0; j < 8; ++j) b[j] = p3 ? a[j + 8] : a[j];
#pragma unroll
  for (int j = 0; j < 4; ++j) c[j] = p2 ? b[j + 4] : b[j];
#pragma unroll
  for (int j = 0; j < 2; ++j) d[j] = p1 ? c[j + 2] : c[j];
  return __uint_as_float(p0 ? d[1] : d[0]);
}

// raw[idx] = -1e30 (kNoColumn), likewise for an index only known at run time.
__device__ __forceinline__ void drop_column(uint32_t (&raw)[32], int idx) {
#pragma unroll
  for (int j = 0; j < 32; ++j)
    asm volatile("{\n\t.reg .pred p;\n\tsetp.eq.s32 p, %1, %2;\n\t@p mov.b32 %0, 0fF149F2CA;\n\t}"
                 : "+r"(raw[j]) : "r"(idx), "r"(j));
}

__device__ __forceinline__ float2 fma2(float2 a, float2 b, float2 c) {
  float2 d;
  asm("{\n\t.reg .b64 ra, rb, rc, rd;\n\tmov.b64 ra, {%2, %3};\n\tmov.b64 rb, {%4, %5};\n\tmov.b64 rc, {%6, %7};\n\t"
      "fma.rn.f32x2 rd, ra, rb, rc;\n\tmov.b64 {%0, %1}, rd;\n\t}"
      : "=f"(d.x), "=f"(d.y) : "f"(a.x), "f"(a.y), "f"(b.x), "f"(b.y), "f"(c.x), "f"(c.y));
  return d;
}
__device__ __forceinline__ float2 add2(float2 a, float2 b) {
  float2 d;
  asm("{\n\t.reg .b64 ra, rb, rd;\n\tmov.b64 ra, {%2, %3};\n\tmov.b64 rb, {%4, %5};\n\t"
      "add.rn.f32x2 rd, ra, rb;\n\tmov.b64 {%0, %1}, rd;\n\t}"
      : "=f"(d.x), "=f"(d.y) : "f"(a.x), "f"(a.y), "f"(b.x), "f"(b.y));
  return d;
}
__device__ __forceinline__ float2 mul2(float2 a, float2 b) {
  float2 d;
  asm("{\n\t.reg .b64 ra, rb, rd;\n\tmov.b64 ra, {%2, %3};\n\tmov.b64 rb, {%4, %5};\n\t"
      "mul.rn.f32x2 rd, ra, rb;\n\tmov.b64 {%0, %1}, rd;\n\t}"
      : "=f"(d.x), "=f"(d.y) : "f"(a.x), "f"(a.y), "f"(b.x), "f"(b.y));
  return d;
}

// One 32-column chunk of dz = 2^L (alpha + beta L), L = c2 (a - m) - log2 s; zero at or beyond nvalid, and for a row that
// is not live (alpha = beta = 0) whatever its logits.  The difference to m is taken first: at a peaked row's maximum L is
// 10^-9, and the term is all there is to the row.
template <bool kFull>
__device__ __forceinline__ void dz_row_chunk(const uint32_t (&raw)[32], int nvalid, float c2, const float4& rp, bool live,
                                             uint32_t* packed) {
  const float2 cc = make_float2(c2, c2), nm = make_float2(-rp.x, -rp.x), ns = make_float2(-rp.y, -rp.y);
  const float2 aa = make_float2(rp.z, rp.z), bb = make_float2(rp.w, rp.w);
#pragma unroll
  for (int j = 0; j < 32; j += 2) {
    const float2 L = fma2(add2(make_float2(__uint_as_float(raw[j]), __uint_as_float(raw[j + 1])), nm), cc, ns);
    float2 v = mul2(make_float2(ex2f(L.x), ex2f(L.y)), fma2(bb, L, aa));
    if (!kFull && j >= nvalid) v.x = 0.f;
    if (!kFull && j + 1 >= nvalid) v.y = 0.f;
    __nv_bfloat162 h = __floats2bfloat162_rn(v.x, v.y);
    packed[j >> 1] = live ? *reinterpret_cast<uint32_t*>(&h) : 0u;
  }
}

// float32 operands: logits above this are the row's maximum itself, whatever the path that recomputes them.  The forward and
// the backward call may have taken different ones, whose logits differ by 10^-6, and at the maximum of a peaked row the
// gradient of an entropy is -e p (ln p + H) with ln p = -10^-8 (8 tokens x 2993, H 336: d_hidden 10^-5 off in all, 10^-6 with
// this).  Where the others add up to less than a quarter of the maximum, each is more than two powers of two below it.
__device__ __forceinline__ float snap_from(const float4& rp, float c2) {
  return rp.y < 0.32f ? rp.x - 1.f / c2 : INFINITY;
}

// The same as float32, in place of the logits.
__device__ __forceinline__ void dz_row_values(uint32_t (&raw)[32], int nvalid, float c2, const float4& rp, bool live) {
  const float from = snap_from(rp, c2);
#pragma unroll
  for (int j = 0; j < 32; ++j) {
    const float a = __uint_as_float(raw[j]);
    const float L = fmaf((a > from ? rp.x : a) - rp.x, c2, -rp.y);
    raw[j] = live && j < nvalid ? __float_as_uint(ex2f(L) * fmaf(rp.w, L, rp.z)) : 0u;
  }
}
// raw[idx] = x for an index only known at run time (see drop_column)
__device__ __forceinline__ void put_value(uint32_t (&raw)[32], int idx, float x) {
#pragma unroll
  for (int j = 0; j < 32; ++j)
    asm volatile("{\n\t.reg .pred p;\n\tsetp.eq.s32 p, %1, %2;\n\t@p mov.b32 %0, %3;\n\t}"
                 : "+r"(raw[j]) : "r"(idx), "r"(j), "f"(x));
}
// packed = the values rounded to bf16, raw = what that took off them
__device__ __forceinline__ void take_plane(uint32_t (&raw)[32], uint32_t* packed) {
#pragma unroll
  for (int j = 0; j < 32; j += 2) {
    const __nv_bfloat162 h = __floats2bfloat162_rn(__uint_as_float(raw[j]), __uint_as_float(raw[j + 1]));
    packed[j >> 1] = *reinterpret_cast<const uint32_t*>(&h);
    raw[j] = __float_as_uint(__uint_as_float(raw[j]) - __low2float(h));
    raw[j + 1] = __float_as_uint(__uint_as_float(raw[j + 1]) - __high2float(h));
  }
}

// One 32-column chunk of dz without its one-hot term: -coef * softmax = -sgn(coef) 2^(c2 a + k_row) with
// k_row = log2|coef| - lse log2(e), so an element costs one fused multiply-add and one exponential; the sign
// is applied to the packed bf16 pairs (sign_mask = 0x80008000 for coef > 0, else 0).  Columns at or beyond
// nvalid give zero, and so does a row with coef = 0 (k_row = -inf).
template <bool kFull>
__device__ __forceinline__ void dz_chunk(const uint32_t (&raw)[32], int nvalid, float c2, float k_row,
                                         uint32_t sign_mask, uint32_t* packed) {
#pragma unroll
  for (int j = 0; j < 32; j += 2) {
    float e0 = 0.f, e1 = 0.f;
    if (kFull || j < nvalid) e0 = ex2f(fmaf(__uint_as_float(raw[j]), c2, k_row));
    if (kFull || j + 1 < nvalid) e1 = ex2f(fmaf(__uint_as_float(raw[j + 1]), c2, k_row));
    __nv_bfloat162 h = __floats2bfloat162_rn(e0, e1);
    packed[j >> 1] = *reinterpret_cast<uint32_t*>(&h) ^ sign_mask;
  }
}

// packed[idx >> 1] with its half (idx & 1) replaced by the bf16 `half_bits`, for an index only known at run
// time; predicated moves over registers for the same reason as pick_column.
__device__ __forceinline__ void put_bf16(uint32_t (&packed)[32], int idx, uint32_t half_bits) {
  const int word = idx >> 1;
  const uint32_t keep = (idx & 1) ? 0x0000FFFFu : 0xFFFF0000u;
  const uint32_t ins = (idx & 1) ? (half_bits << 16) : half_bits;
#pragma unroll
  for (int j = 0; j < 32; ++j) {
    const uint32_t cand = (packed[j] & keep) | ins;
    asm volatile("{\n\t.reg .pred p;\n\tsetp.eq.s32 p, %1, %2;\n\t@p mov.b32 %0, %3;\n\t}"
                 : "+r"(packed[j]) : "r"(word), "r"(j), "r"(cand));
  }
}

// ------------------------------------------------------------------------------------------
// Epilogue of kModeScores* and kModeDistill: eight warps, two per quarter of the accumulator's rows, one taking
// the left and one the right half of a tile's columns (each has its own statistics and list of a row, merged
// afterwards like those of further vocabulary splits).  An element costs one exponential, and that unit gives a
// warp 32 results in eight cycles, 256 cycles a chunk of 32 columns; what else a chunk needs is kept below it with
// packed two-element arithmetic, and the second warp runs while the first waits for tensor memory or a branch.
// With four warps and scalar arithmetic a tile of 256 x 256 took 13400 cycles (8192 tokens x 32768 entries, H 512:
// 393 us), more than its contraction up to H = 1600.
// ------------------------------------------------------------------------------------------
// Stands for a column that does not count (beyond the vocabulary, or on a teacher's list): its exponential is zero
// and, unlike that of -inf, so is the product with its exponent.
constexpr float kNoColumn = -1e30f;

// 2^d for the residue d of a rounded exponent: next to one in float32 unless the scaled logits are in the ten thousands.
__device__ __forceinline__ float residue_ex2(float d) {
  return fabsf(d) < 4.8828125e-4f ? fmaf(d, 0.6931471805599453f, 1.f) : ex2f(d);     // d^2 ln(2)^2 / 2 < 2^-24
}

// Running statistics of a row: m the maximum of the raw accumulators, r = sum 2^(c2 a - ref) over all entries but ONE
// that equals m, u = sum 2^(c2 a - ref) (c2 a - ref).  Leaving the maximum's own 1 out keeps the relative precision of
// 1 - p and of the entropy in sharply peaked rows, where r is 10^-6 and would lose most of its digits beside a one.
// ref is c2 m rounded, so that an exponent is one fused multiply-add; delta is what the rounding took off, and
// finish() puts it back.
struct RestSums {
  float m = kNoColumn, ref = 0.f, delta = 0.f, r = 0.f, u = 0.f;

  // `raw` holds 32 numbers (kNoColumn among them), cmax their maximum.  A chunk of nothing but kNoColumn leaves m and ref
  // as they are: a reference of c2 kNoColumn would be off by its rounding, 10^22
  template <bool kEnt>
  __device__ __forceinline__ void fold(const uint32_t (&raw)[32], float cmax, float c2) {
    const bool risen = cmax > m;
    if (risen) {                                       // a few times per row: harmonic in the number of chunks
      const float ref_new = c2 * cmax;
      if (m > kNoColumn) {
        const float d = fmaxf(ref - ref_new, -1000.f), sc = ex2f(d);
        const float one = residue_ex2(delta);
        if (kEnt) u = sc * (fmaf(d, r + one, u) + one * delta);
        r = (r + one) * sc;
      }
      m = cmax;
      ref = ref_new;
      delta = fmaf(c2, cmax, -ref_new);
    }
    float2 s[4] = {}, v[4] = {};                       // independent chains: two warps a scheduler hide little latency
    const float2 cc = make_float2(c2, c2), nref = make_float2(-ref, -ref);
#pragma unroll
    for (int j = 0; j < 32; j += 8) {
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        const float2 t = fma2(make_float2(__uint_as_float(raw[j + 2 * q]), __uint_as_float(raw[j + 2 * q + 1])), cc, nref);
        const float2 e = make_float2(ex2f(t.x), ex2f(t.y));
        s[q] = add2(s[q], e);
        if (kEnt) v[q] = fma2(e, t, v[q]);
      }
    }
    s[0] = add2(add2(s[0], s[1]), add2(s[2], s[3]));
    float sum = s[0].x + s[0].y;
    if (risen) {
      // The new maximum's own 1 is in the sum.  Where the others are at least a quarter of it, taking it off costs
      // two of the chunk's 24 bits; where they are less the row may be a peaked one, and they are added without it.
      sum -= residue_ex2(delta);
      if (sum < 0.25f) {
        sum = -1.f;                                    // of the entries equal to m one does not count
#pragma unroll
        for (int j = 0; j < 32; ++j) {
          const float a = __uint_as_float(raw[j]);
          sum += a == m ? 1.f : 0.f;
        }
        sum *= residue_ex2(delta);
#pragma unroll
        for (int j = 0; j < 32; ++j) {
          const float a = __uint_as_float(raw[j]);
          sum += a == m ? 0.f : ex2f(fmaf(a, c2, -ref));
        }
      }
    }
    r += sum;
    if (kEnt) {
      v[0] = add2(add2(v[0], v[1]), add2(v[2], v[3]));
      u += (v[0].x + v[0].y) - (risen ? residue_ex2(delta) * delta : 0.f);
    }
  }
  // (m, r, u) relative to c2 m itself; a row of nothing but columns that do not count is (-inf, 0, 0)
  __device__ __forceinline__ float4 finish() const {
    if (!(m > kNoColumn)) return make_float4(-INFINITY, r != r ? r : 0.f, 0.f, 0.f);
    const float f = residue_ex2(-delta);
    return make_float4(m, r * f, fmaf(-delta, r, u) * f, 0.f);
  }
};

// The kTop largest entries of a row seen so far, falling; equal values in the order they came (columns are swept in
// rising order, so ties go to the lower id).  All indices are static, so the list stays in registers.  Entries that
// beat its last one wait in a queue of kQueue slots in shared memory and are inserted together when some
// lane's queue is full: a warp then pays for the most entries of a lane over many chunks, not in every chunk.
constexpr int kQueue = 16;
constexpr int kNoted = 4;
template <int kTop>
struct TopList {
  float val[kTop];
  int id[kTop];
  float best[kNoted];                                  // the largest group maxima, falling
  float bar;                                           // entries that do not exceed it are not wanted
  uint32_t queue, next;                                // shared-memory addresses of the lane's first and next free slot
  static constexpr uint32_t kSlot = 2048;              // bytes from a lane's slot to its next one (256 lanes x 8)
  __device__ __forceinline__ void clear(bool live) {
#pragma unroll
    for (int j = 0; j < kTop; ++j) { val[j] = -INFINITY; id[j] = -1; }
#pragma unroll
    for (int j = 0; j < kNoted; ++j) best[j] = -INFINITY;
    bar = live ? kNoColumn : INFINITY;
    next = queue;
  }
  __device__ __forceinline__ void insert(float x, int i) {
    bool above[kTop];
#pragma unroll
    for (int j = 0; j < kTop; ++j) above[j] = x > val[j];
#pragma unroll
    for (int j = kTop - 1; j > 0; --j) {
      val[j] = above[j - 1] ? val[j - 1] : (above[j] ? x : val[j]);
      id[j] = above[j - 1] ? id[j - 1] : (above[j] ? i : id[j]);
    }
    val[0] = above[0] ? x : val[0];
    id[0] = above[0] ? i : id[0];
  }
  // Notes a group's maximum for what the row's lists publish (see wide_sweep).  A group of NaN has none: min and max both
  // return the number beside a NaN, which would stand in `best` twice.
  __device__ __forceinline__ void note(float x) {
    x = fmaxf(x, -INFINITY);
#pragma unroll
    for (int j = 0; j < kNoted; ++j) {
      const float hi = fmaxf(best[j], x);
      x = fminf(best[j], x);
      best[j] = hi;
    }
  }
  // best[q] for a q only known at run time (see pick_column)
  __device__ __forceinline__ float noted(int q) const {
    float v = -INFINITY;
#pragma unroll
    for (int j = 0; j < kNoted; ++j)
      asm volatile("{\n\t.reg .pred p;\n\tsetp.eq.s32 p, %1, %2;\n\t@p mov.b32 %0, %3;\n\t}"
                   : "+f"(v) : "r"(q), "r"(j), "f"(best[j]));
    return v;
  }
  __device__ __forceinline__ void flush() {            // the whole warp
    const uint32_t end = queue + __reduce_max_sync(0xffffffffu, next - queue);
    for (uint32_t at = queue; at < end; at += kSlot) {
      float x = -INFINITY;
      int i = 0;
      if (at < next) asm volatile("ld.shared.v2.b32 {%0, %1}, [%2];" : "=f"(x), "=r"(i) : "r"(at) : "memory");
      if (__any_sync(0xffffffffu, x > bar)) insert(x > bar ? x : -INFINITY, i);
      bar = fmaxf(bar, val[kTop - 1]);
    }
    next = queue;
  }
  // One chunk, all lanes of a warp together.  A group of eight columns is looked at only where some lane's group
  // maximum is wanted; what it holds goes to the queues in straight-line code.
  __device__ __forceinline__ void fold(const uint32_t (&raw)[32], const float (&gmax)[4], float cmax, int col0, bool note_it) {
    if (!__any_sync(0xffffffffu, cmax > bar)) return;
#pragma unroll
    for (int g = 0; g < 4; ++g) {
      if (!__any_sync(0xffffffffu, gmax[g] > bar)) continue;
      if (__any_sync(0xffffffffu, next > queue + (kQueue - 8) * kSlot)) flush();
      if (note_it) note(gmax[g]);
#pragma unroll
      for (int j = 8 * g; j < 8 * g + 8; ++j)
        asm volatile("{\n\t.reg .pred p;\n\tsetp.gt.f32 p, %1, %2;\n\t@p st.shared.v2.b32 [%0], {%1, %3};\n\t@p add.u32 %0, %0, 2048;\n\t}"
                     : "+r"(next) : "f"(__uint_as_float(raw[j])), "f"(bar), "r"(col0 + j) : "memory");
    }
  }
};
template <>
struct TopList<0> {};

// Keys in the order of the values, for a word that several SMs write and read while they run; -inf is 0, "none".
__device__ __forceinline__ void publish_key(uint32_t* at, float x) {
  const uint32_t b = __float_as_uint(x + 0.f);
  const uint32_t key = x > -INFINITY ? ((b & 0x80000000u) ? ~b : (b | 0x80000000u)) : 0u;
  asm volatile("st.relaxed.gpu.global.u32 [%0], %1;" ::"l"(at), "r"(key) : "memory");
}
__device__ __forceinline__ uint32_t read_key(const uint32_t* at) {
  uint32_t key;
  asm volatile("ld.relaxed.gpu.global.u32 %0, [%1];" : "=r"(key) : "l"(at) : "memory");
  return key;
}
// The least of n keys that lie `stride` words apart.
__device__ __forceinline__ uint32_t least_key(const uint32_t* at, int n, int stride) {
  uint32_t least = 0xFFFFFFFFu;
  int j = 0;
  for (; j + 8 <= n; j += 8) {
    uint32_t key[8];
#pragma unroll
    for (int q = 0; q < 8; ++q) key[q] = read_key(at + (size_t)(j + q) * stride);
#pragma unroll
    for (int q = 0; q < 8; ++q) least = min(least, key[q]);
  }
  for (; j < n; ++j) least = min(least, read_key(at + (size_t)j * stride));
  return least;
}
// Maximum of the chunk's columns [8 g, 8 g + 8).
__device__ __forceinline__ float max_of_group(const uint32_t (&raw)[32], int g) {
  float m = __uint_as_float(raw[8 * g]);
#pragma unroll
  for (int j = 1; j < 8; ++j) m = fmaxf(m, __uint_as_float(raw[8 * g + j]));
  return m;
}
// The largest value below the one with this key; below zero that is a subnormal, not -0, which compares equal to it.
__device__ __forceinline__ float value_below(uint32_t key) {
  const uint32_t k = key == 0x80000000u ? key - 2u : key - 1u;
  return __uint_as_float((k & 0x80000000u) ? (k & 0x7FFFFFFFu) : ~k);
}

template <int kMode, int kCta>
__device__ __forceinline__ void wide_sweep(const UmmaArgs& args, int worker, int n_workers, int n_units, int cta_rank,
                                           uint32_t queues, uint32_t tmem_base, uint32_t bar_full, uint32_t bar_empty,
                                           volatile int* abort_p) {
  using namespace ptx;
  using Tr = ModeTraits<kMode>;
  constexpr bool kEnt = Tr::scores;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int quarter = warp & 3;                       // tensor-memory lanes 32 * quarter ..
  const int half = (warp - 2) >> 2;                   // columns 128 * half .. of a tile
  const float c2 = args.kappa * 1.4426950408889634f;
  [[maybe_unused]] TopList<Tr::top> list;
  if constexpr (Tr::top > 0) list.queue = queues + (threadIdx.x - 64) * 8;
  uint32_t acc_iter = 0;
  for (int unit = worker; unit < n_units; unit += n_workers) {
    const int m_tile = unit / args.n_split, split = unit % args.n_split;
    int n_begin, n_end;
    stats_tile_range(args, split, n_begin, n_end);
    const int row = (m_tile * kCta + cta_rank) * kBM + quarter * 32 + lane;
    const bool row_ok = row < args.M;
    const int grow = args.row0 + row;
    RestSums sums;
    int y = -1;
    if (Tr::scores && row_ok && args.targets != nullptr) {
      y = args.targets[grow];
      if (y < 0 || y >= args.N) {
        atomicOr(args.status, kStatusBadTarget);
        y = y < 0 ? 0 : args.N - 1;
      }
    }
    // What the row's lists have seen bounds its top from below: where each of n of them has q entries of x or more,
    // n q >= top_k, the row has top_k.  Every list publishes its q-th largest group maximum (as an ordered key, 0 for
    // none) and takes the least of the n published ones, in a unit's tiles 0, 1, 2, 4, 8, ... (between them the bound moves
    // little, and the words are a round trip to L2 away); in a unit's first tile the accumulators are read
    // once for their group maxima before they are read for their entries.  Lists of one row run side by side, so nearly
    // all entries that are only large for their own split stay out: with 18 lists of 8448 columns each and k = 32 a
    // list sees about 20 instead of 210.  n is no more than k: the least of 8 maxima is a better bound than the least of 32
    // (1537 tokens x 32768, H 1024, 20 lists of 8: 135 -> 123 us a call).  The keys only rise and an entry of the row's top is never below them,
    // so what the merge picks does not depend on when they are read.  (Few, long lists: q > kNoted, nothing published.)
    [[maybe_unused]] const int n_pub = max(1, min(min(2 * args.n_split, 32), args.top_k)), q_pub = (args.top_k + n_pub - 1) / n_pub;
    if constexpr (Tr::top > 0) list.clear(row_ok);
    [[maybe_unused]] int pos = 0, next_id = INT_MAX;  // kModeDistill: the next id of the row's list in this sweep
    [[maybe_unused]] const int* ids = nullptr;
    if (kMode == kModeDistill && row_ok) {
      ids = args.list_ids + (size_t)grow * args.list_k;
      int hi = args.list_k;
      while (pos < hi) {                              // first id at or behind the split's first column
        const int mid = (pos + hi) >> 1;
        if (ids[mid] < n_begin * kBN) pos = mid + 1; else hi = mid;
      }
      if (pos < args.list_k) next_id = ids[pos];
    }
    for (int n_tile = n_begin; n_tile < n_end; ++n_tile, ++acc_iter) {
      const uint32_t buf = acc_iter & 1u, buf_phase = (acc_iter >> 1) & 1u;
      // the warp gives up together: its tensor-memory loads are collective
      const bool ok = mbar_wait_bounded<true>(bar_full + buf * (uint32_t)sizeof(uint64_t), buf_phase, abort_p, kWaitLimitCycles);
      if (!__all_sync(0xffffffffu, ok)) return;
      tc_fence_after_sync();
      const uint32_t taddr = tmem_base + buf * kBN + half * 128 + ((uint32_t)(quarter * 32) << 16);
      const int first = n_tile * kBN + half * 128;
      if constexpr (Tr::top > 0) {
        if (q_pub <= kNoted) {
          if (n_tile == n_begin) {
#pragma unroll 1
            for (int c = 0; c < 4; ++c) {
              const int col0 = first + c * 32;
              if (col0 + 32 > args.N) break;          // a ragged chunk is left out of the bound
              uint32_t raw[32];
              tmem_ld_32x32(taddr + c * 32, raw);
              tmem_ld_wait();
#pragma unroll
              for (int g = 0; g < 4; ++g) list.note(max_of_group(raw, g));
            }
          }
          if (row_ok && ((n_tile - n_begin) & (n_tile - n_begin - 1)) == 0) {
            uint32_t* pub = args.top_pub + grow;
            const bool mine = 2 * split + half < n_pub;
            if (mine) publish_key(pub + (size_t)(2 * split + half) * args.T_total, list.noted(q_pub - 1));
            uint32_t least = least_key(pub, n_pub, args.T_total);
            // the lists of a row start together: the others' first words are worth a short wait (and only that, nothing
            // depends on them)
            if (n_tile == n_begin)
              for (int q = 0; q < 8 && least == 0u; ++q) {
                __nanosleep(100);
                least = least_key(pub, n_pub, args.T_total);
              }
            // entries that equal the bound may be needed (the lower id wins), those below it are not
            if (least != 0u) list.bar = fmaxf(list.bar, value_below(least));
          }
          __syncwarp();
        }
      }
#pragma unroll 1
      for (int c = 0; c < 4; ++c) {
        const int col0 = first + c * 32;
        if (col0 >= args.N) break;
        const int nvalid = min(32, args.N - col0);
        uint32_t raw[32];
        tmem_ld_32x32(taddr + c * 32, raw);
        tmem_ld_wait();
        if (nvalid < 32) {
#pragma unroll
          for (int j = 0; j < 32; ++j) raw[j] = j < nvalid ? raw[j] : __float_as_uint(kNoColumn);
        }
        if constexpr (kMode == kModeDistill) {
          while (next_id < col0 + 32) {               // INT_MAX: no more ids, or no row
            if (next_id >= col0) {                    // else the other half's
              args.list_z[(size_t)grow * args.list_k + pos] = pick_by_bits(raw, next_id - col0);
              drop_column(raw, next_id - col0);
            }
            ++pos;
            next_id = pos < args.list_k ? ids[pos] : INT_MAX;
          }
          __syncwarp();                               // the next tensor-memory load is the whole warp's
        }
        float gmax[4];
#pragma unroll
        for (int g = 0; g < 4; ++g) gmax[g] = max_of_group(raw, g);
        const float cmax = fmaxf(fmaxf(gmax[0], gmax[1]), fmaxf(gmax[2], gmax[3]));
        sums.fold<kEnt>(raw, cmax, c2);
        if constexpr (Tr::top > 0) {
          list.fold(raw, gmax, cmax, col0, n_tile > n_begin);
        }
        if (Tr::scores && y >= col0 && y < col0 + 32) args.acc_y[grow] = pick_by_bits(raw, y - col0);
        __syncwarp();
      }
      tc_fence_before_sync();
      __syncwarp();
      if (lane == 0) {
        const uint32_t bar = bar_empty + buf * (uint32_t)sizeof(uint64_t);
        if (kCta == 2) mbar_arrive_cluster(map_to_cta(bar, 0));
        else mbar_arrive(bar);
      }
    }
    const size_t at = (size_t)(2 * split + half) * args.T_total + grow;
    if constexpr (Tr::top > 0) {
      list.flush();
      if (row_ok) {
#pragma unroll
        for (int j = 0; j < Tr::top; ++j)
          if (j < args.top_k) { args.top_val[at * args.top_k + j] = list.val[j]; args.top_id[at * args.top_k + j] = list.id[j]; }
      }
    }
    if (row_ok) args.partials[at] = sums.finish();
  }
}

// kModeDHiddenPart: unit -> output tile and the k-blocks of its part (every part has some); else all k-blocks.
template <int kMode>
__device__ __forceinline__ int part_of_unit(int unit, int k_blocks, const UmmaArgs& args, int& kb_begin, int& kb_end) {
  if (kMode != kModeDHiddenPart) return unit;
  const int tiles = args.m_tiles * args.n_tiles, part = unit / tiles;
  kb_begin = part * args.part_blocks;
  kb_end = min(k_blocks, kb_begin + args.part_blocks);
  return unit - part * tiles;
}

template <int kMode, int kCta, int kAcc>
__global__ void __launch_bounds__(ModeTraits<kMode>::threads, 1)
umma_kernel(const __grid_constant__ CUtensorMap map_a, const __grid_constant__ CUtensorMap map_b,
            const __grid_constant__ CUtensorMap map_c, const UmmaArgs args_in) {
  using namespace ptx;
  UmmaArgs args = args_in;
  if (args.dyn_rows != nullptr) {
    // The number of rows is only known on the device (rows kept by the compaction of the backward):
    // this launch was sized for its capacity and shrinks itself to what is really there.
    int n = *args.dyn_rows - args.dyn_base;
    if (ModeTraits<kMode>::dw) {
      n = n < 0 ? 0 : (n > args.K ? args.K : n);
      args.K = n;
    } else {
      n = n < 0 ? 0 : (n > args.M ? args.M : n);
      args.M = n;
      args.m_tiles = (n + kBM * kCta - 1) / (kBM * kCta);
    }
  }
  constexpr int kKA = KAtoms<kMode, kCta, kAcc>::value;
  using Cfg = PipeConfig<kCta, kAcc, kKA>;
  using Tr = ModeTraits<kMode>;
  static_assert(kAcc == 1 || (kCta == 2 && (Tr::dh || Tr::dw)), "two accumulators: gradient modes, CTA pairs");
  constexpr int kBufs = 2 / kAcc;                          // tensor-memory buffers of kAcc accumulators
  constexpr int kUnitN = kBN * kAcc;                       // output columns per unit
  constexpr bool kPair = (kCta == 2);
  constexpr bool kAmn = Tr::a_mn;
  constexpr bool kBmn = Tr::b_mn;
  constexpr int kStagesT = Cfg::stages;
  constexpr int kBNcta = kBN / kCta;                       // rows of B that this CTA loads
  constexpr uint32_t kBBytesCta = kBNcta * kBK * 2;
  constexpr uint32_t kAtomBytesCta = kABytes + kAcc * kBBytesCta;
  constexpr uint32_t kStageBytesCta = kKA * kAtomBytesCta;
  extern __shared__ uint8_t smem_raw[];
  __shared__ __align__(8) uint64_t bar_full[kStagesT];
  __shared__ __align__(8) uint64_t bar_empty[kStagesT];
  __shared__ __align__(8) uint64_t bar_tmem_full[2];
  __shared__ __align__(8) uint64_t bar_tmem_empty[2];
  __shared__ uint32_t tmem_base_slot;
  __shared__ int abort_flag;

  const int warp = threadIdx.x >> 5;
  const int lane = threadIdx.x & 31;
  const uint32_t smem_base = (smem_u32(smem_raw) + 1023u) & ~1023u;
  volatile int* abort_p = &abort_flag;
  const int cta_rank = kPair ? (int)cluster_ctarank() : 0;   // 0 = the CTA that issues the pair's MMAs
  const int worker = kPair ? (int)(blockIdx.x >> 1) : (int)blockIdx.x;
  const int n_workers = kPair ? (int)(gridDim.x >> 1) : (int)gridDim.x;

  if (threadIdx.x == 0) {
    abort_flag = 0;
    for (int s = 0; s < kStagesT; ++s) {
      mbar_init(smem_u32(&bar_full[s]), 1);
      mbar_init(smem_u32(&bar_empty[s]), 1);
    }
    for (int b = 0; b < 2; ++b) {   // with kAcc = 2 only entry 0 is used
      mbar_init(smem_u32(&bar_tmem_full[b]), 1);
      mbar_init(smem_u32(&bar_tmem_empty[b]), Tr::epi_warps * kCta);   // one arrival per epilogue warp of every CTA
    }
    mbar_fence_init();
    fence_async_proxy();
  }
  if (warp == 0 && lane == 0) {
    prefetch_tensormap(&map_a);
    prefetch_tensormap(&map_b);
  }
  if (warp == 1) {
    if (kPair) {
      tmem_alloc_pair(smem_u32(&tmem_base_slot), kTmemCols);
      tmem_relinquish_pair();
    } else {
      tmem_alloc(smem_u32(&tmem_base_slot), kTmemCols);
      tmem_relinquish();
    }
  }
  tc_fence_before_sync();
  __syncthreads();
  if (kPair) cluster_sync_all();                           // the peer's barriers exist before anyone signals them
  tc_fence_after_sync();
  const uint32_t tmem_base = tmem_base_slot;

  const int k_blocks = (args.K + kBK * kKA - 1) / (kBK * kKA);
  const int n_units = (k_blocks == 0) ? 0
                      : Tr::sweep ? args.m_tiles * args.n_split
                      : (kMode == kModeDHiddenPart) ? args.m_tiles * args.n_tiles * args.n_split
                                                    : args.m_tiles * args.n_tiles;

  const int n_products = Tr::may_split && args.n_products > 1 ? args.n_products : 1;

  if (warp == 0) {
    // ------------------------------------------------------------------ TMA producer (every CTA)
    // One thread runs the whole loop: nothing in it needs the other lanes, and a warp-wide
    // rendezvous per k-block would sit on the critical path of the ring.
    if (lane == 0) {
      uint32_t stage = 0, phase = 0;
      uint32_t issued = 0;
      const uint32_t full0 = kPair ? map_to_cta(smem_u32(&bar_full[0]), 0) : smem_u32(&bar_full[0]);
      // which operand is worth keeping in L2: the hidden tile that a pair re-reads for every vocabulary
      // tile (statistics, dz), the slices of W / the hidden panel that every pair sweeps (d_hidden, d_W);
      // the dz stream of the gradient kernels is read by four pairs and then dead
      const uint64_t pol_a = make_l2_policy(args.l2_a);
      const uint64_t pol_b = make_l2_policy(args.l2_b);
      for (int unit = worker; unit < n_units; unit += n_workers) {
        int m_tile, n_begin, n_end, kb_begin = 0, kb_end = k_blocks;
        if (Tr::sweep) {
          m_tile = unit / args.n_split;
          stats_tile_range(args, unit % args.n_split, n_begin, n_end);
        } else {
          unit_to_tile(part_of_unit<kMode>(unit, k_blocks, args, kb_begin, kb_end), args, m_tile, n_begin);
          n_end = n_begin + 1;
        }
        const int a_row = args.a_mn0 + (m_tile * kCta + cta_rank) * kBM;
        for (int n_tile = n_begin; n_tile < n_end; ++n_tile) {
          const int b_row = args.b_mn0 + n_tile * kUnitN + cta_rank * kBNcta;   // + kBN per further accumulator
          for (int product = 0; product < n_products; ++product)
          for (int kb = kb_begin; kb < kb_end; ++kb) {
            if (!mbar_wait_bounded(smem_u32(&bar_empty[stage]), phase ^ 1u, abort_p, kWaitLimitCycles)) goto producer_drain;
            // a plane is a shift along the rows of the matrix, which hold k (K-major) or the operand's own index
            const int pa = Tr::may_split ? (int)((kProductA >> (2 * product)) & 3u) * args.a_plane : 0;
            const int pb = Tr::may_split ? (int)((kProductB >> (2 * product)) & 3u) * args.b_plane : 0;
            const uint32_t full = full0 + stage * (uint32_t)sizeof(uint64_t);
            if (kPair) {
              // both CTAs' bytes are counted on the issuing CTA's barrier, which alone is armed
              if (cta_rank == 0) mbar_arrive_expect_tx(smem_u32(&bar_full[stage]), 2 * kStageBytesCta);
            } else {
              mbar_arrive_expect_tx(full, kStageBytesCta);
            }
#pragma unroll
            for (int t = 0; t < kKA; ++t) {
              const uint32_t sa = smem_base + stage * kStageBytesCta + t * kAtomBytesCta;
              const uint32_t sb = sa + kABytes;
              const int ka = args.a_k0 + (kb * kKA + t) * kBK + (kAmn ? 0 : pa), a_mn = a_row + (kAmn ? pa : 0);
              const int kbb = args.b_k0 + (kb * kKA + t) * kBK + (kBmn ? 0 : pb), b_mn = b_row + (kBmn ? pb : 0);
              if (kPair) {
                if (kAmn) {
#pragma unroll
                  for (int j = 0; j < kBM / 64; ++j) tma_load_2d_pair(sa + j * kChunkBytes, &map_a, full, a_mn + j * 64, ka, pol_a);
                } else {
                  tma_load_2d_pair(sa, &map_a, full, ka, a_mn, pol_a);
                }
#pragma unroll
                for (int q = 0; q < kAcc; ++q) {
                  if (kBmn) {
#pragma unroll
                    for (int j = 0; j < kBNcta / 64; ++j)
                      tma_load_2d_pair(sb + q * kBBytesCta + j * kChunkBytes, &map_b, full, b_mn + q * kBN + j * 64, kbb, pol_b);
                  } else {
                    tma_load_2d_pair(sb + q * kBBytesCta, &map_b, full, kbb, b_mn + q * kBN, pol_b);
                  }
                }
              } else {
                if (kAmn) {
#pragma unroll
                  for (int j = 0; j < kBM / 64; ++j) tma_load_2d(sa + j * kChunkBytes, &map_a, full, a_mn + j * 64, ka);
                } else {
                  tma_load_2d(sa, &map_a, full, ka, a_mn);
                }
                if (kBmn) {
#pragma unroll
                  for (int j = 0; j < kBNcta / 64; ++j) tma_load_2d(sb + j * kChunkBytes, &map_b, full, b_mn + j * 64, kbb);
                } else {
                  tma_load_2d(sb, &map_b, full, kbb, b_mn);
                }
              }
            }
            ++issued;
            if (++stage == kStagesT) { stage = 0; phase ^= 1u; }
          }
        }
      }
      // tail: every slot this CTA filled has been released again, i.e. the MMAs that read this CTA's
      // shared memory are done and no release signal is still on its way to this CTA
      {
        const uint32_t n_tail = issued < (uint32_t)kStagesT ? issued : (uint32_t)kStagesT;
        for (uint32_t b = 0; b < n_tail; ++b) {
          if (!mbar_wait_bounded(smem_u32(&bar_empty[stage]), phase ^ 1u, abort_p, kWaitLimitCycles)) goto producer_drain;
          if (++stage == kStagesT) { stage = 0; phase ^= 1u; }
        }
      }
    producer_drain:
      if (*abort_p && cta_rank == 0) {
        // give the copies still in flight a bounded time to land before the block goes away
        const uint32_t n_back = issued < (uint32_t)kStagesT ? issued : (uint32_t)kStagesT;
        for (uint32_t b = 0; b < n_back; ++b) {
          if (stage == 0) { stage = kStagesT; phase ^= 1u; }
          --stage;
          const long long t0 = clock64();
          while (!mbar_try_wait(smem_u32(&bar_full[stage]), phase) && clock64() - t0 < 200000000LL) {
          }
        }
      }
    }
    __syncwarp();
  } else if (warp == 1) {
    // ------------------------------------------------------------------ MMA issuer (rank 0 of a pair)
    // One thread, and as little as possible between two tcgen05.mma: descriptors advance by
    // constants, and the barrier of the next stage is polled right after this stage's MMAs are
    // queued, so that its latency runs under them.
    if (cta_rank == 0 && lane == 0) {
      constexpr uint32_t idesc = make_idesc_bf16(kBM * kCta, kBN, kAmn ? 1 : 0, kBmn ? 1 : 0);
      // K-major: 16 elements = 32 bytes along the swizzled row; MN-major: 16 k-rows of 128 bytes
      constexpr uint64_t a_step = (kAmn ? kUmmaK * 128 : kUmmaK * 2) >> 4;
      constexpr uint64_t b_step = (kBmn ? kUmmaK * 128 : kUmmaK * 2) >> 4;
      constexpr uint64_t stage_step = kStageBytesCta >> 4;
      constexpr uint64_t atom_step = kAtomBytesCta >> 4;
      const uint64_t da_base = kAmn ? make_smem_desc(smem_base, kChunkBytes, 1024) : make_smem_desc(smem_base, 16, 1024);
      const uint64_t db_base = kBmn ? make_smem_desc(smem_base + kABytes, kChunkBytes, 1024)
                                    : make_smem_desc(smem_base + kABytes, 16, 1024);
      uint32_t stage = 0, phase = 0;
      uint32_t acc_iter = 0;
      bool ready = false;
      for (int unit = worker; unit < n_units; unit += n_workers) {
        int n_tiles_here = 1, kb_begin = 0, kb_end = k_blocks;
        if (Tr::sweep) {
          int n_begin, n_end;
          stats_tile_range(args, unit % args.n_split, n_begin, n_end);
          n_tiles_here = n_end - n_begin;
        } else {
          part_of_unit<kMode>(unit, k_blocks, args, kb_begin, kb_end);
        }
        for (int t = 0; t < n_tiles_here; ++t, ++acc_iter) {
          const uint32_t buf = acc_iter % kBufs;
          const uint32_t buf_phase = (acc_iter / kBufs) & 1u;
          if (!mbar_wait_bounded(smem_u32(&bar_tmem_empty[buf]), buf_phase ^ 1u, abort_p, kWaitLimitCycles)) goto mma_done;
          const uint32_t tmem_d = tmem_base + buf * kUnitN;
          for (int product = 0; product < n_products; ++product)
          for (int kb = kb_begin; kb < kb_end; ++kb) {
            const bool last = kb == kb_end - 1 && product == n_products - 1;
            if (!ready && !mbar_wait_bounded(smem_u32(&bar_full[stage]), phase, abort_p, kWaitLimitCycles)) goto mma_done;
            tc_fence_after_sync();
            const uint64_t da = da_base + stage * stage_step;
            const uint64_t db = db_base + stage * stage_step;
#pragma unroll
            for (int t = 0; t < kKA; ++t) {
#pragma unroll
              for (int q = 0; q < kAcc; ++q) {
#pragma unroll
                for (int k = 0; k < kBK / kUmmaK; ++k) {
                  const uint64_t daq = da + t * atom_step + k * a_step;
                  const uint64_t dbq = db + t * atom_step + q * (uint64_t)(kBBytesCta >> 4) + k * b_step;
                  const uint32_t acc = (product > 0 || kb > kb_begin || t > 0 || k > 0) ? 1u : 0u;
                  if (kPair) umma_bf16_pair(tmem_d + q * kBN, daq, dbq, idesc, acc);
                  else umma_bf16(tmem_d + q * kBN, daq, dbq, idesc, acc);
                }
              }
            }
            if (kPair) {
              umma_commit_pair(smem_u32(&bar_empty[stage]), 3);                        // frees the slot in both CTAs
              if (last) umma_commit_pair(smem_u32(&bar_tmem_full[buf]), 3);  // accumulator ready
            } else {
              umma_commit(smem_u32(&bar_empty[stage]));
              if (last) umma_commit(smem_u32(&bar_tmem_full[buf]));
            }
            if (++stage == kStagesT) { stage = 0; phase ^= 1u; }
            ready = mbar_try_wait(smem_u32(&bar_full[stage]), phase);
          }
        }
      }
    mma_done:;
    }
    __syncwarp();
  } else if constexpr (Tr::wide) {
    wide_sweep<kMode, kCta>(args, worker, n_workers, n_units, cta_rank, smem_base + kStagesT * kStageBytesCta, tmem_base,
                            smem_u32(&bar_tmem_full[0]), smem_u32(&bar_tmem_empty[0]), abort_p);
  } else {
    // ------------------------------------------------------------------ epilogue (warps 2..5, every CTA)
    const int quarter = warp & 3;                       // tensor-memory lanes 32 * quarter ..
    // two_groups: group 0 takes the even 64-column blocks of a tile, group 1 the odd ones, each through a staging tile
    // and a barrier of its own; what one waits for (tensor memory, its barriers, its last copy) the other fills
    const int group = Tr::two_groups ? (warp - 2) >> 2 : 0;
    const int row_in_tile = quarter * 32 + lane;
    const float c2 = args.kappa * 1.4426950408889634f;  // exp(kappa a) = 2^(c2 a)
    uint32_t acc_iter = 0;
    // The dz and d_W epilogues alternate between two staging tiles and only ever wait until at most ONE
    // tile copy is still reading shared memory, so the tile must be chosen by a count of the copies
    // issued that runs across accumulators and units: a last column tile that ends after an odd number
    // of copies would otherwise hand the next unit the tile whose copy is the one still in flight.
    uint32_t stage_iter = 0;
    for (int unit = worker; unit < n_units; unit += n_workers) {
      int m_tile, n_begin, n_end, split = 0;
      if (Tr::sweep) {
        m_tile = unit / args.n_split;
        split = unit % args.n_split;
        stats_tile_range(args, split, n_begin, n_end);
      } else {
        int kb_begin = 0, kb_end = 0;
        unit_to_tile(part_of_unit<kMode>(unit, k_blocks, args, kb_begin, kb_end), args, m_tile, n_begin);
        if (kMode == kModeDHiddenPart) split = unit / (args.m_tiles * args.n_tiles);
        n_end = n_begin + 1;
      }
      const int row = (m_tile * kCta + cta_rank) * kBM + row_in_tile;   // row within this launch's M extent
      const bool row_ok = row < args.M;
      const int grow = args.row0 + row;                 // global token / vocabulary row

      // per-row state
      float run_m = -INFINITY, run_s = 0.f, run_u = 0.f;
      int y = -1;
      float coef = 0.f, lse2 = 0.f;
      if (kMode == kModeStats || kMode == kModeDz || (Tr::dz_row && args.targets != nullptr)) {
        if (row_ok) {
          y = args.targets[grow];
          if (y < 0 || y >= args.N) {
            if (kMode == kModeStats) atomicOr(args.status, kStatusBadTarget);
            y = y < 0 ? 0 : args.N - 1;
          }
        }
      }
      if (kMode == kModeStats && args.resume && row_ok) {  // continue the sweep the launch before left off
        const float4 p = args.partials[(size_t)split * args.T_total + grow];
        run_m = p.x; run_s = p.y; run_u = p.z;
      }
      [[maybe_unused]] float4 rp = make_float4(0.f, 0.f, 0.f, 0.f);   // kModeDzRow, kModeDzRow3
      [[maybe_unused]] float ins = 0.f;
      if (Tr::dz_row && row_ok) {
        rp = args.row_p[grow];
        if (args.targets != nullptr) ins = args.row_ins[grow];
      }
      float k_row = -INFINITY;                          // kModeDz: log2|coef| - lse log2(e); -inf gives a zero row
      uint32_t sign_mask = 0u;
      if (kMode == kModeDzRow && row_ok) {
        if (rp.z != 0.f) k_row = log2f(fabsf(rp.z)) - fmaf(rp.x, c2, rp.y);
        sign_mask = rp.z < 0.f ? 0x80008000u : 0u;
      }
      // beta = 0: alpha goes into the exponent, c2 a + k_row.  What rounding takes off k_row is a factor that a row's entries
      // share, so unlike their rounding to bf16 it does not average out: for |c2 m| up to 64 (logits up to 44, those of
      // trained heads) it is at most 2^-17, next to what the row's statistics carry; beyond, the difference to m is taken first.
      // (One form for a warp's rows; rows without a gradient, padding among them, have no say.)
      [[maybe_unused]] bool flat = false;
      if (kMode == kModeDzRow) flat = args.row_flat && !__any_sync(0xffffffffu, rp.z != 0.f && fabsf(rp.x * c2) > 64.f);
      if (kMode == kModeDz) {
        if (row_ok) {
          const float gl = args.grad_loss ? *args.grad_loss : 1.f;
          coef = args.kappa * gl * args.grad_coef[grow];
          lse2 = args.lse[grow] * 1.4426950408889634f;
          if (coef != 0.f) k_row = log2f(fabsf(coef)) - lse2;
          sign_mask = coef > 0.f ? 0x80008000u : 0u;
        }
      }

      for (int n_tile = n_begin; n_tile < n_end; ++n_tile, ++acc_iter) {
        const uint32_t buf = acc_iter % kBufs;
        const uint32_t buf_phase = (acc_iter / kBufs) & 1u;
        const int col_base = n_tile * kUnitN;
        // The give-up decision is taken by the 128 epilogue threads together: a thread that saw the wait
        // complete while another saw the abort flag would otherwise go on alone to warp-wide tensor-memory
        // loads and to the epilogue barrier, which the others never reach.
        const bool arrived = mbar_wait_bounded<true>(smem_u32(&bar_tmem_full[buf]), buf_phase, abort_p, kWaitLimitCycles);
        if (!(Tr::two_groups ? epilogue_group_all(group, arrived) : epilogue_all(arrived))) goto role_done;
        tc_fence_after_sync();
        const uint32_t taddr = tmem_base + buf * kUnitN + ((uint32_t)(quarter * 32) << 16);
        if (Tr::out_bf16) {
          // 64 columns (one 128-byte row of bf16) at a time: two accumulator chunks -> packed registers ->
          // swizzled staging tile in shared memory -> one TMA store of 128 rows x 128 bytes, so that the
          // panel is written in whole lines by the copy engine instead of 16 bytes a thread
          const int tile_row = (m_tile * kCta + cta_rank) * kBM;
          const bool issuer = (threadIdx.x == 64 + 128 * group);   // first thread of the epilogue warps (of the group)
#pragma unroll 1
          for (int g = group; g < kUnitN / 64; g += Tr::two_groups ? 2 : 1) {
            const int col0 = col_base + g * 64;
            if (col0 >= args.dz_cols) break;
            uint32_t raw0[32], raw1[32];
            tmem_ld_32x32(taddr + g * 64, raw0);
            tmem_ld_32x32(taddr + g * 64 + 32, raw1);
            tmem_ld_wait();
            uint32_t packed[32];
            const int nv0 = args.N - col0, nv1 = args.N - col0 - 32;
            if (kMode == kModeDz) {
              if (nv0 >= 32) dz_chunk<true>(raw0, 32, c2, k_row, sign_mask, packed);
              else dz_chunk<false>(raw0, nv0, c2, k_row, sign_mask, packed);
              if (nv1 >= 32) dz_chunk<true>(raw1, 32, c2, k_row, sign_mask, packed + 16);
              else dz_chunk<false>(raw1, nv1, c2, k_row, sign_mask, packed + 16);
            } else if (kMode == kModeDzRow) {
              if (flat) {
                if (nv0 >= 32) dz_chunk<true>(raw0, 32, c2, k_row, sign_mask, packed);
                else dz_chunk<false>(raw0, nv0, c2, k_row, sign_mask, packed);
                if (nv1 >= 32) dz_chunk<true>(raw1, 32, c2, k_row, sign_mask, packed + 16);
                else dz_chunk<false>(raw1, nv1, c2, k_row, sign_mask, packed + 16);
                if (rp.z == 0.f) {
#pragma unroll
                  for (int j = 0; j < 32; ++j) packed[j] = 0u;
                }
              } else {
                const bool live = rp.z != 0.f || rp.w != 0.f;
                if (nv0 >= 32) dz_row_chunk<true>(raw0, 32, c2, rp, live, packed);
                else dz_row_chunk<false>(raw0, nv0, c2, rp, live, packed);
                if (nv1 >= 32) dz_row_chunk<true>(raw1, 32, c2, rp, live, packed + 16);
                else dz_row_chunk<false>(raw1, nv1, c2, rp, live, packed + 16);
              }
              if (row_ok && y >= col0 && y < col0 + 64) {
                const __nv_bfloat16 hv = __float2bfloat16_rn(ins);
                put_bf16(packed, y - col0, (uint32_t)(*reinterpret_cast<const uint16_t*>(&hv)));
              }
            } else if (kMode == kModeDzRow3) {                 // float32 values in place of the logits
              const bool live = rp.z != 0.f || rp.w != 0.f;
              dz_row_values(raw0, nv0, c2, rp, live);
              dz_row_values(raw1, nv1, c2, rp, live);
              if (row_ok && y >= col0 && y < col0 + 32) put_value(raw0, y - col0, ins);
              if (row_ok && y >= col0 + 32 && y < col0 + 64) put_value(raw1, y - col0 - 32, ins);
            } else {                                           // kModeDWBf16
#pragma unroll
              for (int j = 0; j < 32; j += 2) {
                __nv_bfloat162 h0 = __floats2bfloat162_rn(__uint_as_float(raw0[j]), __uint_as_float(raw0[j + 1]));
                __nv_bfloat162 h1 = __floats2bfloat162_rn(__uint_as_float(raw1[j]), __uint_as_float(raw1[j + 1]));
                packed[j >> 1] = *reinterpret_cast<uint32_t*>(&h0);
                packed[16 + (j >> 1)] = *reinterpret_cast<uint32_t*>(&h1);
              }
            }
            if (kMode == kModeDz && row_ok && y >= col0 && y < col0 + 64) {        // the one-hot term: coef (1 - p_y) at the target column
              const int idx = y - col0;
              const float ay = idx < 32 ? pick_column(raw0, idx) : pick_column(raw1, idx - 32);
              const float vy = coef * (1.f - ex2f(fmaf(ay, c2, -lse2)));
              const __nv_bfloat16 hv = __float2bfloat16_rn(vy);
              put_bf16(packed, idx, (uint32_t)(*reinterpret_cast<const uint16_t*>(&hv)));
            }
#pragma unroll 1
            for (int plane = 0; plane < Tr::out_planes; ++plane) {
            if (Tr::out_planes > 1) {                          // the next plane: the values rounded, and what that left
              take_plane(raw0, packed);
              take_plane(raw1, packed + 16);
            }
            const uint32_t out_buf =
                smem_base + kStagesT * kStageBytesCta + (Tr::two_groups ? (uint32_t)group : (stage_iter++ & 1u)) * kOutStageBytes;
            if (issuer) {                                      // the copy that last read this staging tile is done with it
              if (Tr::two_groups) bulk_wait_read_all();
              else bulk_wait_read_le1();
            }
            if (Tr::two_groups) epilogue_group_sync(group);
            else epilogue_bar_sync();
            const uint32_t row_addr = out_buf + (uint32_t)row_in_tile * 128u;
#pragma unroll
            for (int q = 0; q < 8; ++q) {
              const uint32_t dst = row_addr + ((uint32_t)(q ^ (row_in_tile & 7)) << 4);
              asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(dst), "r"(packed[4 * q]), "r"(packed[4 * q + 1]),
                           "r"(packed[4 * q + 2]), "r"(packed[4 * q + 3])
                           : "memory");
            }
            fence_async_proxy();
            if (Tr::two_groups) epilogue_group_sync(group);
            else epilogue_bar_sync();
            if (issuer) {
              // rows past the panel's capacity (d_W: past the vocabulary) are clipped
              if (Tr::dz || tile_row < args.M) tma_store_2d(&map_c, out_buf, col0 + plane * args.out_plane, (Tr::dz ? 0 : args.row0) + tile_row);
              bulk_commit_group();
            }
            }
          }
        }
#pragma unroll 1
        for (int c = 0; !Tr::out_bf16 && c < kUnitN / 32; ++c) {
          const int col0 = col_base + c * 32;
          if (col0 >= args.N) break;                           // whole chunk beyond the valid columns
          const int nvalid = min(32, args.N - col0);
          uint32_t raw[32];
          tmem_ld_32x32(taddr + c * 32, raw);
          tmem_ld_wait();

          if (kMode == kModeStats) {
            if (nvalid >= 32) stats_chunk<true>(raw, 32, c2, run_m, run_s, run_u);
            else stats_chunk<false>(raw, nvalid, c2, run_m, run_s, run_u);
            if (row_ok && y >= col0 && y < col0 + 32) {
              args.acc_y[grow] = pick_column(raw, y - col0);
            }
          } else if (kMode == kModeDHidden) {
            if (row_ok) {
              uint32_t packed[16];
#pragma unroll
              for (int j = 0; j < 32; j += 2) {
                __nv_bfloat162 h = __floats2bfloat162_rn(__uint_as_float(raw[j]), __uint_as_float(raw[j + 1]));
                packed[j >> 1] = *reinterpret_cast<uint32_t*>(&h);
              }
              uint4* dst = reinterpret_cast<uint4*>(args.d_hidden + (size_t)grow * args.out_ld + col0);
#pragma unroll
              for (int q = 0; q < 4; ++q)
                if (q * 8 < nvalid) dst[q] = make_uint4(packed[4 * q], packed[4 * q + 1], packed[4 * q + 2], packed[4 * q + 3]);
            }
          } else {  // kModeDW, kModeDHiddenPart: swizzled staging tile, then one TMA store (first panel) or reduce-add
            const uint32_t out_buf = smem_base + kStagesT * kStageBytesCta + (stage_iter++ & 1u) * kOutStageBytes;
            const bool issuer = (threadIdx.x == 64);             // first thread of the epilogue warps
            if (issuer) bulk_wait_read_le1();                    // the copy that last read this tile is done with it
            epilogue_bar_sync();
            const uint32_t row_addr = out_buf + (uint32_t)row_in_tile * 128u;
#pragma unroll
            for (int q = 0; q < 8; ++q) {
              const uint32_t dst = row_addr + ((uint32_t)(q ^ (row_in_tile & 7)) << 4);
              asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(dst), "r"(raw[4 * q]), "r"(raw[4 * q + 1]),
                           "r"(raw[4 * q + 2]), "r"(raw[4 * q + 3])
                           : "memory");
            }
            fence_async_proxy();
            epilogue_bar_sync();
            if (issuer) {
              const int tile_row = (m_tile * kCta + cta_rank) * kBM;      // rows past M never reach memory
              if (kMode == kModeDHiddenPart) {                             // rows past M: padding of the part
                tma_store_2d(&map_c, out_buf, col0, split * args.part_rows + tile_row);
              } else if (tile_row < args.M) {
                if (args.accumulate) tma_reduce_add_2d(&map_c, out_buf, col0, args.row0 + tile_row);
                else tma_store_2d(&map_c, out_buf, col0, args.row0 + tile_row);
              }
              bulk_commit_group();
            }
          }
        }
        // accumulator drained: hand the buffer back to the MMA warp (of rank 0)
        tc_fence_before_sync();
        __syncwarp();
        if (lane == 0) {
          if (kPair) mbar_arrive_cluster(map_to_cta(smem_u32(&bar_tmem_empty[buf]), 0));
          else mbar_arrive(smem_u32(&bar_tmem_empty[buf]));
        }
      }

      if (kMode == kModeStats && row_ok)
        args.partials[(size_t)split * args.T_total + grow] = make_float4(run_m, run_s, run_u, 0.f);
    }
  }

[[maybe_unused]] role_done:
  if ((Tr::out_bf16 || Tr::out_f32) && (threadIdx.x == 64 || (Tr::two_groups && threadIdx.x == 192))) bulk_wait_all();   // the tile copies have left shared memory and landed
  if (*abort_p && lane == 0) atomicOr(args.status, kStatusTimeout);
  tc_fence_before_sync();
  __syncthreads();
  if (kPair) cluster_sync_all();       // neither CTA leaves while the other may still signal its barriers
  if (warp == 1) {
    tc_fence_after_sync();
    if (kPair) tmem_dealloc_pair(tmem_base, kTmemCols);
    else tmem_dealloc(tmem_base, kTmemCols);
  }
}

// The bounded wait on its own: one block, one mbarrier on which nobody ever arrives, no copy and no tensor
// memory in flight.  The wait gives up after limit_cycles, the kernel records the timeout in the status word
// and returns normally -- the way umma_kernel reports a stall, exercised without stalling anything.
__global__ void bounded_wait_selftest_kernel(long long limit_cycles, int* status) {
  __shared__ __align__(8) uint64_t bar;
  __shared__ int abort_flag;
  if (threadIdx.x == 0) {
    abort_flag = 0;
    ptx::mbar_init(ptx::smem_u32(&bar), 1);
    ptx::mbar_fence_init();
  }
  __syncthreads();
  if (threadIdx.x == 0) {
    volatile int* abort_p = &abort_flag;
    const bool done = ptx::mbar_wait_bounded(ptx::smem_u32(&bar), 0u, abort_p, limit_cycles);
    if (!done) atomicOr(status, kStatusTimeout);
  }
}

}  // namespace ulorl
