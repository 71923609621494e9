// Host side of token scoring and distillation (included by ulorl_api.cu): validation, workspace, launches.
#pragma once

#include "scores.cuh"
#include "sgemm.cuh"
#include "small_batch.cuh"

namespace ulorl {

constexpr int kHeadMaxSplits = kMaxRowLists / 2;   // a split leaves two partial results of a row

struct HeadPlan {
  bool tensor;
  int planes;                              // tensor path: 1, or 3 for float32 operands (bf16 planes)
  int width;                               // columns of a plane of hidden and of W (H with one plane)
  bool small;                              // tensor path, few tokens: the forward calls go through a panel of logits
  int sms, workers;                        // workers: CTA pairs
  int n_split, tiles_per_split;            // vocabulary splits of the forward sweep
  int n_partial;                           // partial results of a row that it leaves
  int panel_tokens, n_panels;
  size_t dz_ld, logits_ld;
  bool dw_direct;                          // d_W leaves the contraction as bf16: one panel, nothing to add to
  bool dw_acc;                             // d_W summed in float32 in the workspace, rounded at the end
  int dh_acc, dw_acc_tiles;                // accumulators per unit of the two gradient contractions
  int dh_parts, dh_part_blocks, dh_part_rows;
  // forward scratch
  size_t off_status, off_partials, off_acc_y, off_top_val, off_top_id, off_top_pub, off_sorted, off_slots, off_list_z, off_logits, off_planes, fwd_total;
  // backward scratch, over the same bytes
  size_t off_row_p, off_row_ins, off_panel, off_dw_acc, off_parts, off_planes_bwd, bwd_total;
};

static bool aligned8(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 7u) == 0; }

// A column that does not count stands at -1e30: times the scale that has to be far below every exponent, and finite.
static bool scale_supported(float inv_temperature) { return inv_temperature >= 1e-6f && inv_temperature <= 1e6f; }
constexpr int kHeadMaxSize = 1 << 30;              // sizes rounded up to a tile stay within int

// float32 operands as three planes side by side: columns stay within int
static bool split_possible(const ulorl_head_params_t* p) { return p->H <= kHeadMaxSize / 2 && p->V <= kHeadMaxSize / 2; }

static int validate_head(const ulorl_head_params_t* p) {
  if (!p) return ULORL_ERR_INVALID_ARG;
  if (p->T < 0 || p->H <= 0 || p->V <= 0 || p->top_k < 0) return ULORL_ERR_INVALID_ARG;
  if (p->dtype != ULORL_F32 && p->dtype != ULORL_BF16) return ULORL_ERR_UNSUPPORTED;
  if (p->dw_dtype != ULORL_F32 && p->dw_dtype != ULORL_BF16) return ULORL_ERR_INVALID_ARG;
  if (p->kernel_path < ULORL_PATH_AUTO || p->kernel_path > ULORL_PATH_TENSOR_1CTA) return ULORL_ERR_INVALID_ARG;
  if (p->kernel_path == ULORL_PATH_TENSOR_1CTA) return ULORL_ERR_UNSUPPORTED;
  if (!(p->inv_temperature > 0.f) || !std::isfinite(p->inv_temperature)) return ULORL_ERR_INVALID_ARG;
  if (!scale_supported(p->inv_temperature)) return ULORL_ERR_UNSUPPORTED;
  if (p->T > kHeadMaxSize || p->H > kHeadMaxSize || p->V > kHeadMaxSize) return ULORL_ERR_UNSUPPORTED;
  if (!(p->teacher_inv_temperature > 0.f) || !std::isfinite(p->teacher_inv_temperature)) return ULORL_ERR_INVALID_ARG;
  if (p->distill_mode < ULORL_DISTILL_RAW || p->distill_mode > ULORL_DISTILL_TAIL) return ULORL_ERR_INVALID_ARG;
  if (p->distill_mode != ULORL_DISTILL_RENORM && p->teacher_inv_temperature != 1.f) return ULORL_ERR_INVALID_ARG;
  if (p->norm_tokens < 0 || p->bwd_panel_tokens < 0) return ULORL_ERR_INVALID_ARG;
  if (p->dw_accumulate != 0 && p->dw_accumulate != 1) return ULORL_ERR_INVALID_ARG;
  if (p->kernel_path == ULORL_PATH_TENSOR && p->dtype == ULORL_F32 && !split_possible(p)) return ULORL_ERR_UNSUPPORTED;
  if (p->top_k > ULORL_MAX_LIST) return ULORL_ERR_UNSUPPORTED;
  if (p->H % 8 != 0) return ULORL_ERR_UNSUPPORTED;
  return ULORL_OK;
}

// Parts over k of an M x N float32 contraction: as many as there are multiprocessors for, 256 values of k or more each.
static int sgemm_parts(const HeadPlan& pl, int M, int N, int K, int* k_part) {
  const long tiles = (long)((M + kSgTile - 1) / kSgTile) * ((N + kSgTile - 1) / kSgTile);
  long parts = std::max(1L, std::min(pl.sms / std::max(1L, tiles), (long)K / 256));
  *k_part = (int)align_up((size_t)((K + parts - 1) / parts), kSgK);
  return (K + *k_part - 1) / *k_part;
}

// Whether float32 operands go through the tensor cores: six products of bf16 planes against CUDA-core multiply-adds.
// Modelled microseconds of a forward call per 10^6 of V x H, and what the planes cost a small one (measured 39 us for 43 at
// 512 tokens x 4096, H 256; 31 for 29 at 512 x 1000, H 128; 199 for 254 at 1 x 32768, H 1024; 209 for 881 at 512 tokens).
// V x H counts columns as they are, planes are padded to a multiple of 128: at H 64 and below the tensor path does twice the work
// and more of what is modelled here.
static bool split_pays(const ulorl_head_params_t* p, bool backward) {
  if (!split_possible(p)) return false;
  const double vh = 1e-6 * (double)p->V * (double)p->H;
  if (backward) return vh > 0.02;          // three contractions (1 token, H 64: 38 us for 55 at V 1000; H 8, V 100: 33 for 24)
  const double simt = 6.9 * vh * ((p->T + 127) / 128);
  const double tensor = (2.4 * ((p->T + 255) / 256) + 2.0) * vh + 17.0;
  return simt > tensor;
}

// float32 operands: tokens of a panel by default; and tokens (vocabulary entries) that one accumulator of d_W (of d_hidden)
// adds up, the sums of several being added in float32 afterwards.  The tensor core cuts off a sum's last bits, mostly one
// way: an error that grows with the length (d_W of 1024 tokens 1.3e-6 off in one sum, 6.5e-7 in two).  Panels of 512
// tokens would do for d_W, but leave d_hidden few units (2048 tokens x 32768, H 2048: 4.5 ms instead of 3.6).
constexpr int kSplitPanel = 2048, kSplitTokens = 512, kSplitEntries = 2048;

static HeadPlan make_head_plan(const ulorl_head_params_t* p, bool backward) {
  HeadPlan pl{};
  pl.planes = p->dtype == ULORL_F32 ? 3 : 1;
  pl.tensor = p->kernel_path == ULORL_PATH_TENSOR ||
              (p->kernel_path != ULORL_PATH_SIMT && (p->dtype == ULORL_BF16 || split_pays(p, backward)));
  pl.width = pl.planes == 3 ? (int)align_up((size_t)p->H, 2 * kBK) : p->H;
  pl.sms = device_sm_count();
  pl.workers = std::max(1, pl.sms / 2);
  const int T = p->T, V = p->V, H = p->H;
  pl.small = pl.tensor && pl.planes == 1 && T <= kSmallMaxTokens;
  const size_t T1 = (size_t)std::max(T, 1), K = (size_t)p->top_k;
  const int tile_m = 2 * kBM;
  const int m_tiles = std::max(1, (T + tile_m - 1) / tile_m);
  const int n_tiles = (V + kBN - 1) / kBN;
  pl.n_split = 1;
  pl.tiles_per_split = n_tiles;
  if (pl.tensor && !pl.small) {
    // As for the policy loss: enough splits that the live hidden tiles stay in L2, then the count with the shortest
    // modelled time, waves of units x time of a unit, the fewest splits within one percent.  A unit's time is that
    // of its tiles, contraction (8 H cycles a tile) or epilogue, whichever is longer, and, with alternatives, that of
    // its first tiles, where the lists fill faster than the contraction hides (two accumulators are not enough of a
    // cushion): measured 12000 cycles a unit with lists of 8, 105000 with lists of 32 (8192 tokens x 151936, H 2048,
    // 30 splits: 4.47, 4.62 and 5.84 million cycles without alternatives, with 8 and with 32).  Without lists every further
    // split is still a pass over W more: 4.52 ms with 30 splits, 3.8 with 9, under the power cap.
    const int list = p->top_k <= 0 || p->top_k > kMaxTop ? 0 : (p->top_k <= 8 ? 8 : kMaxTop);
    const double contraction = 8.0 * (pl.planes == 3 ? kProducts * pl.width : H);
    const double tile = std::max(contraction, list == 0 ? 5300.0 : (list == 8 ? 6000.0 : 7000.0));
    const double fill = list == 0 ? 10000.0 : (list == 8 ? 12000.0 : 105000.0);
    const size_t live_bytes = (size_t)pl.workers * (size_t)tile_m * (size_t)(pl.planes * pl.width) * 2;
    const int s_max = std::min(kHeadMaxSplits, n_tiles);
    const int s_min = std::max(1, std::min((int)((live_bytes + kStatsHiddenBudget - 1) / kStatsHiddenBudget), s_max));
    auto cost_of = [&](int s) {
      const int tps = (n_tiles + s - 1) / s;
      const int s_eff = (n_tiles + tps - 1) / tps;
      const double unit = tps * tile + fill;
      return (double)(((long)m_tiles * s_eff + pl.workers - 1) / pl.workers) * unit;
    };
    double best = cost_of(s_min);
    for (int s = s_min + 1; s <= s_max; ++s) best = std::min(best, cost_of(s));
    int want = s_min;
    while (want < s_max && cost_of(want) > best * 1.01) ++want;
    pl.tiles_per_split = (n_tiles + want - 1) / want;
    pl.n_split = (n_tiles + pl.tiles_per_split - 1) / pl.tiles_per_split;
  }
  pl.n_partial = pl.tensor && !pl.small ? 2 * pl.n_split : 1;
  // backward panels
  int panel = p->bwd_panel_tokens > 0 ? p->bwd_panel_tokens : (!pl.tensor ? kDefaultPanelSimt : (pl.planes == 3 ? kSplitPanel : pl.workers * tile_m));
  if (!pl.tensor) panel = std::min(panel, 32768);                   // rows are a grid dimension there
  const int unit = pl.tensor ? tile_m : kSimtTile;
  panel = (int)std::min<long>((long)align_up((size_t)panel, (size_t)unit), (long)align_up(T1, (size_t)unit));
  pl.panel_tokens = panel;
  pl.n_panels = (int)((T1 + panel - 1) / panel);
  pl.dz_ld = align_up((size_t)V, pl.tensor ? (pl.planes == 3 ? 2 * kBK : 64) : 4);
  pl.logits_ld = align_up((size_t)V, 4);
  const bool want_bf16 = p->dw_dtype == ULORL_BF16;
  pl.dw_direct = pl.tensor && want_bf16 && pl.n_panels == 1 && !p->dw_accumulate && (pl.planes == 1 || T <= kSplitTokens);
  pl.dw_acc = want_bf16 && !pl.dw_direct;
  // d_hidden: few token tiles make few units (256 x 512 outputs each), so the vocabulary is cut into parts until
  // the units fill the GPU; the parts are float32 and added in order
  pl.dh_parts = 1;
  // Units of 256 x 512 outputs load the row operand once for both halves but cannot hide their epilogue behind the next
  // unit; units of 256 x 256 can.  d_hidden reduces over the vocabulary and its epilogue is small: 512, unless a
  // quarter or more of the columns would be padding.  d_W reduces over the panel's tokens; measured with 512 and with
  // 256 columns, at 151936 x 2048: 64 tokens 184 and 216 us, 200 tokens 282 and 292, 2011 tokens 1072 and 980, 8192 tokens
  // 3990 and 3750; 50000 x 256, 2000 tokens: 74 and 51.  These are of d_W in bf16, before its epilogue had two groups of warps;
  // for float32 d_W and one that is added into the rule is the same and was not measured.
  const size_t h1 = align_up((size_t)H, kBN), h2 = align_up((size_t)H, 2 * kBN);
  pl.dh_acc = 4 * h2 >= 5 * h1 ? 1 : 2;
  pl.dw_acc_tiles = panel > 512 || 4 * h2 >= 5 * h1 ? 1 : 2;
  if (pl.tensor) {
    const int atoms = pl.dh_acc == 1 ? 2 : 1;
    const int k_blocks = (V + kBK * atoms - 1) / (kBK * atoms);
    const int units = ((panel + tile_m - 1) / tile_m) * ((H + pl.dh_acc * kBN - 1) / (pl.dh_acc * kBN));
    int parts = units >= pl.workers ? 1 : pl.workers / units;
    // a part keeps at least 1024 vocabulary entries; six times the work and sums of limited length with float32 operands
    if (pl.planes == 3) parts = std::max(std::min(parts, k_blocks * atoms / 2), (V + kSplitEntries - 1) / kSplitEntries);
    else parts = std::max(1, std::min(parts, k_blocks * atoms / 16));
    parts = std::max(1, std::min(parts, k_blocks));
    pl.dh_part_blocks = (k_blocks + parts - 1) / parts;
    pl.dh_parts = (k_blocks + pl.dh_part_blocks - 1) / pl.dh_part_blocks;
    pl.dh_part_rows = (int)align_up((size_t)panel, (size_t)tile_m);
  }
  size_t off = 256;
  pl.off_status = 0;
  pl.off_top_pub = off;   // behind the status word: cleared together
  if (pl.tensor && !pl.small && K) off = align_up(off + sizeof(uint32_t) * (size_t)std::min(pl.n_partial, 32) * T1, 256);
  pl.off_partials = off;  off = align_up(off + sizeof(float4) * (size_t)pl.n_partial * T1, 256);
  pl.off_acc_y = off;     off = align_up(off + sizeof(float) * T1, 256);
  // the alternatives of a scoring call and the teacher lists of a distillation call are never there together
  size_t lists = off, teacher = off;
  pl.off_top_val = lists; lists = K <= kMaxTop ? align_up(lists + sizeof(float) * (size_t)pl.n_partial * T1 * K, 256) : lists;
  pl.off_top_id = lists;  lists = K <= kMaxTop ? align_up(lists + sizeof(int) * (size_t)pl.n_partial * T1 * K, 256) : lists;
  pl.off_sorted = teacher; teacher = align_up(teacher + sizeof(int) * T1 * K, 256);
  pl.off_list_z = teacher; teacher = align_up(teacher + sizeof(float) * T1 * K, 256);
  pl.off_slots = teacher;  teacher = align_up(teacher + T1 * K, 256);
  off = align_up(std::max(lists, teacher), 1024);
  pl.off_logits = off;    // forward passes that go through a panel of logits
  pl.fwd_total = off;
  pl.off_planes = off;
  const size_t plane_bytes = pl.tensor && pl.planes == 3 ? align_up(sizeof(__nv_bfloat16) * 3 * (size_t)pl.width * (T1 + (size_t)V), 1024) : 0;
  pl.fwd_total += plane_bytes;
  if (pl.small || !pl.tensor) pl.fwd_total = align_up(off + sizeof(float) * (size_t)std::min(panel, (int)T1) * pl.logits_ld, 1024);
  off = 256;
  pl.off_row_p = off;     off = align_up(off + sizeof(float4) * T1, 256);
  pl.off_row_ins = off;   off = align_up(off + sizeof(float) * T1, 1024);
  pl.off_panel = off;
  off = align_up(off + (size_t)panel * pl.dz_ld * (pl.tensor ? 2 * (size_t)pl.planes : 4), 1024);
  if (pl.dw_acc) { pl.off_dw_acc = off; off = align_up(off + sizeof(float) * (size_t)V * (size_t)H, 1024); }
  if (!pl.tensor && p->dtype == ULORL_F32) {      // float32 contractions cut over k
    pl.off_parts = off;
    // tiles x parts is at most the multiprocessor count, and a tile has no more than 128 x min(H, 128) outputs
    off = align_up(off + sizeof(float) * (size_t)pl.sms * kSgTile * (size_t)std::min(H, kSgTile), 1024);
  }
  if (pl.dh_parts > 1) {
    pl.off_parts = off;
    off = align_up(off + sizeof(float) * (size_t)pl.dh_parts * (size_t)pl.dh_part_rows * (size_t)H, 1024);
  }
  pl.off_planes_bwd = off;
  off += plane_bytes;
  pl.bwd_total = off;
  return pl;
}

template <int kMode>
static int launch_pair(const HeadPlan& pl, const CUtensorMap& ma, const CUtensorMap& mb, const CUtensorMap& mc,
                       const UmmaArgs& a, cudaStream_t stream) {
  return launch_umma_impl<kMode, 2, 1>(ma, mb, mc, a, pl.sms, stream);
}

// The gradient contractions: units of 256 x 512 (acc = 2) or 256 x 256 outputs.
template <int kMode>
static int launch_grad(const HeadPlan& pl, int acc, const CUtensorMap& ma, const CUtensorMap& mb, const CUtensorMap& mc,
                       UmmaArgs a, cudaStream_t stream) {
  a.n_tiles = (a.N + acc * kBN - 1) / (acc * kBN);
  return acc == 2 ? launch_umma_impl<kMode, 2, 2>(ma, mb, mc, a, pl.sms, stream)
                  : launch_umma_impl<kMode, 2, 1>(ma, mb, mc, a, pl.sms, stream);
}

// hidden and W as the tensor cores take them: themselves, or their planes, written here.
struct HeadOperands {
  const void *hidden, *W;
  uint64_t ld;                             // columns of a row, all planes
};
static int prepare_operands(const ulorl_head_params_t* p, const HeadPlan& pl, const void* hidden, const void* W, void* planes,
                            HeadOperands* o, cudaStream_t stream) {
  *o = {hidden, W, (uint64_t)p->H};
  if (pl.planes == 1) return ULORL_OK;
  __nv_bfloat16* out = static_cast<__nv_bfloat16*>(planes);
  const size_t rows = (size_t)p->T + (size_t)p->V, blocks = (rows * (size_t)(pl.width / 4) + 255) / 256;
  split_planes_kernel<<<(unsigned)std::min(blocks, (size_t)pl.sms * 16), 256, 0, stream>>>(
      static_cast<const float*>(hidden), (size_t)p->T, static_cast<const float*>(W), (size_t)p->V, p->H, pl.width, out);
  *o = {out, out + (size_t)p->T * 3 * (size_t)pl.width, (uint64_t)(3 * pl.width)};
  return check_launch();
}

// The forward sweep of hidden against W on the tensor cores; `a` carries the mode's own fields.
static int run_sweep(const ulorl_head_params_t* p, const HeadPlan& pl, int mode, UmmaArgs a, const void* hidden,
                     const void* W, uint8_t* ws, cudaStream_t stream) {
  HeadOperands o;
  int st = prepare_operands(p, pl, hidden, W, ws + pl.off_planes, &o, stream);
  if (st != ULORL_OK) return st;
  CUtensorMap map_a, map_b;
  st = make_map_bf16(&map_a, o.hidden, (uint64_t)p->T, o.ld, o.ld, kBK, kBM);
  if (st != ULORL_OK) return st;
  st = make_map_bf16(&map_b, o.W, (uint64_t)p->V, o.ld, o.ld, kBK, kBN / 2);
  if (st != ULORL_OK) return st;
  a.M = p->T; a.N = p->V; a.K = pl.width;
  a.n_products = pl.planes == 3 ? (int)kProducts : 0;
  a.a_plane = a.b_plane = pl.planes == 3 ? pl.width : 0;
  a.m_tiles = (p->T + 2 * kBM - 1) / (2 * kBM);
  a.n_tiles = (p->V + kBN - 1) / kBN;
  a.n_split = pl.n_split;
  a.split_stride = a.tiles_per_split = pl.tiles_per_split;
  a.kappa = p->inv_temperature;
  a.partials = reinterpret_cast<float4*>(ws + pl.off_partials);
  a.T_total = p->T;
  a.status = reinterpret_cast<int*>(ws + pl.off_status);
  switch (mode) {
    case kModeScores: return launch_pair<kModeScores>(pl, map_a, map_b, map_a, a, stream);
    case kModeScoresTop8: return launch_pair<kModeScoresTop8>(pl, map_a, map_b, map_a, a, stream);
    case kModeScoresTop32: return launch_pair<kModeScoresTop32>(pl, map_a, map_b, map_a, a, stream);
    default: return launch_pair<kModeDistill>(pl, map_a, map_b, map_a, a, stream);
  }
}

template <bool kAAlongK, bool kBAlongK>
static int run_sgemm(const HeadPlan& pl, const float* A, size_t lda, const float* B, size_t ldb, float* C, size_t ldc, int M, int N,
                     int K, int accumulate, float* scratch, cudaStream_t stream) {
  SgemmArgs a{};
  a.A = A; a.B = B; a.lda = lda; a.ldb = ldb;
  a.M = M; a.N = N; a.K = K;
  int parts = 1;
  a.k_part = (int)align_up((size_t)K, kSgK);
  if (scratch) parts = sgemm_parts(pl, M, N, K, &a.k_part);
  a.C = parts > 1 ? scratch : C;
  a.ldc = parts > 1 ? (size_t)N : ldc;
  a.part_stride = parts > 1 ? (size_t)M * (size_t)N : 0;
  a.accumulate = parts > 1 ? 0 : accumulate;
  const dim3 grid(tile_blocks(M, N, kSgTile), 1, parts);
  sgemm_kernel<kAAlongK, kBAlongK><<<grid, kSgThreads, 0, stream>>>(a);
  ULORL_LAUNCH_CHECK();
  if (parts > 1) {                                                  // rows of the result are contiguous here: ldc = N
    const size_t n = (size_t)M * (size_t)N;
    sgemm_parts_kernel<<<(unsigned)((n / 4 + 255) / 256), 256, 0, stream>>>(scratch, parts, n, n, C, accumulate);
    ULORL_LAUNCH_CHECK();
  }
  return ULORL_OK;
}

// panel[i, v] = hidden[t0 + i] . W[v] in float32 on CUDA cores (bf16 operands: the cross-check of the tensor path).
static int simt_logits_panel(const ulorl_head_params_t* p, const HeadPlan& pl, const void* hidden, const void* W, int t0, int rows,
                             float* panel, size_t ld, cudaStream_t stream) {
  const size_t H = (size_t)p->H;
  if (p->dtype == ULORL_F32)
    return run_sgemm<true, true>(pl, static_cast<const float*>(hidden) + (size_t)t0 * H, H, static_cast<const float*>(W), H, panel, ld,
                                 rows, p->V, p->H, 0, nullptr, stream);
  const unsigned grid = tile_blocks(rows, p->V, kSimtTile);
  simt_gemm_kernel<__nv_bfloat16, __nv_bfloat16, float><<<grid, kSimtThreads, 0, stream>>>(
      static_cast<const __nv_bfloat16*>(hidden) + (size_t)t0 * H, H, 1, static_cast<const __nv_bfloat16*>(W), 1, H, panel, ld, rows,
      p->V, p->H, 0);
  return check_launch();
}

template <int kN>
static int launch_small(const ulorl_head_params_t* p, const HeadPlan& pl, const void* hidden, const void* W, float* logits,
                        int* status, cudaStream_t stream) {
  using Cfg = SmallConfig<kN>;
  static bool opted_in[kMaxDevices] = {};
  int dev = 0;
  if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= kMaxDevices) return ULORL_ERR_CUDA;
  {
    std::lock_guard<std::mutex> lock(g_setup_mutex);
    if (!opted_in[dev]) {
      if (cudaFuncSetAttribute(small_logits_kernel<kN>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)Cfg::smem_bytes) !=
          cudaSuccess)
        return ULORL_ERR_CUDA;
      opted_in[dev] = true;
    }
  }
  SmallArgs a{};
  a.T = p->T; a.V = p->V; a.K = p->H;
  a.rows_per_cta = (int)align_up((size_t)(p->V + pl.sms - 1) / pl.sms, 16);
  a.logits = logits;
  a.ld = pl.logits_ld;
  a.status = status;
  const int last = a.rows_per_cta - (a.rows_per_cta - 1) / kBM * kBM;
  CUtensorMap map_w, map_last, map_h;
  int st = make_map_bf16(&map_w, W, (uint64_t)p->V, (uint64_t)p->H, (uint64_t)p->H, kBK, kBM);
  if (st != ULORL_OK) return st;
  st = make_map_bf16(&map_last, W, (uint64_t)p->V, (uint64_t)p->H, (uint64_t)p->H, kBK, (uint32_t)last);
  if (st != ULORL_OK) return st;
  st = make_map_bf16(&map_h, hidden, (uint64_t)p->T, (uint64_t)p->H, (uint64_t)p->H, kBK, kN);
  if (st != ULORL_OK) return st;
  const unsigned blocks = (unsigned)((p->V + a.rows_per_cta - 1) / a.rows_per_cta);
  small_logits_kernel<kN><<<blocks, kSmallThreads, Cfg::smem_bytes, stream>>>(map_w, map_last, map_h, a);
  return check_launch();
}

// logits[i, v] = hidden[t0 + i] . W[v] in float32 for the paths that go through a panel of logits.
static int logits_panel(const ulorl_head_params_t* p, const HeadPlan& pl, const void* hidden, const void* W, int t0, int rows,
                        float* logits, uint8_t* ws, cudaStream_t stream) {
  if (!pl.small) return simt_logits_panel(p, pl, hidden, W, t0, rows, logits, pl.logits_ld, stream);
  int* status = reinterpret_cast<int*>(ws + pl.off_status);
  if (p->T <= 16) return launch_small<16>(p, pl, hidden, W, logits, status, stream);
  if (p->T <= 32) return launch_small<32>(p, pl, hidden, W, logits, status, stream);
  return launch_small<64>(p, pl, hidden, W, logits, status, stream);
}

// Rows are spread over clusters until there are two blocks a multiprocessor (four fit; the rule is older), as long as a
// block keeps four loads a thread; more than eight blocks a cluster have to be asked for, once per device.
template <typename T, bool kHeld = false>
static int launch_rows(const RowsArgs& a, int sms, cudaStream_t stream) {
  static bool opted_in[kMaxDevices] = {};
  int dev = 0;
  if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= kMaxDevices) return ULORL_ERR_CUDA;
  {
    std::lock_guard<std::mutex> lock(g_setup_mutex);
    if (!opted_in[dev]) {
      if (cudaFuncSetAttribute(logits_rows_kernel<T, kHeld>, cudaFuncAttributeNonPortableClusterSizeAllowed, 1) != cudaSuccess ||
          cudaFuncSetAttribute(logits_rows_kernel<T, kHeld>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)kRowSmem) != cudaSuccess)
        return ULORL_ERR_CUDA;
      opted_in[dev] = true;
    }
  }
  const int least = kRowThreads * kRowUnroll * RowType<T>::per_vec;
  int cluster = 1;
  while (cluster < kRowMaxCluster && (long)a.T * cluster * 2 <= 2L * sms && a.V >= 2 * cluster * least) cluster *= 2;
  cudaLaunchConfig_t cfg{};
  cfg.gridDim = dim3((unsigned)a.T * (unsigned)cluster, 1, 1);
  cfg.blockDim = dim3(kRowThreads, 1, 1);
  cfg.dynamicSmemBytes = kRowSmem;
  cfg.stream = stream;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeClusterDimension;
  attr[0].val.clusterDim.x = (unsigned)cluster;
  attr[0].val.clusterDim.y = 1;
  attr[0].val.clusterDim.z = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  if (cudaLaunchKernelEx(&cfg, logits_rows_kernel<T, kHeld>, a) != cudaSuccess) {
    (void)cudaGetLastError();
    return ULORL_ERR_CUDA;
  }
  return check_launch();
}

static int clear_status(void* workspace, size_t workspace_bytes, cudaStream_t stream) {
  if (workspace && workspace_bytes >= 256 && cudaMemsetAsync(workspace, 0, 256, stream) != cudaSuccess) return ULORL_ERR_CUDA;
  return ULORL_OK;
}

// Checks what every call shares and clears the first `clear` bytes of the workspace: the status word, by the forward calls
// (what they found stays there while the backward calls run).
static int head_begin(const void* hidden, const void* W, void* workspace, size_t workspace_bytes, size_t need, size_t clear,
                      cudaStream_t stream) {
  if (!hidden || !W || !workspace) return ULORL_ERR_INVALID_ARG;
  if (!aligned16(hidden) || !aligned16(W) || !aligned16(workspace)) return ULORL_ERR_UNSUPPORTED;
  if (workspace_bytes < need) return ULORL_ERR_WORKSPACE;
  if (clear && cudaMemsetAsync(workspace, 0, clear, stream) != cudaSuccess) return ULORL_ERR_CUDA;
  return ULORL_OK;
}

// dz panels and the two gradient contractions.  row_p (and row_ins, targets) say what a row of dz is (flat: with beta = 0
// in all of them); put_list writes the teacher lists' columns of a panel, if there are any.
static int run_head_bwd(const ulorl_head_params_t* p, const HeadPlan& pl, const void* hidden, const void* W,
                        const int32_t* targets, const float4* row_p, const float* row_ins, bool flat,
                        const std::function<int(int, int)>& put_list, void* d_hidden, void* d_W_out, uint8_t* ws,
                        cudaStream_t stream) {
  const int T = p->T, H = p->H, V = p->V;
  float* d_W = pl.dw_acc ? reinterpret_cast<float*>(ws + pl.off_dw_acc) : static_cast<float*>(d_W_out);
  const int acc_into = pl.dw_acc ? 0 : p->dw_accumulate;
  int st;
  if (pl.tensor) {
    __nv_bfloat16* dz = reinterpret_cast<__nv_bfloat16*>(ws + pl.off_panel);
    const int tile_m = 2 * kBM;
    const bool split = pl.planes == 3;
    const int n_products = split ? (int)kProducts : 0, dz_plane = split ? (int)pl.dz_ld : 0, op_plane = split ? pl.width : 0;
    const uint64_t dz_row = (uint64_t)pl.planes * pl.dz_ld;
    HeadOperands o;
    st = prepare_operands(p, pl, hidden, W, ws + pl.off_planes_bwd, &o, stream);
    if (st != ULORL_OK) return st;
    CUtensorMap map_hidden_k, map_w_k, map_w_mn, map_hidden_mn, map_dw, map_parts;
    st = make_map_bf16(&map_hidden_k, o.hidden, (uint64_t)T, o.ld, o.ld, kBK, kBM);
    if (st != ULORL_OK) return st;
    st = make_map_bf16(&map_w_k, o.W, (uint64_t)V, o.ld, o.ld, kBK, kBN / 2);
    if (st != ULORL_OK) return st;
    st = make_map_bf16(&map_w_mn, o.W, (uint64_t)V, o.ld, o.ld, 64, kBK);
    if (st != ULORL_OK) return st;
    st = make_map_bf16(&map_hidden_mn, o.hidden, (uint64_t)T, o.ld, o.ld, 64, kBK);
    if (st != ULORL_OK) return st;
    st = pl.dw_direct ? make_map_bf16(&map_dw, d_W_out, (uint64_t)V, (uint64_t)H, (uint64_t)H, 64, kBM)
                      : make_map(&map_dw, CU_TENSOR_MAP_DATA_TYPE_FLOAT32, 4, d_W, (uint64_t)V, (uint64_t)H, (uint64_t)H, 32, kBM);
    if (st != ULORL_OK) return st;
    float* parts = reinterpret_cast<float*>(ws + pl.off_parts);
    if (pl.dh_parts > 1) {
      st = make_map(&map_parts, CU_TENSOR_MAP_DATA_TYPE_FLOAT32, 4, parts, (uint64_t)pl.dh_parts * pl.dh_part_rows, (uint64_t)H,
                    (uint64_t)H, 32, kBM);
      if (st != ULORL_OK) return st;
    }
    for (int t0 = 0, panel = 0; t0 < T; t0 += pl.panel_tokens, ++panel) {
      const int rows = std::min(T - t0, pl.panel_tokens);
      CUtensorMap dz_out, dz_k, dz_mn;
      st = make_map_bf16(&dz_out, dz, (uint64_t)pl.panel_tokens, dz_row, dz_row, 64, kBM);
      if (st != ULORL_OK) return st;
      st = make_map_bf16(&dz_k, dz, (uint64_t)rows, dz_row, dz_row, kBK, kBM);
      if (st != ULORL_OK) return st;
      st = make_map_bf16(&dz_mn, dz, (uint64_t)rows, dz_row, dz_row, 64, kBK);
      if (st != ULORL_OK) return st;
      UmmaArgs a{};
      a.M = rows; a.N = V; a.K = pl.width;
      a.n_products = n_products; a.a_plane = a.b_plane = op_plane; a.out_plane = dz_plane;
      a.m_tiles = (rows + tile_m - 1) / tile_m;
      a.n_tiles = (int)((pl.dz_ld + kBN - 1) / kBN);
      a.group_m = kRasterGroup;
      a.a_mn0 = a.row0 = t0;
      a.kappa = p->inv_temperature;
      a.targets = targets;
      a.row_p = row_p;
      a.row_ins = row_ins;
      a.row_flat = flat ? 1 : 0;
      a.dz_cols = (int)pl.dz_ld;
      a.status = reinterpret_cast<int*>(ws + pl.off_status);
      st = split ? launch_pair<kModeDzRow3>(pl, map_hidden_k, map_w_k, dz_out, a, stream)
                 : launch_pair<kModeDzRow>(pl, map_hidden_k, map_w_k, dz_out, a, stream);
      if (st != ULORL_OK) return st;
      if (put_list) {
        st = put_list(t0, rows);
        if (st != ULORL_OK) return st;
      }
      // d_hidden[t0 + m, h] = sum_v dz[m, v] W[v, h]
      UmmaArgs b{};
      b.M = rows; b.N = H; b.K = V;
      b.n_products = n_products; b.a_plane = dz_plane; b.b_plane = op_plane;
      b.m_tiles = (rows + tile_m - 1) / tile_m;
      b.group_m = kGradRasterGroup;
      b.row0 = t0;
      b.out_ld = (size_t)H;
      b.status = a.status;
      if (split && pl.dh_parts == 1) {                             // float32 leaves the contraction as it is
        st = make_map(&map_parts, CU_TENSOR_MAP_DATA_TYPE_FLOAT32, 4, static_cast<float*>(d_hidden) + (size_t)t0 * H, (uint64_t)rows,
                      (uint64_t)H, (uint64_t)H, 32, kBM);
        if (st != ULORL_OK) return st;
      }
      if (split || pl.dh_parts > 1) {
        b.n_split = pl.dh_parts;
        b.part_blocks = pl.dh_part_blocks;
        b.part_rows = pl.dh_part_rows;
        st = launch_grad<kModeDHiddenPart>(pl, pl.dh_acc, dz_k, map_w_mn, map_parts, b, stream);
        if (st != ULORL_OK) return st;
        const size_t n = (size_t)rows * (size_t)H, stride = (size_t)pl.dh_part_rows * (size_t)H;
        if (split && pl.dh_parts > 1)
          sgemm_parts_kernel<<<(unsigned)((n / 4 + 255) / 256), 256, 0, stream>>>(parts, pl.dh_parts, stride, n,
                                                                                  static_cast<float*>(d_hidden) + (size_t)t0 * H, 0);
        else if (!split)
          sum_parts_kernel<<<(unsigned)((n / 8 + 255) / 256), 256, 0, stream>>>(
              parts, pl.dh_parts, stride, n, static_cast<__nv_bfloat16*>(d_hidden) + (size_t)t0 * H);
        ULORL_LAUNCH_CHECK();
      } else {
        b.d_hidden = static_cast<__nv_bfloat16*>(d_hidden);
        st = launch_grad<kModeDHidden>(pl, pl.dh_acc, dz_k, map_w_mn, map_w_mn, b, stream);
        if (st != ULORL_OK) return st;
      }
      // d_W[v, h] (+)= sum_m dz[m, v] hidden[t0 + m, h]
      const int terms = split ? kSplitTokens : rows;
      for (int m0 = 0; m0 < rows; m0 += terms) {
        UmmaArgs c{};
        c.M = V; c.N = H; c.K = std::min(terms, rows - m0);
        c.n_products = n_products; c.a_plane = dz_plane; c.b_plane = op_plane;
        c.m_tiles = (V + tile_m - 1) / tile_m;
        c.group_m = kGradRasterGroup;
        c.a_k0 = m0;
        c.b_k0 = t0 + m0;
        c.d_W = d_W;
        c.out_ld = (size_t)H;
        c.dz_cols = H;
        c.accumulate = (panel > 0 || m0 > 0 || acc_into) ? 1 : 0;
        c.status = a.status;
        st = pl.dw_direct ? launch_grad<kModeDWBf16>(pl, pl.dw_acc_tiles, dz_mn, map_hidden_mn, map_dw, c, stream)
                          : launch_grad<kModeDW>(pl, pl.dw_acc_tiles, dz_mn, map_hidden_mn, map_dw, c, stream);
        if (st != ULORL_OK) return st;
      }
    }
  } else {
    float* dz = reinterpret_cast<float*>(ws + pl.off_panel);
    const size_t ld = pl.dz_ld;
    for (int t0 = 0, panel = 0; t0 < T; t0 += pl.panel_tokens, ++panel) {
      const int rows = std::min(T - t0, pl.panel_tokens);
      const int acc = (panel > 0 || acc_into) ? 1 : 0;
      const dim3 gdz((unsigned)std::min((V + 1023) / 1024, 64), rows);
      const unsigned gdh = tile_blocks(rows, H, kSimtTile), gdw = tile_blocks(V, H, kSimtTile);
      const bool f32 = p->dtype == ULORL_F32;
      st = simt_logits_panel(p, pl, hidden, W, t0, rows, dz, ld, stream);
      if (st != ULORL_OK) return st;
      dz_rows_f32_kernel<<<gdz, 256, 0, stream>>>(dz, ld, V, t0, p->inv_temperature, row_p, row_ins, targets);
      ULORL_LAUNCH_CHECK();
      if (put_list) {
        st = put_list(t0, rows);
        if (st != ULORL_OK) return st;
      }
      if (f32) {
        float* scratch = reinterpret_cast<float*>(ws + pl.off_parts);
        st = run_sgemm<true, false>(pl, dz, ld, static_cast<const float*>(W), (size_t)H, static_cast<float*>(d_hidden) + (size_t)t0 * H,
                                    (size_t)H, rows, H, V, 0, scratch, stream);
        if (st != ULORL_OK) return st;
        st = run_sgemm<false, false>(pl, dz, ld, static_cast<const float*>(hidden) + (size_t)t0 * H, (size_t)H, d_W, (size_t)H, V, H,
                                     rows, acc, scratch, stream);
        if (st != ULORL_OK) return st;
      } else {
        simt_gemm_kernel<float, __nv_bfloat16, __nv_bfloat16><<<gdh, kSimtThreads, 0, stream>>>(
            dz, ld, 1, static_cast<const __nv_bfloat16*>(W), (size_t)H, 1,
            static_cast<__nv_bfloat16*>(d_hidden) + (size_t)t0 * H, (size_t)H, rows, H, V, 0);
        ULORL_LAUNCH_CHECK();
        simt_gemm_kernel<float, __nv_bfloat16, float><<<gdw, kSimtThreads, 0, stream>>>(
            dz, 1, ld, static_cast<const __nv_bfloat16*>(hidden) + (size_t)t0 * H, (size_t)H, 1, d_W, (size_t)H, V, H, rows, acc);
        ULORL_LAUNCH_CHECK();
      }
    }
  }
  if (pl.dw_acc) return round_dw_rows(d_W, d_W_out, 0, V, H, p->dw_accumulate, stream);
  return ULORL_OK;
}

// T == 0: the gradient of nothing.
static int empty_head_bwd(const ulorl_head_params_t* p, void* d_W, cudaStream_t stream) {
  if (!d_W) return ULORL_ERR_INVALID_ARG;
  const size_t bytes = (size_t)p->V * (size_t)p->H * (p->dw_dtype == ULORL_BF16 ? 2 : 4);
  if (!p->dw_accumulate && cudaMemsetAsync(d_W, 0, bytes, stream) != cudaSuccess) return ULORL_ERR_CUDA;
  return ULORL_OK;
}

}  // namespace ulorl

extern "C" {

size_t ulorl_head_workspace_bytes(const ulorl_head_params_t* params, int32_t backward) {
  if (validate_head(params) != ULORL_OK) return 0;
  const size_t fwd = make_head_plan(params, false).fwd_total;
  return backward ? std::max(fwd, make_head_plan(params, true).bwd_total) : fwd;
}

int ulorl_token_scores(const ulorl_head_params_t* params, const void* hidden, const void* W, const int32_t* targets,
                       float* logp, float* entropy, float* lse, float* norm, int32_t* top_ids, float* top_logp,
                       void* workspace, size_t workspace_bytes, void* cuda_stream) {
  TraceRange trace("ulorl token scores");
  int st = validate_head(params);
  if (st != ULORL_OK) return st;
  const int T = params->T, V = params->V, k = params->top_k;
  if (k > ULORL_MAX_TOP) return ULORL_ERR_UNSUPPORTED;
  if (k > V) return ULORL_ERR_INVALID_ARG;
  if (T == 0) return clear_status(workspace, workspace_bytes, reinterpret_cast<cudaStream_t>(cuda_stream));
  if ((k > 0) != (top_ids != nullptr) || (k > 0) != (top_logp != nullptr)) return ULORL_ERR_INVALID_ARG;
  if (logp && !targets) return ULORL_ERR_INVALID_ARG;
  if (!aligned8(norm)) return ULORL_ERR_UNSUPPORTED;
  cudaStream_t stream = reinterpret_cast<cudaStream_t>(cuda_stream);
  const HeadPlan pl = make_head_plan(params, false);
  st = head_begin(hidden, W, workspace, workspace_bytes, pl.fwd_total, pl.tensor && !pl.small && k > 0 ? pl.off_partials : 256, stream);
  if (st != ULORL_OK) return st;
  uint8_t* ws = static_cast<uint8_t*>(workspace);
  if (pl.tensor && !pl.small) {
    UmmaArgs a{};
    a.targets = logp ? targets : nullptr;
    a.acc_y = reinterpret_cast<float*>(ws + pl.off_acc_y);
    a.top_k = k;
    a.top_val = reinterpret_cast<float*>(ws + pl.off_top_val);
    a.top_id = reinterpret_cast<int*>(ws + pl.off_top_id);
    a.top_pub = reinterpret_cast<uint32_t*>(ws + pl.off_top_pub);
    st = run_sweep(params, pl, k == 0 ? kModeScores : (k <= 8 ? kModeScoresTop8 : kModeScoresTop32), a, hidden, W, ws, stream);
    if (st != ULORL_OK) return st;
    MergeArgs m{};
    m.T = T; m.n_split = pl.n_partial; m.k = k;
    m.kappa = params->inv_temperature;
    m.partials = reinterpret_cast<const float4*>(ws + pl.off_partials);
    m.acc_y = a.acc_y;
    m.top_val = a.top_val; m.top_id = a.top_id;
    m.logp = logp; m.entropy = entropy; m.lse = lse;
    m.norm = reinterpret_cast<float2*>(norm);
    m.out_ids = top_ids; m.out_logp = top_logp;
    merge_scores_kernel<<<(T + kMergeWarps - 1) / kMergeWarps, 32 * kMergeWarps, 0, stream>>>(m);
    return check_launch();
  }
  float* panel = reinterpret_cast<float*>(ws + pl.off_logits);
  for (int t0 = 0; t0 < T; t0 += pl.panel_tokens) {
    const int rows = std::min(T - t0, pl.panel_tokens);
    st = logits_panel(params, pl, hidden, W, t0, rows, panel, ws, stream);
    if (st != ULORL_OK) return st;
    RowsArgs a{};
    a.logits = panel; a.ld = pl.logits_ld;
    a.T = rows; a.V = V; a.k = k;
    a.kappa = params->inv_temperature;
    a.targets = targets ? targets + t0 : nullptr;
    a.logp = logp ? logp + t0 : nullptr;
    a.entropy = entropy ? entropy + t0 : nullptr;
    a.lse = lse ? lse + t0 : nullptr;
    a.norm = norm ? reinterpret_cast<float2*>(norm) + t0 : nullptr;
    a.top_ids = top_ids ? top_ids + (size_t)t0 * k : nullptr;
    a.top_logp = top_logp ? top_logp + (size_t)t0 * k : nullptr;
    a.status = reinterpret_cast<int*>(ws + pl.off_status);
    st = launch_rows<float>(a, pl.sms, stream);
    if (st != ULORL_OK) return st;
  }
  return ULORL_OK;
}

int ulorl_token_scores_bwd(const ulorl_head_params_t* params, const void* hidden, const void* W,
                           const int32_t* targets, const float* norm, const float* logp, const float* entropy,
                           const float* d_logp, const float* d_entropy, void* d_hidden, void* d_W,
                           void* workspace, size_t workspace_bytes, void* cuda_stream) {
  TraceRange trace("ulorl token scores backward");
  int st = validate_head(params);
  if (st != ULORL_OK) return st;
  cudaStream_t stream = reinterpret_cast<cudaStream_t>(cuda_stream);
  const int T = params->T;
  if (T == 0) return empty_head_bwd(params, d_W, stream);
  if (!norm || !d_hidden || !d_W || (!d_logp && !d_entropy)) return ULORL_ERR_INVALID_ARG;
  if ((d_logp && (!logp || !targets)) || (d_entropy && !entropy)) return ULORL_ERR_INVALID_ARG;
  if (!aligned16(d_hidden) || !aligned16(d_W) || !aligned8(norm)) return ULORL_ERR_UNSUPPORTED;
  const HeadPlan pl = make_head_plan(params, true);
  st = head_begin(hidden, W, workspace, workspace_bytes, pl.bwd_total, 0, stream);
  if (st != ULORL_OK) return st;
  uint8_t* ws = static_cast<uint8_t*>(workspace);
  float4* row_p = reinterpret_cast<float4*>(ws + pl.off_row_p);
  float* row_ins = reinterpret_cast<float*>(ws + pl.off_row_ins);
  row_params_kernel<<<(T + 255) / 256, 256, 0, stream>>>(T, params->inv_temperature, reinterpret_cast<const float2*>(norm), logp, entropy, d_logp, d_entropy,
                                                         row_p, row_ins);
  ULORL_LAUNCH_CHECK();
  return run_head_bwd(params, pl, hidden, W, d_logp ? targets : nullptr, row_p, row_ins, d_entropy == nullptr, nullptr, d_hidden, d_W, ws, stream);
}

int ulorl_logits_scores(const void* logits, int32_t dtype, int32_t T, int32_t V, int64_t ld, int32_t top_k,
                        float inv_temperature, const int32_t* targets, float* logp, float* entropy, float* lse,
                        int32_t* top_ids, float* top_logp, void* cuda_stream) {
  TraceRange trace("ulorl logits scores");
  if (T < 0 || V <= 0 || ld < V || top_k < 0 || top_k > V) return ULORL_ERR_INVALID_ARG;
  if (dtype != ULORL_F32 && dtype != ULORL_BF16 && dtype != ULORL_F16) return ULORL_ERR_UNSUPPORTED;
  if (top_k > ULORL_MAX_TOP) return ULORL_ERR_UNSUPPORTED;
  if (!(inv_temperature > 0.f) || !std::isfinite(inv_temperature)) return ULORL_ERR_INVALID_ARG;
  if (!scale_supported(inv_temperature) || T > kHeadMaxSize || V > kHeadMaxSize) return ULORL_ERR_UNSUPPORTED;
  if (T == 0) return ULORL_OK;
  if ((top_k > 0) != (top_ids != nullptr) || (top_k > 0) != (top_logp != nullptr)) return ULORL_ERR_INVALID_ARG;
  if (logp && !targets) return ULORL_ERR_INVALID_ARG;
  if (!logits || (reinterpret_cast<uintptr_t>(logits) & (dtype == ULORL_F32 ? 3u : 1u))) return ULORL_ERR_INVALID_ARG;
  RowsArgs a{};
  a.logits = logits; a.ld = (size_t)ld;
  a.T = T; a.V = V; a.k = top_k;
  a.kappa = inv_temperature;
  a.targets = targets;
  a.logp = logp; a.entropy = entropy; a.lse = lse;
  a.top_ids = top_ids; a.top_logp = top_logp;
  cudaStream_t stream = reinterpret_cast<cudaStream_t>(cuda_stream);
  const int sms = device_sm_count();
  return dtype == ULORL_F32 ? launch_rows<float>(a, sms, stream)
                            : (dtype == ULORL_BF16 ? launch_rows<__nv_bfloat16>(a, sms, stream) : launch_rows<__half>(a, sms, stream));
}

int ulorl_selftest_logits_wait(const float* logits, int32_t T, int32_t V, int32_t top_k, float* lse, int32_t* top_ids, float* top_logp,
                               void* workspace, int64_t limit_cycles, void* cuda_stream) {
  if (!logits || !lse || !top_ids || !top_logp || !workspace) return ULORL_ERR_INVALID_ARG;
  if (!aligned16(logits) || T < 1 || T > 65536 || V < 4096 || V > kHeadMaxSize || top_k < 1 || top_k > ULORL_MAX_TOP)
    return ULORL_ERR_INVALID_ARG;
  if (limit_cycles < 1000 || limit_cycles > 100000000) return ULORL_ERR_INVALID_ARG;
  RowsArgs a{};
  a.logits = logits; a.ld = (size_t)V;
  a.T = T; a.V = V; a.k = top_k;
  a.kappa = 1.f;
  a.lse = lse;
  a.top_ids = top_ids; a.top_logp = top_logp;
  a.status = static_cast<int*>(workspace);
  a.wait_limit = limit_cycles;
  return launch_rows<float, true>(a, device_sm_count(), reinterpret_cast<cudaStream_t>(cuda_stream));
}

int ulorl_distill_fwd(const ulorl_head_params_t* params, const void* hidden, const void* W,
                      const int32_t* teacher_ids, const float* teacher_logp, const float* weights,
                      float* loss, float* kl, float* lse, float* norm, float* coef, float* entry_grad,
                      void* workspace, size_t workspace_bytes, void* cuda_stream) {
  TraceRange trace("ulorl distillation");
  int st = validate_head(params);
  if (st != ULORL_OK) return st;
  const int T = params->T, V = params->V, K = params->top_k;
  if (K < 1 || !loss) return ULORL_ERR_INVALID_ARG;
  cudaStream_t stream = reinterpret_cast<cudaStream_t>(cuda_stream);
  if (T == 0) {
    if (cudaMemsetAsync(loss, 0, sizeof(float), stream) != cudaSuccess) return ULORL_ERR_CUDA;
    return clear_status(workspace, workspace_bytes, stream);
  }
  if (!teacher_ids || !teacher_logp || !kl || !norm || !coef || !entry_grad) return ULORL_ERR_INVALID_ARG;
  if (!aligned8(norm)) return ULORL_ERR_UNSUPPORTED;
  const HeadPlan pl = make_head_plan(params, false);
  st = head_begin(hidden, W, workspace, workspace_bytes, pl.fwd_total, 256, stream);
  if (st != ULORL_OK) return st;
  uint8_t* ws = static_cast<uint8_t*>(workspace);
  int* status = reinterpret_cast<int*>(ws + pl.off_status);
  int* sorted = reinterpret_cast<int*>(ws + pl.off_sorted);
  uint8_t* slots = ws + pl.off_slots;
  float* list_z = reinterpret_cast<float*>(ws + pl.off_list_z);
  float4* partials = reinterpret_cast<float4*>(ws + pl.off_partials);
  const unsigned row_blocks = (unsigned)((T + 7) / 8);              // eight warps, one token each
  distill_sort_kernel<<<row_blocks, 256, 0, stream>>>(T, K, V, teacher_ids, sorted, slots, status);
  ULORL_LAUNCH_CHECK();
  if (pl.tensor && !pl.small) {
    UmmaArgs a{};
    a.list_k = K;
    a.list_ids = sorted;
    a.list_z = list_z;
    st = run_sweep(params, pl, kModeDistill, a, hidden, W, ws, stream);
    if (st != ULORL_OK) return st;
  } else {
    float* panel = reinterpret_cast<float*>(ws + pl.off_logits);
    for (int t0 = 0; t0 < T; t0 += pl.panel_tokens) {
      const int rows = std::min(T - t0, pl.panel_tokens);
      st = logits_panel(params, pl, hidden, W, t0, rows, panel, ws, stream);
      if (st != ULORL_OK) return st;
      distill_take_kernel<<<(rows + 7) / 8, 256, 0, stream>>>(rows, t0, K, panel, pl.logits_ld, sorted, list_z);
      ULORL_LAUNCH_CHECK();
      RowsArgs a{};
      a.logits = panel; a.ld = pl.logits_ld;
      a.T = rows; a.V = V;
      a.kappa = params->inv_temperature;
      a.partials = partials + t0;
      a.status = status;
      st = launch_rows<float>(a, pl.sms, stream);
      if (st != ULORL_OK) return st;
    }
  }
  DistillRowArgs d{};
  d.T = T; d.K = K; d.n_split = pl.n_partial; d.mode = params->distill_mode;
  d.kappa = params->inv_temperature;
  d.teacher_kappa = params->teacher_inv_temperature;
  d.inv_N = 1.0 / (params->norm_tokens > 0 ? (double)params->norm_tokens : (double)T);
  d.partials = partials;
  d.list_z = list_z; d.slots = slots;
  d.teacher = teacher_logp; d.weights = weights;
  d.kl = kl; d.norm = reinterpret_cast<float2*>(norm); d.lse = lse; d.coef = coef; d.entry_grad = entry_grad;
  d.loss = loss;
  d.done = reinterpret_cast<unsigned int*>(status) + 16;            // cleared with the status word
  distill_rows_kernel<<<row_blocks, kDistillThreads, 0, stream>>>(d);
  return check_launch();
}

int ulorl_distill_bwd(const ulorl_head_params_t* params, const void* hidden, const void* W,
                      const int32_t* teacher_ids, const float* norm, const float* coef, const float* entry_grad,
                      const float* grad_loss, void* d_hidden, void* d_W,
                      void* workspace, size_t workspace_bytes, void* cuda_stream) {
  TraceRange trace("ulorl distillation backward");
  int st = validate_head(params);
  if (st != ULORL_OK) return st;
  const int T = params->T, V = params->V, K = params->top_k;
  if (K < 1) return ULORL_ERR_INVALID_ARG;
  cudaStream_t stream = reinterpret_cast<cudaStream_t>(cuda_stream);
  if (T == 0) return empty_head_bwd(params, d_W, stream);
  if (!teacher_ids || !norm || !coef || !entry_grad || !d_hidden || !d_W) return ULORL_ERR_INVALID_ARG;
  if (!aligned16(d_hidden) || !aligned16(d_W) || !aligned8(norm)) return ULORL_ERR_UNSUPPORTED;
  const HeadPlan pl = make_head_plan(params, true);
  st = head_begin(hidden, W, workspace, workspace_bytes, pl.bwd_total, 0, stream);
  if (st != ULORL_OK) return st;
  uint8_t* ws = static_cast<uint8_t*>(workspace);
  float4* row_p = reinterpret_cast<float4*>(ws + pl.off_row_p);
  distill_params_kernel<<<(T + 255) / 256, 256, 0, stream>>>(T, params->inv_temperature, reinterpret_cast<const float2*>(norm), coef, grad_loss, row_p);
  ULORL_LAUNCH_CHECK();
  auto put_list = [&](int t0, int rows) -> int {
    const size_t n = (size_t)rows * (size_t)K;
    const unsigned blocks = (unsigned)((n + 255) / 256);
    if (pl.tensor)
      distill_put_kernel<<<blocks, 256, 0, stream>>>(rows, t0, K, V, params->inv_temperature, grad_loss, teacher_ids, entry_grad,
                                                     reinterpret_cast<__nv_bfloat16*>(ws + pl.off_panel), pl.dz_ld, pl.planes);
    else
      distill_put_kernel<<<blocks, 256, 0, stream>>>(rows, t0, K, V, params->inv_temperature, grad_loss, teacher_ids, entry_grad,
                                                     reinterpret_cast<float*>(ws + pl.off_panel), pl.dz_ld, 1);
    return check_launch();
  };
  return run_head_bwd(params, pl, hidden, W, nullptr, row_p, nullptr, true, put_list, d_hidden, d_W, ws, stream);
}

}  // extern "C"
