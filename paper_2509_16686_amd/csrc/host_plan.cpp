// Host-side validation, plan selection and workspace layout (no HIP calls).
#include "host_plan.h"

#include <algorithm>
#include <initializer_list>

namespace egmla {

namespace {
constexpr int kMaxRowDim = 640;     // d_c + d_r handled by the VALU kernel's LDS tile
constexpr int kMaxHeadDim = 1024;   // d_h and d_v
constexpr int kTargetWorkItems = 1024;
// Token-split MFMA kernel: one 4-wave work-group per compute unit streams
// longest without gaps between its loads (256 compute units).
constexpr int kTargetWorkItemsTok = 256;
// ... and its smallest automatic split, one unit for each of its four waves
// (measured with few sequences: 8 of 1000 tokens 13.8 us per call with 64-token
// splits, 16.3 with 256), while the partials of a sequence stay few (1 x 32768:
// 18.7 us with 128 partials, 19.8 with 256).
constexpr int kMaxPartialsTok = 128;
constexpr int kMergeValueDim = 128;  // value dim of the MFMA merge kernels (run_decode)
constexpr int kMinSplitTok = 64;
// The d_c 128 kernel takes the balanced schedule from this capacity on, where a
// (sequence, split) item is long enough to pay for the schedule and the second
// work-group per compute unit (up to 2 us):
// from kTokBalancedUneven tokens if the items do not fit one per compute unit
// (some then run two, and the balanced pieces win at equal lengths too), else
// only from kTokBalancedEven, where the longest sequences set the time.
// Measured, us per call without / with, lengths n / 16 to n and all n:
//   72 x 1900 (544-token items, 288 of them)  29.4 / 25.7, 32.9 / 30.7
//   200 x 1900 (two items a sequence, 400)    53.0 / 36.5, 59.2 / 50.8
//   96 x 1000 (384, 288)                      25.2 / 21.3, 27.3 / 27.3
//   64 x 4000 (1024, 256)                     29.8 / 29.9, 35.3 / 37.0
//   128 x 1000 (512, 256)                     23.3 / 25.0, 26.6 / 27.6
//   256 x 1900 (1920, 256)                    45.5 / 41.3, 55.3 / 56.7
constexpr int kTokBalancedMinCap = 1024;
constexpr int kTokBalancedUneven = 448;
constexpr int kTokBalancedEven = 1920;
// fp32 matrix-core kernel: 4-wave work-groups, two per compute unit up to
// d_c 64; above, a work-group's LDS leaves room for one (measured at batch 32,
// d_c 256, lengths to 3003: 384-token splits 42.0 us per call, 192-token 48.7).
constexpr int kTargetWorkItemsF32 = 512;

// Single-launch form: W_UK (and W_UV) bytes of a block of heads, at most.
constexpr int64_t kOneMaxWeightBytes = 128 * 1024;

int ceil_div(int64_t a, int64_t b) { return static_cast<int>((a + b - 1) / b); }
bool aligned16(const void* p) { return reinterpret_cast<uintptr_t>(p) % 16 == 0; }
}  // namespace

bool mfma_shape_supported(const eg_mla_dims& d) {
  if (d.dtype != EG_MLA_BF16) return false;
  if (d.num_heads % 16 != 0) return false;
  if (d.rope_dim != 64) return false;
  return d.latent_dim == 128 || d.latent_dim == 320 || d.latent_dim == 512;
}

bool tok_kernel_shape(const eg_mla_dims& d) { return d.latent_dim == 128 && d.rope_dim == 64; }
bool rows_kernel_shape(const eg_mla_dims& d) { return d.latent_dim == 320 && d.rope_dim == 64; }
bool heads_kernel_shape(const eg_mla_dims& d) {
  return d.latent_dim == 512 && d.rope_dim == 64 && d.head_dim == 128 && d.v_head_dim == 128 &&
         d.num_heads % kHeadsPerItemWide == 0;
}

bool f32_kernel_shape(const eg_mla_dims& d) { return d.latent_dim <= 320 && d.rope_dim <= 64; }

eg_mla_status check_dims(const eg_mla_dims* d) {
  if (!d) return EG_MLA_ERR_INVALID_ARG;
  if (d->dtype != EG_MLA_FP32 && d->dtype != EG_MLA_BF16) return EG_MLA_ERR_INVALID_ARG;
  if (d->num_heads < 1 || d->head_dim < 1 || d->v_head_dim < 1 || d->latent_dim < 1 || d->rope_dim < 0 ||
      d->vocab_size < 1 || d->page_size < 1 || d->gate_dim < 1)
    return EG_MLA_ERR_INVALID_ARG;
  if (d->softmax_scale != d->softmax_scale) return EG_MLA_ERR_INVALID_ARG;  // NaN
  if (d->gate_dim != d->latent_dim) return EG_MLA_ERR_UNSUPPORTED;
  // 16-byte vector access to latent rows, gate rows and query rows.
  const int vec = d->dtype == EG_MLA_BF16 ? 8 : 4;
  if (d->latent_dim % vec != 0 || d->rope_dim % vec != 0 || d->head_dim % vec != 0)
    return EG_MLA_ERR_UNSUPPORTED;
  if (d->latent_dim + d->rope_dim > kMaxRowDim) return EG_MLA_ERR_UNSUPPORTED;
  if (d->head_dim > kMaxHeadDim || d->v_head_dim > kMaxHeadDim) return EG_MLA_ERR_UNSUPPORTED;
  return EG_MLA_OK;
}

eg_mla_status make_decode_plan(const eg_mla_dims& d, int32_t batch, int32_t max_pages_per_seq,
                               const eg_mla_plan* plan, DecodePlan* out, PlanRows rows_rule, int32_t query_rows) {
  DecodePlan p;
  const int heads = query_rows > 0 ? query_rows : d.num_heads;
  const int forced = plan ? plan->path : EG_MLA_PATH_AUTO;
  if (forced != EG_MLA_PATH_AUTO && forced != EG_MLA_PATH_VALU && forced != EG_MLA_PATH_MFMA)
    return EG_MLA_ERR_INVALID_ARG;
  const bool mfma_ok = mfma_shape_supported(d);
  if (forced == EG_MLA_PATH_MFMA && !mfma_ok) return EG_MLA_ERR_UNSUPPORTED;
  p.path = (forced == EG_MLA_PATH_VALU || !mfma_ok) ? EG_MLA_PATH_VALU : EG_MLA_PATH_MFMA;

  const int64_t cap64 = static_cast<int64_t>(max_pages_per_seq) * d.page_size;
  if (cap64 > (1 << 30)) return EG_MLA_ERR_INVALID_ARG;
  p.capacity = static_cast<int>(cap64);

  // The vector kernel stays for the shapes the fp32 matrix-core kernel does
  // not take, for explicit splits past its token list, and when asked for.
  p.f32_mfma = rows_rule != PlanRows::kMost && p.path == EG_MLA_PATH_VALU && forced == EG_MLA_PATH_AUTO &&
               f32_kernel_shape(d) && (plan == nullptr || plan->split_tokens <= kMaxSplitTokens);
  if (p.path == EG_MLA_PATH_MFMA) {
    p.heads_per_group = heads_kernel_shape(d) ? kHeadsPerItemWide : 16;
  } else if (p.f32_mfma) {
    p.heads_per_group = 16;
  } else {
    // Heads per VALU work item: at most 8192 latent accumulators per workgroup.
    p.heads_per_group = std::max(1, std::min({heads, 8192 / d.latent_dim, 256}));
  }
  p.head_groups = ceil_div(heads, p.heads_per_group);

  const int req_slices = plan ? plan->id_slices : 0;
  if (req_slices != 0 && req_slices != 1 && req_slices != kIdSlices) return EG_MLA_ERR_INVALID_ARG;
  const bool sliced_kernel = p.path == EG_MLA_PATH_MFMA && tok_kernel_shape(d);
  // automatic: no slices (measured faster on MI355X: a sliced work item must
  // resolve its token ids before its first cache-row load)
  p.slices = sliced_kernel && req_slices == kIdSlices ? kIdSlices : 1;
  const bool rows_kernel = p.path == EG_MLA_PATH_MFMA && rows_kernel_shape(d);
  // kernels whose waves own whole units of tokens take short splits
  const bool unit_kernel = rows_rule == PlanRows::kFast && ((sliced_kernel && p.slices == 1) || rows_kernel);
  const int max_split = sliced_kernel ? kMaxSliceSplitTokens : kMaxSplitTokens;

  int split = plan ? plan->split_tokens : 0;
  if (split < 0 || split % kTile != 0) return EG_MLA_ERR_INVALID_ARG;
  if (p.path == EG_MLA_PATH_MFMA && split > max_split) return EG_MLA_ERR_UNSUPPORTED;
  if (split == 0) {
    // Work items (splits x slices) to fill the chip: each work item of the
    // sliced kernel handles 1/slices of its split's tokens.
    const int64_t work =
        static_cast<int64_t>(std::max(batch, 1)) * std::max(p.capacity, 1) * p.head_groups * p.slices;
    const int64_t target =
        p.path == EG_MLA_PATH_MFMA && (tok_kernel_shape(d) || heads_kernel_shape(d)) ? kTargetWorkItemsTok
        // (measured: 256 x 2048 117 us per call against 122 with two work-groups
        // per compute unit, 32 x 4096 42.5 against 47.9)
        : rows_kernel && rows_rule != PlanRows::kMost ? kTargetWorkItemsTok
        : p.f32_mfma ? (d.latent_dim <= 64 ? kTargetWorkItemsF32 : kTargetWorkItemsF32 / 2)
                     : kTargetWorkItems;
    int64_t s = (work + target - 1) / target;
    const int gran = p.slices > 1 ? 256 : kTile;  // sliced kernel: whole 256-position scan rows
    s = (s + gran - 1) / gran * gran;
    const int min_split = unit_kernel ? kMinSplitTok
                          : p.path == EG_MLA_PATH_MFMA || p.f32_mfma ? 256
                                                                     : 128;
    p.target_items = static_cast<int>(target);
    p.min_split = min_split;
    p.max_split = max_split;
    s = std::max<int64_t>(s, min_split);
    if (unit_kernel) s = std::max<int64_t>(s, (p.capacity / kMaxPartialsTok + kTile - 1) / kTile * kTile);
    // the general merge reads a sequence's partials one after the other: no more
    // than 16 for the sake of short splits (d_v 64, 1 x 4096: 64 partials 21.6 us
    // per call, 16 18.4; 1 x 2048: 32 18.0, 16 17.0)
    if (unit_kernel && d.v_head_dim != kMergeValueDim && s < 256)
      s = std::max<int64_t>(s, std::min(256, ceil_div(p.capacity, 16 * kTile) * kTile));
    if (sliced_kernel && unit_kernel && s < 256) {
      const int64_t per_split = static_cast<int64_t>(std::max(batch, 1)) * p.head_groups;
      const int cap = std::max(p.capacity, 1);
      auto cut = [&](int n) { return std::max(kMinSplitTok, ceil_div(cap, n * kTile) * kTile); };
      // Short splits only where the items still run one per compute unit (48 x
      // 1000: 288 items of 192 tokens 18.8 us per call, 192 of 256 17.1); up to
      // 4 sequences of 4096 no more than 32 a sequence, which the kernel can
      // absorb the query with (below; 4 x 4096: 32 splits of 128 15.1 us in a
      // graph, 64 of 64 and a launch more 14.5, but a host needs 13 to 17 to
      // enqueue its three launches, 10.5 to 12 for two).  With 17 to 32 sequences 8 a
      // sequence rather than some number between 8 and 16: the absorption is
      // then shared evenly, and 8 partials merge in small work-groups; up to 192
      // tokens each (us per call: as above / 8 splits / of 256 tokens):
      //   20 x 1300  17.6 / 16.1 / 17.2    24 x 1500  18.3 / 16.6 / 17.3
      //   28 x 1100  18.0 / 16.5 / 17.3    20 x 900   16.6 / 15.9 / 17.0
      // and 256 tokens from there to 2048 (24 x 1600 18.2 / 17.7 / 17.3, 28 x
      // 1800 19.9 / 18.6 / 18.7); above, more than 8 splits are due anyway
      // (20 x 2300 18.1 / 18.7 / 19.1).
      if (per_split <= 4 && cap <= 32 * 128)
        s = std::max<int64_t>(s, cut(32));
      else if (per_split > 16 && 8 * per_split <= kTargetWorkItemsTok && cap <= 8 * 256)
        s = cut(8) <= 192 ? cut(8) : 256;
      else if (per_split * ceil_div(cap, static_cast<int>(s)) > kTargetWorkItemsTok)
        s = per_split <= 16 && cut(16) < 256 ? cut(16) : 256;  // (12 x 2048, not 264 items: 16 splits 15.7, 256 tokens 17.0)
    }
    s = std::min<int64_t>(s, max_split);
    split = static_cast<int>(s);
  }
  p.split_tokens = split;
  p.s_max = std::max(1, ceil_div(std::max(p.capacity, 1), split));
  // One launch instead of three where a work-group can afford its heads'
  // weights (read whole by every sequence) and its whole context, and all
  // work-groups are resident at once.
  p.one_launch = p.f32_mfma && (plan == nullptr || plan->split_tokens == 0) && p.capacity > 0 &&
                 p.capacity <= kOneMaxTokens && d.latent_dim <= kOneMaxLatent &&
                 static_cast<int64_t>(std::min(heads, 16)) * std::max(d.head_dim, d.v_head_dim) * d.latent_dim *
                         elem_bytes(d) <= kOneMaxWeightBytes &&
                 static_cast<int64_t>(std::max(batch, 0)) * p.head_groups <= kTargetWorkItemsF32;
  // The head-split kernel balances tokens over its work-groups whatever the
  // length mix; its split size only caps the token list it stages at a time.
  p.balanced = p.path == EG_MLA_PATH_MFMA && heads_kernel_shape(d);
  if (p.balanced && (plan == nullptr || plan->split_tokens == 0)) p.split_tokens = kMaxSplitTokens;

  const size_t B = static_cast<size_t>(std::max(batch, 0));
  const size_t H = static_cast<size_t>(heads);
  const size_t DQ = static_cast<size_t>(d.latent_dim + d.rope_dim);
  // The split kernel absorbs the query itself when that costs each work-group
  // at most 2 heads' W_UK (8 or more splits per sequence, the first 16 of them
  // producers) and every work-group is resident at once (2 per compute unit);
  // otherwise (many splits, whose extra work-groups only wait, or a batch of
  // several rounds of work-groups each reading 4 or more heads' W_UK) the
  // absorption kernel runs first (measured: B32 L4096 25.2 against 25.7 us
  // per call; B4 L32768 28.9 against 27.8; B256 L2048 70.8 against 59.4).  Of
  // 17 to 32 splits the short ones take it, where waiting for the producers
  // costs no more than the launch they save: the two run about as long (2 x
  // 1856 13.6 / 13.7 us in a graph, 12 x 1280 14.7 / 14.5; 8 x 3000, 256 items,
  // 16.0 / 15.4), but a step of append and decode is then four launches, not
  // five, and a host has to enqueue them: 2 x 1856 22.9 us against 25.7.
  const int64_t nblk = static_cast<int64_t>(std::max(batch, 0)) * p.s_max * p.head_groups;
  const bool short_splits = unit_kernel && (plan == nullptr || plan->split_tokens == 0) && p.s_max <= 32 &&
                            (p.split_tokens <= kMinSplitTok || (p.split_tokens <= 128 && nblk <= 224));
  p.fused_absorb = sliced_kernel && p.slices == 1 && d.head_dim == 128 && p.s_max >= 8 &&
                   (p.s_max <= 16 || short_splits) && nblk <= 2 * kTargetWorkItemsTok;
  auto layout = [&]() {
    const size_t rows = p.balanced       ? kWideMaxGroups + B
                        : p.tok_balanced ? static_cast<size_t>(p.pieces)
                                         : B * static_cast<size_t>(p.s_max) * static_cast<size_t>(p.slices);
    size_t off = 0;
    p.off_q = off;
    off = align_up(off + B * H * DQ * 4);
    p.off_ml = off;
    off = align_up(off + rows * H * 2 * 4);
    // partial outputs: fp32 sums, or (wide kernel) fp16 rows normalised by their sums
    p.off_o = off;
    off = align_up(off + rows * H * static_cast<size_t>(d.latent_dim) * (p.balanced ? 2 : 4));
    if (p.balanced || p.tok_balanced) {
      p.off_sched = off;
      off = align_up(off + 16 + (p.balanced ? kWideMaxGroups * 8 : static_cast<size_t>(p.pieces) * 16) + B * 8);
    }
    if (p.fused_absorb) {
      p.off_flags = off;
      off = align_up(off + B * static_cast<size_t>(p.head_groups) * static_cast<size_t>(p.s_max) * 8);
    }
    return off;
  };
  size_t off = layout();
  // Few splits per sequence: a work-group's time follows its sequence's
  // length, so the d_c 128 kernel takes the balanced schedule, two
  // work-groups per compute unit.  Not beyond the batch where the dispatcher
  // itself evens out the work-groups, nor where the search's largest piece (about
  // N / (pieces - batch), see tok_sizes) could outgrow the token list, nor where the extra partial rows would take a call that fits
  // the workspace-free entry's scratch out of it.
  if (rows_rule == PlanRows::kFast && sliced_kernel && p.slices == 1 && !p.fused_absorb && d.head_dim == 128 && batch > 32 && p.s_max < 8 &&
      (plan == nullptr || plan->split_tokens == 0) && p.capacity >= kTokBalancedMinCap &&
      p.split_tokens >= (nblk > kTargetWorkItemsTok ? kTokBalancedUneven : kTokBalancedEven) &&
      batch <= kTokMaxBatch) {
    const int pieces = kTokMaxPieces / p.head_groups / 8 * 8;
    if (pieces > batch &&
        static_cast<int64_t>(batch) * p.capacity / (pieces - batch) < max_split - 128) {
      const size_t plain = off;
      p.tok_balanced = true;
      p.pieces = pieces;
      off = layout();
      if (off > plain && off > EG_MLA_NOALLOC_SCRATCH_BYTES && plain <= EG_MLA_NOALLOC_SCRATCH_BYTES) {
        p.tok_balanced = false;
        p.pieces = 0;
        off = layout();
      }
    }
  }
  p.bytes = std::max<size_t>(off, kAlign);
  *out = p;
  return EG_MLA_OK;
}

eg_mla_status fit_decode_plan(const eg_mla_dims& d, int32_t batch, int32_t max_pages_per_seq, const eg_mla_plan* plan,
                              size_t workspace_bytes, DecodePlan* out) {
  eg_mla_status st = make_decode_plan(d, batch, max_pages_per_seq, plan, out);
  if (st != EG_MLA_OK || out->bytes <= workspace_bytes) return st;
  st = make_decode_plan(d, batch, max_pages_per_seq, plan, out, PlanRows::kFew);
  return st != EG_MLA_OK || out->bytes <= workspace_bytes ? st : EG_MLA_ERR_WORKSPACE;
}

size_t decode_workspace_bytes(const eg_mla_dims& d, int32_t batch, int32_t max_pages_per_seq, const eg_mla_plan* plan) {
  size_t bytes = 0;
  for (const PlanRows rows : {PlanRows::kFast, PlanRows::kFew, PlanRows::kMost}) {
    DecodePlan p;
    if (make_decode_plan(d, batch, max_pages_per_seq, plan, &p, rows) != EG_MLA_OK) return 0;
    bytes = std::max(bytes, p.bytes);
  }
  return bytes;
}

eg_mla_status validate_decode(const eg_mla_dims* d, int32_t batch, const void* q, const void* latent_cache,
                              const int32_t* token_id_cache, const void* gate_table, const void* w_uk,
                              const void* w_uv, const int32_t* seq_lens, int32_t max_pages_per_seq,
                              int64_t num_slots, const int32_t* page_table, const void* workspace,
                              size_t workspace_bytes, const void* out, const eg_mla_plan* plan, DecodePlan* p) {
  eg_mla_status st = check_dims(d);
  if (st != EG_MLA_OK) return st;
  if (batch < 0 || max_pages_per_seq < 0 || num_slots < 0) return EG_MLA_ERR_INVALID_ARG;
  if (num_slots >= (int64_t{1} << 31)) return EG_MLA_ERR_UNSUPPORTED;  // 32-bit row indices in the kernels
  const eg_mla_status fit = fit_decode_plan(*d, batch, max_pages_per_seq, plan, workspace_bytes, p);
  if (fit != EG_MLA_OK && fit != EG_MLA_ERR_WORKSPACE) return fit;
  if (batch == 0) return EG_MLA_OK;
  if (!q || !gate_table || !w_uk || !w_uv || !seq_lens || !out) return EG_MLA_ERR_INVALID_ARG;
  if (max_pages_per_seq > 0 && (!latent_cache || !token_id_cache)) return EG_MLA_ERR_INVALID_ARG;
  if (!page_table) {
    // contiguous rows: every sequence's capacity must fit in the cache
    const int64_t need = static_cast<int64_t>(batch) * max_pages_per_seq * d->page_size;
    if (need > num_slots) return EG_MLA_ERR_INVALID_ARG;
  } else if (num_slots < d->page_size && max_pages_per_seq > 0) {
    return EG_MLA_ERR_INVALID_ARG;
  }
  // 16-byte vector loads of rows and weights
  if (!aligned16(q) || !aligned16(latent_cache) || !aligned16(gate_table) || !aligned16(w_uk) || !aligned16(w_uv))
    return EG_MLA_ERR_INVALID_ARG;
  if (!workspace || fit != EG_MLA_OK) return EG_MLA_ERR_WORKSPACE;
  if (reinterpret_cast<uintptr_t>(workspace) % kAlign != 0) return EG_MLA_ERR_WORKSPACE;
  return EG_MLA_OK;
}

eg_mla_status validate_append(const eg_mla_dims* d, int32_t n_tokens, int32_t hidden, const void* x,
                              const int32_t* token_ids, const int32_t* positions, const int32_t* slots,
                              const void* w_dkv, const void* latent_cache, const int32_t* token_id_cache,
                              int64_t num_slots) {
  eg_mla_status st = check_dims(d);
  if (st != EG_MLA_OK) return st;
  if (n_tokens < 0 || hidden < 1 || num_slots < 0) return EG_MLA_ERR_INVALID_ARG;
  if (hidden > 32768) return EG_MLA_ERR_UNSUPPORTED;  // x row staged in LDS
  if (d->rope_dim % 2 != 0) return EG_MLA_ERR_INVALID_ARG;
  if (n_tokens == 0) return EG_MLA_OK;
  if (!x || !token_ids || !positions || !slots || !w_dkv || !latent_cache || !token_id_cache)
    return EG_MLA_ERR_INVALID_ARG;
  return EG_MLA_OK;
}

eg_mla_status validate_gate_rows(const eg_mla_dims* d, int32_t emb_dim, int32_t emb_vocab, int64_t n,
                                 const int32_t* ids, const void* emb, const void* w_ue, const void* out) {
  eg_mla_status st = check_dims(d);
  if (st != EG_MLA_OK) return st;
  if (emb_dim < 1 || emb_vocab < 1 || n < 0) return EG_MLA_ERR_INVALID_ARG;
  if (emb_dim > 16384) return EG_MLA_ERR_UNSUPPORTED;  // one embedding row staged in LDS (VALU kernel)
  if (n == 0) return EG_MLA_OK;
  if (!ids || !emb || !w_ue || !out) return EG_MLA_ERR_INVALID_ARG;
  return EG_MLA_OK;
}

size_t prefill_workspace_bytes(const eg_mla_dims& d, int32_t seq_len) {
  const size_t T = static_cast<size_t>(std::max(seq_len, 0));
  const size_t H = static_cast<size_t>(d.num_heads);
  // fp32 explicit keys [H, T, d_h + d_r] and values [H, T, d_v]
  size_t k = align_up(H * T * static_cast<size_t>(d.head_dim + d.rope_dim) * 4);
  size_t v = align_up(H * T * static_cast<size_t>(d.v_head_dim) * 4);
  return std::max<size_t>(k + v, kAlign);
}

eg_mla_status validate_prefill(const eg_mla_dims* d, int32_t seq_len, const void* q, const void* latent,
                               const int32_t* token_ids, const void* gate_table, const void* w_uk,
                               const void* w_uv, const void* workspace, size_t workspace_bytes,
                               const void* out) {
  eg_mla_status st = check_dims(d);
  if (st != EG_MLA_OK) return st;
  if (seq_len < 0) return EG_MLA_ERR_INVALID_ARG;
  if (seq_len > 32768) return EG_MLA_ERR_UNSUPPORTED;  // one score row staged in LDS
  if (seq_len == 0) return EG_MLA_OK;
  if (!q || !latent || !token_ids || !gate_table || !w_uk || !w_uv || !out) return EG_MLA_ERR_INVALID_ARG;
  if (!workspace || workspace_bytes < prefill_workspace_bytes(*d, seq_len)) return EG_MLA_ERR_WORKSPACE;
  if (reinterpret_cast<uintptr_t>(workspace) % kAlign != 0) return EG_MLA_ERR_WORKSPACE;
  return EG_MLA_OK;
}

bool prefill_varlen_absorbed(const eg_mla_dims& d) {
  return d.dtype == EG_MLA_BF16 && d.num_heads == 16 && d.head_dim == 128 && d.v_head_dim == 128 &&
         d.latent_dim == 128 && d.rope_dim == 64 && d.gate_dim == d.latent_dim;
}

bool prefill_varlen_shape_ok(const eg_mla_dims& d) {
  if (prefill_varlen_absorbed(d)) return true;
  // the explicit form: any head count, d_c a multiple of 64
  return d.dtype == EG_MLA_BF16 && d.head_dim == 128 && d.v_head_dim == 128 && d.rope_dim == 64 &&
         d.latent_dim % 64 == 0 && d.gate_dim == d.latent_dim;
}

PrefillVarlenLayout prefill_varlen_layout(const eg_mla_dims& d, int32_t total_tokens) {
  const size_t T = static_cast<size_t>(std::max(total_tokens, 0));
  const size_t H = static_cast<size_t>(d.num_heads);
  PrefillVarlenLayout L;
  L.off_seq_start = 0;  // int32 [T]
  if (prefill_varlen_absorbed(d)) {
    // the size is that of query rows of d_c + d_r, whose RoPE part the attention reads from
    // the query: the blocks' order lies in the part of them that is left
    L.off_qf = align_up(T * 4);                                                    // fp16 [T][H][d_c]
    L.off_order = L.off_qf + align_up(T * H * static_cast<size_t>(d.latent_dim) * 2);  // int2 [ceil(T / 8)]
    L.off_olat = L.off_qf + align_up(T * H * static_cast<size_t>(d.latent_dim + d.rope_dim) * 2);  // fp16 [T][H][d_c]
    L.off_ct = L.off_olat + align_up(T * H * static_cast<size_t>(d.latent_dim) * 2);   // fp16 [T][d_c]
    L.bytes = std::max<size_t>(L.off_ct + align_up(T * static_cast<size_t>(d.latent_dim) * 2), kAlign);
  } else {
    L.off_qf = align_up(T * 4);                                                  // K^C: fp16 [H][T][d_h]
    L.off_olat = L.off_qf + align_up(T * H * static_cast<size_t>(d.head_dim) * 2);  // V: fp16 [H][T][d_v]
    L.off_ct = L.off_olat + align_up(T * H * static_cast<size_t>(d.v_head_dim) * 2);  // bf16 hi, lo [2][T][d_c]
    L.bytes = std::max<size_t>(L.off_ct + 2 * align_up(T * static_cast<size_t>(d.latent_dim) * 2), kAlign);
  }
  return L;
}

eg_mla_status validate_prefill_varlen(const eg_mla_dims* d, int32_t batch, int32_t total_tokens,
                                      const int32_t* cu_seqlens, const void* q, const void* latent,
                                      const int32_t* token_ids, const void* gate_table, const void* w_uk,
                                      const void* w_uv, const void* workspace, size_t workspace_bytes,
                                      const void* out) {
  eg_mla_status st = check_dims(d);
  if (st != EG_MLA_OK) return st;
  if (batch < 1 || total_tokens < 0) return EG_MLA_ERR_INVALID_ARG;
  if (!prefill_varlen_shape_ok(*d)) return EG_MLA_ERR_UNSUPPORTED;
  if (total_tokens == 0) return EG_MLA_OK;
  if (!cu_seqlens || !q || !latent || !token_ids || !gate_table || !w_uk || !w_uv || !out)
    return EG_MLA_ERR_INVALID_ARG;
  if (!aligned16(q) || !aligned16(latent) || !aligned16(gate_table) || !aligned16(w_uk) || !aligned16(w_uv) ||
      !aligned16(out))
    return EG_MLA_ERR_INVALID_ARG;
  if (!workspace || workspace_bytes < prefill_varlen_layout(*d, total_tokens).bytes) return EG_MLA_ERR_WORKSPACE;
  if (reinterpret_cast<uintptr_t>(workspace) % kAlign != 0) return EG_MLA_ERR_WORKSPACE;
  return EG_MLA_OK;
}

bool literal_tile_shape(const eg_mla_dims& d) {
  return d.dtype == EG_MLA_BF16 && d.latent_dim == 128 && d.head_dim == 128 && d.v_head_dim == 128 &&
         d.rope_dim == 64 && d.num_heads <= 160 && literal_lds_bytes(d.num_heads, 1) <= 160 * 1024;
}

size_t literal_generic_lds_bytes(const eg_mla_dims& d) {
  // latents of a group of 8 tokens, key dots and weights [8][H], moment sums
  // [4][8][2], per-token figures [3][8], per-head sums [2][H] and softmax
  // state [3][H], value sums [H][d_v] (all fp32)
  const size_t H = static_cast<size_t>(d.num_heads);
  return 4 * (8 * static_cast<size_t>(d.latent_dim) + 16 * H + 64 + 24 + 5 * H +
              H * static_cast<size_t>(d.v_head_dim));
}

size_t literal_lds_bytes(int num_heads, int groups) {
  // per head group: weight / gate-tile region, value sums [4][d_v] and, for two
  // groups, the tokens' moments [3][4][32]; per-wave scores [4][H][32], two
  // sums per head, per-wave figures per head, token means [4][32] (all fp32)
  return static_cast<size_t>(groups) * (272 * 256 + 4 * 128 * 4 + (groups > 1 ? 3 * 4 * 32 * 4 : 0)) +
         4 * static_cast<size_t>(num_heads) * 32 * 4 + static_cast<size_t>(num_heads) * (2 + 12) * 4 + 4 * 32 * 4;
}

int literal_head_groups(int num_heads) {
  return num_heads % 2 == 0 && literal_lds_bytes(num_heads, 2) <= 160 * 1024 ? 2 : 1;
}

size_t literal_workspace_bytes(const eg_mla_dims& d, int32_t batch, int32_t max_pages_per_seq) {
  const int64_t cap = static_cast<int64_t>(std::max(max_pages_per_seq, 0)) * d.page_size;
  const int64_t tiles = (cap + 127) / 128;
  return std::max<size_t>(align_up(static_cast<size_t>(std::max(batch, 0)) * static_cast<size_t>(tiles) *
                                   d.num_heads * (d.v_head_dim + 4) * sizeof(float)),
                          kAlign);
}

eg_mla_status validate_literal(const eg_mla_dims* d, int32_t batch, const void* q, const void* latent_cache,
                               const int32_t* token_id_cache, const void* gate_full, const void* w_uk,
                               const void* w_uv, const void* ln_w, const void* ln_b, uint32_t flags,
                               const int32_t* seq_lens, const int32_t* page_table, int32_t max_pages_per_seq,
                               int64_t num_slots, const void* workspace, size_t workspace_bytes, const void* out) {
  eg_mla_status st = check_dims(d);
  if (st != EG_MLA_OK) return st;
  if (batch < 0 || max_pages_per_seq < 0 || num_slots < 0) return EG_MLA_ERR_INVALID_ARG;
  if ((flags & ~(EG_MLA_LITERAL_NO_LN | EG_MLA_LITERAL_ADD)) != 0) return EG_MLA_ERR_INVALID_ARG;
  if (literal_tile_shape(*d)) {
    // gate rows are addressed by 32-bit byte offsets in the tile kernel
    if (static_cast<int64_t>(d->vocab_size) * d->num_heads * (d->head_dim + d->v_head_dim) * 2 >=
        (int64_t{1} << 32))
      return EG_MLA_ERR_UNSUPPORTED;
  } else if (literal_generic_lds_bytes(*d) > 160 * 1024) {
    return EG_MLA_ERR_UNSUPPORTED;  // the generic kernel's tile state does not fit in LDS
  }
  if (static_cast<int64_t>(max_pages_per_seq) * d->page_size > (int64_t{1} << 30)) return EG_MLA_ERR_UNSUPPORTED;
  if (num_slots >= (int64_t{1} << 31)) return EG_MLA_ERR_UNSUPPORTED;
  if (batch == 0) return EG_MLA_OK;
  if (!q || !gate_full || !w_uk || !w_uv || !seq_lens || !out || !latent_cache || !token_id_cache)
    return EG_MLA_ERR_INVALID_ARG;
  if (max_pages_per_seq < 1 || num_slots < 1) return EG_MLA_ERR_INVALID_ARG;
  if (!page_table && static_cast<int64_t>(batch) * max_pages_per_seq * d->page_size > num_slots)
    return EG_MLA_ERR_INVALID_ARG;  // contiguous rows: every sequence's capacity must fit in the cache
  if ((flags & EG_MLA_LITERAL_NO_LN) == 0 && (!ln_w || !ln_b)) return EG_MLA_ERR_INVALID_ARG;
  if (!aligned16(q) || !aligned16(latent_cache) || !aligned16(gate_full) || !aligned16(w_uk) || !aligned16(w_uv))
    return EG_MLA_ERR_INVALID_ARG;
  if (!workspace || workspace_bytes < literal_workspace_bytes(*d, batch, max_pages_per_seq))
    return EG_MLA_ERR_WORKSPACE;
  if (reinterpret_cast<uintptr_t>(workspace) % kAlign != 0) return EG_MLA_ERR_WORKSPACE;
  return EG_MLA_OK;
}

namespace {

// Arrays of a call that must not overlap (a null one takes no room).
struct Span {
  const void* p;
  int64_t bytes;
};
bool overlap(const Span& a, const Span& b) {
  if (!a.p || !b.p || a.bytes <= 0 || b.bytes <= 0) return false;
  const uintptr_t x = reinterpret_cast<uintptr_t>(a.p), y = reinterpret_cast<uintptr_t>(b.p);
  return x < y ? y - x < static_cast<uintptr_t>(a.bytes) : x - y < static_cast<uintptr_t>(b.bytes);  // (no end wraps round)
}
// Product of non-negative sizes, held at the largest: an array of that many bytes meets every one behind it.
int64_t held_product(int64_t a, int64_t b) {
  int64_t r;
  return __builtin_mul_overflow(a, b, &r) ? INT64_MAX : r;
}
// Whether any of the outputs overlaps another output or an input.
bool outputs_overlap(std::initializer_list<Span> outs, std::initializer_list<Span> ins) {
  for (const Span* o = outs.begin(); o != outs.end(); ++o) {
    for (const Span* q = o + 1; q != outs.end(); ++q)
      if (overlap(*o, *q)) return true;
    for (const Span& i : ins)
      if (overlap(*o, i)) return true;
  }
  return false;
}

constexpr int64_t kMaxCapacity = int64_t{1} << 30;  // tokens of a sequence's row of the page table, array lengths

// The cache and page table of a call over `batch` sequences of max_pages pages.
eg_mla_status check_pages(const eg_mla_dims& d, int32_t batch, int32_t max_pages, int64_t num_slots, bool paged) {
  if (batch < 0 || max_pages < 0 || num_slots < 0) return EG_MLA_ERR_INVALID_ARG;
  if (num_slots >= (int64_t{1} << 31)) return EG_MLA_ERR_UNSUPPORTED;
  const int64_t cap = static_cast<int64_t>(max_pages) * d.page_size;
  if (cap > kMaxCapacity) return EG_MLA_ERR_INVALID_ARG;
  if (batch == 0 || max_pages == 0) return EG_MLA_OK;
  if (!paged && cap > num_slots / batch) return EG_MLA_ERR_INVALID_ARG;  // contiguous rows must fit in the cache
  return num_slots < d.page_size ? EG_MLA_ERR_INVALID_ARG : EG_MLA_OK;
}

}  // namespace

eg_mla_status validate_page_plan(int32_t batch, int32_t page_size, int32_t max_pages_per_seq, int32_t max_tokens,
                                 const int32_t* cached_lens, const int32_t* new_lens, const int32_t* position_base,
                                 const int32_t* page_table, const int32_t* free_pages, const int32_t* free_count,
                                 int32_t free_capacity, const int32_t* seq_lens, const int32_t* cu_seqlens,
                                 const int32_t* positions, const int32_t* slots, const int32_t* free_count_out) {
  if (batch < 0 || page_size < 1 || max_pages_per_seq < 0 || max_tokens < 0 || free_capacity < 0)
    return EG_MLA_ERR_INVALID_ARG;
  if (static_cast<int64_t>(max_pages_per_seq) * page_size > kMaxCapacity || max_tokens > kMaxCapacity ||
      free_capacity > kMaxCapacity)
    return EG_MLA_ERR_INVALID_ARG;
  if (batch > kPageMaxBatch) return EG_MLA_ERR_UNSUPPORTED;
  if (batch == 0) return EG_MLA_OK;
  if (!cached_lens || !new_lens || !free_count || !seq_lens || !cu_seqlens || !free_count_out)
    return EG_MLA_ERR_INVALID_ARG;
  if ((max_pages_per_seq > 0 && !page_table) || (free_capacity > 0 && !free_pages) ||
      (max_tokens > 0 && (!positions || !slots)))
    return EG_MLA_ERR_INVALID_ARG;
  // every work-group reads the inputs for itself while others write
  const int64_t n = 4 * static_cast<int64_t>(batch), t = 4 * static_cast<int64_t>(max_tokens);
  if (outputs_overlap({{seq_lens, n}, {cu_seqlens, n + 4}, {positions, t}, {slots, t}, {free_count_out, 4},
                       {page_table, n * max_pages_per_seq}},
                      {{cached_lens, n}, {new_lens, n}, {position_base, n}, {free_count, 4},
                       {free_pages, 4 * static_cast<int64_t>(free_capacity)}}))
    return EG_MLA_ERR_INVALID_ARG;
  return EG_MLA_OK;
}

eg_mla_status validate_page_release(int32_t batch, int32_t page_size, int32_t max_pages_per_seq,
                                    const int32_t* seq_lens, const int32_t* ended, const int32_t* page_table,
                                    const int32_t* free_pages, const int32_t* free_count, int32_t free_capacity,
                                    const int32_t* seq_lens_out, const int32_t* free_count_out) {
  if (batch < 0 || page_size < 1 || max_pages_per_seq < 0 || free_capacity < 0) return EG_MLA_ERR_INVALID_ARG;
  if (static_cast<int64_t>(max_pages_per_seq) * page_size > kMaxCapacity || free_capacity > kMaxCapacity)
    return EG_MLA_ERR_INVALID_ARG;
  if (batch > kPageMaxBatch) return EG_MLA_ERR_UNSUPPORTED;
  if (batch == 0) return EG_MLA_OK;
  if (!seq_lens || !ended || !free_count || !seq_lens_out || !free_count_out) return EG_MLA_ERR_INVALID_ARG;
  if ((max_pages_per_seq > 0 && !page_table) || (free_capacity > 0 && !free_pages)) return EG_MLA_ERR_INVALID_ARG;
  const int64_t n = 4 * static_cast<int64_t>(batch);
  if (outputs_overlap({{seq_lens_out, n}, {free_count_out, 4}, {free_pages, 4 * static_cast<int64_t>(free_capacity)}},
                      {{seq_lens, n}, {ended, n}, {free_count, 4}, {page_table, n * max_pages_per_seq}}))
    return EG_MLA_ERR_INVALID_ARG;
  return EG_MLA_OK;
}

eg_mla_status validate_qk(const eg_mla_dims* d, int32_t n_tokens, const void* q, int64_t q_stride,
                          const void* q_norm_w, const void* q_out, const void* kv, int64_t kv_stride,
                          const void* kv_norm_w, const void* k_norm_w, const int32_t* token_ids,
                          const int32_t* positions, const int32_t* slots, float rope_theta, const void* latent_cache,
                          const int32_t* token_id_cache, int64_t num_slots) {
  const eg_mla_status st = check_dims(d);
  if (st != EG_MLA_OK) return st;
  if (n_tokens < 0 || num_slots < 0) return EG_MLA_ERR_INVALID_ARG;
  if (rope_theta > 3.4e38f) return EG_MLA_ERR_INVALID_ARG;  // infinite
  if (n_tokens == 0) return EG_MLA_OK;
  if (!q && !kv) return EG_MLA_ERR_INVALID_ARG;
  if (d->rope_dim > 0 && !positions) return EG_MLA_ERR_INVALID_ARG;
  const int eb = elem_bytes(*d), vec = 16 / eb;
  const int64_t row = d->latent_dim + d->rope_dim, n = n_tokens;
  const int64_t q_row = static_cast<int64_t>(d->num_heads) * (d->head_dim + d->rope_dim);
  constexpr int64_t kMaxStride = int64_t{1} << 32;
  if (q) {
    if (!q_out || q_stride < q_row || q_stride % vec != 0 || q_stride > kMaxStride) return EG_MLA_ERR_INVALID_ARG;
    if (!aligned16(q) || !aligned16(q_out) || !aligned16(q_norm_w)) return EG_MLA_ERR_INVALID_ARG;
  }
  if (kv) {
    if (!latent_cache || !token_id_cache || !token_ids || !slots) return EG_MLA_ERR_INVALID_ARG;
    if (kv_stride < row || kv_stride % vec != 0 || kv_stride > kMaxStride) return EG_MLA_ERR_INVALID_ARG;
    if (!aligned16(kv) || !aligned16(kv_norm_w) || !aligned16(k_norm_w) || !aligned16(latent_cache))
      return EG_MLA_ERR_INVALID_ARG;
  }
  // the rotated query may take its source's place where the rows are the same; nothing else may overlap
  const Span qs{q, held_product((n - 1) * q_stride + q_row, eb)}, ks{kv, held_product((n - 1) * kv_stride + row, eb)};
  const Span qo{q ? q_out : nullptr, held_product(n * eb, q_row)}, cache{kv ? latent_cache : nullptr, held_product(num_slots, row * eb)};
  const Span ids{kv ? token_id_cache : nullptr, held_product(num_slots, 4)};
  const Span qw{q ? q_norm_w : nullptr, static_cast<int64_t>(d->head_dim + d->rope_dim) * eb};
  const Span kw{kv ? kv_norm_w : nullptr, static_cast<int64_t>(d->latent_dim) * eb};
  const Span rw{kv ? k_norm_w : nullptr, static_cast<int64_t>(d->rope_dim) * eb};
  const bool in_place = q && q == q_out && q_stride == q_row;
  if ((!in_place && overlap(qs, qo)) || overlap(cache, qs) || overlap(ids, qs) ||
      outputs_overlap({qo, cache, ids}, {ks, qw, kw, rw, {positions, 4 * n}, {kv ? token_ids : nullptr, 4 * n},
                                         {kv ? slots : nullptr, 4 * n}}))
    return EG_MLA_ERR_INVALID_ARG;
  return EG_MLA_OK;
}

bool page_scores_mfma(const eg_mla_dims& d) {
  return d.dtype == EG_MLA_BF16 && (d.head_dim == 64 || d.head_dim == 128);
}

size_t page_scores_workspace_bytes(const eg_mla_dims& d, int32_t batch) {
  const int64_t n = std::max(batch, 0), dq = d.latent_dim + d.rope_dim;
  const int64_t runs = ceil_div(dq, 32) + 2 * ceil_div(d.latent_dim, 32);
  const int64_t bytes = page_scores_mfma(d) ? held_product(n * ceil_div(d.num_heads, 16), runs * 1024)
                                            : held_product(n * d.num_heads, dq * 4);
  return std::max<size_t>(align_up(static_cast<size_t>(bytes)), kAlign);
}

eg_mla_status validate_page_means(const eg_mla_dims* d, int32_t batch, const void* latent_cache,
                                  const int32_t* token_id_cache, const void* gate_table, const int32_t* first_tokens,
                                  const int32_t* seq_lens, const int32_t* page_table, int32_t max_pages_per_seq,
                                  int64_t num_slots, const void* page_means) {
  eg_mla_status st = check_dims(d);
  if (st != EG_MLA_OK) return st;
  st = check_pages(*d, batch, max_pages_per_seq, num_slots, page_table != nullptr);
  if (st != EG_MLA_OK || batch == 0 || max_pages_per_seq == 0) return st;
  if (!latent_cache || !token_id_cache || !gate_table || !seq_lens || !page_means) return EG_MLA_ERR_INVALID_ARG;
  if (!aligned16(latent_cache) || !aligned16(gate_table) || !aligned16(page_means)) return EG_MLA_ERR_INVALID_ARG;
  const int64_t eb = elem_bytes(*d), row = (d->latent_dim + d->rope_dim) * eb, n = 4 * static_cast<int64_t>(batch);
  if (outputs_overlap({{page_means, num_slots / d->page_size * row}},
                      {{latent_cache, num_slots * row}, {token_id_cache, num_slots * 4},
                       {gate_table, eb * d->vocab_size * d->latent_dim}, {first_tokens, n}, {seq_lens, n},
                       {page_table, n * max_pages_per_seq}}))
    return EG_MLA_ERR_INVALID_ARG;
  return EG_MLA_OK;
}

eg_mla_status validate_page_scores(const eg_mla_dims* d, int32_t batch, const void* q, const void* w_uk,
                                   const void* page_means, const int32_t* seq_lens, const int32_t* page_table,
                                   int32_t max_pages_per_seq, int64_t num_slots, const void* workspace,
                                   size_t workspace_bytes, const float* scores) {
  eg_mla_status st = check_dims(d);
  if (st != EG_MLA_OK) return st;
  st = check_pages(*d, batch, max_pages_per_seq, num_slots, page_table != nullptr);
  if (st != EG_MLA_OK || batch == 0 || max_pages_per_seq == 0) return st;
  if (!q || !w_uk || !page_means || !seq_lens || !scores) return EG_MLA_ERR_INVALID_ARG;
  if (!aligned16(q) || !aligned16(w_uk) || !aligned16(page_means)) return EG_MLA_ERR_INVALID_ARG;
  const size_t need = page_scores_workspace_bytes(*d, batch);
  if (!workspace || workspace_bytes < need) return EG_MLA_ERR_WORKSPACE;
  if (reinterpret_cast<uintptr_t>(workspace) % kAlign != 0) return EG_MLA_ERR_WORKSPACE;
  const int64_t eb = elem_bytes(*d), n = 4 * static_cast<int64_t>(batch), h = d->num_heads, dc = d->latent_dim;
  if (outputs_overlap({{scores, n * max_pages_per_seq}, {workspace, static_cast<int64_t>(need)}},
                      {{q, held_product(batch * h, (d->head_dim + d->rope_dim) * eb)}, {w_uk, h * d->head_dim * dc * eb},
                       {page_means, num_slots / d->page_size * (dc + d->rope_dim) * eb}, {seq_lens, n},
                       {page_table, n * max_pages_per_seq}}))
    return EG_MLA_ERR_INVALID_ARG;
  return EG_MLA_OK;
}

eg_mla_status validate_select_pages(const eg_mla_dims* d, int32_t batch, const float* scores, const int32_t* seq_lens,
                                    const int32_t* page_table, int32_t max_pages_per_seq, int32_t keep,
                                    int32_t keep_first, int32_t keep_last, const int32_t* sel_pages,
                                    const int32_t* sel_lens, const int32_t* sel_index) {
  const eg_mla_status st = check_dims(d);
  if (st != EG_MLA_OK) return st;
  if (batch < 0 || max_pages_per_seq < 0 || keep_first < 0 || keep_last < 1 ||
      static_cast<int64_t>(keep_first) + keep_last > keep)
    return EG_MLA_ERR_INVALID_ARG;
  if (static_cast<int64_t>(max_pages_per_seq) * d->page_size > kMaxCapacity) return EG_MLA_ERR_INVALID_ARG;
  const int64_t entries = static_cast<int64_t>(batch) * max_pages_per_seq;
  if (!page_table && entries > 0x7fffffff) return EG_MLA_ERR_INVALID_ARG;  // page numbers are 32-bit
  if (batch == 0) return EG_MLA_OK;
  if (!seq_lens || !sel_pages || !sel_lens || (max_pages_per_seq > 0 && !scores)) return EG_MLA_ERR_INVALID_ARG;
  const int64_t n = 4 * static_cast<int64_t>(batch);
  const int64_t kept = held_product(n, keep), all = held_product(4, entries);
  if (outputs_overlap({{sel_pages, kept}, {sel_lens, n}, {sel_index, kept}},
                      {{seq_lens, n}, {page_table, all}, {scores, all}}))
    return EG_MLA_ERR_INVALID_ARG;
  return EG_MLA_OK;
}

namespace {

// The split kernel of one part of a shared decode, `rows` query rows a
// sequence: the decode's plan without its absorption, the d_c 128 schedule and
// the single-launch form (the call absorbs once for both parts and merges them
// itself).
eg_mla_status shared_part_plan(const eg_mla_dims& d, int32_t batch, int32_t rows, int32_t max_pages, DecodePlan* p) {
  const eg_mla_status st = make_decode_plan(d, batch, max_pages, nullptr, p, PlanRows::kFast, rows);
  if (st != EG_MLA_OK) return st;
  p->fused_absorb = p->one_launch = p->tok_balanced = false;
  p->pieces = 0;
  if (p->path == EG_MLA_PATH_VALU && !p->f32_mfma) {
    // the vector kernel's queries and probabilities of a group of heads lie in LDS
    while (p->heads_per_group > 1 &&
           4 * static_cast<int64_t>(p->heads_per_group) * (d.latent_dim + d.rope_dim + kTile + 1) > 64 * 1024)
      p->heads_per_group /= 2;
    p->head_groups = ceil_div(rows, p->heads_per_group);
  }
  if (p->capacity > 0 && static_cast<int64_t>(batch) * p->s_max * p->head_groups > 0x7fffffff)
    return EG_MLA_ERR_UNSUPPORTED;
  return EG_MLA_OK;
}

// Work-groups of the prefix kernel for `tiles` 64-key tiles over all row blocks.  More of them share the tiles out
// evenly but write more fp32 partial rows for the merge to read; two fit a compute unit at d_c 128, one above.
// Measured, us a call with 128 / 256 / 512 (prefix 8192 but for the last two, 16 to 100 own tokens):
//   d_c 128, 16 heads   1 sequence (128 tiles)  20.2 /  21.4 / 22.2   d_c 320   16 (256)    43.3 / 46.1
//                      16 (256)                 25.7 /  30.1 / 36.9             32 (512)    48.1 / 49.2
//                      32 (512)                 27.1 /  30.4 / 36.2             64 (1024)   56.7 / 54.2
//                      64 (1024)                31.6 /  32.4 / 35.8            128 (2048)   73.6 / 64.1
//                     128 (2048)                44.6 /  37.3 / 39.4
//                     256 (4096)                65.1 /  47.9 / 50.1
//                     256 of 16384 (8192)      107.8 /  71.0 / 70.8
//                     256 of 32768 (16384)     192.8 / 116.1 / 111.4
constexpr int64_t kPrefixFewTiles = 1024, kPrefixManyTiles = 8192;
int prefix_groups(const eg_mla_dims& d, int64_t tiles) {
  if (d.latent_dim < 512 && tiles < kPrefixFewTiles) return 128;
  return d.latent_dim == 128 && tiles >= kPrefixManyTiles ? 512 : 256;
}

// d_c 128: prefix and own tokens in one launch up to this many tiles.  Hiding the own tokens gains less and less, its
// 32-key tiles cost more (us a call in two launches / one, 16 heads, up to 100 own tokens and up to 1000):
//     64 x  8192 (1024 tiles)    39.0 /  32.9     41.3 /  31.4
//    256 x 16384 (8192)          75.9 /  71.6     89.7 /  80.8
//    256 x 32768 (16384)        115.5 / 112.8    129.2 / 122.2
//    256 x 49152 (24576)        155.9 / 155.2    168.9 / 163.4
//    256 x 65536 (32768)        194.6 / 195.6    208.4 / 205.1
constexpr int64_t kBothMaxTiles = 16384;

// Tiled prefix attention: the layers that the decode takes with the same
// roundings, whatever the rows (one sequence of 16 heads, an eighth of a row
// block, prefix 8000: 19.7 us against 86 with the decode's split kernel, whose
// merge reads its many partial rows).
bool prefix_tiled(const eg_mla_dims& d) {
  return mfma_shape_supported(d) && d.head_dim == 128 && d.v_head_dim == 128;
}

// Partial rows that a part's automatic plan has at most for `rows` query rows
// of all its sequences, or for fewer of them or a smaller capacity: whole
// splits of the smallest size, and items of up to `heads` rows, of which there
// are target_items and one more a sequence and group of heads, or those of the
// largest split.  A workspace of this size serves every smaller call too.
int64_t part_rows(const DecodePlan& p, int64_t rows) {
  if (p.capacity == 0) return 0;
  const int64_t heads = p.path == EG_MLA_PATH_VALU && !p.f32_mfma ? 256 : 16;
  return std::min(rows * ceil_div(p.capacity, p.min_split),
                  std::max(heads * p.target_items, rows * p.capacity / p.max_split) + rows);
}

// The same of the decode's own plan, and its workspace in all (make_decode_plan's layout).
size_t plain_bytes(const eg_mla_dims& d, int32_t batch, const DecodePlan& p) {
  const int64_t q_rows = static_cast<int64_t>(batch) * d.num_heads;
  int64_t rows = part_rows(p, q_rows);
  if (p.balanced) rows = (int64_t{kWideMaxGroups} + batch) * d.num_heads;
  else if (p.path == EG_MLA_PATH_MFMA && tok_kernel_shape(d) && batch > 32) rows = std::max<int64_t>(rows, kTokMaxPieces * 16);
  const size_t dq = static_cast<size_t>(d.latent_dim + d.rope_dim);
  return align_up(q_rows * dq * 4) + align_up(rows * 8) + align_up(rows * static_cast<size_t>(d.latent_dim) * (p.balanced ? 2 : 4)) +
         align_up(16 + kTokMaxPieces * 16 + static_cast<size_t>(batch) * 8) + align_up(2 * kTargetWorkItemsTok * 8);
}

}  // namespace

eg_mla_status make_shared_plan(const eg_mla_dims& d, int32_t batch, int32_t max_pages_per_seq,
                               int32_t max_prefix_pages, SharedPlan* out) {
  SharedPlan p;
  // all heads of all sequences are the prefix's heads; merge grid
  const int64_t rows64 = static_cast<int64_t>(batch) * d.num_heads;
  if (rows64 > (1 << 30) || batch > 65535) return EG_MLA_ERR_UNSUPPORTED;
  DecodePlan plain;  // a call without prefix pages is this decode; others leave its room
  eg_mla_status st = make_decode_plan(d, batch, max_pages_per_seq, nullptr, &plain);
  if (st != EG_MLA_OK) return st;
  const size_t least = plain_bytes(d, batch, plain);
  if (max_prefix_pages == 0 && max_pages_per_seq > 0) {
    p.plain = true;
    p.own = plain;
    p.bytes = least;
    *out = p;
    return EG_MLA_OK;
  }
  st = shared_part_plan(d, 1, std::max(1, batch * d.num_heads), max_prefix_pages, &p.pre);
  p.tiled = p.pre.capacity > 0 && rows64 > 0 && prefix_tiled(d);
  if (st == EG_MLA_OK) st = shared_part_plan(d, batch, d.num_heads, max_pages_per_seq, &p.own);
  if (st != EG_MLA_OK) return st;
  const size_t rows = static_cast<size_t>(rows64), dc = static_cast<size_t>(d.latent_dim), dq = dc + d.rope_dim;
  size_t off = 0;
  auto take = [&](size_t bytes) {
    const size_t at = off;
    off = align_up(off + bytes);
    return at;
  };
  if (p.tiled) {
    p.row_blocks = ceil_div(rows64, kPrefixRows);
    const int64_t work = static_cast<int64_t>(p.row_blocks) * ceil_div(p.pre.capacity, 64);  // 64-key tiles of all rows
    p.both = d.latent_dim == 128 && p.own.capacity > 0 && p.own.path == EG_MLA_PATH_MFMA &&
             p.own.split_tokens <= kBothList && work <= kBothMaxTiles &&
             static_cast<int64_t>(batch) * p.own.s_max * p.own.head_groups < (1 << 30);
    p.keys = d.latent_dim == 512 || p.both ? 32 : 64;
    const int tiles = ceil_div(p.pre.capacity, p.keys);
    p.fused = d.latent_dim == 512 && d.num_heads % kPrefixRows == 0;  // a row block within a sequence
    p.half_rows = heads_kernel_shape(d);
    // the fused kernel's work-groups take the own tokens too, whose tiles may be the more
    const int most = p.fused ? std::max(tiles, ceil_div(p.own.capacity, 32)) : tiles;
    const int groups = prefix_groups(d, work);
    p.splits = std::max(1, std::min(groups / p.row_blocks, most));
    if (static_cast<int64_t>(p.row_blocks) * p.splits > 0x3fffffff) return EG_MLA_ERR_UNSUPPORTED;
    p.off_half = take(rows * dq * 2);
    if (!p.own.balanced) p.off_q = take(rows * dq * 4);
    // tiles of either size, and what fewer rows in more splits would need (part_rows)
    p.off_tiles = take(static_cast<size_t>(ceil_div(p.pre.capacity, 64)) * 64 * (prefix_latent_row(d.latent_dim) + 128));
    if (p.fused) p.off_rows = take(static_cast<size_t>(batch) * 8);
    const size_t tiles32 = static_cast<size_t>(ceil_div(std::max(p.pre.capacity, p.fused ? p.own.capacity : 0), 32));
    const size_t n = std::min(rows * tiles32, std::max(rows, static_cast<size_t>(kPrefixRows) * groups));
    p.pre.off_ml = take(n * 8);
    p.pre.off_o = take(n * dc * (p.half_rows ? 2 : 4));
  } else {
    p.off_q = take(rows * dq * 4);
    const size_t n = static_cast<size_t>(part_rows(p.pre, rows64));
    p.pre.off_ml = take(n * 8);
    p.pre.off_o = take(n * dc * 4);
  }
  if (p.own.capacity > 0 && !p.fused) {
    const size_t n = p.own.balanced ? (static_cast<size_t>(kWideMaxGroups) + batch) * d.num_heads
                                    : static_cast<size_t>(part_rows(p.own, rows64));
    p.own.off_ml = take(n * 8);
    p.own.off_o = take(n * dc * (p.own.balanced ? 2 : 4));
    if (p.own.balanced) p.own.off_sched = take(16 + kWideMaxGroups * 8 + static_cast<size_t>(batch) * 8);
  }
  p.bytes = std::max({off, least, kAlign});
  *out = p;
  return EG_MLA_OK;
}

eg_mla_status validate_decode_shared(const eg_mla_dims* d, int32_t batch, const void* q, const void* latent_cache,
                                     const int32_t* token_id_cache, const void* gate_table, const void* w_uk,
                                     const void* w_uv, const int32_t* prefix_len, const int32_t* prefix_table,
                                     int32_t max_prefix_pages, const int32_t* seq_lens, const int32_t* page_table,
                                     int32_t max_pages_per_seq, int64_t num_slots, const void* workspace,
                                     size_t workspace_bytes, const void* out, SharedPlan* p) {
  eg_mla_status st = check_dims(d);
  if (st != EG_MLA_OK) return st;
  st = check_pages(*d, batch, max_pages_per_seq, num_slots, page_table != nullptr);
  if (st == EG_MLA_OK) st = check_pages(*d, std::min(batch, 1), max_prefix_pages, num_slots, true);
  if (st != EG_MLA_OK) return st;
  st = make_shared_plan(*d, batch, max_pages_per_seq, max_prefix_pages, p);
  if (st != EG_MLA_OK || batch == 0) return st;
  if (!q || !gate_table || !w_uk || !w_uv || !out) return EG_MLA_ERR_INVALID_ARG;
  if (max_prefix_pages > 0 && (!prefix_len || !prefix_table)) return EG_MLA_ERR_INVALID_ARG;
  if (max_pages_per_seq > 0 && !seq_lens) return EG_MLA_ERR_INVALID_ARG;
  if ((max_prefix_pages > 0 || max_pages_per_seq > 0) && (!latent_cache || !token_id_cache))
    return EG_MLA_ERR_INVALID_ARG;
  if (!aligned16(q) || !aligned16(latent_cache) || !aligned16(gate_table) || !aligned16(w_uk) || !aligned16(w_uv) ||
      !aligned16(out))
    return EG_MLA_ERR_INVALID_ARG;
  if (!workspace || workspace_bytes < p->bytes) return EG_MLA_ERR_WORKSPACE;
  if (reinterpret_cast<uintptr_t>(workspace) % kAlign != 0) return EG_MLA_ERR_WORKSPACE;
  const int64_t eb = elem_bytes(*d), n = 4 * static_cast<int64_t>(batch), h = d->num_heads, dc = d->latent_dim;
  if (outputs_overlap({{out, batch * h * d->v_head_dim * eb}, {workspace, static_cast<int64_t>(p->bytes)}},
                      {{q, batch * h * (d->head_dim + d->rope_dim) * eb}, {latent_cache, num_slots * (dc + d->rope_dim) * eb},
                       {token_id_cache, num_slots * 4}, {gate_table, d->vocab_size * dc * eb},
                       {w_uk, h * d->head_dim * dc * eb}, {w_uv, h * d->v_head_dim * dc * eb}, {prefix_len, 4},
                       {prefix_table, 4 * static_cast<int64_t>(max_prefix_pages)}, {seq_lens, n},
                       {page_table, n * max_pages_per_seq}}))
    return EG_MLA_ERR_INVALID_ARG;
  return EG_MLA_OK;
}

namespace {

// Frequencies and magnitude of a rotation.
eg_mla_status check_rope(const eg_mla_rope* r, int32_t rope_dim) {
  if (!r) return EG_MLA_ERR_INVALID_ARG;
  if (r->layout != EG_MLA_ROPE_PAIRS && r->layout != EG_MLA_ROPE_HALF) return EG_MLA_ERR_INVALID_ARG;
  if (r->theta != r->theta || r->theta > 3.4e38f || r->magnitude != r->magnitude || r->magnitude > 3.4e38f)
    return EG_MLA_ERR_INVALID_ARG;
  for (int m = 0; r->frequencies && m < rope_dim / 2; ++m)
    if (!(r->frequencies[m] >= -64.0 && r->frequencies[m] <= 64.0)) return EG_MLA_ERR_INVALID_ARG;
  return EG_MLA_OK;
}

constexpr int kMaxRopeDim = 640;
constexpr int kMaxRowHeads = 1 << 30;  // (a head's number and a work-group's step of heads in 32 bits)
constexpr int64_t kMaxRowStride = int64_t{1} << 32;
constexpr int kQ8MaxLatent = 512, kQ8MaxRopeDim = 64;
constexpr int64_t kQ8MaxTiles = int64_t{1} << 23;  // tiles of 16 queries, a head and 64 latent values (work-groups of the absorption)
constexpr int kQ8MaxQueries = 1 << 19;
// Blocks of 128 query rows instead of 16: from so many rows a sequence on average, and so many products (rows x capacity
// x (2 d_c + d_r)), below which their longer start is the time.  us a call with blocks of 16 / 128, tokens of each
// sequence in brackets:
//   16 heads d_c 128, 32 x 4096:  [2] 29.2 / 35.7  [3] 39.3 / 37.0  [4] 37.7 / 37.8  [6] 50.9 / 41.2  [16] 87.1 / 55.0
//   16 heads d_c 128, 8 x 500:    [4] 21.3 / 24.7  [16] 22.3 / 29.0;  4 x 32768:  [4] 38.4 / 38.8  [8] 56.3 / 44.2
//   12 heads d_c 64, 32 x 4096:   [2] 25.9 / 29.1  [3] 33.6 / 29.2  [4] 33.9 / 29.6  [16] 64.3 / 40.4
//   16 heads d_c 320, 32 x 4096:  [1] 35.4 / 50.8  [2] 45.1 / 54.3  [3] 73.2 / 64.4  [4] 66.4 / 60.0  [16] 182 / 98.5
//   128 heads d_c 512, 8 x 4096:  [1] 87.1 / 57.7  [16] 871 / 230;  1 x 30000:  [1] 98.0 / 55.6
//   5 heads d_c 48, 16 x 3000:    [16] 23.3 / 24.5
// (The capacity stands for the lengths, which only the device knows: a table for the longest context takes blocks of 128
// for short ones too.)
constexpr int kQ8ManyRows = 48;
constexpr int64_t kQ8ManyProducts = 600000000;
constexpr int kQ8MaxRuns = 512;

}  // namespace

eg_mla_status validate_rope_rows(const eg_mla_rope* rope, int32_t dtype, int32_t n_tokens, int32_t num_heads,
                                 int32_t head_dim, int32_t rope_offset, int32_t rope_dim, const void* x,
                                 int64_t x_token_stride, int64_t x_head_stride, const int32_t* positions, const void* out,
                                 int64_t out_token_stride, int64_t out_head_stride) {
  if (dtype != EG_MLA_FP32 && dtype != EG_MLA_BF16) return EG_MLA_ERR_INVALID_ARG;
  if (n_tokens < 0 || num_heads < 1 || head_dim < 1 || rope_offset < 0 || rope_dim < 0 || rope_dim % 2 != 0 ||
      rope_dim > head_dim || rope_offset > head_dim - rope_dim)
    return EG_MLA_ERR_INVALID_ARG;
  if (num_heads > kMaxRowHeads) return EG_MLA_ERR_UNSUPPORTED;
  const eg_mla_status st = rope_dim <= kMaxRopeDim ? check_rope(rope, rope_dim) : EG_MLA_ERR_UNSUPPORTED;
  if (st != EG_MLA_OK) return st;
  if (n_tokens == 0) return EG_MLA_OK;
  if (!x || !out || !positions) return EG_MLA_ERR_INVALID_ARG;
  const int64_t eb = dtype == EG_MLA_BF16 ? 2 : 4, n = n_tokens, h = num_heads, d = head_dim;
  if (reinterpret_cast<uintptr_t>(x) % eb != 0 || reinterpret_cast<uintptr_t>(out) % eb != 0) return EG_MLA_ERR_INVALID_ARG;
  for (const int64_t s : {x_token_stride, x_head_stride, out_token_stride, out_head_stride})
    if (s < 0 || s > kMaxRowStride) return EG_MLA_ERR_INVALID_ARG;
  // rows of the output must be apart: heads within tokens, or tokens within heads
  const int64_t ot = n > 1 ? out_token_stride : kMaxRowStride * h, oh = h > 1 ? out_head_stride : kMaxRowStride * n;
  if (!((oh >= d && ot >= (h - 1) * out_head_stride + d) || (ot >= d && oh >= (n - 1) * out_token_stride + d)))
    return EG_MLA_ERR_INVALID_ARG;
  auto room = [&](int64_t ts, int64_t hs) {
    return held_product(eb, std::min(held_product(n - 1, ts), INT64_MAX / 4) + std::min(held_product(h - 1, hs), INT64_MAX / 4) + d);
  };
  const bool in_place = x == out && (n == 1 || x_token_stride == out_token_stride) && (h == 1 || x_head_stride == out_head_stride);
  const Span os{out, room(out_token_stride, out_head_stride)};
  if ((!in_place && overlap(os, {x, room(x_token_stride, x_head_stride)})) || overlap(os, {positions, 4 * n}))
    return EG_MLA_ERR_INVALID_ARG;
  return EG_MLA_OK;
}

eg_mla_status check_q8_dims(const eg_mla_dims* d) {
  const eg_mla_status st = check_dims(d);
  if (st != EG_MLA_OK) return st;
  if (d->dtype != EG_MLA_BF16 || d->latent_dim % 16 != 0 || d->latent_dim > kQ8MaxLatent || d->rope_dim > kQ8MaxRopeDim)
    return EG_MLA_ERR_UNSUPPORTED;
  return EG_MLA_OK;
}

eg_mla_status validate_q8_write(const eg_mla_dims* d, const eg_mla_rope* rope, int32_t n_tokens, const void* kv,
                                int64_t kv_stride, const void* kv_norm_w, const void* k_norm_w, const void* gate_table,
                                const int32_t* token_ids, const int32_t* positions, const int32_t* slots,
                                const uint8_t* codes, const uint8_t* scales, int64_t num_slots) {
  eg_mla_status st = check_q8_dims(d);
  if (st == EG_MLA_OK && rope) st = check_rope(rope, d->rope_dim);
  if (st != EG_MLA_OK) return st;
  if (n_tokens < 0 || num_slots < 0) return EG_MLA_ERR_INVALID_ARG;
  if (n_tokens == 0) return EG_MLA_OK;
  if (!kv || !slots || !codes || !scales || (gate_table && !token_ids) || (rope && d->rope_dim > 0 && !positions))
    return EG_MLA_ERR_INVALID_ARG;
  const int64_t row = d->latent_dim + d->rope_dim, n = n_tokens;
  if (kv_stride < row || kv_stride % 8 != 0 || kv_stride > kMaxRowStride) return EG_MLA_ERR_INVALID_ARG;
  if (!aligned16(kv) || !aligned16(kv_norm_w) || !aligned16(gate_table) || !aligned16(codes)) return EG_MLA_ERR_INVALID_ARG;
  if (outputs_overlap({{codes, held_product(num_slots, q8_row_bytes(*d))}, {scales, num_slots}},
                      {{kv, held_product((n - 1) * kv_stride + row, 2)}, {kv_norm_w, 2 * d->latent_dim},
                       {k_norm_w, 2 * d->rope_dim}, {gate_table, int64_t{2} * d->vocab_size * d->latent_dim},
                       {gate_table ? token_ids : nullptr, 4 * n}, {rope && d->rope_dim ? positions : nullptr, 4 * n},
                       {slots, 4 * n}}))
    return EG_MLA_ERR_INVALID_ARG;
  return EG_MLA_OK;
}

eg_mla_status validate_q8_read(const eg_mla_dims* d, int32_t batch, int32_t total_tokens, const uint8_t* codes,
                               const uint8_t* scales, const int32_t* first_tokens, const int32_t* cu_seqlens,
                               const int32_t* page_table, int32_t max_pages_per_seq, int64_t num_slots, const void* out) {
  eg_mla_status st = check_q8_dims(d);
  if (st != EG_MLA_OK) return st;
  if (total_tokens < 0) return EG_MLA_ERR_INVALID_ARG;
  st = check_pages(*d, batch, max_pages_per_seq, num_slots, page_table != nullptr);
  if (st == EG_MLA_OK && batch > kPageMaxBatch) st = EG_MLA_ERR_UNSUPPORTED;
  if (st != EG_MLA_OK || batch == 0 || total_tokens == 0 || max_pages_per_seq == 0) return st;
  if (!codes || !scales || !cu_seqlens || !out) return EG_MLA_ERR_INVALID_ARG;
  if (!aligned16(codes) || !aligned16(out)) return EG_MLA_ERR_INVALID_ARG;
  const int64_t n = 4 * static_cast<int64_t>(batch);
  if (outputs_overlap({{out, int64_t{2} * total_tokens * (d->latent_dim + d->rope_dim)}},
                      {{codes, num_slots * q8_row_bytes(*d)}, {scales, num_slots}, {first_tokens, n}, {cu_seqlens, n + 4},
                       {page_table, n * max_pages_per_seq}}))
    return EG_MLA_ERR_INVALID_ARG;
  return EG_MLA_OK;
}

eg_mla_status make_q8_plan(const eg_mla_dims& d, int32_t batch, int32_t n_queries, int32_t max_pages_per_seq, Q8Plan* out) {
  if (batch < 0 || n_queries < 0 || max_pages_per_seq < 0) return EG_MLA_ERR_INVALID_ARG;
  const int64_t cap = static_cast<int64_t>(max_pages_per_seq) * d.page_size;
  if (cap > kMaxCapacity) return EG_MLA_ERR_INVALID_ARG;
  const int64_t rows = static_cast<int64_t>(n_queries) * d.num_heads;
  if (batch > kPageMaxBatch || n_queries > kQ8MaxQueries ||
      held_product(ceil_div(n_queries, 16) * int64_t{d.num_heads}, ceil_div(d.latent_dim, 64)) > kQ8MaxTiles)
    return EG_MLA_ERR_UNSUPPORTED;
  Q8Plan p;
  p.capacity = static_cast<int>(cap);
  const bool many = rows >= int64_t{kQ8ManyRows} * batch &&
                    held_product(held_product(rows, cap), 2 * d.latent_dim + d.rope_dim) >= kQ8ManyProducts;
  p.block_rows = many ? 128 : 16;
  p.tile = many ? (d.latent_dim <= 128 ? 64 : 32) : d.latent_dim <= 128 ? 128 : 64;
  // one work-group a compute unit where registers or LDS leave room for one, else two
  p.runs = many && d.latent_dim > 128 ? 256 : kQ8MaxRuns;
  // (us a call at lead 0, 4, 8, 12: 64 x 512-16384 x 128 heads 238, 226, 216, 219; chunks of 200-600 tokens x 16 heads
  // 270, 203, 210, 216; blocks of 16, 256 x 250-8192: 70.7, 69.7, 71.7, 75.8)
  p.lead = many ? 4 : 0;
  p.blocks = rows / p.block_rows + batch;
  if (held_product(p.blocks, cap / p.tile + 1 + p.lead) >= (int64_t{1} << 31)) return EG_MLA_ERR_UNSUPPORTED;
  size_t at = 0;
  auto take = [&](int64_t bytes) {
    const size_t here = at;
    at += align_up(static_cast<size_t>(bytes));
    return here;
  };
  // partial rows: bounds that grow with the batch and the queries, of either size of block, so that a workspace serves
  // every smaller call
  const int64_t small = 16 * (kQ8MaxRuns + rows / 16 + batch);
  const int64_t large = 128 * ((d.latent_dim > 128 ? 256 : kQ8MaxRuns) + rows / 128 + batch);
  p.off_q = take(rows * (d.latent_dim + d.rope_dim) * 2);
  const int64_t most = rows / 16 + batch;
  p.off_info = take(most * 16);
  p.off_rows = take(most * 16);
  p.off_start = take(kQ8MaxRuns * int64_t{48});
  p.off_tokens = take(n_queries * int64_t{8});
  p.off_head = take(16);
  p.off_ml = take(std::max(small, large) * 8);
  p.off_o = take(std::max(small, large) * 4 * d.latent_dim);
  p.bytes = at;
  *out = p;
  return EG_MLA_OK;
}

eg_mla_status validate_q8_attend(const eg_mla_dims* d, int32_t batch, int32_t n_queries, const void* q,
                                 const int32_t* cu_seqlens, const uint8_t* codes, const uint8_t* scales, const void* w_uk,
                                 const void* w_uv, const int32_t* seq_lens, const int32_t* page_table,
                                 int32_t max_pages_per_seq, int64_t num_slots, const void* workspace,
                                 size_t workspace_bytes, const void* out, Q8Plan* p) {
  eg_mla_status st = check_q8_dims(d);
  if (st != EG_MLA_OK) return st;
  st = check_pages(*d, batch, max_pages_per_seq, num_slots, page_table != nullptr);
  if (st == EG_MLA_OK) st = make_q8_plan(*d, batch, n_queries, max_pages_per_seq, p);
  if (st != EG_MLA_OK) return st;
  if (!cu_seqlens && n_queries != batch) return EG_MLA_ERR_INVALID_ARG;
  if (batch == 0 || n_queries == 0) return EG_MLA_OK;
  if (!q || !w_uk || !w_uv || !seq_lens || !out || (max_pages_per_seq > 0 && (!codes || !scales)))
    return EG_MLA_ERR_INVALID_ARG;
  if (!aligned16(q) || !aligned16(codes) || !aligned16(w_uk) || !aligned16(w_uv) || !aligned16(out))
    return EG_MLA_ERR_INVALID_ARG;
  if (!workspace || workspace_bytes < p->bytes) return EG_MLA_ERR_WORKSPACE;
  if (reinterpret_cast<uintptr_t>(workspace) % kAlign != 0) return EG_MLA_ERR_WORKSPACE;
  const int64_t n = 4 * static_cast<int64_t>(batch), h = d->num_heads, dc = d->latent_dim;
  const int64_t rows = n_queries * h;
  if (outputs_overlap({{out, rows * d->v_head_dim * 2}, {workspace, static_cast<int64_t>(p->bytes)}},
                      {{q, rows * (d->head_dim + d->rope_dim) * 2}, {cu_seqlens, n + 4},
                       {codes, num_slots * q8_row_bytes(*d)}, {scales, num_slots},
                       {w_uk, held_product(h, d->head_dim * dc * 2)}, {w_uv, held_product(h, d->v_head_dim * dc * 2)},
                       {seq_lens, n}, {page_table, n * max_pages_per_seq}}))
    return EG_MLA_ERR_INVALID_ARG;
  return EG_MLA_OK;
}

}  // namespace egmla

extern "C" {

const char* eg_mla_status_string(eg_mla_status s) {
  switch (s) {
    case EG_MLA_OK: return "EG_MLA_OK";
    case EG_MLA_ERR_INVALID_ARG: return "EG_MLA_ERR_INVALID_ARG: invalid argument";
    case EG_MLA_ERR_UNSUPPORTED: return "EG_MLA_ERR_UNSUPPORTED: shape or option not supported";
    case EG_MLA_ERR_WORKSPACE: return "EG_MLA_ERR_WORKSPACE: workspace missing, misaligned or too small";
    case EG_MLA_ERR_HIP: return "EG_MLA_ERR_HIP: HIP runtime or launch failure";
  }
  return "EG_MLA_ERR_UNKNOWN";
}

eg_mla_status eg_mla_check_dims(const eg_mla_dims* dims) { return egmla::check_dims(dims); }

size_t eg_mla_decode_workspace_size(const eg_mla_dims* dims, int32_t batch, int32_t max_pages_per_seq,
                                    const eg_mla_plan* plan) {
  if (egmla::check_dims(dims) != EG_MLA_OK || batch < 0 || max_pages_per_seq < 0) return 0;
  return egmla::decode_workspace_bytes(*dims, batch, max_pages_per_seq, plan);
}

size_t eg_mla_prefill_workspace_size(const eg_mla_dims* dims, int32_t seq_len) {
  if (egmla::check_dims(dims) != EG_MLA_OK || seq_len < 0) return 0;
  return egmla::prefill_workspace_bytes(*dims, seq_len);
}

size_t eg_mla_prefill_varlen_workspace_size(const eg_mla_dims* dims, int32_t total_tokens) {
  if (egmla::check_dims(dims) != EG_MLA_OK || total_tokens < 0 || !egmla::prefill_varlen_shape_ok(*dims)) return 0;
  return egmla::prefill_varlen_layout(*dims, total_tokens).bytes;
}

}  // extern "C"
