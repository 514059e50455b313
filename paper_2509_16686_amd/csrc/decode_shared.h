// Decode of a batch whose sequences share a prefix (included by decode.hip).
//
// All heads of all sequences attend to the same latents (App. C Eq. (C.13) in
// the absorbed form), so the batch's attention over the shared prefix is the
// attention of one sequence with B H heads: its rows are read and gated once
// for every query row a work-group holds instead of once per sequence.  Each
// sequence's own tokens run as in eg_mla_decode, and a merge joins both
// parts' partial softmaxes:
//   m = max_s m_s,  o = sum_s o_s 2^(m_s - m) / sum_s l_s 2^(m_s - m)   over the splits of both,
//   out[b,h] = W_UV[h] o.
#pragma once

#include "shared_prefix.h"

namespace egmla {

// Partial rows of one part: row (s, i) of query row i is at s * stride + i * step.
struct SharedPart {
  const float* ml;         // [rows, 2] running max (log2 domain), sum
  const float* o;          // [rows, DC] unnormalised
  const int32_t* lens;     // device lengths: [B] or one
  int32_t cap, split, s_max;
};

// Merge and up-projection of any shape: grid (H, B), 256 threads; the latent
// columns of a row are thread t's t, t + 256, t + 512.
constexpr int kSharedCols = 3;  // d_c <= 640

template <bool BF16>
__global__ __launch_bounds__(256) void shared_combine_kernel(SharedPart pre, SharedPart own,
                                                             const void* __restrict__ w_uv, void* __restrict__ out,
                                                             int B, int H, int DC, int DV) {
  extern __shared__ float o_s[];  // [DC]
  const int h = blockIdx.x, b = blockIdx.y;
  float M = -INFINITY, sum = 0.f, acc[kSharedCols] = {0.f, 0.f, 0.f};
  constexpr int U = 8;  // rows in flight
  auto fold = [&](const SharedPart& p, int64_t row0, int64_t step, int len) {
    const int ns = min((clamp_len(len, p.cap) + p.split - 1) / p.split, p.s_max);
    for (int s0 = 0; s0 < ns; s0 += U) {
      float2 ml[U];
      float v[U][kSharedCols];
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const int64_t row = row0 + min(s0 + u, ns - 1) * step;
        ml[u] = *reinterpret_cast<const float2*>(p.ml + 2 * row);
#pragma unroll
        for (int k = 0; k < kSharedCols; ++k) {
          const int c = threadIdx.x + 256 * k;
          v[u][k] = c < DC ? p.o[row * DC + c] : 0.f;
        }
      }
      float Mn = M;
#pragma unroll
      for (int u = 0; u < U; ++u) Mn = fmaxf(Mn, ml[u].x);  // repeats of the last row change no maximum
      const bool any = Mn > -INFINITY;  // else nothing weighs anything yet; rows are added all the same, for a NaN's sake
      const float keep = any ? exp2f(M - Mn) : 1.f;
      M = Mn;
      sum *= keep;
#pragma unroll
      for (int k = 0; k < kSharedCols; ++k) acc[k] *= keep;
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const float e = any && s0 + u < ns ? exp2f(ml[u].x - Mn) : 0.f;  // exp2(-inf) = 0
        sum = fmaf(e, ml[u].y, sum);
#pragma unroll
        for (int k = 0; k < kSharedCols; ++k) acc[k] = fmaf(e, v[u][k], acc[k]);
      }
    }
  };
  if (pre.s_max > 0) fold(pre, static_cast<int64_t>(b) * H + h, static_cast<int64_t>(B) * H, pre.lens[0]);
  if (own.s_max > 0) fold(own, static_cast<int64_t>(b) * own.s_max * H + h, H, own.lens[b]);
  const float inv = sum == 0.f ? 0.f : 1.f / sum;
#pragma unroll
  for (int k = 0; k < kSharedCols; ++k) {
    const int c = threadIdx.x + 256 * k;
    if (c < DC) o_s[c] = acc[k] * inv;
  }
  __syncthreads();
  const int64_t wbase = static_cast<int64_t>(h) * DV * DC;
  for (int v = threadIdx.x; v < DV; v += 256) {
    float r = 0.f;
    for (int c = 0; c < DC; c += 4) {
      const float4 wv = ld4<BF16>(w_uv, wbase + static_cast<int64_t>(v) * DC + c);
      r = fmaf(wv.x, o_s[c], r);
      r = fmaf(wv.y, o_s[c + 1], r);
      r = fmaf(wv.z, o_s[c + 2], r);
      r = fmaf(wv.w, o_s[c + 3], r);
    }
    st<BF16>(out, (static_cast<int64_t>(b) * H + h) * DV + v, r);
  }
}

namespace {

// Everything a shared decode's launches read.
struct SharedCall {
  const eg_mla_dims& d;
  const SharedPlan& p;
  int32_t batch;
  const void *q, *cache;
  const int32_t* ids;
  const void *gate, *w_uk, *w_uv;
  const int32_t *prefix_len, *prefix_table;
  int32_t max_prefix_pages;
  const int32_t *seq_lens, *page_table;
  int32_t max_pages;
  int64_t num_slots;
  unsigned char* ws;
  void* out;
  hipStream_t stream;
};

// Sequences of a merge work-group: 16, or fewer while that leaves under one work-group per compute unit.
constexpr int kSharedMergeGroups = 256;

// Partial rows of a sequence up to which the fused kernel's go to the wide
// merge, which takes them four at a time and 32 sequences a work-group; more
// go to shared_merge_kernel (us a call with it / the wide merge, prefix 8000:
// 64 sequences, 4 rows, 168.3 / 163.9; 28, 9 rows, 100.5 / 99.0; 20, 12 rows,
// 83.6 / 81.3; 18, 14 rows, 80.7 / 79.3; 16, 16 rows, 73.8 / 75.3; 8, 32 rows,
// 55.9 / 59.2).
constexpr int kFusedWideSplits = 14;

// Arguments of the split kernel of the prefix (part 0, as one sequence of B H heads) or of the own tokens (part 1).
SplitArgs shared_split_args(const SharedCall& c, int part, const float* qfull, SharedPart* rows) {
  const DecodePlan& s = part ? c.p.own : c.p.pre;
  SplitArgs a{};
  a.qfull = qfull;
  a.cache = c.cache;
  a.ids = c.ids;
  a.gate = c.gate;
  a.num_slots = c.num_slots;
  a.DC = c.d.latent_dim;
  a.DR = c.d.rope_dim;
  a.P = c.d.page_size;
  a.V = c.d.vocab_size;
  a.scale_log2 = softmax_scale(c.d) * kLog2e;
  a.DH = c.d.head_dim;
  a.B = part ? c.batch : 1;
  a.H = part ? c.d.num_heads : c.batch * c.d.num_heads;
  a.seq_lens = part ? c.seq_lens : c.prefix_len;
  a.page_table = part ? c.page_table : c.prefix_table;
  a.max_pages = part ? c.max_pages : c.max_prefix_pages;
  a.cap = s.capacity;
  a.split = s.split_tokens;
  a.s_max = s.s_max;
  a.groups = s.head_groups;
  a.hpg = s.heads_per_group;
  a.part_ml = reinterpret_cast<float*>(c.ws + s.off_ml);
  a.part_o = reinterpret_cast<float*>(c.ws + s.off_o);
  if (s.balanced) {
    a.sched_hdr = reinterpret_cast<const int64_t*>(c.ws + s.off_sched);
    a.wg_start = reinterpret_cast<const int2*>(c.ws + s.off_sched + 16);
  }
  *rows = {a.part_ml, a.part_o, a.seq_lens, s.capacity, s.split_tokens, s.s_max};
  return a;
}

hipError_t launch_shared_part(const SharedCall& c, int part, const float* qfull, SharedPart* rows) {
  const SplitArgs a = shared_split_args(c, part, qfull, rows);
  const OneArgs one{c.q, c.w_uk, c.w_uv, c.out, c.d.v_head_dim, 1, 1};
  return launch_split(c.d, part ? c.p.own : c.p.pre, a, one, c.stream, nullptr, nullptr);
}

// Both parts on the fp32 matrix-core kernel: one launch.
template <bool BF16>
hipError_t launch_f32_pair(const SplitArgs& a, const SplitArgs& b, int na, int nb, hipStream_t stream) {
  auto kern = a.DC <= 64    ? split_f32_pair_kernel<BF16, 64>
              : a.DC <= 128 ? split_f32_pair_kernel<BF16, 128>
              : a.DC <= 256 ? split_f32_pair_kernel<BF16, 256>
                            : split_f32_pair_kernel<BF16, 320>;
  hipLaunchKernelGGL(kern, dim3(na + nb), dim3(256), 0, stream, SplitPair{{a, b}}, na);
  return hipGetLastError();
}

template <int DC>
hipError_t launch_tiled(const SharedCall& c) {
  const eg_mla_dims& d = c.d;
  const SharedPlan& p = c.p;
  const bool own_tokens = p.own.capacity > 0;
  const bool wide = p.own.balanced && own_tokens && !p.fused;
  int2* seq_rows = reinterpret_cast<int2*>(c.ws + p.own.off_sched + 16 + kWideMaxGroups * 8);
  PrefixPrepArgs pa{};
  pa.q = static_cast<const uint16_t*>(c.q);
  pa.w_uk = static_cast<const uint16_t*>(c.w_uk);
  pa.qfull = reinterpret_cast<float*>(c.ws + p.off_q);
  pa.qhalf = reinterpret_cast<uint16_t*>(c.ws + p.off_half);
  pa.cache = static_cast<const uint16_t*>(c.cache);
  pa.ids = c.ids;
  pa.gate = static_cast<const uint16_t*>(c.gate);
  pa.len = c.prefix_len;
  pa.table = c.prefix_table;
  pa.tiles = c.ws + p.off_tiles;
  pa.num_slots = c.num_slots;
  if (wide)
    pa.sched = {c.seq_lens, p.own.capacity, wide_groups(p.own.head_groups),
                reinterpret_cast<int64_t*>(c.ws + p.own.off_sched),
                reinterpret_cast<int2*>(c.ws + p.own.off_sched + 16), seq_rows};
  pa.B = c.batch;
  pa.H = d.num_heads;
  pa.DC = DC;
  pa.V = d.vocab_size;
  pa.P = d.page_size;
  pa.cap = p.pre.capacity;
  pa.keys = p.keys;
  pa.splits = p.splits;
  if (p.fused) pa.split_rows = reinterpret_cast<int2*>(c.ws + p.off_rows);
  pa.gate_wgs = std::min((p.pre.capacity + kPrepTokens - 1) / kPrepTokens, kPrepGroups);
  const AbsorbGrid ag = absorb_grid(d, c.batch, p.own.balanced);
  pa.row_blocks = ag.grid.y;
  auto prep = p.own.balanced ? shared_prep_kernel<AbsorbRows::kHalf, kAbsBlocks, kAbsCols>
              : ag.grouped   ? shared_prep_kernel<AbsorbRows::kBoth, kAbsBlocks, kAbsCols>
              : ag.narrow    ? shared_prep_kernel<AbsorbRows::kBoth, 1, kAbsColsNarrow>
                             : shared_prep_kernel<AbsorbRows::kBoth, 1, kAbsCols>;
  const int64_t absorb_wgs = static_cast<int64_t>(ag.grid.x) * ag.grid.y * ag.grid.z;
  if (absorb_wgs > (1 << 30)) return hipErrorInvalidValue;
  pa.absorb_wgs = static_cast<int32_t>(absorb_wgs);
  const unsigned prep_wgs = 1 + pa.absorb_wgs + pa.gate_wgs;
  hipLaunchKernelGGL(prep, dim3(prep_wgs), dim3(256), 0, c.stream, pa);

  PrefixArgs a{};
  a.qhalf = pa.qhalf;
  a.tiles = pa.tiles;
  a.len = c.prefix_len;
  a.part_ml = reinterpret_cast<float*>(c.ws + p.pre.off_ml);
  a.part_o = c.ws + p.pre.off_o;
  a.cap = p.pre.capacity;
  a.rows = c.batch * d.num_heads;
  a.row_blocks = p.row_blocks;
  a.s_max = p.splits;
  a.scale_log2 = softmax_scale(d) * kLog2e;
  SharedPart own{};
  const unsigned prefix_wgs = p.row_blocks * p.splits;
  if (DC == 128 && p.both) {
    const SplitArgs so = shared_split_args(c, 1, pa.qfull, &own);
    const int own_wgs = c.batch * p.own.s_max * p.own.head_groups;
    hipLaunchKernelGGL(shared_both_kernel, dim3(prefix_wgs + own_wgs), dim3(kPrefixThreads), 0, c.stream, a, so, own_wgs);
  } else {
    auto attend = shared_prefix_kernel<DC, DC == 512 ? 32 : 64, false, false>;
    if constexpr (DC == 512) {
      if (p.half_rows) attend = shared_prefix_kernel<DC, 32, false, true>;
      if (p.fused) {
        attend = shared_prefix_kernel<DC, 32, true, true>;
        a.cache = pa.cache;
        a.ids = c.ids;
        a.gate = pa.gate;
        a.own_lens = own_tokens ? c.seq_lens : nullptr;
        a.own_table = c.page_table;
        a.num_slots = c.num_slots;
        a.own_cap = p.own.capacity;
        a.own_pages = c.max_pages;
        a.blocks_per_seq = d.num_heads / kPrefixRows;
        a.P = d.page_size;
        a.V = d.vocab_size;
      }
    }
    hipLaunchKernelGGL(attend, dim3(prefix_wgs), dim3(kPrefixThreads), 0, c.stream, a);
    if (own_tokens && !p.fused) {
      const hipError_t e = launch_shared_part(c, 1, wide ? reinterpret_cast<const float*>(pa.qhalf) : pa.qfull, &own);
      if (e != hipSuccess) return e;
    }
  }
  if constexpr (DC == 512) {
    if (p.fused && p.splits <= kFusedWideSplits) {  // few rows a sequence: the wide kernel's merge
      const hipError_t e = set_lds(combine_wide_kernel, combine_wide_lds_bytes());
      if (e != hipSuccess) return e;
      hipLaunchKernelGGL(combine_wide_kernel, dim3(d.num_heads, (c.batch + kCombWideSeq - 1) / kCombWideSeq),
                         dim3(kCombWideWaves * 64), combine_wide_lds_bytes(), c.stream, a.part_ml,
                         static_cast<const uint16_t*>(a.part_o), static_cast<const uint16_t*>(c.w_uv), pa.split_rows,
                         static_cast<uint16_t*>(c.out), c.batch, d.num_heads);
      return hipGetLastError();
    }
  }
  SharedMergeArgs m{};
  m.pre_ml = a.part_ml;
  m.pre_o = a.part_o;
  m.pre_len = p.fused ? nullptr : c.prefix_len;
  m.pre_step = p.fused ? d.num_heads : static_cast<int64_t>(c.batch) * d.num_heads;
  m.pre_seq = p.fused ? static_cast<int64_t>(p.splits) * d.num_heads : d.num_heads;
  m.own_ml = own.ml;
  m.own_o = own.o;
  m.own_lens = own.lens;
  m.own_rows = wide ? seq_rows : nullptr;
  m.w_uv = static_cast<const uint16_t*>(c.w_uv);
  m.out = static_cast<uint16_t*>(c.out);
  m.B = c.batch;
  m.H = d.num_heads;
  m.pre_cap = p.pre.capacity;
  m.pre_s_max = p.splits;
  m.own_cap = own.cap;
  m.own_split = own.split;
  m.own_s_max = own.s_max;
  m.keys = p.keys;
  m.spw = kSharedMergeSeq;
  while (m.spw > 1 && static_cast<int64_t>(d.num_heads) * ((c.batch + m.spw - 1) / m.spw) < kSharedMergeGroups) m.spw /= 2;
  auto merge = shared_merge_kernel<DC, false>;
  if constexpr (DC == 512) merge = p.half_rows ? shared_merge_kernel<DC, true> : merge;
  hipLaunchKernelGGL(merge, dim3(d.num_heads, (c.batch + m.spw - 1) / m.spw), dim3(kSharedMergeWaves * 64), 0, c.stream, m);
  return hipGetLastError();
}

eg_mla_status run_decode_shared(const SharedCall& c) {
  const eg_mla_dims& d = c.d;
  if (c.p.plain)
    return run_decode(d, c.p.own, c.batch, c.q, c.cache, c.ids, c.gate, c.w_uk, c.w_uv, c.seq_lens, c.page_table,
                      c.max_pages, c.num_slots, c.ws, c.out, c.stream, nullptr);
  (void)hipGetLastError();
  if (c.p.tiled) {
    const hipError_t e = d.latent_dim == 128   ? launch_tiled<128>(c)
                         : d.latent_dim == 320 ? launch_tiled<320>(c)
                                               : launch_tiled<512>(c);
    return e == hipSuccess ? EG_MLA_OK : EG_MLA_ERR_HIP;
  }
  float* qfull = reinterpret_cast<float*>(c.ws + c.p.off_q);
  if (launch_absorb(d, c.batch, c.q, c.w_uk, qfull, c.stream) != hipSuccess) return EG_MLA_ERR_HIP;
  SharedPart parts[2] = {};
  const DecodePlan &pre = c.p.pre, &own = c.p.own;
  const int64_t na = static_cast<int64_t>(pre.s_max) * pre.head_groups;
  const int64_t nb = static_cast<int64_t>(c.batch) * own.s_max * own.head_groups;
  if (pre.f32_mfma && own.f32_mfma && pre.capacity > 0 && own.capacity > 0 && na + nb <= 0x7fffffff) {
    const SplitArgs a = shared_split_args(c, 0, qfull, &parts[0]), b = shared_split_args(c, 1, qfull, &parts[1]);
    const hipError_t e = d.dtype == EG_MLA_BF16 ? launch_f32_pair<true>(a, b, static_cast<int>(na), static_cast<int>(nb), c.stream)
                                                : launch_f32_pair<false>(a, b, static_cast<int>(na), static_cast<int>(nb), c.stream);
    if (e != hipSuccess) return EG_MLA_ERR_HIP;
  } else {
    for (int part = 0; part < 2; ++part)
      if ((part ? own : pre).capacity > 0 && launch_shared_part(c, part, qfull, &parts[part]) != hipSuccess)
        return EG_MLA_ERR_HIP;
  }
  auto kern = d.dtype == EG_MLA_BF16 ? shared_combine_kernel<true> : shared_combine_kernel<false>;
  hipLaunchKernelGGL(kern, dim3(d.num_heads, c.batch), dim3(256), sizeof(float) * d.latent_dim, c.stream, parts[0],
                     parts[1], c.w_uv, c.out, c.batch, d.num_heads, d.latent_dim, d.v_head_dim);
  return hipGetLastError() == hipSuccess ? EG_MLA_OK : EG_MLA_ERR_HIP;
}

}  // namespace
}  // namespace egmla

extern "C" size_t eg_mla_decode_shared_workspace_size(const eg_mla_dims* dims, int32_t batch,
                                                      int32_t max_pages_per_seq, int32_t max_prefix_pages) {
  egmla::SharedPlan p;
  if (egmla::check_dims(dims) != EG_MLA_OK || batch < 0 || max_pages_per_seq < 0 || max_prefix_pages < 0) return 0;
  if (egmla::make_shared_plan(*dims, batch, max_pages_per_seq, max_prefix_pages, &p) != EG_MLA_OK) return 0;
  return p.bytes;
}

extern "C" eg_mla_status eg_mla_decode_shared(const eg_mla_dims* dims, int32_t batch, const void* q,
                                              const void* latent_cache, const int32_t* token_id_cache,
                                              const void* gate_table, const void* w_uk, const void* w_uv,
                                              const int32_t* prefix_len, const int32_t* prefix_table,
                                              int32_t max_prefix_pages, const int32_t* seq_lens,
                                              const int32_t* page_table, int32_t max_pages_per_seq, int64_t num_slots,
                                              void* workspace, size_t workspace_bytes, void* out, void* stream) {
  egmla::SharedPlan p;
  const eg_mla_status st = egmla::validate_decode_shared(
      dims, batch, q, latent_cache, token_id_cache, gate_table, w_uk, w_uv, prefix_len, prefix_table, max_prefix_pages,
      seq_lens, page_table, max_pages_per_seq, num_slots, workspace, workspace_bytes, out, &p);
  if (st != EG_MLA_OK || batch == 0) return st;
  return egmla::run_decode_shared({*dims, p, batch, q, latent_cache, token_id_cache, gate_table, w_uk, w_uv, prefix_len,
                                   prefix_table, max_prefix_pages, seq_lens, page_table, max_pages_per_seq, num_slots,
                                   static_cast<unsigned char*>(workspace), out, static_cast<hipStream_t>(stream)});
}
