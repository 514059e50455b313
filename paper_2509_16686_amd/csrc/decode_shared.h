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
  auto fold = [&](const SharedPart& p, int64_t row0, int64_t step, int len) {
    const int ns = min((clamp_len(len, p.cap) + p.split - 1) / p.split, p.s_max);
    for (int s = 0; s < ns; ++s) {
      const int64_t row = row0 + s * step;
      const float m = p.ml[2 * row];
      const float Mn = fmaxf(M, m);
      if (!(Mn > -INFINITY)) continue;  // nothing weighs anything yet
      const float keep = exp2f(M - Mn), e = exp2f(m - Mn);  // exp2(-inf) = 0
      M = Mn;
      sum = sum * keep + p.ml[2 * row + 1] * e;
#pragma unroll
      for (int k = 0; k < kSharedCols; ++k) {
        const int c = threadIdx.x + 256 * k;
        if (c < DC) acc[k] = acc[k] * keep + p.o[row * DC + c] * e;
      }
    }
  };
  if (pre.s_max > 0) fold(pre, static_cast<int64_t>(b) * H + h, static_cast<int64_t>(B) * H, pre.lens[0]);
  if (own.s_max > 0) fold(own, static_cast<int64_t>(b) * own.s_max * H + h, H, own.lens[b]);
  const float inv = M > -INFINITY ? 1.f / sum : 0.f;
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

eg_mla_status run_decode_shared(const eg_mla_dims& d, const SharedPlan& p, int32_t batch, const void* q,
                                const void* latent_cache, const int32_t* token_id_cache, const void* gate_table,
                                const void* w_uk, const void* w_uv, const int32_t* prefix_len,
                                const int32_t* prefix_table, int32_t max_prefix_pages, const int32_t* seq_lens,
                                const int32_t* page_table, int32_t max_pages_per_seq, int64_t num_slots,
                                void* workspace, void* out, hipStream_t stream) {
  (void)hipGetLastError();
  unsigned char* ws = static_cast<unsigned char*>(workspace);
  float* qfull = reinterpret_cast<float*>(ws + p.off_q);
  if (launch_absorb(d, batch, q, w_uk, qfull, stream) != hipSuccess) return EG_MLA_ERR_HIP;
  SplitArgs a{};
  a.qfull = qfull;
  a.cache = latent_cache;
  a.ids = token_id_cache;
  a.gate = gate_table;
  a.num_slots = num_slots;
  a.DC = d.latent_dim;
  a.DR = d.rope_dim;
  a.P = d.page_size;
  a.V = d.vocab_size;
  a.scale_log2 = softmax_scale(d) * kLog2e;
  a.DH = d.head_dim;
  // the prefix: one sequence of B H heads; then each sequence's own tokens
  SharedPart parts[2] = {};
  for (int part = 0; part < 2; ++part) {
    const DecodePlan& s = part ? p.own : p.pre;
    if (s.capacity == 0) continue;
    eg_mla_dims ds = d;
    if (part == 0) ds.num_heads = batch * d.num_heads;
    a.B = part ? batch : 1;
    a.H = ds.num_heads;
    a.seq_lens = part ? seq_lens : prefix_len;
    a.page_table = part ? page_table : prefix_table;
    a.max_pages = part ? max_pages_per_seq : max_prefix_pages;
    a.cap = s.capacity;
    a.split = s.split_tokens;
    a.s_max = s.s_max;
    a.groups = s.head_groups;
    a.hpg = s.heads_per_group;
    a.part_ml = reinterpret_cast<float*>(ws + s.off_ml);
    a.part_o = reinterpret_cast<float*>(ws + s.off_o);
    const OneArgs one{q, w_uk, w_uv, out, d.v_head_dim, 1, 1};
    if (launch_split(ds, s, a, one, stream, nullptr, nullptr) != hipSuccess) return EG_MLA_ERR_HIP;
    parts[part] = {a.part_ml, a.part_o, a.seq_lens, s.capacity, s.split_tokens, s.s_max};
  }
  const size_t lds = sizeof(float) * static_cast<size_t>(d.latent_dim);
  auto kern = d.dtype == EG_MLA_BF16 ? shared_combine_kernel<true> : shared_combine_kernel<false>;
  hipLaunchKernelGGL(kern, dim3(d.num_heads, batch), dim3(256), lds, stream, parts[0], parts[1], w_uv, out, batch,
                     d.num_heads, d.latent_dim, d.v_head_dim);
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
  return egmla::run_decode_shared(*dims, p, batch, q, latent_cache, token_id_cache, gate_table, w_uk, w_uv, prefix_len,
                                  prefix_table, max_prefix_pages, seq_lens, page_table, max_pages_per_seq, num_slots,
                                  workspace, out, static_cast<hipStream_t>(stream));
}
