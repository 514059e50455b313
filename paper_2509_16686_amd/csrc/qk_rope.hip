// Norms of queries and keys and the position rotation, in one pass (gfx950).
//
// Per token i and head h, with the query's row [q^C | q^R] of d_h + d_r values:
//   q       = q / sqrt(mean(q^2) + 1e-6) * q_norm_w      (where q_norm_w is given)
//   q^R     = RoPE(q^R, positions[i])
// and for the token's key row [c | r] of d_c + d_r values (Sec. 3.1 Eq. (1)):
//   c       = c / sqrt(mean(c^2) + 1e-6) * kv_norm_w     (where kv_norm_w is given)
//   k^R     = RoPE(r / sqrt(mean(r^2) + 1e-6) * k_norm_w, positions[i])   (App. C Eq. (C.10))
//   latent_cache[slots[i]] = [c | k^R],  token_id_cache[slots[i]] = token_ids[i].
//
// Bound by HBM for many tokens (every row in and out once), by latency for
// few.  A wave takes one token and some of its heads: a head's row is one
// 16-byte piece per lane of a group of 8 to 64 lanes (several pieces per lane
// for rows past 64 pieces), so that the sum of squares is a few lane swaps and
// a rotation pair lies within a lane; the sines and cosines, which depend on
// token and piece only, are formed once for all heads of the wave.
//
// Angles: position times frequency in turns, in 64-bit fixed point modulo one
// turn (the frequencies, scaled by 2^64 / 2 pi, come from the host in extended
// precision), off by less than 2^-30 turns for any 32-bit position; the
// remainder, in half turns of (-1, 1), is then rounded to fp32: 2^-26 turns at
// most, wherever the position.  Sine and cosine of it are fp32.  Sums of squares and every product are fp32; the result is rounded
// once to the storage type.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>

#include "device_common.h"
#include "eg_mla.h"
#include "host_plan.h"

namespace egmla {

constexpr int kQkThreads = 256;
constexpr float kQkEps = 1e-6f;
constexpr int kQkMaxPairs = 320;  // d_r <= 640
// Waves that fill the chip (256 compute units, 16 waves each): fewer heads per
// wave while there are not so many.
constexpr int64_t kQkWaves = 4096;

struct QkArgs {
  const void* q;  // [n] rows of q_stride elements, or null
  const void* q_w;
  void* q_out;
  const void* kv;  // [n] rows of kv_stride elements, or null
  const void* kv_w;
  const void* k_w;
  const int32_t* positions;
  const int32_t* token_ids;
  const int32_t* slots;
  void* cache;
  int32_t* ids;
  int64_t q_stride, kv_stride, num_slots, units;
  int32_t H, DH, DC, DR, hpu, upt;  // heads per query unit; units per token (query units and one for the key row)
  uint64_t freq[kQkMaxPairs];       // theta^(-2m/d_r) / 2 pi, in units of 2^-64 turns
};

// 16 bytes of a row as floats and back.
template <bool BF16>
struct Piece {
  static constexpr int N = BF16 ? 8 : 4;
  float v[N];
  __device__ __forceinline__ void load(const void* p, int64_t i) {
    if constexpr (BF16) {
      const u32x4_t w = *reinterpret_cast<const u32x4_t*>(static_cast<const uint16_t*>(p) + i);
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        v[2 * e] = bf16_lo(w[e]);
        v[2 * e + 1] = bf16_hi(w[e]);
      }
    } else {
      const f32x4_t w = *reinterpret_cast<const f32x4_t*>(static_cast<const float*>(p) + i);
#pragma unroll
      for (int e = 0; e < 4; ++e) v[e] = w[e];
    }
  }
  __device__ __forceinline__ void store(void* p, int64_t i) const {
    if constexpr (BF16)
      *reinterpret_cast<u32x4_t*>(static_cast<uint16_t*>(p) + i) =
          u32x4_t{pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3]), pack_bf16x2(v[4], v[5]), pack_bf16x2(v[6], v[7])};
    else
      *reinterpret_cast<f32x4_t*>(static_cast<float*>(p) + i) = f32x4_t{v[0], v[1], v[2], v[3]};
  }
  __device__ __forceinline__ float squares() const {
    float s = 0.f;
#pragma unroll
    for (int e = 0; e < N; ++e) s = fmaf(v[e], v[e], s);
    return s;
  }
  __device__ __forceinline__ void scale(float r, const Piece& w) {
#pragma unroll
    for (int e = 0; e < N; ++e) v[e] = v[e] * r * w.v[e];
  }
};

// Sines and cosines of a piece's pairs, the first of which is pair m of the row.
template <bool BF16>
struct Turns {
  static constexpr int N = Piece<BF16>::N / 2;
  float cs[N], sn[N];
  __device__ __forceinline__ void set(const uint64_t* freq, int m, int32_t position) {
#pragma unroll
    for (int e = 0; e < N; ++e) {
      const uint64_t t = static_cast<uint64_t>(static_cast<int64_t>(position)) * freq[m + e];  // modulo one turn
      sincospif(static_cast<float>(static_cast<int32_t>(t >> 32)) * 0x1p-31f, &sn[e], &cs[e]);
    }
  }
  __device__ __forceinline__ void apply(Piece<BF16>& p) const {
#pragma unroll
    for (int e = 0; e < N; ++e) {
      const float a = p.v[2 * e], b = p.v[2 * e + 1];
      p.v[2 * e] = a * cs[e] - b * sn[e];
      p.v[2 * e + 1] = a * sn[e] + b * cs[e];
    }
  }
};

// Sum over the G lanes of a head's group.
template <int G>
__device__ __forceinline__ float group_sum(float x) {
#pragma unroll
  for (int o = G / 2; o >= 1; o >>= 1) x += __shfl_xor(x, o, 64);
  return x;
}

// G lanes per head, NP pieces per lane.
template <bool BF16, int G, int NP>
__global__ __launch_bounds__(kQkThreads) void qk_norm_rope_kernel(QkArgs a) {
  typedef Piece<BF16> P;
  constexpr int SLOTS = 64 / G;  // heads per pass
  const int lane = threadIdx.x & 63;
  const int64_t unit = static_cast<int64_t>(blockIdx.x) * (kQkThreads / 64) + (threadIdx.x >> 6);
  if (unit >= a.units) return;
  const int64_t t = unit / a.upt;
  const int j = static_cast<int>(unit - t * a.upt);
  const int32_t position = a.DR ? a.positions[t] : 0;

  if (a.kv && j == a.upt - 1) {  // the key row
    constexpr int NK = BF16 ? 2 : 3;  // pieces per lane: d_c + d_r <= 640
    const int64_t slot = a.slots[t];
    if (slot < 0 || slot >= a.num_slots) return;  // out-of-range destination: skipped
    const int DQ = a.DC + a.DR;
    P x[NK];
    float ssc = 0.f, ssr = 0.f;
#pragma unroll
    for (int i = 0; i < NK; ++i) {
      const int at = (lane + 64 * i) * P::N;
      if (at >= DQ) continue;
      x[i].load(a.kv, t * a.kv_stride + at);
      const float ss = x[i].squares();
      if (at < a.DC) ssc += ss;
      else ssr += ss;
    }
    const float rc = a.kv_w ? 1.f / sqrtf(wave_sum(ssc) / static_cast<float>(a.DC) + kQkEps) : 1.f;
    const float rr = a.k_w ? 1.f / sqrtf(wave_sum(ssr) / static_cast<float>(a.DR) + kQkEps) : 1.f;
#pragma unroll
    for (int i = 0; i < NK; ++i) {
      const int at = (lane + 64 * i) * P::N;
      if (at >= DQ) continue;
      P w;
      if (at < a.DC) {
        if (a.kv_w) {
          w.load(a.kv_w, at);
          x[i].scale(rc, w);
        }
      } else {
        if (a.k_w) {
          w.load(a.k_w, at - a.DC);
          x[i].scale(rr, w);
        }
        Turns<BF16> turn;
        turn.set(a.freq, (at - a.DC) / 2, position);
        turn.apply(x[i]);
      }
      x[i].store(a.cache, slot * DQ + at);
    }
    if (lane == 0) a.ids[slot] = a.token_ids[t];
    return;
  }

  // heads h0 .. h1 - 1 of the query, SLOTS at a time
  const int DQ = a.DH + a.DR;
  const int g = lane / G, sub = lane % G;
  const int h0 = j * a.hpu, h1 = min(h0 + a.hpu, a.H);
  bool in[NP], rope[NP];
  P w[NP];
  Turns<BF16> turn[NP];
#pragma unroll
  for (int i = 0; i < NP; ++i) {
    const int at = (sub + G * i) * P::N;
    in[i] = at < DQ;
    rope[i] = in[i] && at >= a.DH;
    if (in[i] && a.q_w) w[i].load(a.q_w, at);
    if (rope[i]) turn[i].set(a.freq, (at - a.DH) / 2, position);
  }
  P x[NP], next[NP];
  auto load = [&](P (&p)[NP], int h) {  // heads past the last repeat it and are not stored
    const int64_t row = t * a.q_stride + static_cast<int64_t>(min(h, h1 - 1)) * DQ;
#pragma unroll
    for (int i = 0; i < NP; ++i)
      if (in[i]) p[i].load(a.q, row + (sub + G * i) * P::N);
  };
  load(next, h0 + g);
  for (int h = h0 + g; h - g < h1; h += SLOTS) {
#pragma unroll
    for (int i = 0; i < NP; ++i) x[i] = next[i];
    if (h - g + SLOTS < h1) load(next, h + SLOTS);
    if (a.q_w) {
      float ss = 0.f;
#pragma unroll
      for (int i = 0; i < NP; ++i)
        if (in[i]) ss += x[i].squares();
      const float r = 1.f / sqrtf(group_sum<G>(ss) / static_cast<float>(DQ) + kQkEps);
#pragma unroll
      for (int i = 0; i < NP; ++i)
        if (in[i]) x[i].scale(r, w[i]);
    }
    const int64_t row = (t * a.H + h) * DQ;
#pragma unroll
    for (int i = 0; i < NP; ++i) {
      if (rope[i]) turn[i].apply(x[i]);
      if (in[i] && h < h1) x[i].store(a.q_out, row + (sub + G * i) * P::N);
    }
  }
}

}  // namespace egmla

using namespace egmla;

namespace {

template <bool BF16>
hipError_t launch_qk(const QkArgs& a, int pieces, dim3 grid, hipStream_t stream) {
  const dim3 block(kQkThreads);
  if (pieces <= 8) hipLaunchKernelGGL((qk_norm_rope_kernel<BF16, 8, 1>), grid, block, 0, stream, a);
  else if (pieces <= 16) hipLaunchKernelGGL((qk_norm_rope_kernel<BF16, 16, 1>), grid, block, 0, stream, a);
  else if (pieces <= 32) hipLaunchKernelGGL((qk_norm_rope_kernel<BF16, 32, 1>), grid, block, 0, stream, a);
  else if (pieces <= 64) hipLaunchKernelGGL((qk_norm_rope_kernel<BF16, 64, 1>), grid, block, 0, stream, a);
  else if (pieces <= 128) hipLaunchKernelGGL((qk_norm_rope_kernel<BF16, 64, 2>), grid, block, 0, stream, a);
  else if (pieces <= 256) hipLaunchKernelGGL((qk_norm_rope_kernel<BF16, 64, 4>), grid, block, 0, stream, a);
  else hipLaunchKernelGGL((qk_norm_rope_kernel<BF16, 64, 8>), grid, block, 0, stream, a);
  return hipGetLastError();
}

// Lanes per head of launch_qk's choice.
int qk_group(int pieces) { return pieces <= 8 ? 8 : pieces <= 16 ? 16 : pieces <= 32 ? 32 : 64; }

}  // namespace

extern "C" eg_mla_status eg_mla_qk_norm_rope(const eg_mla_dims* dims, int32_t n_tokens, const void* q,
                                             int64_t q_stride, const void* q_norm_w, void* q_out, const void* kv,
                                             int64_t kv_stride, const void* kv_norm_w, const void* k_norm_w,
                                             const int32_t* token_ids, const int32_t* positions,
                                             const int32_t* slots, float rope_theta, void* latent_cache,
                                             int32_t* token_id_cache, int64_t num_slots, void* stream_) {
  const eg_mla_status st = validate_qk(dims, n_tokens, q, q_stride, q_norm_w, q_out, kv, kv_stride, kv_norm_w,
                                       k_norm_w, token_ids, positions, slots, rope_theta, latent_cache,
                                       token_id_cache, num_slots);
  if (st != EG_MLA_OK || n_tokens == 0) return st;
  const eg_mla_dims& d = *dims;
  const int pieces = (d.head_dim + d.rope_dim) / (16 / elem_bytes(d));
  QkArgs a;
  a.q = q;
  a.q_w = q_norm_w;
  a.q_out = q_out;
  a.kv = kv;
  a.kv_w = kv_norm_w;
  a.k_w = k_norm_w;
  a.positions = positions;
  a.token_ids = token_ids;
  a.slots = slots;
  a.cache = latent_cache;
  a.ids = token_id_cache;
  a.q_stride = q_stride;
  a.kv_stride = kv_stride;
  a.num_slots = num_slots;
  a.H = d.num_heads;
  a.DH = d.head_dim;
  a.DC = d.latent_dim;
  a.DR = d.rope_dim;
  // heads per wave: whole passes, up to 8 of them while the waves still fill the chip
  const int slots_per_pass = 64 / qk_group(pieces);
  int passes = 1;
  while (passes < 8 && static_cast<int64_t>(n_tokens) * d.num_heads >= kQkWaves * slots_per_pass * passes * 2) passes *= 2;
  a.hpu = slots_per_pass * passes;
  a.upt = (q ? (d.num_heads + a.hpu - 1) / a.hpu : 0) + (kv ? 1 : 0);
  a.units = static_cast<int64_t>(n_tokens) * a.upt;
  const int64_t wgs = (a.units + kQkThreads / 64 - 1) / (kQkThreads / 64);
  if (wgs > 0x7fffffff) return EG_MLA_ERR_UNSUPPORTED;
  const long double theta = rope_theta > 0.f ? rope_theta : 10000.f;
  const long double step = d.rope_dim ? powl(theta, -2.0L / d.rope_dim) : 0.0L;
  long double f = 1.0L / 6.283185307179586476925286766559005768L;
  for (int m = 0; m < d.rope_dim / 2; ++m, f *= step)
    a.freq[m] = static_cast<uint64_t>((f < 1.0L ? f : fmodl(f, 1.0L)) * 18446744073709551616.0L);  // whole turns drop out
  hipStream_t stream = static_cast<hipStream_t>(stream_);
  (void)hipGetLastError();
  const dim3 grid(static_cast<unsigned>(wgs));
  const hipError_t e = d.dtype == EG_MLA_BF16 ? launch_qk<true>(a, pieces, grid, stream)
                                              : launch_qk<false>(a, pieces, grid, stream);
  return e == hipSuccess ? EG_MLA_OK : EG_MLA_ERR_HIP;
}
