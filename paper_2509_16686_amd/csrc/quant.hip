// Rotation of rows, and the 8-bit latent cache written and read back (gfx950).
//
// Rotation of a pair (a, b) of a row's part (App. C Eq. (C.10)):
//   (a, b) -> magnitude (a cos x - b sin x, a sin x + b cos x),  x = positions[i] frequency[m]
// with pair m at (2m, 2m + 1) of the part, or at (m, d_r / 2 + m); `inverse` turns by -x, which is also the gradient's
// way back through the rotation.  x is kept in turns modulo one turn, in 64-bit fixed point (as in qk_rope.hip).
//
// Cache row of a token (Sec. 3.1 Eq. (1), (3)-(5)): the gated latent c~ = c (.) G[id] as d_c e4m3 codes, behind them
// k^R in bf16, and one byte of scale, 127 + e, with e the least power of two that brings the row's largest magnitude
// within e4m3's 448:
//   code = RNE(c~ 2^-e),   c~ ~ code 2^e.
// The gate depends on the token alone, so it is applied once, as the row is written, and neither ids nor gate rows are
// read afterwards.  A power of two costs no accuracy (both formats float) and makes code 2^e exact in bf16, and in fp16
// within its range.  A row with an infinity or NaN among its gated latents gets scale byte 255 and stands for NaN.
//
// All three are bound by HBM for many tokens and by latency for few.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>

#include "device_common.h"
#include "eg_mla.h"
#include "host_plan.h"

namespace egmla {

constexpr int kQ8Threads = 256;
constexpr float kQ8Eps = 1e-6f;
constexpr int kRopeMaxPairs = 320;

// Work-groups of a long call, in two dimensions: a dimension's threads have to stay below 2^32.
dim3 long_grid(int64_t wgs) {
  constexpr int64_t kWide = int64_t{1} << 20;
  return wgs <= kWide ? dim3(static_cast<unsigned>(wgs)) : dim3(kWide, static_cast<unsigned>((wgs + kWide - 1) / kWide));
}
__device__ __forceinline__ int64_t long_block() { return static_cast<int64_t>(blockIdx.y) * gridDim.x + blockIdx.x; }

// Sine and cosine of position * frequency, the frequency in 2^-64 turns a position.
__device__ __forceinline__ void turn_of(uint64_t freq, int32_t position, float& sn, float& cs) {
  const uint64_t t = static_cast<uint64_t>(static_cast<int64_t>(position)) * freq;  // modulo one turn
  sincospif(static_cast<float>(static_cast<int32_t>(t >> 32)) * 0x1p-31f, &sn, &cs);
}

// ---------------------------------------------------------------------------
// Rotation of rows [n, H, D]: a work-group takes one token and `hpu` of its
// heads; a thread takes two pieces of VEC values of a head's row, those of VEC
// pairs or two to copy, for every hpar-th of them, so that its sines are formed
// once, and four heads' loads are in flight (8192 tokens x 128 heads of 192 bf16
// values: 152 us a call, 5.3 TB/s in and out, the rate of a copy; 208 us with one piece to
// copy a thread, two heads in flight and waves that took both branches).
// ---------------------------------------------------------------------------
struct RopeArgs {
  const void* x;
  void* out;
  const int32_t* positions;
  int64_t xt, xh, ot, oh;  // strides of tokens and heads, in elements
  int32_t n, H, D, off, rd, hpu, upt;
  int32_t copy;            // whether the other values are copied (not in place)
  float magnitude, sign;
  uint64_t freq[kRopeMaxPairs];
};

template <bool BF16, int VEC>
struct Values {
  typedef typename std::conditional<BF16, uint16_t, uint32_t>::type E;
  typedef E raw_t __attribute__((ext_vector_type(VEC)));
  raw_t v;
  __device__ __forceinline__ void load(const void* p, int64_t i) {
    v = *reinterpret_cast<const raw_t*>(static_cast<const E*>(p) + i);
  }
  __device__ __forceinline__ void store(void* p, int64_t i) const {
    *reinterpret_cast<raw_t*>(static_cast<E*>(p) + i) = v;
  }
  __device__ __forceinline__ float get(int e) const {
    if constexpr (BF16) return bf16_to_f32(v[e]);
    else return __uint_as_float(v[e]);
  }
  __device__ __forceinline__ void set(int e, float f) {
    if constexpr (BF16) v[e] = f32_to_bf16(f);
    else v[e] = __float_as_uint(f);
  }
};

template <bool BF16, int VEC, bool HALF>
__global__ __launch_bounds__(kQ8Threads) void rope_rows_kernel(RopeArgs a) {
  typedef Values<BF16, VEC> V;
  const int64_t wg = long_block(), t = wg / a.upt;
  if (t >= a.n) return;
  const int u = static_cast<int>(wg - t * a.upt);
  const int h0 = u * a.hpu, h1 = min(h0 + a.hpu, a.H);
  const int32_t position = a.positions[t];
  const int turns = a.rd / (2 * VEC), others = a.copy ? (a.D - a.rd) / VEC : 0;  // items that turn; pieces to copy
  const int items = turns + (others + 1) / 2;
  const int span = min(items, kQ8Threads), hpar = kQ8Threads / span;
  const int hp = threadIdx.x / span;
  if (hp >= hpar) return;
  const int64_t x0 = t * a.xt, o0 = t * a.ot;
  for (int item = threadIdx.x % span; item < items; item += span) {
    const bool turn = item < turns;
    int p, q;
    float sn[VEC], cs[VEC];
    if (turn) {
      p = a.off + (HALF ? item * VEC : 2 * item * VEC);
      q = HALF ? p + a.rd / 2 : p + VEC;
#pragma unroll
      for (int e = 0; e < VEC; ++e) {
        turn_of(a.freq[item * VEC + e], position, sn[e], cs[e]);
        sn[e] *= a.sign * a.magnitude;
        cs[e] *= a.magnitude;
      }
    } else {  // (of an odd number the last one twice)
      const int c = 2 * (item - turns), d = min(c + 1, others - 1);
      p = c * VEC + (c * VEC < a.off ? 0 : a.rd);
      q = d * VEC + (d * VEC < a.off ? 0 : a.rd);
    }
    constexpr int UNROLL = 4;
    for (int h = h0 + hp; h < h1; h += UNROLL * hpar) {
      V x[UNROLL], y[UNROLL];
#pragma unroll
      for (int u = 0; u < UNROLL; ++u) {  // (heads past the last repeat it and are not stored)
        const int64_t at = x0 + min(h + u * hpar, h1 - 1) * a.xh;
        x[u].load(a.x, at + p);
        y[u].load(a.x, at + q);
      }
#pragma unroll
      for (int u = 0; u < UNROLL; ++u) {
        V r = x[u], s = y[u];
        if (turn) {
#pragma unroll
          for (int e = 0; e < VEC; ++e) {
            // pair e: values e of x and y, or values 2e and 2e + 1 of the two side by side
            const int i = HALF ? e : 2 * e, j = HALF ? e + VEC : 2 * e + 1;
            const float f = i < VEC ? x[u].get(i) : y[u].get(i - VEC), g = j < VEC ? x[u].get(j) : y[u].get(j - VEC);
            const float rf = f * cs[e] - g * sn[e], rg = f * sn[e] + g * cs[e];
            if (i < VEC) r.set(i, rf);
            else s.set(i - VEC, rf);
            if (j < VEC) r.set(j, rg);
            else s.set(j - VEC, rg);
          }
        }
        if (h + u * hpar < h1) {
          const int64_t at = o0 + (h + u * hpar) * a.oh;
          r.store(a.out, at + p);
          s.store(a.out, at + q);
        }
      }
    }
  }
}

// ---------------------------------------------------------------------------
// Rows written: LPT lanes a token, 8 latent values a lane (d_c <= 8 LPT), and
// the values of the RoPE key one a lane, LPT apart, with a pair's other value loaded
// beside it.  A chain of slot, row, id and gate row: 12400 tokens of d_c 512 13.8 us
// (2.6 TB/s of rows, gate rows and codes), 32 tokens of d_c 128 5.3.
// ---------------------------------------------------------------------------
constexpr int kQ8MaxRope = 64;

struct Q8WriteArgs {
  const uint16_t* kv;
  const uint16_t* kv_w;
  const uint16_t* k_w;
  const uint16_t* gate;
  const int32_t* ids;
  const int32_t* positions;  // null: no rotation
  const int32_t* slots;
  uint8_t* codes;
  uint8_t* scales;
  int64_t kv_stride, num_slots;
  int32_t n, DC, DR, V, half;
  float magnitude;
  uint64_t freq[kQ8MaxRope / 2];
};

template <int G>
__device__ __forceinline__ float lanes_sum(float x) {
#pragma unroll
  for (int o = G / 2; o >= 1; o >>= 1) x += __shfl_xor(x, o, 64);
  return x;
}

template <int LPT>
__global__ __launch_bounds__(kQ8Threads) void q8_write_kernel(Q8WriteArgs a) {
  constexpr int EPL = kQ8MaxRope / LPT;
  const int sub = threadIdx.x % LPT;
  const int64_t t = long_block() * (kQ8Threads / LPT) + threadIdx.x / LPT;
  if (t >= a.n) return;
  const int64_t slot = a.slots[t];
  if (slot < 0 || slot >= a.num_slots) return;  // out-of-range destination: skipped
  const uint16_t* row = a.kv + t * a.kv_stride;
  const int64_t dst = slot * (a.DC + 2 * a.DR);
  const bool lat = 8 * sub < a.DC;

  // the RoPE key: value r of the lane's and its partner's
  float x[EPL], y[EPL], wx[EPL], wy[EPL];
#pragma unroll
  for (int j = 0; j < EPL; ++j) {
    const int r = sub + LPT * j, m = a.half ? (r < a.DR / 2 ? r + a.DR / 2 : r - a.DR / 2) : r ^ 1;
    x[j] = y[j] = wx[j] = wy[j] = 0.f;
    if (r >= a.DR) continue;
    x[j] = bf16_to_f32(row[a.DC + r]);
    y[j] = bf16_to_f32(row[a.DC + m]);
    if (a.k_w) {
      wx[j] = bf16_to_f32(a.k_w[r]);
      wy[j] = bf16_to_f32(a.k_w[m]);
    }
  }
  const int32_t position = a.positions ? a.positions[t] : 0;
  // the latent
  u32x4_t cv = {0u, 0u, 0u, 0u}, wv = cv, gv = cv;
  if (lat) {
    cv = *reinterpret_cast<const u32x4_t*>(row + 8 * sub);
    if (a.kv_w) wv = *reinterpret_cast<const u32x4_t*>(a.kv_w + 8 * sub);
    if (a.gate) gv = *reinterpret_cast<const u32x4_t*>(a.gate + static_cast<int64_t>(clamp_id(a.ids[t], a.V)) * a.DC + 8 * sub);
  }
  float c[8];
#pragma unroll
  for (int e = 0; e < 8; ++e) c[e] = e & 1 ? bf16_hi(cv[e / 2]) : bf16_lo(cv[e / 2]);
  if (a.kv_w) {
    float ss = 0.f;
#pragma unroll
    for (int e = 0; e < 8; ++e) ss = fmaf(c[e], c[e], ss);
    const float r = 1.f / sqrtf(lanes_sum<LPT>(ss) / static_cast<float>(a.DC) + kQ8Eps);
#pragma unroll
    for (int e = 0; e < 8; ++e) c[e] = c[e] * r * (e & 1 ? bf16_hi(wv[e / 2]) : bf16_lo(wv[e / 2]));
  }
  if (a.gate) {
#pragma unroll
    for (int e = 0; e < 8; ++e) c[e] *= e & 1 ? bf16_hi(gv[e / 2]) : bf16_lo(gv[e / 2]);
  }
  // largest magnitude, as bits (their order is that of magnitudes; an infinity or NaN is the largest)
  uint32_t top = 0;
#pragma unroll
  for (int e = 0; e < 8; ++e) top = max(top, __float_as_uint(c[e]) & 0x7fffffffu);
#pragma unroll
  for (int o = LPT / 2; o >= 1; o >>= 1) top = max(top, static_cast<uint32_t>(__shfl_xor(static_cast<int>(top), o, 64)));
  // 448 = 1.75 2^8: e is the exponent less 8, one more where the fraction is past 1.75; held to powers that fp32 has
  int e = static_cast<int>(top >> 23) - 127 - 8 + ((top & 0x7fffffu) > 0x600000u ? 1 : 0);
  e = top == 0 ? 0 : min(max(e, -126), 120);
  const bool none = top >= 0x7f800000u;
  const float down = none ? 0.f : __uint_as_float(static_cast<uint32_t>(127 - e) << 23);
  if (lat) {
    u32x2_t w = {0u, 0u};
    if (!none) {
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        int p = __builtin_amdgcn_cvt_pk_fp8_f32(c[4 * i] * down, c[4 * i + 1] * down, 0, false);
        w[i] = static_cast<uint32_t>(__builtin_amdgcn_cvt_pk_fp8_f32(c[4 * i + 2] * down, c[4 * i + 3] * down, p, true));
      }
    }
    *reinterpret_cast<u32x2_t*>(a.codes + dst + 8 * sub) = w;
  }
  if (sub == 0) a.scales[slot] = none ? 255 : static_cast<uint8_t>(127 + e);
  if (a.DR == 0) return;
  if (a.k_w) {
    float ss = 0.f;
#pragma unroll
    for (int j = 0; j < EPL; ++j) ss = fmaf(x[j], x[j], ss);
    const float r = 1.f / sqrtf(lanes_sum<LPT>(ss) / static_cast<float>(a.DR) + kQ8Eps);
#pragma unroll
    for (int j = 0; j < EPL; ++j) {
      x[j] = x[j] * r * wx[j];
      y[j] = y[j] * r * wy[j];
    }
  }
#pragma unroll
  for (int j = 0; j < EPL; ++j) {
    const int r = sub + LPT * j;
    if (r >= a.DR) continue;
    float v = x[j];
    if (a.positions) {
      const bool second = a.half ? r >= a.DR / 2 : r & 1;
      const int m = a.half ? (second ? r - a.DR / 2 : r) : r >> 1;
      float sn, cs;
      turn_of(a.freq[m], position, sn, cs);
      sn *= a.magnitude;
      cs *= a.magnitude;
      v = second ? y[j] * sn + x[j] * cs : x[j] * cs - y[j] * sn;
    }
    *reinterpret_cast<uint16_t*>(a.codes + dst + a.DC + 2 * r) = f32_to_bf16(v);
  }
}

// ---------------------------------------------------------------------------
// Rows read back, packed by sequence: a work-group takes kQ8ReadTokens packed
// rows; 16 codes, or 8 values of the RoPE key, an item (270 000 tokens of d_c 512:
// 104 us, 4.7 TB/s).
// ---------------------------------------------------------------------------
constexpr int kQ8ReadTokens = 16;

struct Q8ReadArgs {
  const uint8_t* codes;
  const uint8_t* scales;
  const int32_t* first;
  const int32_t* cu;
  const int32_t* table;
  uint16_t* out;
  int64_t num_slots;
  int32_t batch, total, max_pages, P, DC, DR;
};

// 16 codes times their scale (127 + exponent in a byte; 255: NaN) in bf16, exact.
__device__ __forceinline__ void q8_to_bf16(u32x4_t w, uint32_t byte, u32x4_t& lo, u32x4_t& hi) {
  const float s = __uint_as_float(byte << 23);
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    uint32_t p = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w[i], s, false));
    uint32_t q = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w[i], s, true));
    if (byte == 255u) p = q = 0x7fc07fc0u;
    if (i < 2) {
      lo[2 * i] = p;
      lo[2 * i + 1] = q;
    } else {
      hi[2 * i - 4] = p;
      hi[2 * i - 3] = q;
    }
  }
}

__global__ __launch_bounds__(kQ8Threads) void q8_read_kernel(Q8ReadArgs a) {
  __shared__ int32_t cu_s[kPageMaxBatch + 1];
  __shared__ int32_t slot_s[kQ8ReadTokens];
  __shared__ uint32_t scale_s[kQ8ReadTokens];
  const int tid = threadIdx.x;
  const int64_t first_row = long_block() * kQ8ReadTokens;
  if (first_row >= a.total) return;
  const int i0 = static_cast<int>(first_row);
  for (int i = tid; i <= a.batch; i += kQ8Threads) cu_s[i] = a.cu[i];
  __syncthreads();
  if (tid < kQ8ReadTokens) {
    const int i = i0 + tid;
    int lo = 0, hi = a.batch;  // the first sequence that ends behind i
    while (lo < hi) {
      const int mid = (lo + hi) / 2;
      if (cu_s[mid + 1] > i) hi = mid;
      else lo = mid + 1;
    }
    int slot = -1;
    if (i < a.total && i >= 0 && lo < a.batch && i >= cu_s[lo]) {
      const int64_t cap = static_cast<int64_t>(a.max_pages) * a.P;
      int64_t j = static_cast<int64_t>(i) - cu_s[lo] + (a.first ? max(a.first[lo], 0) : 0);
      j = min(j, cap - 1);
      slot = static_cast<int>(cache_slot(a.table, lo, static_cast<int>(j), a.P, a.max_pages, a.num_slots));
      scale_s[tid] = a.scales[slot];
    }
    slot_s[tid] = slot;
  }
  __syncthreads();
  const int lat = a.DC / 16, items = lat + a.DR / 8, row = a.DC + a.DR;
  for (int it = tid; it < kQ8ReadTokens * items; it += kQ8Threads) {
    const int k = it / items, p = it - k * items;
    const int slot = slot_s[k];
    if (slot < 0) continue;
    const uint8_t* src = a.codes + static_cast<int64_t>(slot) * (a.DC + 2 * a.DR) + 16 * p;
    const u32x4_t w = *reinterpret_cast<const u32x4_t*>(src);
    uint16_t* dst = a.out + static_cast<int64_t>(i0 + k) * row;
    if (p < lat) {
      u32x4_t lo, hi;
      q8_to_bf16(w, scale_s[k], lo, hi);
      *reinterpret_cast<u32x4_t*>(dst + 16 * p) = lo;
      *reinterpret_cast<u32x4_t*>(dst + 16 * p + 8) = hi;
    } else {
      *reinterpret_cast<u32x4_t*>(dst + a.DC + 8 * (p - lat)) = w;
    }
  }
}

}  // namespace egmla

using namespace egmla;

namespace {

// Frequencies of `pairs` pairs in 2^-64 turns a position: whole turns drop out.  (A product with 1 / 2 pi, and nothing
// more where a pair turns less than once a position: a division and a floor for each cost 2.5 us a call.)
void turns_of(const eg_mla_rope& r, int pairs, uint64_t* freq) {
  constexpr long double kTurns = 0.159154943091895335768883763372514362L;
  const long double theta = r.theta > 0.f ? r.theta : 10000.f;
  const long double step = pairs && !r.frequencies ? powl(theta, -1.0L / pairs) : 0.0L;
  long double f = 1.0L;
  for (int m = 0; m < pairs; ++m, f *= step) {
    long double x = (r.frequencies ? static_cast<long double>(r.frequencies[m]) : f) * kTurns;
    if (!(x >= 0.0L && x < 1.0L)) x -= floorl(x);
    freq[m] = x >= 1.0L ? 0 : static_cast<uint64_t>(x * 18446744073709551616.0L);
  }
}

float magnitude_of(const eg_mla_rope& r) { return r.magnitude > 0.f ? r.magnitude : 1.f; }

template <bool BF16, int VEC>
void launch_rope(const RopeArgs& a, bool half, dim3 grid, hipStream_t stream) {
  if (half) hipLaunchKernelGGL((rope_rows_kernel<BF16, VEC, true>), grid, dim3(kQ8Threads), 0, stream, a);
  else hipLaunchKernelGGL((rope_rows_kernel<BF16, VEC, false>), grid, dim3(kQ8Threads), 0, stream, a);
}

}  // namespace

extern "C" eg_mla_status eg_mla_rope_frequencies(int32_t rope_dim, float theta, float factor, int32_t trained_positions,
                                                 float slow_turns, float fast_turns, double* frequencies) {
  if (!frequencies || rope_dim < 2 || rope_dim % 2 != 0 || rope_dim > 2 * kRopeMaxPairs) return EG_MLA_ERR_INVALID_ARG;
  if (!(factor >= 1.f) || factor > 3.4e38f || theta != theta || theta > 3.4e38f || trained_positions < 0)
    return EG_MLA_ERR_INVALID_ARG;
  const double slow = slow_turns > 0.f ? slow_turns : 1.0, fast = fast_turns > 0.f ? fast_turns : 32.0;
  if (!(fast > slow) || fast > 3.4e38) return EG_MLA_ERR_INVALID_ARG;
  const double base = theta > 0.f ? theta : 10000.0;
  for (int m = 0; m < rope_dim / 2; ++m) {
    const double f = pow(base, -2.0 * m / rope_dim);
    const double turns = trained_positions * f / 6.283185307179586;
    const double keep = trained_positions == 0 ? 0.0 : std::min(1.0, std::max(0.0, (turns - slow) / (fast - slow)));
    frequencies[m] = f * (keep + (1.0 - keep) / factor);
  }
  return EG_MLA_OK;
}

extern "C" eg_mla_status eg_mla_rope_rows(const eg_mla_rope* rope, int32_t dtype, int32_t n_tokens, int32_t num_heads,
                                          int32_t head_dim, int32_t rope_offset, int32_t rope_dim, const void* x,
                                          int64_t x_token_stride, int64_t x_head_stride, const int32_t* positions,
                                          int32_t inverse, void* out, int64_t out_token_stride, int64_t out_head_stride,
                                          void* stream_) {
  const eg_mla_status st = validate_rope_rows(rope, dtype, n_tokens, num_heads, head_dim, rope_offset, rope_dim, x,
                                              x_token_stride, x_head_stride, positions, out, out_token_stride,
                                              out_head_stride);
  if (st != EG_MLA_OK || n_tokens == 0) return st;
  RopeArgs a;
  a.copy = x != out;
  if (rope_dim == 0 && !a.copy) return EG_MLA_OK;
  a.x = x;
  a.out = out;
  a.positions = positions;
  a.xt = x_token_stride;
  a.xh = x_head_stride;
  a.ot = out_token_stride;
  a.oh = out_head_stride;
  a.n = n_tokens;
  a.H = num_heads;
  a.D = head_dim;
  a.off = rope_offset;
  a.rd = rope_dim;
  a.magnitude = magnitude_of(*rope);
  a.sign = inverse ? -1.f : 1.f;
  turns_of(*rope, rope_dim / 2, a.freq);
  // values of a load: as many as divide every length and stride and as the pointers are aligned to, up to 16 bytes
  const int eb = dtype == EG_MLA_BF16 ? 2 : 4;
  const bool half = rope->layout == EG_MLA_ROPE_HALF;
  int vec = 16 / eb;
  auto fits = [&](int v) {
    const int64_t all = int64_t{rope_offset} | (rope_dim / 2) | (head_dim - rope_offset - rope_dim) | a.xt | a.xh | a.ot | a.oh;
    return all % v == 0 && (reinterpret_cast<uintptr_t>(x) | reinterpret_cast<uintptr_t>(out)) % (v * eb) == 0;
  };
  while (vec > 1 && !fits(vec)) vec /= 2;
  // heads of a work-group: whole passes, up to 8 of them while there are work-groups enough
  const int items = std::max(1, rope_dim / (2 * vec) + (a.copy ? ((head_dim - rope_dim) / vec + 1) / 2 : 0));
  const int hpar = std::max(1, kQ8Threads / items);
  int passes = 1;
  while (passes < 8 && static_cast<int64_t>(n_tokens) * num_heads >= int64_t{2048} * hpar * passes * 2) passes *= 2;
  a.upt = (num_heads + hpar * passes - 1) / (hpar * passes);
  a.hpu = (num_heads + a.upt - 1) / a.upt;  // (as many in each)
  const int64_t wgs = static_cast<int64_t>(n_tokens) * a.upt;
  if (wgs > (int64_t{1} << 35)) return EG_MLA_ERR_UNSUPPORTED;
  const dim3 grid = long_grid(wgs);
  hipStream_t stream = static_cast<hipStream_t>(stream_);
  (void)hipGetLastError();
  if (dtype == EG_MLA_BF16) {
    if (vec == 8) launch_rope<true, 8>(a, half, grid, stream);
    else if (vec == 4) launch_rope<true, 4>(a, half, grid, stream);
    else if (vec == 2) launch_rope<true, 2>(a, half, grid, stream);
    else launch_rope<true, 1>(a, half, grid, stream);
  } else {
    if (vec == 4) launch_rope<false, 4>(a, half, grid, stream);
    else if (vec == 2) launch_rope<false, 2>(a, half, grid, stream);
    else launch_rope<false, 1>(a, half, grid, stream);
  }
  return hipGetLastError() == hipSuccess ? EG_MLA_OK : EG_MLA_ERR_HIP;
}

extern "C" int64_t eg_mla_quant_row_bytes(const eg_mla_dims* dims) {
  return check_q8_dims(dims) == EG_MLA_OK ? q8_row_bytes(*dims) : 0;
}

extern "C" eg_mla_status eg_mla_quant_write(const eg_mla_dims* dims, const eg_mla_rope* rope, int32_t n_tokens, const void* kv,
                                            int64_t kv_stride, const void* kv_norm_w, const void* k_norm_w,
                                            const void* gate_table, const int32_t* token_ids, const int32_t* positions,
                                            const int32_t* slots, uint8_t* codes, uint8_t* scales, int64_t num_slots,
                                            void* stream_) {
  const eg_mla_status st = validate_q8_write(dims, rope, n_tokens, kv, kv_stride, kv_norm_w, k_norm_w, gate_table,
                                             token_ids, positions, slots, codes, scales, num_slots);
  if (st != EG_MLA_OK || n_tokens == 0) return st;
  const eg_mla_dims& d = *dims;
  Q8WriteArgs a;
  a.kv = static_cast<const uint16_t*>(kv);
  a.kv_w = static_cast<const uint16_t*>(kv_norm_w);
  a.k_w = static_cast<const uint16_t*>(k_norm_w);
  a.gate = static_cast<const uint16_t*>(gate_table);
  a.ids = token_ids;
  a.positions = rope && d.rope_dim ? positions : nullptr;
  a.slots = slots;
  a.codes = codes;
  a.scales = scales;
  a.kv_stride = kv_stride;
  a.num_slots = num_slots;
  a.n = n_tokens;
  a.DC = d.latent_dim;
  a.DR = d.rope_dim;
  a.V = d.vocab_size;
  a.half = rope && rope->layout == EG_MLA_ROPE_HALF;
  a.magnitude = rope ? magnitude_of(*rope) : 1.f;
  if (rope) turns_of(*rope, d.rope_dim / 2, a.freq);
  const int lpt = d.latent_dim <= 128 ? 16 : d.latent_dim <= 256 ? 32 : 64;
  const dim3 grid = long_grid((static_cast<int64_t>(n_tokens) + kQ8Threads / lpt - 1) / (kQ8Threads / lpt)), block(kQ8Threads);
  hipStream_t stream = static_cast<hipStream_t>(stream_);
  (void)hipGetLastError();
  if (lpt == 16) hipLaunchKernelGGL((q8_write_kernel<16>), grid, block, 0, stream, a);
  else if (lpt == 32) hipLaunchKernelGGL((q8_write_kernel<32>), grid, block, 0, stream, a);
  else hipLaunchKernelGGL((q8_write_kernel<64>), grid, block, 0, stream, a);
  return hipGetLastError() == hipSuccess ? EG_MLA_OK : EG_MLA_ERR_HIP;
}

extern "C" eg_mla_status eg_mla_quant_read(const eg_mla_dims* dims, int32_t batch, int32_t total_tokens, const uint8_t* codes,
                                           const uint8_t* scales, const int32_t* first_tokens, const int32_t* cu_seqlens,
                                           const int32_t* page_table, int32_t max_pages_per_seq, int64_t num_slots,
                                           void* out, void* stream_) {
  const eg_mla_status st = validate_q8_read(dims, batch, total_tokens, codes, scales, first_tokens, cu_seqlens,
                                            page_table, max_pages_per_seq, num_slots, out);
  if (st != EG_MLA_OK || batch == 0 || total_tokens == 0 || max_pages_per_seq == 0) return st;
  const eg_mla_dims& d = *dims;
  const Q8ReadArgs a{codes, scales, first_tokens, cu_seqlens, page_table, static_cast<uint16_t*>(out), num_slots, batch,
                     total_tokens, max_pages_per_seq, d.page_size, d.latent_dim, d.rope_dim};
  (void)hipGetLastError();
  hipLaunchKernelGGL(q8_read_kernel, long_grid((static_cast<int64_t>(total_tokens) + kQ8ReadTokens - 1) / kQ8ReadTokens),
                     dim3(kQ8Threads), 0, static_cast<hipStream_t>(stream_), a);
  return hipGetLastError() == hipSuccess ? EG_MLA_OK : EG_MLA_ERR_HIP;
}
