// Attention of new tokens over the 8-bit latent cache (gfx950): one new token a
// sequence (decode) or several, causal among themselves.
//
// With the gated latent c~ and k^R in the cache, query row (i, h) of a sequence
// of n new tokens among its `len` cached ones computes, in the absorbed form of
// App. C Eq. (C.11)-(C.13),
//   s_j = tau (q_lat . c~_j + q^R . k^R_j),  j < len - n + i + 1,  q_lat = W_UK[h]^T q^C
//   out = W_UV[h] sum_j softmax_j(s) c~_j.
// All rows of a sequence share the keys, whatever their head and token.  They
// are cut into blocks of consecutive rows, a block's keys into tiles, and the
// tiles of all blocks, in order, into equal runs, one for each work-group (a run
// may span blocks).  Three launches:
//  1. q8_prep_kernel: the query's absorption, 16-bit rows, and (one work-group) blocks, tiles and runs from the lengths
//     on the device;
//  2. q8_attend_kernel or, for blocks of 128 rows, q8_rows_kernel (quant_rows.h): a partial row (maximum, sum, latent
//     sum) for each row of each piece (the tiles of one block in one run);
//  3. q8_merge_kernel: joins the partial rows of a query row and applies W_UV.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>

#include "absorb.h"
#include "absorb_tile.h"
#include "device_common.h"
#include "eg_mla.h"
#include "host_plan.h"
#include "quant_blocks.h"

namespace egmla {

// ---------------------------------------------------------------------------
// Schedule
// ---------------------------------------------------------------------------
struct Q8Sched {
  const int32_t* cu;        // [B + 1], or null: one new token a sequence
  const int32_t* seq_lens;  // [B]
  // Places: the tiles of all blocks in order, `lead` places left free before each block's (a piece costs about as much
  // as that many tiles before its first and after its last).
  int4* info;               // [blocks]: sequence, first row in it, rows, place of the first tile
  int4* rows;               // [blocks]: first query row, first new token's position (may be negative), length, place
                            // behind the last tile
  int4* start;              // [runs][3]: the first block with tiles from a run's first place on (its number, places of a
                            // run, blocks, places in all; its info; its rows): what a run starts with, in one load
  int2* tokens;             // [T]: the sequence's first block and the token's number in it; -1: no sequence's
  int32_t* head;            // places of a run, blocks
  int32_t B, T, H, cap, block_rows, tile, runs, lead;
};

// Exclusive sum over the work-group's threads, and the total.
template <int THREADS>
__device__ __forceinline__ int group_scan(int v, int* tmp, int& total) {
  const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
  int x = v;
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) {
    const int y = __shfl_up(x, o, 64);
    if (lane >= o) x += y;
  }
  __syncthreads();  // the sums before have been read
  if (lane == 63) tmp[w] = x;
  __syncthreads();
  int before = 0;
  total = 0;
#pragma unroll
  for (int i = 0; i < THREADS / 64; ++i) {
    if (i < w) before += tmp[i];
    total += tmp[i];
  }
  return before + x - v;
}

// First i in [0, n) with a[i + 1] > x (n if none); a is non-decreasing.
__device__ __forceinline__ int first_above(const int* a, int n, int x) {
  int lo = 0, hi = n;
  while (lo < hi) {
    const int mid = (lo + hi) / 2;
    if (a[mid + 1] > x) hi = mid;
    else lo = mid + 1;
  }
  return lo;
}

template <int THREADS>
__device__ __forceinline__ void q8_schedule(const Q8Sched& a) {
  __shared__ int first_s[kPageMaxBatch + 1];  // a sequence's first block
  __shared__ int tmp[THREADS / 64];
  const int tid = threadIdx.x;
  auto first_token = [&](int b) { return a.cu ? clamp_len(a.cu[b], a.T) : min(b, a.T); };
  for (int t = tid; t < a.T; t += THREADS) a.tokens[t] = make_int2(-1, 0);
  for (int g = tid; g < a.runs; g += THREADS) a.start[3 * g] = make_int4(0, 0, 0, 0);  // no places
  const int most = q8_most_blocks(a.T, a.H, a.block_rows, a.B);
  int total = 0, blocks = 0;
  static_assert(THREADS <= 256, "sequences of a step of the count");
  for (int b0 = 0; b0 < a.B; b0 += THREADS) {
    const int b = b0 + tid;
    const int mine = b < a.B ? q8_sequence_blocks(first_token(b), first_token(b + 1), a.H, a.block_rows) : 0;
    const int at = group_scan<THREADS>(mine, tmp, total);
    if (b < a.B) first_s[b] = q8_blocks_behind(blocks, at, most);
    blocks = q8_blocks_behind(blocks, total, most);
  }
  if (tid == 0) first_s[a.B] = blocks;
  __syncthreads();
  int tiles = 0;
  for (int k0 = 0; k0 < blocks; k0 += THREADS) {
    const int k = k0 + tid;
    int n_tiles = 0, b = 0, row0 = 0, rows = 0, first = 0, len = 0, cu = 0;
    if (k < blocks) {
      b = first_above(first_s, a.B, k);
      cu = first_token(b);
      const int n = first_token(b + 1) - cu;
      row0 = (k - first_s[b]) * a.block_rows;
      rows = min(a.block_rows, n * a.H - row0);
      len = clamp_len(a.seq_lens[b], a.cap);
      first = len - n;
      const int most_keys = min(max(first + (row0 + rows - 1) / a.H + 1, 0), len);
      n_tiles = (most_keys + a.tile - 1) / a.tile;
      // the tokens whose first row is in this block
      for (int i = (row0 + a.H - 1) / a.H; i * a.H < row0 + rows; ++i) a.tokens[cu + i] = make_int2(first_s[b], i);
    }
    const int lead = n_tiles ? a.lead : 0;
    const int at = group_scan<THREADS>(n_tiles + lead, tmp, total);
    if (k < blocks) {
      a.info[k] = make_int4(b, row0, rows, tiles + at + lead);
      a.rows[k] = make_int4(cu * a.H + row0, first, len, tiles + at + lead + n_tiles);
    }
    tiles += total;
  }
  const int per = max(1, (tiles + a.runs - 1) / a.runs);
  if (tid == 0) {
    a.head[0] = per;
    a.head[1] = blocks;
  }
  auto put = [&](int g, int k, int4 info, int4 rows) {
    a.start[3 * g] = make_int4(k, per, blocks, tiles);
    a.start[3 * g + 1] = info;
    a.start[3 * g + 2] = rows;
  };
  __threadfence_block();
  __syncthreads();
  if (blocks <= kPageMaxBatch) {  // a thread a run: the first block that ends behind the run's first place
    for (int k = tid; k <= blocks; k += THREADS) first_s[k] = k ? a.rows[k - 1].w : 0;
    __syncthreads();
    for (int g = tid; g < a.runs && static_cast<int64_t>(g) * per < tiles; g += THREADS) {
      const int k = first_above(first_s, blocks, g * per);
      put(g, k, a.info[k], a.rows[k]);
    }
  } else {  // more blocks than runs: few runs start in one
    for (int k = tid; k < blocks; k += THREADS) {
      const int4 info = a.info[k], rows = a.rows[k];
      const int s = rows.w == info.w ? rows.w : info.w - a.lead;
      for (int g = (s + per - 1) / per; g < a.runs && static_cast<int64_t>(g) * per < rows.w; ++g) put(g, k, info, rows);
    }
  }
}

// Schedule (work-group 0) and absorption in one launch: 16-bit rows [q_lat fp16 | q^R bf16].
struct Q8Prep {
  const uint16_t* q;
  const uint16_t* w_uk;
  uint16_t* rows;
  int32_t T, H, DH, DC, DR, row_blocks;
};
template <int DH, int BLOCKS, int COLS>
__global__ __launch_bounds__(256) void q8_prep_kernel(Q8Prep p, Q8Sched a) {
  if (blockIdx.x == 0) {
    q8_schedule<256>(a);
    return;
  }
  const int wg = blockIdx.x - 1, h = wg % p.H, rest = wg / p.H;
  absorb_tile<DH, BLOCKS, COLS, AbsorbRows::kHalf>(p.q, p.w_uk, nullptr, p.rows, p.T, p.H, p.DC, p.DR, h,
                                                   rest % p.row_blocks, rest / p.row_blocks);
}

__global__ __launch_bounds__(256) void q8_prep_any_kernel(Q8Prep p, Q8Sched a) {  // (for any d_h)
  extern __shared__ float smem[];
  if (blockIdx.x == 0) {
    q8_schedule<256>(a);
    return;
  }
  const int wg = blockIdx.x - 1, h = wg % p.H, rest = wg / p.H;
  absorb_any_tile<true, true>(p.q, p.w_uk, reinterpret_cast<float*>(p.rows), p.T, p.H, p.DH, p.DC, p.DR, h,
                              rest / p.row_blocks, rest % p.row_blocks, smem);
}

// ---------------------------------------------------------------------------
// Attention of blocks of 16 rows.  A wave owns units of U tokens of all
// dims: it loads their rows (16 bytes a lane, the next unit's while it computes
// one), turns the codes into fp16 with the row's scale in the conversion (exact
// within fp16's range), stages them in its own LDS tile and takes both MFMA
// operands from there, so the waves share nothing until they merge at a piece's
// end.  The RoPE key stays bf16 and exact; the absorbed query and the
// probabilities are rounded once to fp16; sums, maxima and products are fp32.  A
// row that stands for NaN has zeros for values and a NaN RoPE key, so that it
// reaches the rows that attend to it through their score, and no other; values
// that are not finite: q8_only_finite.  Bound
// by HBM for long calls: 256 sequences of 250-8192 tokens, 16 heads of d_c 128,
// 57 us, 4.9 TB/s.
// ---------------------------------------------------------------------------
// Cache rows of tokens: those of a page table, or contiguous ones.  No index leaves the cache, and no branch is taken
// (a load under one is waited for where the branch ends).
struct Q8Pages {
  const int32_t* table;  // contiguous rows: any readable word
  int32_t paged, P, npages, max_pages, cap;
  uint32_t mul, shift;   // j / P = j mul >> shift for 0 <= j < 2^31
  __device__ __forceinline__ int column(int j) const {
    return static_cast<int>(static_cast<uint64_t>(static_cast<uint32_t>(j)) * mul >> shift);
  }
  __device__ __forceinline__ int page(int b, int j) const {
    return table[paged ? static_cast<int64_t>(b) * max_pages + column(j) : 0];
  }
  __device__ __forceinline__ int row(int b, int j, int page) const {  // given the token's entry of the table
    const int r = min(max(page, 0), npages - 1) * P + (j - column(j) * P);
    return paged ? r : b * cap + j;
  }
};

struct Q8Attend {
  const uint16_t* q;  // [T, H, DC + DR]: q_lat fp16 | q^R bf16
  const uint8_t* codes;
  const uint8_t* scales;
  Q8Pages cache;
  const int4* info;
  const int4* rows;
  const int4* start;
  float* part_ml;  // [piece][block rows][2]
  float* part_o;   // [piece][block rows][DC]: sums O
  int32_t H, DC, DR;
  float scale_log2;
};

constexpr int kQ8AttendThreads = 256;

// Values that are the same in every lane, in scalar registers.
__device__ __forceinline__ int uniform(int x) { return __builtin_amdgcn_readfirstlane(x); }
__device__ __forceinline__ int4 uniform(int4 x) { return make_int4(uniform(x.x), uniform(x.y), uniform(x.z), uniform(x.w)); }

template <int DCP>
struct Q8Cfg {
  static constexpr int NW = kQ8AttendThreads / 64;
  static constexpr int U = DCP <= 128 ? 32 : 16;  // tokens of a unit
  static constexpr int KB = U / 16;
  static constexpr int TILE = NW * U;             // tokens of a tile
  static constexpr int NC = DCP / 32, NR = 2, NB = DCP / 16;
  static constexpr int TS = DCP + 64 + 8;         // row of a tile: latent (fp16) | RoPE key (bf16) | 16 bytes
  static constexpr int PL = DCP / 16;             // 16-byte pieces of a token's codes
  static constexpr int NLI = U * PL / 64, NRI = U * 8 / 64;
  static constexpr int LDS_TILE = NW * U * TS * 2;
  static_assert(U * PL % 64 == 0 && NB % 2 == 0 && NW * (NB / 2) * 1024 <= LDS_TILE, "whole loads; half of the accumulators");
};

// 16 codes times their scale in fp16.
__device__ __forceinline__ void q8_to_f16(u32x4_t w, float s, u32x4_t& lo, u32x4_t& hi) {
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const uint32_t p = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(w[i], s, false));
    const uint32_t q = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(w[i], s, true));
    if (i < 2) {
      lo[2 * i] = p;
      lo[2 * i + 1] = q;
    } else {
      hi[2 * i - 4] = p;
      hi[2 * i - 3] = q;
    }
  }
}

// Values that fp16 does not hold (from 63488 on, which round to codes past 240 2^8, and NaN codes) are infinities or NaN in a
// tile.  Rows that attend to such a token become NaN, as their scores and values do.  One that does not has it in its value
// products all the same where other rows of the block attend to it, with a probability of 0, which an infinity or NaN times
// is none: in the tiles where some row's tokens end such values become zeros and the token's RoPE key a NaN, which reaches
// through their scores the rows that attend to it, and no other.
constexpr u32x4_t kQ8NanKey = {0x7fc07fc0u, 0x7fc07fc0u, 0x7fc07fc0u, 0x7fc07fc0u};
__device__ __forceinline__ void q8_only_finite(u32x4_t* values, u32x4_t* key) {  // (8 fp16 values; a piece of their RoPE key)
  const u32x4_t v = *values;
  uint32_t full = 0;  // exponents of all ones carry
#pragma unroll
  for (int i = 0; i < 4; ++i) full |= (v[i] & 0x7fff7fffu) + 0x04000400u;
  if ((full & 0x80008000u) == 0) return;
  *values = u32x4_t{0u, 0u, 0u, 0u};
  *key = kQ8NanKey;
}

// Eight values of a query row's part of n, zero behind its end.
__device__ __forceinline__ u32x4_t q8_query(const uint16_t* part, int d, int n) {
  return d < n ? *reinterpret_cast<const u32x4_t*>(part + d) : u32x4_t{0u, 0u, 0u, 0u};
}

template <int DCP>
__global__ __launch_bounds__(kQ8AttendThreads, DCP <= 320 ? 2 : 1) void q8_attend_kernel(Q8Attend a) {
  using C = Q8Cfg<DCP>;
  constexpr int NW = C::NW, U = C::U, KB = C::KB, NC = C::NC, NR = C::NR, NB = C::NB, TS = C::TS, PL = C::PL;
  __shared__ __attribute__((aligned(16))) unsigned char lds[C::LDS_TILE + 2 * NW * 16 * 4];
  f32x4_t* obuf = reinterpret_cast<f32x4_t*>(lds);  // [NW][NB / 2][64], at a piece's end
  float* mbuf = reinterpret_cast<float*>(lds + C::LDS_TILE);  // [NW][16]
  float* lbuf = mbuf + NW * 16;
  const int tid = threadIdx.x, lane = tid & 63, r16 = lane & 15, g = lane >> 4;
  const int w = __builtin_amdgcn_readfirstlane(tid >> 6);
  uint16_t* tile = reinterpret_cast<uint16_t*>(lds) + w * U * TS;
  const int row_bytes = a.DC + 2 * a.DR;

  const int run = xcd_logical_block(blockIdx.x, gridDim.x);
  const int4 mine = uniform(a.start[3 * run]);
  int4 info = uniform(a.start[3 * run + 1]), rw = uniform(a.start[3 * run + 2]);
  const int per = mine.y, blocks = mine.z, tiles = mine.w;
  int at = run * per;
  if (static_cast<int64_t>(run) * per >= tiles) return;
  const int end = min(at + per, tiles);
  for (int k = mine.x; k < blocks; ++k) {
    if (k != mine.x) {
      info = uniform(a.info[k]);
      rw = uniform(a.rows[k]);
    }
    at = max(at, info.w);
    if (at >= end) break;
    const int next = rw.w;
    if (next <= at) continue;  // a block without tokens
    const int b = info.x, row0 = info.y, nrows = info.z, first = rw.y, len = rw.z;
    const int most = min(max(first + (row0 + nrows - 1) / a.H + 1, 0), len);
    const int j0 = (at - info.w) * C::TILE, j1 = min((min(end, next) - info.w) * C::TILE, most);
    const int all = min(first + row0 / a.H + 1, len);  // tokens that every row attends to
    at = min(end, next);

    // this lane's query row (rows past the last repeat it and are not stored) and the tokens that it attends to
    const int r = min(r16, nrows - 1);
    const int lim = min(first + (row0 + r) / a.H + 1, len);
    const uint16_t* qrow = a.q + (static_cast<int64_t>(rw.x) + r) * (a.DC + a.DR);
    f16x8_t qv[NC];
    bf16x8_t qr[NR];
#pragma unroll
    for (int c = 0; c < NC; ++c) qv[c] = __builtin_bit_cast(f16x8_t, q8_query(qrow, 32 * c + 8 * g, a.DC));
#pragma unroll
    for (int c = 0; c < NR; ++c) qr[c] = __builtin_bit_cast(bf16x8_t, q8_query(qrow + a.DC, 32 * c + 8 * g, a.DR));

    f32x4_t o[NB];
#pragma unroll
    for (int i = 0; i < NB; ++i) o[i] = f32x4_t{0.f, 0.f, 0.f, 0.f};
    float m_run = -INFINITY, l_run = 0.f;

    const int nunits = (j1 - j0 + U - 1) / U;
    // slot of this lane's token of unit u (tokens past the last repeat it and are masked)
    auto slot_of = [&](int u) {
      const int j = min(j0 + u * U + (lane & (U - 1)), j1 - 1);
      return a.cache.row(b, j, a.cache.page(b, j));
    };
    u32x4_t lat[C::NLI], rop[C::NRI];
    int sc = 0;
    auto issue = [&](int slot) {
      sc = a.scales[slot];
#pragma unroll
      for (int c = 0; c < C::NLI; ++c) {
        const int p = c * 64 + lane, t = p / PL, d = 16 * (p % PL);
        const int64_t s = __shfl(slot, t, 64);
        lat[c] = u32x4_t{0u, 0u, 0u, 0u};
        if (d < a.DC) lat[c] = __builtin_nontemporal_load(reinterpret_cast<const u32x4_t*>(a.codes + s * row_bytes + d));
      }
#pragma unroll
      for (int c = 0; c < C::NRI; ++c) {
        const int p = c * 64 + lane, t = p / 8, d = 8 * (p % 8);
        const int64_t s = __shfl(slot, t, 64);
        rop[c] = u32x4_t{0u, 0u, 0u, 0u};
        if (d < a.DR)
          rop[c] = __builtin_nontemporal_load(reinterpret_cast<const u32x4_t*>(a.codes + s * row_bytes + a.DC + 2 * d));
      }
    };
    if (w < nunits) {
      issue(slot_of(w));
      int slot = slot_of(w + NW);
      const uint16_t* arow = tile + r16 * TS + 8 * g;
      uint16_t* tread = tile + (4 * g + (r16 >> 2)) * TS + 4 * (r16 & 3);
      for (int u = w; u < nunits; u += NW) {
#pragma unroll
        for (int c = 0; c < C::NLI; ++c) {
          const int p = c * 64 + lane, t = p / PL;
          const int e = __shfl(sc, t, 64);
          u32x4_t lo, hi;
          q8_to_f16(lat[c], e == 255 ? 1.f : __uint_as_float(static_cast<uint32_t>(e) << 23), lo, hi);
          u32x4_t* dst = reinterpret_cast<u32x4_t*>(tile + t * TS + 16 * (p % PL));
          dst[0] = lo;
          dst[1] = hi;
        }
#pragma unroll
        for (int c = 0; c < C::NRI; ++c) {
          const int p = c * 64 + lane, t = p / 8;
          const uint32_t none = __shfl(sc, t, 64) == 255 ? 0x7fc07fc0u : 0u;
          *reinterpret_cast<u32x4_t*>(tile + t * TS + DCP + 8 * (p % 8)) = rop[c] | u32x4_t{none, none, none, none};
        }
        if (u + NW < nunits) {
          issue(slot);
          slot = slot_of(u + 2 * NW);
        }
        wave_lds_sync();
        if (min(j0 + (u + 1) * U, j1) > all) {
#pragma unroll 1
          for (int p = lane; p < U * DCP / 8; p += 64) {
            uint16_t* row = tile + p / (DCP / 8) * TS;
            q8_only_finite(reinterpret_cast<u32x4_t*>(row + 8 * (p % (DCP / 8))), reinterpret_cast<u32x4_t*>(row + DCP));
          }
          wave_lds_sync();
        }
        // S^T[token 16 kb + 4g + i][row r16]
        const int left = lim - (j0 + u * U);  // tokens of the unit that the row attends to
        float x[KB][4];
        float mt = -INFINITY;
#pragma unroll
        for (int kb = 0; kb < KB; ++kb) {
          f32x4_t acc = {0.f, 0.f, 0.f, 0.f}, acc2 = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
          for (int c = 0; c < NC; ++c)
            acc = __builtin_amdgcn_mfma_f32_16x16x32_f16(*reinterpret_cast<const f16x8_t*>(arow + 16 * kb * TS + 32 * c),
                                                         qv[c], acc, 0, 0, 0);
#pragma unroll
          for (int c = 0; c < NR; ++c)
            acc2 = __builtin_amdgcn_mfma_f32_16x16x32_bf16(
                *reinterpret_cast<const bf16x8_t*>(arow + 16 * kb * TS + DCP + 32 * c), qr[c], acc2, 0, 0, 0);
          acc += acc2;
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            x[kb][i] = 16 * kb + 4 * g + i < left ? acc[i] * a.scale_log2 : -INFINITY;
            mt = fmaxf(mt, x[kb][i]);
          }
        }
        mt = max_over_row_groups(mt);
        const float m_new = fmaxf(m_run, mt);
        const bool grow = m_new > m_run + kLazyRescale;
        if (__builtin_amdgcn_ballot_w64(grow)) {
          const float alpha = grow ? __builtin_amdgcn_exp2f(m_run - m_new) : 1.0f;
          m_run = grow ? m_new : m_run;
          l_run *= alpha;
#pragma unroll
          for (int db = 0; db < NB; ++db) o[db] *= alpha;
        }
        // (-inf while the row has met no token, or only scores that overflowed to it: those weigh nothing)
        const float m_ref = m_run == -INFINITY ? 0.f : m_run;
        uint32_t pk[KB][2];
#pragma unroll
        for (int kb = 0; kb < KB; ++kb) {
          float p[4];
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            p[i] = __builtin_amdgcn_exp2f(x[kb][i] - m_ref);
            l_run += p[i];
          }
          pk[kb][0] = pack_f16x2(p[0], p[1]);
          pk[kb][1] = pack_f16x2(p[2], p[3]);
        }
#pragma unroll
        for (int db = 0; db < NB; ++db) {
          const s16x4_t a0 =
              __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s16x4_t*)(tread + db * 16));
          if constexpr (KB == 2) {
            const s16x4_t a1 = __builtin_amdgcn_ds_read_tr16_b64_v4i16(
                (__attribute__((address_space(3))) s16x4_t*)(tread + 16 * TS + db * 16));
            o[db] = __builtin_amdgcn_mfma_f32_16x16x32_f16(
                __builtin_bit_cast(f16x8_t, __builtin_shufflevector(a0, a1, 0, 1, 2, 3, 4, 5, 6, 7)),
                __builtin_bit_cast(f16x8_t, u32x4_t{pk[0][0], pk[0][1], pk[KB - 1][0], pk[KB - 1][1]}), o[db], 0, 0, 0);
          } else {
            o[db] = __builtin_amdgcn_mfma_f32_16x16x16f16(
                __builtin_bit_cast(f16x4_t, a0), __builtin_bit_cast(f16x4_t, u32x2_t{pk[0][0], pk[0][1]}), o[db], 0, 0, 0);
          }
        }
        wave_lds_sync();
      }
    }

    // merge of the waves, the value blocks in two halves
    l_run = sum_over_row_groups(l_run);
    if (g == 0) mbuf[w * 16 + r16] = m_run;
    __syncthreads();  // also: every wave is done with its tile (obuf aliases them)
    float M = -INFINITY;
#pragma unroll
    for (int v = 0; v < NW; ++v) M = fmaxf(M, mbuf[v * 16 + r16]);
    // (a wave without a maximum may hold a NaN sum: it stays one)
    const float fold = m_run == -INFINITY ? (M == -INFINITY ? 1.f : 0.f) : __builtin_amdgcn_exp2f(m_run - M);
    if (g == 0) lbuf[w * 16 + r16] = l_run * fold;
    const int64_t prow = (static_cast<int64_t>(run) + k) * 16 + r16;
#pragma unroll
    for (int half = 0; half < 2; ++half) {
      if (half) __syncthreads();  // the first half's sums are read
#pragma unroll
      for (int db = 0; db < NB / 2; ++db) obuf[(w * (NB / 2) + db) * 64 + lane] = o[half * (NB / 2) + db] * fold;
      __syncthreads();
      for (int db = w; db < NB / 2; db += NW) {
        f32x4_t sum = obuf[db * 64 + lane];
#pragma unroll
        for (int v = 1; v < NW; ++v) sum += obuf[(v * (NB / 2) + db) * 64 + lane];
        const int d = (half * (NB / 2) + db) * 16 + 4 * g;
        if (r16 < nrows && d < a.DC) __builtin_nontemporal_store(sum, reinterpret_cast<f32x4_t*>(a.part_o + prow * a.DC + d));
      }
    }
    if (w == 0 && g == 0 && r16 < nrows) {
      float Ls = 0.f;
#pragma unroll
      for (int v = 0; v < NW; ++v) Ls += lbuf[v * 16 + r16];
      *reinterpret_cast<float2*>(a.part_ml + prow * 2) = make_float2(M, Ls);
    }
    __syncthreads();  // the merge's buffers have been read
  }
}

}  // namespace egmla
#include "quant_rows.h"
namespace egmla {

// ---------------------------------------------------------------------------
// Merge and up-projection: grid (H, ceil(T / spt)), one head and spt = 1, 2, 4, ..
// new tokens per work-group (up to 16, or 32 of wide rows).  LPR lanes hold a row, 8 dims each; each group
// of LPR lanes is a worker.  With at least as many tokens as workers a worker takes
// its tokens (up to TPW) side by side, else a token's workers take its partial rows
// in turn and meet in LDS.  Rows are folded online in fp32, two or four loaded together;
// the merged row o / l goes to LDS as bf16 hi + lo, the B operands of out^T[v][token] =
// W_UV[h] o^T on v_mfma_f32_16x16x32_bf16, so that the up-projection adds only
// W_UV's own rounding.  Bound by its chain of loads (token, block, rows), behind
// which W_UV's rows arrive: 8.6 us for 32 and 256 tokens of 16 heads, 28.5 for 64 of
// 128 heads in blocks of 128 rows (half as many bytes a row, O / l in fp16: 23.8;
// W_UV before the rows, 16 tokens a work-group, also in fp16: 37).
// ---------------------------------------------------------------------------
struct Q8Merge {
  const float* part_ml;
  const void* part_o;  // fp32
  const int4* info;
  const int4* rows;
  const int2* tokens;
  const int32_t* head;
  const uint16_t* w_uv;
  uint16_t* out;
  int32_t T, H, DC, DV, block_rows, spt;
};

template <int LPR>
struct Q8MergeCfg {
  static constexpr int WAVES = LPR == 64 ? 8 : 4, WORKERS = WAVES * 64 / LPR;
  static constexpr int TOKENS = LPR == 64 ? 32 : 16;  // of a work-group, at most
  static constexpr int TPW = TOKENS / WORKERS;        // of a worker
  static_assert(TOKENS % WORKERS == 0, "whole rounds");
};

template <int LPR>
__global__ __launch_bounds__(Q8MergeCfg<LPR>::WAVES * 64, LPR == 64 ? 2 : 4) void q8_merge_kernel(Q8Merge a) {
  using C = Q8MergeCfg<LPR>;
  constexpr int DCP = 8 * LPR, NKC = DCP / 32, OS = DCP + 8, GPW = 64 / LPR, TPW = C::TPW, U = LPR == 64 ? 2 : 4;
  __shared__ __attribute__((aligned(16))) uint16_t o_s[2][C::TOKENS][OS];  // merged rows, hi and lo
  __shared__ __attribute__((aligned(16))) float part[C::WORKERS][DCP];
  __shared__ float m_part[C::WORKERS], l_part[C::WORKERS];
  const int h = blockIdx.x, t0 = blockIdx.y * a.spt;
  const int tid = threadIdx.x, w = tid >> 6, lane = tid & 63, r16 = lane & 15, g = lane >> 4;
  const int per = a.head[0], blocks = a.head[1];
  const int wps = max(1, C::WORKERS / a.spt);  // workers a token
  const int worker = w * GPW + lane / LPR, me = worker % wps, col = 8 * (lane % LPR);
  // this worker's tokens worker / wps + j WORKERS: how many partial rows they have, and the first
  int n[TPW];
  int64_t row0[TPW];
  {
    int2 tk[TPW];
    int k[TPW], s[TPW], e[TPW];
#pragma unroll
    for (int j = 0; j < TPW; ++j) {
      const int i = worker / wps + j * C::WORKERS;
      tk[j] = i < a.spt && t0 + i < a.T ? a.tokens[t0 + i] : make_int2(-1, 0);
    }
#pragma unroll
    for (int j = 0; j < TPW; ++j) {
      row0[j] = static_cast<int64_t>(tk[j].y) * a.H + h;
      k[j] = tk[j].x + static_cast<int>(row0[j] / a.block_rows);
      const bool there = tk[j].x >= 0 && k[j] < blocks;
      s[j] = there ? a.info[k[j]].w : 0;
      e[j] = there ? a.rows[k[j]].w : 0;
    }
#pragma unroll
    for (int j = 0; j < TPW; ++j) {
      const int first = s[j] / per;
      n[j] = e[j] > s[j] ? (e[j] - 1) / per - first + 1 : 0;
      row0[j] = (static_cast<int64_t>(first) + k[j]) * a.block_rows + row0[j] % a.block_rows;
    }
  }
  // rows i, i + wps of a token (repeats of the last past its end)
  struct Rows {
    float2 ml[U];
    u32x4_t x[U][2];
  };
  auto load = [&](Rows& r, int64_t first, int i, int n) {
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int64_t row = first + static_cast<int64_t>(min(i + u * wps, n - 1)) * a.block_rows;
      r.ml[u] = *reinterpret_cast<const float2*>(a.part_ml + 2 * row);
#pragma unroll
      for (int q = 0; q < 2; ++q) {
        r.x[u][q] = u32x4_t{0u, 0u, 0u, 0u};
        if (col < a.DC)
          r.x[u][q] = *reinterpret_cast<const u32x4_t*>(static_cast<const unsigned char*>(a.part_o) + (row * a.DC + col) * 4 + 16 * q);
      }
    }
  };
  Rows rows[TPW];
#pragma unroll
  for (int j = 0; j < TPW; ++j)
    if (me < n[j]) load(rows[j], row0[j], me, n[j]);
  // W_UV rows v0 + r16 (columns 32 kc + 8 g ..; zero past d_c, as the merged rows are)
  u32x4_t wa[NKC];
  auto load_w = [&](int v0) {
    const uint16_t* wrow = a.w_uv + (static_cast<int64_t>(h) * a.DV + min(v0 + r16, a.DV - 1)) * a.DC + 8 * g;
#pragma unroll
    for (int kc = 0; kc < NKC; ++kc)
      wa[kc] = 32 * kc + 8 * g < a.DC ? *reinterpret_cast<const u32x4_t*>(wrow + 32 * kc) : u32x4_t{0u, 0u, 0u, 0u};
  };
  load_w(16 * w);

  auto put = [&](int i, int c, const float (&v)[8]) {  // merged values c .. of token i
    bf16x8_t hi, lo;
#pragma unroll
    for (int q = 0; q < 8; ++q) {
      hi[q] = static_cast<__bf16>(v[q]);
      lo[q] = static_cast<__bf16>(v[q] - static_cast<float>(hi[q]));
    }
    *reinterpret_cast<bf16x8_t*>(&o_s[0][i][c]) = hi;
    *reinterpret_cast<bf16x8_t*>(&o_s[1][i][c]) = lo;
  };
#pragma unroll
  for (int j = 0; j < TPW; ++j) {
    float M = -INFINITY, sum = 0.f, acc[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
    for (int i = me; i < n[j]; i += U * wps) {
      const Rows r = rows[j];
      if (i + U * wps < n[j]) load(rows[j], row0[j], i + U * wps, n[j]);
      float top = M;
#pragma unroll
      for (int u = 0; u < U; ++u) top = fmaxf(top, r.ml[u].x);  // repeats change no maximum
      // (where no row has a maximum they are added all the same: a NaN in one stays one)
      const float ref = top == -INFINITY ? 0.f : top;
      const float keep = M > -INFINITY ? __builtin_amdgcn_exp2f(M - ref) : top > -INFINITY ? 0.f : 1.f;
      sum *= keep;
#pragma unroll
      for (int q = 0; q < 8; ++q) acc[q] *= keep;
#pragma unroll
      for (int u = 0; u < U; ++u) {
        if (i + u * wps >= n[j]) continue;
        const float x = top == -INFINITY ? 1.f : __builtin_amdgcn_exp2f(r.ml[u].x - ref);
        sum = fmaf(x, r.ml[u].y, sum);
#pragma unroll
        for (int q = 0; q < 8; ++q) acc[q] = fmaf(x, __uint_as_float(r.x[u][q / 4][q % 4]), acc[q]);
      }
      M = top;
    }
    if (wps == 1) {
      const int i = worker + j * C::WORKERS;
#pragma unroll
      for (int q = 0; q < 8; ++q) acc[q] = sum == 0.f ? 0.f : acc[q] / sum;  // (zero without keys)
      if (i < C::TOKENS) put(i, col, acc);
    } else {  // (one token a worker: j is 0)
      *reinterpret_cast<f32x4_t*>(&part[worker][col]) = f32x4_t{acc[0], acc[1], acc[2], acc[3]};
      *reinterpret_cast<f32x4_t*>(&part[worker][col + 4]) = f32x4_t{acc[4], acc[5], acc[6], acc[7]};
      if (lane % LPR == 0) {
        m_part[worker] = M;
        l_part[worker] = sum;
      }
      break;
    }
  }
  __syncthreads();
  if (wps > 1) {
    for (int i = tid; i < a.spt * LPR; i += C::WAVES * 64) {
      const int kk = i / LPR, c = 8 * (i % LPR);
      float top = -INFINITY, den = 0.f, num[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
      for (int p = 0; p < wps; ++p) top = fmaxf(top, m_part[kk * wps + p]);
      for (int p = 0; p < wps; ++p) {
        const float x = top == -INFINITY ? 1.f : __builtin_amdgcn_exp2f(m_part[kk * wps + p] - top);
        den = fmaf(x, l_part[kk * wps + p], den);
#pragma unroll
        for (int q = 0; q < 8; ++q) num[q] = fmaf(x, part[kk * wps + p][c + q], num[q]);
      }
#pragma unroll
      for (int q = 0; q < 8; ++q) num[q] = den == 0.f ? 0.f : num[q] / den;
      put(kk, c, num);
    }
    __syncthreads();
  }
  for (int v0 = 16 * w; v0 < a.DV; v0 += 16 * C::WAVES) {
    if (v0 != 16 * w) load_w(v0);
#pragma unroll
    for (int i0 = 0; i0 < C::TOKENS; i0 += 16) {
      if (i0 >= a.spt) continue;
      const int i = i0 + r16, rr = min(i, a.spt - 1);  // columns past spt repeat the last and are not stored
      f32x4_t o = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int kc = 0; kc < NKC; ++kc) {
        const bf16x8_t av = __builtin_bit_cast(bf16x8_t, wa[kc]);
#pragma unroll
        for (int part = 0; part < 2; ++part)
          o = __builtin_amdgcn_mfma_f32_16x16x32_bf16(
              av, *reinterpret_cast<const bf16x8_t*>(&o_s[part][rr][32 * kc + 8 * g]), o, 0, 0, 0);
      }
      const int t = t0 + i;
      if (i >= a.spt || t >= a.T || a.tokens[t].x < 0) continue;  // other rows stay as they are
      uint16_t* orow = a.out + (static_cast<int64_t>(t) * a.H + h) * a.DV + v0 + 4 * g;
      if (a.DV % 4 == 0) {
        if (v0 + 4 * g < a.DV) *reinterpret_cast<u32x2_t*>(orow) = u32x2_t{pack_bf16x2(o[0], o[1]), pack_bf16x2(o[2], o[3])};
        continue;
      }
#pragma unroll
      for (int e = 0; e < 4; ++e)
        if (v0 + 4 * g + e < a.DV) orow[e] = f32_to_bf16(o[e]);
    }
  }
}

}  // namespace egmla

using namespace egmla;

namespace {

hipError_t launch_q8_prep(const eg_mla_dims& d, int32_t n, const void* q, const void* w_uk, uint16_t* rows,
                          const Q8Sched& sched, hipStream_t stream) {
  // 64 queries a work-group where those of 16 would be many; narrow column slices where few
  const int64_t tiles = static_cast<int64_t>(d.num_heads) * ((n + kAbsRows - 1) / kAbsRows);
  const bool any = d.head_dim != 64 && d.head_dim != 128, grouped = !any && tiles >= 512, narrow = tiles < kAbsMinWorkGroups;
  const int cols = any ? kAbsorbCols : narrow ? kAbsColsNarrow : kAbsCols;
  const int block = any ? kAbsorbRows : kAbsRows * (grouped ? kAbsBlocks : 1);
  const Q8Prep p{static_cast<const uint16_t*>(q), static_cast<const uint16_t*>(w_uk), rows, n, d.num_heads, d.head_dim,
                 d.latent_dim, d.rope_dim, (n + block - 1) / block};
  const int64_t wgs = int64_t{d.num_heads} * p.row_blocks * ((d.latent_dim + cols - 1) / cols) + 1;
  auto kern = d.head_dim == 64 ? (grouped  ? q8_prep_kernel<64, kAbsBlocks, kAbsCols>
                                  : narrow ? q8_prep_kernel<64, 1, kAbsColsNarrow>
                                           : q8_prep_kernel<64, 1, kAbsCols>)
              : grouped ? q8_prep_kernel<128, kAbsBlocks, kAbsCols>
              : narrow  ? q8_prep_kernel<128, 1, kAbsColsNarrow>
                        : q8_prep_kernel<128, 1, kAbsCols>;
  size_t lds = 0;
  if (any) {
    kern = q8_prep_any_kernel;
    lds = absorb_any_lds(d.head_dim);  // up to 80 KB
    if (lds > 32768) {
      const hipError_t e = hipFuncSetAttribute(reinterpret_cast<const void*>(kern), hipFuncAttributeMaxDynamicSharedMemorySize,
                                               static_cast<int>(lds));
      if (e != hipSuccess) return e;
    }
  }
  hipLaunchKernelGGL(kern, dim3(static_cast<unsigned>(wgs)), dim3(256), lds, stream, p, sched);
  return hipGetLastError();
}

}  // namespace

extern "C" size_t eg_mla_quant_attend_workspace_size(const eg_mla_dims* dims, int32_t batch, int32_t n_queries,
                                                     int32_t max_pages_per_seq) {
  Q8Plan p;
  if (check_q8_dims(dims) != EG_MLA_OK || make_q8_plan(*dims, batch, n_queries, max_pages_per_seq, &p) != EG_MLA_OK) return 0;
  return p.bytes;
}

extern "C" eg_mla_status eg_mla_quant_attend(const eg_mla_dims* dims, int32_t batch, int32_t n_queries, const void* q,
                                             const int32_t* cu_seqlens, const uint8_t* codes, const uint8_t* scales,
                                             const void* w_uk, const void* w_uv, const int32_t* seq_lens,
                                             const int32_t* page_table, int32_t max_pages_per_seq, int64_t num_slots,
                                             void* workspace, size_t workspace_bytes, void* out, void* stream_) {
  Q8Plan p;
  const eg_mla_status st = validate_q8_attend(dims, batch, n_queries, q, cu_seqlens, codes, scales, w_uk, w_uv, seq_lens,
                                              page_table, max_pages_per_seq, num_slots, workspace, workspace_bytes, out, &p);
  if (st != EG_MLA_OK || batch == 0 || n_queries == 0) return st;
  const eg_mla_dims& d = *dims;
  hipStream_t stream = static_cast<hipStream_t>(stream_);
  unsigned char* ws = static_cast<unsigned char*>(workspace);
  uint16_t* qrows = reinterpret_cast<uint16_t*>(ws + p.off_q);
  const Q8Sched sched{cu_seqlens, seq_lens, reinterpret_cast<int4*>(ws + p.off_info), reinterpret_cast<int4*>(ws + p.off_rows),
                      reinterpret_cast<int4*>(ws + p.off_start), reinterpret_cast<int2*>(ws + p.off_tokens),
                      reinterpret_cast<int32_t*>(ws + p.off_head), batch, n_queries, d.num_heads, p.capacity, p.block_rows,
                      p.tile, p.runs, p.lead};
  (void)hipGetLastError();
  if (launch_q8_prep(d, n_queries, q, w_uk, qrows, sched, stream) != hipSuccess) return EG_MLA_ERR_HIP;
  Q8Pages pages{page_table ? page_table : sched.head, page_table != nullptr, d.page_size,
                static_cast<int32_t>(num_slots / d.page_size), max_pages_per_seq, p.capacity, 0, 31};
  while ((int64_t{1} << (pages.shift - 31)) < d.page_size) ++pages.shift;  // l = ceil(log2 P): mul = ceil(2^(31+l) / P) < 2^32
  pages.mul = static_cast<uint32_t>(((uint64_t{1} << pages.shift) + d.page_size - 1) / d.page_size);
  const Q8Attend at{qrows, codes, scales, pages, sched.info, sched.rows, sched.start,
                    reinterpret_cast<float*>(ws + p.off_ml), reinterpret_cast<float*>(ws + p.off_o),
                    d.num_heads, d.latent_dim, d.rope_dim, softmax_scale(d) * 1.4426950408889634f};
  const dim3 grid(p.runs), block(kQ8AttendThreads);
  if (p.block_rows == kQ8Rows) {
    if (d.latent_dim <= 64) hipLaunchKernelGGL((q8_rows_kernel<64>), grid, block, 0, stream, at);
    else if (d.latent_dim <= 128) hipLaunchKernelGGL((q8_rows_kernel<128>), grid, block, 0, stream, at);
    else if (d.latent_dim <= 320) hipLaunchKernelGGL((q8_rows_kernel<320>), grid, block, 0, stream, at);
    else hipLaunchKernelGGL((q8_rows_kernel<512>), grid, block, 0, stream, at);
  } else if (d.latent_dim <= 64) hipLaunchKernelGGL((q8_attend_kernel<64>), grid, block, 0, stream, at);
  else if (d.latent_dim <= 128) hipLaunchKernelGGL((q8_attend_kernel<128>), grid, block, 0, stream, at);
  else if (d.latent_dim <= 320) hipLaunchKernelGGL((q8_attend_kernel<320>), grid, block, 0, stream, at);
  else hipLaunchKernelGGL((q8_attend_kernel<512>), grid, block, 0, stream, at);
  // tokens of a merge work-group: as many as leave two work-groups a compute unit (of wide rows one: 8 waves)
  const bool wide = d.latent_dim > 128;
  int spt = wide ? Q8MergeCfg<64>::TOKENS : Q8MergeCfg<16>::TOKENS;
  while (spt > 1 && static_cast<int64_t>(d.num_heads) * ((n_queries + spt - 1) / spt) < (wide ? 256 : 512)) spt /= 2;
  const Q8Merge mg{at.part_ml, at.part_o, sched.info, sched.rows, sched.tokens, sched.head, static_cast<const uint16_t*>(w_uv),
                   static_cast<uint16_t*>(out), n_queries, d.num_heads, d.latent_dim, d.v_head_dim, p.block_rows, spt};
  const dim3 mgrid(d.num_heads, (n_queries + spt - 1) / spt);
  const dim3 mblock(64 * (wide ? Q8MergeCfg<64>::WAVES : Q8MergeCfg<16>::WAVES));
  auto merge = wide ? q8_merge_kernel<64> : q8_merge_kernel<16>;
  hipLaunchKernelGGL(merge, mgrid, mblock, 0, stream, mg);
  return hipGetLastError() == hipSuccess ? EG_MLA_OK : EG_MLA_ERR_HIP;
}
