// Sparse attention over cache pages (gfx950): the mean key of each page, a
// query's score of every page from it, and the pages that a query attends to.
// The decode over the chosen pages is eg_mla_decode on the table that
// eg_mla_select_pages writes.
//
//   mean[p]     = (1/n) sum_i [c_i (.) G[id_i] | k^R_i]      over the page's n cached tokens
//   score[b,j]  = max_h tau (q_lat[b,h] . mean_c + q^R[b,h] . mean_r)   of page j of sequence b
//
// With the gate in the latent space a page's mean key is one vector for all
// heads (the mean of c~ commutes with W_UK[h]), of the cache row's size.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>

#include "absorb.h"
#include "device_common.h"
#include "eg_mla.h"
#include "host_plan.h"

namespace egmla {

// ---------------------------------------------------------------------------
// Page means.  A work-group takes whole pages of one sequence: thread (r, c)
// adds piece c (16 bytes) of the page's rows r, r + rows, ...; the row lanes
// meet in LDS.  Sums are in 64 bits: the products of two bf16 values are exact
// there and a sum of up to 2^20 of them is off by far less than the last bit
// of its rounding, so that a mean does not depend on the order of its tokens
// (a page whose means are formed again from the same rows keeps its bits).
// Bound by the latency of length, table entry, id, row and gate row for a
// step's pages (so a page's ids load together, and kMeanBatch rows of a thread
// at a time: 8 sequences of the 128-head layer, 2 or 3 pages each, 22 us with
// one row after the other), by HBM for a prompt's.
// ---------------------------------------------------------------------------
constexpr int kMeanThreads = 512;
constexpr int kMeanGroups = 1024;  // work-groups, about
constexpr int kMeanBatch = 4;

struct MeansArgs {
  const void* cache;
  const int32_t* ids;
  const void* gate;
  const int32_t* first;  // or null
  const int32_t* lens;
  const int32_t* table;  // or null
  void* means;
  int64_t num_slots;
  int32_t DC, DR, P, W, V, cap;
};

template <bool BF16>
__device__ __forceinline__ void load_piece(const void* p, int64_t i, float (&v)[BF16 ? 8 : 4]) {
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

template <bool BF16>
__global__ __launch_bounds__(kMeanThreads) void page_means_kernel(MeansArgs a) {
  constexpr int N = BF16 ? 8 : 4;
  __shared__ double red[kMeanThreads * N];
  __shared__ int32_t id_s[kMeanThreads];
  const int b = blockIdx.x;
  const int DQ = a.DC + a.DR, np = DQ / N;  // np <= 160 pieces
  const int rows = kMeanThreads / np;
  const int tid = threadIdx.x, c = tid % np, r = tid / np;
  const int L = clamp_len(a.lens[b], a.cap);
  const int first = a.first ? max(a.first[b], 0) : 0;
  if (first >= L) return;
  const int64_t npages = a.num_slots / a.P;
  const bool gated = c * N < a.DC, adds = r < rows;
  for (int pg = first / a.P + blockIdx.y; static_cast<int64_t>(pg) * a.P < L; pg += gridDim.y) {
    const int n = min(a.P, L - pg * a.P);
    const int64_t page = a.table ? a.table[static_cast<int64_t>(b) * a.W + pg] : static_cast<int64_t>(b) * a.W + pg;
    if (page < 0 || page >= npages) continue;  // uniform: no such page of the cache
    double acc[N];
#pragma unroll
    for (int e = 0; e < N; ++e) acc[e] = 0.0;
    for (int base = 0; base < n; base += kMeanThreads) {  // the ids of up to kMeanThreads tokens at a time
      const int64_t slot0 = page * a.P + base;
      const int m = min(n - base, kMeanThreads);
      const int id = a.ids[slot0 + min(tid, m - 1)];
      for (int i0 = r, round = 0; round * rows * kMeanBatch < m; ++round, i0 += rows * kMeanBatch) {
        float x[kMeanBatch][N], g[kMeanBatch][N];
#pragma unroll
        for (int u = 0; u < kMeanBatch; ++u)  // rows past the last repeat it and are not added
          load_piece<BF16>(a.cache, (slot0 + min(i0 + u * rows, m - 1)) * DQ + c * N, x[u]);
        if (round == 0) {
          id_s[tid] = clamp_id(id, a.V);
          __syncthreads();
        }
        if (gated) {
#pragma unroll
          for (int u = 0; u < kMeanBatch; ++u)
            load_piece<BF16>(a.gate, static_cast<int64_t>(id_s[min(i0 + u * rows, m - 1)]) * a.DC + c * N, g[u]);
        }
#pragma unroll
        for (int u = 0; u < kMeanBatch; ++u) {
          if (!adds || i0 + u * rows >= m) continue;
#pragma unroll
          for (int e = 0; e < N; ++e)
            acc[e] += gated ? static_cast<double>(x[u][e]) * static_cast<double>(g[u][e]) : static_cast<double>(x[u][e]);
        }
      }
      __syncthreads();  // the ids have been read
    }
#pragma unroll
    for (int e = 0; e < N; ++e) red[e * kMeanThreads + tid] = acc[e];
    __syncthreads();
    for (int i = tid; i < DQ; i += kMeanThreads) {
      double s = 0.0;
      for (int k = 0; k < rows; ++k) s += red[(i % N) * kMeanThreads + k * np + i / N];
      // (straight from 64 bits: by way of fp32 it would be rounded twice, but for the compiler's folding the two)
      if constexpr (BF16)
        static_cast<uint16_t*>(a.means)[page * DQ + i] = __builtin_bit_cast(uint16_t, static_cast<__bf16>(s / n));
      else
        static_cast<float*>(a.means)[page * DQ + i] = static_cast<float>(s / n);
    }
    __syncthreads();
  }
}

// ---------------------------------------------------------------------------
// Page scores.  q rows are [q_lat | q^R] in fp32, from the absorption.
// ---------------------------------------------------------------------------
struct ScoreArgs {
  const float* qfull;  // [B, H, DC + DR]
  const void* means;
  const int32_t* lens;
  const int32_t* table;  // or null
  float* scores;         // [B, W]
  int64_t num_slots;
  int32_t H, DQ, P, W, cap;
  float scale;
};

// The page of column j of sequence b, clamped into the cache.
__device__ __forceinline__ int64_t score_page(const ScoreArgs& a, int b, int j) {
  const int64_t npages = a.num_slots / a.P;
  int64_t page = a.table ? a.table[static_cast<int64_t>(b) * a.W + j] : static_cast<int64_t>(b) * a.W + j;
  page = page < 0 ? 0 : page;
  return page < npages ? page : npages - 1;
}

// Any shape, fp32 arithmetic: one wave per page, lanes along the row.
template <bool BF16>
__global__ __launch_bounds__(256) void page_scores_kernel(ScoreArgs a) {
  const int b = blockIdx.x, lane = threadIdx.x & 63;
  const int pages = (clamp_len(a.lens[b], a.cap) + a.P - 1) / a.P;
  for (int j = blockIdx.y * 4 + (threadIdx.x >> 6); j < a.W; j += gridDim.y * 4) {
    float best = -INFINITY;
    if (j < pages) {
      const int64_t row = score_page(a, b, j) * a.DQ;
      float m[10];  // d_c + d_r <= 640
#pragma unroll
      for (int i = 0; i < 10; ++i) m[i] = lane + 64 * i < a.DQ ? ld<BF16>(a.means, row + lane + 64 * i) : 0.f;
      for (int h = 0; h < a.H; ++h) {
        const float* q = a.qfull + (static_cast<int64_t>(b) * a.H + h) * a.DQ;
        float s = 0.f;
#pragma unroll
        for (int i = 0; i < 10; ++i)
          if (lane + 64 * i < a.DQ) s = fmaf(q[lane + 64 * i], m[i], s);
        best = max_or_nan(best, wave_sum(s) * a.scale);
      }
    }
    if (lane == 0) a.scores[static_cast<int64_t>(b) * a.W + j] = best;
  }
}

// Matrix cores, bf16 storage: S[head][page] on v_mfma_f32_16x16x32_bf16, 16
// heads (A: the query's parts) by 16 pages (B: their means), both operands
// straight from global memory.  The products of bf16 values are exact and the
// three parts hold all of the fp32 query, so the scores are fp32 ones.  HW
// waves share a tile of TPW x 16 pages, each with every HW-th block of 16
// heads, and join their maxima in LDS; the other 8 / HW take the next tiles.
// An infinite mean times a zero part, or times parts of both signs, is a NaN
// that the fp32 product does not have: NaN scores are formed again from the
// whole query.
// Bound by latency for few heads, and by the query's parts through L2 for many
// (6 d_c + 2 d_r bytes a head, read once per tile of pages).
constexpr int kScoreWaves = 8;

constexpr int kScoreBatch = 4;

struct ScoreMfmaArgs {
  const uint16_t* parts;  // PartsLayout
  const uint16_t* means;
  ScoreArgs s;
  int32_t B, DC, groups;  // work-groups per sequence
};

// NC > 0: d_c = 32 NC and d_r = 64; 0: any.
template <int HW, int TPW, int NC>
__global__ __launch_bounds__(kScoreWaves * 64) void page_scores_mfma_kernel(ScoreMfmaArgs a) {
  __shared__ float best_s[kScoreWaves][TPW * 16];
  constexpr int PW = kScoreWaves / HW;
  // means that several waves take lie in LDS, rows padded by 16 bytes (the 16 rows of an operand read on distinct banks)
  constexpr bool STAGE = HW > 1 && NC > 0;
  constexpr int MROW = 32 * NC + 64 + 8;
  __shared__ __attribute__((aligned(16))) uint16_t mean_s[STAGE ? PW * TPW * 16 * MROW : 8];
  const int item = xcd_logical_block(blockIdx.x, gridDim.x);  // a sequence's work-groups share its query in an XCD's L2
  const int b = item / a.groups, lane = threadIdx.x & 63, w = threadIdx.x >> 6, r16 = lane & 15, g = lane >> 4;
  const int DC = NC ? 32 * NC : a.DC, DQ = NC ? DC + 64 : a.s.DQ, H = a.s.H;
  const int pages = (clamp_len(a.s.lens[b], a.s.cap) + a.s.P - 1) / a.s.P;
  const int p0 = ((item - b * a.groups) * PW + w / HW) * TPW * 16;  // this wave's first page
  float best[TPW];
#pragma unroll
  for (int t = 0; t < TPW; ++t) best[t] = -INFINITY;
  if constexpr (STAGE) {
    constexpr int PIECES = 4 * NC + 8, ALL = PW * TPW * 16 * PIECES, THREADS = kScoreWaves * 64;
    constexpr int PER = (ALL + THREADS - 1) / THREADS;
    const int wg0 = (item - b * a.groups) * PW * TPW * 16;
    if (wg0 < pages) {
      u32x4_t v[PER];
#pragma unroll
      for (int k = 0; k < PER; ++k) {  // rows past the last page repeat it
        const int i = min(static_cast<int>(threadIdx.x) + k * THREADS, ALL - 1), row = i / PIECES, c = i % PIECES;
        v[k] = *reinterpret_cast<const u32x4_t*>(a.means + score_page(a.s, b, min(wg0 + row, pages - 1)) * DQ + 8 * c);
      }
#pragma unroll
      for (int k = 0; k < PER; ++k) {
        const int i = threadIdx.x + k * THREADS, row = i / PIECES, c = i % PIECES;
        if (i < ALL) *reinterpret_cast<u32x4_t*>(mean_s + row * MROW + 8 * c) = v[k];
      }
    }
    __syncthreads();
  }
  if (p0 < pages) {
    const uint16_t* mrow[TPW];  // columns past the last page repeat it
#pragma unroll
    for (int t = 0; t < TPW; ++t) {
      if constexpr (STAGE) mrow[t] = mean_s + (w / HW * TPW * 16 + 16 * t + r16) * MROW + 8 * g;
      else mrow[t] = a.means + score_page(a.s, b, min(p0 + 16 * t + r16, pages - 1)) * DQ + 8 * g;
    }
    const PartsLayout layout(H, DC, DQ - DC);
    for (int h0 = 16 * (w % HW); h0 < H; h0 += 16 * HW) {
      // A operand of 32 values: this lane's 16 bytes of a run
      const uint16_t* q0 = a.parts + layout(b, h0, 0, 0) + 8 * lane;
      const uint16_t* q1 = a.parts + layout(b, h0, 1, 0) + 8 * lane;
      const uint16_t* q2 = a.parts + layout(b, h0, 2, 0) + 8 * lane;
      f32x4_t acc[TPW];
#pragma unroll
      for (int t = 0; t < TPW; ++t) acc[t] = f32x4_t{0.f, 0.f, 0.f, 0.f};
      const u32x4_t zero = {0u, 0u, 0u, 0u};
      // values k + 8g .. of a mean's row, and of the query's part; zeros past the row's end
      auto mean = [&](const uint16_t* p, int k) {
        return __builtin_bit_cast(bf16x8_t, NC || k + 8 * g < DQ ? *reinterpret_cast<const u32x4_t*>(p + k) : zero);
      };
      auto query = [&](const uint16_t* p, int k, int end) {
        return __builtin_bit_cast(bf16x8_t, NC || k + 8 * g < end ? *reinterpret_cast<const u32x4_t*>(p + 16 * k) : zero);
      };
      if constexpr (NC > 0) {
        // batches of kScoreBatch runs, the next one's loads in flight while one is multiplied; the RoPE runs (the
        // first part holds all of q^R) go out first and are multiplied last
        constexpr int NB = (NC + kScoreBatch - 1) / kScoreBatch;
        bf16x8_t xr[2], mr[2][TPW], x[2][kScoreBatch][3], m[2][kScoreBatch][TPW];
#pragma unroll
        for (int c = 0; c < 2; ++c) {
          xr[c] = query(q0, 32 * (NC + c), DQ);
#pragma unroll
          for (int t = 0; t < TPW; ++t) mr[c][t] = mean(mrow[t], 32 * (NC + c));
        }
        auto load = [&](int n) {
#pragma unroll
          for (int j = 0; j < kScoreBatch; ++j) {
            const int c = n * kScoreBatch + j;
            if (c >= NC) continue;
            x[n & 1][j][0] = query(q0, 32 * c, DQ);
            x[n & 1][j][1] = query(q1, 32 * c, DC);
            x[n & 1][j][2] = query(q2, 32 * c, DC);
#pragma unroll
            for (int t = 0; t < TPW; ++t) m[n & 1][j][t] = mean(mrow[t], 32 * c);
          }
        };
        load(0);
#pragma unroll
        for (int n = 0; n < NB; ++n) {
          if (n + 1 < NB) load(n + 1);
          __builtin_amdgcn_sched_barrier(0);
#pragma unroll
          for (int j = 0; j < kScoreBatch; ++j) {
            if (n * kScoreBatch + j >= NC) continue;
#pragma unroll
            for (int i = 0; i < 3; ++i)
#pragma unroll
              for (int t = 0; t < TPW; ++t)
                acc[t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(x[n & 1][j][i], m[n & 1][j][t], acc[t], 0, 0, 0);
          }
          __builtin_amdgcn_sched_barrier(0);
        }
#pragma unroll
        for (int c = 0; c < 2; ++c)
#pragma unroll
          for (int t = 0; t < TPW; ++t)
            acc[t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(xr[c], mr[c][t], acc[t], 0, 0, 0);
      } else {
        for (int k = 0; k < DQ; k += 32) {
          bf16x8_t m[TPW];
#pragma unroll
          for (int t = 0; t < TPW; ++t) m[t] = mean(mrow[t], k);
          const bf16x8_t x[3] = {query(q0, k, DQ), query(q1, k, DC), query(q2, k, DC)};
#pragma unroll
          for (int i = 0; i < 3; ++i)
#pragma unroll
            for (int t = 0; t < TPW; ++t) acc[t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(x[i], m[t], acc[t], 0, 0, 0);
        }
      }
      // lane: heads h0 + 4 g + 0..3 of page r16
#pragma unroll
      for (int t = 0; t < TPW; ++t) {
        bool lost = false;
#pragma unroll
        for (int r = 0; r < 4; ++r) lost = lost || (h0 + 4 * g + r < H && acc[t][r] != acc[t][r]);
        if (lost) {
          const uint16_t* m = a.means + score_page(a.s, b, min(p0 + 16 * t + r16, pages - 1)) * DQ;
          f32x4_t s = {0.f, 0.f, 0.f, 0.f};
#pragma unroll 1
          for (int c = 0; c < DQ; ++c) {
            const float mv = bf16_to_f32(m[c]);
#pragma unroll
            for (int r = 0; r < 4; ++r) {
              const int h = min(h0 + 4 * g + r, H - 1);
              float q = bf16_to_f32(a.parts[layout(b, h, 0, c)]);
              if (c < DC) q += bf16_to_f32(a.parts[layout(b, h, 1, c)]) + bf16_to_f32(a.parts[layout(b, h, 2, c)]);
              s[r] = fmaf(q, mv, s[r]);
            }
          }
          acc[t] = s;
        }
#pragma unroll
        for (int r = 0; r < 4; ++r)
          if (h0 + 4 * g + r < H) best[t] = max_or_nan(best[t], acc[t][r]);
      }
    }
#pragma unroll
    for (int t = 0; t < TPW; ++t) {  // over the lanes of a page
      best[t] = max_or_nan(best[t], __shfl_xor(best[t], 16, 64));
      best[t] = max_or_nan(best[t], __shfl_xor(best[t], 32, 64)) * a.s.scale;
    }
  }
  if constexpr (HW > 1) {
    if (g == 0) {
#pragma unroll
      for (int t = 0; t < TPW; ++t) best_s[w][16 * t + r16] = best[t];
    }
    __syncthreads();
    if (w % HW) return;
#pragma unroll
    for (int t = 0; t < TPW; ++t)
      for (int k = 1; k < HW; ++k) best[t] = max_or_nan(best[t], best_s[w + k][16 * t + r16]);
  }
#pragma unroll
  for (int t = 0; t < TPW; ++t) {
    const int j = p0 + 16 * t + r16;
    if (g == 0 && j < a.s.W) a.s.scores[static_cast<int64_t>(b) * a.s.W + j] = j < pages ? best[t] : -INFINITY;
  }
}

// ---------------------------------------------------------------------------
// Page selection: one work-group per sequence.  A page's key is its score as
// an unsigned number of the same order (a NaN counts as -inf, -0 as 0; pages
// that are always kept come first); the K-th largest key is found by four
// passes over 8 bits each (a histogram in LDS), then every key above it and
// the first ones equal to it are written in the order of the sequence.  A
// thread keeps its first page's key and number; where the lanes of a wave share a digit,
// as scores of like size do in the first ones, one lane counts for all of them.
// ---------------------------------------------------------------------------
constexpr int kSelThreads = 1024;

struct SelectArgs {
  const float* scores;
  const int32_t* lens;
  const int32_t* table;  // or null
  int32_t* sel;
  int32_t* sel_lens;
  int32_t* sel_index;  // or null
  int32_t W, P, K, cap, keep_first, keep_last;
};

__device__ __forceinline__ uint32_t score_key(float s) {
  if (s != s) s = -INFINITY;
  const uint32_t u = __float_as_uint(s + 0.f);  // -0 + 0 is +0
  return u & 0x80000000u ? ~u : u | 0x80000000u;
}

__global__ __launch_bounds__(kSelThreads) void select_pages_kernel(SelectArgs a) {
  __shared__ uint32_t hist[256];
  __shared__ uint32_t state[2];  // prefix of the K-th key, keys still to take among those with it
  __shared__ uint32_t above_w[kSelThreads / 64], equal_w[kSelThreads / 64];
  const int b = blockIdx.x, tid = threadIdx.x, lane = tid & 63, w = tid >> 6;
  const int L = clamp_len(a.lens[b], a.cap);
  const int n = (L + a.P - 1) / a.P;
  int32_t* sel = a.sel + static_cast<int64_t>(b) * a.K;
  int32_t* index = a.sel_index ? a.sel_index + static_cast<int64_t>(b) * a.K : nullptr;
  auto page_of = [&](int j) { return a.table ? a.table[static_cast<int64_t>(b) * a.W + j] : b * a.W + j; };
  if (tid == 0) a.sel_lens[b] = n <= a.K ? L : L - (n - a.K) * a.P;
  if (n <= a.K) {  // every page
    for (int j = tid; j < a.K; j += kSelThreads) {
      sel[j] = j < n ? page_of(j) : -1;
      if (index) index[j] = j < n ? j : -1;
    }
    return;
  }
  const float* score = a.scores + static_cast<int64_t>(b) * a.W;
  auto load_key = [&](int j) {
    return j < a.keep_first || j >= n - a.keep_last ? 0xffffffffu : score_key(score[j]);
  };
  const uint32_t first_key = tid < n ? load_key(tid) : 0u;
  const int32_t first_page = tid < n ? page_of(tid) : 0;
  auto key_of = [&](int j) { return j == tid ? first_key : load_key(j); };
  uint32_t prefix = 0, want = a.K;
  for (int shift = 24; shift >= 0; shift -= 8) {
    if (tid < 256) hist[tid] = 0;
    __syncthreads();
    for (int j = tid; j < n; j += kSelThreads) {
      const uint32_t k = key_of(j);
      if (shift == 24 || (k >> (shift + 8)) == prefix) {
        const uint32_t digit = (k >> shift) & 255u;
        const uint32_t common = __builtin_amdgcn_readfirstlane(digit);
        const uint64_t same = __ballot(digit == common);
        if (digit != common) atomicAdd(&hist[digit], 1u);
        else if (__builtin_ctzll(same) == lane) atomicAdd(&hist[common], static_cast<uint32_t>(__popcll(same)));
      }
    }
    __syncthreads();
    if (w == 0) {  // the digit whose keys hold the `want`-th from the top: lane l looks at digits 255 - 4 l ...
      uint32_t c[4], sum = 0;
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        c[e] = hist[255 - 4 * lane - e];
        sum += c[e];
      }
      uint32_t incl = sum;
#pragma unroll
      for (int o = 1; o < 64; o <<= 1) {
        const uint32_t u = __shfl_up(incl, o, 64);
        if (lane >= o) incl += u;
      }
      uint32_t before = incl - sum;
      if (before < want && want <= incl) {
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          if (before < want && want <= before + c[e]) {
            state[0] = (prefix << 8) | static_cast<uint32_t>(255 - 4 * lane - e);
            state[1] = want - before;
          }
          before += c[e];
        }
      }
    }
    __syncthreads();
    prefix = state[0];
    want = state[1];
  }
  // keys above `prefix`, and the first `want` equal to it, in order
  uint32_t above = 0, equal = 0;
  for (int j0 = 0; j0 < n; j0 += kSelThreads) {
    const int j = j0 + tid;
    const uint32_t k = j < n ? key_of(j) : 0u;
    const bool is_above = j < n && k > prefix, is_equal = j < n && k == prefix;
    const uint64_t ma = __ballot(is_above), me = __ballot(is_equal);
    __syncthreads();
    if (lane == 0) {
      above_w[w] = __popcll(ma);
      equal_w[w] = __popcll(me);
    }
    __syncthreads();
    uint32_t ra = above, re = equal;
    for (int i = 0; i < kSelThreads / 64; ++i) {
      if (i < w) {
        ra += above_w[i];
        re += equal_w[i];
      }
      above += above_w[i];
      equal += equal_w[i];
    }
    const uint64_t low = (uint64_t{1} << lane) - 1;
    ra += __popcll(ma & low);
    re += __popcll(me & low);
    if (is_above || (is_equal && re < want)) {
      const uint32_t at = ra + min(re, want);
      sel[at] = j == tid ? first_page : page_of(j);
      if (index) index[at] = j;
    }
  }
}

}  // namespace egmla

using namespace egmla;

namespace {

// The instance of a layer's width for HW waves along the heads and TPW tiles of 16 pages a wave.
template <int HW, int TPW>
hipError_t launch_scores(const eg_mla_dims& d, int32_t batch, const uint16_t* parts, const ScoreArgs& a,
                         hipStream_t stream) {
  constexpr int per = kScoreWaves / HW * TPW * 16;  // pages of a work-group
  const int groups = (a.W + per - 1) / per;
  if (static_cast<int64_t>(batch) * groups > 0x7fffffff) return hipErrorInvalidValue;
  const ScoreMfmaArgs m{parts, static_cast<const uint16_t*>(a.means), a, batch, d.latent_dim, groups};
  auto kern = d.rope_dim != 64        ? page_scores_mfma_kernel<HW, TPW, 0>
              : d.latent_dim == 64    ? page_scores_mfma_kernel<HW, TPW, 2>
              : d.latent_dim == 128   ? page_scores_mfma_kernel<HW, TPW, 4>
              : d.latent_dim == 320   ? page_scores_mfma_kernel<HW, TPW, 10>
              : d.latent_dim == 512   ? page_scores_mfma_kernel<HW, TPW, 16>
                                      : page_scores_mfma_kernel<HW, TPW, 0>;
  hipLaunchKernelGGL(kern, dim3(batch * groups), dim3(kScoreWaves * 64), 0, stream, m);
  return hipGetLastError();
}

}  // namespace

extern "C" eg_mla_status eg_mla_page_means(const eg_mla_dims* dims, int32_t batch, const void* latent_cache,
                                           const int32_t* token_id_cache, const void* gate_table,
                                           const int32_t* first_tokens, const int32_t* seq_lens,
                                           const int32_t* page_table, int32_t max_pages_per_seq, int64_t num_slots,
                                           void* page_means, void* stream_) {
  const eg_mla_status st = validate_page_means(dims, batch, latent_cache, token_id_cache, gate_table, first_tokens,
                                               seq_lens, page_table, max_pages_per_seq, num_slots, page_means);
  if (st != EG_MLA_OK || batch == 0 || max_pages_per_seq == 0) return st;
  const eg_mla_dims& d = *dims;
  MeansArgs a{latent_cache, token_id_cache, gate_table, first_tokens, seq_lens, page_table, page_means, num_slots,
              d.latent_dim, d.rope_dim, d.page_size, max_pages_per_seq, d.vocab_size, max_pages_per_seq * d.page_size};
  hipStream_t stream = static_cast<hipStream_t>(stream_);
  (void)hipGetLastError();
  const dim3 grid(batch, std::min(max_pages_per_seq, std::max(1, kMeanGroups / batch)));
  if (d.dtype == EG_MLA_BF16) hipLaunchKernelGGL(page_means_kernel<true>, grid, dim3(kMeanThreads), 0, stream, a);
  else hipLaunchKernelGGL(page_means_kernel<false>, grid, dim3(kMeanThreads), 0, stream, a);
  return hipGetLastError() == hipSuccess ? EG_MLA_OK : EG_MLA_ERR_HIP;
}

extern "C" size_t eg_mla_page_scores_workspace_size(const eg_mla_dims* dims, int32_t batch) {
  if (check_dims(dims) != EG_MLA_OK || batch < 0) return 0;
  return page_scores_workspace_bytes(*dims, batch);
}

extern "C" eg_mla_status eg_mla_page_scores(const eg_mla_dims* dims, int32_t batch, const void* q, const void* w_uk,
                                            const void* page_means, const int32_t* seq_lens,
                                            const int32_t* page_table, int32_t max_pages_per_seq, int64_t num_slots,
                                            void* workspace, size_t workspace_bytes, float* scores, void* stream_) {
  const eg_mla_status st = validate_page_scores(dims, batch, q, w_uk, page_means, seq_lens, page_table,
                                                max_pages_per_seq, num_slots, workspace, workspace_bytes, scores);
  if (st != EG_MLA_OK || batch == 0 || max_pages_per_seq == 0) return st;
  const eg_mla_dims& d = *dims;
  hipStream_t stream = static_cast<hipStream_t>(stream_);
  (void)hipGetLastError();
  ScoreArgs a{static_cast<const float*>(workspace), page_means, seq_lens, page_table, scores, num_slots, d.num_heads,
              d.latent_dim + d.rope_dim, d.page_size, max_pages_per_seq, max_pages_per_seq * d.page_size,
              softmax_scale(d)};
  if (page_scores_mfma(d)) {
    uint16_t* parts = static_cast<uint16_t*>(workspace);
    if (launch_absorb_parts(d, batch, q, w_uk, parts, stream) != hipSuccess) return EG_MLA_ERR_HIP;
    const int blocks = (d.num_heads + 15) / 16;
    const hipError_t e = blocks == 1 ? launch_scores<1, 1>(d, batch, parts, a, stream)
                         : blocks <= 4 ? launch_scores<4, 1>(d, batch, parts, a, stream)
                                       : launch_scores<8, 2>(d, batch, parts, a, stream);
    return e == hipSuccess ? EG_MLA_OK : EG_MLA_ERR_HIP;
  }
  if (launch_absorb(d, batch, q, w_uk, static_cast<float*>(workspace), stream) != hipSuccess) return EG_MLA_ERR_HIP;
  const dim3 grid(batch, std::min((max_pages_per_seq + 3) / 4, std::max(1, 2048 / batch)));
  if (d.dtype == EG_MLA_BF16) hipLaunchKernelGGL(page_scores_kernel<true>, grid, dim3(256), 0, stream, a);
  else hipLaunchKernelGGL(page_scores_kernel<false>, grid, dim3(256), 0, stream, a);
  return hipGetLastError() == hipSuccess ? EG_MLA_OK : EG_MLA_ERR_HIP;
}

extern "C" eg_mla_status eg_mla_select_pages(const eg_mla_dims* dims, int32_t batch, const float* scores,
                                             const int32_t* seq_lens, const int32_t* page_table,
                                             int32_t max_pages_per_seq, int32_t keep, int32_t keep_first,
                                             int32_t keep_last, int32_t* sel_pages, int32_t* sel_lens,
                                             int32_t* sel_index, void* stream_) {
  const eg_mla_status st = validate_select_pages(dims, batch, scores, seq_lens, page_table, max_pages_per_seq, keep,
                                                 keep_first, keep_last, sel_pages, sel_lens, sel_index);
  if (st != EG_MLA_OK || batch == 0) return st;
  SelectArgs a{scores, seq_lens, page_table, sel_pages, sel_lens, sel_index, max_pages_per_seq, dims->page_size, keep,
               max_pages_per_seq * dims->page_size, keep_first, keep_last};
  (void)hipGetLastError();
  hipLaunchKernelGGL(select_pages_kernel, dim3(batch), dim3(kSelThreads), 0, static_cast<hipStream_t>(stream_), a);
  return hipGetLastError() == hipSuccess ? EG_MLA_OK : EG_MLA_ERR_HIP;
}
