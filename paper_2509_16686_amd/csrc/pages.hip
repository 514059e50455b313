// Page tables, slots and positions of a step from the request lengths, and the
// return of ended requests' pages to the free stack (gfx950).
//
//   n_b    = new tokens of sequence b, c_b its cached ones (clamped to the capacity)
//   need_b = ceil((c_b + n_b) / P) - ceil(c_b / P), or 0 where c_b + n_b outgrows the table's row
//   N_b, K_b = sums of n and need over the sequences up to b
//   page k of b's new ones = free_pages[count - 1 - (K_{b-1} + k)]
//
// Every work-group forms both sums for the whole batch (a scan over at most
// kPageMaxBatch lengths, L2 hits but for the first) and then takes its share of
// the new table entries and of the tokens; a token finds its sequence by
// bisection of N in LDS.  One launch and no exchange between work-groups: the
// call is latency-bound (three dependent loads), so a second launch would cost
// more than the repeated scan.
#include <hip/hip_runtime.h>

#include <algorithm>

#include "device_common.h"
#include "eg_mla.h"
#include "host_plan.h"

namespace egmla {

constexpr int kPageThreads = 256;
// Tokens (or pages) of a work-group: one a thread, whose chain of loads is the
// time (51457 tokens of 256 sequences: 11.0 us with four a thread).
constexpr int kPageTokens = kPageThreads;
constexpr int kPageMaxGroups = 1024;

// Sum of two counts in [0, 2^31 - 1], held at 2^31 - 1 (associative, so sums of any order agree).
__device__ __forceinline__ int32_t add_held(int32_t a, int32_t b) {
  const uint32_t s = static_cast<uint32_t>(a) + static_cast<uint32_t>(b);
  return static_cast<int32_t>(min(s, 0x7fffffffu));
}

// Two counts of each thread become their sums over the work-group's threads before it; `red` holds 8 words.
__device__ __forceinline__ void sums_before(int32_t& a, int32_t& b, int32_t* red) {
  const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) {
    const int32_t ua = __shfl_up(a, o, 64), ub = __shfl_up(b, o, 64);
    if (lane >= o) {
      a = add_held(a, ua);
      b = add_held(b, ub);
    }
  }
  if (lane == 63) {
    red[w] = a;
    red[4 + w] = b;
  }
  a = __shfl_up(a, 1, 64);
  b = __shfl_up(b, 1, 64);
  if (lane == 0) a = b = 0;
  __syncthreads();
#pragma unroll
  for (int i = 0; i < kPageThreads / 64 - 1; ++i)
    if (i < w) {
      a = add_held(a, red[i]);
      b = add_held(b, red[4 + i]);
    }
}

// The first b with sum[b] > k (k below the last sum).
__device__ __forceinline__ int find_seq(const int32_t* sum, int B, int32_t k) {
  int lo = 0, hi = B - 1;
  while (lo < hi) {
    const int mid = (lo + hi) >> 1;
    if (sum[mid] > k) hi = mid;
    else lo = mid + 1;
  }
  return lo;
}

struct PagePlanArgs {
  const int32_t* cached;
  const int32_t* fresh;
  const int32_t* base;  // or null
  int32_t* table;
  const int32_t* free_pages;
  const int32_t* free_count;
  int32_t* lens;
  int32_t* cu;
  int32_t* positions;
  int32_t* slots;
  int32_t* count_out;
  int32_t B, P, W, max_tokens, free_cap, cap;
};

__global__ __launch_bounds__(kPageThreads) void page_plan_kernel(PagePlanArgs a) {
  extern __shared__ int32_t page_lds[];  // sums of new tokens [B], of needed pages [B], scratch [8], taken [1]
  int32_t* n_sum = page_lds;
  int32_t* k_sum = page_lds + a.B;
  int32_t* red = page_lds + 2 * a.B;
  int32_t* taken_s = red + 8;
  const int tid = threadIdx.x;
  const int32_t count = clamp_len(a.free_count[0], a.free_cap);
  if (tid == 0) *taken_s = 0;

  // sums over runs of `per` sequences per thread, then over the threads
  const int per = (a.B + kPageThreads - 1) / kPageThreads;
  const int b0 = min(tid * per, a.B), b1 = min(b0 + per, a.B);
  auto pages = [&](int64_t tokens) { return static_cast<int32_t>((tokens + a.P - 1) / a.P); };
  int32_t n_all = 0, k_all = 0;
  for (int b = b0; b < b1; ++b) {
    const int32_t c = clamp_len(a.cached[b], a.cap), n = max(a.fresh[b], 0);
    const int64_t total = static_cast<int64_t>(c) + n;
    n_all = add_held(n_all, n);
    k_all = add_held(k_all, total <= a.cap ? pages(total) - pages(c) : 0);
    n_sum[b] = n_all;
    k_sum[b] = k_all;
  }
  sums_before(n_all, k_all, red);
  for (int b = b0; b < b1; ++b) {
    n_sum[b] = add_held(n_sum[b], n_all);
    k_sum[b] = add_held(k_sum[b], k_all);
  }
  __syncthreads();

  // whether a sequence's tokens are taken in: the row, the token arrays and the free pages have room
  auto served = [&](int b, int32_t c, int32_t n, int32_t need) {
    return static_cast<int64_t>(c) + n <= a.cap && n_sum[b] <= a.max_tokens && (need == 0 || k_sum[b] <= count);
  };
  auto before = [](const int32_t* sum, int b) { return b ? sum[b - 1] : 0; };
  for (int b = tid; b < a.B; b += kPageThreads) {
    const int32_t c = clamp_len(a.cached[b], a.cap), n = max(a.fresh[b], 0), need = k_sum[b] - before(k_sum, b);
    const bool ok = served(b, c, n, need);
    if (ok && need > 0) atomicMax(taken_s, k_sum[b]);
    if (blockIdx.x == 0) {
      a.lens[b] = ok ? c + n : c;
      a.cu[b + 1] = min(n_sum[b], a.max_tokens);
    }
  }
  __syncthreads();
  const int32_t taken = *taken_s;
  if (blockIdx.x == 0 && tid == 0) {
    a.cu[0] = 0;
    a.count_out[0] = count - taken;
  }
  // new entries of the table
  const int stride = gridDim.x * kPageThreads;
  for (int k = blockIdx.x * kPageThreads + tid; k < taken; k += stride) {
    const int b = find_seq(k_sum, a.B, k);
    const int32_t have = pages(clamp_len(a.cached[b], a.cap));
    a.table[static_cast<int64_t>(b) * a.W + have + (k - before(k_sum, b))] = a.free_pages[count - 1 - k];
  }
  // positions and slots
  const int32_t total = min(n_sum[a.B - 1], a.max_tokens);
  const int32_t max_page = 0x7fffffff / a.P;  // pages below it have slots that fit 32 bits
  for (int i = blockIdx.x * kPageThreads + tid; i < a.max_tokens; i += stride) {
    int32_t pos = 0, slot = -1;
    if (i < total) {
      const int b = find_seq(n_sum, a.B, i);
      const int32_t c = clamp_len(a.cached[b], a.cap), n = max(a.fresh[b], 0);
      const int32_t kb = before(k_sum, b), need = k_sum[b] - kb;
      const int32_t at = c + (i - before(n_sum, b));
      pos = static_cast<int32_t>(static_cast<uint32_t>(a.base ? a.base[b] : 0) + static_cast<uint32_t>(at));
      if (served(b, c, n, need)) {
        const int32_t pg = at / a.P, have = pages(c);
        const int32_t page = pg < have ? a.table[static_cast<int64_t>(b) * a.W + pg]
                                       : a.free_pages[count - 1 - (kb + pg - have)];
        if (page >= 0 && page < max_page) slot = page * a.P + at % a.P;
      }
    }
    a.positions[i] = pos;
    a.slots[i] = slot;
  }
}

struct PageReleaseArgs {
  const int32_t* lens;
  const int32_t* ended;
  const int32_t* table;
  int32_t* free_pages;
  const int32_t* free_count;
  int32_t* lens_out;
  int32_t* count_out;
  int32_t B, P, W, free_cap, cap;
};

__global__ __launch_bounds__(kPageThreads) void page_release_kernel(PageReleaseArgs a) {
  extern __shared__ int32_t page_lds[];  // sums of returned pages [B], scratch [8]
  int32_t* k_sum = page_lds;
  int32_t* red = page_lds + a.B;
  const int tid = threadIdx.x;
  const int32_t count = clamp_len(a.free_count[0], a.free_cap);
  const int per = (a.B + kPageThreads - 1) / kPageThreads;
  const int b0 = min(tid * per, a.B), b1 = min(b0 + per, a.B);
  int32_t k_all = 0;
  for (int b = b0; b < b1; ++b) {
    const int32_t len = a.lens[b], gone = a.ended[b];
    if (gone) k_all = add_held(k_all, static_cast<int32_t>((static_cast<int64_t>(clamp_len(len, a.cap)) + a.P - 1) / a.P));
    k_sum[b] = k_all;
    if (blockIdx.x == 0) a.lens_out[b] = gone ? 0 : len;
  }
  int32_t unused = 0;
  sums_before(k_all, unused, red);
  for (int b = b0; b < b1; ++b) k_sum[b] = add_held(k_sum[b], k_all);
  __syncthreads();
  const int32_t back = min(k_sum[a.B - 1], a.free_cap - count);
  if (blockIdx.x == 0 && tid == 0) a.count_out[0] = count + back;
  for (int k = blockIdx.x * kPageThreads + tid; k < back; k += gridDim.x * kPageThreads) {
    const int b = find_seq(k_sum, a.B, k);
    a.free_pages[count + k] = a.table[static_cast<int64_t>(b) * a.W + (k - (b ? k_sum[b - 1] : 0))];
  }
}

}  // namespace egmla

using namespace egmla;

namespace {
int page_groups(int64_t items) {
  return static_cast<int>(std::min<int64_t>(std::max<int64_t>((items + kPageTokens - 1) / kPageTokens, 1), kPageMaxGroups));
}
}  // namespace

extern "C" eg_mla_status eg_mla_page_plan(int32_t batch, int32_t page_size, int32_t max_pages_per_seq,
                                          int32_t max_tokens, const int32_t* cached_lens, const int32_t* new_lens,
                                          const int32_t* position_base, int32_t* page_table,
                                          const int32_t* free_pages, const int32_t* free_count,
                                          int32_t free_capacity, int32_t* seq_lens, int32_t* cu_seqlens,
                                          int32_t* positions, int32_t* slots, int32_t* free_count_out, void* stream) {
  const eg_mla_status st = validate_page_plan(batch, page_size, max_pages_per_seq, max_tokens, cached_lens, new_lens,
                                              position_base, page_table, free_pages, free_count, free_capacity,
                                              seq_lens, cu_seqlens, positions, slots, free_count_out);
  if (st != EG_MLA_OK || batch == 0) return st;
  (void)hipGetLastError();
  PagePlanArgs a{cached_lens, new_lens, position_base, page_table, free_pages, free_count, seq_lens, cu_seqlens,
                 positions, slots, free_count_out, batch, page_size, max_pages_per_seq, max_tokens, free_capacity,
                 max_pages_per_seq * page_size};
  hipLaunchKernelGGL(page_plan_kernel, dim3(page_groups(max_tokens)), dim3(kPageThreads),
                     sizeof(int32_t) * (2 * static_cast<size_t>(batch) + 9), static_cast<hipStream_t>(stream), a);
  return hipGetLastError() == hipSuccess ? EG_MLA_OK : EG_MLA_ERR_HIP;
}

extern "C" eg_mla_status eg_mla_page_release(int32_t batch, int32_t page_size, int32_t max_pages_per_seq,
                                             const int32_t* seq_lens, const int32_t* ended,
                                             const int32_t* page_table, int32_t* free_pages,
                                             const int32_t* free_count, int32_t free_capacity, int32_t* seq_lens_out,
                                             int32_t* free_count_out, void* stream) {
  const eg_mla_status st = validate_page_release(batch, page_size, max_pages_per_seq, seq_lens, ended, page_table,
                                                 free_pages, free_count, free_capacity, seq_lens_out, free_count_out);
  if (st != EG_MLA_OK || batch == 0) return st;
  (void)hipGetLastError();
  PageReleaseArgs a{seq_lens, ended, page_table, free_pages, free_count, seq_lens_out, free_count_out, batch,
                    page_size, max_pages_per_seq, free_capacity, max_pages_per_seq * page_size};
  // at most every sequence's whole row comes back, and no more than the stack holds
  const int64_t most = std::min<int64_t>(static_cast<int64_t>(batch) * max_pages_per_seq, free_capacity);
  hipLaunchKernelGGL(page_release_kernel, dim3(page_groups(most)), dim3(kPageThreads),
                     sizeof(int32_t) * (static_cast<size_t>(batch) + 8), static_cast<hipStream_t>(stream), a);
  return hipGetLastError() == hipSuccess ? EG_MLA_OK : EG_MLA_ERR_HIP;
}
