// Tiles of the query absorption: for any shape, and on MFMA (bf16 storage).
#pragma once

#include "absorb.h"
#include "device_common.h"

namespace egmla {

// ---------------------------------------------------------------------------
// Absorption for any shape: qfull[b,h,:] = [W_UK[h]^T q^C[b,h] | q^R[b,h]]   (fp32)
// grid (H, ceil(DC / 64), ceil(B / 16)), 256 threads = 64 latent columns x
// 4 slices of the head dim.  Each W_UK row segment is read once per 16
// sequences with 128-byte coalesced loads; the 4 slices are summed in LDS.
// ---------------------------------------------------------------------------
constexpr int kAbsorbRows = 16;
constexpr int kAbsorbCols = 64;

inline size_t absorb_any_lds(int DH) { return sizeof(float) * (kAbsorbRows * DH + 4 * kAbsorbRows * kAbsorbCols); }

// Tile (h, by, bz) of it, in `smem`: q rows [kAbsorbRows][DH], partial sums [4][kAbsorbRows][kAbsorbCols].  HALF: 16-bit rows
// [q_lat fp16 | q^R bf16] in the fp32 ones' place.
template <bool BF16, bool HALF>
__device__ __forceinline__ void absorb_any_tile(const void* __restrict__ q, const void* __restrict__ w_uk,
                                                float* __restrict__ qfull, int B, int H, int DH, int DC, int DR, int h,
                                                int by, int bz, float* smem) {
  [[maybe_unused]] uint16_t* qhalf = reinterpret_cast<uint16_t*>(qfull);
  float* q_s = smem;
  float* red = smem + kAbsorbRows * DH;
  const int c0 = by * kAbsorbCols;
  const int b0 = bz * kAbsorbRows;
  const int nb = min(kAbsorbRows, B - b0);
  const int DQin = DH + DR;
  const int DQ = DC + DR;
  const int tid = threadIdx.x;
  for (int i = tid; i < kAbsorbRows * DH; i += 256) {
    const int bb = i / DH, k = i % DH;
    q_s[i] = bb < nb ? ld<BF16>(q, (static_cast<int64_t>(b0 + bb) * H + h) * DQin + k) : 0.f;
  }
  __syncthreads();
  const int cl = tid & (kAbsorbCols - 1);
  const int kq = tid / kAbsorbCols;  // 0..3
  const int c = c0 + cl;
  const int kper = (DH + 3) / 4;
  const int k_lo = kq * kper, k_hi = min(DH, k_lo + kper);
  float acc[kAbsorbRows];
#pragma unroll
  for (int bb = 0; bb < kAbsorbRows; ++bb) acc[bb] = 0.f;
  if (c < DC) {
    const int64_t wbase = static_cast<int64_t>(h) * DH * DC + c;
#pragma unroll 4
    for (int k = k_lo; k < k_hi; ++k) {
      const float wv = ld<BF16>(w_uk, wbase + static_cast<int64_t>(k) * DC);
#pragma unroll
      for (int bb = 0; bb < kAbsorbRows; ++bb) acc[bb] = fmaf(wv, q_s[bb * DH + k], acc[bb]);
    }
  }
#pragma unroll
  for (int bb = 0; bb < kAbsorbRows; ++bb) red[(kq * kAbsorbRows + bb) * kAbsorbCols + cl] = acc[bb];
  __syncthreads();
  for (int i = tid; i < kAbsorbRows * kAbsorbCols; i += 256) {
    const int bb = i / kAbsorbCols, cc = i % kAbsorbCols;
    if (bb < nb && c0 + cc < DC) {
      float v = 0.f;
#pragma unroll
      for (int j = 0; j < 4; ++j) v += red[(j * kAbsorbRows + bb) * kAbsorbCols + cc];
      const int64_t at = (static_cast<int64_t>(b0 + bb) * H + h) * DQ + c0 + cc;
      if constexpr (HALF) qhalf[at] = __builtin_bit_cast(uint16_t, static_cast<_Float16>(v));
      else qfull[at] = v;
    }
  }
  if (by == 0) {
    for (int i = tid; i < nb * DR; i += 256) {
      const int bb = i / DR, r = i % DR;
      const int64_t at = (static_cast<int64_t>(b0 + bb) * H + h) * DQ + DC + r;
      const float v = ld<BF16>(q, (static_cast<int64_t>(b0 + bb) * H + h) * DQin + DH + r);
      if constexpr (HALF) qhalf[at] = f32_to_bf16(v);
      else qfull[at] = v;
    }
  }
}

// ---------------------------------------------------------------------------
// Absorption on MFMA: qfull[b, h, c] = sum_k q^C[b, h, k] W_UK[h, k, c] for
// BLOCKS (1..4) blocks of 16 sequences x COLS (32 or 128) latent columns per
// work-group (grid H x ceil(B / (16 blocks)) x ceil(DC/COLS), 256 threads),
// plus the q^R copy.  More blocks per work-group read W_UK fewer times; fewer
// blocks and narrower column slices spread a small batch over more compute
// units.
// W_UK[h][:, c-block] is read once per work-group with 16-byte row loads and
// stored row-major in LDS; the B operand (8 consecutive k of one column) is
// two ds_read_b64_tr_b16, whose 16-lane transpose hands lane n the column n
// of 4 consecutive rows, and serves every sequence block.  The A operands (8
// consecutive k of one query row) come straight from global.  Every load is
// issued before the first use.  bf16 x bf16 products are exact in fp32 and
// accumulate in fp32.
// ---------------------------------------------------------------------------
constexpr int kAbsRows = 16;    // sequences per MFMA row block
constexpr int kAbsBlocks = 4;   // row blocks per work-group, at most
constexpr int kAbsCols = 128;     // latent columns per work-group, at most
constexpr int kAbsColsNarrow = 32;
// Below this many work-groups the absorption takes the narrow column slices.
constexpr int kAbsMinWorkGroups = 128;

// Rows written: fp32 [B, H, DC + DR], or 16-bit [B, H, DC + DR] = [q_lat in
// fp16 (one rounding) | q^R in bf16 (copied)], the operands of fp16 latent
// products and exact bf16 RoPE products, or both; or the page scores' operands
// (three bf16 parts of q_lat, PartsLayout).
enum class AbsorbRows { kFloat, kHalf, kBoth, kParts };

// Tile (h, by, bz) of the absorption: head h, row block by, column slice bz.
template <int DH, int BLOCKS, int COLS, AbsorbRows ROWS_OUT>
__device__ __forceinline__ void absorb_tile(const uint16_t* __restrict__ q, const uint16_t* __restrict__ w_uk,
                                            float* __restrict__ qfull, uint16_t* __restrict__ qhalf, int B, int H,
                                            int DC, int DR, int h, int by, int bz) {
  static_assert(BLOCKS >= 1 && BLOCKS <= kAbsBlocks, "row blocks per work-group");
  constexpr bool PARTS = ROWS_OUT == AbsorbRows::kParts;
  constexpr bool FLOAT = ROWS_OUT == AbsorbRows::kFloat || ROWS_OUT == AbsorbRows::kBoth;
  constexpr bool HALF = ROWS_OUT == AbsorbRows::kHalf || ROWS_OUT == AbsorbRows::kBoth;
  static_assert(COLS % 16 == 0 && COLS <= 128, "latent columns per work-group");
  constexpr int RS = COLS + 8;  // padded LDS row (bf16 elements)
  constexpr int NK = DH / 32;
  __shared__ __attribute__((aligned(16))) uint16_t wrm[DH * RS];  // [k][c], row-major
  constexpr int ROWS = kAbsRows * BLOCKS;  // sequences of this work-group
  const int b0 = by * ROWS;
  const int c0 = bz * COLS;
  const int nc = min(COLS, DC - c0);
  const int tid = threadIdx.x, w = tid >> 6, lane = tid & 63, r16 = lane & 15, g = lane >> 4;
  const int DQin = DH + DR, DQ = DC + DR;

  // (1) issue every load: this thread's W rows (16 B = 8 columns each), its A
  // operand chunks for every row block, and its RoPE query values
  constexpr int kRowsPerPass = 256 / (COLS / 8);  // e.g. 16 rows of 128 columns per pass
  constexpr int kPasses = (DH + kRowsPerPass - 1) / kRowsPerPass;
  const int cc = (tid % (COLS / 8)) * 8;  // first of this thread's 8 columns
  u32x4_t wv[kPasses];
#pragma unroll
  for (int p = 0; p < kPasses; ++p) {
    const int k = p * kRowsPerPass + tid / (COLS / 8);
    const int kk = min(k, DH - 1);
    const int c = min(c0 + cc, DC - 8);
    wv[p] = *reinterpret_cast<const u32x4_t*>(w_uk + (static_cast<int64_t>(h) * DH + kk) * DC + c);
  }
  u32x4_t qa[BLOCKS][NK];
#pragma unroll
  for (int rb = 0; rb < BLOCKS; ++rb) {
    const int bq = min(b0 + rb * kAbsRows + r16, B - 1);
#pragma unroll
    for (int ks = 0; ks < NK; ++ks)
      qa[rb][ks] = *reinterpret_cast<const u32x4_t*>(q + (static_cast<int64_t>(bq) * H + h) * DQin + ks * 32 + g * 8);
  }
  // RoPE part of the query rows (copied as fp32): when d_r is a multiple of 4
  // and at most 64, thread t loads 4 consecutive values of row t / (d_r / 4)
  // of each row block (8-byte loads, rows clamped so the loads are
  // unconditional); other shapes copy element by element after the product.
  const bool rope_vec = bz == 0 && DR > 0 && DR % 4 == 0 && DR <= 64;
  const int rq_row = rope_vec ? tid / (DR / 4) : 0;  // row within a block
  const int rq_col = rope_vec ? 4 * (tid % (DR / 4)) : 0;
  uint2 rq[BLOCKS];
#pragma unroll
  for (int rb = 0; rb < BLOCKS; ++rb) {
    const int rb_b = min(b0 + rb * kAbsRows + min(rq_row, kAbsRows - 1), B - 1);
    rq[rb] = rope_vec ? *reinterpret_cast<const uint2*>(q + (static_cast<int64_t>(rb_b) * H + h) * DQin + DH + rq_col)
                      : make_uint2(0u, 0u);
  }
  // (2) W rows into LDS as loaded (columns past DC hold unused values)
#pragma unroll
  for (int p = 0; p < kPasses; ++p) {
    const int k = p * kRowsPerPass + tid / (COLS / 8);
    if (k < DH) *reinterpret_cast<u32x4_t*>(wrm + k * RS + cc) = wv[p];
  }
  __syncthreads();
  // (3) wave w computes column tiles w, w+4 (16 columns each) of every row
  // block.  For rows k0 .. k0 + 3 of the tile, lane r16 of group g reads
  // columns 4 (r16 % 4) .. + 3 of row k0 + r16 / 4; the transposed read hands
  // lane r16 column r16 of the 4 rows.
  for (int nt = w; nt * 16 < nc; nt += 4) {
    f32x4_t acc[BLOCKS];
#pragma unroll
    for (int rb = 0; rb < BLOCKS; ++rb) acc[rb] = f32x4_t{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int ks = 0; ks < NK; ++ks) {
      uint16_t* t0 = wrm + (ks * 32 + 8 * g + (r16 >> 2)) * RS + nt * 16 + 4 * (r16 & 3);
      const s16x4_t lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s16x4_t*)t0);
      const s16x4_t hi =
          __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s16x4_t*)(t0 + 4 * RS));
      const u32x2_t l2 = __builtin_bit_cast(u32x2_t, lo), h2 = __builtin_bit_cast(u32x2_t, hi);
      const bf16x8_t bv = __builtin_bit_cast(bf16x8_t, u32x4_t{l2[0], l2[1], h2[0], h2[1]});
#pragma unroll
      for (int rb = 0; rb < BLOCKS; ++rb)
        acc[rb] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(bv, __builtin_bit_cast(bf16x8_t, qa[rb][ks]), acc[rb], 0, 0, 0);
    }
    // lane holds D[c = nt*16 + 4g + r][b = r16] of each row block: 4 columns of a row, stored together (d_c is a
    // multiple of 8)
    const int c = c0 + nt * 16 + 4 * g;
    if (c >= DC) continue;
#pragma unroll
    for (int rb = 0; rb < BLOCKS; ++rb) {
      const int b = b0 + rb * kAbsRows + r16;
      if (b >= B) continue;
      const f32x4_t x = acc[rb];
      const int64_t at = (static_cast<int64_t>(b) * H + h) * DQ + c;
      if constexpr (HALF) {
        typedef __attribute__((ext_vector_type(4))) _Float16 f16x4_t;
        *reinterpret_cast<f16x4_t*>(qhalf + at) = __builtin_convertvector(x, f16x4_t);
      }
      if constexpr (PARTS) {
        const PartsLayout layout(H, DC, DR);
        uint16_t p[3][4];
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          // an infinity has no rest (infinity - infinity), and a finite value past bf16's largest keeps its upper bits
          const bool inf = fabsf(x[r]) == INFINITY;
          p[0][r] = f32_to_bf16(x[r]);
          if (!inf && fabsf(bf16_to_f32(p[0][r])) == INFINITY) p[0][r] = static_cast<uint16_t>(__float_as_uint(x[r]) >> 16);
          const float left = inf ? 0.f : x[r] - bf16_to_f32(p[0][r]);  // exact
          p[1][r] = f32_to_bf16(left);
          p[2][r] = f32_to_bf16(left - bf16_to_f32(p[1][r]));
        }
#pragma unroll
        for (int i = 0; i < 3; ++i)
          *reinterpret_cast<uint2*>(qhalf + layout(b, h, i, c)) =
              make_uint2(p[i][0] | static_cast<uint32_t>(p[i][1]) << 16, p[i][2] | static_cast<uint32_t>(p[i][3]) << 16);
      }
      if constexpr (FLOAT) *reinterpret_cast<f32x4_t*>(qfull + at) = x;
    }
  }
  if (rope_vec) {
#pragma unroll
    for (int rb = 0; rb < BLOCKS; ++rb) {
      const int b = b0 + rb * kAbsRows + rq_row;
      if (rq_row < kAbsRows && b < B) {
        if constexpr (PARTS) *reinterpret_cast<uint2*>(qhalf + PartsLayout(H, DC, DR)(b, h, 0, DC + rq_col)) = rq[rb];
        if constexpr (HALF)
          *reinterpret_cast<uint2*>(qhalf + (static_cast<int64_t>(b) * H + h) * DQ + DC + rq_col) = rq[rb];
        if constexpr (FLOAT)
          *reinterpret_cast<float4*>(qfull + (static_cast<int64_t>(b) * H + h) * DQ + DC + rq_col) =
              make_float4(bf16_lo(rq[rb].x), bf16_hi(rq[rb].x), bf16_lo(rq[rb].y), bf16_hi(rq[rb].y));
      }
    }
  } else if (bz == 0) {
    for (int i = tid; i < ROWS * DR; i += 256) {
      const int bb = i / DR, r = i % DR;
      if (b0 + bb < B) {
        const uint16_t v = q[(static_cast<int64_t>(b0 + bb) * H + h) * DQin + DH + r];
        if constexpr (PARTS) qhalf[PartsLayout(H, DC, DR)(b0 + bb, h, 0, DC + r)] = v;
        if constexpr (HALF) qhalf[(static_cast<int64_t>(b0 + bb) * H + h) * DQ + DC + r] = v;
        if constexpr (FLOAT)
          qfull[(static_cast<int64_t>(b0 + bb) * H + h) * DQ + DC + r] = bf16_to_f32(v);
      }
    }
  }
}

}  // namespace egmla
