// Attention of many query rows over one prefix on gfx950 MFMA (bf16 storage,
// heads a multiple of 16, d_h = d_v = 128, d_r = 64, d_c 128, 320 or 512): the
// prefix part of the shared decode.  Included by decode.hip.
//
// With all heads on one latent, the B H query rows of a batch attend to the
// same keys [c~ | k^R] and values c~: a flash attention with d_c + d_r wide
// keys and d_c wide values, bound by the matrix cores once a few hundred rows
// share a key.  Three launches:
//  1. shared_prep_kernel: the query absorption (16-bit rows [q_lat fp16 | q^R
//     bf16], and fp32 ones where the own tokens' kernel wants them), the own
//     tokens' schedule, and, once per prefix token, the gated latent (the exact
//     fp32 product rounded to fp16) and the RoPE key (bf16), written as tiles of
//     64 or 32 keys that are byte for byte what the attention holds in LDS: page
//     table, gate and bank swizzle are dealt with once, and a tile is copied
//     as one run of memory.
//  2. shared_prefix_kernel: a work-group of 4 waves takes 128 query rows (32
//     per wave, in registers) and a run of tiles.
//  3. shared_merge_kernel (after the own tokens' split kernel): joins both
//     parts' partial rows and applies W_UV.
//
// Attention kernel.  Tiles go straight from global memory into the other of
// two LDS buffers while the current one is computed.  Scores
// S^T[key][row] on v_mfma_f32_32x32x16 (A: 32 keys from LDS, B: the wave's 32
// rows), online softmax per row in the log2 domain with lazy rescale, values
// O^T[dim][row] += C~^T P^T with the probabilities as the B operand as they
// lie in the score accumulators and transposed LDS reads as the A operand.
// Each LDS byte read feeds 32 rows.  A partial row is as the layer's decode has
// it: the fp32 sums O with their maximum and sum l, or, for the layers of the
// head-split kernel (d_c 512, heads a multiple of 64), O / l in fp16, a convex
// combination of fp16 values.
#pragma once

#include "rows32.h"

namespace egmla {

template <int DC, int KEYS_>
struct PrefixCfg {
  static constexpr int KEYS = KEYS_;                   // of a tile
  static constexpr int LROW = prefix_latent_row(DC);   // bytes per key: gated latent, padded to whole 256 bytes
  static constexpr int RROW = 128;                     // RoPE key
  static constexpr int ROPE = KEYS * LROW;             // its rows lie behind the latent rows
  static constexpr int TILE = KEYS * (LROW + RROW);
  static_assert(DC % 32 == 0 && TILE % 4096 == 0 && 2 * TILE <= 160 * 1024, "two tile buffers, copied by 4 waves");
};
constexpr int kPrefixThreads = 256;
constexpr int kPrefixRsrcWord3 = 0x00020000;  // raw buffer resource: 32-bit data format, the record count in bytes
static_assert(kPrefixRows == 32 * kPrefixThreads / 64, "32 rows per wave");

constexpr int kPrepTokens = 16;    // tokens that a work-group gates at a time
constexpr int kPrepGroups = 2048;  // work-groups that gate, at most
constexpr int kPrepBatch = 5;      // pieces of a thread in flight (d_c 512: 72 a token)

struct PrefixPrepArgs {
  const uint16_t* q;
  const uint16_t* w_uk;
  float* qfull;      // fp32 rows, where written
  uint16_t* qhalf;   // 16-bit rows
  const uint16_t* cache;
  const int32_t* ids;
  const uint16_t* gate;
  const int32_t* len;
  const int32_t* table;
  unsigned char* tiles;
  int64_t num_slots;
  WideSchedArgs sched;  // G = 0: none
  int2* split_rows;     // null: none; else each sequence's partial rows, one per split
  int32_t B, H, DC, V, P, cap;
  int32_t absorb_wgs, gate_wgs, row_blocks, keys, splits;
};

template <AbsorbRows ROWS_OUT, int BLOCKS, int COLS>
__global__ __launch_bounds__(256) void shared_prep_kernel(PrefixPrepArgs a) {
  constexpr int DR = 64;
  int wg = blockIdx.x;
  if (wg == 0) {
    if (a.sched.G > 0) wide_schedule<256>(a.sched, a.B);
    if (a.split_rows)
      for (int b = threadIdx.x; b < a.B; b += 256) a.split_rows[b] = make_int2(b * a.splits, a.splits);
    return;
  }
  wg -= 1;
  if (wg < a.absorb_wgs) {
    const int h = wg % a.H, by = (wg / a.H) % a.row_blocks, bz = wg / (a.H * a.row_blocks);
    absorb_tile<128, BLOCKS, COLS, ROWS_OUT>(a.q, a.w_uk, a.qfull, a.qhalf, a.B, a.H, a.DC, DR, h, by, bz);
    return;
  }
  wg -= a.absorb_wgs;
  // pieces of the prefix's tokens, kPrepTokens tokens at a time; those behind the last token, up to the end of its
  // tile, are zero
  const int keys = a.keys;
  const int L = clamp_len(a.len[0], a.cap), end = (L + keys - 1) / keys * keys;
  const int np = a.DC / 8 + DR / 8, lat = a.DC / 8;
  const int lrow = prefix_latent_row(a.DC), tile_bytes = keys * (lrow + 128);
  __shared__ int2 tok_s[kPrepTokens];  // (cache row, id); row -1: behind the last token
  for (int base = wg * kPrepTokens; base < end; base += a.gate_wgs * kPrepTokens) {
    if (threadIdx.x < kPrepTokens) {
      const int t = base + static_cast<int>(threadIdx.x);
      int2 e = make_int2(-1, 0);
      if (t < L) {
        e.x = static_cast<int>(paged_slot(a.table[t / a.P], t, a.P, a.num_slots));
        e.y = clamp_id(a.ids[e.x], a.V);
      }
      tok_s[threadIdx.x] = e;
    }
    __syncthreads();
    for (int i0 = threadIdx.x; i0 < kPrepTokens * np; i0 += 256 * kPrepBatch) {
      u32x4_t v[kPrepBatch], gv[kPrepBatch];
#pragma unroll
      for (int u = 0; u < kPrepBatch; ++u) {
        const int i = i0 + 256 * u, k = min(i / np, kPrepTokens - 1), p = i % np;
        const int2 e = tok_s[k];
        v[u] = gv[u] = u32x4_t{0u, 0u, 0u, 0u};
        if (i < kPrepTokens * np && e.x >= 0) {
          v[u] = *reinterpret_cast<const u32x4_t*>(a.cache + static_cast<int64_t>(e.x) * (a.DC + DR) + 8 * p);
          if (p < lat) gv[u] = *reinterpret_cast<const u32x4_t*>(a.gate + static_cast<int64_t>(e.y) * a.DC + 8 * p);
        }
      }
#pragma unroll
      for (int u = 0; u < kPrepBatch; ++u) {
        const int i = i0 + 256 * u, k = i / np, p = i % np, t = base + k, key = t % keys;
        if (i >= kPrepTokens * np) continue;
        unsigned char* dst = a.tiles + static_cast<int64_t>(t / keys) * tile_bytes +
                             (p < lat ? key * lrow + prefix_latent_byte(key, p)
                                      : keys * lrow + key * 128 + prefix_rope_byte(key, p - lat));
        *reinterpret_cast<u32x4_t*>(dst) = p < lat ? gate_chunk_f16(v[u], gv[u]) : v[u];
      }
    }
    __syncthreads();  // the list has been read
  }
}

// Tiles per split of a prefix of L tokens cut into at most s_max splits, and the splits that have any.
__device__ __forceinline__ int prefix_per_split(int L, int s_max, int keys) {
  const int tiles = (L + keys - 1) / keys;
  return (tiles + s_max - 1) / s_max;
}
__device__ __forceinline__ int prefix_splits(int L, int s_max, int keys) {
  const int tiles = (L + keys - 1) / keys, per = prefix_per_split(L, s_max, keys);
  return per ? (tiles + per - 1) / per : 0;
}

struct PrefixArgs {
  const uint16_t* qhalf;       // [rows][DC + 64]: q_lat fp16 | q^R bf16
  const unsigned char* tiles;  // PrefixCfg<DC>::TILE bytes each
  const int32_t* len;
  float* part_ml;              // [s_max][rows][2]; OWN: [B][s_max][H][2]
  void* part_o;                // [s_max][rows][DC] fp32: O, or (HALF) fp16: O / l; OWN: [B][s_max][H][DC]
  int32_t cap, rows, row_blocks, s_max;
  float scale_log2;
  // OWN: each sequence's own tokens
  const uint16_t* cache;       // [num_slots][DC + 64]
  const int32_t* ids;
  const uint16_t* gate;        // [V][DC]
  const int32_t* own_lens;     // null: none
  const int32_t* own_table;    // or null
  int64_t num_slots;
  int32_t own_cap, own_pages, blocks_per_seq, P, V;
};

// OWN (heads a multiple of 128, so that a row block lies within a sequence): after its run of the prefix a work-group
// takes its share of the sequence's own tokens into the same accumulators.  Their raw rows and gate rows are copied to
// LDS a tile ahead and gated in place there (prefix 8000 x 64 x 128 heads with up to 1500 own tokens: a wave's whole rows
// at a time 208.5 -> 204.5 us a call; raw rows in a buffer of their own, with a barrier more and every piece's address
// formed twice, 209.0, in place 208.1 in the same run).
constexpr int kOwnList = 512;  // own tokens listed at a time

// Work-group `bid` of `nblocks`.  HALF: the form of the partial rows.
template <int DC, int KEYS, bool OWN, bool HALF>
__device__ __forceinline__ void prefix_item(const PrefixArgs& a, int bid, int nblocks) {
#if defined(__HIP_DEVICE_COMPILE__)  // the host pass knows neither the copies to LDS nor the register constraints
  using C = PrefixCfg<DC, KEYS>;
  constexpr int DQ = DC + 64, NC = DC / 16, NR = 4, KB = C::KEYS / 32, NDB = DC / 32;
  // How far the LDS reads run ahead of the products: with two waves per SIMD (d_c 128) the other wave covers their
  // latency, with one (d_c 512: 161 us, prefix 8000 x 64 x 128 heads) they have to (184 one chunk ahead and the values
  // in the compiler's order; 175 six or eight value products ahead).
  constexpr int QA = DC == 512 ? 3 : 1, PA = DC == 128 ? 0 : 4;
  __shared__ __attribute__((aligned(16))) unsigned char lds0[C::TILE];  // two tile buffers
  __shared__ __attribute__((aligned(16))) unsigned char lds1[C::TILE];
  // consecutive items (the row blocks of a split) share an XCD, whose L2 then serves the split's tiles
  const int item = xcd_logical_block(bid, nblocks);
  const int rb = item % a.row_blocks, split = item / a.row_blocks;
  const int L = a.len ? clamp_len(a.len[0], a.cap) : 0;
  const int per = prefix_per_split(L, a.s_max, C::KEYS);
  const int t0 = split * per, t1 = min(t0 + per, (L + C::KEYS - 1) / C::KEYS);
  if (!OWN && t0 >= t1) return;

  const int tid = threadIdx.x, lane = tid & 63, r32 = lane & 31, h = lane >> 5;
  const int w = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int r16 = lane & 15, R1 = (lane >> 4) & 1;
  // this lane's query row; rows past the last repeat it and are not stored
  const int row = rb * kPrefixRows + 32 * w + r32;
  const int64_t qrow = static_cast<int64_t>(min(row, a.rows - 1)) * DQ + 8 * h;
  // d_c 512: q^R and the first QL chunks of q_lat wait in LDS, each lane's own operands (registers are scarce: with them
  // in registers the value operands could not run ahead, and what the compiler spilled it read back in the tile loop,
  // waiting for the tile copies too: prefix 8000 x 64 x 128 heads with own tokens 198 to 272 us, 163 so)
  constexpr int QL = DC == 512 ? 4 : 0;
  constexpr bool QLDS = QL > 0;
  __shared__ __attribute__((aligned(16))) u32x4_t q_s[QLDS ? (NR + QL) * kPrefixThreads : 1];
  f16x8_t qv[NC];   // q_lat
  bf16x8_t qr[NR];  // q^R
#pragma unroll
  for (int c = 0; c < NC; ++c) qv[c] = *reinterpret_cast<const f16x8_t*>(a.qhalf + qrow + 16 * c);
#pragma unroll
  for (int c = 0; c < NR; ++c) qr[c] = *reinterpret_cast<const bf16x8_t*>(a.qhalf + qrow + DC + 16 * c);
  if constexpr (QLDS) {
#pragma unroll
    for (int c = 0; c < NR; ++c) q_s[c * kPrefixThreads + tid] = __builtin_bit_cast(u32x4_t, qr[c]);
#pragma unroll
    for (int c = 0; c < QL; ++c) q_s[(NR + c) * kPrefixThreads + tid] = __builtin_bit_cast(u32x4_t, qv[c]);
  }

  auto lds_ptr = [](unsigned char* p) { return (__attribute__((address_space(3))) void*)p; };
  auto issue_tile = [&](int tile, unsigned char* base) {
    const __amdgpu_buffer_rsrc_t rs = __builtin_amdgcn_make_buffer_rsrc(
        const_cast<unsigned char*>(a.tiles) + static_cast<int64_t>(tile) * C::TILE, 0, C::TILE, kPrefixRsrcWord3);
#pragma unroll
    for (int j = 0; j < C::TILE / 4096; ++j) {
      const int at = 1024 * (C::TILE / 4096 * w + j);
      __builtin_amdgcn_raw_ptr_buffer_load_lds(rs, lds_ptr(base + at), 16, 16 * lane, at, 0, 0);
    }
  };
  // this wave's copies have landed; the barrier after it covers every wave's
  auto tile_landed = []() { asm volatile("s_waitcnt vmcnt(0)" ::: "memory"); };

  // per-lane LDS offsets (bytes within a tile buffer): score operands (key row r32 of a block of 32) ...
  const int swz_l = ((r32 & 3) << 2) | ((r32 >> 2) & 3), swz_r = (r32 >> 1) & 7;
  const int off_l = r32 * C::LROW, off_r = C::ROPE + r32 * C::RROW;
  // ... and value operands (transposed reads): rows 16 m + 4 h + r16 / 4 (+ 8); operand row 16 R1 + 4 j + e is
  // dim 16 R1 + 8 (j % 2) + 4 (j / 2) + e of a block of 32, so that an accumulator lane's outputs are adjacent dims
  const int off_v = (4 * h + (r16 >> 2)) * C::LROW + 8 * ((r16 & 3) >> 1);
  const int vlo = 2 * R1 + (r16 & 1);  // low 2 bits of the logical piece

  px_f32x16_t o[NDB];
#pragma unroll
  for (int db = 0; db < NDB; ++db)
#pragma unroll
    for (int r = 0; r < 16; ++r) o[db][r] = 0.f;
  float m_run = -1e30f, l_run = 0.f;
  // With d_c / 2 values a lane, the accumulators and the query fill the register file: the accumulators stay in the
  // accumulation registers on every path (left to itself the compiler moves them through ordinary ones around the
  // rescale, at each tile, and spills: 875 registers of d_c 512)
  constexpr bool ACC = DC > 128;
  auto hold = [&]() {
    if constexpr (ACC) {
#pragma unroll
      for (int db = 0; db < NDB; ++db) in_agprs(o[db]);
    }
  };

  // attends to the `valid` first keys of the tile in `tb`
  auto attend = [&](const unsigned char* tb, int valid) __attribute__((always_inline)) {
    hold();
    px_f32x16_t s[KB];
#pragma unroll
    for (int kb = 0; kb < KB; ++kb)
#pragma unroll
      for (int r = 0; r < 16; ++r) s[kb][r] = 0.f;
    if constexpr (QLDS) {
#pragma unroll
      for (int c = 0; c < NR; ++c) qr[c] = __builtin_bit_cast(bf16x8_t, q_s[c * kPrefixThreads + tid]);
#pragma unroll
      for (int c = 0; c < QL; ++c) qv[c] = __builtin_bit_cast(f16x8_t, q_s[(NR + c) * kPrefixThreads + tid]);
    }
#pragma unroll
    for (int c = 0; c < NR; ++c)
#pragma unroll
      for (int kb = 0; kb < KB; ++kb) {
        const bf16x8_t av =
            *reinterpret_cast<const bf16x8_t*>(tb + off_r + 32 * kb * C::RROW + 16 * ((2 * c + h) ^ swz_r));
        s[kb] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(av, qr[c], s[kb], 0, 0, 0);
      }
#pragma unroll
    for (int c = 0; c < NC; ++c)
#pragma unroll
      for (int kb = 0; kb < KB; ++kb) {
        const f16x8_t av = *reinterpret_cast<const f16x8_t*>(tb + off_l + 32 * kb * C::LROW + 256 * (c >> 3) +
                                                             16 * ((2 * (c & 7) + h) ^ swz_l));
        s[kb] = __builtin_amdgcn_mfma_f32_32x32x16_f16(av, qv[c], s[kb], 0, 0, 0);
      }
    // issue order: the A operands QA chunks ahead of their products
    __builtin_amdgcn_sched_group_barrier(0x100, (QA + 1) * KB + (QLDS ? NR + QL : 0), 0);
#pragma unroll
    for (int c = 0; c < NC + NR - QA; ++c) {
      __builtin_amdgcn_sched_group_barrier(0x008, KB, 0);
      __builtin_amdgcn_sched_group_barrier(0x100, KB, 0);
    }
    __builtin_amdgcn_sched_group_barrier(0x008, QA * KB, 0);
    if (valid < C::KEYS) {  // the tokens end inside this tile
#pragma unroll
      for (int kb = 0; kb < KB; ++kb)
#pragma unroll
        for (int r = 0; r < 16; ++r)
          if (32 * kb + 8 * (r >> 2) + 4 * h + (r & 3) >= valid) s[kb][r] = -INFINITY;
    }

    // online softmax (row = lane % 32; keys split between lanes l and l ^ 32); the scale (tau log2 e > 0) commutes with
    // the maximum and is applied inside the exponent
    float mt = s[0][0];
#pragma unroll
    for (int kb = 0; kb < KB; ++kb)
#pragma unroll
      for (int r = 0; r < 16; ++r) mt = fmaxf(mt, s[kb][r]);
    mt = half_max(mt) * a.scale_log2;
    const float m_new = fmaxf(m_run, mt);
    const bool grow = m_new > m_run + kLazyRescale;
    const float alpha = grow ? __builtin_amdgcn_exp2f(m_run - m_new) : 1.0f;
    m_run = grow ? m_new : m_run;
    l_run *= alpha;
    if (__builtin_amdgcn_ballot_w64(grow)) {
#pragma unroll
      for (int db = 0; db < NDB; ++db) {
        if constexpr (ACC) {  // one block at a time through ordinary registers
          px_f32x16_t f = o[db];
          in_vgprs(f);
          f *= alpha;
          in_agprs(f);
          o[db] = f;
          __builtin_amdgcn_sched_barrier(0);
        } else {
          o[db] *= alpha;
        }
      }
    }
    hold();
    f16x8_t pb[KB][2];  // [kb][16-key chunk m]: keys 16 m + 8 (e / 4) + 4 h + e % 4 of element e
#pragma unroll
    for (int kb = 0; kb < KB; ++kb)
#pragma unroll
      for (int m = 0; m < 2; ++m) {
        float p[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          p[e] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[kb][8 * m + e], a.scale_log2, -m_run));
          l_run += p[e];
        }
        pb[kb][m] = __builtin_bit_cast(f16x8_t, u32x4_t{pack_f16x2(p[0], p[1]), pack_f16x2(p[2], p[3]),
                                                        pack_f16x2(p[4], p[5]), pack_f16x2(p[6], p[7])});
      }

    // values O^T[dim][row] += C~^T P^T
#pragma unroll
    for (int kb = 0; kb < KB; ++kb)
#pragma unroll
      for (int m = 0; m < 2; ++m) {
        const unsigned char* vp = tb + off_v + (32 * kb + 16 * m) * C::LROW;
#pragma unroll
        for (int db = 0; db < NDB; ++db) {
          // logical piece 4 db + vlo; rows +0 and +8 swizzle with 4 (r16 / 4) + h and + 2
          const int p0 = 256 * (db >> 2) + 16 * (4 * ((db & 3) ^ (r16 >> 2)) + (vlo ^ h));
          const int p1 = 256 * (db >> 2) + 16 * (4 * ((db & 3) ^ (r16 >> 2)) + (vlo ^ (h + 2)));
          const s16x4_t a0 = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s16x4_t*)(vp + p0));
          const s16x4_t a1 = __builtin_amdgcn_ds_read_tr16_b64_v4i16(
              (__attribute__((address_space(3))) s16x4_t*)(vp + 8 * C::LROW + p1));
          const f16x8_t av = __builtin_bit_cast(f16x8_t, __builtin_shufflevector(a0, a1, 0, 1, 2, 3, 4, 5, 6, 7));
          o[db] = __builtin_amdgcn_mfma_f32_32x32x16_f16(av, pb[kb][m], o[db], 0, 0, 0);
        }
      }
    if constexpr (PA > 0) {  // operands PA products ahead
      __builtin_amdgcn_sched_group_barrier(0x100, 2 * PA, 1);
#pragma unroll
      for (int c = 0; c < KB * 2 * NDB - PA; ++c) {
        __builtin_amdgcn_sched_group_barrier(0x008, 1, 1);
        __builtin_amdgcn_sched_group_barrier(0x100, 2, 1);
      }
      __builtin_amdgcn_sched_group_barrier(0x008, PA, 1);
    }
  };

  if (t0 < t1) {
    issue_tile(t0, lds0);
    tile_landed();
    __syncthreads();
  }
  // step i computes tile i from `tb` and copies tile i + 1 into `nb` (last read in step i - 1, which ended in a barrier)
  auto step = [&](int i, const unsigned char* tb, unsigned char* nb) __attribute__((always_inline)) {
    if (i + 1 < t1) issue_tile(i + 1, nb);
    attend(tb, L - i * C::KEYS);
    tile_landed();
    __syncthreads();
  };
  for (int i = t0; i < t1; i += 2) {
    step(i, lds0, lds1);
    if (i + 1 < t1) step(i + 1, lds1, lds0);
  }

  if constexpr (OWN) {
    // own tokens: a tile's raw rows are copied to where the tile's pieces lie (a lane takes the piece that belongs at its
    // place), its gate rows beside them in `gate_s` in the same order, and gated in place; wave w copies and gates rows
    // 8 w .. 8 w + 7, a row's latent one piece (16 bytes) a lane
    static_assert(C::KEYS == 32 && DC == 512 && C::LROW == 1024, "a row's latent is a wave's 64 pieces");
    __shared__ __attribute__((aligned(16))) unsigned char gate_s[32 * DC * 2];
    __shared__ int2 list[kOwnList];  // (cache row, id)
    const int b = rb / a.blocks_per_seq;
    const int own = a.own_lens ? clamp_len(a.own_lens[b], a.own_cap) : 0;
    const int own_tiles = (own + 31) / 32, own_per = (own_tiles + a.s_max - 1) / a.s_max;
    const int k0 = min(32 * split * own_per, own), k1 = min(k0 + 32 * own_per, own);  // this work-group's tokens
    auto fill_list = [&](int base) __attribute__((always_inline)) {  // tokens base .. of this work-group
#pragma unroll
      for (int e = 0; e < kOwnList / kPrefixThreads; ++e) {
        const int t = base + tid + e * kPrefixThreads;
        if (t < k1) {
          const int slot = static_cast<int>(cache_slot(a.own_table, b, t, a.P, a.own_pages, a.num_slots));
          list[t - base] = make_int2(slot, clamp_id(a.ids[slot], a.V));
        }
      }
    };
    auto copy = [&](const uint16_t* from, unsigned char* to) __attribute__((always_inline)) {  // 16 bytes a lane
      __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void*)from, lds_ptr(to), 16, 0, 0);
    };
    // (tokens past the last repeat it and are masked)
    auto issue_raw = [&](int t, int base, unsigned char* tb) __attribute__((always_inline)) {
      int lane = threadIdx.x & 63;  // (not known to be the same each time: the addresses are not kept over `attend`)
      asm volatile("" : "+v"(lane));
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const int k = 8 * w + j;
        const int2 e = list[min(t + k, k1 - 1) - base];
        const int slot = __builtin_amdgcn_readfirstlane(e.x), id = __builtin_amdgcn_readfirstlane(e.y);
        const int at = prefix_latent_byte(k, lane) / 2;  // the swizzle is its own inverse
        copy(a.cache + static_cast<int64_t>(slot) * DQ + at, tb + 1024 * k);
        copy(a.gate + static_cast<int64_t>(id) * DC + at, gate_s + 1024 * k);
      }
      const int k = 8 * w + (lane >> 3);
      const int slot = list[min(t + k, k1 - 1) - base].x;
      copy(a.cache + static_cast<int64_t>(slot) * DQ + DC + prefix_rope_byte(k, lane & 7) / 2, tb + C::ROPE + 1024 * w);
    };
    auto gate_tile = [&](unsigned char* tb) __attribute__((always_inline)) {  // this wave's rows
      int lane = threadIdx.x & 63;
      asm volatile("" : "+v"(lane));
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const int at = 1024 * (8 * w + j) + 16 * lane;
        u32x4_t* x = reinterpret_cast<u32x4_t*>(tb + at);
        *x = gate_chunk_f16(*x, *reinterpret_cast<const u32x4_t*>(gate_s + at));
      }
    };
    for (int base = k0; base < k1; base += kOwnList) {
      fill_list(base);
      __syncthreads();
      const int end = min(base + kOwnList, k1);
      issue_raw(base, base, lds0);
      // the tile of tokens t .. in `tb`; the next one's rows into `nb`, whose last reader's step ended before the barrier
      auto own_step = [&](int t, unsigned char* tb, unsigned char* nb) __attribute__((always_inline)) {
        tile_landed();
        gate_tile(tb);
        __syncthreads();
        if (t + 32 < end) issue_raw(t + 32, base, nb);
        attend(tb, k1 - t);
      };
      for (int t = base; t < end; t += 64) {
        own_step(t, lds0, lds1);
        if (t + 32 < end) own_step(t + 32, lds1, lds0);
      }
      __syncthreads();  // the list and the tiles have been read
    }
  }

  // lane holds dims 32 db + 16 j + 8 h + 0..7 of its row in o[db][8 j + 0..7]; a row whose scores all overflowed to -inf
  // (or that had no token) weighs nothing; a NaN among them stays one
  const float l = half_sum(l_run);
  const bool none = l == 0.f;
  [[maybe_unused]] const float inv = none ? 0.f : 1.0f / l;
  int lane_e = tid & 63;  // (the row is formed anew: nothing of it is kept over the loops)
  asm volatile("" : "+v"(lane_e));
  const int he = lane_e >> 5, row_e = rb * kPrefixRows + 32 * w + (lane_e & 31);
  if (row_e < a.rows) {
    int64_t at = static_cast<int64_t>(split) * a.rows + row_e;
    if constexpr (OWN) {
      const int H = a.blocks_per_seq * kPrefixRows, b = rb / a.blocks_per_seq;
      at = (static_cast<int64_t>(b) * a.s_max + split) * H + (row_e - b * H);
    }
    if (he == 0) *reinterpret_cast<float2*>(a.part_ml + 2 * at) = make_float2(none ? -INFINITY : m_run, l);
    if constexpr (HALF) {
      uint16_t* orow = static_cast<uint16_t*>(a.part_o) + at * DC + 8 * he;
#pragma unroll
      for (int db = 0; db < NDB; ++db)
#pragma unroll
        for (int j = 0; j < 2; ++j)
          *reinterpret_cast<u32x4_t*>(orow + 32 * db + 16 * j) =
              u32x4_t{pack_f16x2(o[db][8 * j] * inv, o[db][8 * j + 1] * inv),
                      pack_f16x2(o[db][8 * j + 2] * inv, o[db][8 * j + 3] * inv),
                      pack_f16x2(o[db][8 * j + 4] * inv, o[db][8 * j + 5] * inv),
                      pack_f16x2(o[db][8 * j + 6] * inv, o[db][8 * j + 7] * inv)};
    } else {
      float* orow = static_cast<float*>(a.part_o) + at * DC + 8 * he;
#pragma unroll
      for (int db = 0; db < NDB; ++db)
#pragma unroll
        for (int j = 0; j < 4; ++j)
          *reinterpret_cast<f32x4_t*>(orow + 32 * db + 16 * (j >> 1) + 4 * (j & 1)) =
              f32x4_t{o[db][4 * j], o[db][4 * j + 1], o[db][4 * j + 2], o[db][4 * j + 3]};
    }
  }
#endif
}

template <int DC, int KEYS, bool OWN, bool HALF>
__global__ __launch_bounds__(kPrefixThreads, DC == 128 ? 2 : 1) void shared_prefix_kernel(PrefixArgs a) {
  prefix_item<DC, KEYS, OWN, HALF>(a, blockIdx.x, gridDim.x);
}

// Both parts of a short call in one launch (d_c 128): the first own_wgs
// work-groups run the own tokens' split kernel, the others the prefix, in 32-key
// tiles so that both fit a compute unit twice over.  Each part alone would
// mostly wait for its own chain of loads.
__global__ __launch_bounds__(kPrefixThreads, 2) void shared_both_kernel(PrefixArgs a, SplitArgs own, int own_wgs) {
  const int bid = blockIdx.x;
  if (bid < own_wgs) split_slice_item<128, 64, 4, 2, 1, false, false, kBothList>(own, bid, own_wgs);
  else prefix_item<128, 32, false, false>(a, bid - own_wgs, gridDim.x - own_wgs);
}

// ---------------------------------------------------------------------------
// Merge and up-projection: grid (H, ceil(B / spw)), 8 waves, one head and
// spw = 1, 2, 4, 8 or 16 sequences per work-group.  DC / 8 lanes hold a row (8
// dims each); with 4 rows to a wave (d_c 128) or one, each group of lanes is a
// worker, and spw sequences share the work-group's workers in rounds.  A
// worker folds every W-th partial row of its sequence (the prefix's, then its
// own tokens') online in fp32, 2, 4 or 8 rows loaded together; the workers
// of a sequence meet in LDS, and the merged row o / l goes there once more as
// bf16 hi + lo, the B operands of out^T[v][b] = W_UV[h] o^T on
// v_mfma_f32_16x16x32_bf16.  Latency-bound: the rows' two round trips, the
// exchanges, W_UV's rows (loaded at the start).
// ---------------------------------------------------------------------------
constexpr int kSharedMergeWaves = 8;
constexpr int kSharedMergeSeq = 16;
template <int N>
struct Batch {
  static constexpr int value = N;
};

struct SharedMergeArgs {
  const float* pre_ml;      // [rows][2]: split i of sequence b and head h at row i pre_step + b pre_seq + h
  const void* pre_o;        // [rows][DC] fp32 sums; HALF: fp16, normalised
  const int32_t* pre_len;   // null: a row in every split
  int64_t pre_step, pre_seq;
  const float* own_ml;
  const void* own_o;        // fp32 sums, [B][own_s_max][H][DC]; HALF: fp16, normalised, rows of own_rows
  const int32_t* own_lens;  // null: no own tokens (HALF: not used)
  const int2* own_rows;     // HALF; null: no own tokens' rows
  const uint16_t* w_uv;
  uint16_t* out;
  int32_t B, H, pre_cap, pre_s_max, own_cap, own_split, own_s_max, spw, keys;
};

template <int DC, bool HALF>
__global__ __launch_bounds__(kSharedMergeWaves * 64) void shared_merge_kernel(SharedMergeArgs a) {
  constexpr int DV = 128, NKC = DC / 32, OS = DC + 8;
  constexpr int LPR = DC / 8, GPW = 64 / LPR;       // lanes per row, rows (workers) per wave
  constexpr int WORKERS = kSharedMergeWaves * GPW;
  __shared__ __attribute__((aligned(16))) uint16_t o_s[2][kSharedMergeSeq][OS];  // merged rows, hi and lo
  __shared__ __attribute__((aligned(16))) float part[WORKERS][DC];
  __shared__ float m_part[WORKERS], l_part[WORKERS];
  const int h = blockIdx.x, b0 = blockIdx.y * a.spw;
  const int tid = threadIdx.x, w = tid >> 6, lane = tid & 63, r16 = lane & 15, g = lane >> 4;
  const int nseq = min(a.spw, a.B - b0);
  // W_UV rows 16 w + r16 (columns 32 kc + 8 g ..) of this wave's output tile
  u32x4_t wa[NKC];
  auto load_w = [&]() {
    const uint16_t* wrow = a.w_uv + (static_cast<int64_t>(h) * DV + 16 * w + r16) * DC + 8 * g;
#pragma unroll
    for (int kc = 0; kc < NKC; ++kc) wa[kc] = *reinterpret_cast<const u32x4_t*>(wrow + 32 * kc);
  };
  if constexpr (DC <= 128) load_w();

  const int pre_n = a.pre_len ? prefix_splits(clamp_len(a.pre_len[0], a.pre_cap), a.pre_s_max, a.keys) : a.pre_s_max;
  const int wps = max(1, WORKERS / a.spw);  // workers per sequence (spw <= WORKERS where GPW > 1, else rounds)
  const int spr = WORKERS / wps;            // sequences per round
  const int worker = w * GPW + (GPW > 1 ? lane / LPR : 0);
  const bool live = GPW > 1 || lane < LPR;  // lanes without a piece of a row
  const int col = 8 * (lane % LPR);
  for (int r0 = 0; r0 < a.spw; r0 += spr) {
    const int k = r0 + worker / wps, me = worker % wps;
    const int b = b0 + k;
    float M = -INFINITY, sum = 0.f, acc[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
    // rows me, me + wps, ... < n of a part, U at a time; load(i, ml, v) reads row i
    auto fold_by = [&](auto batch, int n, auto load) {
      constexpr int U = decltype(batch)::value;
      for (int i0 = me; i0 < n; i0 += wps * U) {
        float2 ml[U];
        float v[U][8];
#pragma unroll
        for (int u = 0; u < U; ++u) load(min(i0 + u * wps, n - 1), ml[u], v[u]);
        float top = M;
#pragma unroll
        for (int u = 0; u < U; ++u) top = fmaxf(top, ml[u].x);  // repeats change no maximum
        const bool any = top > -INFINITY;  // rows without weight have maximum -inf
        const float keep = any ? __builtin_amdgcn_exp2f(M - top) : 1.f;
        sum *= keep;
#pragma unroll
        for (int e = 0; e < 8; ++e) acc[e] *= keep;
#pragma unroll
        for (int u = 0; u < U; ++u) {
          const float x = any && i0 + u * wps < n ? __builtin_amdgcn_exp2f(ml[u].x - top) : 0.f;
          sum = fmaf(x, ml[u].y, sum);
          const float y = HALF ? x * ml[u].y : x;
#pragma unroll
          for (int e = 0; e < 8; ++e) acc[e] = fmaf(y, v[u][e], acc[e]);
        }
        M = top;
      }
    };
    auto fold = [&](int n, auto load) {
      if (n <= 2 * wps) fold_by(Batch<2>{}, n, load);
      else if (n <= 4 * wps) fold_by(Batch<4>{}, n, load);
      else fold_by(Batch<8>{}, n, load);
    };
    auto row = [&](const float* part_ml, const void* part_o, int64_t at, float2& ml, float (&v)[8]) {
      ml = *reinterpret_cast<const float2*>(part_ml + 2 * at);
      if constexpr (HALF) {
        const f16x8_t x = *reinterpret_cast<const f16x8_t*>(static_cast<const uint16_t*>(part_o) + at * DC + col);
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] = static_cast<float>(x[e]);
      } else {
        const f32x4_t* p = reinterpret_cast<const f32x4_t*>(static_cast<const float*>(part_o) + at * DC + col);
        const f32x4_t x = p[0], y = p[1];
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          v[e] = x[e];
          v[4 + e] = y[e];
        }
      }
    };
    if (live && k < nseq) {
      const int64_t pre0 = b * a.pre_seq + h;
      if constexpr (HALF) {  // one list
        const int2 list = a.own_rows ? a.own_rows[b] : make_int2(0, 0);
        fold(pre_n + list.y, [&](int i, float2& ml, float (&v)[8]) {
          const bool own = i >= pre_n;
          const int64_t at = own ? static_cast<int64_t>(list.x + i - pre_n) * a.H + h : i * a.pre_step + pre0;
          row(own ? a.own_ml : a.pre_ml, own ? a.own_o : a.pre_o, at, ml, v);
        });
      } else {
        fold(pre_n, [&](int i, float2& ml, float (&v)[8]) { row(a.pre_ml, a.pre_o, i * a.pre_step + pre0, ml, v); });
        if (a.own_lens) {
          const int L = clamp_len(a.own_lens[b], a.own_cap);
          fold(min((L + a.own_split - 1) / a.own_split, a.own_s_max), [&](int i, float2& ml, float (&v)[8]) {
            row(a.own_ml, a.own_o, (static_cast<int64_t>(b) * a.own_s_max + i) * a.H + h, ml, v);
          });
        }
      }
    }
    if (r0 > 0) __syncthreads();  // the round before has been read
    if (live) {
      *reinterpret_cast<f32x4_t*>(&part[worker][col]) = f32x4_t{acc[0], acc[1], acc[2], acc[3]};
      *reinterpret_cast<f32x4_t*>(&part[worker][col + 4]) = f32x4_t{acc[4], acc[5], acc[6], acc[7]};
      if (lane % LPR == 0) {
        m_part[worker] = M;
        l_part[worker] = sum;
      }
    }
    __syncthreads();
    // merged rows of the round's sequences (zero without tokens and past the batch; rows that weigh nothing are added
    // all the same, for a NaN among them)
    for (int i = tid; i < spr * DC; i += kSharedMergeWaves * 64) {
      const int kk = i / DC, c = i - kk * DC;
      float top = -INFINITY, num = 0.f, den = 0.f;
      for (int p = 0; p < wps; ++p) top = fmaxf(top, m_part[kk * wps + p]);
      const float ref = top > -INFINITY ? top : 0.f;
      for (int p = 0; p < wps; ++p) {
        const float x = __builtin_amdgcn_exp2f(m_part[kk * wps + p] - ref);
        num = fmaf(x, part[kk * wps + p][c], num);
        den = fmaf(x, l_part[kk * wps + p], den);
      }
      const float v = den == 0.f ? 0.f : num / den;
      const __bf16 hi = static_cast<__bf16>(v);
      o_s[0][r0 + kk][c] = __builtin_bit_cast(uint16_t, hi);
      o_s[1][r0 + kk][c] = __builtin_bit_cast(uint16_t, static_cast<__bf16>(v - static_cast<float>(hi)));
    }
  }
  __syncthreads();
  if constexpr (DC > 128) load_w();
  f32x4_t o = {0.f, 0.f, 0.f, 0.f};
  const int rr = min(r16, a.spw - 1);  // columns past spw repeat the last and are not stored
#pragma unroll
  for (int kc = 0; kc < NKC; ++kc) {
    const bf16x8_t av = __builtin_bit_cast(bf16x8_t, wa[kc]);
    o = __builtin_amdgcn_mfma_f32_16x16x32_bf16(av, *reinterpret_cast<const bf16x8_t*>(&o_s[0][rr][32 * kc + 8 * g]), o, 0, 0, 0);
    o = __builtin_amdgcn_mfma_f32_16x16x32_bf16(av, *reinterpret_cast<const bf16x8_t*>(&o_s[1][rr][32 * kc + 8 * g]), o, 0, 0, 0);
  }
  // lane: rows 16 w + 4 g + 0..3 of sequence b0 + r16
  if (r16 < nseq)
    *reinterpret_cast<u32x2_t*>(a.out + (static_cast<int64_t>(b0 + r16) * a.H + h) * DV + 16 * w + 4 * g) =
        u32x2_t{pack_bf16x2(o[0], o[1]), pack_bf16x2(o[2], o[3])};
}

}  // namespace egmla
