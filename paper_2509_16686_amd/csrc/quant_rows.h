// Attention over the 8-bit cache for blocks of 128 query rows (gfx950 MFMA).
// Included by quant_attend.hip.
//
// Bound by the matrix cores, and at d_c up to 128 by the softmax's vector
// instructions, once a few dozen rows share a key.  A work-group of 4 waves holds
// 128 rows, 32 a wave, in registers, and takes its keys in tiles of 64 (32 above
// d_c 128).  Rows are loaded into registers a tile ahead (through the caches:
// blocks of a sequence share them; chunks 202 -> 195 us a call); the wave that loaded
// a row turns it into fp16 with its scale, once for 128 rows, and writes it into one
// of two tile buffers; scores S^T[key][row] on v_mfma_f32_32x32x16 (A: 32 keys from LDS,
// B: the wave's rows), online softmax per row in the log2 domain with lazy rescale,
// and values O^T[dim][row] += C~^T P^T with the probabilities as the B operand as
// they lie in the score accumulators and transposed LDS reads as the A operand: each
// LDS byte feeds 32 rows.
// Kernel times under the profiler, median and best of 20: 64 sequences of 512-16384 tokens x
// 128 heads of d_c 512 247 and 208 us (0.62 and 0.73 PFLOP/s); 8 chunks of 200-600 tokens x 16
// heads of d_c 128 over 600-8192 193 and 171 us (0.72 and 0.82).
#pragma once

#include "rows32.h"

namespace egmla {

constexpr int kQ8Rows = 128;      // rows of a block
constexpr int kQ8RowsThreads = 256;

// A row's scale as a float; of one that stands for NaN (whose codes are 0) a value that no other has.
constexpr int kQ8None = 0x3f800001;
__device__ __forceinline__ int q8_scale(int byte) { return byte == 255 ? kQ8None : byte << 23; }

template <int DC_>
struct Q8RowsCfg : Q8Tile<DC_> {
  using T = Q8Tile<DC_>;
  static constexpr int DC = DC_, KEYS = T::KEYS;
  static constexpr int NC = DC / 16, NR = 4, KB = KEYS / 32, NDB = DC / 32;
  static constexpr int QL = DC == 512 ? 4 : 0;           // query chunks that wait in LDS beside q^R
  static constexpr int Q_LDS = QL ? (NR + QL) * kQ8RowsThreads * 16 : 16;
  static_assert(T::SPARE + 16 + Q_LDS + 4 * KEYS * 8 <= 160 * 1024 && (KEYS & (KEYS - 1)) == 0, "LDS");
};

// The lane's number, formed anew for each i: nothing that follows from it is kept in between (where registers are full it
// would go to scratch memory, and a reload waits for every load before it, the rows of the next tile among them).
__device__ __forceinline__ int lane_anew(int i) {
  uint32_t zero = 0;
  asm("" : "+s"(zero) : "s"(i));
  return __builtin_amdgcn_mbcnt_hi(~0u, __builtin_amdgcn_mbcnt_lo(~0u, zero)) & 63u;
}

template <int DC>
__global__ __launch_bounds__(kQ8RowsThreads, DC <= 128 ? 2 : 1) void q8_rows_kernel(Q8Attend a) {
#if defined(__HIP_DEVICE_COMPILE__)  // the host pass knows neither the copies to LDS nor the register constraints
  using C = Q8RowsCfg<DC>;
  constexpr int NC = C::NC, NR = C::NR, KB = C::KB, NDB = C::NDB, KW = C::KW, PL = C::PL, QL = C::QL;
  constexpr bool ACC = DC > 128;  // the accumulators are held in the accumulation registers (see shared_prefix.h)
  constexpr int QA = DC == 512 ? 3 : 2, PA = DC <= 128 ? 2 : 4;  // how far LDS reads run ahead of the products
  __shared__ __attribute__((aligned(16))) unsigned char lds[C::SPARE + 16];
  __shared__ __attribute__((aligned(16))) u32x4_t q_s[C::Q_LDS / 16];
  __shared__ int2 list[4][C::KEYS];  // (cache row, scale) of the tokens of four tiles
  const int tid = threadIdx.x, lane = tid & 63, r32 = lane & 31, h = lane >> 5;
  const int w = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int row_bytes = a.DC + 2 * a.DR;

  const int run = xcd_logical_block(blockIdx.x, gridDim.x);
  const int4 mine = uniform(a.start[3 * run]);
  int4 info = uniform(a.start[3 * run + 1]), rw = uniform(a.start[3 * run + 2]);
  const int per = mine.y, blocks = mine.z, tiles = mine.w;
  if (static_cast<int64_t>(run) * per >= tiles) return;
  int at = run * per;
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
    const int j0 = (at - info.w) * C::KEYS, j1 = min((min(end, next) - info.w) * C::KEYS, most);
    const int all = min(first + row0 / a.H + 1, len);  // tokens that every row attends to
    at = min(end, next);

    // this lane's query row (rows past the last repeat it and are not stored) and the tokens that it attends to
    const int r = min(32 * w + r32, nrows - 1);
    const int lim = min(first + (row0 + r) / a.H + 1, len);
    const uint16_t* qrow = a.q + (static_cast<int64_t>(rw.x) + r) * (a.DC + a.DR);
    f16x8_t qv[NC];
    bf16x8_t qr[NR];
#pragma unroll
    for (int c = 0; c < NC; ++c) qv[c] = __builtin_bit_cast(f16x8_t, q8_query(qrow, 16 * c + 8 * h, a.DC));
#pragma unroll
    for (int c = 0; c < NR; ++c) qr[c] = __builtin_bit_cast(bf16x8_t, q8_query(qrow + a.DC, 16 * c + 8 * h, a.DR));
    if constexpr (QL > 0) {
#pragma unroll
      for (int c = 0; c < NR; ++c) q_s[c * kQ8RowsThreads + tid] = __builtin_bit_cast(u32x4_t, qr[c]);
#pragma unroll
      for (int c = 0; c < QL; ++c) q_s[(NR + c) * kQ8RowsThreads + tid] = __builtin_bit_cast(u32x4_t, qv[c]);
    }

    px_f32x16_t o[NDB];
#pragma unroll
    for (int db = 0; db < NDB; ++db)
#pragma unroll
      for (int e = 0; e < 16; ++e) o[db][e] = 0.f;
    float m_run = -1e30f, l_run = 0.f;
    auto hold = [&]() {
      if constexpr (ACC) {
#pragma unroll
        for (int db = 0; db < NDB; ++db) in_agprs(o[db]);
      }
    };

    // attends to the keys of tile i in `tb` that the lane's row sees; `beside` runs among the value products
    auto attend = [&](const unsigned char* tb, int i, auto beside) __attribute__((always_inline)) {
      hold();
      // per-lane LDS offsets, as in shared_prefix.h: score operands (key row r32 of a block of 32) and value operands
      // (d_c 512: formed anew for each tile, there is no room to keep them)
      const int ln = QL > 0 ? lane_anew(i) : lane;
      const int valid = lim - (j0 + i * C::KEYS);
      const int r32 = ln & 31, h = ln >> 5, r16 = ln & 15, R1 = (ln >> 4) & 1;
      const int swz_l = ((r32 & 3) << 2) | ((r32 >> 2) & 3), swz_r = (r32 >> 1) & 7;
      const int off_l = r32 * C::LROW, off_r = C::ROPE + r32 * C::RROW;
      // d_c 512: the compiler has products write accumulation registers, which the values fill, and would move a block of
      // them out and back for each tile; the scores' products are written to ordinary ones by hand, and to two
      // accumulators in turn (a product does not wait for the one before it).  The compiler does not know them for
      // products: each is 2 wait states behind any vector instruction that may have written an operand
      constexpr bool HAND = QL > 0;
      constexpr int NS = HAND ? 2 * KB : KB;
      px_f32x16_t s[NS];
#pragma unroll
      for (int kb = 0; kb < NS; ++kb)
#pragma unroll
        for (int e = 0; e < 16; ++e) s[kb][e] = 0.f;
      // chunks of 16 values, the RoPE key's first; operands are read QA chunks ahead of their products
      u32x4_t sa[QA + 1][KB], sq[QA + 1];
      auto read_chunk = [&](int c) __attribute__((always_inline)) {
        const int d = c - NR;
#pragma unroll
        for (int kb = 0; kb < KB; ++kb)
          sa[c % (QA + 1)][kb] = *reinterpret_cast<const u32x4_t*>(
              c < NR ? tb + off_r + 32 * kb * C::RROW + 16 * ((2 * c + h) ^ swz_r)
                     : tb + off_l + 32 * kb * C::LROW + 256 * (d >> 3) + 16 * ((2 * (d & 7) + h) ^ swz_l));
        if (QL > 0 && c < NR + QL) sq[c % (QA + 1)] = q_s[c * kQ8RowsThreads + 64 * w + ln];
      };
#pragma unroll
      for (int c = 0; c < QA; ++c) read_chunk(c);
#pragma unroll
      for (int c = 0; c < NC + NR; ++c) {
        if (c + QA < NC + NR) read_chunk(c + QA);
        __builtin_amdgcn_sched_barrier(0);
        const u32x4_t bv = QL > 0 && c < NR + QL ? sq[c % (QA + 1)]
                           : c < NR              ? __builtin_bit_cast(u32x4_t, qr[c < NR ? c : 0])
                                                 : __builtin_bit_cast(u32x4_t, qv[c < NR ? 0 : c - NR]);
        if constexpr (HAND) {
          const u32x4_t av = sa[c % (QA + 1)][0];
          if (c < NR) asm("s_nop 1\n\tv_mfma_f32_32x32x16_bf16 %0, %1, %2, %0" : "+v"(s[c % 2]) : "v"(av), "v"(bv));
          else asm("s_nop 1\n\tv_mfma_f32_32x32x16_f16 %0, %1, %2, %0" : "+v"(s[c % 2]) : "v"(av), "v"(bv));
        } else {
#pragma unroll
          for (int kb = 0; kb < KB; ++kb) {
            const u32x4_t av = sa[c % (QA + 1)][kb];
            if (c < NR)
              s[kb] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8_t, av),
                                                              __builtin_bit_cast(bf16x8_t, bv), s[kb], 0, 0, 0);
            else
              s[kb] = __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(f16x8_t, av),
                                                             __builtin_bit_cast(f16x8_t, bv), s[kb], 0, 0, 0);
          }
        }
        __builtin_amdgcn_sched_barrier(0);
      }
      if constexpr (HAND) {  // a product's result is read by a vector instruction 18 wait states behind it at the earliest
        asm("s_nop 15\n\ts_nop 7" : "+v"(s[0]), "+v"(s[1]));
        s[0] += s[1];
      }
      if (__builtin_amdgcn_ballot_w64(valid < C::KEYS)) {  // some row's tokens end inside this tile
#pragma unroll
        for (int kb = 0; kb < KB; ++kb)
#pragma unroll
          for (int e = 0; e < 16; ++e)
            if (32 * kb + 8 * (e >> 2) + 4 * h + (e & 3) >= valid) s[kb][e] = -INFINITY;
      }

      // online softmax (row = lane % 32; keys split between lanes l and l ^ 32); the scale (tau log2 e > 0) commutes with
      // the maximum and is applied inside the exponent
      float mt = s[0][0];
#pragma unroll
      for (int kb = 0; kb < KB; ++kb)
#pragma unroll
        for (int e = 0; e < 16; ++e) mt = fmaxf(mt, s[kb][e]);
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

      // values O^T[dim][row] += C~^T P^T: product i of key chunk i / NDB and dims 32 (i % NDB) .., operands PA products
      // ahead, a few instructions of `beside` behind each
      const int off_v = (4 * h + (r16 >> 2)) * C::LROW + 8 * ((r16 & 3) >> 1);
      const int vlo = 2 * R1 + (r16 & 1);
      constexpr int NV = KB * 2 * NDB;
      s16x4_t va[PA + 1][2];
      auto read_values = [&](int i) __attribute__((always_inline)) {
        const int db = i % NDB;
        const unsigned char* vp = tb + off_v + 16 * (i / NDB) * C::LROW;
        // logical piece 4 db + vlo; rows +0 and +8 swizzle with 4 (r16 / 4) + h and + 2
        const int p0 = 256 * (db >> 2) + 16 * (4 * ((db & 3) ^ (r16 >> 2)) + (vlo ^ h));
        const int p1 = 256 * (db >> 2) + 16 * (4 * ((db & 3) ^ (r16 >> 2)) + (vlo ^ (h + 2)));
        va[i % (PA + 1)][0] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s16x4_t*)(vp + p0));
        va[i % (PA + 1)][1] = __builtin_amdgcn_ds_read_tr16_b64_v4i16(
            (__attribute__((address_space(3))) s16x4_t*)(vp + 8 * C::LROW + p1));
      };
#pragma unroll
      for (int i = 0; i < PA; ++i) read_values(i);
#pragma unroll
      for (int i = 0; i < NV; ++i) {
        if (i + PA < NV) read_values(i + PA);
        __builtin_amdgcn_sched_barrier(0);
        const f16x8_t av = __builtin_bit_cast(
            f16x8_t, __builtin_shufflevector(va[i % (PA + 1)][0], va[i % (PA + 1)][1], 0, 1, 2, 3, 4, 5, 6, 7));
        o[i % NDB] = __builtin_amdgcn_mfma_f32_32x32x16_f16(av, pb[i / NDB / 2][i / NDB % 2], o[i % NDB], 0, 0, 0);
        beside(i, NV);
        __builtin_amdgcn_sched_barrier(0);
      }
    };

    // this wave's rows of a tile, from its list (pieces past a row's end are not looked at)
    u32x4_t lat[C::NLI], rop[C::NRI];
    int sc[C::NLI + C::NRI];  // their scales, as the list has them
    auto issue = [&](int i) __attribute__((always_inline)) {
      const int2* l = list[i & 3];
      const int ln = lane_anew(i);
#pragma unroll
      for (int c = 0; c < C::NLI; ++c) {
        const int p = c * 64 + ln, d = 16 * (p % PL);
        const int2 e = l[min(KW * w + p / PL, KW * w + KW - 1)];
        sc[c] = e.y;
        lat[c] = *(
            reinterpret_cast<const u32x4_t*>(a.codes + static_cast<int64_t>(e.x) * row_bytes + (d < a.DC ? d : 0)));
      }
#pragma unroll
      for (int c = 0; c < C::NRI; ++c) {
        const int p = c * 64 + ln, d = 16 * (p % 8);
        const int2 e = l[KW * w + p / 8];
        sc[C::NLI + c] = e.y;
        rop[c] = *(
            reinterpret_cast<const u32x4_t*>(a.codes + static_cast<int64_t>(e.x) * row_bytes + (d < 2 * a.DR ? a.DC + d : 0)));
      }
    };
    // turns them into fp16 in the tile at byte `base`, in SLOTS short pieces (a piece of codes: place, half, half; one of the RoPE key: place,
    // value).  Columns past d_c hold values that no query and no output has.
    constexpr int SLOTS = 3 * C::NLI + 2 * C::NRI;
    unsigned char* to[2];
    auto convert = [&](int base, int ln, int slot) __attribute__((always_inline)) {
      if (slot < 3 * C::NLI) {
        const int c = slot / 3, p = c * 64 + ln;
        if (slot % 3 == 0) {
          to[0] = lds + q8_latent_store<C>(base, w, p, 0);
          to[1] = lds + q8_latent_store<C>(base, w, p, 1);
        } else {
          const int half = slot % 3 - 1;
          u32x4_t v;
#pragma unroll
          for (int i = 0; i < 2; ++i) {
            const uint32_t x = lat[c][2 * half + i];
            const float f = __int_as_float(sc[c]);
            v[2 * i] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(x, f, false));
            v[2 * i + 1] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(x, f, true));
          }
          *reinterpret_cast<u32x4_t*>(to[half]) = v;
        }
      } else {
        const int c = (slot - 3 * C::NLI) / 2, p = c * 64 + ln, key = KW * w + p / 8, pc = p % 8;
        if ((slot - 3 * C::NLI) % 2 == 0) {
          to[0] = lds + base + C::ROPE + key * C::RROW + prefix_rope_byte(key, pc);
        } else {
          u32x4_t v = rop[c];
          if (8 * pc >= a.DR) v = u32x4_t{0u, 0u, 0u, 0u};
          const uint32_t none = sc[C::NLI + c] == kQ8None ? 0x7fc07fc0u : 0u;  // a row that stands for NaN
          *reinterpret_cast<u32x4_t*>(to[0]) = v | u32x4_t{none, none, none, none};
        }
      }
    };
    auto convert_all = [&](int base) __attribute__((always_inline)) {
#pragma unroll
      for (int i = 0; i < SLOTS; ++i) convert(base, threadIdx.x & 63, i);
    };

    // a tile's tokens (those past the last repeat it and are masked) are listed a tile ahead of their rows' loads: page,
    // then scale, then the entry, a tile apart, by every thread alike (no branch to wait at)
    constexpr int KM = C::KEYS - 1;
    auto token_of = [&](int i) __attribute__((always_inline)) {
      return min(j0 + i * C::KEYS + (lane_anew(i) & KM), j1 - 1);
    };
    for (int t = tid; t < 3 * C::KEYS; t += kQ8RowsThreads) {
      const int j = min(j0 + t, j1 - 1), slot = a.cache.row(b, j, a.cache.page(b, j));
      list[t / C::KEYS][t & KM] = make_int2(slot, q8_scale(a.scales[slot]));
    }
    int j_next = token_of(3);
    int slot_next = a.cache.row(b, j_next, a.cache.page(b, j_next)), scale_next = a.scales[slot_next];
    j_next = token_of(4);
    int page_next = a.cache.page(b, j_next);
    __syncthreads();
    issue(0);
    convert_all(0);
    issue(1);
    // (values that are not finite, of tokens that some row does not attend to; any place of a key's RoPE row serves)
    auto only_finite = [&](unsigned char* tb) __attribute__((always_inline)) {
#pragma unroll 1
      for (int p = threadIdx.x; p < C::KEYS * (DC / 8); p += kQ8RowsThreads) {
        const int key = p / (DC / 8);
        q8_only_finite(reinterpret_cast<u32x4_t*>(tb + key * C::LROW + prefix_latent_byte(key, p % (DC / 8))),
                       reinterpret_cast<u32x4_t*>(tb + C::ROPE + key * C::RROW));
      }
      __syncthreads();
    };
    // tile i of the piece from `tb`; the next one's rows go to byte `next` on (last read in step i - 1), the one's after
    // are loaded
    auto step = [&](int i, unsigned char* tb, int next) __attribute__((always_inline)) {
      __syncthreads();
      if (min(j0 + (i + 1) * C::KEYS, j1) > all) only_finite(tb);
      const int ln = lane_anew(i);
      if (w == 0 && ln < C::KEYS) list[(i + 3) & 3][ln] = make_int2(slot_next, q8_scale(scale_next));
      slot_next = a.cache.row(b, j_next, page_next);
      scale_next = a.scales[slot_next];
      j_next = token_of(i + 5);
      page_next = a.cache.page(b, j_next);
      attend(tb, i, [&](int product, int products) __attribute__((always_inline)) {
#pragma unroll
        for (int slot = 0; slot < SLOTS; ++slot)
          if (slot * products / SLOTS == product) convert(next, ln, slot);
      });
      issue(i + 2);
    };
    const int n = (j1 - j0 + C::KEYS - 1) / C::KEYS;
    for (int i = 0; i < n; ++i) step(i, lds + (i & 1) * C::TILE, (~i & 1) * C::TILE);
    __syncthreads();  // the lists and tiles have been read

    // lane holds dims 32 db + 16 j + 8 h + 0..7 of its row in o[db][8 j + 0..7]; a row that met no token (or whose scores
    // all overflowed to -inf) weighs nothing; a NaN among them stays one
    const float l = half_sum(l_run);
    const int ln = lane_anew(n), he = ln >> 5, re = 32 * w + (ln & 31);
    if (re < nrows) {
      const int64_t prow = (static_cast<int64_t>(run) + k) * kQ8Rows + re;
      if (he == 0) *reinterpret_cast<float2*>(a.part_ml + 2 * prow) = make_float2(l == 0.f ? -INFINITY : m_run, l);
      float* orow = a.part_o + prow * a.DC + 8 * he;
#pragma unroll
      for (int db = 0; db < NDB; ++db)
#pragma unroll
        for (int j = 0; j < 2; ++j)
          if (32 * db + 16 * j < a.DC) {
#pragma unroll
            for (int q = 0; q < 2; ++q)
              *reinterpret_cast<f32x4_t*>(orow + 32 * db + 16 * j + 4 * q) =
                  f32x4_t{o[db][8 * j + 4 * q], o[db][8 * j + 4 * q + 1], o[db][8 * j + 4 * q + 2], o[db][8 * j + 4 * q + 3]};
          }
    }
  }
#endif
}

}  // namespace egmla
