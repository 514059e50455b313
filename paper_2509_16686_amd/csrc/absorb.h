// Query absorption shared by the decode and the page scores.
#pragma once

#include <hip/hip_runtime.h>

#include "eg_mla.h"

namespace egmla {

// Enqueues qfull[b, h] = [W_UK[h]^T q^C[b, h] | q^R[b, h]] in fp32, [batch, H, d_c + d_r], for any shape and
// storage type (decode.hip).
hipError_t launch_absorb(const eg_mla_dims& d, int32_t batch, const void* q, const void* w_uk, float* qfull,
                         hipStream_t stream);

// Absorbed query in three bf16 parts that together hold the fp32 q_lat, in the
// order of the A operands of v_mfma_f32_16x16x32_bf16: per sequence and block
// of 16 heads, one run of 1 KB per 32 values of [first part | q^R], then of the
// second and of the third part (d_c values each); in a run the 16 bytes of lane
// 16 g + r are values 8g .. 8g + 7 of head r.  (In rows of d_c values, 1 KB
// apart at d_c 512, the scores of 5100 pages and 128 heads took 22.8 us, 18.4
// with these runs.)  Values past a part's end and heads past the last are not written.
struct PartsLayout {
  int32_t blocks, runs0, runs1;
  __host__ __device__ PartsLayout(int32_t heads, int32_t dc, int32_t dr)
      : blocks((heads + 15) / 16), runs0((dc + dr + 31) / 32), runs1((dc + 31) / 32) {}
  __host__ __device__ int32_t runs() const { return runs0 + 2 * runs1; }  // of a sequence and block of heads
  // 16-bit element of value c of a part of head h of sequence b
  __host__ __device__ int64_t operator()(int32_t b, int32_t h, int32_t part, int32_t c) const {
    const int64_t run = (static_cast<int64_t>(b) * blocks + h / 16) * runs() + (part ? runs0 + (part - 1) * runs1 : 0) + c / 32;
    return run * 512 + (c % 32 / 8 * 16 + h % 16) * 8 + c % 8;
  }
};

// Enqueues the absorption into these parts, for bf16 storage and d_h 64 or 128.
hipError_t launch_absorb_parts(const eg_mla_dims& d, int32_t batch, const void* q, const void* w_uk, uint16_t* parts,
                               hipStream_t stream);

}  // namespace egmla
