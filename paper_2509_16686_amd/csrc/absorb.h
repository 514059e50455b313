// Query absorption shared by the decode and the page scores.
#pragma once

#include <hip/hip_runtime.h>

#include "eg_mla.h"

namespace egmla {

// Enqueues qfull[b, h] = [W_UK[h]^T q^C[b, h] | q^R[b, h]] in fp32, [batch, H, d_c + d_r], for any shape and
// storage type (decode.hip).
hipError_t launch_absorb(const eg_mla_dims& d, int32_t batch, const void* q, const void* w_uk, float* qfull,
                         hipStream_t stream);

}  // namespace egmla
