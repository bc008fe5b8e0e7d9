// Products with 4-bit weights and group scales (csrc/q4.hip).  The launchers check
// nothing: the C entry points do.
#pragma once

#include "gemm.h"

namespace iefwd {

// Bytes of the packed copy: codes of 16 features x 128 weights in 1 KB blocks
// (K rounded up to 128), then a scale and an offset per group in 4 bytes.
size_t q4_packed_bytes(int N, int K, int group);

// codes [N, K / 2]: weight 2 i in the low and 2 i + 1 in the high half of byte i;
// scales bf16 [N, K / group]; zeros uint8 [N, K / group] or null (8 everywhere).
hipError_t launch_q4_pack(const uint8_t *codes, const bf16_t *scales, const uint8_t *zeros, void *dst, int N, int K,
                          int group, hipStream_t stream);

// out = epi(A W^T + b), W = scale (code - zero); M <= 16; bias may be null.
hipError_t launch_q4_gemm(Epi epi, const bf16_t *a, const void *packed, const bf16_t *bias, const float *resid, void *out,
                          int M, int N, int K, int group, hipStream_t stream);

}  // namespace iefwd
