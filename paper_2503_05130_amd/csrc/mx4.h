// Matrices in microscaled 4 bits and their products (csrc/mx4.hip).  The
// launchers check nothing: the C entry points do.
#pragma once

#include "gemm.h"

namespace iefwd {

// Row tiles of 16 rows, each `chunks` blocks of 1 KB (16 rows x 128 columns of codes: lane l's 16 bytes are
// row l % 16, columns 32 (l / 16) and on) and behind them a dword per lane for each 4 chunks, its scale bytes.
inline __host__ __device__ int mx4_chunks(int K) { return (K + 127) / 128; }
inline __host__ __device__ size_t mx4_tile_bytes(int K) {
    const int chunks = mx4_chunks(K);
    return (size_t)chunks * 1024 + (size_t)((chunks + 3) / 4) * 256;
}
inline size_t mx4_bytes(int rows, int K) { return (size_t)((rows + 15) / 16) * mx4_tile_bytes(K); }

// x: bf16 or fp32 rows `stride` elements apart; writes whole row tiles (rows past the last and columns past K as zeros).
hipError_t launch_mx4_quantize(bool f32, const void *x, int64_t stride, void *dst, int rows, int K, hipStream_t stream);
// codes [rows, K / 2], scales [rows, K / 32] row-major; K a multiple of 32.
hipError_t launch_mx4_pack(const uint8_t *codes, const uint8_t *scales, void *dst, int rows, int K, hipStream_t stream);
hipError_t launch_mx4_values(const void *src, bool f32, void *out, int64_t stride, int rows, int K, hipStream_t stream);

// out = epi(A W^T + b), A [M, K] and W [N, K] in 4 bits; bias may be null.
hipError_t launch_mx4_gemm(Epi epi, const void *a, const void *w, const bf16_t *bias, const float *resid, void *out, int M,
                           int N, int K, hipStream_t stream);
// The same of a bf16 A [M, K], quantised in the kernel: M <= 16, K a multiple of 8.
hipError_t launch_mx4_gemm_bf16(Epi epi, const bf16_t *a, const void *w, const bf16_t *bias, const float *resid, void *out,
                                int M, int N, int K, hipStream_t stream);

}  // namespace iefwd
