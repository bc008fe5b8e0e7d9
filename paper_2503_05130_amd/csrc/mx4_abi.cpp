// C ABI of matrices in microscaled 4 bits.  All checks of their arguments are here.
#include <cstdint>

#include "abi.h"
#include "mx4.h"

using namespace iefwd;

namespace {

void check_matrix(uint32_t rows, uint32_t K) {
    if (rows == 0 || rows > (1u << 24) || K == 0 || K > (1u << 20) || (uint64_t)rows * K > (1ull << 36))
        fail(IEFWD_EINVAL, "a matrix has 1 to 2^24 rows, 1 to 2^20 columns and at most 2^36 elements");
}

void check_packed(const char *what, const void *p) {
    if (!p || !aligned16(p)) fail(IEFWD_EINVAL, std::string(what) + " must be 16-byte aligned and not NULL");
}

// Rows of a matrix in memory: its type and stride, in elements.
void check_rows(uint32_t type, const void *p, uint64_t stride, uint32_t K) {
    if (type > IEFWD_F32) fail(IEFWD_EINVAL, "unknown type");
    if (!p) fail(IEFWD_EINVAL, "NULL pointer");
    if ((uintptr_t)p % (type == IEFWD_F32 ? 4 : 2)) fail(IEFWD_EINVAL, "elements must be aligned");
    if (stride < K || stride > (1ull << 40)) fail(IEFWD_EINVAL, "the row stride must be at least K and at most 2^40");
}

void check_product(uint32_t epilogue, const void *w, const float *resid, const void *out, uint32_t M, uint32_t N, uint32_t K) {
    check_matrix(M, K);
    check_matrix(N, K);
    if ((uint64_t)M * N > (1ull << 36)) fail(IEFWD_EINVAL, "M * N must be at most 2^36");
    if (epilogue > IEFWD_EPI_BIAS_RESID_F32) fail(IEFWD_EINVAL, "unknown epilogue");
    check_packed("w", w);
    check_packed("out", out);
    if (epilogue == IEFWD_EPI_BIAS_RESID_F32) check_packed("resid", resid);
}

}  // namespace

extern "C" {

int iefwd_mx4_bytes(uint32_t rows, uint32_t K, size_t *bytes) {
    return guarded([&] {
        if (!bytes) fail(IEFWD_EINVAL, "bytes is NULL");
        check_matrix(rows, K);
        *bytes = mx4_bytes((int)rows, (int)K);
    });
}

int iefwd_mx4_quantize(uint32_t type, const void *x, uint64_t x_stride, void *dst, uint32_t rows, uint32_t K, void *stream) {
    return guarded([&] {
        check_matrix(rows, K);
        check_rows(type, x, x_stride, K);
        check_packed("dst", dst);
        hip_check(launch_mx4_quantize(type == IEFWD_F32, x, (int64_t)x_stride, dst, (int)rows, (int)K, (hipStream_t)stream),
                  "microscaled quantisation launch");
    });
}

int iefwd_mx4_pack(const void *codes, const void *scales, void *dst, uint32_t rows, uint32_t K, void *stream) {
    return guarded([&] {
        check_matrix(rows, K);
        if (K % 32) fail(IEFWD_EINVAL, "K must be a multiple of 32");
        check_packed("codes", codes);
        if (!scales) fail(IEFWD_EINVAL, "scales is NULL");
        check_packed("dst", dst);
        hip_check(launch_mx4_pack((const uint8_t *)codes, (const uint8_t *)scales, dst, (int)rows, (int)K, (hipStream_t)stream),
                  "microscaled pack launch");
    });
}

int iefwd_mx4_values(const void *src, uint32_t type, void *out, uint64_t out_stride, uint32_t rows, uint32_t K, void *stream) {
    return guarded([&] {
        check_matrix(rows, K);
        check_rows(type, out, out_stride, K);
        check_packed("src", src);
        hip_check(launch_mx4_values(src, type == IEFWD_F32, out, (int64_t)out_stride, (int)rows, (int)K, (hipStream_t)stream),
                  "microscaled values launch");
    });
}

int iefwd_mx4_gemm(uint32_t epilogue, const void *a, const void *w, const void *bias, const float *resid, void *out,
                   uint32_t M, uint32_t N, uint32_t K, void *stream) {
    return guarded([&] {
        check_product(epilogue, w, resid, out, M, N, K);
        check_packed("a", a);
        hip_check(launch_mx4_gemm((Epi)epilogue, a, w, (const bf16_t *)bias, resid, out, (int)M, (int)N, (int)K,
                                  (hipStream_t)stream),
                  "microscaled product launch");
    });
}

int iefwd_mx4_gemm_bf16(uint32_t epilogue, const void *a, const void *w, const void *bias, const float *resid, void *out,
                        uint32_t M, uint32_t N, uint32_t K, void *stream) {
    return guarded([&] {
        check_product(epilogue, w, resid, out, M, N, K);
        check_packed("a", a);
        if (M > 16) fail(IEFWD_EINVAL, "M must be in [1, 16]");
        if (K % 8) fail(IEFWD_EINVAL, "K must be a multiple of 8");
        hip_check(launch_mx4_gemm_bf16((Epi)epilogue, (const bf16_t *)a, w, (const bf16_t *)bias, resid, out, (int)M, (int)N,
                                       (int)K, (hipStream_t)stream),
                  "microscaled product launch");
    });
}

}  // extern "C"
