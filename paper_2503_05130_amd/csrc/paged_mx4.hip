// New tokens to a paged cache in microscaled 4 bits, and tokens of every kind of cache read back, for gfx950.
#include "mx4_device.h"
#include "paged.h"

namespace iefwd {
namespace {

constexpr int kThreads = 256;

// The place of 8 columns' codes (4 bytes) and of their block's scale in a head's part of a page.
struct Mx4Place {
    uint32_t codes, scale;
};

__device__ inline Mx4Place mx4_place(bool v, int page, int dh, int place, int eighth) {
    const uint32_t scales = page * dh / 2, block = eighth >> 2;
    if (v)
        return {(uint32_t)(((place >> 2) * (dh / 8) + eighth) * 16 + (place & 3) * 4),
                scales + ((place >> 2) * (dh / 32) + block) * 4 + (place & 3)};
    return {(block * page + place) * 16 + (eighth & 3) * 4, scales + block * page + place};
}

// A thread takes 8 columns of K or V of a token and head, a quad of lanes a block.
__global__ __launch_bounds__(kThreads) void paged_append_mx4_kernel(PagedCache c, const bf16_t *__restrict__ k,
                                                                    const bf16_t *__restrict__ v,
                                                                    const int64_t *__restrict__ slots, int64_t threads,
                                                                    int64_t k_stride, int64_t v_stride) {
    const int64_t i = (int64_t)blockIdx.x * kThreads + threadIdx.x;
    if (i >= threads) return;      // whole quads
    const int eighths = c.head_dim / 8, page = 1 << c.page_log2;
    const int64_t row = i / eighths;      // token, head, K or V
    const int eighth = (int)(i - row * eighths);
    const bool is_v = row & 1;
    const int64_t token = (row >> 1) / c.kv_heads;
    const int head = (int)((row >> 1) - token * c.kv_heads);
    const int64_t slot = slots[token];
    if (slot < 0 || slot >= (int64_t)c.n_pages << c.page_log2) return;
    Eight x{};
    x.lo = *reinterpret_cast<const u32x4 *>((is_v ? v + token * v_stride : k + token * k_stride) + head * c.head_dim + 8 * eighth);
    const uint32_t scale = mx4_scale<false>(x);
    const Mx4Place at = mx4_place(is_v, page, c.head_dim, (int)(slot & (page - 1)), eighth);
    char *dst = static_cast<char *>(is_v ? c.v : c.k) + ((size_t)(slot >> c.page_log2) * c.kv_heads + head) * (page * c.head_dim / 32 * 17);
    *reinterpret_cast<uint32_t *>(dst + at.codes) = mx4_codes<false>(x, scale);
    if ((eighth & 3) == 0) dst[at.scale] = (char)scale;
}

template <KvKind KIND>
__global__ __launch_bounds__(kThreads) void paged_read_kernel(PagedCache c, const int64_t *__restrict__ slots,
                                                              bf16_t *__restrict__ k, bf16_t *__restrict__ v, int64_t threads,
                                                              int64_t k_stride, int64_t v_stride) {
    const int64_t i = (int64_t)blockIdx.x * kThreads + threadIdx.x;
    if (i >= threads) return;
    const int dh = c.head_dim, eighths = dh / 8, page = 1 << c.page_log2;
    const int64_t row = i / eighths;
    const int eighth = (int)(i - row * eighths);
    const bool is_v = row & 1;
    const int64_t token = (row >> 1) / c.kv_heads;
    const int head = (int)((row >> 1) - token * c.kv_heads);
    const int64_t slot = slots[token];
    u32x4 out = {0, 0, 0, 0};
    if (slot >= 0 && slot < (int64_t)c.n_pages << c.page_log2) {
        const int place = (int)(slot & (page - 1));
        const size_t part = (size_t)(slot >> c.page_log2) * c.kv_heads + head, elements = (size_t)page * dh;
        const char *src = static_cast<const char *>(is_v ? c.v : c.k);
        if constexpr (KIND == KvKind::Mx4) {
            src += part * (elements / 32 * 17);
            const Mx4Place at = mx4_place(is_v, page, dh, place, eighth);
            out = mx4_bf16(*reinterpret_cast<const uint32_t *>(src + at.codes), (uint8_t)src[at.scale]);
        } else if constexpr (KIND == KvKind::Bf16) {
            src += part * elements * 2;
            if (is_v) {
                const bf16_t *p = reinterpret_cast<const bf16_t *>(src) + ((place >> 2) * dh + 8 * eighth) * 4 + (place & 3);
#pragma unroll
                for (int e = 0; e < 4; ++e) out[e] = p[8 * e] | (uint32_t)p[8 * e + 4] << 16;
            } else {
                out = *reinterpret_cast<const u32x4 *>(src + (eighth * page + place) * 16);
            }
        } else {
            src += part * elements;
            uint32_t b[2] = {0, 0};      // 8 bytes
            if (is_v) {
                const uint8_t *p = reinterpret_cast<const uint8_t *>(src) + ((place >> 2) * dh + 8 * eighth) * 4 + (place & 3);
#pragma unroll
                for (int e = 0; e < 8; ++e) b[e / 4] |= (uint32_t)p[4 * e] << (8 * (e & 3));
            } else {
                const u32x2 w = *reinterpret_cast<const u32x2 *>(src + ((eighth >> 1) * page + place) * 16 + (eighth & 1) * 8);
                b[0] = w[0];
                b[1] = w[1];
            }
            const float s = is_v ? c.v_scale[head] : c.k_scale[head];
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                const f32x2 lo = __builtin_amdgcn_cvt_pk_f32_fp8((int)b[e], false), hi = __builtin_amdgcn_cvt_pk_f32_fp8((int)b[e], true);
                out[2 * e] = pack2(lo[0] * s, lo[1] * s);
                out[2 * e + 1] = pack2(hi[0] * s, hi[1] * s);
            }
        }
    }
    *reinterpret_cast<u32x4 *>((is_v ? v + token * v_stride : k + token * k_stride) + head * dh + 8 * eighth) = out;
}

int64_t threads_of(const PagedCache &c, int tokens) { return (int64_t)tokens * c.kv_heads * 2 * (c.head_dim / 8); }

}  // namespace

hipError_t launch_paged_append_mx4(const PagedCache &c, const bf16_t *k, const bf16_t *v, const int64_t *slots, int tokens,
                                   int64_t k_stride, int64_t v_stride, hipStream_t stream) {
    const int64_t threads = threads_of(c, tokens);
    return launch_kernel(paged_append_mx4_kernel, dim3((unsigned)((threads + kThreads - 1) / kThreads)), dim3(kThreads), stream,
                         c, k, v, slots, threads, k_stride, v_stride);
}

hipError_t launch_paged_read(const PagedCache &c, const int64_t *slots, bf16_t *k, bf16_t *v, int tokens, int64_t k_stride,
                             int64_t v_stride, hipStream_t stream) {
    const int64_t threads = threads_of(c, tokens);
    const dim3 grid((unsigned)((threads + kThreads - 1) / kThreads));
    auto launch = [&](auto kernel) { return launch_kernel(kernel, grid, dim3(kThreads), stream, c, slots, k, v, threads, k_stride, v_stride); };
    switch (c.kind) {
    case KvKind::Bf16: return launch(paged_read_kernel<KvKind::Bf16>);
    case KvKind::E4m3: return launch(paged_read_kernel<KvKind::E4m3>);
    case KvKind::Mx4: return launch(paged_read_kernel<KvKind::Mx4>);
    }
    return hipErrorInvalidValue;
}

}  // namespace iefwd
