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

// A workgroup takes a tile of following tokens of one head, a thread 8 columns of K and of V of one of them, a quad of lanes a block of
// 32: neighbouring lanes have neighbouring addresses on the bf16 side, which is the most of the bytes.
//
// Bound by its bytes for prompts: 24001 tokens of 8 x 128 are written in 26 us (4.75 TB/s) and 26000 read back in 33 us (4.0; lanes
// in the order of the pages' pieces 36); 48 tokens take 2.5 us either way, a launch and two loads in a row.
template <int DH>
struct Tile {
    static constexpr int EIGHTHS = DH / 8, TOKENS = kThreads / EIGHTHS;
    int token, head, eighth;

    __device__ Tile(int kv_heads) {
        const int tile = blockIdx.x / kv_heads;
        head = blockIdx.x - tile * kv_heads;
        token = tile * TOKENS + threadIdx.x / EIGHTHS;
        eighth = threadIdx.x % EIGHTHS;
    }
};

template <int DH>
__global__ __launch_bounds__(kThreads) void paged_append_mx4_kernel(PagedCache c, const bf16_t *__restrict__ k,
                                                                    const bf16_t *__restrict__ v,
                                                                    const int64_t *__restrict__ slots, int tokens,
                                                                    int64_t k_stride, int64_t v_stride) {
    const Tile<DH> at(c.kv_heads);
    const int page = 1 << c.page_log2;
    if (at.token >= tokens) return;      // whole quads
    const int64_t slot = slots[at.token];
    const int col = at.head * DH + 8 * at.eighth;
    Eight x[2] = {};
    x[0].lo = *reinterpret_cast<const u32x4 *>(k + at.token * k_stride + col);
    x[1].lo = *reinterpret_cast<const u32x4 *>(v + at.token * v_stride + col);
    if (slot < 0 || slot >= (int64_t)c.n_pages << c.page_log2) return;
    const size_t part = ((size_t)(slot >> c.page_log2) * c.kv_heads + at.head) * (page * (DH / 32 * 17));
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        const uint32_t scale = mx4_scale<false>(x[i]);
        const Mx4Place p = mx4_place(i, page, DH, (int)(slot & (page - 1)), at.eighth);
        char *dst = static_cast<char *>(i ? c.v : c.k) + part;
        *reinterpret_cast<uint32_t *>(dst + p.codes) = mx4_codes<false>(x[i], scale);
        if ((at.eighth & 3) == 0) dst[p.scale] = (char)scale;
    }
}

// 8 columns of K (of V) of a place as bf16.
template <int DH, KvKind KIND>
__device__ inline u32x4 read_eight(const PagedCache &c, bool is_v, size_t part, int page, int place, int eighth, int head) {
    const char *src = static_cast<const char *>(is_v ? c.v : c.k);
    const size_t elements = (size_t)page * DH;
    if constexpr (KIND == KvKind::Mx4) {
        src += part * (elements / 32 * 17);
        const Mx4Place at = mx4_place(is_v, page, DH, place, eighth);
        return mx4_bf16(*reinterpret_cast<const uint32_t *>(src + at.codes), (uint8_t)src[at.scale]);
    } else if constexpr (KIND == KvKind::Bf16) {
        src += part * elements * 2;
        if (!is_v) return *reinterpret_cast<const u32x4 *>(src + (eighth * page + place) * 16);
        const bf16_t *p = reinterpret_cast<const bf16_t *>(src) + ((place >> 2) * DH + 8 * eighth) * 4 + (place & 3);
        u32x4 out;
#pragma unroll
        for (int e = 0; e < 4; ++e) out[e] = p[8 * e] | (uint32_t)p[8 * e + 4] << 16;
        return out;
    } else {
        src += part * elements;
        uint32_t b[2] = {0, 0};      // 8 bytes
        if (is_v) {
            const uint8_t *p = reinterpret_cast<const uint8_t *>(src) + ((place >> 2) * DH + 8 * eighth) * 4 + (place & 3);
#pragma unroll
            for (int e = 0; e < 8; ++e) b[e / 4] |= (uint32_t)p[4 * e] << (8 * (e & 3));
        } else {
            const u32x2 w = *reinterpret_cast<const u32x2 *>(src + ((eighth >> 1) * page + place) * 16 + (eighth & 1) * 8);
            b[0] = w[0];
            b[1] = w[1];
        }
        const float s = is_v ? c.v_scale[head] : c.k_scale[head];
        u32x4 out;
#pragma unroll
        for (int e = 0; e < 2; ++e) {
            const f32x2 lo = __builtin_amdgcn_cvt_pk_f32_fp8((int)b[e], false), hi = __builtin_amdgcn_cvt_pk_f32_fp8((int)b[e], true);
            out[2 * e] = pack2(lo[0] * s, lo[1] * s);
            out[2 * e + 1] = pack2(hi[0] * s, hi[1] * s);
        }
        return out;
    }
}

template <int DH, KvKind KIND>
__global__ __launch_bounds__(kThreads) void paged_read_kernel(PagedCache c, const int64_t *__restrict__ slots,
                                                              bf16_t *__restrict__ k, bf16_t *__restrict__ v, int tokens,
                                                              int64_t k_stride, int64_t v_stride) {
    const Tile<DH> at(c.kv_heads);
    const int page = 1 << c.page_log2;
    if (at.token >= tokens) return;
    const int64_t slot = slots[at.token];
    u32x4 x[2] = {};
    if (slot >= 0 && slot < (int64_t)c.n_pages << c.page_log2) {
        const size_t part = (size_t)(slot >> c.page_log2) * c.kv_heads + at.head;
#pragma unroll
        for (int i = 0; i < 2; ++i) x[i] = read_eight<DH, KIND>(c, i, part, page, (int)(slot & (page - 1)), at.eighth, at.head);
    }
    const int col = at.head * DH + 8 * at.eighth;
    *reinterpret_cast<u32x4 *>(k + at.token * k_stride + col) = x[0];
    *reinterpret_cast<u32x4 *>(v + at.token * v_stride + col) = x[1];
}

dim3 grid_of(const PagedCache &c, int tokens) {
    const int per_tile = kThreads / (c.head_dim / 8);
    return dim3((unsigned)((int64_t)((tokens + per_tile - 1) / per_tile) * c.kv_heads));
}

template <KvKind KIND>
hipError_t launch_read(const PagedCache &c, const int64_t *slots, bf16_t *k, bf16_t *v, int tokens, int64_t k_stride,
                       int64_t v_stride, hipStream_t stream) {
    auto launch = [&](auto kernel) {
        return launch_kernel(kernel, grid_of(c, tokens), dim3(kThreads), stream, c, slots, k, v, tokens, k_stride, v_stride);
    };
    return c.head_dim == 64 ? launch(paged_read_kernel<64, KIND>) : launch(paged_read_kernel<128, KIND>);
}

}  // namespace

hipError_t launch_paged_append_mx4(const PagedCache &c, const bf16_t *k, const bf16_t *v, const int64_t *slots, int tokens,
                                   int64_t k_stride, int64_t v_stride, hipStream_t stream) {
    auto launch = [&](auto kernel) {
        return launch_kernel(kernel, grid_of(c, tokens), dim3(kThreads), stream, c, k, v, slots, tokens, k_stride, v_stride);
    };
    return c.head_dim == 64 ? launch(paged_append_mx4_kernel<64>) : launch(paged_append_mx4_kernel<128>);
}

hipError_t launch_paged_read(const PagedCache &c, const int64_t *slots, bf16_t *k, bf16_t *v, int tokens, int64_t k_stride,
                             int64_t v_stride, hipStream_t stream) {
    switch (c.kind) {
    case KvKind::Bf16: return launch_read<KvKind::Bf16>(c, slots, k, v, tokens, k_stride, v_stride, stream);
    case KvKind::E4m3: return launch_read<KvKind::E4m3>(c, slots, k, v, tokens, k_stride, v_stride, stream);
    case KvKind::Mx4: return launch_read<KvKind::Mx4>(c, slots, k, v, tokens, k_stride, v_stride, stream);
    }
    return hipErrorInvalidValue;
}

}  // namespace iefwd
