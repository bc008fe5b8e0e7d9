// What the paged attention kernels (paged.hip, paged_mx4.h) share on the device.
#pragma once

#include "mx4_device.h"
#include "paged.h"
#include "paged_split.h"

namespace iefwd {

// One call of the attention.
struct AttnArgs {
    PagedCache c;
    const bf16_t *q;
    int64_t q_stride;
    const int32_t *table;
    const int32_t *lens;
    bf16_t *ctx;
    float *part_o;       // [batch, heads, slots, head_dim]
    float *part_ml;      // [batch, heads, slots, 2]
    int table_stride, batch, heads, max_keys, slots;
    PagedSplit split;
    float scale_log2e;
    float cap_log2e, cap_inv;      // cap * log2(e) and its inverse; 0: no cap
    const float *slopes;           // [heads] or null
};

namespace {

__device__ inline float bf16_of(uint32_t w, int half) { return __uint_as_float(half ? w & 0xffff0000u : w << 16); }

// Inclusive scan over the wave's lanes: row shifts by 1, 2, 4, 8, then lane 15's row
// result to the next row and lane 31's to the upper half.  0 is neutral to `add`.
template <class T, class Add>
__device__ inline T wave_scan(T v, Add add) {
    v = add(v, (T)__builtin_amdgcn_update_dpp(0, (int)v, 0x111, 0xf, 0xf, false));
    v = add(v, (T)__builtin_amdgcn_update_dpp(0, (int)v, 0x112, 0xf, 0xf, false));
    v = add(v, (T)__builtin_amdgcn_update_dpp(0, (int)v, 0x114, 0xf, 0xf, false));
    v = add(v, (T)__builtin_amdgcn_update_dpp(0, (int)v, 0x118, 0xf, 0xf, false));
    v = add(v, (T)__builtin_amdgcn_update_dpp(0, (int)v, 0x142, 0xa, 0xf, false));
    v = add(v, (T)__builtin_amdgcn_update_dpp(0, (int)v, 0x143, 0xc, 0xf, false));
    return v;
}

// The lane, hidden from the compiler: what is computed from it inside the loop over
// items stays there instead of being held in registers through it (153 -> 140 VGPRs).
__device__ inline int opaque_lane() {
    int lane = threadIdx.x & 63;
    asm volatile("" : "+v"(lane));
    return lane;
}

struct AttnItem {
    int b, part, keys;
};

// The item-th (request, part) of the batch, requests in order; false past the last.
// Every wave finds it by itself from the lengths, 64 requests at a time.  A request
// without keys has one part, which writes its zeros.
__device__ inline bool find_item(const AttnArgs &a, int item, int &b0, int &before, AttnItem &out) {
    const int lane = opaque_lane();
    for (; b0 < a.batch; b0 += 64) {
        const bool in = b0 + lane < a.batch;
        const int n = in ? min(max(a.lens[b0 + lane], 0), a.max_keys) : 0;
        const int parts = in ? paged_parts(n, a.split) : 0;
        const int to = before + wave_scan(parts, [](int x, int y) { return x + y; });
        const int total = __builtin_amdgcn_readlane(to, 63);
        if (item < total) {
            const int src = __builtin_ctzll(__ballot(to > item));
            out.b = __builtin_amdgcn_readfirstlane(b0 + src);
            out.part = __builtin_amdgcn_readfirstlane(item - __builtin_amdgcn_readlane(to, src) +
                                                      __builtin_amdgcn_readlane(parts, src));
            out.keys = __builtin_amdgcn_readlane(n, src);
            return true;
        }
        before = total;
    }
    return false;
}

// v of lanes l, l ^ 16, l ^ 32 and l ^ 48 together: each swap leaves a row's (half's) value
// in one result and its neighbour's in the other.
__device__ inline float across_rows_max(float v) {
    const uint32_t x = __float_as_uint(v);
    const auto a = __builtin_amdgcn_permlane16_swap(x, x, false, false);
    const uint32_t y = __float_as_uint(fmaxf(__uint_as_float(a[0]), __uint_as_float(a[1])));
    const auto b = __builtin_amdgcn_permlane32_swap(y, y, false, false);
    return fmaxf(__uint_as_float(b[0]), __uint_as_float(b[1]));
}

__device__ inline float across_rows_sum(float v) {
    const uint32_t x = __float_as_uint(v);
    const auto a = __builtin_amdgcn_permlane16_swap(x, x, false, false);
    const uint32_t y = __float_as_uint(__uint_as_float(a[0]) + __uint_as_float(a[1]));
    const auto b = __builtin_amdgcn_permlane32_swap(y, y, false, false);
    return __uint_as_float(b[0]) + __uint_as_float(b[1]);
}

// A page of one head as a buffer: its base in scalar registers, so that a load needs one
// 32-bit offset a lane.
__device__ inline __amdgpu_buffer_rsrc_t page_buffer(const char *base, size_t at, uint32_t bytes) {
    const uint32_t lo = __builtin_amdgcn_readfirstlane((uint32_t)at), hi = __builtin_amdgcn_readfirstlane((uint32_t)(at >> 32));
    return __builtin_amdgcn_make_buffer_rsrc(const_cast<char *>(base + ((uint64_t)hi << 32 | lo)), 0, bytes, 0x00027000);
}

// cap tanh(s / cap) of a score s in powers of two: tanh(x) = 1 - 2 / (e^2x + 1), good to 2^-22 of the cap, which up to 64 is less
// than what the probabilities are kept to; beyond, small scores by the power series of tanh, good to 2^-20 of their value.
__device__ inline float capped(const AttnArgs &a, float s) {
    const float x = s * a.cap_inv;
    float t = fmaf(-2.f, __builtin_amdgcn_rcpf(__builtin_amdgcn_exp2f(x * (2.f * kLog2e)) + 1.f), 1.f);
    if (a.cap_log2e > 64.f * kLog2e) {
        const float y = x * x;
        float series = fmaf(y, 62.f / 2835.f, -17.f / 315.f);
        series = fmaf(y, series, 2.f / 15.f);
        series = fmaf(y, series, -1.f / 3.f);
        series = fmaf(x * y, series, x);
        t = fabsf(x) < 0.25f ? series : t;
    }
    return a.cap_log2e * t;
}

// A head's slope in powers of two.  From 2^96 on one step of the distance is more than scores differ by, and up to there no product
// with a distance leaves fp32's range.
__device__ inline float slope_log2e(float slope) {
    return __builtin_elementwise_minimum(__builtin_elementwise_maximum(slope * kLog2e, -0x1p96f), 0x1p96f);
}

// The score s less the slope times the distance, which counts from the end that the slope favours: from the newest key, of a negative slope
// from the first, whose scores are all lower by the same.  The product's rounding is then small where the probabilities are
// large (from the other end a slope of -1 over 2^20 keys had them off by some 4%).
__device__ inline float lowered(float s, float slope, int key, int newest) {
    return fmaf(-fabsf(slope), (float)(slope < 0.f ? key : newest - key), s);
}

}  // namespace
}  // namespace iefwd
