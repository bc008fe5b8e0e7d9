// A paged cache in microscaled 4 bits for gfx950: new tokens, attention of one query per request, and tokens of
// every kind of cache read back.  Part of paged.hip.
#pragma once

#include <algorithm>

#include "paged_device.h"

namespace iefwd {
namespace {

constexpr int kTileThreads = 256;

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
// Bound by its bytes for prompts: 24001 tokens of 8 x 128 are written in 26.5 us (4.7 TB/s) and 26000 read back in 21.6 (6.2; with lanes
// in the order of the pages' pieces a tenth more); 48 tokens take 2.6 us either way, a launch and two loads in a row.
template <int DH>
struct Tile {
    static constexpr int EIGHTHS = DH / 8, TOKENS = kTileThreads / EIGHTHS;
    int token, head, eighth;

    __device__ Tile(int kv_heads) {
        const int tile = blockIdx.x / kv_heads;
        head = blockIdx.x - tile * kv_heads;
        token = tile * TOKENS + threadIdx.x / EIGHTHS;
        eighth = threadIdx.x % EIGHTHS;
    }
};

template <int DH, bool FAR>
__global__ __launch_bounds__(kTileThreads) void paged_append_mx4_kernel(PagedCache c, const bf16_t *__restrict__ k,
                                                                    const bf16_t *__restrict__ v,
                                                                    const int64_t *__restrict__ slots, int tokens,
                                                                    int64_t k_stride, int64_t v_stride) {
    const Tile<DH> at(c.kv_heads);
    const int page = 1 << c.page_log2;
    if (at.token >= tokens) return;      // whole quads
    const int64_t slot = slots[at.token];
    const int col = at.head * DH + 8 * at.eighth;
    Eight x[2] = {};
    const u32x4 *kp = reinterpret_cast<const u32x4 *>(k + at.token * k_stride + col);
    const u32x4 *vp = reinterpret_cast<const u32x4 *>(v + at.token * v_stride + col);
    x[0].lo = FAR ? __builtin_nontemporal_load(kp) : *kp;
    x[1].lo = FAR ? __builtin_nontemporal_load(vp) : *vp;
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

// 8 columns of K (of V) of a place as bf16.  V of the 16- and 8-bit caches comes in single elements, which lie 4 apart: 26000 tokens of
// 8 x 128 are read back in 58 and 55 us (3.7 and 2.9 TB/s), in 80 and 55 where the slots are in any order; 4-bit ones in 20 and 22.
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

template <int DH, KvKind KIND, bool FAR>
__global__ __launch_bounds__(kTileThreads) void paged_read_kernel(PagedCache c, const int64_t *__restrict__ slots,
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
    u32x4 *kp = reinterpret_cast<u32x4 *>(k + at.token * k_stride + col), *vp = reinterpret_cast<u32x4 *>(v + at.token * v_stride + col);
    if (FAR) {
        __builtin_nontemporal_store(x[0], kp);
        __builtin_nontemporal_store(x[1], vp);
    } else {
        *kp = x[0];
        *vp = x[1];
    }
}

// ------------------------------------------------------------------------------ attention
//
// As over the other caches (paged.hip): a workgroup takes one part of one request's keys for one key-value head and up to HC of its
// query heads, its waves steps of 64 keys in turn, and what they have is joined through LDS, parts by a second kernel.
//
// S = Q K^T goes to the matrix cores with the stored codes and scales as an operand (4 bits by 8), the heads as rows and 16 keys as
// columns.  Row i is head i % HC, so that lane (r, c) gets the scores of key r and heads 4 c .. 4 c + 3 (mod HC) of every tile of 16
// keys; of 16 / HC tiles each lane keeps one by its c, and no score is worked on twice: with 4 heads a lane has 4 of the 64 x 4
// scores of a step.  The probabilities go through 1 KB of LDS to the lanes that need them as an operand of O^T = V^T P^T, as bf16 and its
// bf16 rest (see paged.hip).  V becomes bf16 on the way, by v_cvt_scalef32_pk_bf16_fp4 under the scale as it is stored.
//
// 64 requests of 4000 to 8192 keys, 32 / 8 heads of 128, 408 MB, take 87 us with capped scores (4.7 TB/s, 51% of the issue slots) and
// 4.3 to 5.2 for the joining; calls from a graph 93, with slopes as well 96, with neither 88; 56 / 8 heads 110, 115 and 92.  Neither the
// memory nor the issue is full: a step waits for its own pages, with nothing of the next one on its way.  One request of 300 keys
// takes 6.7, a chain of loads (length, table, page) and the joining of 8 waves.  Not kept: every lane working on all scores of its
// heads (103 and 115 us); steps of 32 keys; the next step's loads asked for ahead, or the first one's before q is converted, whose
// registers spill (137 us uncapped) or halve the waves.  (Copies of the next step straight to LDS, which take no registers, have not
// been tried.)
//
// The reference of the exponents need not be the largest score: it is raised, and sums and context scaled down, when a score
// exceeds it by 2^8, which in a row of many keys is rare; probabilities up to 2^8 are as exact as those up to 1.
// A head's query for the product with 4-bit keys: q = hi + lo in e4m3 (4 bits of significance each), under scales per 32 columns
// that bring the block's largest to 128 .. 256 and let lo have 2^-4 of hi's.  bf16 has 8 bits: hi and lo are exact down to 2^-13
// of the block's largest and off by 2^-21 of it below.  Lane (r, c) holds columns 16 c to 16 c + 15 and 64 + 16 c
// to 64 + 16 c + 15 of head r, and the scale of block c.  A block with an infinity or a NaN becomes NaN.
struct Q8 {
    i32x8 hi, lo;
    int hi_scale, lo_scale;
};

template <int DH>
struct Q16 {      // the lane's columns as they are
    u32x4 w[DH / 64][2];
    __device__ Q16(const bf16_t *qh, int c) {
#pragma unroll
        for (int h = 0; h < DH / 64; ++h)
#pragma unroll
            for (int i = 0; i < 2; ++i) w[h][i] = *reinterpret_cast<const u32x4 *>(qh + 64 * h + 16 * c + 8 * i);
    }
};

template <int DH>
__device__ inline Q8 q8_operand(const Q16<DH> &q16, int r, int c) {
    Q8 q{};
    int scale[2] = {127, 127};      // of the blocks that the lane's two pieces lie in
#pragma unroll
    for (int h = 0; h < DH / 64; ++h) {
        const u32x4 (&w)[2] = q16.w[h];
        uint32_t top = 0;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const uint32_t x = w[i / 4][i % 4] & 0x7fff7fffu;
            top = max(top, max(x & 0xffffu, x >> 16));
        }
        const auto both = __builtin_amdgcn_permlane16_swap(top, top, false, false);      // a block is two lanes' pieces, l and l ^ 16
        const int field = (int)(max(both[0], both[1]) >> 7);
        scale[h] = field == 255 ? 255 : max(field - 7, 4);
        const float unit = __uint_as_float((uint32_t)(254 - min(scale[h], 250)) << 23);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            float x[4], hi[4];
#pragma unroll
            for (int e = 0; e < 4; ++e) x[e] = bf16_of(w[i / 2][2 * (i % 2) + e / 2], e % 2) * unit;
            int b = __builtin_amdgcn_cvt_pk_fp8_f32(x[0], x[1], 0, false);
            b = __builtin_amdgcn_cvt_pk_fp8_f32(x[2], x[3], b, true);
            const f32x2 back[2] = {__builtin_amdgcn_cvt_pk_f32_fp8(b, false), __builtin_amdgcn_cvt_pk_f32_fp8(b, true)};
#pragma unroll
            for (int e = 0; e < 4; ++e) hi[e] = back[e / 2][e % 2];
            int l = __builtin_amdgcn_cvt_pk_fp8_f32((x[0] - hi[0]) * 16.f, (x[1] - hi[1]) * 16.f, 0, false);
            l = __builtin_amdgcn_cvt_pk_fp8_f32((x[2] - hi[2]) * 16.f, (x[3] - hi[3]) * 16.f, l, true);
            q.hi[4 * h + i] = b;
            q.lo[4 * h + i] = l;
        }
    }
    // block c of 64 columns' two is that of the pieces of lanes 2 c and 2 c + 1
    const int from = r + 32 * (c & 1);
    const int first = __shfl(scale[0], from), second = __shfl(scale[1], from);
    q.hi_scale = c < 2 ? first : second;
    q.lo_scale = q.hi_scale == 255 ? 255 : q.hi_scale - 4;
    return q;
}

// Columns 2 m and 2 m + 1 of the lane's W of token e of a quad, as bf16.  The conversion reads of its scale the exponent field alone,
// whatever the other bits: a shift puts the token's byte there.
template <int W>
__device__ inline uint32_t v_pair(uint32_t codes, uint32_t scales, int e, int m, int r) {
    const float s = __uint_as_float(e == 3 ? scales >> 1 : scales << (23 - 8 * e));
    if (W == 4) codes >>= 16 * (r & 1);
    const bf16x2 x = m == 0   ? __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, s, 0)
                     : m == 1 ? __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, s, 1)
                     : m == 2 ? __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, s, 2)
                              : __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, s, 3);
    return __builtin_bit_cast(uint32_t, x);
}

// max and sum over the 16 lanes of a row, in each of them.
__device__ inline float row_max(float v) {
    v = fmaxf(v, __uint_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(v), 0x121, 0xf, 0xf, true)));
    v = fmaxf(v, __uint_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(v), 0x122, 0xf, 0xf, true)));
    v = fmaxf(v, __uint_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(v), 0x124, 0xf, 0xf, true)));
    return fmaxf(v, __uint_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(v), 0x128, 0xf, 0xf, true)));
}
__device__ inline float row_sum(float v) {
    v += __uint_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(v), 0x121, 0xf, 0xf, true));
    v += __uint_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(v), 0x122, 0xf, 0xf, true));
    v += __uint_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(v), 0x124, 0xf, 0xf, true));
    return v + __uint_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(v), 0x128, 0xf, 0xf, true));
}
// and over the rows that have the same heads: all (4 heads), c and c ^ 2 (8), the row itself (16).
template <int HC>
__device__ inline float same_heads_max(float v) {
    v = row_max(v);
    if (HC == 4) return across_rows_max(v);
    if (HC == 8) {
        const auto b = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
        return fmaxf(__uint_as_float(b[0]), __uint_as_float(b[1]));
    }
    return v;
}
template <int HC>
__device__ inline float same_heads_sum(float v) {
    v = row_sum(v);
    if (HC == 4) return across_rows_sum(v);
    if (HC == 8) {
        const auto b = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
        return __uint_as_float(b[0]) + __uint_as_float(b[1]);
    }
    return v;
}

// HC: 4, 8 or 16 heads at most.  STREAM, SCORED: as in paged.hip.  128 registers for 4 waves a SIMD; the 16 scores a lane that 16 heads
// come to need more.
template <int DH, int HC, int WAVES, bool STREAM, bool SCORED>
__global__ __launch_bounds__(64 * WAVES, HC < 16 ? 4 : WAVES == 8 ? 2 : 3) void paged_attention_mx4_kernel(AttnArgs a) {
    constexpr int T = 4, TPV = 16 / HC, SETS = T / TPV;      // tiles of a step, tiles of a set of scores that a lane keeps one of, sets
    constexpr int W = DH / 16;                               // columns of V that a lane takes
    constexpr int ROW = DH + 4;
    __shared__ __attribute__((aligned(16))) float o_lds[WAVES][HC][ROW];
    __shared__ float m_lds[WAVES][HC], l_lds[WAVES][HC];
    static_assert(ROW > 16 * T, "a wave's probabilities lie where its context will");
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int r = lane & 15, c = lane >> 4;
    const int group = a.heads / a.c.kv_heads, tiles = (group + 15) / 16;
    // the heads of one item next to each other: their parts of a page are neighbours in memory
    const int rows = a.c.kv_heads * tiles, step = gridDim.x / rows;
    const int item0 = blockIdx.x / rows, row = blockIdx.x - item0 * rows;
    const int kvh = row / tiles, tile = row - kvh * tiles;
    const int head0 = kvh * group + tile * 16, n_heads = min(HC, group - tile * 16);
    const int page = 1 << a.c.page_log2;
    const uint32_t page_bytes = page * (DH / 32 * 17), codes = page * (DH / 2);
    const char *K = static_cast<const char *>(a.c.k), *V = static_cast<const char *>(a.c.v);
    // lane (r, c): columns 32 c and on of key r (heads of 64 have two such blocks: the others are read twice and dropped); of V the
    // tokens 4 c to 4 c + 3 and columns W r and on, for heads of 64 half of a load
    const int k_block = DH == 64 ? c & 1 : c;
    const uint32_t k_lane = (k_block * page + r) * 16, ks_lane = codes + k_block * page + r;
    const uint32_t v_lane = (c * (DH / 8) + r * W / 8) * 16, vs_lane = codes + (c * (DH / 32) + r * W / 32) * 4;
    uint32_t (*p_lds)[ROW] = reinterpret_cast<uint32_t (*)[ROW]>(o_lds[wave]);      // [head][key of the step]
    const int own_heads = 4 * (c % (HC / 4)), own_tile = c / (HC / 4);      // of its scores: heads from, tile of the set

    int b0 = 0, before = 0;
    AttnItem it;
    for (int item = item0; find_item(a, item, b0, before, it); item += step) {
        const int part_log2 = paged_part_log2(it.keys, a.split);
        const int k0 = it.part << part_log2, k1 = min(it.keys, k0 + (1 << part_log2));
        const int32_t *ids = a.table + (size_t)it.b * a.table_stride;
        const Q16<DH> q16(a.q + (int64_t)it.b * a.q_stride + (head0 + min(r % HC, n_heads - 1)) * DH, c);
        // the heads' slopes wait behind the wave's probabilities: in four registers they made more of the others spill, also where there is
        // but a cap (2 to 3 registers do now, with 5 to 8 heads of 128 eight)
        if constexpr (SCORED) {
            if (a.slopes && lane < HC) p_lds[lane][16 * T] = __float_as_uint(slope_log2e(a.slopes[head0 + min(lane, n_heads - 1)]));
            wave_lds_fence();
        }
        float m[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY}, l[4] = {0.f, 0.f, 0.f, 0.f};      // of its scores' heads
        f32x4 o[W] = {};                                                                            // of head r % HC
        const int steps = (k1 - k0 + 16 * T - 1) / (16 * T), own = (steps - wave + WAVES - 1) / WAVES;      // this wave's
        // lane 4 (i % 16) + t: the page of tile t of this wave's i-th step
        auto load_pages = [&](int i0) {
            const int key = k0 + (wave + WAVES * (i0 + (lane >> 2))) * 16 * T + (lane & 3) * 16;
            int id = key < k1 ? ids[key >> a.c.page_log2] : -1;
            return id >= a.c.n_pages ? -1 : id;
        };
        int pages = own > 0 ? load_pages(0) : -1, more = -1;      // those of the next 16 steps
        auto key_of = [&](int i, int t) { return k0 + (wave + WAVES * i) * 16 * T + 16 * t; };
        u32x4 kr[T], vr[T];
        uint32_t ks[T], vs[T];
        auto load_k = [&](int i) {
#pragma unroll
            for (int t = 0; t < T; ++t) {
                const int id = __builtin_amdgcn_readlane(pages, 4 * (i & 15) + t), off = key_of(i, t) & (page - 1);
                const __amdgpu_buffer_rsrc_t kp = page_buffer(K, ((size_t)max(id, 0) * a.c.kv_heads + kvh) * page_bytes, page_bytes);
                kr[t] = __builtin_amdgcn_raw_buffer_load_b128(kp, k_lane, off * 16, STREAM ? 2 : 0);
                ks[t] = (uint8_t)__builtin_amdgcn_raw_buffer_load_b8(kp, ks_lane, off, STREAM ? 2 : 0);
            }
        };
        auto load_v = [&](int i) {
#pragma unroll
            for (int t = 0; t < T; ++t) {
                const int id = __builtin_amdgcn_readlane(pages, 4 * (i & 15) + t), off = key_of(i, t) & (page - 1);
                const __amdgpu_buffer_rsrc_t vp = page_buffer(V, ((size_t)max(id, 0) * a.c.kv_heads + kvh) * page_bytes, page_bytes);
                vr[t] = __builtin_amdgcn_raw_buffer_load_b128(vp, v_lane, off * (DH / 2), STREAM ? 2 : 0);
                vs[t] = __builtin_amdgcn_raw_buffer_load_b32(vp, vs_lane, off * (DH / 32), STREAM ? 2 : 0);
            }
        };
        // keys of each tile of a step that take part
        auto limits = [&](int i, int (&limit)[T]) {
            int least = 16;
#pragma unroll
            for (int t = 0; t < T; ++t) {
                limit[t] = __builtin_amdgcn_readlane(pages, 4 * (i & 15) + t) < 0 ? 0 : min(16, k1 - key_of(i, t));
                least = min(least, limit[t]);
            }
            return least;
        };
        const Q8 q8 = q8_operand<DH>(q16, r, c);
        for (int i = 0; i < own; ++i) {
            const int key0 = key_of(i, 0);
            if (i > 0 && (i & 15) == 0) pages = more;
            load_k(i);
            load_v(i);
            int limit[T];
            const int least = limits(i, limit);
            if ((i & 15) == 8 && i + 8 < own) more = load_pages((i & ~15) + 16);
            float p[SETS][4];
            bool above = false;
#pragma unroll
            for (int s = 0; s < SETS; ++s) {
                f32x4 z = {0.f, 0.f, 0.f, 0.f};
                int tile_of = 0, keys = 0;
#pragma unroll
                for (int u = 0; u < TPV; ++u) {
                    const int t = s * TPV + u;
                    const bool there = DH == 128 || c < 2;
                    const i32x8 x = {there ? (int)kr[t][0] : 0, there ? (int)kr[t][1] : 0, there ? (int)kr[t][2] : 0,
                                     there ? (int)kr[t][3] : 0, 0, 0, 0, 0};
                    const int x_scale = there ? (int)ks[t] : 127;
                    f32x4 d = {0.f, 0.f, 0.f, 0.f};
                    d = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(q8.lo, x, d, 0, 4, 0, q8.lo_scale, 0, x_scale);
                    d = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(q8.hi, x, d, 0, 4, 0, q8.hi_scale, 0, x_scale);
                    if (u == 0 || own_tile == u) {
                        z = d;
                        tile_of = t;
                        keys = limit[t];
                    }
                }
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    float y = z[e] * a.scale_log2e;
                    if constexpr (SCORED) {
                        if (a.cap_log2e != 0.f) y = capped(a, y);
                        if (a.slopes) y = lowered(y, __uint_as_float(p_lds[own_heads + e][16 * T]), key0 + 16 * tile_of + r, it.keys - 1);
                    }
                    if (least < 16 && r >= keys) y = -INFINITY;
                    p[s][e] = y;
                    above |= y > m[e] + 8.f;
                }
            }
            if (__any(above)) {
                float f[4];
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    float top = p[0][e];
#pragma unroll
                    for (int s = 1; s < SETS; ++s) top = fmaxf(top, p[s][e]);
                    top = fmaxf(m[e], same_heads_max<HC>(top));
                    f[e] = __builtin_amdgcn_exp2f(m[e] - (top == -INFINITY ? 0.f : top));
                    l[e] *= f[e];
                    m[e] = top;
                }
                // the factor of head h = r % HC is element h % 4 of the lanes whose heads begin at h - h % 4
                const int from = r % HC / 4 * 16;
                const float f0 = __shfl(f[0], from), f1 = __shfl(f[1], from), f2 = __shfl(f[2], from), f3 = __shfl(f[3], from);
                const float mine = r & 2 ? (r & 1 ? f3 : f2) : (r & 1 ? f1 : f0);
#pragma unroll
                for (int w = 0; w < W; ++w) o[w] *= mine;
            }
#pragma unroll
            for (int s = 0; s < SETS; ++s)
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    // nothing but -inf so far: any finite reference gives p = 0
                    const float x = __builtin_amdgcn_exp2f(p[s][e] - (m[e] == -INFINITY ? 0.f : m[e]));
                    l[e] += x;
                    const uint32_t hi = __float_as_uint(x) & 0xffff0000u;
                    const uint32_t lo = f32_to_bf16(fmaf(x, 1.f + 0x1p-22f, -__uint_as_float(hi)));
                    p_lds[own_heads + e][16 * (s * TPV + own_tile) + r] = hi | lo;
                }
            wave_lds_fence();
            // places past the last key hold any bits: any codes are finite under a finite scale
            if (least < 16)
#pragma unroll
                for (int t = 0; t < T; ++t) {
                    const int n = min(max(limit[t] - 4 * c, 0), 4);
                    vs[t] &= n == 4 ? 0xffffffffu : (1u << (8 * n)) - 1u;
                }
#pragma unroll
            for (int g = 0; g < T / 2; ++g) {
                const u32x4 pa = *reinterpret_cast<const u32x4 *>(&p_lds[r % HC][32 * g + 4 * c]);
                const u32x4 pb = *reinterpret_cast<const u32x4 *>(&p_lds[r % HC][32 * g + 16 + 4 * c]);
                auto halves = [&](uint32_t pick) {
                    return __builtin_bit_cast(
                        bf16x8, u32x4{__builtin_amdgcn_perm(pa[1], pa[0], pick), __builtin_amdgcn_perm(pa[3], pa[2], pick),
                                      __builtin_amdgcn_perm(pb[1], pb[0], pick), __builtin_amdgcn_perm(pb[3], pb[2], pick)});
                };
                const bf16x8 p_hi = halves(0x07060302u), p_lo = halves(0x05040100u);
                // a byte holds two columns of one token: the pairs of tokens that the operand wants come of two bytes
#pragma unroll
                for (int j = 0; j < W / 2; ++j) {
                    uint32_t lo_col[4], hi_col[4];
#pragma unroll
                    for (int t = 0; t < 2; ++t)
#pragma unroll
                        for (int e = 0; e < 2; ++e) {
                            const uint32_t x = v_pair<W>(vr[2 * g + t][2 * e], vs[2 * g + t], 2 * e, j, r);
                            const uint32_t y = v_pair<W>(vr[2 * g + t][2 * e + 1], vs[2 * g + t], 2 * e + 1, j, r);
                            lo_col[2 * t + e] = __builtin_amdgcn_perm(y, x, 0x05040100u);
                            hi_col[2 * t + e] = __builtin_amdgcn_perm(y, x, 0x07060302u);
                        }
                    const bf16x8 x0 = __builtin_bit_cast(bf16x8, u32x4{lo_col[0], lo_col[1], lo_col[2], lo_col[3]});
                    const bf16x8 x1 = __builtin_bit_cast(bf16x8, u32x4{hi_col[0], hi_col[1], hi_col[2], hi_col[3]});
                    o[2 * j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(x0, p_hi, o[2 * j], 0, 0, 0);
                    o[2 * j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(x0, p_lo, o[2 * j], 0, 0, 0);
                    o[2 * j + 1] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(x1, p_hi, o[2 * j + 1], 0, 0, 0);
                    o[2 * j + 1] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(x1, p_lo, o[2 * j + 1], 0, 0, 0);
                }
            }
            wave_lds_fence();
        }
        // join the waves.  Lane (r, c) holds of head r % HC the columns W (4 c + e) + w
#pragma unroll
        for (int e = 0; e < 4; ++e) l[e] = same_heads_sum<HC>(l[e]);
        const int late = opaque_lane(), head = late & 15, quad = late >> 4;
        if (head == 0 && own_tile == 0) {
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                m_lds[wave][own_heads + e] = m[e];
                l_lds[wave][own_heads + e] = l[e];
            }
        }
        if (head < n_heads) {
            float *dst = &o_lds[wave][head][4 * W * quad];
            float flat[4 * W];
#pragma unroll
            for (int e = 0; e < 4; ++e)
#pragma unroll
                for (int w = 0; w < W; ++w) flat[W * e + w] = o[w][e];
#pragma unroll
            for (int e = 0; e < W; ++e)
                *reinterpret_cast<f32x4 *>(dst + 4 * e) = f32x4{flat[4 * e], flat[4 * e + 1], flat[4 * e + 2], flat[4 * e + 3]};
        }
        __syncthreads();
        const bool whole = it.keys <= 1 << part_log2;
        for (int i = wave * 64 + late; i < n_heads * (DH / 4); i += 64 * WAVES) {
            const int h = i / (DH / 4), d = (i - h * (DH / 4)) * 4;
            float top = m_lds[0][h];
#pragma unroll
            for (int w = 1; w < WAVES; ++w) top = fmaxf(top, m_lds[w][h]);
            const float ref = top == -INFINITY ? 0.f : top;
            float sum = 0.f;
            f32x4 acc = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int w = 0; w < WAVES; ++w) {
                const float f = __builtin_amdgcn_exp2f(m_lds[w][h] - ref);
                sum += f * l_lds[w][h];
                acc += f * *reinterpret_cast<const f32x4 *>(&o_lds[w][h][d]);
            }
            const size_t bh = (size_t)it.b * a.heads + head0 + h;
            if (whole) {
                const float inv = sum == 0.f ? 0.f : 1.f / sum;     // nothing to attend to: zeros
                *reinterpret_cast<u32x2 *>(a.ctx + bh * DH + d) =
                    u32x2{pack2(acc[0] * inv, acc[1] * inv), pack2(acc[2] * inv, acc[3] * inv)};
            } else {
                const size_t slot = bh * a.slots + it.part;
                *reinterpret_cast<f32x4 *>(a.part_o + slot * DH + d) = acc;
                if (d == 0) *reinterpret_cast<f32x2 *>(a.part_ml + 2 * slot) = f32x2{top, sum};
            }
        }
        __syncthreads();
    }
}

template <int DH, int HC, int WAVES>
hipError_t launch_mx4_w(const AttnArgs &a, bool stream_pages, dim3 grid, hipStream_t stream) {
    auto launch = [&](auto kernel) { return launch_kernel(kernel, grid, dim3(64 * WAVES), stream, a); };
    if (a.cap_log2e != 0.f || a.slopes)
        return stream_pages ? launch(paged_attention_mx4_kernel<DH, HC, WAVES, true, true>)
                            : launch(paged_attention_mx4_kernel<DH, HC, WAVES, false, true>);
    return stream_pages ? launch(paged_attention_mx4_kernel<DH, HC, WAVES, true, false>)
                        : launch(paged_attention_mx4_kernel<DH, HC, WAVES, false, false>);
}

template <int DH, int WAVES>
hipError_t launch_mx4_heads(const AttnArgs &a, bool stream_pages, dim3 grid, hipStream_t stream) {
    const int group = a.heads / a.c.kv_heads;
    return group <= 4   ? launch_mx4_w<DH, 4, WAVES>(a, stream_pages, grid, stream)
           : group <= 8 ? launch_mx4_w<DH, 8, WAVES>(a, stream_pages, grid, stream)
                        : launch_mx4_w<DH, 16, WAVES>(a, stream_pages, grid, stream);
}

// launch(grid, first token, tokens), in one go but for the very most tokens: a grid holds less than 2^32 threads.
template <class Launch>
hipError_t in_grids(const PagedCache &c, int tokens, Launch launch) {
    const int per_tile = kTileThreads / (c.head_dim / 8), most = (1 << 23) / c.kv_heads * per_tile;
    hipError_t e = hipSuccess;
    for (int64_t at = 0; at < tokens && e == hipSuccess; at += most) {
        const int n = (int)std::min<int64_t>(most, tokens - at);
        e = launch(dim3((unsigned)((n + per_tile - 1) / per_tile * c.kv_heads)), at, n);
    }
    return e;
}

// Of the tokens' keys and values in bf16.  From 64 MiB on new ones are read, from 32 MiB on read ones written past the last cache:
// append and read of tokens of 8 x 128, us, without a hint / stores / both:
//   2000  7.7  7.4  7.0     4000 10.9  9.8  9.8     8000 18.7 16.8 17.9     16000 41.2 33.3 33.7     24001 and 26000 62.2 53.3 49.4
int64_t bytes_of(const PagedCache &c, int tokens) { return (int64_t)tokens * c.kv_heads * c.head_dim * 4; }

template <KvKind KIND>
hipError_t launch_read(const PagedCache &c, const int64_t *slots, bf16_t *k, bf16_t *v, int tokens, int64_t k_stride,
                       int64_t v_stride, hipStream_t stream) {
    auto launch = [&](auto kernel) {
        return in_grids(c, tokens, [&](dim3 grid, int64_t at, int n) {
            return launch_kernel(kernel, grid, dim3(kTileThreads), stream, c, slots + at, k + at * k_stride, v + at * v_stride, n, k_stride,
                                 v_stride);
        });
    };
    const bool far = bytes_of(c, tokens) >= 32 << 20;
    if (c.head_dim == 64) return far ? launch(paged_read_kernel<64, KIND, true>) : launch(paged_read_kernel<64, KIND, false>);
    return far ? launch(paged_read_kernel<128, KIND, true>) : launch(paged_read_kernel<128, KIND, false>);
}

}  // namespace

// Up to the joining of parts.
hipError_t launch_attention_mx4(const AttnArgs &a, bool stream_pages, dim3 grid, hipStream_t stream) {
    const bool narrow = a.c.head_dim == 64;
    switch (a.split.waves) {
    case 8:
        return narrow ? launch_mx4_heads<64, 8>(a, stream_pages, grid, stream)
                      : launch_mx4_heads<128, 8>(a, stream_pages, grid, stream);
    case 4:
        return narrow ? launch_mx4_heads<64, 4>(a, stream_pages, grid, stream)
                      : launch_mx4_heads<128, 4>(a, stream_pages, grid, stream);
    }
    return narrow ? launch_mx4_heads<64, 2>(a, stream_pages, grid, stream) : launch_mx4_heads<128, 2>(a, stream_pages, grid, stream);
}

hipError_t launch_paged_append_mx4(const PagedCache &c, const bf16_t *k, const bf16_t *v, const int64_t *slots, int tokens,
                                   int64_t k_stride, int64_t v_stride, hipStream_t stream) {
    auto launch = [&](auto kernel) {
        return in_grids(c, tokens, [&](dim3 grid, int64_t at, int n) {
            return launch_kernel(kernel, grid, dim3(kTileThreads), stream, c, k + at * k_stride, v + at * v_stride, slots + at, n, k_stride,
                                 v_stride);
        });
    };
    const bool far = bytes_of(c, tokens) >= 64 << 20;
    if (c.head_dim == 64) return far ? launch(paged_append_mx4_kernel<64, true>) : launch(paged_append_mx4_kernel<64, false>);
    return far ? launch(paged_append_mx4_kernel<128, true>) : launch(paged_append_mx4_kernel<128, false>);
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
