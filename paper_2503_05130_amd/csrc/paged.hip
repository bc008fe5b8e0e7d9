// The paged key-value cache's kernels for gfx950: planning of pages and slots,
// appending new tokens, and attention of one query per request over pages.
#include "paged.h"

#include <algorithm>

#include "paged_mx4.h"

namespace iefwd {
namespace {

constexpr int kThreads = 256;
constexpr int kWaves = kThreads / 64;

// ------------------------------------------------------------------------------ plan
//
// For request b with o cached and n wanted tokens in pages of P: it holds
// ceil(o / P) pages and needs ceil(n / P).  Every workgroup makes the same
// prefix sums over the batch (new tokens, pages taken, pages given back) from
// the lengths, which it reads from L2; they say where each request's slots begin and
// which entries of the ring of free pages are its own.  The slots are then
// spread over the workgroups whatever request they belong to (a binary search
// in the sums finds it), so that one long prompt is as parallel as many short
// ones; the slot that opens a page also writes the table's entry.  One launch, no
// scratch, no atomics between workgroups: what one writes none reads.
//
// Bound by latency, a launch and four loads that depend on each other (lengths, LDS sums, ring or table entry): 4 requests 3.0 us,
// 512 of which 16 end 5.4, 192 prompts with 90000 slots 4.7.
//
// The sums saturate at 2^32 - 1, which is past everything they are compared with (below 2^31);
// saturating sums of such numbers are the same in any order.
constexpr int kPlanGiveBack = 16;      // requests a wave looks through for pages to give back

__device__ inline uint32_t add_sat(uint32_t a, uint32_t b) { return __builtin_elementwise_add_sat(a, b); }

struct PlanRequest {
    int held, want;
    uint32_t tokens;
    bool valid;
};

__device__ inline PlanRequest plan_request(const PlanArgs &p, int o, int n) {
    const int cap = p.max_pages << p.page_log2, up = (1 << p.page_log2) - 1;      // at most 2^30
    PlanRequest r{0, 0, 0, o >= 0 && n >= 0 && o <= cap && n <= cap};
    if (r.valid) {
        r.held = (o + up) >> p.page_log2;
        r.want = (n + up) >> p.page_log2;
        r.tokens = n > o ? n - o : 0;
    }
    return r;
}

__global__ __launch_bounds__(kThreads) void paged_plan_kernel(PlanArgs p) {
    __shared__ int ends[kPlanMaxBatch];      // new tokens up to and with request b, at most room
    __shared__ int at[kPlanMaxBatch];        // the request's first entry of the ring (taken from or given to), -1: refused
    __shared__ uint32_t wave_sum[2][kWaves][3];
    __shared__ int granted_total[2], refused_total;
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    int o = tid < p.batch ? p.lens[tid] : 0, n = tid < p.batch ? p.new_lens[tid] : 0;
    const int64_t head = p.counters[0], tail = p.counters[1];
    const bool sane = head >= 0 && tail >= head && tail - head <= p.ring_size;
    const uint32_t avail = sane ? (uint32_t)(tail - head) : 0, space = sane ? p.ring_size - avail : 0;
    const uint32_t head_at = sane ? (uint32_t)(head % p.ring_size) : 0, tail_at = sane ? (uint32_t)(tail % p.ring_size) : 0;
    if (tid < 2) granted_total[tid] = 0;
    if (tid == 2) refused_total = 0;

    // kThreads requests at a time; sum: of all before them
    uint32_t sum[3] = {0, 0, 0};
    for (int b0 = 0; b0 < p.batch; b0 += kThreads) {
        const int b = b0 + tid, next = b + kThreads;
        const PlanRequest r = plan_request(p, o, n);
        const int o_now = o, n_now = n;
        if (next < p.batch) {
            o = p.lens[next];
            n = p.new_lens[next];
        }
        const bool in = b < p.batch;
        const uint32_t take = in ? max(0, r.want - r.held) : 0, give = in ? max(0, r.held - r.want) : 0;
        const uint32_t mine[3] = {in ? r.tokens : 0, take, give};
        uint32_t to[3];
        uint32_t (*waves)[3] = wave_sum[(b0 / kThreads) & 1];      // the other half may still be read
#pragma unroll
        for (int i = 0; i < 3; ++i) {
            to[i] = wave_scan(mine[i], add_sat);
            if (lane == 63) waves[wave][i] = to[i];
        }
        __syncthreads();
#pragma unroll
        for (int i = 0; i < 3; ++i) {
            uint32_t below = sum[i];
#pragma unroll
            for (int w = 0; w < kWaves; ++w) {
                if (w == wave) to[i] = add_sat(below, to[i]);
                below = add_sat(below, waves[w][i]);
            }
            sum[i] = below;
        }
        const bool ok = in && r.valid && (take == 0 || to[1] <= avail) && (r.tokens == 0 || to[0] <= (uint32_t)p.room) &&
                        (give == 0 || to[2] <= space);
        if (in) {
            // where the request's own pages begin in the ring: a granted request's sums are at most the ring's size
            const int end = (int)min(to[0], (uint32_t)p.room);
            uint32_t place = give ? tail_at + (to[2] - give) : take ? head_at + (to[1] - take) : 0;
            if (place >= (uint32_t)p.ring_size) place -= p.ring_size;
            ends[b] = end;
            at[b] = ok ? (int)place : -1;
            if (blockIdx.x == 0) {
                p.lens_out[b] = ok ? n_now : o_now;
                p.starts[b + 1] = end;
                if (b == 0) p.starts[0] = 0;
            }
        }
        if (blockIdx.x == 0) {      // whole numbers in LDS: any order gives the same
            if (ok && take) atomicAdd(&granted_total[0], (int)take);
            if (ok && give) atomicAdd(&granted_total[1], (int)give);
            if (in && !ok) atomicAdd(&refused_total, 1);
        }
    }
    __syncthreads();
    if (blockIdx.x == 0 && tid == 0) {
        p.counters_out[0] = head + granted_total[0];
        p.counters_out[1] = tail + granted_total[1];
        *p.refused = refused_total;
    }

    // slots and the table's new entries
    const int page = 1 << p.page_log2, total = ends[p.batch - 1];
    for (int64_t i = (int64_t)blockIdx.x * kThreads + tid; i < p.room; i += (int64_t)gridDim.x * kThreads) {
        int64_t slot = -1;
        if (i < total) {
            int lo = 0, hi = p.batch - 1;            // the first request whose tokens end past i
            while (lo < hi) {
                const int mid = (lo + hi) >> 1;
                if (ends[mid] > i) hi = mid;
                else lo = mid + 1;
            }
            if (at[lo] >= 0) {
                const int cached = p.lens[lo], pos = cached + (int)(i - (lo ? ends[lo - 1] : 0));
                const int held = (cached + page - 1) >> p.page_log2, column = pos >> p.page_log2;
                int32_t *entry = p.table + (int64_t)lo * p.table_stride + column;
                int32_t id;
                if (column < held) {
                    id = *entry;
                } else {
                    const uint32_t place = (uint32_t)at[lo] + column - held;
                    id = p.ring[place >= (uint32_t)p.ring_size ? place - p.ring_size : place];
                    if ((pos & (page - 1)) == 0) *entry = id;
                }
                if (id >= 0 && id < p.ring_size) slot = ((int64_t)id << p.page_log2) + (pos & (page - 1));
            }
        }
        p.slots[i] = slot;
    }
    // pages given back: a wave finds them among some requests and copies them one request after the other
    for (int b0 = (blockIdx.x * kWaves + wave) * kPlanGiveBack; b0 < p.batch; b0 += gridDim.x * kWaves * kPlanGiveBack) {
        const int b = b0 + lane;
        const bool in = lane < kPlanGiveBack && b < p.batch;
        const PlanRequest r = plan_request(p, in ? p.lens[b] : 0, in ? p.new_lens[b] : 0);
        const int to = in && r.want < r.held ? at[b] : -1;
        for (uint64_t left = __ballot(to >= 0); left; left &= left - 1) {
            const int src = __builtin_ctzll(left);
            const int first = __builtin_amdgcn_readlane(r.want, src), count = __builtin_amdgcn_readlane(r.held, src) - first;
            const uint32_t begin = (uint32_t)__builtin_amdgcn_readlane(to, src);
            const int32_t *pages = p.table + (int64_t)(b0 + src) * p.table_stride + first;
            for (int j = lane; j < count; j += 64) {
                const uint32_t place = begin + j;
                p.ring[place >= (uint32_t)p.ring_size ? place - p.ring_size : place] = pages[j];
            }
        }
    }
}

// ------------------------------------------------------------------------------ append
//
// A workgroup copies `tile` following tokens of one key-value head.  K: a thread takes a
// 16-byte piece of one token; neighbouring threads take neighbouring tokens, whose pieces
// are neighbours in a page.  V holds 4 tokens of a column together, so a thread takes 16 bytes of
// such quads (2 or 4 columns) from 4 rows and writes them at once.  The quads are found from the slots: a unit is a
// run of tokens in following places of one quad, whole in the middle of a prompt, a single
// token in a decode step; one that is not whole is written element by element.
//
// Bound by its bytes for prompts: 24001 tokens of 8 x 128 in 8 bits 30 - 33 us, 16000 in bf16 22 - 28 us, by where the memory
// lies (4.5 - 4.9 and 4.7 - 5.9 TB/s of reads and writes; a copy of 4 GiB reaches 4.8, but a plain kernel that reads and writes
// the same amounts in a row and leaves them in the last cache in part takes 21 and 16 us).  Pages written by much are not read
// soon: from kAppendStream bytes on they are stored with the non-temporal hint (34.6 -> 32.6 us and 30.7 -> 23.4; but 12 MB
// 7.3 -> 7.5).  48 tokens of a decode step take 3.5 us, a launch and two loads in a row.
constexpr int kAppendTile = 32;      // most tokens of a workgroup
constexpr int64_t kAppendStream = 32 << 20;

// x / scale, rounded as a division is, within e4m3's range; NaN stays NaN.  `inv` is the
// rounded 1 / scale: one Newton step on the quotient by its remainder gives the correctly
// rounded one (Markstein, IBM J. Res. Dev. 34, 1990; checked for every scale's with every bf16's mantissa), in 3
// operations for the division's dozen.
// That holds where neither leaves fp32's range, which `near` says of the scale; then a quotient of 2^-11
// to 512 is exact so, a larger one is cut off and a smaller one is 0 in either form.
struct E4m3Scale {
    float scale, inv;
    bool near;
};

__device__ inline E4m3Scale e4m3_scale(float scale) {
    const float size = fabsf(scale);
    return {scale, 1.f / scale, size >= 0x1p-60f && size <= 0x1p60f};
}

__device__ inline float to_e4m3_range(float x, const E4m3Scale &s) {
    float y;
    if (s.near) {
        const float q = x * s.inv;
        y = fabsf(q) < 512.f ? fmaf(-fmaf(q, s.scale, -x), s.inv, q) : q;      // in this form -0 stays -0
    } else {
        y = x / s.scale;
    }
    return __builtin_elementwise_minimum(__builtin_elementwise_maximum(y, -448.f), 448.f);
}

// Two 32-bit words of bf16 pairs as 4 e4m3 values
__device__ inline uint32_t narrow(uint32_t a, uint32_t b, const E4m3Scale &scale) {
    const int w = __builtin_amdgcn_cvt_pk_fp8_f32(to_e4m3_range(bf16_of(a, 0), scale), to_e4m3_range(bf16_of(a, 1), scale), 0,
                                                  false);
    return __builtin_amdgcn_cvt_pk_fp8_f32(to_e4m3_range(bf16_of(b, 0), scale), to_e4m3_range(bf16_of(b, 1), scale), w, true);
}

// STREAM: pages are stored with the non-temporal hint.
template <bool E4M3, bool STREAM>
__global__ __launch_bounds__(kThreads) void paged_append_kernel(PagedCache c, const bf16_t *__restrict__ k,
                                                                const bf16_t *__restrict__ v,
                                                                const int64_t *__restrict__ slots, int tokens, int tile,
                                                                int64_t k_stride, int64_t v_stride) {
    constexpr int E = E4M3 ? 16 : 8, W = E4M3 ? 4 : 2;      // columns in 16 bytes of K and (of 4 tokens) of V
    __shared__ int64_t slot_of[kAppendTile];                // -1: outside the pool
    __shared__ int unit[kAppendTile];                       // first token in the tile, count << 8
    __shared__ int n_units;
    const int tid = threadIdx.x, dh = c.head_dim, page = 1 << c.page_log2;
    // the heads of a tile next to each other: their parts of a row are neighbours in memory
    const int64_t tile_at = blockIdx.x / c.kv_heads, t0 = tile_at * tile, limit = (int64_t)c.n_pages << c.page_log2;
    const int head = (int)(blockIdx.x - tile_at * c.kv_heads), n = (int)min((int64_t)tile, tokens - t0);
    if (tid < 64) {
        // lane 63: the slot before the tile; lanes up to tile + 2: the tile's and the three after it
        const int64_t i = tid == 63 ? t0 - 1 : t0 + tid;
        const int64_t s = i >= 0 && i < tokens && (tid < tile + 3 || tid == 63) ? slots[i] : -2;
        const bool in = tid < n && s >= 0 && s < limit;
        if (tid < tile) slot_of[tid] = in ? s : -1;
        // a token that follows its predecessor within a quad belongs to that one's unit, whatever tile it is in
        const int64_t before = __shfl(s, (tid + 63) & 63);
        const bool follows = (s & 3) != 0 && before == s - 1;
        const bool starts = in && !follows;
        const uint64_t chain = __ballot(s >= 0 && s < limit && follows) >> tid;      // bit j: token tid + j follows
        const int count = chain & 2 ? (chain & 4 ? (chain & 8 ? 4 : 3) : 2) : 1;
        const uint64_t all = __ballot(starts);
        if (starts) unit[__popcll(all & ((1ull << tid) - 1))] = tid | count << 8;
        if (tid == 0) n_units = __popcll(all);
    }
    __syncthreads();
    const size_t head_elems = (size_t)page * dh;
    auto base = [&](int64_t s) { return ((size_t)(s >> c.page_log2) * c.kv_heads + head) * head_elems; };
    auto store = [&](char *dst, u32x4 x) {
        if constexpr (STREAM)
            __builtin_nontemporal_store(x, reinterpret_cast<u32x4 *>(dst));
        else
            *reinterpret_cast<u32x4 *>(dst) = x;
    };
    const E4m3Scale ks = e4m3_scale(E4M3 ? c.k_scale[head] : 1.f), vs = e4m3_scale(E4M3 ? c.v_scale[head] : 1.f);
    const bf16_t *kh = k + t0 * k_stride + head * dh, *vh = v + t0 * v_stride + head * dh;
    for (int i = tid; i < tile * (dh / E); i += kThreads) {
        const int t = i % tile, j = i / tile;
        if (t >= n) continue;
        const int64_t s = slot_of[t];
        if (s < 0) continue;
        const u32x4 *src = reinterpret_cast<const u32x4 *>(kh + t * k_stride + j * E);
        u32x4 x = src[0];
        if constexpr (E4M3) {
            const u32x4 y = src[1];
            x = u32x4{narrow(x[0], x[1], ks), narrow(x[2], x[3], ks), narrow(y[0], y[1], ks), narrow(y[2], y[3], ks)};
        }
        char *dst = static_cast<char *>(c.k) + base(s) * (16 / E) + ((size_t)j * page + (s & (page - 1))) * 16;
        store(dst, x);
    }
    // V: a unit's W columns a thread
    const int per_unit = dh / W;
    for (int i = tid; i < n_units * per_unit; i += kThreads) {
        const int u = i / per_unit, d = (i - u * per_unit) * W, t = unit[u] & 255, count = unit[u] >> 8;
        const int64_t s = slot_of[t];
        uint32_t x[4][W / 2];
#pragma unroll
        for (int e = 0; e < 4; ++e)
#pragma unroll
            for (int h = 0; h < W / 2; ++h)      // rows past the unit repeat its last one and are not stored
                x[e][h] = reinterpret_cast<const uint32_t *>(vh + (t + min(e, count - 1)) * v_stride + d)[h];
        const int place = (int)(s & (page - 1));
        char *dst = static_cast<char *>(c.v) + (base(s) + ((size_t)(place >> 2) * dh + d) * 4) * (16 / E);
        // column w of the 4 rows: 4 elements that lie together
        u32x4 q;
        if constexpr (E4M3) {
#pragma unroll
            for (int w = 0; w < 4; ++w) {
                float f[4];
#pragma unroll
                for (int e = 0; e < 4; ++e) f[e] = to_e4m3_range(bf16_of(x[e][w / 2], w % 2), vs);
                const int lo = __builtin_amdgcn_cvt_pk_fp8_f32(f[0], f[1], 0, false);
                q[w] = __builtin_amdgcn_cvt_pk_fp8_f32(f[2], f[3], lo, true);
            }
        } else {
#pragma unroll
            for (int w = 0; w < 4; ++w) {        // rows 2 (w % 2) and the next of column w / 2
                const uint32_t lo = x[2 * (w % 2)][0], hi = x[2 * (w % 2) + 1][0];
                q[w] = w / 2 ? (lo >> 16) | (hi & 0xffff0000u) : (lo & 0xffffu) | (hi << 16);
            }
        }
        if (count == 4) {
            store(dst, q);
            continue;
        }
#pragma unroll
        for (int e = 0; e < 3; ++e) {
            if (e >= count) break;
            const int at = (place & 3) + e;      // the element's place in the quad; the value is row e's
#pragma unroll
            for (int w = 0; w < W; ++w) {
                if constexpr (E4M3)
                    reinterpret_cast<uint8_t *>(dst)[4 * w + at] = (uint8_t)(q[w] >> (8 * e));
                else
                    reinterpret_cast<bf16_t *>(dst)[4 * w + at] = (bf16_t)(x[e][0] >> (16 * w));
            }
        }
    }
}

// ------------------------------------------------------------------------------ attention
//
// One query per request and head, ctx = sum_j softmax_j(scale q . k_j) v_j over
// the request's pages.  A workgroup takes one part of one request's keys for one
// key-value head and up to 16 of its query heads; its waves take steps
// of 32 keys in turn, each with its own running maximum, sum and context, and
// join them through LDS.  A request of several parts is joined by a second kernel.
//
// Both products run on the matrix cores with the query heads as columns:
// S^T = K Q^T (rows: keys), O^T = V^T P^T (rows: columns of V).  A lane then
// holds the scores of one head and of the keys 4 c .. 4 c + 3 of two tiles of 16
// (c = lane / 16), which is just what the second product wants from it as its
// operand, so the probabilities never leave the lane's registers; the
// pages are laid out so that K's and V's operands are 16-byte loads in the
// same sense.  P goes in as two bf16 numbers, its first 8 bits and the rounded
// rest, which keeps 16 bits of it (the result has 8) for two products where there is ample room (the matrix cores
// are busy for 6% of the time).  Neither part is ever negative, nor the rest zero, for which it gets 2^-22 of P more: both
// times an infinite element of V are infinities of its sign, and so is their sum.
//
// Bound by reading the pages once: 64 requests of 4000 - 8192 keys, 32 / 8 heads of 128, 250 us with the joining kernel (6.1
// TB/s, what a plain read reaches), in 8 bits 134 us; one request of 32001 keys 26 us (5.0 TB/s); 96 of 5 - 12000, 16 / 4 heads
// of 64 in 8 bits, 22 us (3.3 TB/s: 784 workgroups in one round, whose longest have 4 steps in a row, and 4 us of joining).
// Changed scores cost little: the 64 requests capped, and lowered as well, 262 us in calls from a graph, 259 as they are, in 8 bits 139 and
// 137 (heads of 128 in bf16 need 135 registers then in place of 124, and a SIMD holds 3 waves).
// Each 16 query heads of a key-value head read the pages for themselves: 64 x 6000 keys with 40 / 2 heads of 128 take 141 us, with
// 32 / 2 (one tile) 74; 64 / 1 145, 16 / 1 41.
// Not kept: K of the next step requested before this step's V is used, and 2 or 4 steps at once (249 registers and 18% slower
// in bf16, no faster in 8 bits).
// four e4m3 values as four bf16 (exact)
__device__ inline u32x2 widen(uint32_t w) {
    typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
    const bf16x2 lo = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, 1.0f, false);
    const bf16x2 hi = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, 1.0f, true);
    return u32x2{__builtin_bit_cast(uint32_t, lo), __builtin_bit_cast(uint32_t, hi)};
}

__device__ inline bf16x8 operand(u32x2 a, u32x2 b) { return __builtin_bit_cast(bf16x8, u32x4{a[0], a[1], b[0], b[1]}); }

// STREAM: pages are read with the non-temporal hint (see kStreamBytes).  SCORED: scores have a cap or a slope.
template <int DH, KvKind KIND, int WAVES, bool STREAM, bool SCORED>
__global__ __launch_bounds__(64 * WAVES, 2) void paged_attention_kernel(AttnArgs a) {
    constexpr bool E4M3 = KIND == KvKind::E4m3;
    constexpr int ES = E4M3 ? 1 : 2;             // bytes per element
    constexpr int NK = DH * ES / 64;             // 16-byte loads per lane and key tile: DH columns of 16 keys
    constexpr int W = E4M3 ? 4 : 2;              // columns of V in a 16-byte load
    constexpr int NV = DH / (16 * W);            // such loads per key tile
    constexpr int ROW = DH + 4;
    __shared__ __attribute__((aligned(16))) float o_lds[WAVES][16][ROW];
    __shared__ float m_lds[WAVES][16], l_lds[WAVES][16];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int r = lane & 15, c = lane >> 4;
    const int group = a.heads / a.c.kv_heads, tiles = (group + 15) / 16;
    // the heads of one item next to each other: their parts of a page are neighbours in memory
    const int rows = a.c.kv_heads * tiles, step = gridDim.x / rows;
    const int item0 = blockIdx.x / rows, row = blockIdx.x - item0 * rows;
    const int kvh = row / tiles, tile = row - kvh * tiles;
    const int head0 = kvh * group + tile * 16, n_heads = min(16, group - tile * 16);
    const int page = 1 << a.c.page_log2;
    const uint32_t page_bytes = page * DH * ES;
    const char *K = static_cast<const char *>(a.c.k), *V = static_cast<const char *>(a.c.v);
    const float scale = E4M3 ? a.scale_log2e * a.c.k_scale[kvh] : a.scale_log2e;
    const float v_scale = E4M3 ? a.c.v_scale[kvh] : 1.f;
    const uint32_t k_lane = (c * page + r) * 16, v_lane = c * DH * 4 * ES + r * 16;

    int b0 = 0, before = 0;
    AttnItem it;
    for (int item = item0; find_item(a, item, b0, before, it); item += step) {
        const int part_log2 = paged_part_log2(it.keys, a.split);
        const int k0 = it.part << part_log2, k1 = min(it.keys, k0 + (1 << part_log2));
        const int32_t *ids = a.table + (size_t)it.b * a.table_stride;
        // the queries as the first product's second operand: column r, rows as K's pieces have them
        bf16x8 q[DH / 32];
        {
            const bf16_t *qh = a.q + (int64_t)it.b * a.q_stride + (head0 + min(r, n_heads - 1)) * DH;
#pragma unroll
            for (int i = 0; i < DH / 32; ++i) {
                const int d = E4M3 ? 16 * (4 * (i / 2) + c) + 8 * (i % 2) : 8 * (4 * i + c);
                q[i] = *reinterpret_cast<const bf16x8 *>(qh + d);
            }
        }
        const float slope = SCORED && a.slopes ? slope_log2e(a.slopes[head0 + min(r, n_heads - 1)]) : 0.f;
        float m = -INFINITY, l = 0.f;
        f32x4 o[NV][W] = {};
        const int steps = (k1 - k0 + 31) / 32;
        for (int s0 = 0; s0 < steps; s0 += 32 * WAVES) {
            // lane 2 i + t: the page of key tile t of this wave's i-th step from s0 on
            int pages;
            {
                const int key = k0 + (s0 + wave + WAVES * (lane >> 1)) * 32 + (lane & 1) * 16;
                pages = key < k1 ? ids[key >> a.c.page_log2] : -1;
                if (pages >= a.c.n_pages) pages = -1;
            }
            for (int i = 0; i < 32 && s0 + wave + WAVES * i < steps; ++i) {
                const int key0 = k0 + (s0 + wave + WAVES * i) * 32;
                u32x4 kr[2][NK], vr[2][NV];
                int limit[2];     // keys of each tile that take part
#pragma unroll
                for (int t = 0; t < 2; ++t) {
                    const int id = __builtin_amdgcn_readlane(pages, 2 * i + t);
                    const int key = key0 + 16 * t, off = key & (page - 1);
                    limit[t] = id < 0 ? 0 : min(16, k1 - key);
                    const size_t at = ((size_t)max(id, 0) * a.c.kv_heads + kvh) * page_bytes;
                    const __amdgpu_buffer_rsrc_t kp = page_buffer(K, at, page_bytes), vp = page_buffer(V, at, page_bytes);
#pragma unroll
                    for (int j = 0; j < NK; ++j)
                        kr[t][j] = __builtin_amdgcn_raw_buffer_load_b128(kp, k_lane, off * 16 + j * 64 * page,
                                                                         STREAM ? 2 : 0);
#pragma unroll
                    for (int j = 0; j < NV; ++j)
                        vr[t][j] = __builtin_amdgcn_raw_buffer_load_b128(vp, v_lane, off * DH * ES + j * 256,
                                                                         STREAM ? 2 : 0);
                }
                float p[8];
                float mx = m;
#pragma unroll
                for (int t = 0; t < 2; ++t) {
                    f32x4 s = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
                    for (int j = 0; j < NK; ++j) {
                        if constexpr (E4M3) {
                            s = __builtin_amdgcn_mfma_f32_16x16x32_bf16(operand(widen(kr[t][j][0]), widen(kr[t][j][1])),
                                                                        q[2 * j], s, 0, 0, 0);
                            s = __builtin_amdgcn_mfma_f32_16x16x32_bf16(operand(widen(kr[t][j][2]), widen(kr[t][j][3])),
                                                                        q[2 * j + 1], s, 0, 0, 0);
                        } else {
                            s = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, kr[t][j]), q[j], s, 0,
                                                                        0, 0);
                        }
                    }
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        float z = s[e] * scale;
                        if constexpr (SCORED) {
                            if (a.cap_log2e != 0.f) z = capped(a, z);
                            if (a.slopes) z = lowered(z, slope, key0 + 16 * t + 4 * c + e, it.keys - 1);
                        }
                        p[4 * t + e] = 4 * c + e < limit[t] ? z : -INFINITY;
                        mx = fmaxf(mx, p[4 * t + e]);
                    }
                }
                mx = across_rows_max(mx);
                // nothing but -inf so far: any finite maximum gives p = 0
                const float ref = mx == -INFINITY ? 0.f : mx;
                if (__any(mx > m)) {
                    const float f = __builtin_amdgcn_exp2f(m - ref);
                    l *= f;
#pragma unroll
                    for (int j = 0; j < NV; ++j)
#pragma unroll
                        for (int w = 0; w < W; ++w) o[j][w] *= f;
                    m = mx;
                }
                uint32_t hi[4], lo[4];
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const float x = __builtin_amdgcn_exp2f(p[2 * e] - ref), y = __builtin_amdgcn_exp2f(p[2 * e + 1] - ref);
                    l += x + y;
                    hi[e] = __builtin_amdgcn_perm(__float_as_uint(y), __float_as_uint(x), 0x07060302u);     // upper halves
                    lo[e] = pack2(fmaf(x, 1.f + 0x1p-22f, -__uint_as_float(hi[e] << 16)),
                                  fmaf(y, 1.f + 0x1p-22f, -__uint_as_float(hi[e] & 0xffff0000u)));
                }
                const bf16x8 p_hi = __builtin_bit_cast(bf16x8, u32x4{hi[0], hi[1], hi[2], hi[3]});
                const bf16x8 p_lo = __builtin_bit_cast(bf16x8, u32x4{lo[0], lo[1], lo[2], lo[3]});
                // places past the last key hold any bits: cleared, since 0 times NaN is NaN
#pragma unroll
                for (int t = 0; t < 2; ++t) {
                    if (limit[t] < 16) {
                        const int n = min(max(limit[t] - 4 * c, 0), 4);
#pragma unroll
                        for (int j = 0; j < NV; ++j)
#pragma unroll
                            for (int e = 0; e < 4; ++e) {
                                const int have = E4M3 ? 8 * n : min(max(16 * n - 32 * (e % 2), 0), 32);
                                vr[t][j][e] &= have == 32 ? 0xffffffffu : (1u << have) - 1u;
                            }
                    }
                }
#pragma unroll
                for (int j = 0; j < NV; ++j)
#pragma unroll
                    for (int w = 0; w < W; ++w) {
                        bf16x8 x;
                        if constexpr (E4M3)
                            x = operand(widen(vr[0][j][w]), widen(vr[1][j][w]));
                        else
                            x = operand(u32x2{vr[0][j][2 * w], vr[0][j][2 * w + 1]},
                                        u32x2{vr[1][j][2 * w], vr[1][j][2 * w + 1]});
                        o[j][w] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(x, p_hi, o[j][w], 0, 0, 0);
                        o[j][w] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(x, p_lo, o[j][w], 0, 0, 0);
                    }
            }
        }
        // join the waves.  Lane (r, c) holds of head r the columns 16 W j + 4 W c + W e + w
        l = across_rows_sum(l);
        const int late = opaque_lane(), head = late & 15, quad = late >> 4;
        if (head < n_heads) {
            if (quad == 0) {
                m_lds[wave][head] = m;
                l_lds[wave][head] = l;
            }
#pragma unroll
            for (int j = 0; j < NV; ++j) {
                float *dst = &o_lds[wave][head][16 * W * j + 4 * W * quad];
                float flat[4 * W];
#pragma unroll
                for (int e = 0; e < 4; ++e)
#pragma unroll
                    for (int w = 0; w < W; ++w) flat[W * e + w] = o[j][w][e];
#pragma unroll
                for (int e = 0; e < W; ++e)
                    *reinterpret_cast<f32x4 *>(dst + 4 * e) =
                        f32x4{flat[4 * e], flat[4 * e + 1], flat[4 * e + 2], flat[4 * e + 3]};
            }
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
                const float inv = sum == 0.f ? 0.f : v_scale / sum;     // nothing to attend to: zeros
                *reinterpret_cast<u32x2 *>(a.ctx + bh * DH + d) =
                    u32x2{pack2(acc[0] * inv, acc[1] * inv), pack2(acc[2] * inv, acc[3] * inv)};
            } else {
                const size_t slot = bh * a.slots + it.part;
                *reinterpret_cast<f32x4 *>(a.part_o + slot * DH + d) = acc * v_scale;
                if (d == 0) *reinterpret_cast<f32x2 *>(a.part_ml + 2 * slot) = f32x2{top, sum};
            }
        }
        __syncthreads();
    }
}

// Joins a request's parts: M = max m, ctx = sum 2^(m - M) o / sum 2^(m - M) l.
// One workgroup per (request, head); a group of DH / 4 threads takes every
// (4 * kThreads / DH)-th part, in order.
template <int DH>
__global__ __launch_bounds__(kThreads) void paged_join_kernel(AttnArgs a) {
    constexpr int TPP = DH / 4, PAR = kThreads / TPP;
    __shared__ __attribute__((aligned(16))) f32x4 acc_lds[PAR][TPP];
    __shared__ float sum_lds[PAR];
    const int bh = blockIdx.x, b = bh / a.heads;
    const int parts = paged_parts(min(max(a.lens[b], 0), a.max_keys), a.split);
    if (parts == 1) return;
    const float *ml = a.part_ml + (size_t)bh * a.slots * 2;
    const int lane = threadIdx.x & 63;
    float top = -INFINITY;
    for (int i = lane; i < parts; i += 64) top = fmaxf(top, ml[2 * i]);
#pragma unroll
    for (int s = 32; s >= 1; s >>= 1) top = fmaxf(top, __shfl_xor(top, s));
    const float ref = top == -INFINITY ? 0.f : top;
    const int g = threadIdx.x / TPP, d = threadIdx.x % TPP;
    f32x4 acc = {0.f, 0.f, 0.f, 0.f};
    float sum = 0.f;
    const f32x4 *o = reinterpret_cast<const f32x4 *>(a.part_o + (size_t)bh * a.slots * DH) + d;
#pragma unroll 4      // four parts' loads at once (one request of 64000 keys, one key-value head: 15.9 -> 15.5 us in all)
    for (int i = g; i < parts; i += PAR) {
        const f32x2 x = *reinterpret_cast<const f32x2 *>(ml + 2 * i);
        const float f = __builtin_amdgcn_exp2f(x[0] - ref);
        sum += f * x[1];
        acc += f * o[(size_t)i * TPP];
    }
    acc_lds[g][d] = acc;
    if (d == 0) sum_lds[g] = sum;
    __syncthreads();
    if (g != 0) return;
#pragma unroll
    for (int i = 1; i < PAR; ++i) {
        acc += acc_lds[i][d];
        sum += sum_lds[i];
    }
    const float inv = sum == 0.f ? 0.f : 1.f / sum;
    *reinterpret_cast<u32x2 *>(a.ctx + (size_t)bh * DH + 4 * d) =
        u32x2{pack2(acc[0] * inv, acc[1] * inv), pack2(acc[2] * inv, acc[3] * inv)};
}

// A call that may read this much is taken to stream its pages past the chip's last cache (256 MiB, for which the other
// layers' pages compete as well), and reads them with the non-temporal hint; what a smaller one reads may still be there at the
// next call.  us without / with the hint, calls on three caches in turn: 1534 MB 269 / 250 (6.1 TB/s, what a plain read
// of the memory reaches), 767 MB 145 / 134, 135 MB 27.3 / 24.5, 131 MB 30.7 / 27.1; but 72 MB 22.4 / 23.1, 44 MB in short requests
// 14.7 / 15.9 (and 74 MB in long ones 15.3 / 15.3, 16 MB 10.3 / 10.1).
// The host knows the table's width and the pool's size, not the lengths: short requests under a wide table of a large pool count as
// long ones (96 x 5 - 500 keys, 16 heads of 128: 14.4 us under their own table, 17.0 under one of 12000 keys, by the
// joining launch, and 18.8 with 24000 pages, by the hint).
constexpr int64_t kStreamBytes = 96 << 20;

template <int DH, KvKind KIND, int WAVES, bool SCORED>
hipError_t launch_attention_w(const AttnArgs &a, bool stream_pages, dim3 grid, hipStream_t stream) {
    return stream_pages ? launch_kernel(paged_attention_kernel<DH, KIND, WAVES, true, SCORED>, grid, dim3(64 * WAVES), stream, a)
                        : launch_kernel(paged_attention_kernel<DH, KIND, WAVES, false, SCORED>, grid, dim3(64 * WAVES), stream, a);
}

template <int DH, KvKind KIND>
hipError_t launch_attention(const AttnArgs &a, bool stream_pages, dim3 grid, hipStream_t stream) {
    if (a.cap_log2e != 0.f || a.slopes)
        return a.split.waves == 8 ? launch_attention_w<DH, KIND, 8, true>(a, stream_pages, grid, stream)
                                  : launch_attention_w<DH, KIND, 2, true>(a, stream_pages, grid, stream);
    return a.split.waves == 8 ? launch_attention_w<DH, KIND, 8, false>(a, stream_pages, grid, stream)
                              : launch_attention_w<DH, KIND, 2, false>(a, stream_pages, grid, stream);
}

}  // namespace

hipError_t launch_paged_plan(const PlanArgs &p, hipStream_t stream) {
    // a thread a slot, and waves for the requests, up to 4 workgroups a CU
    const int64_t groups = std::max<int64_t>((p.room + (int64_t)kThreads - 1) / kThreads,
                                             (p.batch + kWaves * kPlanGiveBack - 1) / (kWaves * kPlanGiveBack));
    return launch_kernel(paged_plan_kernel, dim3((unsigned)std::min<int64_t>(groups, 1024)), dim3(kThreads), stream, p);
}

hipError_t launch_paged_append(const PagedCache &c, const bf16_t *k, const bf16_t *v, const int64_t *slots, int tokens,
                               int64_t k_stride, int64_t v_stride, hipStream_t stream) {
    // few tokens: more workgroups of fewer (48 tokens of 8 heads 3.6 us in tiles of 8, 4.3 of 16, 5.7 of 32; 24001 in 8 bits
    // 31.7 us in tiles of 32, 32.4 of 16, 40 of 8; 16000 in bf16 22.2, 22.7 and 27)
    const int tile = (int64_t)tokens * c.kv_heads <= 16 * 1024 ? 8 : kAppendTile;
    const dim3 grid((unsigned)((tokens + tile - 1) / tile * c.kv_heads));
    const bool e4m3 = c.kind == KvKind::E4m3;
    const bool stream_out = (int64_t)tokens * c.kv_heads * c.head_dim * (e4m3 ? 2 : 4) >= kAppendStream;
    auto launch = [&](auto kernel) {
        return launch_kernel(kernel, grid, dim3(kThreads), stream, c, k, v, slots, tokens, tile, k_stride, v_stride);
    };
    if (e4m3) return stream_out ? launch(paged_append_kernel<true, true>) : launch(paged_append_kernel<true, false>);
    return stream_out ? launch(paged_append_kernel<false, true>) : launch(paged_append_kernel<false, false>);
}

size_t paged_workspace_floats(const PagedCache &c, int batch, int heads, int max_keys) {
    const size_t slots = paged_most_parts(max_keys, paged_split(batch, heads, c.kv_heads, c.kind == KvKind::Mx4));
    return slots == 1 ? 0 : (size_t)batch * heads * slots * (c.head_dim + 2);
}

hipError_t launch_paged_attention(const PagedCache &c, const bf16_t *q, int64_t q_stride, const int32_t *table,
                                  int table_stride, int max_pages, const int32_t *lens, bf16_t *ctx, float *partials,
                                  int batch, int heads, float scale, ScoreForm form, hipStream_t stream) {
    AttnArgs a{};
    a.c = c;
    a.q = q;
    a.q_stride = q_stride;
    a.table = table;
    a.table_stride = table_stride;
    a.lens = lens;
    a.ctx = ctx;
    a.batch = batch;
    a.heads = heads;
    a.max_keys = max_pages << c.page_log2;
    a.split = paged_split(batch, heads, c.kv_heads, c.kind == KvKind::Mx4);
    a.slots = paged_most_parts(a.max_keys, a.split);
    a.scale_log2e = scale * kLog2e;
    a.cap_log2e = form.cap * kLog2e;
    a.cap_inv = form.cap == 0.f ? 0.f : 1.f / a.cap_log2e;
    a.slopes = form.slopes;
    a.part_o = partials;
    a.part_ml = partials + (size_t)batch * heads * a.slots * c.head_dim;
    // The lengths are the device's: a workgroup for every part that there could be, up to 8 a CU, which then
    // go on to further items.  (4, 8 and 16 a CU, us: 64 x 4000 - 8192 keys 255, 250 and 250; 96 x 5 - 12000 keys,
    // where most workgroups find nothing to do, 21.6, 21.6 and 26.3.)
    const int rows = c.kv_heads * paged_tiles(heads, c.kv_heads);
    const int64_t items = (int64_t)batch * a.slots;
    const dim3 grid((unsigned)(std::min<int64_t>(items, std::max(1, 2048 / rows)) * rows));
    const int64_t pages = std::min((int64_t)c.n_pages, (int64_t)batch * max_pages);
    const bool stream_pages = pages * c.kv_heads * 2 * (int64_t)c.page_bytes() >= kStreamBytes;      // K and V
    const bool narrow = c.head_dim == 64;
    hipError_t e;
    switch (c.kind) {
    case KvKind::Bf16:
        e = narrow ? launch_attention<64, KvKind::Bf16>(a, stream_pages, grid, stream)
                   : launch_attention<128, KvKind::Bf16>(a, stream_pages, grid, stream);
        break;
    case KvKind::E4m3:
        e = narrow ? launch_attention<64, KvKind::E4m3>(a, stream_pages, grid, stream)
                   : launch_attention<128, KvKind::E4m3>(a, stream_pages, grid, stream);
        break;
    default: e = launch_attention_mx4(a, stream_pages, grid, stream);
    }
    if (e != hipSuccess || a.slots == 1) return e;     // no request can have a second part
    const dim3 join_grid(batch * heads);
    return narrow ? launch_kernel(paged_join_kernel<64>, join_grid, dim3(kThreads), stream, a)
                  : launch_kernel(paged_join_kernel<128>, join_grid, dim3(kThreads), stream, a);
}

}  // namespace iefwd
