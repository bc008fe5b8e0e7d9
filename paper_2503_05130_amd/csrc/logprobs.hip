// Log probabilities of given tokens, entropy and the most probable alternatives over a
// vocabulary, and the gradient of the first two, for gfx950.
//
// For a row x of logits, with m = max x, d_j = x_j - m and a scale s > 0 (the inverse of a temperature):
//   S = sum e^(s d_j),  T = sum e^(s d_j) d_j
//   log p_j = s d_j - log S,  entropy = -sum p_j log p_j = log S - s T / S
// Both are differences of small numbers where the row is sure of a token: relative to m nothing large cancels.
//   gradient of g_l log p_t + g_h entropy:  s (g_l (1[j = t] - p_j) - g_h p_j (log p_j + entropy))
// Bound by reading the logits once (and writing the gradient): 4095 x 65003 bf16 in 105 us between gradients (median of a profile, 5.1
// TB/s; alone from a graph 100; 8.9 vector instructions an element, 81% of the issue slots) and its gradient in 193 (5.5 TB/s; 11.6 an
// element, 51%).  Few rows by latency and issue: 48 x 131072 with 5 alternatives 9.1 us and 3.4 for joining the parts, of which the
// bytes are 2.1.  Alternatives cost many rows too: 1000 x 128000 with 32 of them 78 us, without 56; fp32 500 x 128000 64 and 50.
#include "logprobs.h"

#include <algorithm>
#include <cmath>
#include <type_traits>

#include "mx4_device.h"

namespace iefwd {
namespace {

constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f, kLeast = -3.0e38f;
constexpr int kThreads = 256;
constexpr int kBuffer = 128;      // candidates of a wave
constexpr int kSlack = 16;       // more than n of them are cut to n after a tile

// Rows may begin anywhere: 16-byte loads and stores of any alignment, which the memory of gfx950 takes.
typedef uint32_t u32x4_any __attribute__((ext_vector_type(4), aligned(2)));

// `count` elements of a 16-byte piece, the first `valid` of which exist; the others are -inf.
template <bool F32> struct Piece {
    static constexpr int N = F32 ? 4 : 8;
    u32x4 raw;

    __device__ void load(const char *p, int valid) {
        if (valid >= N) {
            raw = *reinterpret_cast<const u32x4_any *>(p);
            return;
        }
        const uint32_t none = F32 ? 0xff800000u : 0xff80ff80u;
        raw = u32x4{none, none, none, none};
#pragma unroll
        for (int e = 0; e < N; ++e) {
            if (e >= valid) continue;
            if (F32) raw[e] = reinterpret_cast<const uint32_t *>(p)[e];
            else raw[e / 2] = (raw[e / 2] & (e & 1 ? 0x0000ffffu : 0xffff0000u)) |
                              (uint32_t) reinterpret_cast<const uint16_t *>(p)[e] << (16 * (e & 1));
        }
    }
    __device__ float value(int e) const {
        if (F32) return __uint_as_float(raw[e]);
        return __uint_as_float(e & 1 ? raw[e / 2] & 0xffff0000u : raw[e / 2] << 16);
    }
};

// Numbers as whole ones of the same order, from 1 on: NaN above all, -0 as 0; and back.
__device__ inline uint32_t order_of(float x) {
    const uint32_t u = __float_as_uint(x + 0.f);
    return x != x ? 0xffffffffu : (u >> 31) ? ~u : u | 0x80000000u;
}
// (bf16: of the upper 16 bits alone, which decide between them)
template <bool F32>
__device__ inline uint32_t key_of(float x) { return F32 ? order_of(x) : order_of(x) & 0xffff0000u; }
__device__ inline float value_of(uint32_t k, bool f32) {
    if (!f32 && !(k >> 31)) k |= 0xffffu;
    return __uint_as_float(k >> 31 ? k & 0x7fffffffu : ~k);
}

// maximum with NaN if one is
__device__ inline float top_of(float a, float b) { return __builtin_elementwise_maximum(a, b); }

struct Sums {
    float m, s, t;

    // relative to `to`, at least as large as m
    __device__ void rescale(float to, float c) {
        const float ref = to == -INFINITY ? 0.f : to, d = m - ref, f = __builtin_amdgcn_exp2f(d * c);
        t = f == 0.f ? 0.f : f * (t + s * d);
        s *= f;
        m = to;
    }
};

// Over all lanes by row shifts of 1, 2, 4 and 8, then lane 15's row result to the next row and lane 31's to the upper half.
template <class Op>
__device__ inline uint32_t over_wave(uint32_t v, uint32_t neutral, Op op) {
    v = op(v, (uint32_t)__builtin_amdgcn_update_dpp((int)neutral, (int)v, 0x111, 0xf, 0xf, false));
    v = op(v, (uint32_t)__builtin_amdgcn_update_dpp((int)neutral, (int)v, 0x112, 0xf, 0xf, false));
    v = op(v, (uint32_t)__builtin_amdgcn_update_dpp((int)neutral, (int)v, 0x114, 0xf, 0xf, false));
    v = op(v, (uint32_t)__builtin_amdgcn_update_dpp((int)neutral, (int)v, 0x118, 0xf, 0xf, false));
    v = op(v, (uint32_t)__builtin_amdgcn_update_dpp((int)neutral, (int)v, 0x142, 0xa, 0xf, false));
    v = op(v, (uint32_t)__builtin_amdgcn_update_dpp((int)neutral, (int)v, 0x143, 0xc, 0xf, false));
    return __builtin_amdgcn_readlane(v, 63);
}

__device__ inline uint32_t largest_of(uint32_t v) {
    return over_wave(v, 0, [](uint32_t x, uint32_t y) { return max(x, y); });
}
__device__ inline float sum_of(float v) {
    return __uint_as_float(over_wave(__float_as_uint(v), 0, [](uint32_t x, uint32_t y) {
        return __float_as_uint(__uint_as_float(x) + __uint_as_float(y));
    }));
}

// All lanes' sums together, in every lane.
__device__ inline Sums across_wave(Sums a, float c) {
    a.rescale(__uint_as_float(over_wave(__float_as_uint(a.m), __float_as_uint(-INFINITY), [](uint32_t x, uint32_t y) {
                  return __float_as_uint(top_of(__uint_as_float(x), __uint_as_float(y)));
              })),
              c);
    a.s = sum_of(a.s);
    a.t = sum_of(a.t);
    return a;
}

// The row's given token and its logit, asked for early: two loads in a row.
struct Given {
    float logit;
    bool there;

    __device__ Given(const LogprobArgs &a, int row) {
        const int64_t token = a.tokens[row];
        there = token >= 0 && token < a.vocab;
        const int64_t at = row * a.stride + (there ? token : 0);
        logit = a.f32 ? static_cast<const float *>(a.logits)[at]
                      : __uint_as_float((uint32_t) static_cast<const bf16_t *>(a.logits)[at] << 16);
    }
};

// What a row's sums and its given logit come to; one lane.
__device__ inline void write_row(const LogprobArgs &a, int row, const Given &given, const Sums &s, float log_s) {
    const bool empty = s.m == -INFINITY;      // every token masked
    a.logprobs[row] = !given.there ? 0.f : empty ? -INFINITY : (given.logit - s.m) * a.scale - log_s;
    if (a.entropy) a.entropy[row] = empty ? 0.f : top_of(log_s - a.scale * (s.t / s.s), 0.f);
    if (a.stats) {
        a.stats[2 * row] = s.m;
        a.stats[2 * row + 1] = log_s;
    }
}

__device__ inline float log_sum(const Sums &s) { return s.m == -INFINITY ? 0.f : logf(s.s); }

// A token that may be among the most probable: its logit's key above the complement of its index, so that the larger number comes
// before the other.  0: none.
typedef unsigned long long Candidate;
typedef Candidate Candidate2 __attribute__((ext_vector_type(2)));

__device__ inline Candidate candidate(uint32_t key, uint32_t id) { return (Candidate)key << 32 | (0xffffffffu - id); }

__device__ inline void write_top(const LogprobArgs &a, int row, int place, Candidate c, float m, float log_s) {
    const float x = value_of((uint32_t)(c >> 32), a.f32);
    a.top_ids[(int64_t)row * a.top + place] = (int)(0xffffffffu - (uint32_t)c);
    a.top_logprobs[(int64_t)row * a.top + place] = x == -INFINITY ? (log_s != log_s ? log_s : x) : (x - m) * a.scale - log_s;
}

// Sorts a wave's first `count` candidates (in LDS, 16-byte aligned) and keeps n of them: a lane counts those before its own two,
// eight at a time.
__device__ inline int keep_best(Candidate *list, int count, int n) {
    const int lane = threadIdx.x & 63;
    if (lane < 8 && count + lane < kBuffer) list[count + lane] = 0;
    wave_lds_fence();
    Candidate own[2];
    int rank[2] = {0, 0};
#pragma unroll
    for (int h = 0; h < 2; ++h) own[h] = lane + 64 * h < count ? list[lane + 64 * h] : 0;
    for (int i = 0; i < count; i += 8) {
        Candidate2 c[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) c[j] = *reinterpret_cast<const Candidate2 *>(list + i + 2 * j);
#pragma unroll
        for (int j = 0; j < 8; ++j)
#pragma unroll
            for (int h = 0; h < 2; ++h) rank[h] += c[j / 2][j % 2] > own[h];
    }
    wave_lds_fence();
#pragma unroll
    for (int h = 0; h < 2; ++h)
        if (own[h] && rank[h] < n) list[rank[h]] = own[h];
    wave_lds_fence();
    return min(count, n);
}

// The workspace of a call whose rows are cut into parts: per row and part its best candidates, and its sums.
struct Parts {
    Candidate *best;
    Sums *sums;
};

__device__ __host__ inline Parts parts_in(void *ws, int64_t row_parts, int top) {
    Parts p;
    p.best = static_cast<Candidate *>(ws);
    p.sums = reinterpret_cast<Sums *>(p.best + row_parts * top);
    return p;
}

// A workgroup takes a part of a row, its waves tiles of it in turn: kUnits loads of 16 bytes a lane, whose elements a lane
// adds to its own sums under its own maximum.
//
// The best n: the largest number that n lanes' own maxima of the first tile reach is at most the n-th largest
// element; what reaches it becomes a candidate.  From then on only larger numbers do, which few are: one comparison a lane and tile
// finds that there are none.  A full buffer is sorted and cut to n, whose last is the new border.
// LISTS: 0 no such tokens; 1 each wave goes by its own lanes; 2 by all of the workgroup's, which leaves the waves a quarter of the
// candidates for a barrier and three more ballots a bit: taken for n > 8.  us, 1 / 2:
//   48 x 131072, n = 5 12.7 13.1     300 x 50001, 20 37.8 22.6     1000 x 128000, 32 117 79     500 x 128000 fp32, 20 78 65
template <bool F32, int LISTS, int WAVES>
__global__ __launch_bounds__(64 * WAVES) void logprobs_kernel(LogprobArgs a, int parts, int part) {
    constexpr int N = Piece<F32>::N, kUnits = F32 ? 6 : 4, kTile = 64 * N * kUnits;
    constexpr bool TOP = LISTS > 0, SHARED = LISTS == 2 && WAVES > 1;
    __shared__ __attribute__((aligned(16))) Candidate best[TOP ? WAVES : 1][kBuffer];
    __shared__ u32x4 stage[TOP ? WAVES : 1][TOP ? kUnits : 1][64];      // a wave's tile
    __shared__ uint32_t tops[SHARED ? 64 * WAVES : 1];
    __shared__ int counts[WAVES];
    __shared__ Sums sums[WAVES];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int row = blockIdx.x / parts, p = blockIdx.x - row * parts;
    const int first = p * part, end = min(a.vocab, first + part);
    const char *x = static_cast<const char *>(a.logits) + row * a.stride * (F32 ? 4 : 2);
    const float c = a.scale * kLog2e;
    const Given given(a, row);
    Sums own{-INFINITY, 0.f, 0.f};
    Candidate *mine = best[TOP ? wave : 0];
    int count = 0;
    Candidate border = 0;      // what comes before it is a candidate
    uint32_t reach = 0;        // its key, or the first tile's
    bool begun = false;
    auto cut = [&] {      // n or more candidates to the best n
        count = keep_best(mine, count, a.top);
        border = mine[a.top - 1];
        reach = __builtin_amdgcn_readfirstlane((uint32_t)(border >> 32));
        border = (Candidate)reach << 32 | (uint32_t)__builtin_amdgcn_readfirstlane((uint32_t)border);
    };
    for (int at = first + wave * kTile; at < end; at += WAVES * kTile) {
        Piece<F32> v[kUnits];
        const int e0 = at + lane * N;
        if (at + kTile <= end) {
#pragma unroll
            for (int u = 0; u < kUnits; ++u) v[u].load(x + (int64_t)(e0 + u * 64 * N) * (F32 ? 4 : 2), N);
        } else {
#pragma unroll
            for (int u = 0; u < kUnits; ++u) v[u].load(x + (int64_t)(e0 + u * 64 * N) * (F32 ? 4 : 2), end - (e0 + u * 64 * N));
        }
        float top = v[0].value(0);
#pragma unroll
        for (int i = 1; i < kUnits * N; ++i) top = top_of(top, v[i / N].value(i % N));
        if (__any(!(top <= own.m))) own.rescale(top_of(own.m, top), c);
        const float ref = own.m == -INFINITY ? 0.f : own.m;
#pragma unroll
        for (int i = 0; i < kUnits * N; ++i) {
            const float d = v[i / N].value(i % N) - ref, e = __builtin_amdgcn_exp2f(d * c);
            own.s += e;
            own.t = fmaf(e, fmaxf(d, kLeast), own.t);      // 0 times -inf would be NaN
        }
        if constexpr (TOP) {
            const uint32_t lane_top = e0 < end ? key_of<F32>(top) : 0;
            bool take = __any(lane_top > reach);
            const bool first_tile = !begun;
            if (first_tile) {
                // the largest number that at least n lanes of the workgroup reach, 0 if fewer have an element
                uint32_t of[SHARED ? WAVES : 1] = {lane_top};
                if constexpr (SHARED) {
                    tops[threadIdx.x] = lane_top;
                    __syncthreads();
#pragma unroll
                    for (int w = 0; w < WAVES; ++w) of[w] = tops[64 * w + lane];
                }
                for (int bit = 31; bit >= (F32 ? 0 : 16); --bit) {
                    const uint32_t t = reach | 1u << bit;
                    int lanes = 0;
#pragma unroll
                    for (int w = 0; w < (SHARED ? WAVES : 1); ++w) lanes += __popcll(__ballot(of[w] >= t));
                    if (lanes >= a.top) reach = t;
                }
                reach = __builtin_amdgcn_readfirstlane(reach);
                border = reach ? ((Candidate)reach << 32) - 1 : 0;      // it and larger ones, whatever the index
                begun = take = true;
            }
            if (take) {
                // which of the lane's elements may be: by the numbers; at no border, or one of NaN, all of them
                const float low = reach && reach != key_of<F32>(NAN) ? value_of(reach, F32) : NAN;
                uint32_t left = 0;
#pragma unroll
                for (int i = kUnits * N - 1; i >= 0; --i) left = 2 * left + !(v[i / N].value(i % N) < low);
                if (low == -INFINITY && first_tile) {
                    // fewer than n lanes have another number: the first n of -inf are in the lanes' first pieces, whose indices are
                    // the lowest
                    uint32_t others = 0;
#pragma unroll
                    for (int i = kUnits * N - 1; i >= N; --i) others = 2 * others + (v[i / N].value(i % N) != low);
                    left &= others << N | ((1u << N) - 1);
                }
#pragma unroll
                for (int u = 0; u < kUnits; ++u) stage[wave][u][lane] = v[u].raw;
                wave_lds_fence();
                // a lane's next such element from LDS (in a loop: code that runs once costs more for being fetched)
#pragma unroll 1
                while (__any(left != 0)) {
                    Candidate own_c = 0;
                    if (left) {
                        const int i = __builtin_ctz(left), id = e0 + i / N * 64 * N + i % N;
                        left &= left - 1;
                        const void *piece = &stage[wave][i / N][lane];
                        const float w = F32 ? static_cast<const float *>(piece)[i % N]
                                            : __uint_as_float((uint32_t) static_cast<const uint16_t *>(piece)[i % N] << 16);
                        if (id < end) own_c = candidate(key_of<F32>(w), id);
                    }
                    uint64_t who = __ballot(own_c > border);
                    if (count + __popcll(who) > kBuffer) {
                        cut();
                        who = __ballot(own_c > border);
                    }
                    if (who >> lane & 1) mine[count + __popcll(who & ((1ull << lane) - 1))] = own_c;
                    count += __popcll(who);
                }
                wave_lds_fence();
                if (count >= a.top + kSlack) cut();
            }
        }
    }
    if constexpr (SHARED)
        if (!begun) {      // no tile: the others wait for this wave's part of theirs
            tops[threadIdx.x] = 0;
            __syncthreads();
        }
    own = across_wave(own, c);
    if constexpr (TOP) count = keep_best(mine, count, a.top);
    Sums all = own;
    if constexpr (WAVES > 1) {
        if (lane == 0) {
            sums[wave] = own;
            counts[wave] = count;
        }
        __syncthreads();
        all = sums[0];
        float m = all.m;
#pragma unroll
        for (int w = 1; w < WAVES; ++w) m = top_of(m, sums[w].m);
        all.rescale(m, c);
#pragma unroll
        for (int w = 1; w < WAVES; ++w) {
            Sums o = sums[w];
            o.rescale(m, c);
            all.s += o.s;
            all.t += o.t;
        }
    }
    const float log_s = log_sum(all);
    const Parts out = parts_in(a.workspace, (int64_t)a.rows * parts, a.top);
    const int64_t slot = (int64_t)row * parts + p;
    if (threadIdx.x == 0) {
        if (parts == 1) write_row(a, row, given, all, log_s);
        else out.sums[slot] = all;
    }
    if constexpr (TOP) {
        // a candidate's place: those before it in every wave's sorted list
        const int i = lane;
        if (i < count) {
            const Candidate own_c = mine[i];
            int place = i;
            if constexpr (WAVES > 1) {
                int before[WAVES] = {};
#pragma unroll
                for (int step = kMaxTop; step >= 1; step >>= 1)
#pragma unroll
                    for (int o = 0; o < WAVES; ++o) {
                        const int to = before[o] + step;
                        if (to <= counts[o] && best[o][to - 1] > own_c) before[o] = to;
                    }
                place = 0;
#pragma unroll
                for (int o = 0; o < WAVES; ++o) place += before[o];      // of its own list: i
            }
            if (place < a.top) {
                if (parts == 1) write_top(a, row, place, own_c, all.m, log_s);
                else out.best[slot * a.top + place] = own_c;
            }
        }
        if (parts > 1) {
            int total = count;
            if constexpr (WAVES > 1) {
                total = 0;
#pragma unroll
                for (int o = 0; o < WAVES; ++o) total += counts[o];
            }
            if ((int)threadIdx.x >= total && (int)threadIdx.x < a.top) out.best[slot * a.top + threadIdx.x] = 0;      // no further ones
        }
    }
}

// A row's parts together: a wave a row, a lane a part (at most 64).  Their sorted lists are merged from their heads.
template <bool TOP>
__global__ __launch_bounds__(64) void logprobs_join_kernel(LogprobArgs a, int parts) {
    __shared__ Candidate lists[TOP ? 64 * kMaxTop : 1];
    const int row = blockIdx.x, lane = threadIdx.x;
    const Given given(a, row);
    const Parts in = parts_in(a.workspace, (int64_t)a.rows * parts, a.top);
    const int64_t slot = (int64_t)row * parts;
    if constexpr (TOP)
        for (int i = lane; i < parts * a.top; i += 64) lists[i] = in.best[slot * a.top + i];
    Sums own{-INFINITY, 0.f, 0.f};
    if (lane < parts) own = in.sums[slot + lane];
    own = across_wave(own, a.scale * kLog2e);
    const float log_s = log_sum(own);
    if (lane == 0) write_row(a, row, given, own, log_s);
    if constexpr (TOP) {
        __syncthreads();
        int next = lane * a.top;
        const int last = lane < parts ? next + a.top : next;
        Candidate head = next < last ? lists[next] : 0, second = next + 1 < last ? lists[next + 1] : 0, mine = 0;
        next += 2;
        for (int place = 0; place < a.top; ++place) {
            const uint32_t key = largest_of((uint32_t)(head >> 32));
            const uint32_t low = largest_of((uint32_t)(head >> 32) == key ? (uint32_t)head : 0);
            const Candidate first = (Candidate)key << 32 | low;
            if (lane == place) mine = first;
            if (head == first) {      // one lane: indices differ
                head = second;
                second = next < last ? lists[next] : 0;
                ++next;
            }
        }
        if (lane < a.top) write_top(a, row, lane, mine, own.m, log_s);
    }
}

// The gradient: a workgroup takes 4 pieces a thread of a row.  With u = log2 p_j = c (x_j - m) - log2 e log S, an element is
// p_j (a + b u), a = -s (g_l + g_h entropy), b = -s g_h ln 2, and s g_l more at the given token.
//
// FAR: logits and gradient are more than the last cache's 256 MiB.  The last rows go first, which the pass before has
// left there, and the gradient past the cache: forward and backward of 4095 x 65003 bf16 320 -> 293 us by the stores, 282 by both (512 x
// 32000: 22.5, 21.2 and 22.5).
template <bool F32, bool FAR>
__global__ __launch_bounds__(kThreads) void logprobs_grad_kernel(LogprobGradArgs g, int segments) {
    constexpr int N = Piece<F32>::N, kUnits = 4, kTile = kThreads * N * kUnits, ES = F32 ? 4 : 2;
    const int id = FAR ? gridDim.x - 1 - blockIdx.x : blockIdx.x;
    const int row = id / segments, at = (id - row * segments) * kTile;
    const char *x = static_cast<const char *>(g.logits) + row * g.stride * ES;
    char *out = static_cast<char *>(g.out) + row * g.out_stride * ES;
    Piece<F32> v[kUnits];
#pragma unroll
    for (int u = 0; u < kUnits; ++u) {
        const int e0 = at + (u * kThreads + threadIdx.x) * N;
        v[u].load(x + (int64_t)e0 * ES, g.vocab - e0);
    }
    const float m = g.stats[2 * row], c = g.scale * kLog2e, log2_s = g.stats[2 * row + 1] * kLog2e;
    const bool empty = m == -INFINITY;      // zeros: every p is
    const int64_t token = g.tokens[row];
    const bool given = token >= 0 && token < g.vocab && !empty;
    const float gl = given && g.grad_logprobs ? g.scale * g.grad_logprobs[row] : 0.f;
    const float gh = g.grad_entropy && !empty ? g.scale * g.grad_entropy[row] : 0.f;
    const float a = -fmaf(gh, g.grad_entropy ? g.entropy[row] : 0.f, gl), b = -gh * kLn2, ref = empty ? 0.f : m;
#pragma unroll
    for (int u = 0; u < kUnits; ++u) {
        const int e0 = at + (u * kThreads + threadIdx.x) * N;
        float d[N];
#pragma unroll
        for (int e = 0; e < N; ++e) {
            const float l = fmaf(v[u].value(e) - ref, c, -log2_s);
            d[e] = __builtin_amdgcn_exp2f(l) * fmaf(b, fmaxf(l, -1e4f), a);      // p is 0 long before
        }
        const int64_t own = token - e0;
        if (own >= 0 && own < N)
#pragma unroll
            for (int e = 0; e < N; ++e) d[e] += e == own ? gl : 0.f;
        u32x4 w;
        if constexpr (F32) w = u32x4{__float_as_uint(d[0]), __float_as_uint(d[1]), __float_as_uint(d[2]), __float_as_uint(d[3])};
        else w = u32x4{pack2(d[0], d[1]), pack2(d[2], d[3]), pack2(d[4 % N], d[5 % N]), pack2(d[6 % N], d[7 % N])};
        if (e0 + N <= g.vocab) {
            u32x4_any *to = reinterpret_cast<u32x4_any *>(out + (int64_t)e0 * ES);
            if (FAR) __builtin_nontemporal_store((u32x4_any)w, to);
            else *to = w;
        } else {
#pragma unroll
            for (int e = 0; e < N; ++e) {
                if (e0 + e >= g.vocab) continue;
                if constexpr (F32) reinterpret_cast<float *>(out)[e0 + e] = d[e];
                else reinterpret_cast<bf16_t *>(out)[e0 + e] = f32_to_bf16(d[e]);
            }
        }
    }
}

// Few rows are cut into parts that the whole chip works on: up to 2048 workgroups, whole rounds of their waves' tiles each (bf16: of
// 8192 elements, taken for fp32 as well, whose rounds are of 6144 and whose last round in a part is a third full.  fp32, us, in parts of
// 8192 / 6144: 48 x 131072 9.5 9.5, with 5 alternatives 15.1 14.9, 1 x 131072 5.5 4.6, with 5 10.5 9.1, 300 x 50001 15.3 14.9).
struct Split {
    int parts, part;
};

Split split_of(int rows, int vocab) {
    constexpr int kRound = 8192;
    const int rounds = (vocab + kRound - 1) / kRound, most = std::max(1, std::min({64, rounds, 2048 / std::max(rows, 1)}));
    const int each = (rounds + most - 1) / most;
    return {(rounds + each - 1) / each, each * kRound};
}

}  // namespace

size_t logprobs_workspace(int rows, int vocab, int top) {
    const int parts = split_of(rows, vocab).parts;
    return parts == 1 ? 0 : (size_t)rows * parts * (sizeof(Sums) + (size_t)top * sizeof(Candidate));
}

hipError_t launch_logprobs(const LogprobArgs &a, hipStream_t stream) {
    const Split s = split_of(a.rows, a.vocab);
    const int parts = s.parts;
    const dim3 grid((unsigned)((int64_t)a.rows * parts));
    // a wave a row where its tiles are two at most (of bf16; three of fp32)
    const int waves = a.vocab <= 4096 ? 1 : 4;
    auto launch = [&](auto kernel) { return launch_kernel(kernel, grid, dim3(64 * waves), stream, a, s.parts, s.part); };
    const int lists = a.top == 0 ? 0 : a.top <= 8 || waves == 1 ? 1 : 2;
    auto choose = [&](auto f32) {
        constexpr bool F32 = decltype(f32)::value;
        if (waves == 1) return lists ? launch(logprobs_kernel<F32, 1, 1>) : launch(logprobs_kernel<F32, 0, 1>);
        return lists == 2   ? launch(logprobs_kernel<F32, 2, 4>)
               : lists == 1 ? launch(logprobs_kernel<F32, 1, 4>)
                            : launch(logprobs_kernel<F32, 0, 4>);
    };
    const hipError_t e = a.f32 ? choose(std::true_type{}) : choose(std::false_type{});
    if (e != hipSuccess || parts == 1) return e;
    return a.top ? launch_kernel(logprobs_join_kernel<true>, dim3(a.rows), dim3(64), stream, a, parts)
                 : launch_kernel(logprobs_join_kernel<false>, dim3(a.rows), dim3(64), stream, a, parts);
}

hipError_t launch_logprobs_grad(const LogprobGradArgs &a, hipStream_t stream) {
    const int tile = kThreads * 4 * (a.f32 ? 4 : 8), segments = (a.vocab + tile - 1) / tile;
    const dim3 grid((unsigned)((int64_t)a.rows * segments));
    const bool far = (int64_t)a.rows * a.vocab * (a.f32 ? 8 : 4) > 256 << 20;
    auto launch = [&](auto kernel) { return launch_kernel(kernel, grid, dim3(kThreads), stream, a, segments); };
    if (a.f32) return far ? launch(logprobs_grad_kernel<true, true>) : launch(logprobs_grad_kernel<true, false>);
    return far ? launch(logprobs_grad_kernel<false, true>) : launch(logprobs_grad_kernel<false, false>);
}

}  // namespace iefwd
