// Log probabilities of given tokens, entropy and the most probable alternatives over a
// vocabulary, and the gradient of the first two, for gfx950.
//
// For a row x of logits, with m = max x, d_j = x_j - m and a scale s > 0 (the inverse of a temperature):
//   S = sum e^(s d_j),  T = sum e^(s d_j) d_j
//   log p_j = s d_j - log S,  entropy = -sum p_j log p_j = log S - s T / S
// Both are differences of small numbers where the row is sure of a token: relative to m nothing large cancels.
//   gradient of g_l log p_t + g_h entropy:  s (g_l (1[j = t] - p_j) - g_h p_j (log p_j + entropy))
// Bound by reading the logits once (and writing the gradient).
#include "logprobs.h"

#include <algorithm>
#include <cmath>

#include "gemm_device.h"

namespace iefwd {
namespace {

constexpr float kLog2e = 1.4426950408889634f, kLeast = -3.0e38f;
constexpr int kWaves = 4, kThreads = 64 * kWaves;
constexpr int kBuffer = 128;      // candidates of a wave

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

// All lanes' sums together, in every lane.
__device__ inline Sums across_wave(Sums a, float c) {
    float m = a.m;
#pragma unroll
    for (int i = 32; i >= 1; i >>= 1) m = top_of(m, __shfl_xor(m, i));
    a.rescale(m, c);
#pragma unroll
    for (int i = 32; i >= 1; i >>= 1) {
        a.s += __shfl_xor(a.s, i);
        a.t += __shfl_xor(a.t, i);
    }
    return a;
}

// What a row's sums and its given logit come to; one lane.
__device__ inline void write_row(const LogprobArgs &a, int row, const Sums &s, float log_s) {
    const bool empty = s.m == -INFINITY;      // every token masked
    const int64_t token = a.tokens[row];
    float lp = 0.f;
    if (token >= 0 && token < a.vocab) {
        const int64_t at = row * a.stride + token;
        const float x = a.f32 ? static_cast<const float *>(a.logits)[at]
                              : __uint_as_float((uint32_t) static_cast<const bf16_t *>(a.logits)[at] << 16);
        lp = empty ? -INFINITY : (x - s.m) * a.scale - log_s;
    }
    a.logprobs[row] = lp;
    if (a.entropy) a.entropy[row] = empty ? 0.f : top_of(log_s - a.scale * (s.t / s.s), 0.f);
    if (a.stats) {
        a.stats[2 * row] = s.m;
        a.stats[2 * row + 1] = log_s;
    }
}

__device__ inline float log_sum(const Sums &s) { return s.m == -INFINITY ? 0.f : logf(s.s); }

__device__ inline void write_top(const LogprobArgs &a, int row, int place, uint32_t key, int id, float m, float log_s) {
    const float x = value_of(key, a.f32);
    a.top_ids[(int64_t)row * a.top + place] = id;
    a.top_logprobs[(int64_t)row * a.top + place] = x == -INFINITY ? (log_s != log_s ? log_s : x) : (x - m) * a.scale - log_s;
}

// A wave's candidates for the row's largest, in LDS.
struct Candidates {
    uint32_t key[kBuffer];
    int id[kBuffer];
};

__device__ inline bool before(uint32_t ka, int ia, uint32_t kb, int ib) { return ka > kb || (ka == kb && ia < ib); }

// Sorts the first `count` candidates, the largest first and of equal ones the lowest index, and keeps n of them.
__device__ inline int keep_best(Candidates &b, int count, int n) {
    const int lane = threadIdx.x & 63;
    uint32_t key[2];
    int id[2], rank[2] = {0, 0};
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");      // other lanes' candidates
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        const int i = min(lane + 64 * h, kBuffer - 1);
        key[h] = b.key[i];
        id[h] = b.id[i];
    }
    for (int i = 0; i < count; ++i) {
        const uint32_t k = b.key[i];
        const int j = b.id[i];
#pragma unroll
        for (int h = 0; h < 2; ++h) rank[h] += before(k, j, key[h], id[h]);
    }
#pragma unroll
    for (int h = 0; h < 2; ++h)
        if (lane + 64 * h < count && rank[h] < n) {
            b.key[rank[h]] = key[h];
            b.id[rank[h]] = id[h];
        }
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    return min(count, n);
}

// The workspace of a call whose rows are cut into parts: per row and part its sums, and its best candidates.
struct Parts {
    Sums *sums;
    uint32_t *keys;
    int *ids;
};

__device__ __host__ inline Parts parts_in(void *ws, int64_t row_parts, int top) {
    Parts p;
    p.sums = static_cast<Sums *>(ws);
    p.keys = reinterpret_cast<uint32_t *>(p.sums + row_parts);
    p.ids = reinterpret_cast<int *>(p.keys + row_parts * top);
    return p;
}

// A workgroup takes a part of a row, its waves tiles of it in turn: kUnits loads of 16 bytes a lane, whose elements a lane
// adds to its own sums under its own maximum.
//
// The best n: of a wave's first tile, the largest number that n lanes' own maxima reach is at most its n-th largest
// element; what exceeds it becomes a candidate, and equal ones up to n in the order of their indices.  From then on only
// larger numbers do, which few are: one comparison a lane and tile finds that there are none.  A full buffer is sorted and cut to n, whose
// last is the new border.
template <bool F32, bool TOP>
__global__ __launch_bounds__(kThreads) void logprobs_kernel(LogprobArgs a, int parts, int part) {
    constexpr int N = Piece<F32>::N, kUnits = F32 ? 6 : 4, kTile = 64 * N * kUnits;
    __shared__ Candidates best[TOP ? kWaves : 1];
    __shared__ int counts[kWaves];
    __shared__ Sums sums[kWaves];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int row = blockIdx.x / parts, p = blockIdx.x - row * parts;
    const int first = p * part, end = min(a.vocab, first + part);
    const char *x = static_cast<const char *>(a.logits) + row * a.stride * (F32 ? 4 : 2);
    const float c = a.scale * kLog2e;
    Sums own{-INFINITY, 0.f, 0.f};
    Candidates &mine = best[TOP ? wave : 0];
    int count = 0, border_id = 0;      // a candidate comes before (border, border_id)
    uint32_t border = 0;
    bool begun = false;
    for (int at = first + wave * kTile; at < end; at += kWaves * kTile) {
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
            bool take = __any(lane_top > border), ties = false;
            if (!begun) {
                begun = take = ties = true;
                // the largest number that at least n lanes reach, 0 if fewer have an element
                for (int bit = 31; bit >= (F32 ? 0 : 16); --bit) {
                    const uint32_t t = border | 1u << bit;
                    if (__popcll(__ballot(lane_top >= t)) >= a.top) border = t;
                }
                border = __builtin_amdgcn_readfirstlane(border);
            }
            if (take) {
#pragma unroll 1
                for (int u = 0; u < kUnits; ++u) {
                    Piece<F32> w = v[0];
#pragma unroll
                    for (int i = 1; i < kUnits; ++i)
                        if (i == u) w = v[i];
#pragma unroll
                    for (int e = 0; e < N; ++e) {
                        const int id = e0 + u * 64 * N + e;
                        const uint32_t k = id < end ? key_of<F32>(w.value(e)) : 0;
                        uint64_t who = __ballot(k != 0 && before(k, id, border, border_id));
                        if (!who) continue;
                        if (count + __popcll(who) > kBuffer) {
                            count = keep_best(mine, count, a.top);
                            border = __builtin_amdgcn_readfirstlane(mine.key[a.top - 1]);
                            border_id = __builtin_amdgcn_readfirstlane(mine.id[a.top - 1]);
                            ties = false;
                            who = __ballot(k != 0 && before(k, id, border, border_id));
                        }
                        if (who >> lane & 1) {
                            const int i = count + __popcll(who & ((1ull << lane) - 1));
                            mine.key[i] = k;
                            mine.id[i] = id;
                        }
                        count += __popcll(who);
                    }
                }
                if (ties && count < a.top && border != 0) {
#pragma unroll 1
                    for (int u = 0; u < kUnits && count < a.top; ++u) {
                        Piece<F32> w = v[0];
#pragma unroll
                        for (int i = 1; i < kUnits; ++i)
                            if (i == u) w = v[i];
                        uint32_t same = 0;
#pragma unroll
                        for (int e = 0; e < N; ++e)
                            if (e0 + u * 64 * N + e < end && key_of<F32>(w.value(e)) == border) same |= 1u << e;
                        int to = __popc(same);      // of this lane and those before it
#pragma unroll
                        for (int s = 1; s < 64; s <<= 1) {
                            const int o = __shfl_up(to, s);
                            if (lane >= s) to += o;
                        }
                        const int all = __builtin_amdgcn_readlane(to, 63);
                        for (int i = count + to - __popc(same); same && i < a.top; ++i, same &= same - 1) {
                            mine.key[i] = border;
                            mine.id[i] = e0 + u * 64 * N + __builtin_ctz(same);
                        }
                        count = min(count + all, a.top);
                    }
                }
            }
        }
    }
    own = across_wave(own, c);
    if constexpr (TOP) count = keep_best(mine, count, a.top);
    if (lane == 0) {
        sums[wave] = own;
        counts[wave] = count;
    }
    __syncthreads();
    Sums all = sums[0];
    float m = all.m;
#pragma unroll
    for (int w = 1; w < kWaves; ++w) m = top_of(m, sums[w].m);
    all.rescale(m, c);
#pragma unroll
    for (int w = 1; w < kWaves; ++w) {
        Sums o = sums[w];
        o.rescale(m, c);
        all.s += o.s;
        all.t += o.t;
    }
    const float log_s = log_sum(all);
    const Parts out = parts_in(a.workspace, (int64_t)a.rows * parts, a.top);
    const int64_t slot = (int64_t)row * parts + p;
    if (threadIdx.x == 0) {
        if (parts == 1) write_row(a, row, all, log_s);
        else out.sums[slot] = all;
    }
    if constexpr (TOP) {
        // a candidate's place: those before it in every wave's sorted list
        const int w = threadIdx.x / kMaxTop, i = threadIdx.x % kMaxTop;
        int total = 0;
#pragma unroll
        for (int o = 0; o < kWaves; ++o) total += counts[o];
        if (w < kWaves && i < counts[w]) {
            const uint32_t k = best[w].key[i];
            const int id = best[w].id[i];
            int place = i;
#pragma unroll
            for (int o = 0; o < kWaves; ++o)
                if (o != w)
                    for (int j = 0; j < counts[o] && before(best[o].key[j], best[o].id[j], k, id); ++j) ++place;
            if (place < a.top) {
                if (parts == 1) {
                    write_top(a, row, place, k, id, all.m, log_s);
                } else {
                    out.keys[slot * a.top + place] = k;
                    out.ids[slot * a.top + place] = id;
                }
            }
        }
        if (parts > 1 && threadIdx.x >= total && threadIdx.x < a.top) out.keys[slot * a.top + threadIdx.x] = 0;      // no further ones
    }
}

// A row's parts together: a wave a row, a lane a part (at most 64).  Their sorted lists are merged from their heads.
template <bool TOP>
__global__ __launch_bounds__(64) void logprobs_join_kernel(LogprobArgs a, int parts) {
    __shared__ uint32_t keys[TOP ? 64 * kMaxTop : 1];
    __shared__ int ids[TOP ? 64 * kMaxTop : 1];
    const int row = blockIdx.x, lane = threadIdx.x;
    const Parts in = parts_in(a.workspace, (int64_t)a.rows * parts, a.top);
    const int64_t slot = (int64_t)row * parts;
    if constexpr (TOP) {
        for (int i = lane; i < parts * a.top; i += 64) {
            keys[i] = in.keys[slot * a.top + i];
            ids[i] = in.ids[slot * a.top + i];
        }
    }
    Sums own{-INFINITY, 0.f, 0.f};
    if (lane < parts) own = in.sums[slot + lane];
    own = across_wave(own, a.scale * kLog2e);
    const float log_s = log_sum(own);
    if (lane == 0) write_row(a, row, own, log_s);
    if constexpr (TOP) {
        __syncthreads();
        int at = 0;
        for (int place = 0; place < a.top; ++place) {
            uint32_t k = lane < parts && at < a.top ? keys[lane * a.top + at] : 0;
            int id = k ? ids[lane * a.top + at] : 0x7fffffff;
            const uint32_t k0 = k;
            const int id0 = id;
#pragma unroll
            for (int s = 32; s >= 1; s >>= 1) {
                const uint32_t ok = __shfl_xor(k, s);
                const int oid = __shfl_xor(id, s);
                if (before(ok, oid, k, id)) {
                    k = ok;
                    id = oid;
                }
            }
            if (k0 && k0 == k && id0 == id) ++at;
            if (lane == 0) write_top(a, row, place, k, id, own.m, log_s);
        }
    }
}

// The gradient: a workgroup takes kGradTile elements of a row.
template <bool F32>
__global__ __launch_bounds__(kThreads) void logprobs_grad_kernel(LogprobGradArgs a, int segments) {
    constexpr int N = Piece<F32>::N, kUnits = 4, kTile = kThreads * N * kUnits, ES = F32 ? 4 : 2;
    const int row = blockIdx.x / segments, at = (blockIdx.x - row * segments) * kTile;
    const float m = a.stats[2 * row], log_s = a.stats[2 * row + 1];
    const int64_t token = a.tokens[row];
    const bool given = token >= 0 && token < a.vocab;
    const float gl = given && a.grad_logprobs ? a.grad_logprobs[row] : 0.f, gh = a.grad_entropy ? a.grad_entropy[row] : 0.f;
    const float h = a.grad_entropy ? a.entropy[row] : 0.f;
    const bool empty = m == -INFINITY;
    const char *x = static_cast<const char *>(a.logits) + row * a.stride * ES;
    char *out = static_cast<char *>(a.out) + row * a.out_stride * ES;
    Piece<F32> v[kUnits];
#pragma unroll
    for (int u = 0; u < kUnits; ++u) {
        const int e0 = at + (u * kThreads + threadIdx.x) * N;
        v[u].load(x + (int64_t)e0 * ES, a.vocab - e0);
    }
#pragma unroll
    for (int u = 0; u < kUnits; ++u) {
        const int e0 = at + (u * kThreads + threadIdx.x) * N;
        float g[N];
#pragma unroll
        for (int e = 0; e < N; ++e) {
            const float lp = fmaf(v[u].value(e) - m, a.scale, -log_s), p = __builtin_amdgcn_exp2f(lp * kLog2e);
            float d = p * fmaf(-gh, fmaxf(lp, -1e4f) + h, -gl);      // p is 0 long before
            if (given && e0 + e == token) d += gl;
            g[e] = empty ? 0.f : a.scale * d;
        }
        u32x4 w;
        if constexpr (F32) w = u32x4{__float_as_uint(g[0]), __float_as_uint(g[1]), __float_as_uint(g[2]), __float_as_uint(g[3])};
        else w = u32x4{pack2(g[0], g[1]), pack2(g[2], g[3]), pack2(g[4 % N], g[5 % N]), pack2(g[6 % N], g[7 % N])};
        if (e0 + N <= a.vocab) {
            *reinterpret_cast<u32x4_any *>(out + (int64_t)e0 * ES) = w;
        } else {
#pragma unroll
            for (int e = 0; e < N; ++e) {
                if (e0 + e >= a.vocab) continue;
                if constexpr (F32) reinterpret_cast<float *>(out)[e0 + e] = g[e];
                else reinterpret_cast<bf16_t *>(out)[e0 + e] = f32_to_bf16(g[e]);
            }
        }
    }
}

// Few rows are cut into parts that the whole chip works on, each of at least kLeastPart elements.
constexpr int kLeastPart = 8192;

int parts_of(int rows, int vocab) {
    const int most = std::min(64, (vocab + kLeastPart - 1) / kLeastPart);
    return std::max(1, std::min(most, 1024 / std::max(rows, 1)));
}

}  // namespace

size_t logprobs_workspace(int rows, int vocab, int top) {
    const int parts = parts_of(rows, vocab);
    return parts == 1 ? 0 : (size_t)rows * parts * (sizeof(Sums) + (size_t)top * 8);
}

hipError_t launch_logprobs(const LogprobArgs &a, hipStream_t stream) {
    const int parts = parts_of(a.rows, a.vocab);
    const int part = ((a.vocab + parts - 1) / parts + 7) / 8 * 8;
    const dim3 grid((unsigned)((int64_t)a.rows * parts));
    auto launch = [&](auto kernel) { return launch_kernel(kernel, grid, dim3(kThreads), stream, a, parts, part); };
    const hipError_t e = a.f32 ? (a.top ? launch(logprobs_kernel<true, true>) : launch(logprobs_kernel<true, false>))
                               : (a.top ? launch(logprobs_kernel<false, true>) : launch(logprobs_kernel<false, false>));
    if (e != hipSuccess || parts == 1) return e;
    return a.top ? launch_kernel(logprobs_join_kernel<true>, dim3(a.rows), dim3(64), stream, a, parts)
                 : launch_kernel(logprobs_join_kernel<false>, dim3(a.rows), dim3(64), stream, a, parts);
}

hipError_t launch_logprobs_grad(const LogprobGradArgs &a, hipStream_t stream) {
    const int tile = kThreads * 4 * (a.f32 ? 4 : 8), segments = (a.vocab + tile - 1) / tile;
    const dim3 grid((unsigned)((int64_t)a.rows * segments));
    return a.f32 ? launch_kernel(logprobs_grad_kernel<true>, grid, dim3(kThreads), stream, a, segments)
                 : launch_kernel(logprobs_grad_kernel<false>, grid, dim3(kThreads), stream, a, segments);
}

}  // namespace iefwd
