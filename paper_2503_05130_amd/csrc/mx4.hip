// Matrices in microscaled 4 bits for gfx950: quantisation, layout and values.
#include "mx4.h"

#include <algorithm>

#include "mx4_device.h"

namespace iefwd {
namespace {

constexpr int kWaves = 4;      // of a workgroup at most

// ------------------------------------------------------------------------------ to the form and back
//
// A block's scale byte is max(exponent field of its largest magnitude - 2, 0); v_cvt_scalef32_pk_fp4 divides by 2^(byte - 127),
// rounds to the nearest (ties to even codes) and cuts off at 6, the inverse conversion is exact.  Bound by bytes: 8191 x 8192 bf16
// become codes in 28.6 us (5.95 TB/s) and codes bf16 in 25.9 (6.6, the codes from the last cache); few rows by
// latency: one of 2048 in 3.1 and 1.5 us.
//
// A wave takes a row tile's 4 chunks, 16 rows x 512 columns: a row's 512 columns are one load of 16 bytes a lane (two
// in fp32), so that 4 lanes hold a block and neighbouring lanes neighbouring addresses.  The codes change places in 4
// KB of LDS of the wave's own, and leave as whole 1 KB blocks.  Place p of block c and chunk s in the wave's LDS is
// turned by c + 4 s, which spreads the 16 pieces of a row over the banks.
__device__ inline int turned(int r, int c, int s) { return s * 1024 + (c * 16 + ((r + c + 4 * s) & 15)) * 16; }

// VECTOR: rows begin at multiples of 16 bytes and have a multiple of 8 elements.  FAR: more than the caches hold (far_reads).
template <bool F32, bool VECTOR, bool FAR>
__device__ inline Eight load_eight(const void *row, int col, int K) {
    Eight x = {};
    if (VECTOR) {
        if (col < K) {
            const u32x4 *p = reinterpret_cast<const u32x4 *>(static_cast<const char *>(row) + (size_t)col * (F32 ? 4 : 2));
            x.lo = FAR ? __builtin_nontemporal_load(p) : p[0];
            if (F32) x.hi = FAR ? __builtin_nontemporal_load(p + 1) : p[1];
        }
    } else {
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            if (col + e >= K) continue;
            if (F32) {
                const uint32_t v = static_cast<const uint32_t *>(row)[col + e];
                if (e < 4) x.lo[e] = v;
                else x.hi[e - 4] = v;
            } else {
                x.lo[e / 2] |= (uint32_t) static_cast<const uint16_t *>(row)[col + e] << (16 * (e & 1));
            }
        }
    }
    return x;
}

template <bool F32, bool VECTOR, bool FAR>
__global__ __launch_bounds__(64 * kWaves) void mx4_quantize_kernel(const char *__restrict__ x, int64_t row_bytes,
                                                                   char *__restrict__ dst, int rows, int K, int64_t items) {
    __shared__ __attribute__((aligned(16))) char lds[kWaves][4096 + 256];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int64_t item = (int64_t)blockIdx.x * (blockDim.x >> 6) + wave;
    if (item >= items) return;
    const int chunks = mx4_chunks(K), groups = (chunks + 3) / 4;
    const int tile = (int)(item / groups), g = (int)(item - (int64_t)tile * groups);
    const int s = lane >> 4, c = (lane >> 2) & 3, part = lane & 3, col = 512 * g + 8 * lane;
    const int n = min(16, rows - 16 * tile);
    const char *row0 = x + (int64_t)tile * 16 * row_bytes;
    char *stage = lds[wave];
    constexpr int kAhead = F32 ? 4 : 8;      // rows whose loads are on their way together
    for (int r0 = 0; r0 < 16; r0 += kAhead) {
        Eight v[kAhead];
#pragma unroll
        for (int i = 0; i < kAhead; ++i) {
            v[i] = Eight{};
            if (r0 + i < n) v[i] = load_eight<F32, VECTOR, FAR>(row0 + (r0 + i) * row_bytes, col, K);
        }
#pragma unroll
        for (int i = 0; i < kAhead; ++i) {
            const int r = r0 + i;
            const uint32_t scale = mx4_scale<F32>(v[i]);
            *reinterpret_cast<uint32_t *>(stage + turned(r, c, s) + part * 4) = mx4_codes<F32>(v[i], scale);
            if (part == 0) stage[4096 + (r + 16 * c) * 4 + s] = (char)scale;
        }
    }
    wave_lds_fence();
    char *out = dst + (size_t)tile * mx4_tile_bytes(K);
    const int r = lane & 15, cc = lane >> 4;
#pragma unroll
    for (int j = 0; j < 4; ++j)
        if (4 * g + j < chunks)
            *reinterpret_cast<u32x4 *>(out + (size_t)(4 * g + j) * 1024 + lane * 16) =
                *reinterpret_cast<const u32x4 *>(stage + turned(r, cc, j));
    *reinterpret_cast<uint32_t *>(out + (size_t)chunks * 1024 + (size_t)g * 256 + lane * 4) =
        *reinterpret_cast<const uint32_t *>(stage + 4096 + lane * 4);
}

template <bool F32, bool VECTOR, bool FAR>
__global__ __launch_bounds__(64 * kWaves) void mx4_values_kernel(const char *__restrict__ src, char *__restrict__ out,
                                                                 int64_t row_bytes, int rows, int K, int64_t items) {
    __shared__ __attribute__((aligned(16))) char lds[kWaves][4096 + 256];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int64_t item = (int64_t)blockIdx.x * (blockDim.x >> 6) + wave;
    if (item >= items) return;
    const int chunks = mx4_chunks(K), groups = (chunks + 3) / 4;
    const int tile = (int)(item / groups), g = (int)(item - (int64_t)tile * groups);
    const char *in = src + (size_t)tile * mx4_tile_bytes(K);
    char *stage = lds[wave];
    {
        const int r = lane & 15, c = lane >> 4;
        u32x4 w[4];
#pragma unroll
        for (int j = 0; j < 4; ++j)
            w[j] = *reinterpret_cast<const u32x4 *>(in + (size_t)min(4 * g + j, chunks - 1) * 1024 + lane * 16);
        const uint32_t scales = *reinterpret_cast<const uint32_t *>(in + (size_t)chunks * 1024 + (size_t)g * 256 + lane * 4);
#pragma unroll
        for (int j = 0; j < 4; ++j) *reinterpret_cast<u32x4 *>(stage + turned(r, c, j)) = w[j];
        *reinterpret_cast<uint32_t *>(stage + 4096 + lane * 4) = scales;
    }
    wave_lds_fence();
    const int s = lane >> 4, c = (lane >> 2) & 3, part = lane & 3, col = 512 * g + 8 * lane;
    if (col >= K) return;
    const int n = min(16, rows - 16 * tile);
    for (int r = 0; r < n; ++r) {
        const uint32_t codes = *reinterpret_cast<const uint32_t *>(stage + turned(r, c, s) + part * 4);
        const uint32_t scale = (uint8_t)stage[4096 + (r + 16 * c) * 4 + s];
        char *row = out + (int64_t)(tile * 16 + r) * row_bytes;
        if constexpr (F32) {
            const float sc = __uint_as_float(scale << 23);
            const f32x2 v[4] = {
                __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(codes, sc, 0), __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(codes, sc, 1),
                __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(codes, sc, 2), __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(codes, sc, 3)};
            float *p = reinterpret_cast<float *>(row) + col;
            if (VECTOR) {
                *reinterpret_cast<f32x4 *>(p) = f32x4{v[0][0], v[0][1], v[1][0], v[1][1]};
                *reinterpret_cast<f32x4 *>(p + 4) = f32x4{v[2][0], v[2][1], v[3][0], v[3][1]};
            } else {
#pragma unroll
                for (int e = 0; e < 8; ++e)
                    if (col + e < K) p[e] = v[e / 2][e % 2];
            }
        } else {
            const u32x4 v = mx4_bf16(codes, scale);
            bf16_t *p = reinterpret_cast<bf16_t *>(row) + col;
            if (VECTOR) {
                if (FAR) __builtin_nontemporal_store(v, reinterpret_cast<u32x4 *>(p));
                else *reinterpret_cast<u32x4 *>(p) = v;
            } else {
#pragma unroll
                for (int e = 0; e < 8; ++e)
                    if (col + e < K) p[e] = (bf16_t)(v[e / 2] >> (16 * (e & 1)));
            }
        }
    }
}

// A thread: 4 chunks of a lane, from row-major codes and scales.  8192 x 8192 in 14.1 us (5.1 TB/s, the last cache holding both sides).
__global__ __launch_bounds__(256) void mx4_pack_kernel(const uint8_t *__restrict__ codes, const uint8_t *__restrict__ scales,
                                                       char *__restrict__ dst, int rows, int K, int64_t threads) {
    const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x;
    if (i >= threads) return;
    const int chunks = mx4_chunks(K), groups = (chunks + 3) / 4, lane = (int)(i & 63);
    const int64_t item = i >> 6;
    const int tile = (int)(item / groups), g = (int)(item - (int64_t)tile * groups);
    const int row = tile * 16 + (lane & 15);
    char *out = dst + (size_t)tile * mx4_tile_bytes(K);
    uint32_t bytes = 0;
#pragma unroll
    for (int s = 0; s < 4; ++s) {
        if (4 * g + s >= chunks) break;
        const int col = (4 * g + s) * 128 + 32 * (lane >> 4);
        u32x4 w = {0, 0, 0, 0};
        if (row < rows && col < K) {
            w = *reinterpret_cast<const u32x4 *>(codes + ((size_t)row * K + col) / 2);
            bytes |= (uint32_t)scales[((size_t)row * K + col) / 32] << (8 * s);
        }
        *reinterpret_cast<u32x4 *>(out + (size_t)(4 * g + s) * 1024 + lane * 16) = w;
    }
    *reinterpret_cast<uint32_t *>(out + (size_t)chunks * 1024 + (size_t)g * 256 + lane * 4) = bytes;
}

// What a call reads once and what it writes for later goes past the last cache from here on.  Quantised and back, bf16, us,
// without a hint / stores / loads / both:
//   2000 x 8192  16.9  16.7  17.6  17.4      4000 x 8192  38.4  28.6  29.8  30.7
//   6000 x 8192  51.3  44.8  43.6  43.1      8191 x 8192  68.5  61.6  58.1  55.6
constexpr int64_t kFarReads = 96 << 20, kFarWrites = 32 << 20;

int64_t items_of(int rows, int K) { return (int64_t)((rows + 15) / 16) * ((mx4_chunks(K) + 3) / 4); }

// A wave a workgroup spreads few items over the chip: 100 x 2048 there and back 6.7 -> 6.3 us; many of them are better off in fours
// (4000 x 8192 of fp32 63 -> 70), and 4 items as one workgroup (1 x 2048 5.1, else 5.4).
int waves_of(int64_t items) { return items > 4 && items <= 2048 ? 1 : kWaves; }

}  // namespace

hipError_t launch_mx4_quantize(bool f32, const void *x, int64_t stride, void *dst, int rows, int K, hipStream_t stream) {
    const int es = f32 ? 4 : 2;
    const int64_t items = items_of(rows, K);
    const int waves = waves_of(items);
    const dim3 grid((unsigned)((items + waves - 1) / waves)), block(64 * waves);
    const bool vector = K % 8 == 0 && stride * es % 16 == 0 && (uintptr_t)x % 16 == 0;
    const bool far = (int64_t)rows * K * es > kFarReads;
    auto launch = [&](auto kernel) {
        return launch_kernel(kernel, grid, block, stream, static_cast<const char *>(x), stride * es, static_cast<char *>(dst),
                             rows, K, items);
    };
    if (!vector) return f32 ? launch(mx4_quantize_kernel<true, false, false>) : launch(mx4_quantize_kernel<false, false, false>);
    if (f32) return far ? launch(mx4_quantize_kernel<true, true, true>) : launch(mx4_quantize_kernel<true, true, false>);
    return far ? launch(mx4_quantize_kernel<false, true, true>) : launch(mx4_quantize_kernel<false, true, false>);
}

hipError_t launch_mx4_pack(const uint8_t *codes, const uint8_t *scales, void *dst, int rows, int K, hipStream_t stream) {
    const int64_t threads = (int64_t)((rows + 15) / 16) * ((mx4_chunks(K) + 3) / 4) * 64;
    return launch_kernel(mx4_pack_kernel, dim3((unsigned)((threads + 255) / 256)), dim3(256), stream, codes, scales,
                         static_cast<char *>(dst), rows, K, threads);
}

hipError_t launch_mx4_values(const void *src, bool f32, void *out, int64_t stride, int rows, int K, hipStream_t stream) {
    const int es = f32 ? 4 : 2;
    const int64_t items = items_of(rows, K);
    const int waves = waves_of(items);
    const dim3 grid((unsigned)((items + waves - 1) / waves)), block(64 * waves);
    const bool vector = K % 8 == 0 && stride * es % 16 == 0 && (uintptr_t)out % 16 == 0;
    auto launch = [&](auto kernel) {
        return launch_kernel(kernel, grid, block, stream, static_cast<const char *>(src), static_cast<char *>(out), stride * es,
                             rows, K, items);
    };
    // fp32: a lane's two stores leave halves of the lines, which the hint makes 91 us of 63 for 4000 x 8192
    if (f32) return vector ? launch(mx4_values_kernel<true, true, false>) : launch(mx4_values_kernel<true, false, false>);
    if (!vector) return launch(mx4_values_kernel<false, false, false>);
    return (int64_t)rows * K * es >= kFarWrites ? launch(mx4_values_kernel<false, true, true>)
                                                : launch(mx4_values_kernel<false, true, false>);
}

}  // namespace iefwd
