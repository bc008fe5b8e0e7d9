// Matrices in microscaled 4 bits for gfx950: quantisation, layout, values and products.
#include "mx4.h"

#include <algorithm>

#include "mx4_device.h"

namespace iefwd {
namespace {

constexpr int kWaves = 4;

// ------------------------------------------------------------------------------ to the form and back
//
// A wave takes a row tile's 4 chunks, 16 rows x 512 columns: a row's 512 columns are one load of 16 bytes a lane (two
// in fp32), so that 4 lanes hold a block and neighbouring lanes neighbouring addresses.  The codes change places in 4
// KB of LDS of the wave's own, and leave as whole 1 KB blocks.  Place p of block c and chunk s in the wave's LDS is
// turned by c + 4 s, which spreads the 16 pieces of a row over the banks.
__device__ inline int turned(int r, int c, int s) { return s * 1024 + (c * 16 + ((r + c + 4 * s) & 15)) * 16; }

// VECTOR: rows begin at multiples of 16 bytes and have a multiple of 8 elements.
template <bool F32, bool VECTOR>
__device__ inline Eight load_eight(const void *row, int col, int K) {
    Eight x = {};
    if (VECTOR) {
        if (col < K) {
            const u32x4 *p = reinterpret_cast<const u32x4 *>(static_cast<const char *>(row) + (size_t)col * (F32 ? 4 : 2));
            x.lo = p[0];
            if (F32) x.hi = p[1];
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

template <bool F32, bool VECTOR>
__global__ __launch_bounds__(64 * kWaves) void mx4_quantize_kernel(const char *__restrict__ x, int64_t row_bytes,
                                                                   char *__restrict__ dst, int rows, int K, int64_t items) {
    __shared__ __attribute__((aligned(16))) char lds[kWaves][4096 + 256];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int64_t item = (int64_t)blockIdx.x * kWaves + wave;
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
            if (r0 + i < n) v[i] = load_eight<F32, VECTOR>(row0 + (r0 + i) * row_bytes, col, K);
        }
#pragma unroll
        for (int i = 0; i < kAhead; ++i) {
            const int r = r0 + i;
            const uint32_t scale = mx4_scale<F32>(v[i]);
            *reinterpret_cast<uint32_t *>(stage + turned(r, c, s) + part * 4) = mx4_codes<F32>(v[i], scale);
            if (part == 0) stage[4096 + (r + 16 * c) * 4 + s] = (char)scale;
        }
    }
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

template <bool F32, bool VECTOR>
__global__ __launch_bounds__(64 * kWaves) void mx4_values_kernel(const char *__restrict__ src, char *__restrict__ out,
                                                                 int64_t row_bytes, int rows, int K, int64_t items) {
    __shared__ __attribute__((aligned(16))) char lds[kWaves][4096 + 256];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int64_t item = (int64_t)blockIdx.x * kWaves + wave;
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
    const int s = lane >> 4, c = (lane >> 2) & 3, part = lane & 3, col = 512 * g + 8 * lane;
    if (col >= K) return;
    const int n = min(16, rows - 16 * tile);
    for (int r = 0; r < n; ++r) {
        const uint32_t codes = *reinterpret_cast<const uint32_t *>(stage + turned(r, c, s) + part * 4);
        const uint32_t scale = (uint8_t)stage[4096 + (r + 16 * c) * 4 + s];
        char *row = out + (int64_t)(tile * 16 + r) * row_bytes;
        if constexpr (F32) {
            const float sc = __uint_as_float(scale << 23);
            const f32x2 v[4] = {__builtin_amdgcn_cvt_scalef32_pk_f32_fp4(codes, sc, 0), __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(codes, sc, 1),
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
                *reinterpret_cast<u32x4 *>(p) = v;
            } else {
#pragma unroll
                for (int e = 0; e < 8; ++e)
                    if (col + e < K) p[e] = (bf16_t)(v[e / 2] >> (16 * (e & 1)));
            }
        }
    }
}

// A thread: 4 chunks of a lane, from row-major codes and scales.
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

// ------------------------------------------------------------------------------ products
//
// out^T = W A^T on the matrix cores, which take the codes and the scales as they are stored: a product of 16 features x 16
// rows x 128 of K is one instruction of two 16-byte operands and a scale byte a lane, exact products summed in fp32.
struct Mx4Params {
    const char *a, *w;
    const bf16_t *a16;           // A in bf16 instead
    const bf16_t *bias;
    const float *resid;
    void *out;
    int M, N, K;
    int row_tiles;               // workgroups' tiles along M
    Epi epi;
};

// Four features n .. n + 3 of row m.
__device__ inline void mx4_store(const Mx4Params &p, int m, int n, f32x4 v) {
    if (m >= p.M) return;
    const int count = min(4, p.N - n);
#pragma unroll
    for (int e = 0; e < 4; ++e)
        if (e < count && p.bias) v[e] += __uint_as_float((uint32_t)p.bias[n + e] << 16);
    const size_t i = (size_t)m * p.N + n;
    if (p.epi == Epi::BiasResidF32) {
        float *out = static_cast<float *>(p.out) + i;
        if ((p.N & 3) == 0) {
            if (count > 0) *reinterpret_cast<f32x4 *>(out) = *reinterpret_cast<const f32x4 *>(p.resid + i) + v;
        } else {
#pragma unroll
            for (int e = 0; e < 4; ++e)
                if (e < count) out[e] = p.resid[i + e] + v[e];
        }
        return;
    }
    if (p.epi == Epi::BiasGeluBf16)
#pragma unroll
        for (int e = 0; e < 4; ++e) v[e] = gelu(v[e]);
    bf16_t *out = static_cast<bf16_t *>(p.out) + i;
    if ((p.N & 3) == 0) {
        if (count > 0) *reinterpret_cast<u32x2 *>(out) = u32x2{pack2(v[0], v[1]), pack2(v[2], v[3])};
    } else {
#pragma unroll
        for (int e = 0; e < 4; ++e)
            if (e < count) out[e] = f32_to_bf16(v[e]);
    }
}

// A workgroup's tile of 16 FT features x 16 RT rows with K spread over its waves, chunk by chunk, and the waves' sums
// added in wave order through LDS.  Operands go from memory to registers.  NL > 0: A is bf16, 4 NL >= M rows: a chunk of them is loaded in
// rows, quantised by quads of lanes and laid out as the operand in the wave's LDS.
template <int FT, int RT, int WAVES, int NL>
__global__ __launch_bounds__(64 * WAVES) void mx4_split_kernel(Mx4Params p) {
    static_assert(NL == 0 || RT == 1, "bf16 rows are one tile");
    constexpr int kStage = 1024 + 64;
    constexpr int kLds = WAVES * FT * RT * 1024 > WAVES * kStage || NL == 0 ? WAVES * FT * RT * 1024 : WAVES * kStage;
    __shared__ __attribute__((aligned(16))) char lds[kLds];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int r = lane & 15, c = lane >> 4;
    const int chunks = mx4_chunks(p.K);
    const size_t tile_bytes = mx4_tile_bytes(p.K);
    const int ft0 = blockIdx.x / p.row_tiles * FT, rt0 = blockIdx.x % p.row_tiles * RT;
    const int last_f = (p.N + 15) / 16 - 1, last_r = (p.M + 15) / 16 - 1;
    const char *w[FT], *a[RT];      // a tile past the last reads the last one and is not stored
#pragma unroll
    for (int f = 0; f < FT; ++f) w[f] = p.w + (size_t)min(ft0 + f, last_f) * tile_bytes;
    if (NL == 0)
#pragma unroll
        for (int t = 0; t < RT; ++t) a[t] = p.a + (size_t)min(rt0 + t, last_r) * tile_bytes;
    char *stage = lds + wave * kStage;
    f32x4 acc[FT][RT] = {};
    for (int j = wave; j < chunks; j += WAVES) {
        const size_t scales = (size_t)chunks * 1024 + (size_t)(j >> 2) * 256 + lane * 4;
        const int shift = 8 * (j & 3);
        u32x4 wf[FT], af[RT];
        uint32_t ws[FT], as[RT];
#pragma unroll
        for (int f = 0; f < FT; ++f) {
            wf[f] = *reinterpret_cast<const u32x4 *>(w[f] + (size_t)j * 1024 + lane * 16);
            ws[f] = *reinterpret_cast<const uint32_t *>(w[f] + scales) >> shift;
        }
        if constexpr (NL == 0) {
#pragma unroll
            for (int t = 0; t < RT; ++t) {
                af[t] = *reinterpret_cast<const u32x4 *>(a[t] + (size_t)j * 1024 + lane * 16);
                as[t] = *reinterpret_cast<const uint32_t *>(a[t] + scales) >> shift;
            }
        } else {
            const int piece = lane & 15, col = j * 128 + 8 * piece;
            Eight x[NL];
#pragma unroll
            for (int i = 0; i < NL; ++i) {
                x[i] = Eight{};
                if (col < p.K)
                    x[i].lo = *reinterpret_cast<const u32x4 *>(p.a16 + (size_t)min(4 * i + (lane >> 4), p.M - 1) * p.K + col);
            }
#pragma unroll
            for (int i = 0; i < NL; ++i) {
                const int row = 4 * i + (lane >> 4), at = row + 16 * (piece >> 2);
                const uint32_t scale = mx4_scale<false>(x[i]);
                *reinterpret_cast<uint32_t *>(stage + at * 16 + (piece & 3) * 4) = mx4_codes<false>(x[i], scale);
                if ((piece & 3) == 0) stage[1024 + at] = (char)scale;
            }
            // columns of rows past 4 NL hold whatever was there: they are sums of their own and not stored
            af[0] = *reinterpret_cast<const u32x4 *>(stage + lane * 16);
            as[0] = (uint8_t)stage[1024 + lane];
        }
#pragma unroll
        for (int f = 0; f < FT; ++f)
#pragma unroll
            for (int t = 0; t < RT; ++t) acc[f][t] = mfma_mx4(wf[f], af[t], acc[f][t], ws[f], as[t]);
    }
    __syncthreads();
    f32x4 (*part)[FT * RT][64] = reinterpret_cast<f32x4 (*)[FT * RT][64]>(lds);
#pragma unroll
    for (int f = 0; f < FT; ++f)
#pragma unroll
        for (int t = 0; t < RT; ++t) part[wave][f * RT + t][lane] = acc[f][t];
    __syncthreads();
    for (int b = wave; b < FT * RT; b += WAVES) {
        f32x4 v = part[0][b][lane];
#pragma unroll
        for (int i = 1; i < WAVES; ++i) v += part[i][b][lane];
        mx4_store(p, (rt0 + b % RT) * 16 + r, (ft0 + b / RT) * 16 + 4 * c, v);
    }
}

template <int FT, int RT, int WAVES, int NL>
hipError_t launch_split(Mx4Params p, hipStream_t stream) {
    const int f_groups = ((p.N + 15) / 16 + FT - 1) / FT;
    p.row_tiles = ((p.M + 15) / 16 + RT - 1) / RT;
    return launch_kernel(mx4_split_kernel<FT, RT, WAVES, NL>, dim3((unsigned)((int64_t)f_groups * p.row_tiles)),
                         dim3(64 * WAVES), stream, p);
}

}  // namespace

hipError_t launch_mx4_quantize(bool f32, const void *x, int64_t stride, void *dst, int rows, int K, hipStream_t stream) {
    const int es = f32 ? 4 : 2;
    const int64_t items = (int64_t)((rows + 15) / 16) * ((mx4_chunks(K) + 3) / 4);
    const dim3 grid((unsigned)((items + kWaves - 1) / kWaves)), block(64 * kWaves);
    const bool vector = K % 8 == 0 && stride * es % 16 == 0 && (uintptr_t)x % 16 == 0;
    auto launch = [&](auto kernel) {
        return launch_kernel(kernel, grid, block, stream, static_cast<const char *>(x), stride * es, static_cast<char *>(dst),
                             rows, K, items);
    };
    if (f32) return vector ? launch(mx4_quantize_kernel<true, true>) : launch(mx4_quantize_kernel<true, false>);
    return vector ? launch(mx4_quantize_kernel<false, true>) : launch(mx4_quantize_kernel<false, false>);
}

hipError_t launch_mx4_pack(const uint8_t *codes, const uint8_t *scales, void *dst, int rows, int K, hipStream_t stream) {
    const int64_t threads = (int64_t)((rows + 15) / 16) * ((mx4_chunks(K) + 3) / 4) * 64;
    return launch_kernel(mx4_pack_kernel, dim3((unsigned)((threads + 255) / 256)), dim3(256), stream, codes, scales,
                         static_cast<char *>(dst), rows, K, threads);
}

hipError_t launch_mx4_values(const void *src, bool f32, void *out, int64_t stride, int rows, int K, hipStream_t stream) {
    const int es = f32 ? 4 : 2;
    const int64_t items = (int64_t)((rows + 15) / 16) * ((mx4_chunks(K) + 3) / 4);
    const dim3 grid((unsigned)((items + kWaves - 1) / kWaves)), block(64 * kWaves);
    const bool vector = K % 8 == 0 && stride * es % 16 == 0 && (uintptr_t)out % 16 == 0;
    auto launch = [&](auto kernel) {
        return launch_kernel(kernel, grid, block, stream, static_cast<const char *>(src), static_cast<char *>(out), stride * es,
                             rows, K, items);
    };
    if (f32) return vector ? launch(mx4_values_kernel<true, true>) : launch(mx4_values_kernel<true, false>);
    return vector ? launch(mx4_values_kernel<false, true>) : launch(mx4_values_kernel<false, false>);
}

hipError_t launch_mx4_gemm(Epi epi, const void *a, const void *w, const bf16_t *bias, const float *resid, void *out, int M,
                           int N, int K, hipStream_t stream) {
    Mx4Params p{static_cast<const char *>(a), static_cast<const char *>(w), nullptr, bias, resid, out, M, N, K, 0, epi};
    if (M <= 16) return launch_split<1, 1, 8, 0>(p, stream);
    if (M <= 32) return launch_split<2, 2, 8, 0>(p, stream);
    return launch_split<4, 4, 4, 0>(p, stream);
}

hipError_t launch_mx4_gemm_bf16(Epi epi, const bf16_t *a, const void *w, const bf16_t *bias, const float *resid, void *out,
                                int M, int N, int K, hipStream_t stream) {
    Mx4Params p{nullptr, static_cast<const char *>(w), a, bias, resid, out, M, N, K, 0, epi};
    if (M <= 4) return launch_split<1, 1, 8, 1>(p, stream);
    if (M <= 8) return launch_split<1, 1, 8, 2>(p, stream);
    return launch_split<1, 1, 8, 4>(p, stream);
}

}  // namespace iefwd
