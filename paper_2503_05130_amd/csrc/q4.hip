// Products of a decode step with 4-bit weights for gfx950:
// out = epilogue(A W^T + b), W[n][k] = s[n][g] (code[n][k] - z[n][g]), g = k / group,
// for at most 16 rows of A.  Bound by reading the codes once.
//
// The codes go to the matrix cores as bf16 numbers 16 + code: the four bits are
// set into the mantissa of 16.0 (16 (1 + code / 16) = 16 + code), which is exact and
// takes a shift and one and-or for two weights.  Per group g the product then is
//   s_g (sum_k a_k (16 + code_k) - (16 + z_g) sum_k a_k),
// the second sum from a matrix product with ones.  Both sums are fp32; the
// subtraction cancels at most the five bits that 16 + code has over code, so
// some 19 bits of the result are left.
#include "q4.h"

#include "gemm_device.h"

namespace iefwd {
namespace {

constexpr int kWaves = 8;
constexpr int kChunk = 128;      // weights of a feature in one block: 4 K steps of 32

struct Q4Params {
    const bf16_t *a;
    const u32x4 *codes;          // [N / 16][chunks][64 lanes]
    const uint32_t *meta;        // [N / 16][chunks][16 features][128 / group]
    const bf16_t *bias;
    const float *resid;
    void *out;
    int M, N, K, chunks;
};

// Lane l of a block holds of feature l % 16 the weights 32 s + 8 (l / 16) + e in
// word s, e = 0 .. 7; the even ones lie in the word's low half, the odd ones in
// its high half, so that a pair comes out as the two halves of a register.
template <int GROUP>
__global__ __launch_bounds__(256) void q4_pack_kernel(const uint8_t *codes, const bf16_t *scales, const uint8_t *zeros,
                                                      u32x4 *dst, uint32_t *meta, int N, int K, int chunks) {
    constexpr int GPC = kChunk / GROUP;
    const size_t i = (size_t)blockIdx.x * 256 + threadIdx.x;
    const size_t pieces = (size_t)N / 16 * chunks * 64;
    if (i >= pieces) return;
    const int l = (int)(i % 64);
    const size_t block = i / 64;
    const int chunk = (int)(block % chunks), n = (int)(block / chunks) * 16 + l % 16;
    u32x4 out = {0, 0, 0, 0};
#pragma unroll
    for (int s = 0; s < 4; ++s) {
        const int k = chunk * kChunk + 32 * s + 8 * (l / 16);
        if (k < K)
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const uint32_t byte = codes[((size_t)n * K + k) / 2 + e];
                out[s] |= (byte & 15) << (4 * e) | (byte >> 4) << (16 + 4 * e);
            }
    }
    dst[i] = out;
    if (l / 16 < GPC) {      // this lane's group of the chunk
        const int g = l / 16, groups = K / GROUP, at = chunk * GPC + g;
        uint32_t w = 0;      // past K: scale 0
        if (at < groups) {
            const size_t j = (size_t)n * groups + at;
            const float off = 16.f + (zeros ? (float)(zeros[j] & 15) : 8.f);
            w = scales[j] | (__float_as_uint(off) & 0xffff0000u);
        }
        meta[(block * 16 + l % 16) * GPC + g] = w;
    }
}

template <int N>
__device__ inline bf16x8 rotate_rows(bf16x8 v) {     // lane i of each 16 gets lane (i - N) mod 16's value
    if constexpr (N == 0) return v;
    u32x4 w = __builtin_bit_cast(u32x4, v);
#pragma unroll
    for (int e = 0; e < 4; ++e) w[e] = __builtin_amdgcn_update_dpp(0, w[e], 0x120 + N, 0xf, 0xf, false);
    return __builtin_bit_cast(bf16x8, w);
}

__device__ inline bf16x8 widen(uint32_t x) {
    constexpr uint32_t mask = 0x00780078u, one = 0x41804180u;
    return __builtin_bit_cast(bf16x8, u32x4{((x << 3) & mask) | one, ((x >> 1) & mask) | one, ((x >> 5) & mask) | one,
                                            ((x >> 9) & mask) | one});
}

// MC: row class (4, 8 or 16 rows).  With at most 4 (8) rows a 16-byte load per lane
// takes a chunk's 4 (2) steps of all rows at once: lane column s MC + m holds
// row m's piece of step s, and a rotation within the 16 lanes brings it to
// columns 0 .. MC - 1, the only ones that are stored.
// T: tiles of 16 features a workgroup works on together.  U: chunks a wave requests at once.
template <int GROUP, int MC, int T, int U>
__global__ __launch_bounds__(64 * kWaves) void q4_kernel(Q4Params p, Epi epi) {
    constexpr int GPC = kChunk / GROUP, SPG = 4 / GPC;      // groups of a chunk, steps of a group
    constexpr int NL = MC / 4, SPL = 4 / NL;                // activation loads per chunk, steps per load
    __shared__ f32x4 part[kWaves * T][64];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int r = lane & 15, c = lane >> 4;
    const int tile0 = blockIdx.x * T;
    f32x4 acc[T] = {};
    const bf16x8 zero = {}, ones = __builtin_bit_cast(bf16x8, u32x4{0x3f803f80u, 0x3f803f80u, 0x3f803f80u, 0x3f803f80u});
    const bf16_t *arow = p.a + (size_t)min(r % MC, p.M - 1) * p.K;
    const int k_lane = 32 * (r / MC) + 8 * c;      // of this lane's piece in a chunk, plus 32 SPL per load

    bf16x8 af[U][NL];
    u32x4 wf[U][T];
    uint32_t mf[U][T][GPC];
    auto load = [&](int u, int j) {
#pragma unroll
        for (int i = 0; i < NL; ++i) {
            const int k = j * kChunk + 32 * SPL * i + k_lane;
            af[u][i] = *reinterpret_cast<const bf16x8 *>(arow + min(k, p.K - 8));
        }
#pragma unroll
        for (int t = 0; t < T; ++t) {
            const size_t block = (size_t)min(tile0 + t, p.N / 16 - 1) * p.chunks + j;
            wf[u][t] = p.codes[block * 64 + lane];
            const uint32_t *m = p.meta + (block * 16 + r) * GPC;
            if constexpr (GPC == 4) {
                const u32x4 x = *reinterpret_cast<const u32x4 *>(m);
#pragma unroll
                for (int g = 0; g < 4; ++g) mf[u][t][g] = x[g];
            } else if constexpr (GPC == 2) {
                const u32x2 x = *reinterpret_cast<const u32x2 *>(m);
                mf[u][t][0] = x[0];
                mf[u][t][1] = x[1];
            } else {
                mf[u][t][0] = *m;
            }
        }
    };
    auto use = [&](int u, int j) {
        bf16x8 a[4];
#pragma unroll
        for (int i = 0; i < NL; ++i) {
            bf16x8 x = af[u][i];
            // the part of the last chunk past K
            if (j * kChunk + 32 * SPL * i + k_lane >= p.K) x = zero;
            if constexpr (MC == 4) {
                a[0] = x;
                a[1] = rotate_rows<12>(x);
                a[2] = rotate_rows<8>(x);
                a[3] = rotate_rows<4>(x);
            } else if constexpr (MC == 8) {
                a[2 * i] = x;
                a[2 * i + 1] = rotate_rows<8>(x);
            } else {
                a[i] = x;
            }
        }
#pragma unroll
        for (int g = 0; g < GPC; ++g) {
            f32x4 sum = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int s = 0; s < SPG; ++s)
                sum = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a[g * SPG + s], ones, sum, 0, 0, 0);
#pragma unroll
            for (int t = 0; t < T; ++t) {
                f32x4 d = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
                for (int s = 0; s < SPG; ++s)
                    d = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a[g * SPG + s], widen(wf[u][t][g * SPG + s]), d, 0, 0, 0);
                const float scale = __uint_as_float(mf[u][t][g] << 16), off = __uint_as_float(mf[u][t][g] & 0xffff0000u);
#pragma unroll
                for (int e = 0; e < 4; ++e) acc[t][e] = fmaf(scale, fmaf(-off, sum[e], d[e]), acc[t][e]);
            }
        }
    };
    for (int j0 = wave; j0 < p.chunks; j0 += kWaves * U) {
#pragma unroll
        for (int u = 0; u < U; ++u) load(u, min(j0 + u * kWaves, p.chunks - 1));
#pragma unroll
        for (int u = 0; u < U; ++u)
            if (j0 + u * kWaves < p.chunks) use(u, j0 + u * kWaves);
    }
    // the waves' sums in wave order, wave t for tile t
#pragma unroll
    for (int t = 0; t < T; ++t) part[wave * T + t][lane] = acc[t];
    __syncthreads();
    const int n = (tile0 + wave) * 16 + r;
    if (wave >= T || n >= p.N) return;
    f32x4 sum = part[wave][lane];
#pragma unroll
    for (int w = 1; w < kWaves; ++w) sum += part[w * T + wave][lane];
    // this lane: feature n of rows 4 c .. 4 c + 3
    const float bias = p.bias ? __uint_as_float((uint32_t)p.bias[n] << 16) : 0.f;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        const int row = 4 * c + e;
        if (row >= p.M) break;
        const size_t i = (size_t)row * p.N + n;
        const float v = sum[e] + bias;
        if (epi == Epi::BiasResidF32)
            static_cast<float *>(p.out)[i] = p.resid[i] + v;
        else
            static_cast<bf16_t *>(p.out)[i] = f32_to_bf16(epi == Epi::BiasGeluBf16 ? gelu(v) : v);
    }
}

template <int GROUP, int MC, int T>
hipError_t launch_q4_t(Epi epi, const Q4Params &p, hipStream_t stream) {
    const dim3 grid((p.N / 16 + T - 1) / T), block(64 * kWaves);
    const int per_wave = (p.chunks + kWaves - 1) / kWaves;
    if (per_wave == 1) return launch_kernel(q4_kernel<GROUP, MC, T, 1>, grid, block, stream, p, epi);
    if (per_wave == 2) return launch_kernel(q4_kernel<GROUP, MC, T, 2>, grid, block, stream, p, epi);
    return launch_kernel(q4_kernel<GROUP, MC, T, 4>, grid, block, stream, p, epi);
}

template <int GROUP, int MC>
hipError_t launch_q4_m(Epi epi, const Q4Params &p, hipStream_t stream) {
    // more tiles a workgroup read the activations fewer times, while enough workgroups are left for the chip
    const int tiles = p.N / 16;
    if (tiles >= 1024) return launch_q4_t<GROUP, MC, 4>(epi, p, stream);
    if (tiles >= 512) return launch_q4_t<GROUP, MC, 2>(epi, p, stream);
    return launch_q4_t<GROUP, MC, 1>(epi, p, stream);
}

template <int GROUP>
hipError_t launch_q4_g(Epi epi, const Q4Params &p, hipStream_t stream) {
    if (p.M <= 4) return launch_q4_m<GROUP, 4>(epi, p, stream);
    if (p.M <= 8) return launch_q4_m<GROUP, 8>(epi, p, stream);
    return launch_q4_m<GROUP, 16>(epi, p, stream);
}

int q4_chunks(int K) { return (K + kChunk - 1) / kChunk; }
size_t q4_code_bytes(int N, int K) { return (size_t)N / 16 * q4_chunks(K) * 1024; }

}  // namespace

size_t q4_packed_bytes(int N, int K, int group) {
    return q4_code_bytes(N, K) + (size_t)N * q4_chunks(K) * (kChunk / group) * 4;
}

hipError_t launch_q4_pack(const uint8_t *codes, const bf16_t *scales, const uint8_t *zeros, void *dst, int N, int K,
                          int group, hipStream_t stream) {
    const int chunks = q4_chunks(K);
    const size_t pieces = (size_t)N / 16 * chunks * 64;
    const dim3 grid((unsigned)((pieces + 255) / 256)), block(256);
    u32x4 *out = static_cast<u32x4 *>(dst);
    uint32_t *meta = reinterpret_cast<uint32_t *>(static_cast<char *>(dst) + q4_code_bytes(N, K));
    switch (group) {
    case 32: return launch_kernel(q4_pack_kernel<32>, grid, block, stream, codes, scales, zeros, out, meta, N, K, chunks);
    case 64: return launch_kernel(q4_pack_kernel<64>, grid, block, stream, codes, scales, zeros, out, meta, N, K, chunks);
    case 128:
        return launch_kernel(q4_pack_kernel<128>, grid, block, stream, codes, scales, zeros, out, meta, N, K, chunks);
    }
    return hipErrorInvalidValue;
}

hipError_t launch_q4_gemm(Epi epi, const bf16_t *a, const void *packed, const bf16_t *bias, const float *resid, void *out,
                          int M, int N, int K, int group, hipStream_t stream) {
    Q4Params p{};
    p.a = a;
    p.codes = static_cast<const u32x4 *>(packed);
    p.meta = reinterpret_cast<const uint32_t *>(static_cast<const char *>(packed) + q4_code_bytes(N, K));
    p.bias = bias;
    p.resid = resid;
    p.out = out;
    p.M = M;
    p.N = N;
    p.K = K;
    p.chunks = q4_chunks(K);
    switch (group) {
    case 32: return launch_q4_g<32>(epi, p, stream);
    case 64: return launch_q4_g<64>(epi, p, stream);
    case 128: return launch_q4_g<128>(epi, p, stream);
    }
    return hipErrorInvalidValue;
}

}  // namespace iefwd
