// Products of a decode step with 4-bit weights for gfx950:
// out = epilogue(A W^T + b), W[n][k] = s[n][g] (code[n][k] - z[n][g]), g = k / group,
// for at most 16 rows of A.  Bound by reading the codes once.
//
// code - z, a whole number from -15 to 15, is exact in bf16 and goes to the matrix cores as such: a weight
// that equals its zero point adds nothing, an infinite activation gives what the definition gives. The sums
// are fp32, the scale is applied to a group's sum.  Relative to 64 bits the fp32 result is off by 8.5e-8 in
// the mean (16 x 4096 -> 1024, groups of 128, activations of either or of one sign; sums of a (16 + code) less
// (16 + z) sum a, which need no subtraction a weight, were off by 1.3e-7 and 3.9e-7 at the same times).
// The matrix cores subtract: as an e4m3 bit pattern a byte 0 .. 15 is the number 2^-9 code, and an 8-bit product
// with a matrix that has 2^9 in the right places and with -z as its addend leaves each lane its own eight code - z
// in fp32 (exact), four to a product, whose upper halves are the bf16 operand.
//
// Measured (us; a plain read of the same bytes, launch included, takes 7.6 for the last two): 1 x 1024 -> 1024 2.9,
// 1 x 2048 -> 8192 3.8, 1 x 4096 -> 16384 8.8, 16 x 4096 -> 16384 10.0 and, in groups of 32, 11.3, where the vector
// units have 4.2 us of work (for 8 weights of a lane 16 operations, 3 to part and 4 to pack the codes, 4 for the
// addend, 5 for the scale; and 4 of other work) and the matrix cores 2.6.  With weights that are not in the last cache (430 MB read in turn)
// the last three take 9.8, 12.8 and 14.0.  Short rows are bound by the latency of a launch and two loads in a row.
// Loading the next chunk before using this one: 8.9, 10.4, 12.1, and 10.9, 12.8, 13.8 from memory; not kept.
#include "q4.h"

#include "gemm_device.h"

namespace iefwd {
namespace {

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
// word s: e = 0 .. 3 in the low and e = 4 .. 7 in the high halves of its bytes, in order.
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
            for (int e = 0; e < 4; ++e) {      // the pair 2 e, 2 e + 1
                const uint32_t byte = codes[((size_t)n * K + k) / 2 + e], pair = (byte & 15) | (byte >> 4) << 8;
                out[s] |= pair << (e < 2 ? 16 * e : 16 * e - 28);
            }
    }
    dst[i] = out;
    if (l / 16 < GPC) {      // this lane's group of the chunk
        const int g = l / 16, groups = K / GROUP, at = chunk * GPC + g;
        uint32_t w = 0;      // past K: scale 0
        if (at < groups) {
            const size_t j = (size_t)n * groups + at;
            const float off = zeros ? -(float)(zeros[j] & 15) : -8.f;
            w = scales[j] | (__float_as_uint(off) & 0xffff0000u);
        }
        meta[(block * 16 + l % 16) * GPC + g] = w;
    }
}

__device__ inline __amdgpu_buffer_rsrc_t buffer(const void *p, uint32_t bytes) {
    return __builtin_amdgcn_make_buffer_rsrc(const_cast<void *>(p), 0, bytes, 0x00027000);
}

// The lane's eight codes of a word, each less the zero point: off holds -z four times.  pick, this lane's part of the
// product's first operand (e5m2), is 2^9 at its row's weight: row 4 c + e takes weight 8 c + e with it in the
// lower word and 8 c + 4 + e in the upper one.
__device__ inline bf16x8 widen(uint32_t x, uint32_t pick, f32x4 off) {
    const long bytes = (long)((uint64_t)((x >> 4) & 0x0f0f0f0fu) << 32 | (x & 0x0f0f0f0fu));
    const f32x4 lo = __builtin_amdgcn_mfma_f32_16x16x32_bf8_fp8((long)pick, bytes, off, 0, 0, 0);
    const f32x4 hi = __builtin_amdgcn_mfma_f32_16x16x32_bf8_fp8((long)((uint64_t)pick << 32), bytes, off, 0, 0, 0);
    auto pair = [](float a, float b) { return __builtin_amdgcn_perm(__float_as_uint(b), __float_as_uint(a), 0x07060302u); };
    return __builtin_bit_cast(bf16x8, u32x4{pair(lo[0], lo[1]), pair(lo[2], lo[3]), pair(hi[0], hi[1]), pair(hi[2], hi[3])});
}

// NL: 16-byte activation loads a lane and chunk, 4 rows each (1, 2 or 4: up to 4, 8 or 16 rows).
// A load takes 256 consecutive bytes of each of 4 rows, 16 lanes a row: only neighbouring
// lanes' addresses are merged, and loading a matrix operand as it stands (neighbouring lanes in
// different rows) reached 16 bytes a clock and CU where this reaches 50.  The pieces come to
// their lanes through 1 KB of LDS a load, the wave's own; XORed with the row, a piece's place puts the
// 16 lanes that read together into different banks.
// The operand's 16 rows are the 4 NL rows of A, each 4 / NL times, so that a lane's results are
// rows NL c .. NL c + NL - 1 of one feature and nothing is computed twice but by the matrix cores.
// T: tiles of 16 features a workgroup works on together.
template <int GROUP, int NL, int T, int WAVES>
__global__ __launch_bounds__(64 * WAVES) void q4_kernel(Q4Params p, Epi epi) {
    constexpr int GPC = kChunk / GROUP, SPG = 4 / GPC;      // groups of a chunk, steps of a group
    constexpr int kStage = NL * 1024, kLds = WAVES * (kStage > T * NL * 256 ? kStage : T * NL * 256);
    __shared__ __attribute__((aligned(16))) char lds[kLds];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int r = lane & 15, c = lane >> 4;
    const int tile0 = blockIdx.x * T;
    f32x4 acc[T] = {};
    const uint32_t pick = r >> 2 == c ? 0x60u << (8 * (r & 3)) : 0u;
    char *stage = lds + wave * kStage;
    const int own = r * NL / 4;                             // the row of A that this lane's operand row is
    // Operands as buffers: a scalar base and step, one 32-bit offset a lane.  Every offset lies inside
    // them by itself: a tile past N reads the last one's operands and is not stored.
    const int n_tiles = min(T, p.N / 16 - tile0);
    const size_t block0 = (size_t)tile0 * p.chunks;
    const __amdgpu_buffer_rsrc_t a_buf = buffer(p.a, (uint32_t)p.M * p.K * 2);
    const __amdgpu_buffer_rsrc_t code_buf = buffer(p.codes + block0 * 64, (uint32_t)n_tiles * p.chunks * 1024);
    const __amdgpu_buffer_rsrc_t meta_buf = buffer(p.meta + block0 * 16 * GPC, (uint32_t)n_tiles * p.chunks * 64 * GPC);
    uint32_t a_lane[NL];
#pragma unroll
    for (int i = 0; i < NL; ++i) a_lane[i] = (uint32_t)min(4 * i + c, p.M - 1) * p.K * 2 + r * 16;

    // this lane's piece of chunk j lies past K: the chunk's first is read in its place and not used
    auto past = [&](int j) { return (j + 1) * kChunk > p.K && j * kChunk + 8 * r >= p.K; };

    u32x4 af[NL], wf[T];
    uint32_t mf[T][GPC];
    auto load = [&](int j) {
#pragma unroll
        for (int i = 0; i < NL; ++i)
            af[i] = __builtin_amdgcn_raw_buffer_load_b128(a_buf, a_lane[i] - (past(j) ? r * 16 : 0), j * 256, 0);
#pragma unroll
        for (int t = 0; t < T; ++t) {
            const int block = min(t, n_tiles - 1) * p.chunks + j;
            wf[t] = __builtin_amdgcn_raw_buffer_load_b128(code_buf, lane * 16, block * 1024, 0);
            if constexpr (GPC == 4) {
                const u32x4 x = __builtin_amdgcn_raw_buffer_load_b128(meta_buf, r * 16, block * 256, 0);
#pragma unroll
                for (int g = 0; g < 4; ++g) mf[t][g] = x[g];
            } else if constexpr (GPC == 2) {
                const u32x2 x = __builtin_amdgcn_raw_buffer_load_b64(meta_buf, r * 8, block * 128, 0);
                mf[t][0] = x[0];
                mf[t][1] = x[1];
            } else {
                mf[t][0] = __builtin_amdgcn_raw_buffer_load_b32(meta_buf, r * 4, block * 64, 0);
            }
        }
    };
    auto use = [&](int j) {
        if ((j + 1) * kChunk > p.K) {
#pragma unroll
            for (int i = 0; i < NL; ++i)
                if (past(j)) af[i] = u32x4{0, 0, 0, 0};
        }
#pragma unroll
        for (int i = 0; i < NL; ++i)
            *reinterpret_cast<u32x4 *>(stage + (4 * i + c) * 256 + (r ^ (4 * i + c)) * 16) = af[i];
        bf16x8 a[4];
#pragma unroll
        for (int s = 0; s < 4; ++s)
            a[s] = *reinterpret_cast<const bf16x8 *>(stage + own * 256 + ((4 * s + c) ^ own) * 16);
#pragma unroll
        for (int g = 0; g < GPC; ++g) {
#pragma unroll
            for (int t = 0; t < T; ++t) {
                const float scale = __uint_as_float(mf[t][g] << 16), z = __uint_as_float(mf[t][g] & 0xffff0000u);
                f32x4 d = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
                for (int s = 0; s < SPG; ++s)
                    d = __builtin_amdgcn_mfma_f32_16x16x32_bf16(
                        a[g * SPG + s], widen(wf[t][g * SPG + s], pick, f32x4{z, z, z, z}), d, 0, 0, 0);
#pragma unroll
                for (int e = 0; e < NL; ++e) acc[t][e * 4 / NL] = fmaf(scale, d[e * 4 / NL], acc[t][e * 4 / NL]);
            }
        }
    };
    for (int j = wave; j < p.chunks; j += WAVES) {
        load(j);
        use(j);
    }
    // the waves' sums in wave order, wave t for tile t
    float (*part)[T][NL][64] = reinterpret_cast<float (*)[T][NL][64]>(lds);
    __syncthreads();
#pragma unroll
    for (int t = 0; t < T; ++t)
#pragma unroll
        for (int e = 0; e < NL; ++e) part[wave][t][e][lane] = acc[t][e * 4 / NL];
    __syncthreads();
    const int n = (tile0 + wave) * 16 + r;
    if (wave >= T || n >= p.N) return;
    const float bias = p.bias ? __uint_as_float((uint32_t)p.bias[n] << 16) : 0.f;
#pragma unroll
    for (int e = 0; e < NL; ++e) {
        const int row = NL * c + e;
        if (row >= p.M) break;
        float v = part[0][wave][e][lane];
#pragma unroll
        for (int w = 1; w < WAVES; ++w) v += part[w][wave][e][lane];
        v += bias;
        const size_t i = (size_t)row * p.N + n;
        if (epi == Epi::BiasResidF32)
            static_cast<float *>(p.out)[i] = p.resid[i] + v;
        else
            static_cast<bf16_t *>(p.out)[i] = f32_to_bf16(epi == Epi::BiasGeluBf16 ? gelu(v) : v);
    }
}

template <int GROUP, int NL, int T, int WAVES>
hipError_t launch_q4_w(Epi epi, const Q4Params &p, hipStream_t stream) {
    const dim3 grid((p.N / 16 + T - 1) / T), block(64 * WAVES);
    return launch_kernel(q4_kernel<GROUP, NL, T, WAVES>, grid, block, stream, p, epi);
}

// Two tiles a workgroup halve the reads of the activations, which each CU takes in whole, and are taken
// where the workgroups still fill the chip; 16 waves have more of a long row in flight where one workgroup a
// CU is all there is.  The waves, and with them the order of the sums, follow from N and K alone.
// us with 8 waves and 1 tile / 8 and 2 / 16 and 1 / 16 and 2, groups of 128:
//   1 x 1024 -> 1024    2.8  3.1  2.9  3.1     16 x 4096 -> 4096    5.6  6.5  5.4  6.1
//   1 x 8192 -> 2048    7.1  8.5  5.4  7.2     16 x 8192 -> 2048    7.9  9.6  6.9  8.3
//   1 x 2048 -> 8192    4.0  4.0  4.1  4.0     16 x 2048 -> 8192    5.4  5.0  5.4  5.1
//   1 x 4096 -> 16384   8.7  8.6  9.5  8.7     16 x 4096 -> 16384  11.4 10.0 12.3 11.4
template <int GROUP, int NL>
hipError_t launch_q4_m(Epi epi, const Q4Params &p, hipStream_t stream) {
    const int tiles = p.N / 16;
    if (tiles > 512) return launch_q4_w<GROUP, NL, 2, 8>(epi, p, stream);
    if (p.chunks < 16) return launch_q4_w<GROUP, NL, 1, 8>(epi, p, stream);
    if (tiles > 256) return launch_q4_w<GROUP, NL, 2, 16>(epi, p, stream);
    return launch_q4_w<GROUP, NL, 1, 16>(epi, p, stream);
}

template <int GROUP>
hipError_t launch_q4_g(Epi epi, const Q4Params &p, hipStream_t stream) {
    if (p.M <= 4) return launch_q4_m<GROUP, 1>(epi, p, stream);
    if (p.M <= 8) return launch_q4_m<GROUP, 2>(epi, p, stream);
    return launch_q4_m<GROUP, 4>(epi, p, stream);
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
