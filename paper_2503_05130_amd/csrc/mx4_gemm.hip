// Products of matrices in microscaled 4 bits for gfx950.
#include <algorithm>
#include <type_traits>

#include "mx4.h"
#include "mx4_device.h"

namespace iefwd {
namespace {

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

// Many rows: a workgroup's tile of BM rows x BN features, through LDS.
//
// The operands' 1 KB blocks are copied from global memory straight into a ring of S chunks of K, each block by one
// instruction, in the lane order in which the fragments are read (contiguous in both, no bank conflicts); a group of 4 chunks' scales
// goes into one of two buffers ahead of the group's first chunk.  Step j: read the second half of the rows' fragments of
// chunk j; products of the first half; wait for the own copies of chunk j + 1 and the own reads, barrier (chunk j + 1 is
// there, nobody reads chunk j's slot any more); copy chunk j + S into that slot, read chunk j + 1's features and
// first half; products of the second half.
template <int BM_, int BN_, int WM_, int WN_>
struct TileCfg {
    static constexpr int BM = BM_, BN = BN_, WM = WM_, WN = WN_, NW = WM * WN, S = 4;
    static constexpr int TA = BM / 16, TW = BN / 16, FM = TA / WM, FN = TW / WN, H = FM / 2;
    static constexpr int COPIES = (TA + TW) / NW;       // of a wave and chunk
    static constexpr int SLOT = (TA + TW) * 1024, SCALES = (TA + TW) * 256, LDS = S * SLOT + 2 * SCALES;
    static_assert(TA % NW == 0 && TW % NW == 0 && NW * 4 == TA + TW && FM % 2 == 0, "tile");
    static constexpr int ROW = BN + 8;                  // of the staged output, in bf16
    static_assert(BM * ROW * 2 <= LDS, "output tile");
};

template <int I, int S, int COPIES>
constexpr int tile_waits() {      // copies younger than chunk j + 1's while chunks up to j + S - 1 are on their way, j % 4 = I
    int n = 0;
    for (int t = I + 2; t < I + S; ++t) n += COPIES + (t % 4 == 0);
    return n;
}

template <class C>
__global__ __launch_bounds__(64 * C::NW, 2) void mx4_tile_kernel(Mx4Params p, int tiles_m, int tiles_n) {
    constexpr int NW = C::NW, FM = C::FM, FN = C::FN, H = C::H, S = C::S;
    __shared__ __attribute__((aligned(16))) char lds[C::LDS];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int wm = wave % C::WM, wn = wave / C::WM;
    int tm, tn;
    grouped_tile(xcd_contiguous(blockIdx.x, gridDim.x), tiles_m, tiles_n, tm, tn);
    const int chunks = mx4_chunks(p.K), groups = (chunks + 3) / 4;
    const size_t tile_bytes = mx4_tile_bytes(p.K);
    const int rt0 = tm * C::TA, ft0 = tn * C::TW;
    const int last_r = (p.M + 15) / 16 - 1, last_f = (p.N + 15) / 16 - 1;      // tiles past them read the last and are not stored

    // copies: block wave + NW i of a slot, whose first TA are rows
    const char *base[C::COPIES];
#pragma unroll
    for (int i = 0; i < C::COPIES; ++i) {
        const int b = wave + NW * i;
        base[i] = b < C::TA ? p.a + (size_t)min(rt0 + b, last_r) * tile_bytes : p.w + (size_t)min(ft0 + b - C::TA, last_f) * tile_bytes;
    }
    // scales: 4 tiles a wave
    const bool of_rows = wave < C::TA / 4;
    const int st0 = of_rows ? rt0 + 4 * wave : ft0 + 4 * wave - C::TA, st_last = of_rows ? last_r : last_f;
    const char *scale_base = (of_rows ? p.a : p.w) + (size_t)min(st0, st_last) * tile_bytes + (size_t)chunks * 1024;
    const uint32_t scale_off = (uint32_t)(min(st0 + (lane >> 4), st_last) - min(st0, st_last)) * (uint32_t)tile_bytes + (lane & 15) * 16;
    const uint32_t lds0 = (uint32_t)(size_t)(lds_ptr_t)lds, scales0 = lds0 + S * C::SLOT;
    auto copy = [&](int j) {
        if ((j & 3) == 0) dma16(scale_base + (j >> 2) * 256, scale_off, scales0 + ((j >> 2) & 1) * C::SCALES + wave * 1024);
#pragma unroll
        for (int i = 0; i < C::COPIES; ++i)
            dma16(base[i] + (size_t)j * 1024, lane * 16, lds0 + (j % S) * C::SLOT + (wave + NW * i) * 1024);
    };
    u32x4 w[2][FN], lo[H], hi[H];
    uint32_t ws[FN], as[FM];
    auto read_w = [&](u32x4 (&f)[FN], int j) {
        const char *s = lds + (j % S) * C::SLOT + (C::TA + wn * FN) * 1024 + lane * 16;
#pragma unroll
        for (int i = 0; i < FN; ++i) f[i] = *reinterpret_cast<const u32x4 *>(s + i * 1024);
    };
    auto read_a = [&](u32x4 (&f)[H], int j, int first) {
        const char *s = lds + (j % S) * C::SLOT + (wm * FM + first) * 1024 + lane * 16;
#pragma unroll
        for (int i = 0; i < H; ++i) f[i] = *reinterpret_cast<const u32x4 *>(s + i * 1024);
    };
    auto read_scales = [&](uint32_t (&fw)[FN], uint32_t (&fa)[FM], int g) {
        const char *s = lds + S * C::SLOT + (g & 1) * C::SCALES + lane * 4;
#pragma unroll
        for (int i = 0; i < FN; ++i) fw[i] = *reinterpret_cast<const uint32_t *>(s + (C::TA + wn * FN + i) * 256);
#pragma unroll
        for (int i = 0; i < FM; ++i) fa[i] = *reinterpret_cast<const uint32_t *>(s + (wm * FM + i) * 256);
    };
    f32x4 acc[FN][FM] = {};
    auto barrier = [&] {
        __builtin_amdgcn_s_barrier();
        asm volatile("" ::: "memory");      // LDS accesses stay on their side
    };

#pragma unroll
    for (int j = 0; j < S; ++j)
        if (j < chunks) copy(j);
    __builtin_amdgcn_s_waitcnt(waitcnt_imm(0, 15));
    barrier();
    read_w(w[0], 0);
    read_a(lo, 0, 0);
    read_scales(ws, as, 0);
    // chunk j, j % 4 = I; w[I % 2] and lo are its own
    auto step = [&](auto place, int j) {
        constexpr int I = decltype(place)::value;
        read_a(hi, j, H);
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int f = 0; f < FN; ++f)
#pragma unroll
            for (int t = 0; t < H; ++t) acc[f][t] = mfma_mx4<I>(w[I % 2][f], lo[t], acc[f][t], ws[f], as[t]);
        __builtin_amdgcn_sched_barrier(0);
        uint32_t ws2[FN], as2[FM];
        if (j + 1 < chunks) {
            if (j + S - 1 < chunks) __builtin_amdgcn_s_waitcnt(waitcnt_imm(tile_waits<I, S, C::COPIES>(), 0));
            else __builtin_amdgcn_s_waitcnt(waitcnt_imm(0, 0));
            barrier();
            if (j + S < chunks) copy(j + S);
            read_w(w[(I + 1) % 2], j + 1);
            read_a(lo, j + 1, 0);
            if (I == 3) read_scales(ws2, as2, (j + 1) >> 2);
        }
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int f = 0; f < FN; ++f)
#pragma unroll
            for (int t = 0; t < H; ++t) acc[f][H + t] = mfma_mx4<I>(w[I % 2][f], hi[t], acc[f][H + t], ws[f], as[H + t]);
        __builtin_amdgcn_sched_barrier(0);
        if (I == 3 && j + 1 < chunks) {
#pragma unroll
            for (int f = 0; f < FN; ++f) ws[f] = ws2[f];
#pragma unroll
            for (int t = 0; t < FM; ++t) as[t] = as2[t];
        }
    };
    for (int g = 0; g < groups; ++g) {
        const int j = 4 * g;
        step(std::integral_constant<int, 0>{}, j);
        if (j + 1 < chunks) step(std::integral_constant<int, 1>{}, j + 1);
        if (j + 2 < chunks) step(std::integral_constant<int, 2>{}, j + 2);
        if (j + 3 < chunks) step(std::integral_constant<int, 3>{}, j + 3);
    }
    // lane (r, c): row r of a row tile, features 4 c .. 4 c + 3
    const int r = lane & 15, c = lane >> 4;
#pragma unroll
    for (int f = 0; f < FN; ++f)
#pragma unroll
        for (int t = 0; t < FM; ++t)
            mx4_store(p, (rt0 + wm * FM + t) * 16 + r, (ft0 + wn * FN + f) * 16 + 4 * c, acc[f][t]);
}

template <class C>
hipError_t launch_tile(const Mx4Params &p, hipStream_t stream) {
    const int tiles_m = (p.M + C::BM - 1) / C::BM, tiles_n = (p.N + C::BN - 1) / C::BN;
    return launch_kernel(mx4_tile_kernel<C>, dim3((unsigned)((int64_t)tiles_m * tiles_n)), dim3(64 * C::NW), stream, p, tiles_m, tiles_n);
}

}  // namespace

hipError_t launch_mx4_gemm(Epi epi, const void *a, const void *w, const bf16_t *bias, const float *resid, void *out, int M,
                           int N, int K, hipStream_t stream) {
    Mx4Params p{static_cast<const char *>(a), static_cast<const char *>(w), nullptr, bias, resid, out, M, N, K, 0, epi};
    if (M <= 16) return launch_split<1, 1, 8, 0>(p, stream);
    if (M <= 32) return launch_split<2, 2, 8, 0>(p, stream);
    if ((int64_t)M * N <= 1024 * 1024) return launch_split<4, 4, 4, 0>(p, stream);
    if ((int64_t)((M + 255) / 256) * ((N + 255) / 256) >= 192) return launch_tile<TileCfg<256, 256, 2, 4>>(p, stream);
    return launch_tile<TileCfg<128, 128, 2, 2>>(p, stream);
}

hipError_t launch_mx4_gemm_bf16(Epi epi, const bf16_t *a, const void *w, const bf16_t *bias, const float *resid, void *out,
                                int M, int N, int K, hipStream_t stream) {
    Mx4Params p{nullptr, static_cast<const char *>(w), a, bias, resid, out, M, N, K, 0, epi};
    if (M <= 4) return launch_split<1, 1, 8, 1>(p, stream);
    if (M <= 8) return launch_split<1, 1, 8, 2>(p, stream);
    return launch_split<1, 1, 8, 4>(p, stream);
}

}  // namespace iefwd
