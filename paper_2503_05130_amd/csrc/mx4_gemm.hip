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

// What is added to four features n .. n + 3 of row m, asked for before the sums.
struct Tail {
    f32x4 bias, resid;
};

typedef u32x2 u32x2_any __attribute__((aligned(2)));

__device__ inline f32x4 mx4_bias(const Mx4Params &p, int n) {
    f32x4 b = {0.f, 0.f, 0.f, 0.f};
    if (!p.bias) return b;
    if (n + 4 <= p.N) {
        const u32x2 w = *reinterpret_cast<const u32x2_any *>(p.bias + n);
#pragma unroll
        for (int e = 0; e < 4; ++e) b[e] = __uint_as_float(e % 2 ? w[e / 2] & 0xffff0000u : w[e / 2] << 16);
    } else {
#pragma unroll
        for (int e = 0; e < 4; ++e)
            if (n + e < p.N) b[e] = __uint_as_float((uint32_t)p.bias[n + e] << 16);
    }
    return b;
}

__device__ inline f32x4 mx4_resid(const Mx4Params &p, int m, int n) {
    f32x4 x = {0.f, 0.f, 0.f, 0.f};
    if (p.epi != Epi::BiasResidF32 || m >= p.M) return x;
    const float *resid = p.resid + (size_t)m * p.N + n;
    if ((p.N & 3) == 0) {
        if (n < p.N) x = *reinterpret_cast<const f32x4 *>(resid);
    } else {
#pragma unroll
        for (int e = 0; e < 4; ++e)
            if (n + e < p.N) x[e] = resid[e];
    }
    return x;
}

template <bool FAR, class T>
__device__ inline void put(T *to, T v) {
    if constexpr (FAR) __builtin_nontemporal_store(v, to);
    else *to = v;
}

// Four features n .. n + 3 of row m.
template <bool FAR = false>
__device__ inline void mx4_store(const Mx4Params &p, int m, int n, f32x4 v, const Tail &t) {
    if (m >= p.M) return;
    const int count = min(4, p.N - n);
    v += t.bias;
    const size_t i = (size_t)m * p.N + n;
    if (p.epi == Epi::BiasResidF32) {
        float *out = static_cast<float *>(p.out) + i;
        v = t.resid + v;
        if ((p.N & 3) == 0) {
            if (count > 0) put<FAR>(reinterpret_cast<f32x4 *>(out), v);
        } else {
#pragma unroll
            for (int e = 0; e < 4; ++e)
                if (e < count) out[e] = v[e];
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

// Few rows: bound by the weights' bytes and, below some 10 MB, by latency (launch, a chain of two loads, the joining of the waves).
// 4 x 4096 -> 16384 takes 5.9 us of 4-bit rows (6.1 TB/s), 6.4 of bf16 ones; 1 x 2048 -> 8192 3.2 and 3.4 us; 32 x 8192 -> 8192
// 6.7 (5.4 TB/s).  Bias and residual are asked for first: at the end they cost 0.3 to 0.6 us.
//
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
    static_assert(FT * RT <= WAVES, "a wave stores one block at most");
    const int m = (rt0 + wave % RT) * 16 + r, n = (ft0 + wave / RT) * 16 + 4 * c;
    Tail tail = {};
    if (wave < FT * RT) tail = {mx4_bias(p, n), mx4_resid(p, m, n)};
    struct Chunk {
        u32x4 w[FT], a[NL ? 1 : RT];
        uint32_t ws[FT], as[NL ? 1 : RT];
        Eight x[NL ? NL : 1];
    };
    const int piece = lane & 15;
    auto load = [&](Chunk &k, int j) {
        const size_t scales = (size_t)chunks * 1024 + (size_t)(j >> 2) * 256 + lane * 4;
#pragma unroll
        for (int f = 0; f < FT; ++f) {
            k.w[f] = *reinterpret_cast<const u32x4 *>(w[f] + (size_t)j * 1024 + lane * 16);
            k.ws[f] = *reinterpret_cast<const uint32_t *>(w[f] + scales);
        }
        if constexpr (NL == 0) {
#pragma unroll
            for (int t = 0; t < RT; ++t) {
                k.a[t] = *reinterpret_cast<const u32x4 *>(a[t] + (size_t)j * 1024 + lane * 16);
                k.as[t] = *reinterpret_cast<const uint32_t *>(a[t] + scales);
            }
        } else {
            const int col = j * 128 + 8 * piece;
#pragma unroll
            for (int i = 0; i < NL; ++i) {
                k.x[i] = Eight{};
                if (col < p.K)
                    k.x[i].lo = *reinterpret_cast<const u32x4 *>(p.a16 + (size_t)min(4 * i + (lane >> 4), p.M - 1) * p.K + col);
            }
        }
    };
    auto use = [&](Chunk &k, int j) {
        const int shift = 8 * (j & 3);
        if constexpr (NL > 0) {
#pragma unroll
            for (int i = 0; i < NL; ++i) {
                const int row = 4 * i + (lane >> 4), at = row + 16 * (piece >> 2);
                const uint32_t scale = mx4_scale<false>(k.x[i]);
                *reinterpret_cast<uint32_t *>(stage + at * 16 + (piece & 3) * 4) = mx4_codes<false>(k.x[i], scale);
                if ((piece & 3) == 0) stage[1024 + at] = (char)scale;
            }
            wave_lds_fence();
            // columns of rows past 4 NL hold whatever was there: they are sums of their own and not stored
            k.a[0] = *reinterpret_cast<const u32x4 *>(stage + lane * 16);
            k.as[0] = (uint32_t)(uint8_t)stage[1024 + lane] << shift;
            wave_lds_fence();
        }
#pragma unroll
        for (int f = 0; f < FT; ++f)
#pragma unroll
            for (int t = 0; t < RT; ++t) acc[f][t] = mfma_mx4(k.w[f], k.a[t], acc[f][t], k.ws[f] >> shift, k.as[t] >> shift);
    };
    // a chunk's loads ahead of the chunk in use
    Chunk k0, k1;
    int j = wave;
    if (j < chunks) load(k0, j);
    for (; j < chunks; j += 2 * WAVES) {
        if (j + WAVES < chunks) load(k1, j + WAVES);
        use(k0, j);
        if (j + WAVES >= chunks) break;
        if (j + 2 * WAVES < chunks) load(k0, j + 2 * WAVES);
        use(k1, j + WAVES);
    }
    __syncthreads();
    f32x4 (*part)[FT * RT][64] = reinterpret_cast<f32x4 (*)[FT * RT][64]>(lds);
#pragma unroll
    for (int f = 0; f < FT; ++f)
#pragma unroll
        for (int t = 0; t < RT; ++t) part[wave][f * RT + t][lane] = acc[f][t];
    __syncthreads();
    if (wave < FT * RT) {
        f32x4 v = part[0][wave][lane];
#pragma unroll
        for (int i = 1; i < WAVES; ++i) v += part[i][wave][lane];
        mx4_store(p, m, n, v, tail);
    }
}

template <int FT, int RT, int WAVES, int NL>
hipError_t launch_split(Mx4Params p, hipStream_t stream) {
    const int f_groups = ((p.N + 15) / 16 + FT - 1) / FT;
    p.row_tiles = ((p.M + 15) / 16 + RT - 1) / RT;
    return launch_kernel(mx4_split_kernel<FT, RT, WAVES, NL>, dim3((unsigned)((int64_t)f_groups * p.row_tiles)),
                         dim3(64 * WAVES), stream, p);
}

// Many rows: a workgroup's tile of BM rows x BN features, through LDS.  A lane's operand is 16 bytes for 16 x 16 x 128 x 2 / 64
// operations, so that a wave of 128 x 64 reads 12 KB of LDS for 32 products of 16 cycles each; registers alone (the kernel above) come
// to half the rate.  8192^3 takes 240 us from a graph (4.6 PFLOP/s) and 255 between quantisations (median of a profile, least 242; 4.3) at
// a clock that falls to 1.8 GHz: the matrix cores are busy for 62% of the whole and 67% of the loop, some 40 us are the first stages'
// loads and the output of 4 rounds of workgroups.  4096^3 37 us (3.7 PFLOP/s).  A 256 x 256 tile has a CU for itself (144 KB of LDS), so
// that its epilogue follows its products: 8192 x 16384 x 2048 with bias 175 us, with GELU 228; 4096^3 38, 45 and with the fp32 residual 58.
// (The compiler spills 4 of its registers.)
// A ring of four stages in place of two for 64 x 64 tiles gained nothing (201 x 4096 x 4096, 250 x 4096 x 4096, 150 x 2048 x 8192).
//
// The operands' 1 KB blocks are copied from global memory straight into a ring of S stages of CH chunks of K, each block by one
// instruction, in the lane order in which the fragments are read (contiguous in both, no bank conflicts); a group of 4 chunks' scales
// goes into a ring of buffers ahead of the group's first chunk.  Step j: read the second half of the rows' fragments of
// chunk j; products of the first half; where chunk j + 1 begins a stage, wait for the own copies of it and the own reads,
// barrier (the stage is there, nobody reads chunk j's any more), and copy the stage S further into that slot; read chunk j +
// 1's features and first half; products of the second half.
template <int BM_, int BN_, int WM_, int WN_, int CH_, int S_, bool FAR_ = false>
struct TileCfg {
    static constexpr bool FAR = FAR_;      // the output past the last cache
    static constexpr int BM = BM_, BN = BN_, WM = WM_, WN = WN_, NW = WM * WN, CH = CH_, S = S_;
    static constexpr int TA = BM / 16, TW = BN / 16, FM = TA / WM, FN = TW / WN, H = FM / 2;
    static constexpr int COPIES = (TA + TW) / NW;                        // of a wave and chunk
    static constexpr int SCALE_COPIES = ((TA + TW) / 4 + NW - 1) / NW;   // of a wave and group
    static constexpr int BUFFERS = (S * CH + 3) / 4 + 1;                 // of scales: the group in use and those on their way
    static constexpr int SLOT = (TA + TW) * 1024, SCALES = (TA + TW) * 256, LDS = S * CH * SLOT + BUFFERS * SCALES;
    static constexpr int WAVES_SIMD = 163840 / LDS * NW / 4 < 1 ? 1 : 163840 / LDS * NW / 4 > 4 ? 4 : 163840 / LDS * NW / 4;
    // bias and residual are asked for before the sums where the registers have room: 512 x 4096 x 4096 with residual 19.1 -> 18.0 us with
    // its quantisation; for 128 x 128 they would spill (1000 x 4096 x 4096 22.9 -> 26.1)
    static constexpr bool EARLY = FN * FM <= 4;
    static_assert((TA + TW) % NW == 0 && TA % 4 == 0 && TW % 4 == 0 && FM % 2 == 0 && 4 % CH == 0 && S >= 2, "tile");
    static constexpr int ROW = BN * 2 + 16;                              // bytes of a row of the staged output
    static_assert(BM * ROW <= LDS, "output tile");
    static_assert(S * CH * (COPIES + SCALE_COPIES) < 64, "copies on their way (vmcnt holds 6 bits)");

    // copies of a wave for chunks [from, to), counted from a group's first
    static constexpr int copies(int from, int to) {
        int n = 0;
        for (int t = from; t < to; ++t) n += COPIES + (t % 4 == 0 ? SCALE_COPIES : 0);
        return n;
    }
};

template <class C>
__global__ __launch_bounds__(64 * C::NW, C::WAVES_SIMD) void mx4_tile_kernel(Mx4Params p, int tiles_m, int tiles_n) {
    constexpr int NW = C::NW, FM = C::FM, FN = C::FN, H = C::H, S = C::S, CH = C::CH;
    __shared__ __attribute__((aligned(16))) char lds[C::LDS];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int wm = wave % C::WM, wn = wave / C::WM;
    int tm, tn;
    grouped_tile(xcd_contiguous(blockIdx.x, gridDim.x), tiles_m, tiles_n, tm, tn);
    const int chunks = mx4_chunks(p.K);
    const size_t tile_bytes = mx4_tile_bytes(p.K);
    const int rt0 = tm * C::TA, ft0 = tn * C::TW;
    const int last_r = (p.M + 15) / 16 - 1, last_f = (p.N + 15) / 16 - 1;      // tiles past them read the last and are not stored

    // copies: block wave + NW i of a chunk, whose first TA are rows
    const char *base[C::COPIES];
#pragma unroll
    for (int i = 0; i < C::COPIES; ++i) {
        const int b = wave + NW * i;
        base[i] = b < C::TA ? p.a + (size_t)min(rt0 + b, last_r) * tile_bytes : p.w + (size_t)min(ft0 + b - C::TA, last_f) * tile_bytes;
    }
    // scales: 4 tiles a copy (copies past the last tile repeat it)
    const char *scale_base[C::SCALE_COPIES];
    uint32_t scale_off[C::SCALE_COPIES], scale_at[C::SCALE_COPIES];
    const uint32_t lds0 = (uint32_t)(size_t)(lds_ptr_t)lds, scales0 = lds0 + S * CH * C::SLOT;
#pragma unroll
    for (int i = 0; i < C::SCALE_COPIES; ++i) {
        const int four = min(wave + NW * i, (C::TA + C::TW) / 4 - 1);
        const bool of_rows = four < C::TA / 4;
        const int t0 = of_rows ? rt0 + 4 * four : ft0 + 4 * four - C::TA, last = of_rows ? last_r : last_f;
        scale_base[i] = (of_rows ? p.a : p.w) + (size_t)min(t0, last) * tile_bytes + (size_t)chunks * 1024;
        scale_off[i] = (uint32_t)(min(t0 + (lane >> 4), last) - min(t0, last)) * (uint32_t)tile_bytes + (lane & 15) * 16;
        scale_at[i] = scales0 + four * 1024;
    }
    auto copy_stage = [&](int j0, auto full) {      // the chunks from j0 on; full: all of them are there
#pragma unroll
        for (int d = 0; d < CH; ++d) {
            const int j = j0 + d;
            if (!decltype(full)::value && j >= chunks) break;
            if ((j & 3) == 0)
#pragma unroll
                for (int i = 0; i < C::SCALE_COPIES; ++i)
                    dma16(scale_base[i] + (j >> 2) * 256, scale_off[i], scale_at[i] + (j >> 2) % C::BUFFERS * C::SCALES);
#pragma unroll
            for (int i = 0; i < C::COPIES; ++i)
                dma16(base[i] + (size_t)j * 1024, lane * 16, lds0 + j % (S * CH) * C::SLOT + (wave + NW * i) * 1024);
        }
    };
    // the n-th copy of the stage of chunks from j0 on, j0 % 4 = I0, all of which are there
    auto copy_nth = [&](auto place, int j0, int n) {
        constexpr int I0 = decltype(place)::value;
        int k = 0;
#pragma unroll
        for (int d = 0; d < CH; ++d) {
            const int j = j0 + d;
            if ((I0 + d) % 4 == 0)
#pragma unroll
                for (int i = 0; i < C::SCALE_COPIES; ++i)
                    if (k++ == n) dma16(scale_base[i] + (j >> 2) * 256, scale_off[i], scale_at[i] + (j >> 2) % C::BUFFERS * C::SCALES);
#pragma unroll
            for (int i = 0; i < C::COPIES; ++i)
                if (k++ == n) dma16(base[i] + (size_t)j * 1024, lane * 16, lds0 + j % (S * CH) * C::SLOT + (wave + NW * i) * 1024);
        }
    };
    u32x4 w[2][FN], lo[H], hi[H];
    uint32_t ws[FN], as[FM];
    auto read_w = [&](u32x4 (&f)[FN], int j) {
        const char *s = lds + j % (S * CH) * C::SLOT + (C::TA + wn * FN) * 1024 + lane * 16;
#pragma unroll
        for (int i = 0; i < FN; ++i) f[i] = *reinterpret_cast<const u32x4 *>(s + i * 1024);
    };
    auto read_a = [&](u32x4 (&f)[H], int j, int first) {
        const char *s = lds + j % (S * CH) * C::SLOT + (wm * FM + first) * 1024 + lane * 16;
#pragma unroll
        for (int i = 0; i < H; ++i) f[i] = *reinterpret_cast<const u32x4 *>(s + i * 1024);
    };
    auto read_scales = [&](uint32_t (&fw)[FN], uint32_t (&fa)[FM], int g) {
        const char *s = lds + S * CH * C::SLOT + g % C::BUFFERS * C::SCALES + lane * 4;
#pragma unroll
        for (int i = 0; i < FN; ++i) fw[i] = *reinterpret_cast<const uint32_t *>(s + (C::TA + wn * FN + i) * 256);
#pragma unroll
        for (int i = 0; i < FM; ++i) fa[i] = *reinterpret_cast<const uint32_t *>(s + (wm * FM + i) * 256);
    };
    f32x4 acc[FN][FM] = {};
    // lane (r, c): row r of a row tile, features 4 c .. 4 c + 3
    const int r = lane & 15, c = lane >> 4;
    auto row_of = [&](int t) { return (rt0 + wm * FM + t) * 16 + r; };
    auto feature_of = [&](int f) { return (ft0 + wn * FN + f) * 16 + 4 * c; };
    f32x4 bias[FN], resid[C::EARLY ? FN : 1][C::EARLY ? FM : 1];
    if constexpr (C::EARLY)
#pragma unroll
        for (int f = 0; f < FN; ++f) {
            bias[f] = mx4_bias(p, feature_of(f));
#pragma unroll
            for (int t = 0; t < FM; ++t) resid[f][t] = mx4_resid(p, row_of(t), feature_of(f));
        }
    auto barrier = [&] {
        __builtin_amdgcn_s_barrier();
        asm volatile("" ::: "memory");      // LDS accesses stay on their side
    };

#pragma unroll
    for (int s = 0; s < S; ++s) copy_stage(s * CH, std::false_type{});
    if (chunks >= S * CH) __builtin_amdgcn_s_waitcnt(waitcnt_imm(C::copies(CH, S * CH), 15));
    else __builtin_amdgcn_s_waitcnt(waitcnt_imm(0, 15));
    barrier();
    read_w(w[0], 0);
    read_a(lo, 0, 0);
    read_scales(ws, as, 0);
    // chunk j, j % 4 = I; w[I % 2] and lo are its own.  full: chunks up to j + S CH are there, and nothing is asked (the
    // compiler would sink the first half's products past the barrier into the branches behind it).
    auto step = [&](auto place, auto full, int j) {
        constexpr int I = decltype(place)::value;
        constexpr bool FULL = decltype(full)::value;
        read_a(hi, j, H);
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int f = 0; f < FN; ++f)
#pragma unroll
            for (int t = 0; t < H; ++t) acc[f][t] = mfma_mx4<I>(w[I % 2][f], lo[t], acc[f][t], ws[f], as[t]);
        __builtin_amdgcn_sched_barrier(0);
        uint32_t ws2[FN], as2[FM];
        constexpr bool STAGE = (I + 1) % CH == 0;      // chunk j + 1 begins one
        constexpr int I0 = (I + 1 + (S - 1) * CH) % 4, READS = FN + H, ACTS = READS + (STAGE ? C::copies(I0, I0 + CH) : 0), NM = FN * H;
        if (FULL || j + 1 < chunks) {
            if constexpr (STAGE) {
                // chunks up to j + (S - 1) CH are on their way or there; j + 1 to j + CH have to be
                if (FULL || j + (S - 1) * CH < chunks)
                    __builtin_amdgcn_s_waitcnt(waitcnt_imm(C::copies(I + 1 + CH, I + 1 + (S - 1) * CH), 0));
                else __builtin_amdgcn_s_waitcnt(waitcnt_imm(0, 0));
                barrier();
            }
            if (!FULL) {
                if (STAGE) copy_stage(j + 1 + (S - 1) * CH, full);
                read_w(w[(I + 1) % 2], j + 1);
                read_a(lo, j + 1, 0);
            }
            if (I == 3) read_scales(ws2, as2, (j + 1) >> 2);
        }
        __builtin_amdgcn_sched_barrier(0);
        // the second half's products, between them the next chunk's reads and then the copies
        const char *next = lds + (j + 1) % (S * CH) * C::SLOT + lane * 16;
#pragma unroll
        for (int f = 0; f < FN; ++f)
#pragma unroll
            for (int t = 0; t < H; ++t) {
                if constexpr (FULL) {
                    const int q = f * H + t;
#pragma unroll
                    for (int d = q * ACTS / NM; d < (q + 1) * ACTS / NM; ++d) {
                        if (d < H) lo[d] = *reinterpret_cast<const u32x4 *>(next + (wm * FM + d) * 1024);
                        else if (d < READS)
                            w[(I + 1) % 2][d - H] = *reinterpret_cast<const u32x4 *>(next + (C::TA + wn * FN + d - H) * 1024);
                        else copy_nth(std::integral_constant<int, I0>{}, j + 1 + (S - 1) * CH, d - READS);
                        __builtin_amdgcn_sched_barrier(0);
                    }
                }
                acc[f][H + t] = mfma_mx4<I>(w[I % 2][f], hi[t], acc[f][H + t], ws[f], as[H + t]);
                if (FULL) __builtin_amdgcn_sched_barrier(0);
            }
        __builtin_amdgcn_sched_barrier(0);
        if (I == 3 && (FULL || j + 1 < chunks)) {
#pragma unroll
            for (int f = 0; f < FN; ++f) ws[f] = ws2[f];
#pragma unroll
            for (int t = 0; t < FM; ++t) as[t] = as2[t];
        }
    };
    int j = 0;
    for (; j + 3 + S * CH < chunks; j += 4) {
        step(std::integral_constant<int, 0>{}, std::true_type{}, j);
        step(std::integral_constant<int, 1>{}, std::true_type{}, j + 1);
        step(std::integral_constant<int, 2>{}, std::true_type{}, j + 2);
        step(std::integral_constant<int, 3>{}, std::true_type{}, j + 3);
    }
    for (; j < chunks; j += 4) {
        step(std::integral_constant<int, 0>{}, std::false_type{}, j);
        if (j + 1 < chunks) step(std::integral_constant<int, 1>{}, std::false_type{}, j + 1);
        if (j + 2 < chunks) step(std::integral_constant<int, 2>{}, std::false_type{}, j + 2);
        if (j + 3 < chunks) step(std::integral_constant<int, 3>{}, std::false_type{}, j + 3);
    }
    if constexpr (!C::EARLY)
#pragma unroll
        for (int f = 0; f < FN; ++f) bias[f] = mx4_bias(p, feature_of(f));
    if (p.epi == Epi::BiasResidF32 || (p.N & 7) != 0) {
        // a column of tiles' residual ahead of the one that is stored: the compiler cannot know that none of it is overwritten
        f32x4 x[2][FM];
        auto load = [&](int f) {
#pragma unroll
            for (int t = 0; t < FM; ++t) {
                if constexpr (C::EARLY) x[f & 1][t] = resid[f][t];
                else x[f & 1][t] = mx4_resid(p, row_of(t), feature_of(f));
            }
        };
        load(0);
#pragma unroll
        for (int f = 0; f < FN; ++f) {
            if (f + 1 < FN) load(f + 1);
#pragma unroll
            for (int t = 0; t < FM; ++t) mx4_store<C::FAR>(p, row_of(t), feature_of(f), acc[f][t], {bias[f], x[f & 1][t]});
        }
        return;
    }
    // bf16 by way of LDS: a store straight from the registers would cover 16 rows x 32 bytes
    __syncthreads();
#pragma unroll
    for (int f = 0; f < FN; ++f) {
#pragma unroll
        for (int t = 0; t < FM; ++t) {
            f32x4 v = acc[f][t];
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                v[e] += bias[f][e];
                if (p.epi == Epi::BiasGeluBf16) v[e] = gelu(v[e]);
            }
            *reinterpret_cast<u32x2 *>(lds + ((wm * FM + t) * 16 + r) * C::ROW + ((wn * FN + f) * 16 + 4 * c) * 2) =
                u32x2{pack2(v[0], v[1]), pack2(v[2], v[3])};
        }
    }
    __syncthreads();
    constexpr int PIECES = C::BN / 8;      // of a row
    bf16_t *out = static_cast<bf16_t *>(p.out);
    for (int i = threadIdx.x; i < C::BM * PIECES; i += 64 * NW) {
        const int m = rt0 * 16 + i / PIECES, n = ft0 * 16 + i % PIECES * 8;
        if (m < p.M && n < p.N)
            put<C::FAR>(reinterpret_cast<u32x4 *>(out + (size_t)m * p.N + n),
                        *reinterpret_cast<const u32x4 *>(lds + i / PIECES * C::ROW + i % PIECES * 16));
    }
}

template <class C>
hipError_t launch_tile(const Mx4Params &p, hipStream_t stream) {
    const int tiles_m = (p.M + C::BM - 1) / C::BM, tiles_n = (p.N + C::BN - 1) / C::BN;
    return launch_kernel(mx4_tile_kernel<C>, dim3((unsigned)((int64_t)tiles_m * tiles_n)), dim3(64 * C::NW), stream, p, tiles_m, tiles_n);
}


// Up to 16 rows (tiles: of features): two tiles a workgroup halve what is read and made of the rows, and are taken where the
// workgroups still fill the chip, four where 16 bf16 rows have to be quantised besides; 16 waves have more of a long row in flight
// where there is one workgroup a CU.  us, FT 1 / 2 / 4 with 8 waves, 1 with 16:
//   bf16  1 x 2048 -> 8192    3.8  3.5  4.2  4.4      16 x 2048 -> 8192    5.6  4.7  4.9  6.7
//         1 x 4096 -> 16384   6.6  6.2  6.3  8.0      16 x 4096 -> 16384  14.3  9.4  8.5 16.8
//         1 x 8192 -> 2048    4.7  5.1  6.5  4.6      16 x 11008 -> 4096  11.2 11.2 12.7  9.9
//   mx4  16 x 4096 -> 16384   6.3  5.8  6.1  7.7      16 x 8192 -> 2048    4.0  4.5  5.9  4.1
template <int NL>
hipError_t launch_few(const Mx4Params &p, hipStream_t stream) {
    const int tiles = (p.N + 15) / 16;
    if constexpr (NL == 4)
        if (tiles >= 1024) return launch_split<4, 1, 8, NL>(p, stream);
    if (tiles >= 512) return launch_split<2, 1, 8, NL>(p, stream);
    if constexpr (NL > 0)
        if (mx4_chunks(p.K) >= 64) return launch_split<1, 1, 16, NL>(p, stream);
    return launch_split<1, 1, 8, NL>(p, stream);
}

int64_t tiles_of(int M, int N, int side) { return (int64_t)((M + side - 1) / side) * ((N + side - 1) / side); }

}  // namespace

// More rows: the largest tile whose workgroups fill the chip, 32 x 32 with the waves along K where even 64 x 64 do not.  us, 32 / 64 /
// 128 / 256 tiles (M x N x K), with a bias alone:
//    64 x  4096 x 4096   4.5  8.8 12.1            201 x  4096 x 4096  12.2  7.7 10.0
//   201 x  1024 x 4096   4.5  7.4  9.8            512 x  4096 x 4096  16.8  9.9 10.5
//   128 x  8192 x 2048   7.7  5.9  7.4           1000 x  4096 x 4096  28.2 19.6 13.3
//  4096 x  4096 x 4096             42.2 37.1     2048 x  8192 x 2048             27.4 24.2
// The rule does not look at how much of a tile the rows fill: a few dozen of them by a vocabulary go to 256 x 256 tiles as well, where
// 128 x 128 would be faster (48 x 131072 x 4096 in 64 / 128 / 256 tiles 62 57 83, 128 x 131072 x 4096 111 66 82, 48 x 65536 x 2048
// 17 16 23; but 200 x 65536 x 4096 75 43 38).
// An output of more than 32 MiB goes past the last cache, which the operands need (with quantisation, us, without / with the hint):
//   8192 x 16384 x 2048, GELU 274 233     4096 x 4096 x 4096, fp32 residual 83 74
//   8192 x 8192 x 8192 285 278            4096 x 4096 x 4096 bf16 45.6 46.2
hipError_t launch_mx4_gemm(Epi epi, const void *a, const void *w, const bf16_t *bias, const float *resid, void *out, int M,
                           int N, int K, hipStream_t stream) {
    const Mx4Params p{static_cast<const char *>(a), static_cast<const char *>(w), nullptr, bias, resid, out, M, N, K, 0, epi};
    if (M <= 16) return launch_few<0>(p, stream);
    if (M <= 32) return N > 8176 ? launch_split<2, 2, 8, 0>(p, stream) : launch_split<1, 2, 8, 0>(p, stream);
    if (tiles_of(M, N, 32) <= 320) return launch_split<2, 2, 8, 0>(p, stream);
    if (tiles_of(M, N, 64) <= 512) return launch_tile<TileCfg<64, 64, 2, 2, 4, 2>>(p, stream);
    if (tiles_of(M, N, 256) >= 192) {
        const bool far = (int64_t)M * N * (epi == Epi::BiasResidF32 ? 4 : 2) > 32 << 20;
        return far ? launch_tile<TileCfg<256, 256, 2, 4, 1, 4, true>>(p, stream) : launch_tile<TileCfg<256, 256, 2, 4, 1, 4>>(p, stream);
    }
    return launch_tile<TileCfg<128, 128, 4, 2, 1, 4>>(p, stream);
}

hipError_t launch_mx4_gemm_bf16(Epi epi, const bf16_t *a, const void *w, const bf16_t *bias, const float *resid, void *out,
                                int M, int N, int K, hipStream_t stream) {
    const Mx4Params p{nullptr, static_cast<const char *>(w), a, bias, resid, out, M, N, K, 0, epi};
    if (M <= 4) return launch_few<1>(p, stream);
    if (M <= 8) return launch_few<2>(p, stream);
    return launch_few<4>(p, stream);
}

}  // namespace iefwd
