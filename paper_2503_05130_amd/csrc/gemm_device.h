// What the products (gemm.hip, decode.hip, mx4_gemm.hip) share on the device:
// vector types, the kernels' parameters, the order of their tiles, the
// global-to-LDS copies and the bf16 conversions.
#pragma once

#include "gelu.h"
#include "gemm.h"

namespace iefwd {
namespace {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef __attribute__((address_space(3))) void *lds_ptr_t;

struct GemmParams {
    const bf16_t *a;
    const bf16_t *w;
    const bf16_t *bias;
    const float *resid;
    void *out;
    int M, N, K;
    int tiles_m, tiles_n;
    QkvDst qkv;
    LnResid ln;
    LnIn lnin;
    const bf16_t *aux;   // Epi::GeluBwdBf16: the GELU's input [M, N]
    bf16_t *out2;        // Epi::BiasGelu2Bf16: GELU(out) [M, N]
};

// Workgroups are dispatched round-robin over the 8 XCDs.  Renumber them so
// that each XCD receives a contiguous range of logical tiles (bijective for
// any grid size), which keeps tiles that share operands in one XCD's L2.
__device__ inline int xcd_contiguous(int i, int g) {
    constexpr int X = 8;
    const int q = g / X, r = g % X;
    const int x = i % X, local = i / X;
    return x < r ? x * (q + 1) + local : r * (q + 1) + (x - r) * q + local;
}

// Logical tile -> (token tile, feature tile), grouped 4 token tiles deep so
// that workgroups running together share both A rows and W rows.
__device__ inline void grouped_tile(int l, int tiles_m, int tiles_n, int &tm, int &tn) {
    constexpr int G = 4;
    const int per_group = G * tiles_n;
    const int g = l / per_group;
    const int first = g * G;
    const int gsize = min(tiles_m - first, G);
    const int in = l - g * per_group;
    tm = first + in % gsize;
    tn = in / gsize;
}

// One global->LDS copy of 16 bytes per lane (1 KB per wave) to the
// wave-uniform LDS byte address `lds`.  Issued through inline asm: the
// compiler's wait-count model treats these copies as LDS traffic that may
// complete out of order with LDS reads, and would then drain every
// outstanding LDS read before each use of any of them; the main loop orders
// the copies itself (s_waitcnt vmcnt before each barrier).  The M0 write
// needs one wait state before the copy reads it.
__device__ inline void dma16(const void *base, uint32_t off, uint32_t lds) {
    uint32_t m0;   // the asm writes M0; naming it as an output tells the compiler so
    asm volatile("s_mov_b32 %0, %3\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2"
                 : "={m0}"(m0)
                 : "v"(off), "s"(base), "s"(lds)
                 : "memory");
    (void)m0;
}

// s_waitcnt immediate: wait until at most vm vector-memory and lgkm LDS
// operations of this wave are outstanding (expcnt left unconstrained).
constexpr int waitcnt_imm(int vm, int lgkm) { return (vm & 15) | (7 << 4) | ((lgkm & 15) << 8) | ((vm >> 4) << 14); }

__device__ inline bf16_t f32_to_bf16(float f) {
    __bf16 b = (__bf16)f;   // round to nearest even
    return __builtin_bit_cast(bf16_t, b);
}

__device__ inline uint32_t pack2(float lo, float hi) {
    return (uint32_t)f32_to_bf16(lo) | ((uint32_t)f32_to_bf16(hi) << 16);
}

}  // namespace
}  // namespace iefwd
