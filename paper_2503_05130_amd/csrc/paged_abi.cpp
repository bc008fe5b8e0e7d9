// C ABI of token generation over a paged cache: planning, append, attention and the
// products with 4-bit weights.  All checks of their arguments are here.
#include <cmath>
#include <cstdint>
#include <string>

#include "abi.h"
#include "paged.h"
#include "paged_split.h"
#include "q4.h"

using namespace iefwd;

namespace {

bool aligned16(const void *p) { return ((uintptr_t)p & 15) == 0; }

int log2_page(uint32_t page_size) {
    for (int i = 4; i <= 8; ++i)
        if (page_size == 1u << i) return i;
    fail(IEFWD_EINVAL, "page_size must be 16, 32, 64, 128 or 256");
}

// The checked, device-side form of a cache descriptor.
PagedCache paged_cache(const iefwd_paged_cache *c) {
    if (!c) fail(IEFWD_EINVAL, "cache is NULL");
    if (c->abi_version != IEFWD_ABI_VERSION) fail(IEFWD_EVERSION, "cache: ABI version mismatch");
    if (c->kv_type > IEFWD_KV_E4M3) fail(IEFWD_EINVAL, "unknown kv_type");
    if (c->n_pages == 0 || c->n_pages > 0x7fffffffu) fail(IEFWD_EINVAL, "n_pages must be in [1, 2^31 - 1]");
    if (c->n_kv_heads == 0 || c->n_kv_heads > 1024) fail(IEFWD_EINVAL, "n_kv_heads must be in [1, 1024]");
    if (c->head_dim != 64 && c->head_dim != 128) fail(IEFWD_EINVAL, "head_dim must be 64 or 128");
    const int log2 = log2_page(c->page_size);
    if (!c->k || !c->v || !aligned16(c->k) || !aligned16(c->v)) fail(IEFWD_EINVAL, "k and v must be 16-byte aligned");
    const bool e4m3 = c->kv_type == IEFWD_KV_E4M3;
    if (e4m3 && (!c->k_scale || !c->v_scale)) fail(IEFWD_EINVAL, "an 8-bit cache needs k_scale and v_scale");
    return {c->k, c->v, c->k_scale, c->v_scale, (int)c->n_pages, log2, (int)c->n_kv_heads, (int)c->head_dim, e4m3};
}

void check_table(uint32_t table_stride, uint32_t max_pages, int page_log2) {
    if (max_pages == 0 || ((uint64_t)max_pages << page_log2) > (1u << 30))
        fail(IEFWD_EINVAL, "max_pages * page_size must be in [1, 2^30]");
    if (table_stride < max_pages || table_stride > 0x7fffffffu)
        fail(IEFWD_EINVAL, "table_stride must be at least max_pages and below 2^31");
}

void check_row_stride(const char *what, const void *p, uint64_t stride, uint64_t row) {
    if (!p) fail(IEFWD_EINVAL, std::string(what) + " is NULL");
    if (!aligned16(p) || stride < row || stride % 8 || stride > (1ull << 40))
        fail(IEFWD_EINVAL, std::string(what) + ": rows must be 16-byte aligned and not overlap");
}

void check_batch_heads(uint32_t batch, uint32_t n_heads, uint32_t n_kv_heads) {
    if (batch == 0 || batch > 65535) fail(IEFWD_EINVAL, "batch must be in [1, 65535]");
    if (n_heads == 0 || n_heads > 1024 || n_kv_heads == 0 || n_heads % n_kv_heads)
        fail(IEFWD_EINVAL, "n_heads must be a multiple of n_kv_heads, at most 1024");
    if ((uint64_t)batch * n_heads > (1u << 22)) fail(IEFWD_EINVAL, "batch * n_heads must be at most 2^22");
}

// The workspace's size, with the argument checks that it shares with the launch.
size_t paged_workspace(const PagedCache &c, uint32_t batch, uint32_t n_heads, uint32_t max_pages) {
    check_batch_heads(batch, n_heads, (uint32_t)c.kv_heads);
    return 4 * paged_workspace_floats((int)batch, (int)n_heads, c.kv_heads, c.head_dim, (int)(max_pages << c.page_log2));
}

void check_q4(uint32_t N, uint32_t K, uint32_t group) {
    if (group != 32 && group != 64 && group != 128) fail(IEFWD_EINVAL, "group must be 32, 64 or 128");
    if (N == 0 || N % 16 || K == 0 || K % group) fail(IEFWD_EINVAL, "N must be a positive multiple of 16, K of group");
    if ((uint64_t)N * K >= (1ull << 31) || K > (1u << 24)) fail(IEFWD_EINVAL, "too large");
}

}  // namespace

extern "C" {

int iefwd_paged_plan(uint32_t batch, uint32_t page_size, const int32_t *lens, const int32_t *new_lens, int32_t *table,
                     uint32_t table_stride, uint32_t max_pages, int32_t *ring, uint32_t ring_size,
                     const int64_t *counters, int32_t *lens_out, int64_t *counters_out, int64_t *slots,
                     uint32_t max_new, int32_t *starts, int32_t *refused, void *stream) {
    return guarded([&] {
        if (!lens || !new_lens || !table || !ring || !counters || !lens_out || !counters_out || !starts || !refused)
            fail(IEFWD_EINVAL, "NULL pointer");
        if (!slots && max_new) fail(IEFWD_EINVAL, "slots is NULL");
        if (batch == 0 || batch > (uint32_t)kPlanMaxBatch) fail(IEFWD_EINVAL, "batch must be in [1, 4096]");
        const int log2 = log2_page(page_size);
        check_table(table_stride, max_pages, log2);
        if (ring_size == 0 || ring_size > 0x7fffffffu || max_new > 0x7fffffffu)
            fail(IEFWD_EINVAL, "ring_size must be in [1, 2^31 - 1] and max_new below 2^31");
        if (lens_out == lens || lens_out == new_lens || counters_out == counters)
            fail(IEFWD_EINVAL, "lens_out and counters_out must be buffers of their own");
        PlanArgs p{};
        p.lens = lens;
        p.new_lens = new_lens;
        p.lens_out = lens_out;
        p.table = table;
        p.ring = ring;
        p.counters = counters;
        p.counters_out = counters_out;
        p.slots = slots;
        p.starts = starts;
        p.refused = refused;
        p.batch = (int)batch;
        p.table_stride = (int)table_stride;
        p.max_pages = (int)max_pages;
        p.ring_size = (int)ring_size;
        p.room = (int)max_new;
        p.page_log2 = log2;
        hip_check(launch_paged_plan(p, (hipStream_t)stream), "paged plan launch");
    });
}

int iefwd_paged_append(const iefwd_paged_cache *cache, const void *k, const void *v, const int64_t *slots,
                       uint32_t n_tokens, uint64_t k_stride, uint64_t v_stride, void *stream) {
    return guarded([&] {
        const PagedCache c = paged_cache(cache);
        const uint64_t row = (uint64_t)c.kv_heads * c.head_dim;
        if (n_tokens == 0) return;
        check_row_stride("k", k, k_stride, row);
        check_row_stride("v", v, v_stride, row);
        if (!slots) fail(IEFWD_EINVAL, "slots is NULL");
        if ((uint64_t)n_tokens * c.kv_heads > (1u << 28)) fail(IEFWD_EINVAL, "n_tokens * n_kv_heads must be at most 2^28");
        hip_check(launch_paged_append(c, (const bf16_t *)k, (const bf16_t *)v, slots, (int)n_tokens, (int64_t)k_stride,
                                      (int64_t)v_stride, (hipStream_t)stream),
                  "paged append launch");
    });
}

int iefwd_paged_attention_workspace(const iefwd_paged_cache *cache, uint32_t batch, uint32_t n_heads,
                                    uint32_t max_pages, size_t *bytes) {
    return guarded([&] {
        if (!bytes) fail(IEFWD_EINVAL, "bytes is NULL");
        const PagedCache c = paged_cache(cache);
        check_table(max_pages, max_pages, c.page_log2);
        *bytes = paged_workspace(c, batch, n_heads, max_pages);
    });
}

int iefwd_paged_attention(const iefwd_paged_cache *cache, const void *q, uint64_t q_stride, uint32_t n_heads,
                          const int32_t *table, uint32_t table_stride, uint32_t max_pages, const int32_t *lens,
                          uint32_t batch, float scale, void *ctx, void *workspace, size_t workspace_bytes,
                          void *stream) {
    return guarded([&] {
        const PagedCache c = paged_cache(cache);
        check_table(table_stride, max_pages, c.page_log2);
        const size_t need = paged_workspace(c, batch, n_heads, max_pages);
        check_row_stride("q", q, q_stride, (uint64_t)n_heads * c.head_dim);
        if (!table || !lens || !ctx) fail(IEFWD_EINVAL, "NULL pointer");
        if (!aligned16(ctx)) fail(IEFWD_EINVAL, "ctx must be 16-byte aligned");
        // the kernel's exponent is in powers of two; infinity times a product of 0 would be NaN
        if (!std::isfinite(scale * kLog2e)) fail(IEFWD_EINVAL, "scale * log2(e) must be finite");
        if (workspace_bytes < need || (need && (!workspace || !aligned16(workspace))))
            fail(IEFWD_EINVAL, "workspace of " + std::to_string(need) + " bytes (16-byte aligned) needed, " +
                                   std::to_string(workspace_bytes) + " given");
        hip_check(launch_paged_attention(c, (const bf16_t *)q, (int64_t)q_stride, table, (int)table_stride, (int)max_pages,
                                         lens, (bf16_t *)ctx, static_cast<float *>(workspace), (int)batch, (int)n_heads,
                                         scale, (hipStream_t)stream),
                  "paged attention launch");
    });
}

int iefwd_test_paged_split(uint32_t batch, uint32_t n_heads, uint32_t n_kv_heads, uint32_t n_keys, uint32_t *part_keys) {
    return guarded([&] {
        if (!part_keys) fail(IEFWD_EINVAL, "NULL pointer");
        check_batch_heads(batch, n_heads, n_kv_heads);
        if (n_keys > (1u << 30)) fail(IEFWD_EINVAL, "n_keys must be at most 2^30");
        *part_keys = 1u << paged_part_log2((int)n_keys, paged_split((int)batch, (int)n_heads, (int)n_kv_heads));
    });
}

int iefwd_q4_packed_bytes(uint32_t N, uint32_t K, uint32_t group, size_t *bytes) {
    return guarded([&] {
        if (!bytes) fail(IEFWD_EINVAL, "bytes is NULL");
        check_q4(N, K, group);
        *bytes = q4_packed_bytes((int)N, (int)K, (int)group);
    });
}

int iefwd_q4_pack(const void *codes, const void *scales, const void *zeros, void *dst, uint32_t N, uint32_t K,
                  uint32_t group, void *stream) {
    return guarded([&] {
        check_q4(N, K, group);
        if (!codes || !scales || !dst) fail(IEFWD_EINVAL, "NULL pointer");
        if (!aligned16(dst)) fail(IEFWD_EINVAL, "dst must be 16-byte aligned");
        hip_check(launch_q4_pack((const uint8_t *)codes, (const bf16_t *)scales, (const uint8_t *)zeros, dst, (int)N,
                                 (int)K, (int)group, (hipStream_t)stream),
                  "4-bit pack launch");
    });
}

int iefwd_q4_gemm(uint32_t epilogue, const void *a, const void *packed, const void *bias, const float *resid, void *out,
                  uint32_t M, uint32_t N, uint32_t K, uint32_t group, void *stream) {
    return guarded([&] {
        check_q4(N, K, group);
        if (epilogue > IEFWD_EPI_BIAS_RESID_F32) fail(IEFWD_EINVAL, "unknown epilogue");
        if (!a || !packed || !out) fail(IEFWD_EINVAL, "NULL pointer");
        if (epilogue == IEFWD_EPI_BIAS_RESID_F32 && !resid) fail(IEFWD_EINVAL, "resid is NULL");
        if (M == 0 || M > 16) fail(IEFWD_EINVAL, "M must be in [1, 16]");
        if (!aligned16(a) || !aligned16(packed)) fail(IEFWD_EINVAL, "a and packed must be 16-byte aligned");
        hip_check(launch_q4_gemm((Epi)epilogue, (const bf16_t *)a, packed, (const bf16_t *)bias, resid, out, (int)M, (int)N,
                                 (int)K, (int)group, (hipStream_t)stream),
                  "4-bit product launch");
    });
}

}  // extern "C"
