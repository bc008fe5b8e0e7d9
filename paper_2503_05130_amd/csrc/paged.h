// Launchers of the paged key-value cache's kernels (csrc/paged.hip).  They
// check nothing: the C entry points do.
#pragma once

#include "launch.h"

namespace iefwd {

enum class KvKind : int { Bf16 = 0, E4m3 = 1, Mx4 = 3 };      // as IEFWD_KV_*

// A pool of pages of `page` tokens.  K [n_pages, kv_heads, dh / E, page, E]
// with E = 16 bytes' worth of elements, V [n_pages, kv_heads, page / 4, dh, 4].
// Mx4: per page and head, K [dh / 32, page, 16 bytes] and then its scales [dh / 32, page]; V [page / 4, dh / 8, 4 tokens,
// 4 bytes of 8 columns] and then its scales [page / 4, dh / 32, 4 tokens].
struct PagedCache {
    void *k, *v;
    const float *k_scale, *v_scale;   // [kv_heads], 8-bit caches only
    int n_pages, page_log2, kv_heads, head_dim;
    KvKind kind;

    // of K (or V) of one head of a page
    size_t page_bytes() const {
        const size_t elements = (size_t)head_dim << page_log2;
        return kind == KvKind::Mx4 ? elements / 32 * 17 : kind == KvKind::E4m3 ? elements : elements * 2;
    }
};

constexpr int kPlanMaxBatch = 4096;
constexpr float kLog2e = 1.4426950408889634f;

struct PlanArgs {
    const int32_t *lens, *new_lens;
    int32_t *lens_out;
    int32_t *table;
    int32_t *ring;
    const int64_t *counters;
    int64_t *counters_out;
    int64_t *slots;
    int32_t *starts;
    int32_t *refused;
    int batch, table_stride, max_pages, ring_size, room, page_log2;
};
hipError_t launch_paged_plan(const PlanArgs &p, hipStream_t stream);

// k, v: bf16 rows of kv_heads * head_dim elements, k_stride / v_stride apart
// (multiples of 8); slots[i] = page * page size + place, anything outside the
// pool is skipped.
hipError_t launch_paged_append(const PagedCache &c, const bf16_t *k, const bf16_t *v, const int64_t *slots, int tokens,
                               int64_t k_stride, int64_t v_stride, hipStream_t stream);

// The same for a Mx4 cache.
hipError_t launch_paged_append_mx4(const PagedCache &c, const bf16_t *k, const bf16_t *v, const int64_t *slots, int tokens,
                                   int64_t k_stride, int64_t v_stride, hipStream_t stream);

// The inverse: the slots' keys and values in bf16, rows of kv_heads * head_dim elements, strides as above; zeros for a slot
// outside the pool.
hipError_t launch_paged_read(const PagedCache &c, const int64_t *slots, bf16_t *k, bf16_t *v, int tokens, int64_t k_stride,
                             int64_t v_stride, hipStream_t stream);

// What becomes of a score s = scale q . k before the softmax: cap tanh(s / cap) (cap 0: s), less slopes[head] times the
// distance of the key from the newest one (null: 0).
struct ScoreForm {
    float cap;
    const float *slopes;
};

// q bf16 rows of heads * head_dim elements q_stride apart (a multiple of 8);
// ctx bf16 [batch, heads * head_dim]; partials: paged_workspace_floats floats.
size_t paged_workspace_floats(const PagedCache &c, int batch, int heads, int max_keys);
hipError_t launch_paged_attention(const PagedCache &c, const bf16_t *q, int64_t q_stride, const int32_t *table,
                                  int table_stride, int max_pages, const int32_t *lens, bf16_t *ctx, float *partials,
                                  int batch, int heads, float scale, ScoreForm form, hipStream_t stream);

}  // namespace iefwd
