// Host-side checks of the paged cache's and the 4-bit product's entry points, built with AddressSanitizer and
// UndefinedBehaviorSanitizer (tests/test_paged_sanitizers.py builds and runs it): every refusal with a descriptor in a heap
// block of its own size, the sizes and the split over their whole range.  Nothing is launched: each call is refused.
#include <cmath>
#include <cstdint>
#include <cstdio>
#include <cstring>
#include <memory>
#include <vector>

#include "iefwd.h"

static int failures = 0;
#define CHECK(c)                                                              \
    do {                                                                      \
        if (!(c)) {                                                           \
            std::fprintf(stderr, "check failed at line %d: %s\n", __LINE__, #c); \
            ++failures;                                                       \
        }                                                                     \
    } while (0)

template <class T>
static T *at(uintptr_t a) { return reinterpret_cast<T *>(a); }      // an address that nothing reads

static std::unique_ptr<iefwd_paged_cache> cache() {
    auto c = std::make_unique<iefwd_paged_cache>();
    std::memset(c.get(), 0, sizeof *c);
    c->abi_version = IEFWD_ABI_VERSION;
    c->n_pages = 10;
    c->page_size = 16;
    c->n_kv_heads = 4;
    c->head_dim = 64;
    c->k = at<void>(4096);
    c->v = at<void>(8192);
    return c;
}

static int append(const iefwd_paged_cache *c, uintptr_t k, uint64_t stride, uint32_t n) {
    return iefwd_paged_append(c, at<void>(k), at<void>(4096), at<int64_t>(4096), n, stride, stride, nullptr);
}

static int attention(const iefwd_paged_cache *c, uint64_t q_stride, uint32_t heads, uint32_t stride, uint32_t pages, uint32_t batch,
                     float scale, uintptr_t ws, size_t bytes) {
    return iefwd_paged_attention(c, at<void>(4096), q_stride, heads, at<int32_t>(4096), stride, pages, at<int32_t>(4096), batch, scale,
                                 at<void>(4096), at<void>(ws), bytes, nullptr);
}

static void check_caches() {
    struct Bad {
        void (*edit)(iefwd_paged_cache &);
        int status;
    } bad[] = {
        {[](iefwd_paged_cache &c) { c.abi_version = 0; }, IEFWD_EVERSION},
        {[](iefwd_paged_cache &c) { c.kv_type = 2; }, IEFWD_EINVAL},
        {[](iefwd_paged_cache &c) { c.kv_type = IEFWD_KV_E4M3; }, IEFWD_EINVAL},
        {[](iefwd_paged_cache &c) { c.n_pages = 0; }, IEFWD_EINVAL},
        {[](iefwd_paged_cache &c) { c.n_pages = 0xffffffffu; }, IEFWD_EINVAL},
        {[](iefwd_paged_cache &c) { c.page_size = 48; }, IEFWD_EINVAL},
        {[](iefwd_paged_cache &c) { c.page_size = 0xffffffffu; }, IEFWD_EINVAL},
        {[](iefwd_paged_cache &c) { c.n_kv_heads = 0; }, IEFWD_EINVAL},
        {[](iefwd_paged_cache &c) { c.n_kv_heads = 0xffffffffu; }, IEFWD_EINVAL},
        {[](iefwd_paged_cache &c) { c.head_dim = 96; }, IEFWD_EINVAL},
        {[](iefwd_paged_cache &c) { c.k = nullptr; }, IEFWD_EINVAL},
        {[](iefwd_paged_cache &c) { c.v = at<void>(4097); }, IEFWD_EINVAL},
    };
    for (const Bad &b : bad) {
        auto c = cache();
        b.edit(*c);
        auto bytes = std::make_unique<size_t>(7);
        CHECK(append(c.get(), 4096, 256, 3) == b.status);
        CHECK(attention(c.get(), 512, 8, 10, 10, 2, 1.f, 4096, 1 << 20) == b.status);
        CHECK(iefwd_paged_attention_workspace(c.get(), 2, 8, 10, bytes.get()) == b.status && *bytes == 7);
        CHECK(std::strlen(iefwd_last_error()) > 0);
    }
    CHECK(append(nullptr, 4096, 256, 3) == IEFWD_EINVAL);
    CHECK(attention(nullptr, 512, 8, 10, 10, 2, 1.f, 4096, 1 << 20) == IEFWD_EINVAL);
    CHECK(iefwd_paged_attention_workspace(cache().get(), 2, 8, 10, nullptr) == IEFWD_EINVAL);
}

static void check_sizes() {
    auto c = cache();
    CHECK(append(c.get(), 4096, 256, 0) == IEFWD_OK);
    CHECK(append(c.get(), 0, 256, 3) == IEFWD_EINVAL);
    CHECK(append(c.get(), 4098, 256, 3) == IEFWD_EINVAL);
    for (uint64_t stride : {0ull, 248ull, 257ull, 1ull << 41, ~0ull, ~7ull}) CHECK(append(c.get(), 4096, stride, 3) == IEFWD_EINVAL);
    CHECK(append(c.get(), 4096, 256, 0xffffffffu) == IEFWD_EINVAL);
    // sizes whose products pass 32 and 64 bits
    const uint32_t big[] = {0u, 1u << 27, 0x7fffffffu, 0x80000000u, 0xffffffffu};
    for (uint32_t x : big) {
        CHECK(attention(c.get(), 512, 8, x, x, 2, 1.f, 4096, 1 << 20) == IEFWD_EINVAL);
        CHECK(attention(c.get(), 512, x, 10, 10, 2, 1.f, 4096, 1 << 20) == IEFWD_EINVAL);
        CHECK(attention(c.get(), 512, 8, 10, 10, x, 1.f, 4096, 1 << 20) == IEFWD_EINVAL);
        CHECK(iefwd_paged_attention_workspace(c.get(), 2, 8, x, std::make_unique<size_t>().get()) == IEFWD_EINVAL);
    }
    CHECK(attention(c.get(), 504, 8, 10, 10, 2, 1.f, 4096, 1 << 20) == IEFWD_EINVAL);
    for (float scale : {INFINITY, -INFINITY, NAN, 3e38f}) CHECK(attention(c.get(), 512, 8, 10, 10, 2, scale, 4096, 1 << 20) == IEFWD_EINVAL);
    CHECK(attention(c.get(), 512, 8, 200, 200, 2, 1.f, 4096, 8) == IEFWD_EINVAL);
    CHECK(attention(c.get(), 512, 8, 200, 200, 2, 1.f, 0, 1 << 30) == IEFWD_EINVAL);
    CHECK(attention(c.get(), 512, 8, 200, 200, 2, 1.f, 4100, 1 << 30) == IEFWD_EINVAL);
    // the workspace holds the parts of every length, for every shape and up to the longest table
    for (uint32_t batch : {1u, 3u, 64u, 255u, 4096u})
        for (uint32_t heads : {4u, 8u, 68u, 1024u})
            for (uint32_t pages : {1u, 33u, 1000u, 1u << 20, 1u << 26}) {
                auto bytes = std::make_unique<size_t>();
                auto keys = std::make_unique<uint32_t>();
                CHECK(iefwd_paged_attention_workspace(c.get(), batch, heads, pages, bytes.get()) == IEFWD_OK);
                for (uint64_t n = 1; n <= 16ull * pages; n = n * 5 / 4 + 1) {
                    CHECK(iefwd_test_paged_split(batch, heads, 4, (uint32_t)n, keys.get()) == IEFWD_OK);
                    const uint64_t parts = (n + *keys - 1) / *keys;
                    CHECK(parts == 1 || parts * batch * heads * (64 + 2) * 4 <= *bytes);
                }
            }
    CHECK(iefwd_test_paged_split(1, 4, 4, 1, nullptr) == IEFWD_EINVAL);
    CHECK(iefwd_test_paged_split(1, 4, 4, 0xffffffffu, std::make_unique<uint32_t>().get()) == IEFWD_EINVAL);
    CHECK(iefwd_test_paged_split(1, 4, 0, 1, std::make_unique<uint32_t>().get()) == IEFWD_EINVAL);
}

static int plan(uint32_t batch, uint32_t page, uint32_t stride, uint32_t pages, uint32_t ring, uint32_t room, uintptr_t lens_out) {
    return iefwd_paged_plan(batch, page, at<int32_t>(4096), at<int32_t>(8192), at<int32_t>(4096), stride, pages, at<int32_t>(4096), ring,
                            at<int64_t>(4096), at<int32_t>(lens_out), at<int64_t>(8192), at<int64_t>(room ? 4096 : 0), room,
                            at<int32_t>(4096), at<int32_t>(4096), nullptr);
}

static void check_plan() {
    const uint32_t m = 0xffffffffu;
    CHECK(plan(0, 16, 9, 9, 9, 9, 12288) == IEFWD_EINVAL);
    CHECK(plan(m, 16, 9, 9, 9, 9, 12288) == IEFWD_EINVAL);
    CHECK(plan(4, m, 9, 9, 9, 9, 12288) == IEFWD_EINVAL);
    CHECK(plan(4, 16, 8, 9, 9, 9, 12288) == IEFWD_EINVAL);
    CHECK(plan(4, 16, m, 9, 9, 9, 12288) == IEFWD_EINVAL);
    CHECK(plan(4, 256, m, m, 9, 9, 12288) == IEFWD_EINVAL);
    CHECK(plan(4, 16, 9, 9, 0, 9, 12288) == IEFWD_EINVAL);
    CHECK(plan(4, 16, 9, 9, m, 9, 12288) == IEFWD_EINVAL);
    CHECK(plan(4, 16, 9, 9, 9, m, 12288) == IEFWD_EINVAL);
    CHECK(plan(4, 16, 9, 9, 9, 9, 0) == IEFWD_EINVAL);
    CHECK(plan(4, 16, 9, 9, 9, 9, 4096) == IEFWD_EINVAL);
    CHECK(plan(4, 16, 9, 9, 9, 9, 8192) == IEFWD_EINVAL);
}

static void check_q4() {
    const uint32_t bad[][3] = {{0, 128, 64}, {24, 128, 64}, {32, 0, 64}, {32, 96, 64}, {32, 128, 0}, {32, 128, 48}, {1u << 20, 4096, 64},
                               {16, (1u << 24) + 128, 128}, {0xfffffff0u, 0xffffff80u, 128}};
    for (const auto &b : bad) {
        auto bytes = std::make_unique<size_t>(7);
        CHECK(iefwd_q4_packed_bytes(b[0], b[1], b[2], bytes.get()) == IEFWD_EINVAL && *bytes == 7);
        CHECK(iefwd_q4_pack(at<void>(4096), at<void>(4096), nullptr, at<void>(4096), b[0], b[1], b[2], nullptr) == IEFWD_EINVAL);
        CHECK(iefwd_q4_gemm(0, at<void>(4096), at<void>(4096), nullptr, nullptr, at<void>(4096), 1, b[0], b[1], b[2], nullptr) == IEFWD_EINVAL);
    }
    auto bytes = std::make_unique<size_t>();
    for (uint32_t group : {32u, 64u, 128u})
        for (uint32_t n : {16u, 1u << 20, (1u << 26) - 16})
            for (uint64_t k = group; k <= 1u << 24 && (uint64_t)n * k < 1ull << 31; k = k * 3 / group * group) {
                CHECK(iefwd_q4_packed_bytes(n, (uint32_t)k, group, bytes.get()) == IEFWD_OK);
                CHECK(*bytes >= (uint64_t)n * k / 2 + (uint64_t)n * (k / group) * 4);
            }
    CHECK(iefwd_q4_packed_bytes(16, 128, 64, nullptr) == IEFWD_EINVAL);
    CHECK(iefwd_q4_pack(nullptr, at<void>(4096), nullptr, at<void>(4096), 16, 128, 64, nullptr) == IEFWD_EINVAL);
    CHECK(iefwd_q4_pack(at<void>(4096), at<void>(4096), nullptr, at<void>(4104), 16, 128, 64, nullptr) == IEFWD_EINVAL);
    for (uint32_t m : {0u, 17u, 0xffffffffu})
        CHECK(iefwd_q4_gemm(0, at<void>(4096), at<void>(4096), nullptr, nullptr, at<void>(4096), m, 16, 128, 64, nullptr) == IEFWD_EINVAL);
    for (uint32_t epi : {3u, 0xffffffffu, (uint32_t)IEFWD_EPI_BIAS_RESID_F32})
        CHECK(iefwd_q4_gemm(epi, at<void>(4096), at<void>(4096), nullptr, nullptr, at<void>(4096), 1, 16, 128, 64, nullptr) == IEFWD_EINVAL);
}

int main() {
    check_caches();
    check_sizes();
    check_plan();
    check_q4();
    if (failures) return 1;
    std::printf("paged host sanitizer checks passed\n");
    return 0;
}
