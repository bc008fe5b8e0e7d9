// Host-side checks of the entry points of the 4-bit matrices, the 4-bit cache and the log probabilities, built with AddressSanitizer
// and UndefinedBehaviorSanitizer (tests/test_mx4_sanitizers.py builds and runs it): refusals and sizes over their
// whole range.  Nothing is launched: each call is refused.
#include <cmath>
#include <cstdint>
#include <cstdio>
#include <cstring>
#include <memory>

#include "iefwd.h"

static int failures = 0;
#define CHECK(c)                                                              \
    do {                                                                      \
        if (!(c)) {                                                           \
            std::fprintf(stderr, "check failed at line %d: %s\n", __LINE__, #c); \
            ++failures;                                                       \
        }                                                                     \
    } while (0)

template <class T = void>
static T *at(uintptr_t a) { return reinterpret_cast<T *>(a); }      // an address that nothing reads

static const uint32_t kSizes[] = {0, 1, 2, 15, 16, 17, 31, 128, 129, 4096, 65535, 1u << 20, (1u << 20) + 1, 1u << 22, (1u << 22) + 1, 1u << 24,
                                  (1u << 24) + 1, 0x7fffffffu, 0x80000000u, 0xffffffffu};

static bool matrix(uint32_t rows, uint32_t k) {
    return rows >= 1 && rows <= 1u << 24 && k >= 1 && k <= 1u << 20 && (uint64_t)rows * k <= 1ull << 36;
}

static void check_matrices() {
    CHECK(iefwd_mx4_bytes(1, 1, nullptr) == IEFWD_EINVAL);
    for (uint32_t rows : kSizes)
        for (uint32_t k : kSizes) {
            size_t bytes = 7;
            const bool good = matrix(rows, k);
            CHECK(iefwd_mx4_bytes(rows, k, &bytes) == (good ? IEFWD_OK : IEFWD_EINVAL));
            if (good) {
                CHECK(bytes % 16 == 0 && bytes / 17 * 32 >= (size_t)rows * k && bytes < ((size_t)rows + 15) * (k + 511) * 5 / 8);
            } else {
                CHECK(bytes == 7);
                CHECK(iefwd_mx4_quantize(IEFWD_BF16, at(4096), 1ull << 40, at(4096), rows, k, nullptr) == IEFWD_EINVAL);
                CHECK(iefwd_mx4_values(at(4096), IEFWD_F32, at(4096), 1ull << 40, rows, k, nullptr) == IEFWD_EINVAL);
                CHECK(iefwd_mx4_pack(at(4096), at(4096), at(4096), rows, k, nullptr) == IEFWD_EINVAL);
                CHECK(iefwd_mx4_gemm(0, at(4096), at(4096), nullptr, nullptr, at(4096), rows, 16, k, nullptr) == IEFWD_EINVAL);
                CHECK(iefwd_mx4_gemm_bf16(0, at(4096), at(4096), nullptr, nullptr, at(4096), 1, rows, k, nullptr) == IEFWD_EINVAL);
            }
        }
    CHECK(iefwd_mx4_gemm(0, at(4096), at(4096), nullptr, nullptr, at(4096), 1u << 24, 1u << 24, 32, nullptr) == IEFWD_EINVAL);
    for (uint64_t stride : {0ull, 31ull, (1ull << 40) + 1, ~0ull})
        CHECK(iefwd_mx4_quantize(IEFWD_BF16, at(4096), stride, at(4096), 3, 32, nullptr) == IEFWD_EINVAL);
    for (uint32_t type : {2u, 0xffffffffu}) CHECK(iefwd_mx4_values(at(4096), type, at(4096), 32, 3, 32, nullptr) == IEFWD_EINVAL);
    for (uint32_t epi : {3u, 0xffffffffu}) CHECK(iefwd_mx4_gemm(epi, at(4096), at(4096), nullptr, at<float>(4096), at(4096), 3, 3, 32, nullptr) == IEFWD_EINVAL);
    CHECK(iefwd_mx4_gemm(2, at(4096), at(4096), nullptr, nullptr, at(4096), 3, 3, 32, nullptr) == IEFWD_EINVAL);
    CHECK(iefwd_mx4_gemm_bf16(0, at(4096), at(4096), nullptr, nullptr, at(4096), 17, 3, 32, nullptr) == IEFWD_EINVAL);
    CHECK(iefwd_mx4_gemm_bf16(0, at(4096), at(4096), nullptr, nullptr, at(4096), 1, 3, 36, nullptr) == IEFWD_EINVAL);
    CHECK(std::strlen(iefwd_last_error()) > 0);
}

static void check_cache() {
    auto c = std::make_unique<iefwd_paged_cache>();
    std::memset(c.get(), 0, sizeof *c);
    c->abi_version = IEFWD_ABI_VERSION;
    c->kv_type = IEFWD_KV_MX4;
    c->n_pages = 10;
    c->page_size = 16;
    c->n_kv_heads = 4;
    c->head_dim = 64;
    c->k = at(4096);
    c->v = at(8192);
    size_t before = 0;
    for (uint32_t pages = 1; pages <= 1u << 20; pages = pages * 3 / 2 + 1) {
        size_t bytes = 7;
        CHECK(iefwd_paged_attention_workspace(c.get(), 3, 16, pages, &bytes) == IEFWD_OK && bytes >= before);
        before = bytes;
        if (bytes)
            CHECK(iefwd_paged_attention_scored(c.get(), at(4096), 1024, 16, at<int32_t>(4096), pages, pages, at<int32_t>(4096), 3, 1.f, 5.f, nullptr,
                                               at(4096), at(4096), bytes - 1, nullptr) == IEFWD_EINVAL);
    }
    for (float cap : {-1.f, 0x1p-61f, 0x1p61f, INFINITY, NAN})
        CHECK(iefwd_paged_attention_scored(c.get(), at(4096), 1024, 16, at<int32_t>(4096), 8, 8, at<int32_t>(4096), 3, 1.f, cap, nullptr, at(4096),
                                           nullptr, 0, nullptr) == IEFWD_EINVAL);
    CHECK(iefwd_paged_read(c.get(), nullptr, at(4096), at(4096), 5, 256, 256, nullptr) == IEFWD_EINVAL);
    CHECK(iefwd_paged_read(c.get(), at<int64_t>(4096), at(4096), at(4096), 5, 255, 256, nullptr) == IEFWD_EINVAL);
    CHECK(iefwd_paged_read(c.get(), at<int64_t>(4096), at(4096), at(4098), 5, 256, 256, nullptr) == IEFWD_EINVAL);
    CHECK(iefwd_paged_read(c.get(), at<int64_t>(4096), at(4096), at(4096), 0xffffffffu, 256, 256, nullptr) == IEFWD_EINVAL);
    CHECK(iefwd_paged_append(c.get(), at(4096), at(4096), at<int64_t>(4096), 5, 256, 0, nullptr) == IEFWD_EINVAL);
    CHECK(iefwd_paged_read(c.get(), nullptr, nullptr, nullptr, 0, 0, 0, nullptr) == IEFWD_OK);
    c->head_dim = 96;
    CHECK(iefwd_paged_read(c.get(), at<int64_t>(4096), at(4096), at(4096), 5, 384, 384, nullptr) == IEFWD_EINVAL);
}

static void check_logprobs() {
    CHECK(iefwd_token_logprobs_workspace(1, 1, 0, nullptr) == IEFWD_EINVAL);
    for (uint32_t rows : kSizes)
        for (uint32_t vocab : kSizes)
            for (uint32_t n : {0u, 1u, 32u, 33u, 0xffffffffu}) {
                size_t bytes = 7;
                const bool good = rows >= 1 && rows <= 1u << 22 && vocab >= 1 && vocab <= 1u << 24 && (uint64_t)rows * vocab <= 1ull << 35 &&
                                  n <= 32 && n <= vocab;
                CHECK(iefwd_token_logprobs_workspace(rows, vocab, n, &bytes) == (good ? IEFWD_OK : IEFWD_EINVAL));
                // no more than 2048 parts and one more a row, whatever the sizes
                CHECK(good ? bytes <= (size_t)2 * 2048 * (12 + 8 * n) : bytes == 7);
                if (!good || bytes)
                    CHECK(iefwd_token_logprobs(IEFWD_BF16, at(4096), 1ull << 24, rows, vocab, at<int64_t>(4096), 1.f, at<float>(4096), nullptr, nullptr, n,
                                               at<int32_t>(4096), at<float>(4096), at(4096), bytes - 1, nullptr) == IEFWD_EINVAL);
            }
    for (float scale : {0.f, -1.f, 0x1p31f, 0x1p-31f, INFINITY, NAN}) {
        CHECK(iefwd_token_logprobs(IEFWD_BF16, at(4096), 100, 3, 100, at<int64_t>(4096), scale, at<float>(4096), nullptr, nullptr, 0, nullptr, nullptr,
                                   nullptr, 0, nullptr) == IEFWD_EINVAL);
        CHECK(iefwd_token_logprobs_grad(IEFWD_BF16, at(4096), 100, 3, 100, at<int64_t>(4096), scale, at<float>(4096), nullptr, at<float>(4096), nullptr,
                                        at(8192), 100, nullptr) == IEFWD_EINVAL);
    }
    CHECK(iefwd_token_logprobs_grad(IEFWD_BF16, at(4096), 100, 3, 100, at<int64_t>(4096), 1.f, at<float>(4096), nullptr, nullptr, nullptr, at(8192), 100,
                                    nullptr) == IEFWD_EINVAL);
    CHECK(iefwd_token_logprobs_grad(IEFWD_BF16, at(4096), 100, 3, 100, at<int64_t>(4096), 1.f, at<float>(4096), nullptr, at<float>(4096), at<float>(4096),
                                    at(8192), 100, nullptr) == IEFWD_EINVAL);
    CHECK(iefwd_token_logprobs_grad(IEFWD_BF16, at(4096), 100, 3, 100, at<int64_t>(4096), 1.f, at<float>(4096), nullptr, at<float>(4096), nullptr,
                                    at(4096), 101, nullptr) == IEFWD_EINVAL);
}

int main() {
    check_matrices();
    check_cache();
    check_logprobs();
    if (failures) return 1;
    std::puts("4-bit host sanitizer checks passed");
    return 0;
}
