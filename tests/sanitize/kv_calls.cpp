// The host side of the key-value cache and attention calls against a stand-in HIP
// runtime: launches are recorded and not run, device pointers are never touched.
// Built with AddressSanitizer and UndefinedBehaviorSanitizer on the host code; no GPU.
#include <cstdio>
#include <cstdlib>
#include <cstring>
#include <random>
#include <vector>

#include <hip/hip_runtime.h>

#include "lora.h"
#include "lora_internal.h"
#include "lora_kv.h"

namespace lora {
hipError_t launch_shrink(const KernelArgs&, const uint32_t*, int, hipStream_t) { return hipSuccess; }
hipError_t launch_expand(const KernelArgs&, const uint32_t*, int, hipStream_t) { return hipSuccess; }
hipError_t launch_reduce(const KernelArgs&, const uint32_t*, hipStream_t) { return hipSuccess; }
hipError_t launch_step(const KernelArgs&, const uint32_t*, int, hipStream_t) { return hipSuccess; }
hipError_t launch_fill(uint32_t*, uint32_t, uint64_t, hipStream_t) { return hipSuccess; }
hipError_t launch_base(const BaseArgs&, int, hipStream_t) { return hipSuccess; }
}  // namespace lora

namespace {
int g_launches, g_fail_at, g_allocs;
uint64_t g_threads;                        // of the launches
hipError_t g_error = hipSuccess;
bool g_no_memory, g_capturing;
dim3 g_grid, g_block;
int failures = 0;
#define CHECK(cond, ...)                                   \
    do {                                                   \
        if (!(cond)) {                                     \
            std::fprintf(stderr, "FAIL %s:%d: ", __FILE__, __LINE__); \
            std::fprintf(stderr, __VA_ARGS__);             \
            std::fprintf(stderr, "\n");                    \
            ++failures;                                    \
        }                                                  \
    } while (0)
}  // namespace

// The runtime calls of the library's host code (defined here, they take the
// place of the HIP library's).
extern "C" {
hipError_t hipGetDevice(int* d) { *d = 0; return hipSuccess; }
hipError_t hipSetDevice(int d) { return d == 0 ? hipSuccess : hipErrorInvalidDevice; }
hipError_t hipDeviceGetAttribute(int* v, hipDeviceAttribute_t, int) { *v = 256; return hipSuccess; }
hipError_t hipMalloc(void** p, size_t) {
    if (g_no_memory && g_allocs == 1) return hipErrorOutOfMemory;
    ++g_allocs;
    return (*p = std::malloc(256)) ? hipSuccess : hipErrorOutOfMemory;
}
hipError_t hipFree(void* p) {
    if (p) --g_allocs;
    std::free(p);
    return hipSuccess;
}
hipError_t hipStreamSynchronize(hipStream_t) { return hipSuccess; }
hipError_t hipStreamIsCapturing(hipStream_t, hipStreamCaptureStatus* c) {
    *c = g_capturing ? hipStreamCaptureStatusActive : hipStreamCaptureStatusNone;
    return hipSuccess;
}
hipError_t hipGetLastError() {
    const hipError_t e = g_error;
    g_error = hipSuccess;
    return e;
}
hipError_t __hipPushCallConfiguration(dim3 grid, dim3 block, size_t, hipStream_t) {
    g_grid = grid;
    g_block = block;
    return hipSuccess;
}
hipError_t __hipPopCallConfiguration(dim3* grid, dim3* block, size_t* lds, hipStream_t* s) {
    *grid = g_grid;
    *block = g_block;
    *lds = 0;
    *s = nullptr;
    return hipSuccess;
}
hipError_t hipLaunchKernel(const void*, dim3 grid, dim3 block, void**, size_t, hipStream_t) {
    ++g_launches;
    CHECK(grid.x > 0 && grid.y > 0 && grid.z == 1 && grid.y <= 65535, "grid %u %u %u", grid.x, grid.y, grid.z);
    CHECK((uint64_t)grid.x * block.x < (1ull << 32), "grid of %u x %u threads", grid.x, block.x);
    g_threads += (uint64_t)grid.x * grid.y * block.x;
    if (g_fail_at > 0 && --g_fail_at == 0) g_error = hipErrorInvalidConfiguration;
    return hipSuccess;
}
}

namespace {

void* const P = (void*)(uintptr_t)(1 << 20);

lora_kv_cache_t cache(int layers, int pages, int kv_heads, int page_rows, int dim) {
    const int64_t head = (int64_t)page_rows * dim, page = head * kv_heads;
    return {P, (char*)P + (1ll << 40), page * pages, page, head, dim, LORA_BF16, layers, pages, kv_heads, page_rows, dim};
}

// Id lists of every length around what one launch carries: nothing is read past
// their ends, and the launches are as many as the ids need.
void check_id_lists() {
    const lora_kv_cache_t c = cache(2, 4000, 2, 16, 64);
    const lora_kv_book_t b{(int32_t*)P, (int32_t*)P, (int32_t*)P, 3000, 8, 4000, 16};
    size_t bytes = 0;
    CHECK(lora_kv_workspace_bytes(&b, &bytes) == LORA_OK && bytes >= 4 * (3u * 4000 + 3000 + 2), "%zu bytes", bytes);
    for (int n : {0, 1, 239, 240, 241, 479, 480, 481, 961, 1500}) {
        std::vector<int32_t> from(n), to(n);
        for (int i = 0; i < n; ++i) from[i] = i % 700, to[i] = 1400 + i;
        g_launches = 0;
        CHECK(lora_kv_copy(&c, n, from.data(), to.data(), nullptr) == LORA_OK, "%s", lora_last_error());
        CHECK(g_launches == (n + 239) / 240, "copy of %d: %d launches", n, g_launches);
        g_launches = 0;
        CHECK(lora_kv_fork(&c, &b, n, from.data(), to.data(), nullptr, P, bytes, nullptr) == LORA_OK, "%s", lora_last_error());
        CHECK(g_launches == (n ? 3 * ((n + 239) / 240) : 1), "fork of %d: %d launches", n, g_launches);
        g_launches = 0;
        CHECK(lora_kv_free(&b, n, to.data(), nullptr) == LORA_OK, "%s", lora_last_error());
        CHECK(g_launches == (n + 479) / 480, "free of %d: %d launches", n, g_launches);
        if (n < 2) continue;
        to[n - 1] = to[0];
        g_launches = 0;
        CHECK(lora_kv_copy(&c, n, from.data(), to.data(), nullptr) == LORA_E_ARG, "a page twice");
        CHECK(lora_kv_free(&b, n, to.data(), nullptr) == LORA_E_ARG, "a sequence twice");
        to[n - 1] = from[0];
        CHECK(lora_kv_fork(&c, &b, n, from.data(), to.data(), nullptr, P, bytes, nullptr) == LORA_E_ARG, "a child that is a parent");
        to[n - 1] = 4000;
        CHECK(lora_kv_copy(&c, n, from.data(), to.data(), nullptr) == LORA_E_INDEX, "a page past the last");
        CHECK(g_launches == 0, "%d launches of refused calls", g_launches);
    }
    g_fail_at = 2;
    std::vector<int32_t> from(500), to(500);
    for (int i = 0; i < 500; ++i) from[i] = i, to[i] = 600 + i;
    CHECK(lora_kv_copy(&c, 500, from.data(), to.data(), nullptr) == LORA_E_HIP, "a launch that fails");
}

// Sizes of every order: a call is refused or launches a grid within the limits.
void check_sizes(lora_attn_t h) {
    std::mt19937_64 rng(7);
    auto size = [&](int64_t most) {
        const double f = std::uniform_real_distribution<double>(0, 1)(rng);
        return (int64_t)std::min((double)most, std::exp2(f * std::log2((double)most + 1)));
    };
    int64_t ran = 0, refused = 0;
    for (int i = 0; i < 200000; ++i) {
        const int page_rows = 16 << (size(13) - 1), kv_heads = (int)size(1 << 12), dim = 8 * (int)size(32);
        const lora_kv_cache_t c = cache((int)size(100), (int)size(1 << 20), kv_heads, page_rows, dim);
        const int n_seqs = (int)size(0x7fffffff), ld = (int)size(0x7fffffff);
        const int max_len = (int)size(0x7fffffff), group = (int)size(1 << 10);
        const lora_kv_seqs_t s{(int32_t*)P, (int32_t*)P, n_seqs, ld, max_len};
        const int64_t w = (int64_t)kv_heads * dim, qw = w * group;
        const int n_rows = (int)size(0x7fffffff);
        const int window = i & 1 ? (int)size(0x7fffffff) : 0, sinks = (int)size(0x7fffffff) - 1;
        void* const out = (void*)((uintptr_t)1 << 62);
        for (int call = 0; call < 6; ++call) {
            g_launches = 0;
            int rc = 0;
            const int heads = (int)std::min<int64_t>((int64_t)group * kv_heads, 0x7fffffff / kv_heads * kv_heads);
            if (call == 0) rc = lora_attn_decode(h, &c, 0, &s, heads, P, qw, out, qw, 0.1f, window, sinks, nullptr);
            if (call == 1) rc = lora_attn_prompt(h, &c, 0, &s, (int32_t*)P, n_rows, heads, P, qw, out, qw, 0.1f, window, sinks, nullptr);
            if (call == 2) rc = lora_kv_append(&c, 0, &s, (int32_t*)P, n_rows, P, w, P, w, nullptr);
            const lora_kv_book_t b{(int32_t*)P, (int32_t*)P, (int32_t*)P, n_seqs, ld, c.n_pages, page_rows};
            size_t bytes = 0;
            const bool book = lora_kv_workspace_bytes(&b, &bytes) == LORA_OK;
            if (call == 3) rc = lora_kv_grow(&b, (int32_t*)P, nullptr, P, bytes, nullptr);
            if (call == 4) rc = lora_kv_compact(&c, &b, (int32_t*)P, (int32_t*)P, nullptr, P, bytes, nullptr);
            if (call == 5 && n_seqs < (1 << 24)) rc = lora_kv_trim(&b, 1 + size(1 << 30), 0, nullptr);
            CHECK(book || call < 3 || call == 5 || rc != LORA_OK, "call %d without a workspace", call);
            CHECK((rc == LORA_OK) == (g_launches > 0) || (call == 5 && n_seqs >= (1 << 24)), "call %d: %d, %d launches", call, rc,
                  g_launches);
            ++(rc == LORA_OK ? ran : refused);
        }
    }
    std::printf("%lld calls launched, %lld refused\n", (long long)ran, (long long)refused);
    CHECK(ran > 1000 && refused > 1000, "one-sided sizes");
}

void check_handles() {
    lora_attn_t h = nullptr;
    g_no_memory = true;
    CHECK(lora_attn_create(&h, 0, nullptr) == LORA_E_NOMEM && !h && g_allocs == 0, "%d allocations left", g_allocs);
    g_no_memory = false;
    g_capturing = true;
    CHECK(lora_attn_create(&h, 0, nullptr) == LORA_E_CAPTURE && !h && g_allocs == 0, "on a capturing stream");
    g_capturing = false;
    g_fail_at = 1;
    CHECK(lora_attn_create(&h, 0, nullptr) == LORA_E_HIP && !h && g_allocs == 0, "with a launch that fails");
    CHECK(lora_attn_create(&h, 0, nullptr) == LORA_OK && h, "%s", lora_last_error());
    check_sizes(h);
    CHECK(lora_attn_destroy(h) == LORA_OK && g_allocs == 0, "%d allocations left", g_allocs);
    CHECK(lora_attn_destroy(nullptr) == LORA_E_ARG, "no handle");
}

}  // namespace

int main() {
    check_id_lists();
    check_handles();
    if (failures) return 1;
    std::puts("all checks passed");
    return 0;
}
