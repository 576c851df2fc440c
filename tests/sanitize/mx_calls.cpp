// The host side of the calls on rows in blocks, of the norm and of the choice of tokens against a
// stand-in HIP runtime: launches are recorded and not run, device pointers are never touched.
// Built with AddressSanitizer and UndefinedBehaviorSanitizer on the host code; no GPU.
#include <cmath>
#include <cstdio>
#include <cstdlib>
#include <random>

#include <hip/hip_runtime.h>

#include "lora.h"
#include "lora_internal.h"
#include "lora_mx.h"
#include "lora_sample.h"

namespace lora {
hipError_t launch_shrink(const KernelArgs&, const uint32_t*, int, hipStream_t) { return hipSuccess; }
hipError_t launch_expand(const KernelArgs&, const uint32_t*, int, hipStream_t) { return hipSuccess; }
hipError_t launch_reduce(const KernelArgs&, const uint32_t*, hipStream_t) { return hipSuccess; }
hipError_t launch_step(const KernelArgs&, const uint32_t*, int, hipStream_t) { return hipSuccess; }
hipError_t launch_fill(uint32_t*, uint32_t, uint64_t, hipStream_t) { return hipSuccess; }
hipError_t launch_base(const BaseArgs&, int, hipStream_t) { return hipSuccess; }
}  // namespace lora

namespace {
int g_launches, g_fail_at;
uint64_t g_threads;                        // of the launches
hipError_t g_error = hipSuccess;
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
    CHECK((uint64_t)grid.x * block.x < (1ull << 32) && block.x <= 1024, "grid of %u x %u threads", grid.x, block.x);
    g_threads += (uint64_t)grid.x * grid.y * block.x;
    if (g_fail_at > 0 && --g_fail_at == 0) g_error = hipErrorInvalidConfiguration;
    return hipSuccess;
}
}

namespace {

// Matrices of 2^54 bytes and less, 2^55 apart.
void* at(int i) { return (void*)((uintptr_t)(i + 1) << 55); }

// Sizes of every order: a call is refused or launches grids within the limits, whose threads
// are as many as its elements and rows need.
void check_sizes() {
    std::mt19937_64 rng(7);
    auto size = [&](int64_t most) {
        const double f = std::uniform_real_distribution<double>(0, 1)(rng);
        return (int64_t)std::min((double)most, std::exp2(f * std::log2((double)most + 1)));
    };
    int64_t ran = 0, refused = 0;
    for (int i = 0; i < 20000; ++i) {
        // (2^42 elements and less: what a card's memory can hold, and some more)
        const int h = (int)std::min<int64_t>(8 * size(1 << 28), 0x7ffffff8);
        const int n = (int)size(std::min<int64_t>(0x7fffffff, (1ll << 42) / h));
        const int h_out = (int)std::min<int64_t>({8 * size(1 << 28), 0x7ffffff8, std::max<int64_t>(8, (1ll << 42) / n / 8 * 8)});
        const int fmt = i & 1, type = i % 3;
        const int64_t blocks = (h + 31) / 32, most = std::min<int64_t>(1ll << 40, (1ll << 52) / n);
        auto ld = [&](int64_t least, int64_t of) { return std::max((least + of - 1) / of * of, size(most) / of * of); };
        const int64_t row = blocks * (fmt == LORA_E4M3 ? 32 : 16);
        const lora_mx_t x{at(0), at(1), ld(row, 16), ld(blocks, 4), n, h, fmt};
        const lora_mx_t w{at(2), at(3), (blocks * 16 + 15) / 16 * 16, (blocks + 3) / 4 * 4, h_out, h, LORA_E2M1};
        for (int call = 0; call < 5; ++call) {
            g_launches = 0;
            g_threads = 0;
            int rc = 0;
            uint64_t need = 0;
            size_t bytes = 0;
            if (call == 0) {
                rc = lora_mx_quantize(at(4), ld(h, 8), type, &x, nullptr);
                need = (uint64_t)n * blocks * 4;
            }
            if (call == 1) {
                rc = lora_mx_dequantize(&x, at(4), ld(h, 8), type, nullptr);
                need = (uint64_t)n * h / 8;
            }
            if (call == 2) {
                const int narrow = std::min(h, 8 * (int)size(1 << 13));
                lora_mx_t q = x;
                q.h = narrow;
                q.ld_codes = std::max<int64_t>(q.ld_codes, 2 * 65536);
                q.ld_scales = std::max<int64_t>(q.ld_scales, 4096);
                rc = lora_norm(at(4), ld(narrow, 8), i & 4 ? at(5) : nullptr, ld(narrow, 8), nullptr, 1e-5f, n, narrow, fmt,
                               i & 8 ? at(6) : nullptr, ld(narrow, 8), at(7), ld(narrow, 8), i & 16 ? &q : nullptr, nullptr);
                CHECK(rc == LORA_OK, "%s", lora_last_error());
                need = (uint64_t)n * 64;
            }
            if (call == 3) {
                rc = lora_mx_workspace_bytes(&x, &w, &bytes);
                                if (rc == LORA_OK) rc = lora_mx_apply(&x, &w, at(4), ld(h_out, 8), type, at(5), bytes, nullptr);
                if (rc == LORA_OK && bytes > 16) CHECK(g_launches == 2, "%d launches of split K", g_launches);
                need = (uint64_t)n * h_out / 1024;
            }
            if (call == 4) {
                const int v = (int)size(1 << 19);
                rc = lora_sample_workspace_bytes(n, v, type, &bytes);
                CHECK(rc == LORA_OK && bytes < 1ull << 32, "%zu bytes", bytes);
                rc = lora_sample(at(4), ld(v, 1), type, n, v, nullptr, (float*)at(5), (int32_t*)at(6), (float*)at(7), at(8), bytes, nullptr);
                CHECK(rc == LORA_OK, "%s", lora_last_error());
                need = (uint64_t)n * 1024;
            }
            CHECK((rc == LORA_OK) == (g_launches > 0), "call %d: %d, %d launches", call, rc, g_launches);
            CHECK(rc != LORA_OK || g_threads >= need, "call %d, %d rows of %d: %llu threads", call, n, h, (unsigned long long)g_threads);
            ++(rc == LORA_OK ? ran : refused);
        }
    }
    std::printf("%lld calls launched, %lld refused\n", (long long)ran, (long long)refused);
    CHECK(ran > 1000 && refused > 1000, "one-sided sizes");
}

// A launch that fails is the call's error, whichever of its launches it is; nothing is launched after it.
void check_failures() {
    const lora_mx_t x{at(0), at(1), 8192, 256, 40, 8192, LORA_E4M3}, w{at(2), at(3), 4096, 256, 1024, 8192, LORA_E2M1};
    size_t bytes = 0;
    CHECK(lora_mx_workspace_bytes(&x, &w, &bytes) == LORA_OK && bytes > 16, "%zu bytes", bytes);
    for (int k = 1; k <= 2; ++k) {
        g_fail_at = k;
        g_launches = 0;
        CHECK(lora_mx_apply(&x, &w, at(4), 1024, LORA_F16, at(5), bytes, nullptr) == LORA_E_HIP && g_launches == k, "launch %d", k);
    }
    const lora_mx_t big{at(0), at(1), 128, 4, 0x7fffffff, 128, LORA_E4M3};
    for (int k = 1; k <= 3; ++k) {
        g_fail_at = k;
        g_launches = 0;
        CHECK(lora_mx_quantize(at(4), 128, LORA_F16, &big, nullptr) == LORA_E_HIP && g_launches == k, "launch %d", k);
        g_fail_at = k;
        g_launches = 0;
        CHECK(lora_norm(at(4), 128, nullptr, 0, nullptr, 1e-5f, 0x7fffffff, 128, LORA_F16, nullptr, 0, at(5), 128, nullptr, nullptr) ==
                  LORA_E_HIP && g_launches == k, "launch %d", k);
    }
    for (int k = 1; k <= 4; ++k) {
        CHECK(lora_sample_workspace_bytes(3, 128000, LORA_BF16, &bytes) == LORA_OK, "%s", lora_last_error());
        g_fail_at = k;
        CHECK(lora_sample(at(4), 128000, LORA_BF16, 3, 128000, nullptr, (float*)at(5), (int32_t*)at(6), nullptr, at(8), bytes, nullptr) ==
                  LORA_E_HIP, "launch %d", k);
    }
}

}  // namespace

int main() {
    check_sizes();
    check_failures();
    if (failures) return 1;
    std::puts("all checks passed");
    return 0;
}
