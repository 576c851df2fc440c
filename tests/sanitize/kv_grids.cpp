// Books of very many sequences against the stand-in runtime of kv_calls.cpp, which checks every
// launch's grid: each call is refused or stays within what a grid may have.
#define main kv_calls_main
#include "kv_calls.cpp"
#undef main

int main() {
    for (int n_seqs : {1, (1 << 20) - 1, 1 << 20, (1 << 20) + 1, (1 << 24) - 1, 1 << 24, (1 << 24) + 1, 1 << 30, 0x7fffffff})
        for (int ld : {0, 1}) {
            const lora_kv_book_t b{(int32_t*)P, (int32_t*)P, (int32_t*)P, n_seqs, ld, 100, 16};
            size_t bytes = 0;
            CHECK(lora_kv_workspace_bytes(&b, &bytes) == LORA_OK, "%s", lora_last_error());
            const int32_t id = n_seqs - 1;
            int32_t* const step = (int32_t*)((uintptr_t)1 << 62);
            for (int call = 0; call < 4; ++call) {
                g_launches = 0;
                g_threads = 0;
                int rc = LORA_OK;
                if (call == 0) rc = lora_kv_trim(&b, 5, 2, nullptr);
                if (call == 1) rc = lora_kv_free(&b, 1, &id, nullptr);
                if (call == 2) rc = lora_kv_grow(&b, (int32_t*)P, nullptr, P, bytes, nullptr);
                if (call == 3) rc = lora_kv_grow_step(&b, (int32_t*)P, 16 * ld, step, nullptr, P, bytes, nullptr);
                CHECK(rc == LORA_OK && g_launches == 1, "call %d, %d sequences: %d, %d launches (%s)", call, n_seqs, rc, g_launches,
                      lora_last_error());
            }
        }
    if (failures) return 1;
    std::puts("all checks passed");
    return 0;
}
