// Shared by the sources behind include/lora_kv.h: argument checks and launch
// helpers of the host side, and the device code's view of tables and lengths.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include <string>

#include "lora.h"
#include "lora_internal.h"
#include "lora_kv.h"
#include "lora_stream.h"

namespace lora {

int set_error(int code, const std::string& msg);

// Argument checks: LORA_OK, or the code set with its message.
int check_kv_cache(const lora_kv_cache_t* c);
int check_kv_layer(const lora_kv_cache_t* c, int32_t layer);
int check_kv_seqs(const lora_kv_cache_t* c, const lora_kv_seqs_t* s);
// a [n_rows, ld] operand of h elements per row
int check_kv_rows(const char* name, const void* p, const char* ld_name, int64_t ld, int64_t h, int32_t n_rows);
int check_launch(const char* what);

inline bool is_aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }

// A length as the kernels use it.
__device__ __forceinline__ int kv_len(const int32_t* lens, int s, int max_len) {
    const int v = lens[s];
    return v < 0 ? 0 : v < max_len ? v : max_len;
}

}  // namespace lora
