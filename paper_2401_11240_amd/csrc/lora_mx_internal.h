// Shared by the sources behind include/lora_mx.h and lora_sample.h: argument checks
// of the host side.
#pragma once
#include <stdint.h>

#include "lora_kv_internal.h"
#include "lora_mx.h"

namespace lora {

// Bytes of a row's codes, and its blocks.
inline int64_t mx_blocks(int64_t h) { return (h + 31) / 32; }
inline int64_t mx_row_bytes(int64_t h, int32_t format) { return mx_blocks(h) * (format == LORA_E4M3 ? 32 : 16); }

// Argument checks: LORA_OK, or the code set with its message.
int check_mx(const char* name, const lora_mx_t* q);

// The bytes from a matrix's first to behind its last.
struct Span {
    uintptr_t lo = 0, hi = 0;
    Span() = default;
    Span(const void* p, int64_t rows, int64_t ld_bytes, int64_t row_bytes) {
        if (!p || rows <= 0) return;
        lo = (uintptr_t)p;
        hi = lo + (uintptr_t)(rows - 1) * (uintptr_t)ld_bytes + (uintptr_t)row_bytes;
    }
    bool meets(const Span& o) const { return lo < o.hi && o.lo < hi; }
};
inline Span codes_span(const lora_mx_t* q) { return Span(q->codes, q->n_rows, q->ld_codes, mx_row_bytes(q->h, q->format)); }
inline Span scales_span(const lora_mx_t* q) { return Span(q->scales, q->n_rows, q->ld_scales, mx_blocks(q->h)); }

}  // namespace lora
