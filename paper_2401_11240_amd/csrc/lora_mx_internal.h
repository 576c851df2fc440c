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

// A matrix's bytes: its rows, a leading dimension apart.
struct Span {
    uintptr_t lo = 0, hi = 0;              // from the first to behind the last
    uintptr_t ld = 0, row = 0;             // ld 0: one row
    Span() = default;
    Span(const void* p, int64_t rows, int64_t ld_bytes, int64_t row_bytes) {
        if (!p || rows <= 0) return;
        lo = (uintptr_t)p;
        hi = lo + (uintptr_t)(rows - 1) * (uintptr_t)ld_bytes + (uintptr_t)row_bytes;
        ld = rows > 1 ? (uintptr_t)ld_bytes : 0;
        row = (uintptr_t)row_bytes;
    }
    // Whether two have a byte in common, exactly where their rows are equally far apart (columns of one buffer) or one
    // of them is a single row; otherwise from first to last.
    bool meets(const Span& o) const {
        if (!(lo < o.hi && o.lo < hi)) return false;
        const uintptr_t step = ld ? ld : o.ld;
        if (!step || (ld && o.ld && ld != o.ld)) return true;
        const uintptr_t at = o.lo >= lo ? (o.lo - lo) % step : (step - (lo - o.lo) % step) % step;   // of o's rows in this one's
        return at < row || o.row > step - at;
    }
};
inline Span codes_span(const lora_mx_t* q) { return Span(q->codes, q->n_rows, q->ld_codes, mx_row_bytes(q->h, q->format)); }
inline Span scales_span(const lora_mx_t* q) { return Span(q->scales, q->n_rows, q->ld_scales, mx_blocks(q->h)); }

}  // namespace lora
