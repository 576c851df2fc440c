// gfx950 kernels of attention over the paged key-value cache (include/lora_kv.h).
#include <algorithm>
#include <cmath>
#include <new>

#include "lora_device.h"
#include "lora_kv_internal.h"

using namespace lora;

struct lora_attn_s {
    int device = 0;
    int n_cu = 0;
};

namespace {

struct AttnArgs {
    const uint16_t *k, *v;                 // the layer's
    const uint16_t* q;
    uint16_t* out;
    const int32_t *tables, *lens, *seg_offset;
    int64_t page_stride, head_stride, row_stride, ldq, ldo;
    int32_t n_rows, n_seqs, ld_table, max_len, n_pages, page_shift;
    int32_t n_heads, group, head_dim;
    int32_t window, n_sinks;
    float scale;
};

// One wave per row and head: 4 elements of the head per lane, one token at a time.
template <class Fmt>
__global__ void __launch_bounds__(64) lora_attn_row_kernel(AttnArgs a) {
    const int l = threadIdx.x, row = blockIdx.x, h = blockIdx.y;
    int s = row, n = 1, i = 0;
    if (a.seg_offset) {
        int lo = 0, hi = a.n_seqs;
        while (lo < hi) {
            const int mid = (lo + hi) >> 1;
            if (a.seg_offset[mid + 1] > row) hi = mid;
            else lo = mid + 1;
        }
        s = lo;
        if (s >= a.n_seqs) return;
        const int first = a.seg_offset[s];
        n = min(a.seg_offset[s + 1], a.n_rows) - first;
        i = row - first;
        if (first < 0 || i < 0) return;
    }
    const int len = kv_len(a.lens, s, a.max_len);
    const int p = len - n + i;
    const int d = 4 * l;
    const bool in = d < a.head_dim;
    float q[4] = {0, 0, 0, 0}, o[4] = {0, 0, 0, 0}, m = -INFINITY, sum = 0.f;
    if (in)
        for (int e = 0; e < 4; ++e) q[e] = Fmt::to_f32(a.q[row * a.ldq + (int64_t)h * a.head_dim + d + e]);
    for (int j = 0; j <= p; ++j) {
        if (a.window && j <= p - a.window && j >= a.n_sinks) continue;
        const int page = a.tables[(int64_t)s * a.ld_table + (j >> a.page_shift)];
        if ((uint32_t)page >= (uint32_t)a.n_pages) continue;
        const int64_t at = page * a.page_stride + (h / a.group) * a.head_stride +
                           (j & ((1 << a.page_shift) - 1)) * a.row_stride + d;
        float x = 0.f;
        if (in)
            for (int e = 0; e < 4; ++e) x += q[e] * Fmt::to_f32(a.k[at + e]);
        for (int b = 1; b < 64; b <<= 1) x += __shfl_xor(x, b, 64);
        x *= a.scale;
        const float mn = fmaxf(m, x), f = m == -INFINITY ? 0.f : expf(m - mn), w = mn == -INFINITY ? 0.f : expf(x - mn);
        m = mn;
        sum = sum * f + w;
        if (in)
            for (int e = 0; e < 4; ++e) o[e] = o[e] * f + w * Fmt::to_f32(a.v[at + e]);
    }
    if (!in) return;
    const float r = sum != 0.f ? 1.f / sum : 0.f;
    for (int e = 0; e < 4; e += 2)
        *(uint32_t*)(a.out + row * a.ldo + (int64_t)h * a.head_dim + d + e) = Fmt::pack2(o[e] * r, o[e + 1] * r);
}

// ---------------------------------------------------------------------------
// host side
// ---------------------------------------------------------------------------

int check_attn(const lora_attn_s* h, const lora_kv_cache_t* c, int32_t layer, const lora_kv_seqs_t* s, int32_t n_rows,
               int32_t n_heads, const void* q, int64_t ldq, const void* out, int64_t ldo, float scale, int32_t window,
               int32_t n_sinks) {
    if (!h) return set_error(LORA_E_ARG, "attention handle is NULL");
    if (int rc = check_kv_cache(c)) return rc;
    if (int rc = check_kv_layer(c, layer)) return rc;
    if (int rc = check_kv_seqs(c, s)) return rc;
    if (n_rows < 0) return set_error(LORA_E_ARG, "negative n_rows");
    if (n_heads < 1 || n_heads % c->n_kv_heads)
        return set_error(LORA_E_SHAPE, "n_heads must be a positive multiple of n_kv_heads");
    const int64_t width = (int64_t)n_heads * c->head_dim;
    if (width > (1 << 24)) return set_error(LORA_E_SHAPE, "n_heads * head_dim exceeds 2^24");
    if (int rc = check_kv_rows("q", q, "ldq", ldq, width, n_rows)) return rc;
    if (int rc = check_kv_rows("out", out, "ldo", ldo, width, n_rows)) return rc;
    if (!(scale > 0.f) || !std::isfinite(scale)) return set_error(LORA_E_ARG, "scale must be positive and finite");
    if (window < 0 || n_sinks < 0) return set_error(LORA_E_ARG, "negative window or n_sinks");
    if (n_rows > 0) {
        const uintptr_t qs = (uintptr_t)q, os = (uintptr_t)out;
        const uintptr_t qe = qs + ((uintptr_t)(n_rows - 1) * ldq + width) * 2;
        const uintptr_t oe = os + ((uintptr_t)(n_rows - 1) * ldo + width) * 2;
        if (qs < oe && os < qe) return set_error(LORA_E_OVERLAP, "q and out overlap");
    }
    return LORA_OK;
}

AttnArgs attn_args(const lora_kv_cache_t* c, int32_t layer, const lora_kv_seqs_t* s, const int32_t* seg_offset,
                   int32_t n_rows, int32_t n_heads, const void* q, int64_t ldq, void* out, int64_t ldo, float scale,
                   int32_t window, int32_t n_sinks) {
    AttnArgs a;
    a.k = (const uint16_t*)c->k + layer * c->layer_stride;
    a.v = (const uint16_t*)c->v + layer * c->layer_stride;
    a.q = (const uint16_t*)q;
    a.out = (uint16_t*)out;
    a.tables = s->tables;
    a.lens = s->lens;
    a.seg_offset = seg_offset;
    a.page_stride = c->page_stride;
    a.head_stride = c->head_stride;
    a.row_stride = c->row_stride;
    a.ldq = ldq;
    a.ldo = ldo;
    a.n_rows = n_rows;
    a.n_seqs = s->n_seqs;
    a.ld_table = s->ld_table;
    a.max_len = s->max_len;
    a.n_pages = c->n_pages;
    a.page_shift = 0;
    while ((1 << a.page_shift) < c->page_rows) ++a.page_shift;
    a.n_heads = n_heads;
    a.group = n_heads / c->n_kv_heads;
    a.head_dim = c->head_dim;
    a.window = window;
    a.n_sinks = n_sinks;
    a.scale = scale;
    return a;
}

struct HandleDevice {
    int prev = -1;
    bool ok = false;
    explicit HandleDevice(int device) {
        if (hipGetDevice(&prev) != hipSuccess) return;
        ok = prev == device || hipSetDevice(device) == hipSuccess;
    }
    ~HandleDevice() {
        if (prev >= 0) (void)hipSetDevice(prev);
    }
};

}  // namespace

extern "C" {

int lora_attn_create(lora_attn_t* out, int device, void* stream) {
    if (!out) return set_error(LORA_E_ARG, "out is NULL");
    *out = nullptr;
    if (device < 0) return set_error(LORA_E_ARG, "negative device");
    HandleDevice g(device);
    if (!g.ok) return set_error(LORA_E_HIP, "lora_attn_create: cannot select the device");
    hipStreamCaptureStatus cs = hipStreamCaptureStatusNone;
    if (hipStreamIsCapturing((hipStream_t)stream, &cs) != hipSuccess)
        return set_error(LORA_E_HIP, "lora_attn_create: the stream's capture status");
    if (cs != hipStreamCaptureStatusNone) return set_error(LORA_E_CAPTURE, "lora_attn_create cannot be recorded in a graph");
    auto* h = new (std::nothrow) lora_attn_s();
    if (!h) return set_error(LORA_E_NOMEM, "handle allocation failed");
    h->device = device;
    *out = h;
    return LORA_OK;
}

int lora_attn_destroy(lora_attn_t a) {
    if (!a) return set_error(LORA_E_ARG, "attention handle is NULL");
    delete a;
    return LORA_OK;
}

int lora_attn_decode(lora_attn_t h, const lora_kv_cache_t* c, int32_t layer, const lora_kv_seqs_t* s, int32_t n_heads,
                     const void* q, int64_t ldq, void* out, int64_t ldo, float scale, int32_t window, int32_t n_sinks,
                     void* stream) {
    if (int rc = check_attn(h, c, layer, s, s ? s->n_seqs : 0, n_heads, q, ldq, out, ldo, scale, window, n_sinks)) return rc;
    if (s->n_seqs == 0) return LORA_OK;
    HandleDevice g(h->device);
    if (!g.ok) return set_error(LORA_E_HIP, "lora_attn_decode: cannot select the device");
    const AttnArgs a = attn_args(c, layer, s, nullptr, s->n_seqs, n_heads, q, ldq, out, ldo, scale, window, n_sinks);
    if (c->dtype == LORA_F16)
        hipLaunchKernelGGL(lora_attn_row_kernel<FmtF16>, dim3(a.n_rows, n_heads), dim3(64), 0, (hipStream_t)stream, a);
    else
        hipLaunchKernelGGL(lora_attn_row_kernel<FmtBF16>, dim3(a.n_rows, n_heads), dim3(64), 0, (hipStream_t)stream, a);
    return check_launch("lora_attn_decode");
}

int lora_attn_prompt(lora_attn_t h, const lora_kv_cache_t* c, int32_t layer, const lora_kv_seqs_t* s,
                     const int32_t* seg_offset, int32_t n_rows, int32_t n_heads, const void* q, int64_t ldq, void* out,
                     int64_t ldo, float scale, int32_t window, int32_t n_sinks, void* stream) {
    if (int rc = check_attn(h, c, layer, s, n_rows, n_heads, q, ldq, out, ldo, scale, window, n_sinks)) return rc;
    if (!seg_offset) return set_error(LORA_E_ARG, "seg_offset is NULL");
    if ((uintptr_t)seg_offset & 3) return set_error(LORA_E_ALIGN, "seg_offset not 4-byte aligned");
    if (n_rows == 0 || s->n_seqs == 0) return LORA_OK;
    HandleDevice g(h->device);
    if (!g.ok) return set_error(LORA_E_HIP, "lora_attn_prompt: cannot select the device");
    const AttnArgs a = attn_args(c, layer, s, seg_offset, n_rows, n_heads, q, ldq, out, ldo, scale, window, n_sinks);
    if (c->dtype == LORA_F16)
        hipLaunchKernelGGL(lora_attn_row_kernel<FmtF16>, dim3(n_rows, n_heads), dim3(64), 0, (hipStream_t)stream, a);
    else
        hipLaunchKernelGGL(lora_attn_row_kernel<FmtBF16>, dim3(n_rows, n_heads), dim3(64), 0, (hipStream_t)stream, a);
    return check_launch("lora_attn_prompt");
}

}  // extern "C"
