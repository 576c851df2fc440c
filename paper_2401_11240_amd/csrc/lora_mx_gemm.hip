// gfx950 kernel of the product of rows in blocks (include/lora_mx.h): y = x W^T with
// x in E4M3 or E2M1 and W in E2M1 blocks, on v_mfma_scale_f32_16x16x128_f8f6f4, which takes
// codes and scale bytes as they are stored.
//
// The instruction, as measured (A here the weight, B the rows x): lane l holds row l % 16 of
// its operand; of 4-bit codes K 32 g .. + 31 (g = l / 16: one block, 16 bytes), of 8-bit codes
// K 16 g .. + 15 and 64 + 16 g .. + 15; its scale byte is that of block g of row l % 16;
// accumulator i is D[4 g + i][l % 16].
#include <stddef.h>

#include "lora_device.h"
#include "lora_mx_internal.h"

namespace lora {
namespace {

typedef int i32x8 __attribute__((ext_vector_type(8)));

struct GemmArgs {
    const unsigned char *x, *xs, *w, *ws;
    void* y;
    int64_t ldx, ldxs, ldw, ldws, ldy;     // bytes; ldy elements
    int n_rows, h_out, blocks;
    int dtype;
};

__device__ __forceinline__ void store4(const GemmArgs& a, int row, int n, const f32x4& v) {
    if (row >= a.n_rows || n >= a.h_out) return;
    const int64_t at = row * a.ldy + n;
    if (a.dtype == LORA_F32) *(f32x4*)((float*)a.y + at) = v;
    else if (a.dtype == LORA_F16) *(u32x2*)((uint16_t*)a.y + at) = u32x2{FmtF16::pack2(v[0], v[1]), FmtF16::pack2(v[2], v[3])};
    else *(u32x2*)((uint16_t*)a.y + at) = u32x2{FmtBF16::pack2(v[0], v[1]), FmtBF16::pack2(v[2], v[3])};
}

// One wave, 16 rows of x by 16 of W.
template <int XF>
__global__ void __launch_bounds__(64) lora_mx_tile_kernel(GemmArgs a) {
    const int l = threadIdx.x, r = l & 15, g = l >> 4;
    const int n = blockIdx.x * 16 + r, t = blockIdx.y * 16 + r;
    const bool nw = n < a.h_out, tx = t < a.n_rows;
    f32x4 acc = {0.f, 0.f, 0.f, 0.f};
    for (int k = 0; k < a.blocks; k += 4) {
        const u32x4 zero = {0, 0, 0, 0};
        const bool wb = nw && k + g < a.blocks, xb = tx && k + g < a.blocks;
        u32x4 w = zero, x0 = zero, x1 = zero;
        uint32_t sw = 0, sx = 0;
        if (wb) {
            w = *(const u32x4*)(a.w + n * a.ldw + 16 * (int64_t)(k + g));
            sw = a.ws[n * a.ldws + k + g];
        }
        if (xb) sx = a.xs[t * a.ldxs + k + g];
        if (XF == LORA_E4M3) {
            const int b = k + (g >> 1);
            if (tx && b < a.blocks) x0 = *(const u32x4*)(a.x + t * a.ldx + 32 * (int64_t)b + 16 * (g & 1));
            if (tx && b + 2 < a.blocks) x1 = *(const u32x4*)(a.x + t * a.ldx + 32 * (int64_t)(b + 2) + 16 * (g & 1));
        } else if (xb) {
            x0 = *(const u32x4*)(a.x + t * a.ldx + 16 * (int64_t)(k + g));
        }
        const i32x8 A = {(int)w[0], (int)w[1], (int)w[2], (int)w[3], 0, 0, 0, 0};
        const i32x8 B = {(int)x0[0], (int)x0[1], (int)x0[2], (int)x0[3], (int)x1[0], (int)x1[1], (int)x1[2], (int)x1[3]};
        acc = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(A, B, acc, 4, XF == LORA_E4M3 ? 0 : 4, 0, (int)sw, 0, (int)sx);
    }
    store4(a, t, blockIdx.x * 16 + 4 * g, acc);
}

int check_product(const lora_mx_t* x, const lora_mx_t* w) {
    if (int rc = check_mx("x", x)) return rc;
    if (int rc = check_mx("w", w)) return rc;
    if (w->format != LORA_E2M1) return set_error(LORA_E_ARG, "w: format must be LORA_E2M1");
    if (x->h != w->h) return set_error(LORA_E_SHAPE, "x and w differ in h");
    if (w->n_rows < 8 || w->n_rows % 8) return set_error(LORA_E_SHAPE, "w: n_rows must be a positive multiple of 8");
    return LORA_OK;
}

}  // namespace
}  // namespace lora

using namespace lora;

extern "C" {

int lora_mx_workspace_bytes(const lora_mx_t* x, const lora_mx_t* w, size_t* bytes) {
    if (int rc = check_product(x, w)) return rc;
    if (!bytes) return set_error(LORA_E_ARG, "bytes is NULL");
    *bytes = 16;
    return LORA_OK;
}

int lora_mx_apply(const lora_mx_t* x, const lora_mx_t* w, void* y, int64_t ldy, int32_t dtype, void* ws,
                  size_t ws_bytes, void* stream) {
    size_t need = 0;
    if (int rc = lora_mx_workspace_bytes(x, w, &need)) return rc;
    if (dtype != LORA_F16 && dtype != LORA_BF16 && dtype != LORA_F32)
        return set_error(LORA_E_ARG, "dtype must be LORA_F16, LORA_BF16 or LORA_F32");
    if (int rc = check_kv_rows("y", y, "ldy", ldy, w->n_rows, x->n_rows)) return rc;
    if (ldy > (1ll << 40)) return set_error(LORA_E_SHAPE, "ldy exceeds 2^40");
    if (!ws || ws_bytes < need) return set_error(LORA_E_WORKSPACE, "workspace smaller than lora_mx_workspace_bytes");
    if (!is_aligned16(ws)) return set_error(LORA_E_ALIGN, "ws not 16-byte aligned");
    const int64_t e = dtype == LORA_F32 ? 4 : 2;
    const Span out[2] = {Span(y, x->n_rows, ldy * e, w->n_rows * e), Span(ws, 1, 0, (int64_t)need)};
    const Span in[4] = {codes_span(x), scales_span(x), codes_span(w), scales_span(w)};
    for (const Span& o : out)
        for (const Span& i : in)
            if (o.meets(i)) return set_error(LORA_E_OVERLAP, "y or ws overlaps x or w");
    if (out[0].meets(out[1])) return set_error(LORA_E_OVERLAP, "y and ws overlap");
    if (x->n_rows == 0) return LORA_OK;
    hipStream_t st = (hipStream_t)stream;
    StreamDevice g(st);
    if (!g.ok) return set_error(LORA_E_HIP, "lora_mx_apply: no device for the stream");
    GemmArgs a;
    a.x = (const unsigned char*)x->codes;
    a.xs = (const unsigned char*)x->scales;
    a.w = (const unsigned char*)w->codes;
    a.ws = (const unsigned char*)w->scales;
    a.y = y;
    a.ldx = x->ld_codes;
    a.ldxs = x->ld_scales;
    a.ldw = w->ld_codes;
    a.ldws = w->ld_scales;
    a.ldy = ldy;
    a.n_rows = x->n_rows;
    a.h_out = w->n_rows;
    a.blocks = (int)mx_blocks(x->h);
    a.dtype = dtype;
    const int64_t gy = ((int64_t)a.n_rows + 15) / 16;
    if (gy > 65535) return set_error(LORA_E_SHAPE, "lora_mx_apply: too many rows");
    const dim3 grid((a.h_out + 15) / 16, (unsigned)gy);
    if (x->format == LORA_E4M3) hipLaunchKernelGGL(lora_mx_tile_kernel<LORA_E4M3>, grid, dim3(64), 0, st, a);
    else hipLaunchKernelGGL(lora_mx_tile_kernel<LORA_E2M1>, grid, dim3(64), 0, st, a);
    return check_launch("lora_mx_apply");
}

}  // extern "C"
