/*
 * lora_mx.h - Rows in blocks of 8- and 4-bit elements with a scale, and what a
 * serving step does with them, on MI355X (gfx950).
 *
 * Equation 1 adds each request's adapter to a base weight that all requests share.
 * Here that weight is kept in 4 bits: a step runs, for every projection,
 *
 *     h, hq = norm(x + residual)             lora_norm: 16 bits for the adapters, 8 for the base
 *     y     = hq W                           lora_mx_apply, W [h_out, h_in] from lora_mx_quantize
 *     y    += s_g (h A_g) B_g                lora_plan_apply (lora.h)
 *
 * and lora_mx_quantize makes ready what does not come out of a norm (attention's
 * output in front of the o projection).  lora_mx_dequantize is the way back.
 *
 * Blocks.  A row of h elements is ceil(h / 32) blocks of 32 elements.  Element e of
 * block b is code * 2^(scale - 127), where scale is the block's byte; a block whose scale
 * is 255 is NaN.  Formats:
 *
 *   LORA_E4M3   one byte an element: sign, 4 exponent bits (bias 7), 3 mantissa bits; up
 *               to 448, 0x7f and 0xff are NaN.  32 bytes a block.
 *   LORA_E2M1   4 bits an element: sign, 2 exponent bits (bias 1), 1 mantissa bit: 0, 0.5,
 *               1, 1.5, 2, 3, 4, 6.  16 bytes a block, the even element in a byte's low half.
 *
 * Byte i of row r is codes[r * ld_codes + i], its blocks' scales are scales[r * ld_scales + b].
 * The elements of the last block past h have zero codes; the calls that write blocks write
 * them so, and never write past the last block.
 *
 * Quantisation.  With m the largest magnitude of a block and emax 8 (E4M3) or 2 (E2M1),
 *
 *     scale = max(0, floor(log2 m) - emax + 127)   (0 for a block of zeros)
 *
 * and every element is divided by 2^(scale - 127), exactly, rounded to the nearest code (ties
 * to even) and held to the largest one.  A block with a NaN or an infinity gets the scale 255
 * and zero codes.
 *
 * Requirements, checked on the host before anything is enqueued (negative code,
 * lora_last_error() set, nothing enqueued):
 *   - h, h_out and leading dimensions in elements: positive multiples of 8, a leading
 *     dimension at least the row's width; 16-bit and 32-bit rows 16-byte aligned (32-bit
 *     leading dimensions too);
 *   - codes 16-byte aligned, ld_codes a multiple of 16 and at least a row's bytes;
 *     scales 4-byte aligned, ld_scales a multiple of 4 and at least a row's blocks;
 *     (the product reads scales in whole 4-byte words, behind the last row's last block up to 3 bytes more, which
 *     may hold anything but have to be readable);
 *   - codes and scales of the product's x and w: 256 leading dimensions within 0x7fff0000 bytes; rows of x
 *     times rows of w at most 2^42;
 *   - element types LORA_F16, LORA_BF16, and LORA_F32 where it is named;
 *   - outputs do not overlap inputs or each other, but where it is said.  Matrices whose rows are equally far
 *     apart may be columns of one buffer; of others the memory from the first byte to the last counts.
 *
 * Asynchrony, errors and thread safety are lora.h's: calls are enqueued on the caller's
 * stream, allocate nothing, copy nothing to the host and never wait.  All may be recorded
 * in a HIP graph.  The same inputs give the same bits.
 */
#ifndef LORA_MX_H
#define LORA_MX_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

#define LORA_F32 2              /* beside LORA_F16 and LORA_BF16 */

#define LORA_E4M3 0
#define LORA_E2M1 1

/* Rows in blocks (HOST structure of DEVICE pointers). */
typedef struct {
    void* codes;
    void* scales;
    int64_t ld_codes, ld_scales;   /* bytes from row to row     */
    int32_t n_rows;
    int32_t h;                     /* elements of a row         */
    int32_t format;                /* LORA_E4M3 or LORA_E2M1    */
} lora_mx_t;

/*
 * For every row, in float32 and more, with one rounding at each output:
 *
 *     s = x + residual          total gets s
 *     y = s * weight / sqrt(mean(s^2) + eps)
 *
 * and q gets y in blocks (from y before its rounding to `dtype`).  residual, weight and total may be NULL (no
 * addition, ones, s not kept); y or q may be NULL, not both.  x, residual, total and y
 * [n_rows, ld] and weight [h] are of `dtype` (LORA_F16 or LORA_BF16), q of LORA_E4M3 or
 * LORA_E2M1 with n_rows rows.  total may be x or residual itself, and y may be x or residual itself
 * (the same pointer and leading dimension; total and y not the same).  h at most 65536; eps
 * positive and finite.  A row whose squares pass float32's range comes out as zeros (its infinities as NaN).
 */
int lora_norm(const void* x, int64_t ldx, const void* residual, int64_t ldr, const void* weight, float eps,
              int32_t n_rows, int32_t h, int32_t dtype, void* total, int64_t ldt, void* y, int64_t ldy,
              const lora_mx_t* q, void* stream);

/* Rows x [q->n_rows, ldx] of `dtype` (LORA_F16, LORA_BF16 or LORA_F32) into blocks. */
int lora_mx_quantize(const void* x, int64_t ldx, int32_t dtype, const lora_mx_t* q, void* stream);

/* Blocks into rows y [q->n_rows, ldy] of `dtype` (LORA_F16, LORA_BF16 or LORA_F32), rounded
 * to nearest even. */
int lora_mx_dequantize(const lora_mx_t* q, void* y, int64_t ldy, int32_t dtype, void* stream);

/* Device workspace of lora_mx_apply for these rows and this weight, in bytes: any contents, 16-byte
 * aligned, overwritten.  Calls that share it must be ordered on one stream. */
int lora_mx_workspace_bytes(const lora_mx_t* x, const lora_mx_t* w, size_t* bytes);

/*
 * y[t, n] = sum_k x[t, k] w[n, k]: rows x [n_rows, h_in] (LORA_E4M3 or LORA_E2M1) times a
 * weight w [h_out, h_in] (LORA_E2M1, the layout of a linear layer), y [n_rows, ldy] of `dtype`
 * (LORA_F16, LORA_BF16 or LORA_F32) is output only.  Sums are float32, rounded once.  With x in
 * E4M3 the matrix instruction adds eight consecutive products at a time and cuts off what lies
 * below 2^-13 of the largest of them (measured: 4.4e-6 of y for normal rows, where a
 * rounding to bfloat16 is 1.7e-3, one to binary16 2e-4, and float32 sums would be off by some 1e-7).
 * About one in 250 values of y in bfloat16 is then the other neighbour of its exact value; y in
 * LORA_F32 is as exact as that and no more.  With x in E2M1 it adds exactly.
 */
int lora_mx_apply(const lora_mx_t* x, const lora_mx_t* w, void* y, int64_t ldy, int32_t dtype, void* ws,
                  size_t ws_bytes, void* stream);

#ifdef __cplusplus
}
#endif

#endif /* LORA_MX_H */
