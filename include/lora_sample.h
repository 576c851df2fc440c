/*
 * lora_sample.h - The next token of every row of a step's logits, on MI355X (gfx950).
 *
 * For a row with logits l_0 .. l_(V-1), temperature T, and l_max the largest logit:
 *
 *     w_i = round(2^43 exp((l_i - l_max) / T))              a whole number
 *     K   = the top_k largest logits
 *     P   = of K in falling order, the shortest start with sum w >= top_p * sum_K w (at
 *           least one logit): i is in P if the weights before it sum to less than top_p * sum_K w
 *     M   = { i : w_i >= 2^43 min_p }
 *     token = the first i of P and M, in the order of i, whose weights up to and with its own
 *             sum to more than floor(u * total), total = the sum over P and M
 *     prob  = w_token / total
 *
 * Equal logits are ordered by index, the lowest first.  Weights are whole numbers so that
 * their sums are exact in whatever order they are added: the same inputs give the same token
 * however the work is divided.  The weight of a token less likely than the likeliest by
 * 2^44 is zero.  Sums are compared in binary64.
 *
 *   - T below 2^-100 (0, less and NaN too): the largest logit, prob 1.  T above 2^100 is read as
 *     2^100.
 *   - top_k below 1 or not below V: all.  top_p not below 1 (or NaN): all; not above 0: one
 *     logit.  min_p not above 0 (or NaN): all; 1 and more: those of weight 2^43.
 *   - u outside [0, 1) (or NaN) is read as 0 below and as the last token that is left above.
 *   - A logit of -infinity or NaN is never chosen.  Where the largest is +infinity, all of that
 *     value weigh 2^43 and the others nothing.  A row with nothing left gets token -1, prob 0.
 *
 * Parameters and random numbers are in DEVICE memory and are read when a launch runs, so a
 * recorded step may be replayed with new ones.
 *
 * Requirements, checked on the host before anything is enqueued (negative code,
 * lora_last_error() set, nothing enqueued): n_vocab in [1, 2^19], ld at least n_vocab; logits aligned
 * to their elements, parameters, u, tokens and probs to 4 bytes; the workspace of
 * lora_sample_workspace_bytes, 16-byte aligned.  Any vocabulary size, leading dimension and row
 * alignment is taken (the widest loads need 16-byte aligned rows).
 *
 * Asynchrony, errors and thread safety are lora.h's: calls are enqueued on the caller's
 * stream, allocate nothing, copy nothing to the host and never wait.  They may be recorded in a
 * HIP graph.  Calls that share a workspace must be ordered on one stream.
 */
#ifndef LORA_SAMPLE_H
#define LORA_SAMPLE_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

/* Parameters of every row (HOST structure of DEVICE arrays [n_rows]); NULL for 1, all, 1 and 0. */
typedef struct {
    const float* temperature;
    const int32_t* top_k;
    const float* top_p;
    const float* min_p;
} lora_sample_t;

/* Device workspace of lora_sample in bytes; any contents, overwritten. */
int lora_sample_workspace_bytes(int32_t n_rows, int32_t n_vocab, int32_t dtype, size_t* bytes);

/*
 * logits [n_rows, ld] of `dtype` (LORA_F16, LORA_BF16 or LORA_F32), u [n_rows] random numbers
 * in [0, 1); tokens [n_rows] and, unless NULL, probs [n_rows] are written.
 */
int lora_sample(const void* logits, int64_t ld, int32_t dtype, int32_t n_rows, int32_t n_vocab,
                const lora_sample_t* params, const float* u, int32_t* tokens, float* probs, void* ws, size_t ws_bytes,
                void* stream);

#ifdef __cplusplus
}
#endif

#endif /* LORA_SAMPLE_H */
