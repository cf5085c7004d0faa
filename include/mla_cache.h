/*
 * mla_cache.h -- C ABI of the compact latent cache around the mixed-step
 * attention (libmlastep.so): appends that rotate the positions on the way, a
 * cache held in 8 bits, attention over it, and attention through a sliding
 * window with a few first tokens that stay visible.
 *
 * Batches, row order, positions, streams, errors, device flags and check mode
 * are those of mla_step.h.  Row i of request r has position p_r + i.
 *
 * Rotation.  new_latents holds, per row, 512 compressed dims as they are cached
 * and 64 rope dims x before rotation; with base b > 1 the cached rope dims of a
 * token at position t are, for i < 32,
 *     (x_2i cos a - x_2i+1 sin a,  x_2i sin a + x_2i+1 cos a),  a = t b^(-2i / 64).
 * The angle is reduced in 64 bits, its sine and cosine and the rotation are
 * computed in fp32.  Queries are the caller's (rotated before the attention).
 *
 * The 8-bit cache.
 *   data    DEVICE uint8 [num_pages][P][576]: e4m3 codes (sign, 4 exponent bits
 *           with bias 7, 3 mantissa bits; 0x7F / 0xFF is NaN, no infinity).
 *   scales  DEVICE bf16 [num_pages][P / 16][2]: every block of 16 tokens of a
 *           page has one scale for its 512 compressed dims and one for its 64
 *           rope dims, each a power of two in [2^-100, 2^120].  A key's value is
 *           code x scale (exact in bf16; of magnitude below 2^128, so at a scale of
 *           2^120 codes are at most 240).
 *   The page size P is at least 16.
 * Append (append_latent_kv8) takes the rows' values (rotated, in fp32, if asked)
 * and, for every block that it writes into and each of the two parts, the
 * smallest scale of that range with which no finite value exceeds 448, the
 * largest e4m3 value; a block that holds earlier tokens of the request (p_r
 * inside it) keeps its own scale if that is larger, otherwise those earlier
 * tokens are rounded again to the new scale.  Values are rounded to nearest,
 * ties to even, once (at a scale of 2^120 to at most 240, which is within half a
 * step of every finite bf16: 2^-4 of it); NaN and infinities are stored as NaN.
 * Other tokens of the pool are left as they are.
 *   What mla_step.h says about written slots holds for blocks here: a block
 *   that one request writes into belongs to it alone in that step.
 *
 * Window.  With a window of W keys and S sinks, the row at position t sees the
 * keys j <= t with j > t - W or j < S.  W >= 1, so a row always sees itself.
 * Block-table entries of pages that hold no key that a row of the request sees
 * may be anything, in appends as well; page 0 is read in place of a page outside
 * the pool.  Keys are read in tiles of 32: up to 31 hidden keys behind the sinks
 * and as many before the window of a block of 8 rows are read with the seen ones
 * (whatever they hold, it does not reach a result), the tiles between are not.
 *
 * Values that are not finite.  Keys that a row does not see never reach it,
 * whatever they hold.  Those that it sees count as the sums say: a score of NaN
 * or +inf makes the row's output and lse of that head NaN, one of -inf has a
 * weight of 0, and 0 x inf is NaN in the dims whose value is infinite.
 *
 * Probabilities meet the values with 22 bits or more; in chunk rows with bf16
 * output, which rounds to fewer, with 11.  Sums are fp32.
 */
#ifndef MLA_CACHE_H
#define MLA_CACHE_H

#include "mla_step.h"

#ifdef __cplusplus
extern "C" {
#endif

#define MLA_CACHE8_BLOCK 16 /* tokens that share a pair of scales */

typedef struct mla_cache8 {
    uint8_t *data;
    uint16_t *scales;
} mla_cache8;

typedef struct mla_window {
    int32_t window; /* W >= 1 */
    int32_t sinks;  /* S >= 0 */
} mla_window;

/* Bytes of the scales of a pool, rounded up to a multiple of 16 (0 on invalid
 * arguments: num_pages < 1, or a page size that is not a power of two in [16,
 * 1024]).  Nothing outside the scales themselves is read. */
size_t mla_cache8_scale_bytes(int32_t num_pages, int32_t page_size);

/* append_latent_kv with the rotation applied on the way.
 *   new_latents  DEVICE bf16 [T][576], rope dims not rotated.
 *   rope_base    b, finite, > 1.
 *   kv_cache     DEVICE bf16 [num_pages][P][576]; only the T written slots
 *                change (rotated dims rounded to nearest even once, the others
 *                copied).
 * Errors: as append_latent_kv, and MLA_ERR_INVALID_ARG for a bad base. */
int append_latent_kv_rope(const mla_batch *batch, const uint16_t *new_latents, float rope_base, uint16_t *kv_cache,
                          void *stream);

/* Append into the 8-bit cache (the rules above).
 *   rope_base    b, finite, > 1; or 0: the rope dims are rotated already
 *                (the new_latents of mla_pre_attn).
 * Errors: MLA_ERR_INVALID_ARG (null or misaligned pointer with T > 0: 16 bytes;
 * a bad base), MLA_ERR_UNSUPPORTED (page size not a power of two in [16, 1024]),
 * MLA_ERR_HIP. */
int append_latent_kv8(const mla_batch *batch, const uint16_t *new_latents, float rope_base, const mla_cache8 *cache,
                      void *stream);

/* Workspace bytes of mixed_step_attn8 (window NULL: none) and of
 * mixed_step_attn_window for this batch: rules as for
 * mixed_step_workspace_bytes, its first 256 bytes zeroed once before the first
 * use; a workspace may serve all the entry points in turn if it is large
 * enough for each.  0 on invalid arguments (then mla_last_error says why). */
size_t mixed_step_attn8_workspace_bytes(const mla_batch *batch, const mla_window *window);
size_t mixed_step_attn_window_workspace_bytes(const mla_batch *batch, const mla_window *window);

/* mixed_step_attn over the 8-bit cache, which already holds the step's tokens
 * (call append_latent_kv8 first, on the same stream).
 *   window       NULL: every earlier key is visible.
 *   other arguments as for mixed_step_attn.  Scores are sums in fp32, as there.
 *   Value dims (code x scale) go through fp16 relative to a scale of the blocks
 *   read, and rows that are cut into parts keep the parts' averages, so no value
 *   below 2^128 is too large; those of a decode row are off by at most 2^-25 of
 *   the largest compressed scale that it sees, those of a chunk row by at most
 *   2^-25 of the largest that its block of 8 rows sees (rows 8 k .. 8 k + 7 of
 *   the request).  Scales at most 2^15 apart lose nothing.
 * Errors: as mixed_step_attn, and MLA_ERR_INVALID_ARG for a bad window,
 * MLA_ERR_UNSUPPORTED for a page size below 16. */
int mixed_step_attn8(const mla_batch *batch, const uint16_t *q, const mla_cache8 *cache, const mla_window *window,
                     float softmax_scale, void *out, int32_t out_dtype, float *lse, void *workspace,
                     size_t workspace_bytes, void *stream);

/* mixed_step_attn (bf16 cache) through a window.
 * Errors: as mixed_step_attn, and MLA_ERR_INVALID_ARG for a bad window. */
int mixed_step_attn_window(const mla_batch *batch, const uint16_t *q, const uint16_t *kv_cache, const mla_window *window,
                           float softmax_scale, void *out, int32_t out_dtype, float *lse, void *workspace,
                           size_t workspace_bytes, void *stream);

#ifdef __cplusplus
}
#endif

#endif /* MLA_CACHE_H */
