/*
 * mla_ffn.h -- C ABI of the feed-forward half of a layer (libmlastep.so): the
 * gated feed-forward block that follows the attention layer of mla_layer.h,
 * and products with weights held in 4 bits.
 *
 * For each row t of x [T][H]:
 *   g = x[t] Wg^T, u = x[t] Wu^T          [I]   (gate and up projections)
 *   h = g / (1 + exp(-g)) * u             [I]
 *   out[t] = h Wd^T                       [H]   (down projection)
 * and, for a product on its own, out[t] = x[t] W^T.
 *
 * Weights are row-major with the reduction dimension contiguous, as the model
 * stores its linear layers: w_gate and w_up [I][H], w_down [H][I], w [N][K].
 *
 * 4-bit weights (mla_mx4).
 *   codes   DEVICE uint8 [N][K / 2]: two codes a byte, the even one in the low
 *           half.  A code is a sign (8) and a magnitude out of
 *           0, 0.5, 1, 1.5, 2, 3, 4, 6 (two exponent bits, one mantissa bit).
 *   scales  DEVICE uint8 [N][K / 32]: each 32 neighbouring weights of a row
 *           share one byte b, which stands for 2^(b - 127); 255 makes its 32
 *           weights NaN.
 *   A weight is code x scale.  Every such value below 2^128 is exact in bf16,
 *   so a product with 4-bit weights is the product with those bf16 values;
 *   the values from 2^128 on (b = 253 and 254 only) count as infinite.
 *
 * Precision: bf16 inputs, fp32 sums.  h is computed in fp32 and meets w_down
 * as one bf16, rounded to nearest even, where out is bf16.  Where out is fp32 it
 * meets it as the sum of three bf16: with all its 24 bits from 2^-110 on, below
 * that as the nearest multiple of 2^-133, and no smaller than 3 x 2^-133 unless
 * it is 0.  Values that are not finite count as the formulas say, in every row
 * that they belong to and no other.
 *
 * Conventions, errors and streams are those of mla_step.h.  Device arrays are
 * contiguous and 16-byte aligned; out overlaps no input and no workspace.
 * Calls read their inputs and write out and the workspace, nothing else.
 *
 * Workspaces are caller-allocated device memory.  The first
 * MLA_FFN_COUNTER_BYTES bytes are counters: they must be zero when a workspace
 * is first used, and every completed call leaves them zero again.  The rest is
 * ignored on entry: 64 MiB for parts of sums whatever the sizes, and in a
 * block's 6 T I bytes more whatever out's type.  A workspace for T rows serves
 * calls of fewer rows with weights of the same sizes, and the same workspace may
 * serve all entry points in turn; calls that overlap in time need distinct ones.
 * Results do not depend on what ran before: sums that are cut into parts are
 * joined in one order.
 */
#ifndef MLA_FFN_H
#define MLA_FFN_H

#include "mla_step.h"

#ifdef __cplusplus
extern "C" {
#endif

#define MLA_MX4_GROUP 32 /* weights that share a scale */
#define MLA_FFN_COUNTER_BYTES 4096

typedef struct mla_mx4 {
    const uint8_t *codes;
    const uint8_t *scales;
} mla_mx4;

/* Sizes: hidden (H) and inner (I) are positive multiples of 8 with bf16 weights,
 * of 32 with 4-bit ones. */
typedef struct mla_ffn_weights {
    const uint16_t *w_gate; /* bf16 [I][H] */
    const uint16_t *w_up;   /* bf16 [I][H] */
    const uint16_t *w_down; /* bf16 [H][I] */
    int32_t hidden;
    int32_t inner;
} mla_ffn_weights;

typedef struct mla_ffn4_weights {
    mla_mx4 w_gate; /* [I][H] */
    mla_mx4 w_up;   /* [I][H] */
    mla_mx4 w_down; /* [H][I] */
    int32_t hidden;
    int32_t inner;
} mla_ffn4_weights;

/* Workspace bytes of mla_linear4 for T rows (0 on sizes that it refuses, and if
 * T <= 0). */
size_t mla_linear4_workspace_bytes(int32_t num_rows, int32_t in_features, int32_t out_features);

/* out = x W^T with 4-bit weights, for T rows.
 *   x             DEVICE bf16 [T][K].
 *   in_features   K, a positive multiple of 32.
 *   out_features  N, a positive multiple of 8.
 *   out           DEVICE [T][N] fp32 or bf16 (out_dtype).
 * Errors: MLA_ERR_INVALID_ARG (a null or misaligned pointer with T > 0, T < 0,
 * an unknown out_dtype, a size < 1), MLA_ERR_UNSUPPORTED (sizes that are not
 * such multiples, or above 2^24, more than 2^28 rows, more tiles of outputs
 * than a launch takes), MLA_ERR_WORKSPACE, MLA_ERR_HIP. */
int mla_linear4(int32_t num_rows, const uint16_t *x, const mla_mx4 *w, int32_t in_features, int32_t out_features, void *out,
                int32_t out_dtype, void *workspace, size_t workspace_bytes, void *stream);

/* Workspace bytes of mla_gated_ffn and mla_gated_ffn4 for T rows, either output
 * type (0 on sizes that they refuse, and if T <= 0). */
size_t mla_gated_ffn_workspace_bytes(int32_t num_rows, int32_t hidden, int32_t inner);

/* The gated feed-forward block, for T rows.
 *   x    DEVICE bf16 [T][H].
 *   out  DEVICE [T][H] fp32 or bf16 (out_dtype).
 * Errors: as mla_linear4. */
int mla_gated_ffn(int32_t num_rows, const uint16_t *x, const mla_ffn_weights *w, void *out, int32_t out_dtype, void *workspace,
                  size_t workspace_bytes, void *stream);
int mla_gated_ffn4(int32_t num_rows, const uint16_t *x, const mla_ffn4_weights *w, void *out, int32_t out_dtype, void *workspace,
                   size_t workspace_bytes, void *stream);

#ifdef __cplusplus
}
#endif

#endif /* MLA_FFN_H */
