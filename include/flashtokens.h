/*
 * flashtokens.h -- C ABI of the operators on token tables in libflashkmeans.so
 * (AMD Instinct MI355X, gfx950).
 *
 * A table W holds one row per token: a codebook that kmeans_lloyd found and
 * kmeans_assign encodes with, or the embedding or output matrix of a model that
 * learns such tokens.  The calls look rows up and train them, and score rows
 * against a whole table.
 *
 * The conventions of flashkmeans.h hold (types, status codes, ownership, stream,
 * capture, determinism, workspaces), and these:
 * - W holds B tables of V rows of D elements, [B, V, D]; the other arrays hold B
 *   instances of M positions.  Tokens are int32 and local to an instance.
 * - A position whose token lies outside [0, V) (kmeans_assign's -1, padding) has
 *   no token: a zero row, log probability 0, no gradient.
 * - Tables and rows of elements are 16-byte aligned; arrays of one 4-byte value a
 *   position or token (tokens, offsets, statistics, alternatives) start anywhere.
 * - Offsets are 64 bits wide: no array has a size limit of its own.  B up to
 *   65,535, M up to 2^24 (2^23 - 64 for tokens_logprobs_grad), V up to 2^20, D up
 *   to 8,192.
 * - Outputs overlap neither inputs, nor each other, nor the workspace.
 */
#ifndef FLASHTOKENS_H_
#define FLASHTOKENS_H_

#include "flashkmeans.h"

#ifdef __cplusplus
extern "C" {
#endif

/*
 * Rows of a table, times a factor.
 *   W      [B, V, D] dtype  table (read)
 *   idx    [B, M]    int32  tokens (read)
 *   out    [B, M, D] dtype  written: scale * W[b, idx[b, m]], the product in fp32
 *                           rounded once; zeros where there is no token
 * dtype fp32, bf16 or fp16.  No workspace.
 */
int tokens_embed(const void* W, int dtype, const int32_t* idx, int64_t B, int64_t M, int64_t V,
                 int64_t D, float scale, void* out, void* stream);

/*
 * The gradient of tokens_embed in the table: the positions sorted by token
 * (stable), a segmented sum in fp32 in a fixed order, no floating-point atomics.
 *   G      [B, M, D] gdtype  gradients of the rows (read); positions without a
 *                            token are not read
 *   idx    [B, M]    int32   tokens (read)
 *   dW     [B, V, D] wdtype  accumulate 0: written, scale * the sum of G over the
 *                            token's positions (zeros for a token without one);
 *                            accumulate 1: that is added to dW (in fp32, rounded
 *                            once), and rows of tokens without a position are
 *                            left as they are
 * wdtype is gdtype or FKM_F32.  Workspace: tokens_embed_grad_workspace_bytes
 * (0 for arguments that the call would reject); for fixed B and D it never
 * decreases as M or V grows.
 */
size_t tokens_embed_grad_workspace_bytes(int64_t B, int64_t M, int64_t V, int64_t D, int gdtype);
int tokens_embed_grad(const void* G, int gdtype, const int32_t* idx, int64_t B, int64_t M,
                      int64_t V, int64_t D, float scale, int accumulate, void* dW, int wdtype,
                      void* ws, size_t ws_bytes, void* stream);

/*
 * Scores of rows against a whole table, z = scale * <x, w_v> + bias_v, and of
 * each row's softmax over them the log probability of a given token, the
 * entropy, the log-sum-exp and the k best tokens.  Products are exact, their
 * sums, the scores and the softmax's statistics fp32; the scores are not stored
 * (except for k > 0, a block of rows at a time, in the workspace).
 *   X           [B, M, D] xdtype  rows (read)
 *   W           [B, V, D] xdtype  table (read)
 *   bias        [B, V]    fp32    added to the scores (read); NULL: none.  -inf
 *                                 forbids a token, whatever its row of W holds
 *                                 (NaN and infinities too)
 *   target      [B, M]    int32   tokens (read); NULL: logprob is not written
 *   logprob     [B, M]    fp32    z[target] - lse; -inf for a forbidden token
 *   entropy     [B, M]    fp32    -sum p log p, in nats; may be NULL
 *   lse         [B, M]    fp32    log sum exp z
 *   top_idx     [B, M, k] int32   the k tokens of the largest scores, largest
 *                                 first, ties to the lowest token; -1 (and -inf)
 *                                 past the tokens that are not forbidden
 *   top_logprob [B, M, k] fp32    their log probabilities
 * 0 <= k <= min(V, 32) (more than 32 is FKM_ERR_UNSUPPORTED, more than V invalid);
 * with k = 0 the last two are not used.  A row all of whose tokens are forbidden
 * has lse and logprob -inf and entropy 0.  xdtype bf16 or fp16 (fp32 is
 * FKM_ERR_UNSUPPORTED).  A row of X with a NaN has NaN results and no other
 * row has; its top_idx are valid or -1.  D that is no multiple of 8 runs on padded
 * copies.  scale must be finite.  Products scale * <x, w> of magnitude 2^100 and
 * more are outside the contract; offsets may have any value but NaN and +inf.
 * Workspace: tokens_logprobs_workspace_bytes.
 */
size_t tokens_logprobs_workspace_bytes(int64_t B, int64_t M, int64_t V, int64_t D, int k,
                                       int xdtype);
int tokens_logprobs(const void* X, const void* W, int xdtype, const float* bias,
                    const int32_t* target, int64_t B, int64_t M, int64_t V, int64_t D, float scale,
                    int k, float* logprob, float* entropy, float* lse, int32_t* top_idx,
                    float* top_logprob, void* ws, size_t ws_bytes, void* stream);

/*
 * The gradient of sum_m g_m logprob_m + h_m entropy_m in X and W (bias is a
 * constant).  The scores are computed again; with p = exp(z - lse) (with offsets, a
 * row whose |lse| is 4,096 or more has its own maximum and sum taken again, as
 * fp32 holds neither p nor the number of tokens in such an lse),
 *   dz = g (1[v = target] - p) - h p (z - lse + entropy)
 *   dX = scale * dz W,   dW = scale * dz^T X.
 *   lse       [B, M] fp32  of tokens_logprobs (read)
 *   entropy   [B, M] fp32  of tokens_logprobs (read); NULL with grad_entropy NULL
 *   grad_logprob [B, M] fp32   g (read)
 *   grad_entropy [B, M] fp32   h (read); NULL: 0
 *   dX        [B, M, D] xdtype  written
 *   dW        [B, V, D] xdtype  written
 * A position without a token, or whose token is forbidden, has no gradient of
 * its log probability; a row with neither gradient, or with lse -inf, is not
 * used at all (it may hold anything) and gets dX 0.  Forbidden tokens get dW 0.
 * The two products take dz, X and W in fp16, sum in fp32 in a fixed order and round
 * once.  X and W are brought to fp16's range by the power of two of their instance's
 * largest value (half of 2^-39 of that is rounded off), dz by one of its
 * position's larger gradient (calls of up to 64 fp16 positions: by the target's dz, no
 * power of two).  bf16 results are as far off as their own rounding, fp16 ones up to
 * twice that.  A dz below 3e-8 of its position's larger gradient has fewer than 11
 * bits; below 1.5e-11 of it, it is 0.  In dW a position counts with fewer bits of small
 * values (of X and of dz) if its larger gradient is below 2^-12 of the instance's
 * largest, of all values below 2^-40, and not at all below 2^-54.
 * Workspace: tokens_logprobs_grad_workspace_bytes.
 */
size_t tokens_logprobs_grad_workspace_bytes(int64_t B, int64_t M, int64_t V, int64_t D, int xdtype);
int tokens_logprobs_grad(const void* X, const void* W, int xdtype, const float* bias,
                         const int32_t* target, const float* lse, const float* entropy,
                         const float* grad_logprob, const float* grad_entropy, int64_t B, int64_t M,
                         int64_t V, int64_t D, float scale, void* dX, void* dW, void* ws,
                         size_t ws_bytes, void* stream);

#ifdef __cplusplus
}
#endif

#endif /* FLASHTOKENS_H_ */
