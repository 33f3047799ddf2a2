/*
 * espace_train.h - the two ends of a model that is retrained around projected
 * layers: token embeddings, and the losses on the logits of its head.
 *
 * The head is a linear layer S = W·X over a vocabulary of V entries: the dense
 * one, or a projected one's folded weight with Z in place of X.  Its logits S
 * [N][V] are never kept: the losses read them in pieces of the vocabulary, and the
 * gradient calls compute them again, piece by piece, next to the gradients'
 * products.  The gradients with respect to the activations are also what the
 * NL-MSE calibration of espace.h takes.
 *
 * Letters: K features, N tokens, V vocabulary entries, T teacher entries a token.
 *     X       [N][K]   activations (rows are tokens)
 *     W       [V][K]   head or embedding, a row per vocabulary entry
 *     labels  [N]      int64
 *     index   [N][T]   int64, the teacher's entries; logits [N][T] float32, theirs
 *     loss, lse, dloss [N] float32
 *
 * The conventions of espace.h hold (device pointers, leading dimensions, dtypes,
 * workspaces, statuses, streams; the same call on the same operands gives the same
 * bits again), with these additions: int64 and float32 arrays need their natural
 * alignment alone, a leading dimension of index, logits and picked any value >= T.
 * Most float32 products run on the bfloat16 matrix cores, a value as the sum of three
 * bfloat16, to at most 2^-23 of each product beside the sums' roundings: an infinity, or
 * a value that rounds to one in bfloat16, gives NaN there, and values below 2^-110 lose
 * their last bits.
 * Limits: 1 <= V <= 2^30, 1 <= K <= 2^21, N < 2^21 (more tokens: several calls, whose
 * dW, each rounded to its type, the caller adds).
 *
 * Tokens without a target are part of the call and have no loss: it is 0, their row
 * of dX is 0, and they add nothing to dW, whatever their rows of X and their dloss
 * hold (NaN and infinities included).
 *
 * Targets outside the vocabulary (>= V) are a caller's error that only the device
 * sees.  The token's loss is NaN, and so are, of the gradients,
 *     a label             the token's row of dX and every row of dW
 *     a teacher's entry   the token's row of dX and the rows of dW of all its entries,
 *                         where the last one, V - 1, stands for those past the
 *                         vocabulary (none of them where the token's dloss is 0)
 * lse, the other tokens' losses and rows of dX, and the other rows of dW are right.
 */
#ifndef ESPACE_TRAIN_H
#define ESPACE_TRAIN_H

#include "espace.h"

#ifdef __cplusplus
extern "C" {
#endif

#define ESPACE_MAX_TEACHER_ENTRIES 1024

/* ---- Cross entropy ----------------------------------------------------------
 * With s_v = x_n·w_v (float32 sums, not rounded):
 *     lse[n]  = log Σ_v exp(s_v)
 *     loss[n] = lse[n] - s_label,  0 for a label < 0
 * In: X [N][K] (ldx), W [V][K] (ldw), labels [N].  Out: loss [N], lse [N] (both
 * required; the backward pass takes lse).
 * Needs espace_linear_loss_workspace_bytes(0, N, K, V, 0, dt). */
espace_status espace_linear_cross_entropy(const void* X, int64_t ldx, const void* W, int64_t ldw,
                                          const int64_t* labels, float* loss, float* lse,
                                          int64_t N, int64_t K, int64_t V, espace_dtype dt,
                                          void* workspace, size_t workspace_bytes, hipStream_t stream);

/* Gradients for an upstream gradient dloss[n] = ∂ℓ/∂loss[n] (1/N for a mean):
 *     G[n][v] = dloss[n]·(exp(s_v - lse[n]) - [v = label])
 *     dX = G·W       dW = Gᵀ·X
 * bf16: G, taken relative to the largest |dloss|, is rounded to bfloat16 once (up to
 * 128 tokens: kept as the sum of two bfloat16); the sums are float32 and rounded once
 * (dX of several pieces: added in float32).  In norm, the results' own rounding leaves
 * dX and dW 1.7e-3 off.  Of more than 128 tokens G's adds next to nothing to that where
 * all dloss are alike (the entry of an improbable label is exact then), and makes it
 * 2.2e-3 with unlike ones, up to 2.6e-3 where many tokens share one.
 * In: dloss [N], X, W, labels, lse [N] as the forward call gave it.  Out: dX [N][K]
 * (lddx) and/or dW [V][K] (lddw) (either may be NULL).
 * Needs espace_linear_loss_workspace_bytes(1, N, K, V, 0, dt). */
espace_status espace_linear_cross_entropy_backward(const float* dloss, const void* X, int64_t ldx,
                                                   const void* W, int64_t ldw, const int64_t* labels,
                                                   const float* lse, void* dX, int64_t lddx, void* dW,
                                                   int64_t lddw, int64_t N, int64_t K, int64_t V,
                                                   espace_dtype dt, void* workspace, size_t workspace_bytes,
                                                   hipStream_t stream);

/* ---- Distillation from a teacher's top logits ---------------------------------
 * The student's logits are those of the head, s_v = x_n·w_v / t at the temperature
 * t.  The teacher gives token n up to T vocabulary entries i_j = index[n][j] with
 * its logits z_j; an index < 0 marks an empty place.  Its distribution is the
 * softmax of its entries, p_j = exp(z_j / t) / Σ exp(z / t) (an entry of -infinity
 * has probability 0; a token whose places are all empty or -infinity has no target).
 *     lse[n]  = log Σ_v exp(s_v)
 *     loss[n] = t²·Σ_j p_j·(log p_j - s_{i_j} + lse[n])
 *     picked[n][j] = s_{i_j}, 0 in empty places (kept for the backward pass)
 * An entry that occurs more than once counts each time.
 * In: X, W, index [N][T] (ldi), logits [N][T] (ldl).  Out: loss [N], lse [N],
 * picked [N][T] (ldpk).  1 <= T <= ESPACE_MAX_TEACHER_ENTRIES; t > 0 and finite
 * (another t: ESPACE_ERR_SHAPE).
 * Needs espace_linear_loss_workspace_bytes(0, N, K, V, T, dt). */
espace_status espace_linear_distillation(const void* X, int64_t ldx, const void* W, int64_t ldw,
                                         const int64_t* index, int64_t ldi, const float* logits, int64_t ldl,
                                         float* loss, float* lse, float* picked, int64_t ldpk,
                                         int64_t N, int64_t K, int64_t V, int64_t T, float temperature,
                                         espace_dtype dt, void* workspace, size_t workspace_bytes,
                                         hipStream_t stream);

/* Its gradients, as above with
 *     G[n][v] = dloss[n]·t·(exp(s_v - lse[n]) - Σ_{j: i_j = v} p_j)
 * (bf16, more than 128 tokens: the probabilities' rounding in G leaves dX and dW 2.1e-3
 * to 2.6e-3 off in norm, with any dloss).
 * In: dloss [N], X, W, index, logits, lse, picked as the forward call had and gave
 * them.  Out: dX [N][K] and/or dW [V][K].
 * Needs espace_linear_loss_workspace_bytes(1, N, K, V, T, dt). */
espace_status espace_linear_distillation_backward(const float* dloss, const void* X, int64_t ldx,
                                                  const void* W, int64_t ldw, const int64_t* index, int64_t ldi,
                                                  const float* logits, int64_t ldl, const float* lse,
                                                  const float* picked, int64_t ldpk, void* dX, int64_t lddx,
                                                  void* dW, int64_t lddw, int64_t N, int64_t K, int64_t V,
                                                  int64_t T, float temperature, espace_dtype dt,
                                                  void* workspace, size_t workspace_bytes, hipStream_t stream);

/* Workspace bytes of the four calls above: backward 0 or 1, T = 0 for cross
 * entropy.  SIZE_MAX for invalid sizes. */
size_t espace_linear_loss_workspace_bytes(int backward, int64_t N, int64_t K, int64_t V, int64_t T,
                                          espace_dtype dt);

/* ---- Embedding -----------------------------------------------------------------
 * X[n] = scale·E[tokens[n]] (the product in float32, rounded once; with scale 1 the
 * row itself), a row of zeros for a token < 0 (padding), of NaN for one >= V.
 * In: tokens [N], E [V][K] (lde).  Out: X [N][K] (ldx).  No workspace. */
espace_status espace_embedding(const int64_t* tokens, const void* E, int64_t lde, void* X, int64_t ldx,
                               int64_t N, int64_t K, int64_t V, float scale, espace_dtype dt,
                               hipStream_t stream);

/* Its gradient: dE[v] = scale·Σ_{n: tokens[n] = v} dX[n], float32 sums in the order
 * of n, rounded once.  accumulate = 0: every row of dE is written (zeros for an
 * entry that no token names); accumulate != 0: dE[v] + scale·Σ is rounded once, and
 * rows that no token names are not touched (a head tied to the embedding: dE is the
 * head's dW).  Tokens outside [0, V) add nothing.
 * In: tokens [N], dX [N][K] (lddx).  Out (in/out): dE [V][K] (ldde).
 * Needs espace_embedding_workspace_bytes(N, K, V). */
espace_status espace_embedding_backward(const int64_t* tokens, const void* dX, int64_t lddx, void* dE,
                                        int64_t ldde, int64_t N, int64_t K, int64_t V, float scale,
                                        int accumulate, espace_dtype dt, void* workspace,
                                        size_t workspace_bytes, hipStream_t stream);
size_t espace_embedding_workspace_bytes(int64_t N, int64_t K, int64_t V);

#ifdef __cplusplus
}
#endif

#endif /* ESPACE_TRAIN_H */
