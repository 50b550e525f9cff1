/*
 * ze.h -- C ABI of libzc, the vocabulary's operators: the two ends of a model on a
 * tensor-parallel rank that has a part of the vocabulary (MI355X, gfx950).
 *
 * A rank has the rows first .. first + rows - 1 of the embedding and of the output matrix.  Its
 * part of the embedding (zeros for other ranks' tokens) is the first message that is reduced over
 * the tensor-parallel ranks (Sec. II-A, Table I); the loss needs three floats for each token and
 * rank, and leaves the gradient of the last hidden states, which is reduced as well, and the gradients of the
 * rows, which go into the gradient bucket that include/zc.h compresses and include/zt.h clips.
 *
 * Conventions
 *   - d_* are DEVICE pointers owned by the caller, aligned to their elements unless said
 *     otherwise.  The library neither allocates, frees nor keeps them.
 *   - `stream` is a hipStream_t as void*; calls enqueue kernels on it and return without
 *     synchronising.  They only launch kernels, so sequences of them can be captured in a HIP
 *     graph.  Calls on different streams may run concurrently where they share no output and no workspace.
 *   - Return value: ZC_OK or a negative code of include/zc.h; on error nothing is launched.
 *   - Sums, exponentials and products are held in fp32; a value is rounded once, to the nearest with ties
 *     to even, where it is stored, but for what ze_vocab_loss_backward says.  Results do not depend on the
 *     order in which workgroups run.
 *   - A workspace is aligned to 256 bytes; its contents before and after a call do not matter.
 *   - No output overlaps an input or another output, and no two rows of an output overlap.  (One may take the place of another: d_dhidden that of
 *     d_hidden, at the same address with the same stride.)
 */
#ifndef ZE_H
#define ZE_H

#include <stddef.h>

#include "zc.h"

#ifdef __cplusplus
extern "C" {
#endif

enum ze_id_dtype { ZE_I32 = 0, ZE_I64 = 1 };
enum { ZE_MAX_TOKENS = 1 << 25, ZE_MAX_ROWS = 1 << 28, ZE_MAX_COLS = 65536 };

/* What the calls have in common.  `tokens` rows of `cols` values (the lookup's output, the hidden states) go with
 * an id each: a token or a label of the whole vocabulary.  The table (embedding or output matrix) has `rows` rows of
 * `cols` values.  A stride is the number of elements from one row to the next, 0 for cols. */
struct ze_form {
  size_t tokens, rows, cols;
  long long first;                       /* the id of the table's first row: from 0 to 2^63 - 1 - ZE_MAX_ROWS */
  int dtype;                             /* enum zc_dtype: of the table and of the tokens' rows */
  int grad_dtype;                        /* of ze_embedding_backward's d_dtable: dtype or ZC_F32; the others do not read it */
  int id_dtype;                          /* enum ze_id_dtype */
  float scale;                           /* finite: of the embedding, or of the logits */
  size_t stride_table, stride_tokens;    /* inputs: of the table; of hidden states and of the gradient of the lookup's output */
  size_t stride_dtable, stride_dtokens;  /* outputs: of the table's gradient; of the lookup and of the hidden states' gradient */
};

/* d_out[n] = scale * d_table[id[n] - first], a row of zeros where the id is not one of this rank's (other ranks', padding's: any).
 * stride_table is that of d_table, stride_dtokens that of d_out. */
int ze_embedding(const struct ze_form* form, const void* d_ids, const void* d_table, void* d_out, void* stream);

/* d_dtable[v] = scale * (the sum of d_dout[n] over the tokens with id[n] = first + v), zeros where there is none; with
 * `accumulate` added to what d_dtable holds (rows that no token has stay as they are, and are not read).  The sum is taken in the order of
 * the tokens, cut into pieces at places that depend on the ids alone.  stride_tokens is that of d_dout. */
size_t ze_embedding_work_bytes(const struct ze_form* form);
int ze_embedding_backward(const struct ze_form* form, const void* d_ids, const void* d_dout, void* d_dtable, int accumulate,
                          void* d_work, size_t work_bytes, void* stream);

/*
 * Softmax cross entropy of hidden states h against the output matrix w,
 *
 *     l[n][v] = scale * h[n] . w[v]      loss[n] = log(sum over the whole vocabulary of exp(l[n][v])) - l[n][label[n]]
 *
 * in three calls.  The logits are made tile by tile and not kept.  A token whose label is negative has no part in any of it, whatever its
 * hidden state holds: loss, lse and gradients are 0, and nothing is computed for it.  cols >= 1.
 *
 * ze_vocab_loss leaves what this rank's rows have of it in d_stats, three arrays of `tokens` floats: the greatest logit m (-inf
 * without rows), the sum of exp(l - m), and the label's logit (-inf where the label is not one of this rank's). A
 * token without a label gets -inf, 0, 0.  A logit of +inf counts as not a number.
 *
 * How much workspace a call needs depends on whether d_hidden and d_table can be read as they are (rows that start at multiples of 4 bytes; the
 * table's, that do not overlap) or have to be copied; ze_loss_work_bytes and ze_loss_backward_work_bytes look at the pointers'
 * values for that, and give enough for any place where one is NULL.  The forward call keeps 8 bytes for each token and 16 to 128 rows.
 */
size_t ze_loss_work_bytes(const struct ze_form* form, const void* d_hidden, const void* d_table);
int ze_vocab_loss(const struct ze_form* form, const void* d_hidden, const void* d_table, const void* d_labels, float* d_stats,
                  void* d_work, size_t work_bytes, void* stream);

/* Joins the d_stats of all ranks, [ranks][3][tokens]: d_lse[n], the logarithm of the sum, and d_loss[n].  A label that is no rank's gives a
 * loss of +inf.  d_loss may be NULL. */
int ze_join_loss(size_t tokens, int ranks, int id_dtype, const float* d_stats, const void* d_labels, float* d_loss, float* d_lse, void* stream);

/* From d_lse and the gradient of the losses, with g[n][v] = dloss[n] (exp(l[n][v] - lse[n]) - (first + v == label[n])),
 *
 *     d_dhidden[n] = scale * sum over this rank's v of g[n][v] w[v]      d_dtable[v] = scale * sum over n of g[n][v] h[n]
 *
 * both of type dtype.  The first is this rank's part, to be added up over the ranks.  The logits are made anew, in pieces of the vocabulary:
 * `piece` rows at a time, 0 for the library's choice (at least 4096 and as many as keep g below 128 Mi values).
 * g / max |dloss| of a piece lies in the workspace in type dtype: half-precision products take half-precision operands, so each g is rounded once more
 * (fp16: times 2^15, so that small probabilities stay normal numbers; what is below 2^-40 max |dloss| is lost).
 * Either output may be NULL if it is not wanted. */
size_t ze_loss_backward_work_bytes(const struct ze_form* form, const void* d_hidden, const void* d_table, size_t piece);
int ze_vocab_loss_backward(const struct ze_form* form, const void* d_hidden, const void* d_table, const void* d_labels, const float* d_lse,
                           const float* d_dloss, void* d_dhidden, void* d_dtable, size_t piece, void* d_work, size_t work_bytes, void* stream);

#ifdef __cplusplus
}
#endif
#endif /* ZE_H */
