/*
 * cos_draft.h -- C ABI of the proposer's operators for NVIDIA B200 (sm_100a), in the library of cos_verify.h.
 *
 * What stands before and behind a verification: a draft token is drawn from the proposer's
 * logits (cos_sample), and a proposer learns to have more of its drafts accepted from the
 * largest logits of the models it is verified against (cos_top_logits, cos_distill).
 *
 * All pointers are DEVICE pointers owned by the caller.  Every function enqueues one launch (two for
 * cos_distill_loss and cos_distill_step) on `cuda_stream`, on the device named in its arguments (the calling thread's current device stays as it
 * is), allocates nothing, keeps nothing between calls and returns without waiting; calls on any
 * number of streams may overlap, and a call may be captured into a CUDA graph.  Problems the host can
 * see are returned (the reason is in cos_verify_last_error(NULL)) and nothing is enqueued then;
 * problems of the data are reported row by row.
 */
#ifndef COS_DRAFT_H
#define COS_DRAFT_H

#include "cos_verify.h"

#ifdef __cplusplus
extern "C" {
#endif

#define COS_DISTILL_STATISTICS 8 /* floats of a row beside its lists' shares */
#define COS_TOP_MAX 1024 /* most entries cos_top_logits lists for a row, and cos_distill takes for one */

typedef struct {
  const void* logits;     /* [rows][vocab], element (r, x) at r * stride_row + x (in elements)          */
  int64_t stride_row;     /* >= vocab where rows > 1, or 0: all rows are the same one                   */
  int32_t rows, vocab;    /* >= 1                                                                       */
  int32_t dtype;          /* COS_DTYPE_* of the logits                                                  */
  int32_t device;         /* CUDA device ordinal                                                        */
  const float* uniforms;  /* [rows], in [0, 1): u of the row's draw (outside: taken to the next bound)  */
  /* the parameters of every row, or, where the pointer is not NULL, of each row ([rows])               */
  float temperature;      /* T >= 0; 0: the largest logit, the lowest index among equals                */
  int32_t top_k;          /* <= 0: no limit                                                             */
  float top_p;            /* >= 1: no limit; else > 0                                                   */
  float min_p;            /* in [0, 1]; 0: no limit                                                     */
  const float* row_temperature;
  const int32_t* row_top_k;
  const float* row_top_p; /* entries below 0 count as 0 (the most likely token alone is kept)           */
  const float* row_min_p; /* entries outside [0, 1] count as the next bound                             */
  int32_t* tokens;        /* out [rows]: the token, -1 where the row has none                           */
  float* prob;            /* optional out [rows]: its probability under the law it was drawn from; NaN  */
                          /* where there is no token                                                    */
  int32_t* kept;          /* optional out [rows]: how many tokens that law is made of                   */
  uint32_t* row_status;   /* optional out [rows]: COS_ROW_NONFINITE where the row holds a NaN or +inf,  */
                          /* where it holds nothing but -inf, and where its temperature is negative or  */
                          /* NaN                                                                        */
  void* filtered;         /* optional out [rows][vocab], of the logits' type: the logits of the tokens  */
                          /* that were kept, -inf elsewhere (rows without a token are copied as they    */
                          /* are): the logits whose softmax at T is the law of the draw, which a        */
                          /* verification takes as the proposer's.  May be `logits` itself with the     */
                          /* same stride; must not overlap them otherwise                               */
  int64_t stride_filtered;
} cos_sample_args;

/*
 * Draw a token for every row.  With w(x) = exp((l(x) - max l) / T), tokens in order of their logits (the lowest index first
 * among equals; +0 and -0 are equal, -inf is no token):
 *   top-k   the first top_k of them are kept;
 *   top-p   of these, a token is kept while the w of those before it sum to less than top_p times the sum over what top-k
 *           kept (so the first one always is);
 *   min-p   of these, a token is kept where w(x) >= min_p.
 * The draw is the inverse of the cumulative sum in order of the index: the lowest kept x with sum_{y <= x} w(y) >= u * S.
 * Weights are evaluated in 64 bits (those below 2^-36 of the largest one in 32, to 2^-17 of themselves) and summed as whole
 * multiples of 2^-(63 - ceil(log2 vocab)) (2^-46 at the least) of the largest one, so sums do not depend on any order: two calls
 * on the same inputs agree bit by bit.
 */
cos_status cos_sample(const cos_sample_args* args, void* cuda_stream);

typedef struct {
  const void* logits; /* as in cos_sample_args */
  int64_t stride_row;
  int32_t rows, vocab;
  int32_t dtype;
  int32_t device;
  int32_t k;          /* 1 .. min(COS_TOP_MAX, vocab)                                                   */
  double temperature; /* T > 0: of the log-sum-exp only                                                 */
  float* values;      /* out [rows][k]: the k largest logits, the largest first, the lowest index first */
                      /* among equals; -inf where the row has fewer tokens                              */
  int32_t* ids;       /* out [rows][k]: their tokens, -1 where there is none                            */
  float* lse;         /* out [rows]: ln sum_x exp(l(x) / T); -inf where every logit is -inf.  A row     */
                      /* with a NaN or +inf has NaN here, and lists nothing                             */
} cos_top_args;

/* The k largest logits of every row and the log-sum-exp behind its softmax: what cos_distill reads of a teacher. */
cos_status cos_top_logits(const cos_top_args* args, void* cuda_stream);

typedef struct {
  const void* student;    /* [rows][vocab] logits, element (n, x) at n * stride_student + x             */
  int64_t stride_student; /* >= vocab where rows > 1, or 0: all rows are the same one                   */
  int32_t rows, vocab;    /* >= 1                                                                       */
  int32_t dtype;          /* COS_DTYPE_* of the student's logits and of their gradient                  */
  int32_t device;         /* CUDA device ordinal                                                        */
  int32_t lists;          /* 1..COS_MAX_MODELS: teachers                                                */
  int32_t k;              /* entries of a list; lists * k <= COS_TOP_MAX                                */
  const int32_t* ids;     /* [rows][lists][k]: tokens; a negative one is an empty entry.  A token may   */
                          /* come up any number of times: its shares add up.  One >= vocab makes the    */
                          /* row's loss and gradient NaN                                                */
  const float* values;    /* [rows][lists][k]: the teachers' logits of these tokens; -inf: empty        */
  const float* lse;       /* [rows][lists]: ln sum_x exp(v(x) / T) of each teacher over its whole       */
                          /* vocabulary: shares are the teacher's probabilities, what is not listed is  */
                          /* left out.  NULL: shares are the softmax over the list                      */
  float weights[COS_MAX_MODELS]; /* >= 0, of the lists (Eq. 4)                                          */
  double temperature;     /* T > 0, of teachers and student                                             */
  const float* row_weights; /* [rows]: what the loss of each row counts in the sum whose gradient is    */
                          /* wanted; rows of weight 0 have gradient 0 whatever they hold                */
  float* loss;            /* out [rows] */
  float* statistics;      /* rows * (COS_DISTILL_STATISTICS + lists * k) floats, 16-byte aligned: what  */
                          /* cos_distill_loss leaves for cos_distill_grad; cos_distill_step's own       */
  void* grad;             /* out [rows][vocab], of the student's type; may be `student` itself with the */
                          /* same stride; must not overlap it otherwise                                 */
  int64_t stride_grad;
} cos_distill_args;

/*
 * Distillation of a student (the proposer) from the largest logits of its teachers (the models its drafts are verified against).  With the
 * target t(x) = sum_g w_g p_g(x) over the listed tokens, p_g(x) = exp(v(x) / T - lse_g), and q = softmax(s / T):
 *   loss = sum_x t(x) (ln t(x) - ln q(x)),   gradient = row_weight / T * (P q(x) - t(x)),  P = sum_x t(x).
 * +inf where a token with a share has the logit -inf.  A row without a share (padding) has loss 0 and gradient 0 whatever its logits are; the first rows of a call may be read
 * before that is known, so `student` has to hold all of them.  A teacher whose row holds a NaN or +inf lists nothing (cos_top_logits) and counts as one that is absent: its share of the
 * target is missing, or the row is padding where no other teacher lists anything.  Its lse tells it, which is not looked at here where no entry refers to it.
 *   cos_distill_loss  loss and statistics (row_weights, grad are not looked at)
 *   cos_distill_grad  the gradient, from the statistics of the same student, lists and T (loss is not looked at)
 *   cos_distill_step  loss and gradient, reading the student once
 */
cos_status cos_distill_loss(const cos_distill_args* args, void* cuda_stream);
cos_status cos_distill_grad(const cos_distill_args* args, void* cuda_stream);
cos_status cos_distill_step(const cos_distill_args* args, void* cuda_stream);

#ifdef __cplusplus
}
#endif

#endif /* COS_DRAFT_H */
