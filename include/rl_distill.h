/*
 * rl_distill.h - C ABI of scoring with top alternatives and of distillation from a teacher's top entries (MI355X / gfx950).
 *
 * Both run on the LM head of rl_policy.h, z_t = W x_t, q_t = softmax(z_t / temperature), never with more than a chunk of the logits in memory:
 *   rl_token_top_logprobs    log q_t of a given token, logsumexp, entropy and the K most probable tokens with their log-probabilities
 *   rl_distill_loss_fwd_bwd  for every row a list of up to K entries (token, log-probability) of a teacher, as the first call writes it; the
 *                            Kullback-Leibler divergence from the teacher to q_t, its loss over the batch and the gradients of hidden and weight
 *
 * Conventions are those of rl_policy.h: device pointers owned by the caller, nothing allocated, kept or synchronised, all work on `stream`,
 * host-checkable errors returned before anything is launched, rows that do not count (mask, sequences, data errors) read 0, results the same
 * bits every run.  Of rl_batch they read R, H, V, B, dtype, hidden, weight, mask, cu_seqlens and, the first one, token_ids.
 * No output may overlap an input or another output (RL_ERR_RANGE), but d_hidden may be hidden.
 */
#ifndef RL_DISTILL_H
#define RL_DISTILL_H

#include "rl_policy.h"

#ifdef __cplusplus
extern "C" {
#endif

#define RL_TOP_MAX_K 128          /* most alternatives, or entries of a list   */
#define RL_TOP_MAX_V 524288       /* largest vocabulary of these two calls     */

typedef struct rl_top_params {
  int32_t top_k;                  /* alternatives, 1 <= top_k <= min(RL_TOP_MAX_K, V)                             */
  int32_t chunk_rows;             /* rows whose logits are held at once (4 bytes per row and vocabulary entry);   */
                                  /* 0 = rl_default_chunk_rows_distill; rounded up to a multiple of 256, 2^20 at most */
  float   temperature;            /* 0 = 1.0; otherwise 4.3e-39 to 3e38 (log2(e) / temperature is finite in f32)  */
} rl_top_params;

typedef struct rl_top_outputs {   /* NULL = not wanted; one at least                                              */
  float*   logprob;               /* [R]  log q_t[token_ids[t]]; needs token_ids, which may be NULL without it    */
  float*   lse;                   /* [R]  logsumexp of z / temperature                                            */
  float*   entropy;               /* [R]  a logit of -inf has probability 0 and no part in it                       */
  int32_t* top_ids;               /* [R, top_k]  the most probable tokens, most probable first; among equal logits the lower token first; */
                                  /*             -1 on rows that do not count, and where a row's logits are not numbers                   */
  float*   top_logprob;           /* [R, top_k]  their log-probabilities; 0 on rows that do not count             */
} rl_top_outputs;

/* Logits are added up in f32; "most probable" is by these values.  A row whose token is outside [0, V) does not count. */
rl_status rl_token_top_logprobs_workspace_bytes(const rl_batch* batch, const rl_top_params* params, size_t* bytes);
rl_status rl_token_top_logprobs(const rl_batch* batch, const rl_top_params* params, const rl_top_outputs* outputs,
                                void* workspace, size_t workspace_bytes, void* stream);

/* What stands for the tokens that a teacher's list does not name. */
typedef enum rl_distill_rest {
  RL_REST_BUCKET = 0,             /* one entry for all of them, with the probability that the list leaves: p_r = max(0, 1 - sum p_i)      */
  RL_REST_RENORMALISE = 1         /* nothing: the p_i are divided by their sum (log-probabilities or logits will do)                      */
} rl_distill_rest;

/* p_i = exp(teacher_logprob) of the entries i of a row's list.  An entry whose token is -1 is none; one outside [0, V), or whose token an earlier
 * entry of the row has, is left out and counted (n_bad_entry).  With q_r the probability of all tokens that the list does not name,
 *     KL_t = sum_i p_i (log p_i - log q_t[i]) + p_r (log p_r - log q_r)        (terms of p = 0 are 0; p_r = 0 where the list names all tokens)
 *     loss = scale sum_t c_t KL_t,    c_t = 1 / (B |y_i|) (RL_AGG_SEQUENCE: mean over the B sequences of the mean over a sequence's rows)
 *                                       or 1 / T (RL_AGG_TOKEN)
 *     dS[t,v] = scale c_t / temperature (P q_t[v] - p_v) for listed v, scale c_t / temperature q_t[v] (P - p_r / q_r) for others,  P = sum p_i + p_r
 * and d_hidden = dS W, d_weight = dS^T X.  A row with an empty list, or whose entries all have p = 0 under RL_REST_RENORMALISE, counts with
 * KL_t = 0 and no gradient, whatever its hidden states or the weight hold. */
typedef struct rl_distill_params {
  int32_t top_k;                  /* length of the lists, 1 <= top_k <= RL_TOP_MAX_K                              */
  int32_t rest;                   /* rl_distill_rest                                                              */
  int32_t aggregation;            /* rl_aggregation                                                               */
  int32_t chunk_rows;             /* as above; sizes the workspace                                                */
  float   temperature;            /* of the student, as above; the lists are taken as they are                    */
  float   scale;                  /* 0 = 1.0; otherwise finite                                                    */
  int32_t d_weight_dtype;         /* rl_dtype of d_weight: RL_F32, or RL_BF16 with bf16 inputs (else RL_ERR_DTYPE)  */
} rl_distill_params;

typedef struct rl_distill_stats { /* device struct                                                                */
  int32_t n_tokens;               /* rows that counted (T)                                                        */
  int32_t n_bad_entry;            /* entries left out: token outside [0, V) (but -1), or named before             */
  int32_t n_empty_row;            /* rows that counted with KL_t = 0 for want of entries                          */
  int32_t n_bad_seq;              /* sequences treated as empty                                                   */
} rl_distill_stats;

typedef struct rl_distill_outputs { /* NULL = not wanted, except loss                                             */
  float* loss;                    /* [1]                                                                          */
  float* row_loss;                /* [R]  KL_t                                                                    */
  float* lse;                     /* [R]  logsumexp of the student's z / temperature                              */
  void*  d_hidden;                /* [R,H] in dtype; d_hidden and d_weight NULL together skips the backward       */
  void*  d_weight;                /* [V,H] in d_weight_dtype, overwritten (may start at any element)              */
  rl_distill_stats* stats;        /* [1]                                                                          */
} rl_distill_outputs;

/* teacher_ids, teacher_logprob: [R, top_k].  With bf16 inputs dS is staged in bf16, rounded once, and both gradients are added up in f32; chunks add
 * to d_weight in f32, which is rounded once if it leaves in bf16. */
rl_status rl_distill_workspace_bytes(const rl_batch* batch, const rl_distill_params* params, int32_t want_backward, size_t* bytes);
rl_status rl_distill_loss_fwd_bwd(const rl_batch* batch, const int32_t* teacher_ids, const float* teacher_logprob,
                                  const rl_distill_params* params, const rl_distill_outputs* outputs,
                                  void* workspace, size_t workspace_bytes, void* stream);

/* Chunk size used when chunk_rows = 0. */
int32_t rl_default_chunk_rows_distill(void);

#ifdef __cplusplus
}
#endif
#endif /* RL_DISTILL_H */
