/*
 * grumpy_hip_attention.h -- attention and rotary positions beside the lazy arrays of grumpy_hip.h.
 *
 * A softmax over products of rows is what the lazy arrays record as dot, max, sub, exp, sum, div, dot; fused
 * per sub-graph, the N x M scores between the two contractions still pass through memory, several times for the
 * gradient.  These calls are that program, and its gradient, as kernels that never store a score.
 *
 * Conventions, beyond those of grumpy_hip.h
 *   - Like gr_assign, the calls launch at once: operands that are still unevaluated are evaluated first, results
 *     are WRITTEN into the arrays given for them, which must be materialised arrays or slice / transpose views of
 *     some; recorded but unevaluated arrays that read that storage are evaluated first, so they keep the values
 *     they had when recorded.  Everything runs asynchronously on the context's stream.
 *   - Element types: f32 or bf16 (GR_BF16) for tensors, one type for all tensors of a call; i32 for whole numbers;
 *     f32 for lse and slopes.  bf16 arrays are leaves and views of leaves: no other call computes with them
 *     (GR_ERR_DTYPE).  Products of f32 are formed of three bf16 pieces of each value, right to 2^-24; a value that bf16 rounds
 *     to infinity (2^128 - 2^119 = 3.396e38 and more) counts as infinite and gives NaN.  Scores, probabilities, statistics and sums are
 *     f32; with bf16 tensors a probability, or a score's gradient, is rounded to bf16 where it enters the next product (not the probabilities of
 *     gr_attention with rest, nor of calls of at most 32 queries times heads per head of k).  The gradient forms
 *     probabilities from lse, which f32 holds to |lse| 2^-24, and is off by as much relatively (keys all 10^6 away from a query under a slope of 1: 6 %); and it carries sums 2^32 times as large: dv, dq / scale and dk / scale
 *     (with no part of their sums) may not pass 2^95 in size, beyond it they are infinite or NaN.
 *   - Shapes: q, out, rest, dout, dq (B, N, H, D); k, v, dk, dv (B, M, HK, D) with H a multiple of HK: head h of q reads head
 *     h / (H / HK) of k and v.  1 <= D <= 256.  Any strides, as long as the D values of a row are neighbours
 *     (GR_ERR_UNSUPPORTED otherwise); rows of whole, aligned 16-byte vectors are the fast ones.
 *   - Results may be views of one buffer (the three parts of a packed gradient) but must not overlap one another
 *     or an operand (GR_ERR_ALIAS); only gr_rotary may be given its operand as its result.
 *   - Temporary memory comes from the context's allocator, is kept by the context, and grows with the largest call so
 *     far.  A call whose stream is being captured into a HIP graph allocates nothing: run it once before with
 *     the same arguments, else GR_ERR_OOM.  Memory that a captured call has used stays as it is until the context
 *     goes; replays and other attention calls of that context must not overlap in time.
 *   - Results do not depend on timing: every sum is taken in an order fixed by the shapes.
 */
#ifndef GRUMPY_HIP_ATTENTION_H
#define GRUMPY_HIP_ATTENTION_H

#include "grumpy_hip.h"

#ifdef __cplusplus
extern "C" {
#endif

/* How scores are formed and which keys a query sees.  The query of row i stands at position p = position + i, key j
 * at position j (gr_attention_step: p = lengths[b] - 1).
 *   score = scale * (q . k);  capped: cap * tanh(score / cap);  then - slopes[h] * |p - j|
 *   (the distance as f32 holds it: beyond 2^24 neighbouring keys may share one)
 *   key j is seen if (not causal, or j <= p, or j < prefix[b]), and j < lengths[b], and the documents are the same
 * Rows of k and v from lengths[b] on are not read, and a score that is masked is replaced whatever it is: a k that is infinite
 * or NaN has no say in out and lse of the queries that do not see it.  (A v below lengths[b], or in the gradient a k, v, q or dout, that
 * is infinite or NaN may reach rows of its tile that do not see it, as 0 * inf does in a plain product.)
 * A query that sees a score that is NaN or +inf (which a q that is NaN makes of all) has NaN in out and lse, at every size. */
typedef struct {
  double scale;         /* 1e-28 .. 1e30 */
  double cap;           /* 0 = none; 1e-30 .. 1e30, and scale / cap 1e-37 .. 1e38 */
  gr_array slopes;      /* f32 (H), not trained: no gradient; 0 = none */
  int causal;           /* 1: a query sees keys up to its own position */
  int64_t position;     /* of query 0, -2^31 .. 2^31; with slopes no further than 2^24 from where the keys begin and end */
  gr_array prefix;      /* i32 (B): keys before it are seen by every query; 0 = none.  Only with causal */
  gr_array q_documents; /* i32 (B, N) and (B, M): a query sees keys of its own document; numbers below zero stand for */
  gr_array k_documents; /*   no document: such rows see nothing, such keys are not seen.  0, 0 = none */
  gr_array lengths;     /* i32 (B): keys there are, taken as 0 .. M; 0 = all M */
} gr_scores;

/* out = softmax(scores) v.  lse (f32 (B, H, N), C-contiguous; 0 = not wanted) gets log(sum(exp(score))) of each row; rest
 * (bf16 only; 0 = not wanted) what the rounding of out to bf16 lost.  A query that sees nothing gets out = 0,
 * lse = -inf. */
gr_status gr_attention(gr_ctx* ctx, const gr_scores* scores, gr_array q, gr_array k, gr_array v, gr_array out, gr_array lse, gr_array rest);

/* The gradients of q, k and v for the gradient `dout` of out, from out and lse of gr_attention with the same
 * scores.  rest (0 = none): makes sum(dout * out) that of the unrounded output; without it dq and dk of queries that see only a
 * few keys are off by bf16's rounding of out.  Heads that share a head of k and v add up in its dk and dv. */
gr_status gr_attention_grad(gr_ctx* ctx, const gr_scores* scores, gr_array q, gr_array k, gr_array v, gr_array out, gr_array rest, gr_array lse,
                            gr_array dout, gr_array dq, gr_array dk, gr_array dv);

/* One new token per sequence against a cache: q and out (B, H, D), k and v (B, M, HK, D) of which sequence b holds
 * lengths[b] rows, the new token's own among them.  Of the scores, scale, cap, slopes and lengths are used (lengths must be given);
 * causal, position, prefix and documents must be 0. */
gr_status gr_attention_step(gr_ctx* ctx, const gr_scores* scores, gr_array q, gr_array k, gr_array v, gr_array out);

/* Rotary positions: out = x with pair i of every head turned by the angle p * frequencies[i] and times factor,
 *   lo' = factor (lo cos - hi sin), hi' = factor (hi cos + lo sin).
 * x, out (B, N, H, D); pair i is (x[i], x[pairs + i]), or with interleaved = 1 (x[2 i], x[2 i + 1]); the D - 2 pairs
 * values behind the pairs are copied.  p = positions[b][n] (i32 (B, N), any strides), or position + n where
 * positions = 0.  frequencies: host array of `pairs` <= 256 finite doubles, radians per position, copied before the call
 * returns; angles are formed in 64 bits.  inverse = 1 turns the other way: the gradient of the same call without it.
 * out may be x itself (the same view). */
gr_status gr_rotary(gr_ctx* ctx, gr_array x, gr_array positions, int64_t position, const double* frequencies, int pairs, int interleaved, int inverse,
                    double factor, gr_array out);

#ifdef __cplusplus
}
#endif
#endif /* GRUMPY_HIP_ATTENTION_H */
