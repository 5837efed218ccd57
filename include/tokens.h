/*
 * tokens.h - C ABI of libslide for transformers over the tiles of slides: attention over packed slides, and the norms and
 * rotation of its queries and keys, each with its gradients.
 *
 * Rows are tokens: the tiles of one or many slides, one slide's rows behind the other's, class or register tokens among them.
 * Queries, keys and values are matrices [rows][heads * head_dim] of dtype, mostly column ranges of one matrix that a linear layer wrote:
 * "ld" counts elements between rows.  heads_q is a multiple of heads_k; query head h belongs to key (and value) head
 * h / (heads_q / heads_k).
 *
 * Conventions as in slide.h and act8.h: device pointers unless a comment says "host"; `hip_stream` is a hipStream_t passed as void*, of the
 * current device; every call only enqueues work and returns; the library never allocates device memory: work space is the
 * caller's, needs no clearing, is 256-byte aligned, holds nothing from one call to the next, and must not be shared by calls
 * that may run at the same time (two captured graphs that may).  Return value 0 or a negative SLIDE_E* code.  `dtype` is 0 = float32,
 * 1 = bfloat16; sums, norms, softmax statistics and angles are held in 32 bits or more, and results are the same bits on every run.
 * Matrices are 16-byte aligned and ld is a multiple of 8 (bfloat16) or 4 (float32), below 2^21.  bfloat16: products of bfloat16 operands with
 * sums in float32; probabilities and the gradients of scores are rounded to bfloat16 where they are multiplied.  Unless a comment allows it, outputs must not
 * overlap inputs or each other.
 */
#ifndef SLIDE_TOKENS_H_
#define SLIDE_TOKENS_H_

#include "slide.h"

#ifdef __cplusplus
extern "C" {
#endif

/* How columns of a head are paired for the rotation: pair p is columns p and p + head_dim / 2, or 2 p and 2 p + 1. */
#define SLIDE_ROPE_HALVES     0
#define SLIDE_ROPE_NEIGHBOURS 1

/* Norm and rotation of a head's vector x (host).  head_dim: a multiple of 16 up to 256.  axes: 0 to 3 coordinates of a position;
 * axis a has pairs[a] >= 0 pairs, those of axis 0 first, at most head_dim / 2 in all (the others are not rotated).  The j-th pair of an axis with n
 * turns by position * theta^(-j / n) radians; theta >= 1.  Angles are right to 2^-31 of a turn for every position that 32 bits hold.
 * With a gain g:  n = x / sqrt(mean(x^2) + eps) * g, eps > 0; without: n = x.  Result: n, rotated. */
typedef struct slide_head_rope {
  int64_t rows;
  int32_t heads_q, heads_k, head_dim, dtype;   /* heads_k 0: queries only, all pointers of the keys NULL */
  int32_t axes, pairing;
  int32_t pairs[3];
  float eps;
  double theta;
} slide_head_rope;

/* yq, yk = the heads of q and k, normalised where gq / gk [head_dim] float32 (16-byte aligned) is not NULL, and rotated.  pos: [rows][axes] (NULL where axes
 * is 0).  yq may be q and yk may be k (same pointer and stride). */
int slide_head_rope_fwd(const slide_head_rope* s, const void* q, int64_t ldq, const void* k, int64_t ldk, const float* gq,
                        const float* gk, const int32_t* pos, void* yq, int64_t ldyq, void* yk, int64_t ldyk, void* hip_stream);

/* Gradients: dq, dk of dtype; dgq, dgk [head_dim] float32 where the gain is not NULL (then not NULL, else NULL), written
 * (accumulate == 0) or added to.  q and k are the forward's inputs; they may be NULL where the gain is.  dq may be dyq and dk may be dyk (same pointer
 * and stride).  work: slide_head_rope_workspace_bytes(s) bytes (0 for what is refused). */
size_t slide_head_rope_workspace_bytes(const slide_head_rope* s);
int slide_head_rope_bwd(const slide_head_rope* s, const void* dyq, int64_t lddyq, const void* dyk, int64_t lddyk, const void* q,
                        int64_t ldq, const void* k, int64_t ldk, const float* gq, const float* gk, const int32_t* pos, void* dq,
                        int64_t lddq, void* dk, int64_t lddk, float* dgq, float* dgk, int accumulate, void* work,
                        size_t work_bytes, void* hip_stream);

/* Attention inside each of `docs` slides (host).  head_dim: a multiple of 16 up to 128; heads_q / heads_k up to 128, times rows_q below 2^31 - 256.
 * Row i of slide b is rows q_start[b] + i of the queries and k_start[b] + i of the keys.  Score of a query and a key of the same slide:
 *     x = scale * q.k;   where cap > 0: x = cap * tanh(x / cap);   where there are slopes: x -= slopes[head] * distance(pos_q, pos_k)
 * The first lead_q queries and lead_k keys of a slide have no place (class tokens): their distances are 0 and their positions are not used.
 * Scores are float32, right to some units of 2^-24 of their terms: a row's largest score has to be below 2^24 in size (its other ones may be as low as they like). */
typedef struct slide_tokens_attn {
  int64_t rows_q, rows_k;                      /* 1 to 2^31 - 1 - 256 */
  int32_t docs;                                /* 1 to 2^20 */
  int32_t heads_q, heads_k, head_dim, dtype;
  int32_t lead_q, lead_k;
  float scale, cap;                            /* scale, and cap where it is not 0 (none): 2^-40 to 2^40 */
  int32_t reserved;                            /* 0 */
} slide_tokens_attn;

/* For the forward, or for both directions; 0 for what is refused. */
size_t slide_tokens_attn_workspace_bytes(const slide_tokens_attn* s, int backward);

/* o [rows_q][heads_q * head_dim] = softmax(scores) v, lse [heads_q][rows_q] float32 = log of the sum of exp(scores).  A slide without keys has
 * o = 0 and lse = -infinity.  q_start, k_start: [docs + 1], not decreasing, from 0 to rows_q / rows_k; rows before the first slide and behind the last
 * one are neither read nor written.  (What does not fit is taken as if cut to that range: never out of the matrices.)
 * pos_q [rows_q][2], pos_k [rows_k][2] float32, 8-byte aligned, below 2^40 in size, and slopes [heads_q] float32, below 2^20 in size: all of them or
 * none. */
int slide_tokens_attn_fwd(const slide_tokens_attn* s, const void* q, int64_t ldq, const void* k, int64_t ldk, const void* v,
                          int64_t ldv, const int32_t* q_start, const int32_t* k_start, const float* pos_q, const float* pos_k,
                          const float* slopes, void* o, int64_t ldo, float* lse, void* work, size_t work_bytes, void* hip_stream);

/* Gradients of the queries, keys and values from the output's, dout, with the o and lse that the forward left.  Rows of slides without queries
 * (keys) have zero gradients; rows of no slide are not written.  Probabilities are made again out of lse and carry its rounding: they are off by up to
 * 2^-22 of its size, so rows' largest scores belong below 2^16.  bfloat16: the rounding of o is taken off the keys' gradients, and off the queries' in slides of
 * 256 keys or fewer. */
int slide_tokens_attn_bwd(const slide_tokens_attn* s, const void* dout, int64_t lddo, const void* q, int64_t ldq, const void* k,
                          int64_t ldk, const void* v, int64_t ldv, const void* o, int64_t ldo, const float* lse,
                          const int32_t* q_start, const int32_t* k_start, const float* pos_q, const float* pos_k,
                          const float* slopes, void* dq, int64_t lddq, void* dk, int64_t lddk, void* dv, int64_t lddv, void* work,
                          size_t work_bytes, void* hip_stream);

#ifdef __cplusplus
}
#endif
#endif /* SLIDE_TOKENS_H_ */
