// Internal declarations of the operators over tokens (include/tokens.h; gfx950 only).
#pragma once
#include "../../include/tokens.h"
#include "slide_internal.h"

namespace sl {

constexpr int64_t TOK_LD_MAX = (1 << 21) - 1;   // 64 rows of 4-byte elements within a buffer's 32-bit offsets
constexpr int64_t TOK_ROWS_MAX = (1LL << 31) - 1 - 256;

// ---- norm and rotation of heads ------------------------------------------------------------------
constexpr int ROPE_PAIRS = 128;
struct HeadRope {
  long long rows;
  int hq, hk, dim, axes, neighbours;
  int bound[2];                       // first pair of axis 1, of axis 2
  float eps;
  const void *q, *k; long long ldq, ldk;        // forward: inputs; backward: the forward's inputs
  const void *dyq, *dyk; long long lddyq, lddyk;
  void *yq, *yk; long long ldyq, ldyk;          // outputs: values, or gradients
  const float *gq, *gk;
  const int* pos;
  float *dgq, *dgk; int accumulate;
  float* work;
  const unsigned long long* freq;               // host: a pair's turns for a step of its position, as a fraction of 2^64; [ROPE_PAIRS]
};
size_t head_rope_work_bytes(const slide_head_rope& s);
hipError_t launch_head_rope_fwd(int dt, const HeadRope& g, hipStream_t s);
hipError_t launch_head_rope_bwd(int dt, const HeadRope& g, hipStream_t s);

// ---- attention -----------------------------------------------------------------------------------
struct TokAttn {
  int rows_q, rows_k, docs, hq, hk, group, dim;
  int lead_q, lead_k;
  float scale, cap;
  const void *q, *k, *v, *o_in, *dout;
  int ldq, ldk, ldv, ldo, lddo, lddq, lddk, lddv;
  const int *q_start, *k_start;
  const float *pos_q, *pos_k, *slopes;
  void *o, *dq, *dk, *dv;
  float* lse;           // [hq][rows_q]
  float* delta;         // [hq][rows_q]: dout . o
  const long long* table;   // first units of the slides, where there are more than 64
  void* joins;              // column tiles of several workgroups
  float *part, *part2, *part3;   // their partial results: two tiles a workgroup
};
// How a pass is cut: `blocks` workgroups of `waves` wavefronts with 32 columns each (packed queries, or keys) and `heads` heads at a time
struct TokCut { int waves, blocks, heads; };
enum { TOK_FWD = 0, TOK_DQ = 1, TOK_DKV = 2 };
TokCut tok_cut(int pass, const slide_tokens_attn& s, bool bias);
inline size_t tok_table_bytes(int docs) { return docs > 64 ? ((size_t)docs + 1) * 8 : 0; }
inline size_t tok_joins_bytes(TokCut c) { return (size_t)c.blocks * 16; }
inline size_t tok_columns(TokCut c) { return (size_t)2 * c.blocks * c.waves * 32 * c.heads; }   // of partial results
// first units of the slides of a pass, where a table is used
hipError_t launch_tok_table(int pass, int dt, const TokAttn& g, TokCut c, long long* table, hipStream_t s);
hipError_t launch_tok_fwd(int dt, const TokAttn& g, TokCut c, hipStream_t s);
hipError_t launch_tok_dq(int dt, const TokAttn& g, TokCut c, hipStream_t s);
hipError_t launch_tok_dkv(int dt, const TokAttn& g, TokCut c, hipStream_t s);
// results of the column tiles that several workgroups share, out of their parts
hipError_t launch_tok_join(int pass, int dt, const TokAttn& g, TokCut c, hipStream_t s);

}  // namespace sl
