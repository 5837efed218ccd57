// C entry points of include/tokens.h: checks of the arguments, then the launches.
#include "run_internal.h"
#include "tokens_internal.h"

#include <cmath>

using namespace sl;

namespace {

constexpr float FACTOR_MIN = 0x1p-40f, FACTOR_MAX = 0x1p40f;   // their quotients, and slopes over them, stay within float32

bool dtype_ok(int dt) { return dt == DT_F32 || dt == DT_BF16; }
// rows of `cols` elements that 16-byte accesses reach
bool matrix_ok(const void* p, int dt, int64_t ld, int64_t cols) {
  return p && ((uintptr_t)p & 15) == 0 && ld >= cols && ld <= TOK_LD_MAX && ld % (16 / (int64_t)elem_size(dt)) == 0;
}
bool aligned(const void* p, unsigned n) { return ((uintptr_t)p & (n - 1)) == 0; }
int work_ok(const void* work, size_t have, size_t need) {
  if (!work || have < need) return SLIDE_EARENA;
  return aligned(work, 256) ? SLIDE_OK : SLIDE_EINVAL;
}
int status(hipError_t e) {
  if (e == hipSuccess) return SLIDE_OK;
  g_last_hip = (int)e;
  return SLIDE_EHIP;
}

int rope_ok(const slide_head_rope* s) {
  if (!s || s->rows < 1 || s->rows > TOK_ROWS_MAX || s->heads_q < 1 || s->heads_q > 4096 || s->heads_k < 0 || s->heads_k > 4096 || s->head_dim < 1 ||
      !dtype_ok(s->dtype) || s->axes < 0 || s->axes > 3 || (s->pairing != SLIDE_ROPE_HALVES && s->pairing != SLIDE_ROPE_NEIGHBOURS) ||
      !(s->eps > 0.f) || !std::isfinite(s->eps) || !(s->theta >= 1.0) || !std::isfinite(s->theta))
    return SLIDE_EINVAL;
  int64_t pairs = 0;
  for (int a = 0; a < s->axes; ++a) {
    if (s->pairs[a] < 0) return SLIDE_EINVAL;
    pairs += s->pairs[a];
  }
  if (2 * pairs > s->head_dim) return SLIDE_EINVAL;
  return s->head_dim % 16 || s->head_dim > 2 * ROPE_PAIRS ? SLIDE_EUNSUPPORTED : SLIDE_OK;
}
HeadRope rope_of(const slide_head_rope& s, unsigned long long (&freq)[ROPE_PAIRS]) {
  HeadRope g{};
  g.freq = freq;
  g.rows = s.rows; g.hq = s.heads_q; g.hk = s.heads_k; g.dim = s.head_dim; g.axes = s.axes; g.neighbours = s.pairing; g.eps = s.eps;
  int at = 0;
  for (int a = 0; a < s.axes; ++a) {
    const int n = s.pairs[a];
    // theta^(-j / n) / 2 pi, below a sixth, as a fraction of 2^64, 64-bit mantissas: every eighth by itself, the others by products with the ratio
    // (2 us for 32 exponentials, a sixth of a small call)
    const long double step = n ? -std::log((long double)s.theta) / n : 0, ratio = std::exp(step);
    long double turns = 0;
    for (int j = 0; j < n; ++j) {
      turns = j % 8 == 0 ? std::exp(step * j) * 0.159154943091895335768883763372514362L : turns * ratio;
      freq[at++] = (unsigned long long)(turns * 18446744073709551616.0L);
    }
    if (a < 2) g.bound[a] = at;
  }
  for (int a = s.axes; a < 2; ++a) g.bound[a] = at;
  return g;
}

int attn_ok(const slide_tokens_attn* s) {
  if (!s || s->rows_q < 1 || s->rows_q > TOK_ROWS_MAX || s->rows_k < 1 || s->rows_k > TOK_ROWS_MAX || s->docs < 1 || s->docs > (1 << 20) ||
      s->heads_q < 1 || s->heads_q > 4096 || s->heads_k < 1 || s->heads_q % s->heads_k || s->head_dim < 1 || !dtype_ok(s->dtype) || s->lead_q < 0 ||
      s->lead_k < 0 || !(s->scale >= FACTOR_MIN && s->scale <= FACTOR_MAX) || !(s->cap == 0.f || (s->cap >= FACTOR_MIN && s->cap <= FACTOR_MAX)) || s->reserved != 0)
    return SLIDE_EINVAL;
  const int64_t group = s->heads_q / s->heads_k;
  if (s->head_dim % 16 || s->head_dim > 128 || group > 128) return SLIDE_EUNSUPPORTED;
  // packed columns are counted in 32 bits
  if (s->rows_q * group > TOK_ROWS_MAX) return SLIDE_EUNSUPPORTED;
  return SLIDE_OK;
}
size_t up256(size_t n) { return (n + 255) / 256 * 256; }
// Work space of a pass: the slides' table, the shared tiles, their parts and what goes with them (maxima and sums, sums of P k and the errors of delta, or
// the values' parts).  The
// backward's passes follow one another in the same place, behind the deltas.
struct PassWork { size_t joins, part, part2, part3, bytes; };
PassWork pass_work(const slide_tokens_attn& s, int pass, TokCut c) {
  const size_t part = up256(tok_columns(c) * s.head_dim * 4);
  PassWork w;
  w.joins = up256(tok_table_bytes(s.docs));
  w.part = w.joins + up256(tok_joins_bytes(c));
  w.part2 = w.part + part;
  w.part3 = w.part2 + (pass == TOK_FWD ? up256(tok_columns(c) * 8) : part);
  w.bytes = w.part3 + (pass == TOK_DQ ? up256(tok_columns(c) * 4) : 0);
  return w;
}
// for a call with a bias and for one without
size_t pass_bytes(const slide_tokens_attn& s, int pass) {
  const size_t a = pass_work(s, pass, tok_cut(pass, s, false)).bytes, b = pass_work(s, pass, tok_cut(pass, s, true)).bytes;
  return a > b ? a : b;
}
size_t delta_bytes(const slide_tokens_attn& s) { return up256((size_t)s.rows_q * s.heads_q * 4); }
size_t bwd_bytes(const slide_tokens_attn& s) {
  const size_t a = pass_bytes(s, TOK_DQ), b = pass_bytes(s, TOK_DKV);
  return delta_bytes(s) + (a > b ? a : b);
}
hipError_t run_pass(int pass, const slide_tokens_attn& s, TokAttn g, char* work, hipStream_t st) {
  const TokCut c = tok_cut(pass, s, g.slopes != nullptr);
  const PassWork w = pass_work(s, pass, c);
  g.table = (const long long*)work; g.joins = work + w.joins; g.part = (float*)(work + w.part); g.part2 = (float*)(work + w.part2); g.part3 = (float*)(work + w.part3);
  hipError_t e = launch_tok_table(pass, s.dtype, g, c, (long long*)work, st);
  if (e != hipSuccess) return e;
  e = pass == TOK_FWD ? launch_tok_fwd(s.dtype, g, c, st) : pass == TOK_DQ ? launch_tok_dq(s.dtype, g, c, st) : launch_tok_dkv(s.dtype, g, c, st);
  return e != hipSuccess ? e : launch_tok_join(pass, s.dtype, g, c, st);
}
// pos_q, pos_k, slopes: all or none
bool bias_ok(const float* a, const float* b, const float* slopes) {
  if (!a && !b && !slopes) return true;
  return a && b && slopes && aligned(a, 8) && aligned(b, 8) && aligned(slopes, 4);
}
TokAttn attn_of(const slide_tokens_attn& s) {
  TokAttn g{};
  g.rows_q = (int)s.rows_q; g.rows_k = (int)s.rows_k; g.docs = s.docs; g.hq = s.heads_q; g.hk = s.heads_k; g.group = s.heads_q / s.heads_k;
  g.dim = s.head_dim; g.lead_q = s.lead_q; g.lead_k = s.lead_k; g.scale = s.scale; g.cap = s.cap;
  return g;
}

}  // namespace

extern "C" {

int slide_head_rope_fwd(const slide_head_rope* s, const void* q, int64_t ldq, const void* k, int64_t ldk, const float* gq,
                        const float* gk, const int32_t* pos, void* yq, int64_t ldyq, void* yk, int64_t ldyk, void* stream) {
  const int rc = rope_ok(s);
  if (rc) return rc;
  const int64_t cq = (int64_t)s->heads_q * s->head_dim, ck = (int64_t)s->heads_k * s->head_dim;
  if (!matrix_ok(q, s->dtype, ldq, cq) || !matrix_ok(yq, s->dtype, ldyq, cq) || (yq == q && ldyq != ldq) || !aligned(gq, 16)) return SLIDE_EINVAL;
  if (s->heads_k ? !matrix_ok(k, s->dtype, ldk, ck) || !matrix_ok(yk, s->dtype, ldyk, ck) || (yk == k && ldyk != ldk) || yk == yq || yk == q || yq == k || !aligned(gk, 16)
                 : k || yk || gk)
    return SLIDE_EINVAL;
  if (s->axes ? !pos || !aligned(pos, 4) : pos != nullptr) return SLIDE_EINVAL;
  (void)hipGetLastError();
  unsigned long long freq[ROPE_PAIRS] = {};
  HeadRope g = rope_of(*s, freq);
  g.q = q; g.ldq = ldq; g.k = k; g.ldk = ldk; g.gq = gq; g.gk = gk; g.pos = pos; g.yq = yq; g.ldyq = ldyq; g.yk = yk; g.ldyk = ldyk;
  return status(launch_head_rope_fwd(s->dtype, g, (hipStream_t)stream));
}

size_t slide_head_rope_workspace_bytes(const slide_head_rope* s) { return rope_ok(s) == SLIDE_OK ? head_rope_work_bytes(*s) : 0; }

int slide_head_rope_bwd(const slide_head_rope* s, const void* dyq, int64_t lddyq, const void* dyk, int64_t lddyk, const void* q,
                        int64_t ldq, const void* k, int64_t ldk, const float* gq, const float* gk, const int32_t* pos, void* dq,
                        int64_t lddq, void* dk, int64_t lddk, float* dgq, float* dgk, int accumulate, void* work,
                        size_t work_bytes, void* stream) {
  int rc = rope_ok(s);
  if (rc) return rc;
  const int64_t cq = (int64_t)s->heads_q * s->head_dim, ck = (int64_t)s->heads_k * s->head_dim;
  if (!matrix_ok(dyq, s->dtype, lddyq, cq) || !matrix_ok(dq, s->dtype, lddq, cq) || (dq == dyq && lddq != lddyq)) return SLIDE_EINVAL;
  if (gq ? !matrix_ok(q, s->dtype, ldq, cq) || !aligned(gq, 16) || !dgq || !aligned(dgq, 4) || dq == q : dgq != nullptr) return SLIDE_EINVAL;
  if (s->heads_k) {
    if (!matrix_ok(dyk, s->dtype, lddyk, ck) || !matrix_ok(dk, s->dtype, lddk, ck) || (dk == dyk && lddk != lddyk) || dk == dq ||
        dk == dyq || dq == dyk || (gq && dk == q) || (gk && dq == k))
      return SLIDE_EINVAL;
    if (gk ? !matrix_ok(k, s->dtype, ldk, ck) || !aligned(gk, 16) || !dgk || !aligned(dgk, 4) || dk == k || dgk == dgq : dgk != nullptr) return SLIDE_EINVAL;
  } else if (dyk || dk || k || gk || dgk) {
    return SLIDE_EINVAL;
  }
  if (s->axes ? !pos || !aligned(pos, 4) : pos != nullptr) return SLIDE_EINVAL;
  rc = work_ok(work, work_bytes, head_rope_work_bytes(*s));
  if (rc) return rc;
  (void)hipGetLastError();
  unsigned long long freq[ROPE_PAIRS] = {};
  HeadRope g = rope_of(*s, freq);
  g.dyq = dyq; g.lddyq = lddyq; g.dyk = dyk; g.lddyk = lddyk; g.q = q; g.ldq = ldq; g.k = k; g.ldk = ldk; g.gq = gq; g.gk = gk; g.pos = pos;
  g.yq = dq; g.ldyq = lddq; g.yk = dk; g.ldyk = lddk; g.dgq = dgq; g.dgk = dgk; g.accumulate = accumulate != 0; g.work = (float*)work;
  return status(launch_head_rope_bwd(s->dtype, g, (hipStream_t)stream));
}

size_t slide_tokens_attn_workspace_bytes(const slide_tokens_attn* s, int backward) {
  if (attn_ok(s) != SLIDE_OK) return 0;
  const size_t f = pass_bytes(*s, TOK_FWD), b = backward ? bwd_bytes(*s) : 0;
  return b > f ? b : f;
}

int slide_tokens_attn_fwd(const slide_tokens_attn* s, const void* q, int64_t ldq, const void* k, int64_t ldk, const void* v,
                          int64_t ldv, const int32_t* q_start, const int32_t* k_start, const float* pos_q, const float* pos_k,
                          const float* slopes, void* o, int64_t ldo, float* lse, void* work, size_t work_bytes, void* stream) {
  int rc = attn_ok(s);
  if (rc) return rc;
  const int64_t cq = (int64_t)s->heads_q * s->head_dim, ck = (int64_t)s->heads_k * s->head_dim;
  if (!matrix_ok(q, s->dtype, ldq, cq) || !matrix_ok(k, s->dtype, ldk, ck) || !matrix_ok(v, s->dtype, ldv, ck) || !matrix_ok(o, s->dtype, ldo, cq) ||
      !q_start || !k_start || !aligned(q_start, 4) || !aligned(k_start, 4) || !lse || !aligned(lse, 4) || !bias_ok(pos_q, pos_k, slopes) || o == q || o == k || o == v)
    return SLIDE_EINVAL;
  rc = work_ok(work, work_bytes, pass_bytes(*s, TOK_FWD));
  if (rc) return rc;
  (void)hipGetLastError();
  TokAttn g = attn_of(*s);
  g.q = q; g.ldq = (int)ldq; g.k = k; g.ldk = (int)ldk; g.v = v; g.ldv = (int)ldv; g.q_start = q_start; g.k_start = k_start;
  g.pos_q = pos_q; g.pos_k = pos_k; g.slopes = slopes; g.o = o; g.ldo = (int)ldo; g.lse = lse;
  return status(run_pass(TOK_FWD, *s, g, (char*)work, (hipStream_t)stream));
}

int slide_tokens_attn_bwd(const slide_tokens_attn* s, const void* dout, int64_t lddo, const void* q, int64_t ldq, const void* k,
                          int64_t ldk, const void* v, int64_t ldv, const void* o, int64_t ldo, const float* lse,
                          const int32_t* q_start, const int32_t* k_start, const float* pos_q, const float* pos_k,
                          const float* slopes, void* dq, int64_t lddq, void* dk, int64_t lddk, void* dv, int64_t lddv, void* work,
                          size_t work_bytes, void* stream) {
  int rc = attn_ok(s);
  if (rc) return rc;
  const int64_t cq = (int64_t)s->heads_q * s->head_dim, ck = (int64_t)s->heads_k * s->head_dim;
  const int dt = s->dtype;
  if (!matrix_ok(dout, dt, lddo, cq) || !matrix_ok(q, dt, ldq, cq) || !matrix_ok(k, dt, ldk, ck) || !matrix_ok(v, dt, ldv, ck) || !matrix_ok(o, dt, ldo, cq) ||
      !matrix_ok(dq, dt, lddq, cq) || !matrix_ok(dk, dt, lddk, ck) || !matrix_ok(dv, dt, lddv, ck) || !lse || !aligned(lse, 4) || !q_start || !k_start ||
      !aligned(q_start, 4) || !aligned(k_start, 4) || !bias_ok(pos_q, pos_k, slopes))
    return SLIDE_EINVAL;
  const void* const in[5] = {dout, q, k, v, o};
  for (const void* p : in)
    if (p == dq || p == dk || p == dv) return SLIDE_EINVAL;
  if (dq == dk || dq == dv || dk == dv) return SLIDE_EINVAL;
  rc = work_ok(work, work_bytes, bwd_bytes(*s));
  if (rc) return rc;
  (void)hipGetLastError();
  const hipStream_t st = (hipStream_t)stream;
  TokAttn g = attn_of(*s);
  g.q = q; g.ldq = (int)ldq; g.k = k; g.ldk = (int)ldk; g.v = v; g.ldv = (int)ldv; g.o_in = o; g.ldo = (int)ldo; g.dout = dout; g.lddo = (int)lddo;
  g.q_start = q_start; g.k_start = k_start; g.pos_q = pos_q; g.pos_k = pos_k; g.slopes = slopes; g.lse = const_cast<float*>(lse);
  g.dq = dq; g.lddq = (int)lddq; g.dk = dk; g.lddk = (int)lddk; g.dv = dv; g.lddv = (int)lddv;
  g.delta = (float*)work;
  char* const rest = (char*)work + delta_bytes(*s);
  hipError_t e = run_pass(TOK_DQ, *s, g, rest, st);
  if (e == hipSuccess) e = run_pass(TOK_DKV, *s, g, rest, st);
  return status(e);
}

}  // extern "C"
