// Attention over packed slides: the table of the slides' first units, and the column tiles whose rows several workgroups shared (tokens_attn.h).
#include "tokens_attn.h"

namespace sl {

namespace {

__global__ void __launch_bounds__(1024) tok_table_k(const TokSide c, const TokSide r, int docs, long long* __restrict__ table) {
  __shared__ long long sums[16];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  long long before = 0;
  for (int base = 0; base < docs; base += 1024) {
    const int i = base + threadIdx.x;
    const long long n = i < docs ? tok_units(c, r, i) : 0;
    long long v = n;
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
      const long long x = __shfl_up(v, o, 64);
      if (lane >= o) v += x;
    }
    if (lane == 63) sums[wave] = v;
    __syncthreads();
    long long all = 0;
#pragma unroll
    for (int w = 0; w < 16; ++w) {
      if (w < wave) v += sums[w];
      all += sums[w];
    }
    if (i < docs) table[i] = before + v - n;
    before += all;
    __syncthreads();
  }
  if (threadIdx.x == 0) table[docs] = before;
}

// A workgroup joins COLS columns of a tile.  A column's threads are groups of `lanes` with four of its values each, group z of them takes every
// `zs`-th piece; the groups' results meet in LDS, in their order.  blockIdx.z: the head of a group (forward), keys' or values' gradient.
// Forward: pieces are sums under references of their own.  TOK_DQ, bfloat16 (ERR): beside the sums the error of delta and, where the slide's `keys` are
// few or the wavefronts single, sums of P k to mend them with (tokens_attn_dq.hip).
struct Sum { f32x4 o, k; float m, l; };
template <int PASS>
__device__ __forceinline__ void add(Sum& a, const Sum& b, bool mend) {
  if (PASS == TOK_FWD) {
    const float n = fmaxf(a.m, b.m), ns = n == -INFINITY ? 0.f : n;
    const float wa = __builtin_amdgcn_exp2f(a.m - ns), wb = __builtin_amdgcn_exp2f(b.m - ns);
    a.m = n;
    a.l = fmaf(a.l, wa, b.l * wb);
#pragma unroll
    for (int i = 0; i < 4; ++i) a.o[i] = fmaf(a.o[i], wa, b.o[i] * wb);
  } else {
    a.o += b.o;
    if (mend) a.k += b.k;
    if (PASS == TOK_DQ) a.l += b.l;
  }
}
struct JoinOut { void* out; int ld; };
template <typename T, int W, int PASS>
__global__ void __launch_bounds__(W == 32 ? 512 : 256) tok_join_k(const TokAttn g, const TokSide side, const TokSide keys, const TokHeads hs, int hstep, int blocks,
                                                                  JoinOut out0, JoinOut out1) {
  constexpr int COLS = 8, NT = W == 32 ? 512 : 256;   // few columns mean many pieces
  constexpr bool ERR = PASS == TOK_DQ && sizeof(T) == 2;
  __shared__ f32x4 sums[NT], sums2[ERR ? NT : 1];
  __shared__ float2 stats[PASS == TOK_DKV ? 1 : NT];
  const TokJoin j = ((const TokJoin*)g.joins)[blockIdx.x];
  if (j.pieces == 0) return;
  const bool second = PASS == TOK_DKV && blockIdx.z;
  const int n = PASS == TOK_DKV ? 0 : blockIdx.z, heads = PASS == TOK_DKV ? 1 : gridDim.z;
  const float* const part = second ? g.part2 : g.part;
  const JoinOut out = second ? out1 : out0;
  const TokSpan c = tok_span(side, j.doc);
  const int first = j.tile * W + blockIdx.y * COLS, here = c.n - first < COLS ? c.n - first : COLS;   // columns of this workgroup
  if (here <= 0) return;
  const bool mend = ERR && (W == 32 || tok_span(keys, j.doc).n <= TOK_MEND_KEYS);   // uniform
  const int quads = g.dim >> 2, lanes = quads <= 4 ? 4 : quads <= 8 ? 8 : quads <= 16 ? 16 : 32;
  const int cols = here <= 1 ? 1 : here <= 2 ? 2 : here <= 4 ? 4 : 8, zs = NT / (lanes * cols);
  const int quad = threadIdx.x & (lanes - 1), col = (threadIdx.x / lanes) & (cols - 1), z = threadIdx.x / (lanes * cols);
  const bool on = quad < quads && col < here;
  Sum a = {{0.f, 0.f, 0.f, 0.f}, {0.f, 0.f, 0.f, 0.f}, -INFINITY, 0.f};
  if (on) {
#pragma unroll 4
    for (int p = z; p < j.pieces; p += zs) {
      const long long slot = p == 0 ? blocks + (int)blockIdx.x : (int)blockIdx.x + p;   // the first piece is the end of its workgroup's units
      const long long at = (slot * heads + n) * W + blockIdx.y * COLS + col;
      Sum b = {};
      b.o = *reinterpret_cast<const f32x4*>(part + at * g.dim + quad * 4);
      if (PASS == TOK_FWD) {
        const float2 s = *reinterpret_cast<const float2*>(g.part2 + 2 * at);
        b.m = s.x; b.l = s.y;
      }
      if (mend) b.k = *reinterpret_cast<const f32x4*>(g.part2 + at * g.dim + quad * 4);
      if (ERR) b.l = g.part3[at];
      add<PASS>(a, b, mend);
    }
  }
  if (zs > 1) {
    sums[threadIdx.x] = a.o;
    if (mend) sums2[threadIdx.x] = a.k;
    if (PASS != TOK_DKV) stats[threadIdx.x] = float2{a.m, a.l};
    __syncthreads();
    if (z) return;
    const int stride = lanes * cols;
    for (int k = 1; k < zs; ++k) {
      const int at = threadIdx.x + k * stride;
      Sum b = {};
      b.o = sums[at];
      if (mend) b.k = sums2[at];
      if (PASS != TOK_DKV) { b.m = stats[at].x; b.l = stats[at].y; }
      add<PASS>(a, b, mend);
    }
  }
  if (!on) return;
  const int at = first + col, qi = at / side.group, head = j.head * hstep + n * hs.step + (at - qi * side.group);
  const long long row = c.lo + qi;
  const float f = PASS != TOK_FWD ? 1.f : a.l == 0.f ? 0.f : 1.f / a.l;
  typedef T T4 __attribute__((ext_vector_type(4)));
  T4 v;
#pragma unroll
  for (int i = 0; i < 4; ++i) v[i] = from_f<T>(mend ? fmaf(-a.l, a.k[i], a.o[i]) : a.o[i] * f);
  *reinterpret_cast<T4*>((T*)out.out + row * out.ld + head * g.dim + quad * 4) = v;
  if (PASS == TOK_FWD && quad == 0) g.lse[head * (long long)g.rows_q + row] = a.l == 0.f ? -INFINITY : (a.m + __builtin_amdgcn_logf(a.l)) * TOK_LN2;
  if (ERR && quad == 0) g.delta[head * (long long)g.rows_q + row] += a.l;
}

// rows of a block in LDS (the kernels' KB)
int tok_block_rows(int pass, int dt, int dim, TokCut c) { return dt == DT_F32 || c.heads == 2 || (pass != TOK_DKV && dim > 96) ? 32 : 64; }
TokSide side_of(const TokAttn& g, bool queries, int pack, int per) { return queries ? TokSide{g.q_start, g.rows_q, pack, per} : TokSide{g.k_start, g.rows_k, 1, per}; }

template <typename T, int PASS>
hipError_t join(const TokAttn& g, TokCut c, JoinOut out, JoinOut out1, hipStream_t s) {
  constexpr bool KEYS = PASS == TOK_DKV;
  const dim3 grid(c.blocks, c.waves * 32 / 8, KEYS ? 2 : c.heads);
  const TokHeads hs = tok_heads(g, c.heads);
  const TokSide side = side_of(g, !KEYS, hs.pack, c.waves * 32);
  const int hstep = KEYS ? 1 : g.group * (hs.kv_step + 1);   // heads from one group to the next
  const TokSide keys = side_of(g, false, 1, 1);
  if (c.waves == 4) tok_join_k<T, 128, PASS><<<grid, 256, 0, s>>>(g, side, keys, hs, hstep, c.blocks, out, out1);
  else tok_join_k<T, 32, PASS><<<grid, 512, 0, s>>>(g, side, keys, hs, hstep, c.blocks, out, out1);
  return hipGetLastError();
}
template <typename T>
hipError_t join_pass(int pass, const TokAttn& g, TokCut c, hipStream_t s) {
  if (pass == TOK_FWD) return join<T, TOK_FWD>(g, c, {g.o, g.ldo}, {}, s);
  if (pass == TOK_DQ) return join<T, TOK_DQ>(g, c, {g.dq, g.lddq}, {}, s);
  return join<T, TOK_DKV>(g, c, {g.dk, g.lddk}, {g.dv, g.lddv}, s);
}

}  // namespace

// Few columns a slide leave three of four wavefronts idle: a wavefront a workgroup then.  As many workgroups as the card holds at a time: one or
// two of four wavefronts on each of 256 units, four or eight of one; fewer where there is less to do.  (Where there is, down to one unit each: 12 slides' tokens against 1 to 8192 keys,
// 12 heads: 27.7 us with four units at least, 20.9 with two, 17.9 with one.)
// Two heads at a time: a key head's, or two key heads', where the kernels are built for it.
TokCut tok_cut(int pass, const slide_tokens_attn& s, bool bias) {
  const int group = s.heads_q / s.heads_k;
  const bool queries = pass != TOK_DKV;
  TokCut c;
  c.heads = pass == TOK_FWD && bias && s.dtype == DT_BF16 && s.head_dim > 32 && s.head_dim <= 64 && (group == 1 ? s.heads_k % 2 == 0 : group % 2 == 0) ? 2 : 1;
  long long cols = queries ? s.rows_q * (group > 1 ? group / c.heads : 1) : s.rows_k;
  c.waves = cols <= 32LL * s.docs ? 1 : 4;
  if (c.waves == 1 && c.heads == 2) {   // built for four wavefronts
    c.heads = 1;
    cols = s.rows_q * group;
    c.waves = cols <= 32LL * s.docs ? 1 : 4;
  }
  const long long rows = queries ? s.rows_k : s.rows_q * group, width = 32 * c.waves, kb = tok_block_rows(pass, s.dtype, s.head_dim, c);
  // no more units than these: a slide's last tile and block are partly empty
  const double units = ((double)cols / width + s.docs) * ((double)rows / kb + 1) * s.heads_k;
  // two wavefronts a SIMD where 256 registers do, which is where the kernels' launch bounds say so; else one
  const bool two = c.waves == 4 ? s.head_dim <= 64 || (pass == TOK_FWD && s.dtype == DT_BF16) : pass == TOK_FWD && s.head_dim <= 64;
  const long long most = (c.waves == 4 ? 256 : 1024) * (two ? 2 : 1), n = units < (double)most ? (long long)units + 1 : most;
  c.blocks = (int)((n + 7) / 8 * 8);
  return c;
}

hipError_t launch_tok_table(int pass, int dt, const TokAttn& g, TokCut c, long long* table, hipStream_t s) {
  if (g.docs <= 64) return hipSuccess;
  const int kb = tok_block_rows(pass, dt, g.dim, c), pack = tok_heads(g, c.heads).pack;
  const bool queries = pass != TOK_DKV;
  tok_table_k<<<1, 1024, 0, s>>>(side_of(g, queries, pack, c.waves * 32), side_of(g, !queries, g.group, kb), g.docs, table);
  return hipGetLastError();
}

hipError_t launch_tok_join(int pass, int dt, const TokAttn& g, TokCut c, hipStream_t s) {
  return dt == DT_F32 ? join_pass<float>(pass, g, c, s) : join_pass<bf16>(pass, g, c, s);
}

}  // namespace sl
