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
// `zs`-th piece; blockIdx.z is the head of a group; the groups' results meet in LDS.  SOFTMAX: pieces are sums under maxima of their own.
// TWO: two results of the same columns, one after the other in blockIdx.z (keys' and values' gradients).
template <typename T, int W, bool SOFTMAX, bool TWO>
__global__ void __launch_bounds__(W == 32 ? 512 : 256) tok_join_k(const TokAttn g, const TokSide side, const TokHeads hs, int hstep, int blocks,
                                                                  const float* __restrict__ part0, const float* __restrict__ stat, T* __restrict__ out0, int ld0, T* __restrict__ out1, int ld1) {
  constexpr int COLS = 8, NT = W == 32 ? 512 : 256;   // few columns mean many pieces
  __shared__ f32x4 sums[NT];
  __shared__ float2 stats[NT];
  const TokJoin j = ((const TokJoin*)g.joins)[blockIdx.x];
  if (j.pieces == 0) return;
  const int n = TWO ? 0 : blockIdx.z, heads = TWO ? 1 : gridDim.z;
  const float* const part = TWO && blockIdx.z ? stat : part0;
  T* const out = TWO && blockIdx.z ? out1 : out0;
  const int ld = TWO && blockIdx.z ? ld1 : ld0;
  const TokSpan c = tok_span(side, j.doc);
  const int first = j.tile * W + blockIdx.y * COLS, here = c.n - first < COLS ? c.n - first : COLS;   // columns of this workgroup
  if (here <= 0) return;
  const int quads = g.dim >> 2, lanes = quads <= 4 ? 4 : quads <= 8 ? 8 : quads <= 16 ? 16 : 32;
  const int cols = here <= 1 ? 1 : here <= 2 ? 2 : here <= 4 ? 4 : 8, zs = NT / (lanes * cols);
  const int quad = threadIdx.x & (lanes - 1), col = (threadIdx.x / lanes) & (cols - 1), z = threadIdx.x / (lanes * cols);
  const bool on = quad < quads && col < here;
  f32x4 o = {0.f, 0.f, 0.f, 0.f};
  float m = -INFINITY, l = 0.f;
  if (on) {
#pragma unroll 4
    for (int p = z; p < j.pieces; p += zs) {
      const long long slot = p == 0 ? blocks + (int)blockIdx.x : (int)blockIdx.x + p;   // the first piece is the end of its workgroup's units
      const long long at = (slot * heads + n) * W + blockIdx.y * COLS + col;
      const f32x4 v = *reinterpret_cast<const f32x4*>(part + at * g.dim + quad * 4);
      if (SOFTMAX) {
        const float2 s = *reinterpret_cast<const float2*>(stat + 2 * at);
        const float n = fmaxf(m, s.x), ns = n == -INFINITY ? 0.f : n;
        const float wa = __builtin_amdgcn_exp2f(m - ns), wb = __builtin_amdgcn_exp2f(s.x - ns);
        m = n;
        l = fmaf(l, wa, s.y * wb);
#pragma unroll
        for (int i = 0; i < 4; ++i) o[i] = fmaf(o[i], wa, v[i] * wb);
      } else {
        o += v;
      }
    }
  }
  if (zs > 1) {
    sums[threadIdx.x] = o;
    if (SOFTMAX) stats[threadIdx.x] = float2{m, l};
    __syncthreads();
    if (z) return;
    const int stride = lanes * cols;
    for (int k = 1; k < zs; ++k) {   // in the groups' order
      const f32x4 v = sums[threadIdx.x + k * stride];
      if (SOFTMAX) {
        const float2 s = stats[threadIdx.x + k * stride];
        const float n = fmaxf(m, s.x), ns = n == -INFINITY ? 0.f : n;
        const float wa = __builtin_amdgcn_exp2f(m - ns), wb = __builtin_amdgcn_exp2f(s.x - ns);
        m = n;
        l = fmaf(l, wa, s.y * wb);
#pragma unroll
        for (int i = 0; i < 4; ++i) o[i] = fmaf(o[i], wa, v[i] * wb);
      } else {
        o += v;
      }
    }
  }
  if (!on) return;
  const int at = first + col, qi = at / side.group, head = j.head * hstep + n * hs.step + (at - qi * side.group);
  const long long row = c.lo + qi;
  const float f = !SOFTMAX ? 1.f : l == 0.f ? 0.f : 1.f / l;
  typedef T T4 __attribute__((ext_vector_type(4)));
  T4 v;
#pragma unroll
  for (int i = 0; i < 4; ++i) v[i] = from_f<T>(o[i] * f);
  *reinterpret_cast<T4*>(out + row * ld + head * g.dim + quad * 4) = v;
  if (SOFTMAX && quad == 0) g.lse[head * (long long)g.rows_q + row] = l == 0.f ? -INFINITY : (m + __builtin_amdgcn_logf(l)) * TOK_LN2;
}

// rows of a block in LDS (the kernels' KB)
int tok_block_rows(int pass, int dt, int dim, TokCut c) { return dt == DT_F32 || c.heads == 2 || (pass == TOK_FWD && dim > 96) ? 32 : 64; }
TokSide side_of(const TokAttn& g, bool queries, int pack, int per) { return queries ? TokSide{g.q_start, g.rows_q, pack, per} : TokSide{g.k_start, g.rows_k, 1, per}; }

template <typename T, bool SOFTMAX, bool TWO>
hipError_t join(const TokAttn& g, TokCut c, void* out, int ld, void* out1, int ld1, hipStream_t s) {
  const dim3 grid(c.blocks, c.waves * 32 / 8, TWO ? 2 : c.heads);
  const TokHeads hs = tok_heads(g, c.heads);
  const TokSide side = side_of(g, !TWO, hs.pack, c.waves * 32);
  const int hstep = TWO ? 1 : g.group * (hs.kv_step + 1);   // heads from one group to the next
  if (c.waves == 4) tok_join_k<T, 128, SOFTMAX, TWO><<<grid, 256, 0, s>>>(g, side, hs, hstep, c.blocks, g.part, g.part2, (T*)out, ld, (T*)out1, ld1);
  else tok_join_k<T, 32, SOFTMAX, TWO><<<grid, 512, 0, s>>>(g, side, hs, hstep, c.blocks, g.part, g.part2, (T*)out, ld, (T*)out1, ld1);
  return hipGetLastError();
}
template <typename T>
hipError_t join_pass(int pass, const TokAttn& g, TokCut c, hipStream_t s) {
  if (pass == TOK_FWD) return join<T, true, false>(g, c, g.o, g.ldo, nullptr, 0, s);
  if (pass == TOK_DQ) return join<T, false, false>(g, c, g.dq, g.lddq, nullptr, 0, s);
  return join<T, false, true>(g, c, g.dk, g.lddk, g.dv, g.lddv, s);
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
