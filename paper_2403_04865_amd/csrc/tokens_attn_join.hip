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
// `zs`-th piece; the groups' results meet in LDS.  SOFTMAX: pieces are sums under maxima of their own.
template <typename T, int W, bool SOFTMAX>
__global__ void __launch_bounds__(256) tok_join_k(const TokAttn g, const TokSide side, int blocks, const float* __restrict__ part,
                                                  const float* __restrict__ stat, T* __restrict__ out, int ld) {
  constexpr int COLS = 8;
  __shared__ f32x4 sums[256];
  __shared__ float2 stats[256];
  const TokJoin j = ((const TokJoin*)g.joins)[blockIdx.x];
  if (j.pieces == 0) return;
  const TokSpan c = tok_span(side, j.doc);
  const int first = j.tile * W + blockIdx.y * COLS, here = c.n - first < COLS ? c.n - first : COLS;   // columns of this workgroup
  if (here <= 0) return;
  const int quads = g.dim >> 2, lanes = quads <= 4 ? 4 : quads <= 8 ? 8 : quads <= 16 ? 16 : 32;
  const int cols = here <= 1 ? 1 : here <= 2 ? 2 : here <= 4 ? 4 : 8, zs = 256 / (lanes * cols);
  const int quad = threadIdx.x & (lanes - 1), col = (threadIdx.x / lanes) & (cols - 1), z = threadIdx.x / (lanes * cols);
  const bool on = quad < quads && col < here;
  f32x4 o = {0.f, 0.f, 0.f, 0.f};
  float m = -INFINITY, l = 0.f;
  if (on) {
#pragma unroll 4
    for (int p = z; p < j.pieces; p += zs) {
      const long long slot = p == 0 ? blocks + (int)blockIdx.x : (int)blockIdx.x + p;   // the first piece is the end of its workgroup's units
      const long long at = slot * W + blockIdx.y * COLS + col;
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
  const int at = first + col, qi = at / side.group, head = j.head * side.group + (at - qi * side.group);
  const long long row = c.lo + qi;
  const float f = !SOFTMAX ? 1.f : l == 0.f ? 0.f : 1.f / l;
  typedef T T4 __attribute__((ext_vector_type(4)));
  T4 v;
#pragma unroll
  for (int i = 0; i < 4; ++i) v[i] = from_f<T>(o[i] * f);
  *reinterpret_cast<T4*>(out + row * ld + head * g.dim + quad * 4) = v;
  if (SOFTMAX && quad == 0) g.lse[head * (long long)g.rows_q + row] = l == 0.f ? -INFINITY : (m + __builtin_amdgcn_logf(l)) * TOK_LN2;
}

TokSide side_of(const TokAttn& g, bool queries, int per) { return queries ? TokSide{g.q_start, g.rows_q, g.group, per} : TokSide{g.k_start, g.rows_k, 1, per}; }

template <typename T, bool SOFTMAX>
hipError_t join(const TokAttn& g, TokCut c, bool queries, const float* part, const float* stat, void* out, int ld, hipStream_t s) {
  const dim3 grid(c.blocks, c.waves * 32 / 8);
  const TokSide side = side_of(g, queries, c.waves * 32);
  if (c.waves == 4) tok_join_k<T, 128, SOFTMAX><<<grid, 256, 0, s>>>(g, side, c.blocks, part, stat, (T*)out, ld);
  else tok_join_k<T, 32, SOFTMAX><<<grid, 256, 0, s>>>(g, side, c.blocks, part, stat, (T*)out, ld);
  return hipGetLastError();
}
template <typename T>
hipError_t join_pass(int pass, const TokAttn& g, TokCut c, hipStream_t s) {
  if (pass == TOK_FWD) return join<T, true>(g, c, true, g.part, g.part2, g.o, g.ldo, s);
  if (pass == TOK_DQ) return join<T, false>(g, c, true, g.part, nullptr, g.dq, g.lddq, s);
  const hipError_t e = join<T, false>(g, c, false, g.part, nullptr, g.dk, g.lddk, s);
  return e != hipSuccess ? e : join<T, false>(g, c, false, g.part2, nullptr, g.dv, g.lddv, s);
}

}  // namespace

// Few columns a slide leave three of four wavefronts idle: a wavefront a workgroup then.  Two workgroups of four wavefronts are on each of 256 units
// at a time, or eight of one; fewer where there is less to do.
TokCut tok_cut(long long cols, long long rows, int docs, int heads, int dt) {
  TokCut c;
  c.waves = cols <= 32LL * docs ? 1 : 4;
  const long long width = 32 * c.waves, kb = dt == DT_F32 ? 32 : 64;
  // no more units than these: a slide's last tile and block are partly empty
  const double units = ((double)cols / width + docs) * ((double)rows / kb + 1) * heads;
  const long long most = c.waves == 4 ? 512 : 2048, n = units / TOK_LEAST < (double)most ? (long long)(units / TOK_LEAST) + 1 : most;
  c.blocks = (int)((n + 7) / 8 * 8);
  return c;
}

hipError_t launch_tok_table(int pass, int dt, const TokAttn& g, TokCut c, long long* table, hipStream_t s) {
  if (g.docs <= 64) return hipSuccess;
  const int kb = dt == DT_F32 ? TokType<float>::KB : TokType<bf16>::KB;
  const bool queries = pass != TOK_DKV;
  tok_table_k<<<1, 1024, 0, s>>>(side_of(g, queries, c.waves * 32), side_of(g, !queries, kb), g.docs, table);
  return hipGetLastError();
}

hipError_t launch_tok_join(int pass, int dt, const TokAttn& g, TokCut c, hipStream_t s) {
  return dt == DT_F32 ? join_pass<float>(pass, g, c, s) : join_pass<bf16>(pass, g, c, s);
}

}  // namespace sl
