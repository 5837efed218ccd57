// Group normalisation with its activation over channels-last tiles, forward and backward (gfx950).
//
// A unit is one tile's slice of whole groups.  Bound by memory traffic: forward x in, y out (and one byte of checkpoint), backward
// dy and x in, dx out; everything else is to keep a value from being read twice.
//   * Where a unit fits the registers of one workgroup it is loaded once and stays there: sums of every channel over the rows,
//     the groups' means out of these, squares of the distances from the mean the same way, then the result (forward);
//     the two sums per channel that the gradients need, then dx (backward).
//   * Larger units are split over rows: partial statistics per channel (count, mean, sum of squared distances: merged, never a
//     difference of large sums), one small kernel for the groups, one pass for the result.
// A thread owns V neighbouring channels (16 bytes of bfloat16) and strides over rows.  All statistics and sums are float32; the
// gradients of gain and shift add the workgroups' sums in double, in a fixed order.
#include "act8_internal.h"

namespace sl {

namespace {

// V values of a row as they are in memory
template <typename T, int V> struct Vec;
template <> struct Vec<bf16, 8> {
  u32x4 r;
  __device__ __forceinline__ void load(const bf16* p) { r = *reinterpret_cast<const u32x4*>(p); }
  __device__ __forceinline__ void zero() { r = u32x4{0, 0, 0, 0}; }
  __device__ __forceinline__ void get(float (&v)[8]) const {
#pragma unroll
    for (int w = 0; w < 4; ++w) {
      v[2 * w] = __uint_as_float(r[w] << 16);
      v[2 * w + 1] = __uint_as_float(r[w] & 0xffff0000u);
    }
  }
};
template <> struct Vec<float, 8> {
  f32x4 lo, hi;
  __device__ __forceinline__ void load(const float* p) {
    lo = *reinterpret_cast<const f32x4*>(p); hi = *reinterpret_cast<const f32x4*>(p + 4);
  }
  __device__ __forceinline__ void zero() { lo = hi = f32x4{0.f, 0.f, 0.f, 0.f}; }
  __device__ __forceinline__ void get(float (&v)[8]) const {
#pragma unroll
    for (int e = 0; e < 4; ++e) { v[e] = lo[e]; v[4 + e] = hi[e]; }
  }
};
template <typename T> struct Vec<T, 1> {
  T r;
  __device__ __forceinline__ void load(const T* p) { r = *p; }
  __device__ __forceinline__ void zero() { r = (T)0.f; }
  __device__ __forceinline__ void get(float (&v)[1]) const { v[0] = to_f(r); }
};
__device__ __forceinline__ void store_vec(bf16* p, const float (&v)[8]) {
  bf16x8 t;
#pragma unroll
  for (int e = 0; e < 8; ++e) t[e] = (bf16)v[e];
  *reinterpret_cast<bf16x8*>(p) = t;
}
__device__ __forceinline__ void store_vec(float* p, const float (&v)[8]) {
  *reinterpret_cast<f32x4*>(p) = f32x4{v[0], v[1], v[2], v[3]};
  *reinterpret_cast<f32x4*>(p + 4) = f32x4{v[4], v[5], v[6], v[7]};
}
template <typename T> __device__ __forceinline__ void store_vec(T* p, const float (&v)[1]) { *p = from_f<T>(v[0]); }

// eight codes of a checkpoint and their scale byte, or (V = 1) one
template <int V> struct Vec8;
template <> struct Vec8<8> {
  u32x2 q; unsigned b;
  __device__ __forceinline__ void load(const A8& a, long long row, int c) {
    q = *reinterpret_cast<const u32x2*>(a.codes + row * a.ldc + c);
    b = a.scales[row * a.lds + (c >> 7)];
  }
  __device__ __forceinline__ void zero() { q = u32x2{0, 0}; b = 127; }
  __device__ __forceinline__ void get(float (&v)[8]) const {
    const float s = a8_scale(b);
    float t[4];
    a8_value4(q[0], s, t);
#pragma unroll
    for (int e = 0; e < 4; ++e) v[e] = t[e];
    a8_value4(q[1], s, t);
#pragma unroll
    for (int e = 0; e < 4; ++e) v[4 + e] = t[e];
  }
};
template <> struct Vec8<1> {
  unsigned q, b;
  __device__ __forceinline__ void load(const A8& a, long long row, int c) {
    q = a.codes[row * a.ldc + c];
    b = a.scales[row * a.lds + (c >> 7)];
  }
  __device__ __forceinline__ void zero() { q = 0; b = 127; }
  __device__ __forceinline__ void get(float (&v)[1]) const { v[0] = __builtin_amdgcn_cvt_f32_fp8((int)q, 0) * a8_scale(b); }
};

__device__ __forceinline__ float act_any(float u, int act) {   // act: uniform
  switch (act) {
    case SLIDE_ACT_RELU: return act_f<SLIDE_ACT_RELU>(u);
    case SLIDE_ACT_SILU: return act_f<SLIDE_ACT_SILU>(u);
    case SLIDE_ACT_GELU: return act_f<SLIDE_ACT_GELU>(u);
    default: return u;
  }
}

struct P {
  GroupNorm g;
  A8 x8;
  int S, slices, G, per, C, hw;   // channels of a slice, slices, groups, channels of a group
  long long n;
  int units_p;                    // workgroups per slice that share out the tiles (resident kernels)
  int chunks, rows_chunk;         // split kernels: pieces of a tile's rows
  float* part;                    // [..][2][C]
  float* sums;                    // [n][G][2]
};

// What a thread of a workgroup of TH owns: channels c0 .. c0 + V - 1 of the slice, rows tr, tr + rpp, ...
template <int V> struct Own {
  int vpr, rpp, tr, tc;
  bool on;
  __device__ __forceinline__ Own(int S, int th) {
    vpr = S / V; rpp = th / vpr;
    tr = (int)threadIdx.x / vpr; tc = (int)threadIdx.x - tr * vpr;
    on = tr < rpp;
  }
};

// Sums over the rows of the workgroup: s[V] per thread -> ch[S] per channel of the slice.  red: TH V floats, red2: TH (or S, where
// larger) floats.  Ends with a barrier.
template <int TH, int V>
__device__ __forceinline__ void channel_sums(const float (&s)[V], const Own<V>& o, int S, float* red, float* red2, float* ch) {
  if (o.on) {
#pragma unroll
    for (int v = 0; v < V; ++v) red[o.tr * S + o.tc * V + v] = s[v];
  }
  __syncthreads();
  const int Q = S < TH ? TH / S : 1;
  if (Q == 1) {
    for (int c = threadIdx.x; c < S; c += TH) {
      float a = 0.f;
      for (int r = 0; r < o.rpp; ++r) a += red[r * S + c];
      ch[c] = a;
    }
  } else {
    const int q = (int)threadIdx.x / S, c = (int)threadIdx.x - q * S;
    if (q < Q) {
      float a = 0.f;
      for (int r = q; r < o.rpp; r += Q) a += red[r * S + c];
      red2[q * S + c] = a;
    }
    __syncthreads();
    if ((int)threadIdx.x < S) {
      float a = 0.f;
      for (int k = 0; k < Q; ++k) a += red2[k * S + threadIdx.x];
      ch[threadIdx.x] = a;
    }
  }
  __syncthreads();
}

// per-channel values ch[S] (times w[S] where w is not null) -> their sum over each group of the slice, gs[groups].  Ends with a barrier.
template <int TH>
__device__ __forceinline__ void group_sums(const float* ch, const float* w, int S, int per, float* gs) {
  const int gl = S / per;
  int L = 64;
  while (L > 1 && L * gl > TH) L >>= 1;
  const int sub = (int)threadIdx.x / L, lane = (int)threadIdx.x & (L - 1);
  for (int g = sub; g < gl; g += TH / L) {
    float a = 0.f;
    for (int c = lane; c < per; c += L) a += w ? ch[g * per + c] * w[g * per + c] : ch[g * per + c];
    for (int k = L >> 1; k > 0; k >>= 1) a += __shfl_xor(a, k, 64);
    if (lane == 0) gs[g] = a;
  }
  __syncthreads();
}

// ---- resident units -------------------------------------------------------------------------------------------------

constexpr int SMAX = 2048;   // most channels of a slice

template <typename T, int V, int TH, int E>
__global__ void __launch_bounds__(TH) gn_fwd_k(P p) {
  __shared__ __attribute__((aligned(16))) float red[TH * V];
  __shared__ float red2[TH], ch[TH * V], gs[TH * V];
  const GroupNorm& g = p.g;
  const Own<V> o(p.S, TH);
  const int j = blockIdx.x >> 3, slice = j % p.slices, first = (int)(blockIdx.x & 7) + 8 * (j / p.slices);
  if (first >= p.units_p) return;
  const int c0 = slice * p.S + o.tc * V, per = p.per;
  const float count = (float)p.hw * (float)per;
  float gam[V], bet[V];
  int gi[V];
#pragma unroll
  for (int v = 0; v < V; ++v) {
    gam[v] = o.on ? g.gamma[c0 + v] : 0.f;
    bet[v] = o.on ? g.beta[c0 + v] : 0.f;
    gi[v] = (o.tc * V + v) / per;
  }
  for (long long tile = first; tile < p.n; tile += p.units_p) {
    const long long r0 = tile * p.hw;
    const T* x = (const T*)g.x + r0 * g.ldx + c0;
    Vec<T, V> buf[E];
#pragma unroll
    for (int e = 0; e < E; ++e) {
      const int r = o.tr + e * o.rpp;
      if (o.on && r < p.hw) buf[e].load(x + (long long)r * g.ldx);
      else buf[e].zero();
    }
    float s[V];
#pragma unroll
    for (int v = 0; v < V; ++v) s[v] = 0.f;
#pragma unroll
    for (int e = 0; e < E; ++e) {
      float t[V];
      buf[e].get(t);
#pragma unroll
      for (int v = 0; v < V; ++v) s[v] += t[v];
    }
    channel_sums<TH, V>(s, o, p.S, red, red2, ch);
    group_sums<TH>(ch, nullptr, p.S, per, gs);
    float m[V];
#pragma unroll
    for (int v = 0; v < V; ++v) { m[v] = o.on ? gs[gi[v]] / count : 0.f; s[v] = 0.f; }
    const float my_mean = (int)threadIdx.x < p.S / per ? gs[threadIdx.x] / count : 0.f;
#pragma unroll
    for (int e = 0; e < E; ++e) {
      if (!(o.on && o.tr + e * o.rpp < p.hw)) continue;
      float t[V];
      buf[e].get(t);
#pragma unroll
      for (int v = 0; v < V; ++v) { const float d = t[v] - m[v]; s[v] = fmaf(d, d, s[v]); }
    }
    channel_sums<TH, V>(s, o, p.S, red, red2, ch);
    group_sums<TH>(ch, nullptr, p.S, per, gs);
    for (int k = threadIdx.x; k < p.S / per; k += TH) {
      const long long at = tile * p.G + slice * (p.S / per) + k;
      g.mean[at] = my_mean;    // S / per <= TH: one group per thread
      g.rstd[at] = 1.0f / sqrtf(gs[k] / count + g.s.eps);
    }
    float a[V];
#pragma unroll
    for (int v = 0; v < V; ++v) a[v] = o.on ? gam[v] * (1.0f / sqrtf(gs[gi[v]] / count + g.s.eps)) : 0.f;
#pragma unroll
    for (int e = 0; e < E; ++e) {
      const int r = o.tr + e * o.rpp;
      if (!(o.on && r < p.hw)) continue;
      float t[V], u[V];
      buf[e].get(t);
#pragma unroll
      for (int v = 0; v < V; ++v) u[v] = fmaf(t[v] - m[v], a[v], bet[v]);
      if (g.resid) {
        Vec<T, V> q;
        q.load((const T*)g.resid + (r0 + r) * g.ldr + c0);
        q.get(t);
#pragma unroll
        for (int v = 0; v < V; ++v) u[v] += t[v];
      }
#pragma unroll
      for (int v = 0; v < V; ++v) u[v] = act_any(u[v], g.s.act);
      store_vec((T*)g.y + (r0 + r) * g.ldy + c0, u);
    }
    __syncthreads();
  }
}

// du = dy act'(u) of one value.  A rectifier asks which side of zero u is on: where float32 cannot tell, it is formed again in
// double (mean and rstd are what the forward stored; products of two floats are exact there).
__device__ __forceinline__ float slope(float u, float mag, int act, float x, float mean, float rstd, float gam, float bet, float res) {
  switch (act) {
    case SLIDE_ACT_RELU: {
      bool pos = u > 0.f;
      if (fabsf(u) <= 1e-6f * mag)
        pos = (((double)x - (double)mean) * (double)rstd) * (double)gam + (double)bet + (double)res > 0.0;
      return pos ? 1.f : 0.f;
    }
    case SLIDE_ACT_SILU: {
      const float s = sigmoid_f(u);
      return s * fmaf(u, 1.0f - s, 1.0f);
    }
    case SLIDE_ACT_GELU: return gelu_grad_f(u);
    default: return 1.f;
  }
}

// du and xhat of a thread's V values of one row
template <int V>
__device__ __forceinline__ void du_xhat(const float (&x)[V], const float (&dy)[V], const float (&res)[V], const float (&mean)[V],
                                        const float (&rstd)[V], const float (&gam)[V], const float (&bet)[V], int act,
                                        float (&du)[V], float (&xh)[V]) {
#pragma unroll
  for (int v = 0; v < V; ++v) {
    xh[v] = (x[v] - mean[v]) * rstd[v];
    const float z = xh[v] * gam[v], u = z + bet[v] + res[v];
    const float mag = fabsf(z) + fabsf(bet[v]) + fabsf(res[v]);
    du[v] = act == SLIDE_ACT_NONE ? dy[v] : dy[v] * slope(u, mag, act, x[v], mean[v], rstd[v], gam[v], bet[v], res[v]);
  }
}

// X8: the input is the checkpoint
template <typename T, int V, bool X8> struct Input { typedef Vec<T, V> type; };
template <typename T, int V> struct Input<T, V, true> { typedef Vec8<V> type; };
template <typename T, int V>
__device__ __forceinline__ void load_in(Vec<T, V>& b, const P& p, long long row, int c) { b.load((const T*)p.g.x + row * p.g.ldx + c); }
template <int V>
__device__ __forceinline__ void load_in(Vec8<V>& b, const P& p, long long row, int c) { b.load(p.x8, row, c); }

template <typename T, int V, int TH, int E, bool X8>
__global__ void __launch_bounds__(TH) gn_bwd_k(P p) {
  __shared__ __attribute__((aligned(16))) float red[TH * V];
  __shared__ float red2[TH], ca[TH * V], cb[TH * V], ga[TH * V], gb[TH * V], wg[TH * V];
  const GroupNorm& g = p.g;
  const Own<V> o(p.S, TH);
  const int j = blockIdx.x >> 3, slice = j % p.slices, first = (int)(blockIdx.x & 7) + 8 * (j / p.slices);
  if (first >= p.units_p) return;
  const int c0 = slice * p.S + o.tc * V, per = p.per, act = g.s.act;
  const float inv = 1.0f / ((float)p.hw * (float)per);
  float gam[V], bet[V];
  int gi[V];
#pragma unroll
  for (int v = 0; v < V; ++v) {
    gam[v] = o.on ? g.gamma[c0 + v] : 0.f;
    bet[v] = o.on ? g.beta[c0 + v] : 0.f;
    gi[v] = (o.tc * V + v) / per;
  }
  for (int c = threadIdx.x; c < p.S; c += TH) wg[c] = g.gamma[slice * p.S + c];
  // sums of this workgroup's tiles for the gain and the shift: thread t keeps those of channels t, t + TH, ...
  float tg[V], tb[V];
#pragma unroll
  for (int v = 0; v < V; ++v) tg[v] = tb[v] = 0.f;
  for (long long tile = first; tile < p.n; tile += p.units_p) {
    const long long r0 = tile * p.hw;
    typename Input<T, V, X8>::type bx[E];
    Vec<T, V> bd[E];
#pragma unroll
    for (int e = 0; e < E; ++e) {
      const int r = o.tr + e * o.rpp;
      if (o.on && r < p.hw) {
        load_in(bx[e], p, r0 + r, c0);
        bd[e].load((const T*)g.dy + (r0 + r) * g.lddy + c0);
      } else { bx[e].zero(); bd[e].zero(); }
    }
    float mean[V], rstd[V];
#pragma unroll
    for (int v = 0; v < V; ++v) {
      const long long at = tile * p.G + slice * (p.S / per) + gi[v];
      mean[v] = o.on ? g.mean[at] : 0.f;
      rstd[v] = o.on ? g.rstd[at] : 0.f;
    }
    float s[V], q[V];
#pragma unroll
    for (int v = 0; v < V; ++v) s[v] = q[v] = 0.f;
    auto one = [&](int e, float (&du)[V], float (&xh)[V]) __attribute__((always_inline)) {
      float x[V], dy[V], res[V];
      bx[e].get(x);
      bd[e].get(dy);
#pragma unroll
      for (int v = 0; v < V; ++v) res[v] = 0.f;
      if (g.resid) {
        Vec<T, V> b;
        b.load((const T*)g.resid + (r0 + o.tr + e * o.rpp) * g.ldr + c0);
        b.get(res);
      }
      du_xhat<V>(x, dy, res, mean, rstd, gam, bet, act, du, xh);
    };
#pragma unroll
    for (int e = 0; e < E; ++e) {
      if (!(o.on && o.tr + e * o.rpp < p.hw)) continue;
      float du[V], xh[V];
      one(e, du, xh);
#pragma unroll
      for (int v = 0; v < V; ++v) { s[v] += du[v]; q[v] = fmaf(du[v], xh[v], q[v]); }
    }
    channel_sums<TH, V>(s, o, p.S, red, red2, cb);
    channel_sums<TH, V>(q, o, p.S, red, red2, ca);
    group_sums<TH>(cb, wg, p.S, per, gb);
    group_sums<TH>(ca, wg, p.S, per, ga);
#pragma unroll
    for (int v = 0; v < V; ++v) {
      const int c = threadIdx.x + v * TH;
      if (c < p.S) { tg[v] += ca[c]; tb[v] += cb[c]; }
    }
    float m1[V], m2[V];
#pragma unroll
    for (int v = 0; v < V; ++v) { m1[v] = o.on ? gb[gi[v]] * inv : 0.f; m2[v] = o.on ? ga[gi[v]] * inv : 0.f; }
#pragma unroll
    for (int e = 0; e < E; ++e) {
      const int r = o.tr + e * o.rpp;
      if (!(o.on && r < p.hw)) continue;
      float du[V], xh[V];
      one(e, du, xh);
      if (g.dresid) store_vec((T*)g.dresid + (r0 + r) * g.lddr + c0, du);
#pragma unroll
      for (int v = 0; v < V; ++v) du[v] = rstd[v] * ((du[v] * gam[v] - m1[v]) - xh[v] * m2[v]);
      store_vec((T*)g.y + (r0 + r) * g.ldy + c0, du);
    }
    __syncthreads();
  }
#pragma unroll
  for (int v = 0; v < V; ++v) {
    const int c = threadIdx.x + v * TH;
    if (c < p.S) {
      p.part[((long long)first * 2 + 0) * p.C + slice * p.S + c] = tg[v];
      p.part[((long long)first * 2 + 1) * p.C + slice * p.S + c] = tb[v];
    }
  }
}

// dgamma, dbeta = (accumulate ? what is there : 0) + the partials [rows][2][C], added in double in a fixed order; 16 channels per workgroup
__global__ void __launch_bounds__(1024) gn_sum_k(const float* __restrict__ part, long long rows, int C, float* dgamma, float* dbeta,
                                                 int accumulate) {
  __shared__ double ra[64][17], rb[64][17];
  const int c = threadIdx.x & 15, q = threadIdx.x >> 4, ch = blockIdx.x * 16 + c;
  double a = 0.0, b = 0.0;
  if (ch < C)
    for (long long r = q; r < rows; r += 64) { a += (double)part[r * 2 * C + ch]; b += (double)part[(r * 2 + 1) * C + ch]; }
  ra[q][c] = a; rb[q][c] = b;
  __syncthreads();
  if (threadIdx.x < 16 && ch < C) {
    a = b = 0.0;
    for (int k = 0; k < 64; ++k) { a += ra[k][c]; b += rb[k][c]; }
    dgamma[ch] = accumulate ? dgamma[ch] + (float)a : (float)a;
    dbeta[ch] = accumulate ? dbeta[ch] + (float)b : (float)b;
  }
}

// ---- units split over rows --------------------------------------------------------------------------------------------

constexpr int ST = 256, SE = 8;   // threads; rows of a thread whose loads are in flight together

// (count, mean, squared distances) of two disjoint sets, merged into the first
__device__ __forceinline__ void merge(float& n, float& m, float& q, float nb, float mb, float qb) {
  const float t = n + nb;
  if (t == 0.f) return;
  const float d = mb - m, f = nb / t;
  m = fmaf(d, f, m);
  q += qb + d * d * n * f;
  n = t;
}

struct Where { long long tile; int slice, chunk, lo, hi; };
__device__ __forceinline__ Where where(const P& p, long long unit) {
  Where w;
  w.slice = (int)(unit % p.slices);
  const long long k = unit / p.slices;
  w.chunk = (int)(k % p.chunks);
  w.tile = k / p.chunks;
  w.lo = w.chunk * p.rows_chunk;
  w.hi = w.lo + p.rows_chunk < p.hw ? w.lo + p.rows_chunk : p.hw;
  return w;
}

// partial statistics of a chunk: part[tile * chunks + chunk][0 mean, 1 squared distances][C]
template <typename T, int V>
__global__ void __launch_bounds__(ST) gn_stat_k(P p) {
  __shared__ float sn[ST], sm[ST * V], sq[ST * V];
  const GroupNorm& g = p.g;
  for (long long unit = blockIdx.x; unit < p.n * p.chunks * p.slices; unit += gridDim.x) {
    const Where w = where(p, unit);
    const int S = p.C - w.slice * p.S < p.S ? p.C - w.slice * p.S : p.S;   // the last slice may be short
    const Own<V> o(S, ST);
    const int c0 = w.slice * p.S + o.tc * V;
    const T* x = (const T*)g.x + w.tile * p.hw * g.ldx + c0;
    float n = 0.f, m[V], q[V];
#pragma unroll
    for (int v = 0; v < V; ++v) m[v] = q[v] = 0.f;
    if (o.on)
      for (int r = w.lo + o.tr; r < w.hi; r += SE * o.rpp) {
        Vec<T, V> buf[SE];
        int have = 0;
#pragma unroll
        for (int e = 0; e < SE; ++e) {
          const int k = r + e * o.rpp;
          if (k < w.hi) { buf[e].load(x + (long long)k * g.ldx); ++have; }
          else buf[e].zero();
        }
        float s[V], d2[V];
#pragma unroll
        for (int v = 0; v < V; ++v) s[v] = d2[v] = 0.f;
#pragma unroll
        for (int e = 0; e < SE; ++e) {
          float t[V];
          buf[e].get(t);
#pragma unroll
          for (int v = 0; v < V; ++v) s[v] += t[v];
        }
#pragma unroll
        for (int v = 0; v < V; ++v) s[v] /= (float)have;
#pragma unroll
        for (int e = 0; e < SE; ++e) {
          if (r + e * o.rpp >= w.hi) continue;
          float t[V];
          buf[e].get(t);
#pragma unroll
          for (int v = 0; v < V; ++v) { const float d = t[v] - s[v]; d2[v] = fmaf(d, d, d2[v]); }
        }
        const float n0 = n;
#pragma unroll
        for (int v = 0; v < V; ++v) { float k = n0; merge(k, m[v], q[v], (float)have, s[v], d2[v]); }
        n = n0 + (float)have;
      }
    if (o.on) {
      if (o.tc == 0) sn[o.tr] = n;
#pragma unroll
      for (int v = 0; v < V; ++v) { sm[o.tr * S + o.tc * V + v] = m[v]; sq[o.tr * S + o.tc * V + v] = q[v]; }
    }
    __syncthreads();
    float* out = p.part + (w.tile * p.chunks + w.chunk) * 2 * p.C + w.slice * p.S;
    for (int c = threadIdx.x; c < S; c += ST) {
      float cn = 0.f, cm = 0.f, cq = 0.f;
      for (int r = 0; r < o.rpp; ++r) merge(cn, cm, cq, sn[r], sm[r * S + c], sq[r * S + c]);
      out[c] = cm;
      out[p.C + c] = cq;
    }
    __syncthreads();
  }
}

__device__ __forceinline__ double block_sum(double v, double* red) {
#pragma unroll
  for (int k = 32; k > 0; k >>= 1) v += __shfl_xor(v, k, 64);
  __syncthreads();
  if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = v;
  __syncthreads();
  return red[0] + red[1] + red[2] + red[3];
}

// mean and rstd of a group from the partials of its channels and chunks
__global__ void __launch_bounds__(256) gn_stat_group_k(P p) {
  __shared__ double red[4];
  for (long long u = blockIdx.x; u < p.n * p.G; u += gridDim.x) {
    const long long tile = u / p.G;
    const int gr = (int)(u - tile * p.G);
    const float* part = p.part + tile * p.chunks * 2 * p.C + gr * p.per;
    const int all = p.chunks * p.per;
    double s = 0.0;
    for (int i = threadIdx.x; i < all; i += 256) {
      const int k = i / p.per, c = i - k * p.per;
      const int rows = p.hw - k * p.rows_chunk < p.rows_chunk ? p.hw - k * p.rows_chunk : p.rows_chunk;
      s += (double)rows * (double)part[(long long)k * 2 * p.C + c];
    }
    const double count = (double)p.hw * p.per, mean = block_sum(s, red) / count;
    double q = 0.0;
    for (int i = threadIdx.x; i < all; i += 256) {
      const int k = i / p.per, c = i - k * p.per;
      const int rows = p.hw - k * p.rows_chunk < p.rows_chunk ? p.hw - k * p.rows_chunk : p.rows_chunk;
      const double d = (double)part[(long long)k * 2 * p.C + c] - mean;
      q += (double)part[((long long)k * 2 + 1) * p.C + c] + d * d * rows;
    }
    q = block_sum(q, red);
    if (threadIdx.x == 0) {
      p.g.mean[u] = (float)mean;
      p.g.rstd[u] = (float)(1.0 / sqrt(q / count + (double)p.g.s.eps));
    }
    __syncthreads();
  }
}

template <int V>
__device__ __forceinline__ void group_stats(const P& p, long long tile, int c0, float (&mean)[V], float (&rstd)[V]) {
#pragma unroll
  for (int v = 0; v < V; ++v) {
    const long long at = tile * p.G + (c0 + v) / p.per;
    mean[v] = p.g.mean[at];
    rstd[v] = p.g.rstd[at];
  }
}

template <typename T, int V>
__global__ void __launch_bounds__(ST) gn_apply_k(P p) {
  const GroupNorm& g = p.g;
  for (long long unit = blockIdx.x; unit < p.n * p.chunks * p.slices; unit += gridDim.x) {
    const Where w = where(p, unit);
    const int S = p.C - w.slice * p.S < p.S ? p.C - w.slice * p.S : p.S;
    const Own<V> o(S, ST);
    if (!o.on) continue;
    const int c0 = w.slice * p.S + o.tc * V;
    float mean[V], a[V], bet[V];
    group_stats<V>(p, w.tile, c0, mean, a);
#pragma unroll
    for (int v = 0; v < V; ++v) { a[v] *= g.gamma[c0 + v]; bet[v] = g.beta[c0 + v]; }
#pragma unroll 4
    for (int r = w.lo + o.tr; r < w.hi; r += o.rpp) {
      const long long row = w.tile * p.hw + r;
      Vec<T, V> b;
      float t[V], u[V];
      b.load((const T*)g.x + row * g.ldx + c0);
      b.get(t);
#pragma unroll
      for (int v = 0; v < V; ++v) u[v] = fmaf(t[v] - mean[v], a[v], bet[v]);
      if (g.resid) {
        b.load((const T*)g.resid + row * g.ldr + c0);
        b.get(t);
#pragma unroll
        for (int v = 0; v < V; ++v) u[v] += t[v];
      }
#pragma unroll
      for (int v = 0; v < V; ++v) u[v] = act_any(u[v], g.s.act);
      store_vec((T*)g.y + row * g.ldy + c0, u);
    }
  }
}

// DX false: the chunk's sums of du xhat and du per channel -> part; true: dx (and dresidual) out of the groups' sums
template <typename T, int V, bool X8, bool DX>
__global__ void __launch_bounds__(ST) gn_bwd_split_k(P p) {
  __shared__ __attribute__((aligned(16))) float red[DX ? 1 : ST * V];
  __shared__ float red2[DX ? 1 : ST], ch[DX ? 1 : ST * V];
  const GroupNorm& g = p.g;
  const int act = g.s.act;
  const float inv = 1.0f / ((float)p.hw * (float)p.per);
  for (long long unit = blockIdx.x; unit < p.n * p.chunks * p.slices; unit += gridDim.x) {
    const Where w = where(p, unit);
    const int S = p.C - w.slice * p.S < p.S ? p.C - w.slice * p.S : p.S;
    const Own<V> o(S, ST);
    const int c0 = w.slice * p.S + o.tc * V;
    float mean[V], rstd[V], gam[V], bet[V], s[V], q[V];
#pragma unroll
    for (int v = 0; v < V; ++v) { mean[v] = rstd[v] = gam[v] = bet[v] = s[v] = q[v] = 0.f; }
    if (o.on) {
      group_stats<V>(p, w.tile, c0, mean, rstd);
#pragma unroll
      for (int v = 0; v < V; ++v) {
        gam[v] = g.gamma[c0 + v]; bet[v] = g.beta[c0 + v];
        if constexpr (DX) {
          const float* gsum = p.sums + (w.tile * p.G + (c0 + v) / p.per) * 2;
          q[v] = gsum[0] * inv;   // of du gamma xhat
          s[v] = gsum[1] * inv;   // of du gamma
        }
      }
#pragma unroll 2
      for (int r = w.lo + o.tr; r < w.hi; r += o.rpp) {
        const long long row = w.tile * p.hw + r;
        typename Input<T, V, X8>::type bx;
        Vec<T, V> b;
        float x[V], dy[V], res[V], du[V], xh[V];
        load_in(bx, p, row, c0);
        b.load((const T*)g.dy + row * g.lddy + c0);
        bx.get(x);
        b.get(dy);
#pragma unroll
        for (int v = 0; v < V; ++v) res[v] = 0.f;
        if (g.resid) { b.load((const T*)g.resid + row * g.ldr + c0); b.get(res); }
        du_xhat<V>(x, dy, res, mean, rstd, gam, bet, act, du, xh);
        if constexpr (DX) {
          if (g.dresid) store_vec((T*)g.dresid + row * g.lddr + c0, du);
#pragma unroll
          for (int v = 0; v < V; ++v) du[v] = rstd[v] * ((du[v] * gam[v] - s[v]) - xh[v] * q[v]);
          store_vec((T*)g.y + row * g.ldy + c0, du);
        } else {
#pragma unroll
          for (int v = 0; v < V; ++v) { s[v] += du[v]; q[v] = fmaf(du[v], xh[v], q[v]); }
        }
      }
    }
    if constexpr (!DX) {
      float* out = p.part + (w.tile * p.chunks + w.chunk) * 2 * p.C + w.slice * p.S;
      channel_sums<ST, V>(q, o, S, red, red2, ch);
      for (int c = threadIdx.x; c < S; c += ST) out[c] = ch[c];
      __syncthreads();
      channel_sums<ST, V>(s, o, S, red, red2, ch);
      for (int c = threadIdx.x; c < S; c += ST) out[p.C + c] = ch[c];
      __syncthreads();
    }
  }
}

// sums[tile][group] = sums over chunks and channels of the partials times the gain
__global__ void __launch_bounds__(256) gn_bwd_group_k(P p) {
  __shared__ double red[4];
  for (long long u = blockIdx.x; u < p.n * p.G; u += gridDim.x) {
    const long long tile = u / p.G;
    const int gr = (int)(u - tile * p.G);
    const float* part = p.part + tile * p.chunks * 2 * p.C + gr * p.per;
    double a = 0.0, b = 0.0;
    for (int i = threadIdx.x; i < p.chunks * p.per; i += 256) {
      const int k = i / p.per, c = i - k * p.per;
      const double w = p.g.gamma[gr * p.per + c];
      a += w * (double)part[(long long)k * 2 * p.C + c];
      b += w * (double)part[((long long)k * 2 + 1) * p.C + c];
    }
    a = block_sum(a, red);
    b = block_sum(b, red);
    if (threadIdx.x == 0) { p.sums[u * 2] = (float)a; p.sums[u * 2 + 1] = (float)b; }
    __syncthreads();
  }
}

// ---- host -------------------------------------------------------------------------------------------------------------

constexpr int FWD_E = 49, BWD_E = 20;   // most rows of a thread that stay in registers (bfloat16; float32: half)
constexpr int WANT = 1024;              // workgroups of a split launch

int gcd(int a, int b) { while (b) { const int t = a % b; a = b; b = t; } return a; }

// The channels of a resident slice: whole groups and whole pieces of V, the fewest that are 128 bytes of a row and 256 pieces in all, as
// long as they divide the channels.  0: a unit does not fit.
int resident_slice(const slide_group_norm& s, int V, int es, int most_e, int th) {
  const int per = s.channels / s.groups, base = per / gcd(per, V) * V;   // lcm
  if (base > s.channels || s.channels % base) return 0;
  int pick = 0;
  for (int k = 1; k <= s.channels / base; ++k) {
    if ((s.channels / base) % k) continue;
    const int S = base * k, vpr = S / V;
    if (vpr > th || S / per > th) break;
    const long long rpp = th / vpr, e = (s.hw + rpp - 1) / rpp;
    if (e > most_e) break;
    pick = S;
    if ((long long)S * es >= 128 && s.hw * vpr >= 256) break;
  }
  return pick;
}

int pieces(const GroupNorm& g, bool bwd) {   // 8: every row can be read and written in pieces of eight channels
  const size_t es = elem_size(g.s.dtype);
  auto ok = [&](const void* q, long long ld) { return !q || (((uintptr_t)q & 15) == 0 && ld * es % 16 == 0); };
  bool v = g.s.channels % 8 == 0 && ok(g.y, g.ldy) && ok(g.resid, g.ldr) && ok(g.x, g.ldx);
  if (bwd) v = v && ok(g.dy, g.lddy) && ok(g.dresid, g.lddr);
  return v ? 8 : 1;
}

void split_plan(const slide_group_norm& s, int V, P* p) {
  const int most = ST * V < SMAX ? ST * V : SMAX;
  p->S = s.channels < most ? s.channels : most;
  p->slices = (s.channels + p->S - 1) / p->S;
  const long long have = s.n * p->slices;
  long long chunks = have >= WANT ? 1 : (WANT + have - 1) / have;
  // 16 rows of a thread at least
  const int vpr = p->S / V > 0 ? p->S / V : 1;
  const long long rpp = ST / vpr, by_rows = (s.hw + 16 * rpp - 1) / (16 * rpp);
  if (chunks > by_rows) chunks = by_rows;
  if (chunks < 1) chunks = 1;
  p->rows_chunk = (int)((s.hw + chunks - 1) / chunks);
  p->chunks = (int)((s.hw + p->rows_chunk - 1) / p->rows_chunk);
}

P base(const GroupNorm& g) {
  P p{};
  p.g = g;
  if (g.x8) p.x8 = a8_view(*g.x8);
  p.C = g.s.channels; p.G = g.s.groups; p.per = p.C / p.G; p.hw = (int)g.s.hw; p.n = g.s.n;
  return p;
}

constexpr long long MOST_P = 4096;   // rows of partial sums that the resident backward leaves

size_t part_floats(const slide_group_norm& s) {
  P a{}, b{};
  split_plan(s, 8, &a);
  split_plan(s, 1, &b);
  long long rows = s.n * (a.chunks > b.chunks ? a.chunks : b.chunks);
  return (size_t)rows * 2 * s.channels;
}

template <typename T, int V, int E>
hipError_t fwd_e(const P& p, unsigned grid, bool small, hipStream_t s) {
  if (small) gn_fwd_k<T, V, 256, E><<<grid, 256, 0, s>>>(p);
  else gn_fwd_k<T, V, 512, E><<<grid, 512, 0, s>>>(p);
  return hipGetLastError();
}
template <typename T, int V, int E>
hipError_t bwd_e(const P& p, unsigned grid, bool small, hipStream_t s) {
  if (p.g.x) {
    if (small) gn_bwd_k<T, V, 256, E, false><<<grid, 256, 0, s>>>(p);
    else gn_bwd_k<T, V, 512, E, false><<<grid, 512, 0, s>>>(p);
  } else {
    if (small) gn_bwd_k<T, V, 256, E, true><<<grid, 256, 0, s>>>(p);
    else gn_bwd_k<T, V, 512, E, true><<<grid, 512, 0, s>>>(p);
  }
  return hipGetLastError();
}

unsigned split_grid(const P& p) {
  const long long u = p.n * p.chunks * p.slices;
  return (unsigned)(u < (1 << 20) ? u : (1 << 20));
}
unsigned group_grid(const P& p) {
  const long long u = p.n * p.G;
  return (unsigned)(u < (1 << 20) ? u : (1 << 20));
}

// slice, threads and rows per thread of the resident kernels; false: the unit is split
template <typename T>
bool resident(P* p, int V, int most_e, int* rows, bool* small, unsigned* grid) {
  const slide_group_norm& s = p->g.s;
  p->S = 0;
  // 256 threads with up to eight rows of a thread, else 512
  for (int t = 0; t < 2 && !p->S; ++t) {
    *small = t == 0;
    p->S = resident_slice(s, V, sizeof(T), t == 0 ? (most_e < 8 ? most_e : 8) : most_e, t == 0 ? 256 : 512);
  }
  if (!p->S) return false;
  p->slices = p->C / p->S;
  const int rpp = (*small ? 256 : 512) / (p->S / V);
  *rows = (p->hw + rpp - 1) / rpp;
  p->units_p = (int)(s.n < MOST_P ? s.n : MOST_P);
  *grid = (unsigned)((p->units_p + 7) / 8 * 8 * p->slices);
  return true;
}

template <typename T, int V>
hipError_t fwd(const GroupNorm& g, hipStream_t s) {
  P p = base(g);
  int e;
  bool small;
  unsigned grid;
  constexpr int MOST = V == 1 ? FWD_E : FWD_E / ((int)sizeof(T) / 2);
  if (resident<T>(&p, V, MOST, &e, &small, &grid)) {
    if (e <= 2) return fwd_e<T, V, 2>(p, grid, small, s);
    if (e <= 4) return fwd_e<T, V, 4>(p, grid, small, s);
    if (e <= 8) return fwd_e<T, V, 8>(p, grid, small, s);
    if (e <= 13) return fwd_e<T, V, 13>(p, grid, small, s);
    if (e <= 24) return fwd_e<T, V, 24>(p, grid, small, s);
    if constexpr (MOST > 24) return e <= 36 ? fwd_e<T, V, 36>(p, grid, small, s) : fwd_e<T, V, 49>(p, grid, small, s);
  }
  split_plan(g.s, V, &p);
  p.part = g.work;
  gn_stat_k<T, V><<<split_grid(p), ST, 0, s>>>(p);
  hipError_t err = hipGetLastError();
  if (err != hipSuccess) return err;
  gn_stat_group_k<<<group_grid(p), 256, 0, s>>>(p);
  err = hipGetLastError();
  if (err != hipSuccess) return err;
  gn_apply_k<T, V><<<split_grid(p), ST, 0, s>>>(p);
  return hipGetLastError();
}

template <typename T, int V>
hipError_t bwd(const GroupNorm& g, hipStream_t s) {
  P p = base(g);
  int e;
  bool small;
  unsigned grid;
  long long rows;
  constexpr int MOST = V == 1 ? BWD_E : BWD_E / ((int)sizeof(T) / 2);
  hipError_t err;
  p.part = g.work;
  if (resident<T>(&p, V, MOST, &e, &small, &grid)) {
    rows = p.units_p;
    if (e <= 2) err = bwd_e<T, V, 2>(p, grid, small, s);
    else if (e <= 4) err = bwd_e<T, V, 4>(p, grid, small, s);
    else if (e <= 8) err = bwd_e<T, V, 8>(p, grid, small, s);
    else if constexpr (MOST > 10) err = e <= 13 ? bwd_e<T, V, 13>(p, grid, small, s) : bwd_e<T, V, 20>(p, grid, small, s);
    else err = bwd_e<T, V, 10>(p, grid, small, s);
  } else {
    split_plan(g.s, V, &p);
    rows = p.n * p.chunks;
    p.sums = g.work + part_floats(g.s);
    const unsigned sg = split_grid(p);
    if (g.x) gn_bwd_split_k<T, V, false, false><<<sg, ST, 0, s>>>(p);
    else gn_bwd_split_k<T, V, true, false><<<sg, ST, 0, s>>>(p);
    err = hipGetLastError();
    if (err != hipSuccess) return err;
    gn_bwd_group_k<<<group_grid(p), 256, 0, s>>>(p);
    err = hipGetLastError();
    if (err != hipSuccess) return err;
    if (g.x) gn_bwd_split_k<T, V, false, true><<<sg, ST, 0, s>>>(p);
    else gn_bwd_split_k<T, V, true, true><<<sg, ST, 0, s>>>(p);
    err = hipGetLastError();
  }
  if (err != hipSuccess) return err;
  gn_sum_k<<<(p.C + 15) / 16, 1024, 0, s>>>(p.part, rows, p.C, g.dgamma, g.dbeta, g.accumulate);
  return hipGetLastError();
}

}  // namespace

size_t group_norm_bytes(const slide_group_norm& s) {
  return ((part_floats(s) + (size_t)s.n * s.groups * 2) * 4 + 255) & ~(size_t)255;
}

hipError_t launch_group_norm_fwd(const GroupNorm& g, hipStream_t s) {
  const int V = pieces(g, false);
  if (g.x8) {   // before y, which may be x, is written
    const hipError_t e = launch_act8_pack(g.x, g.s.dtype, g.ldx, false, *g.x8, s);
    if (e != hipSuccess) return e;
  }
  if (g.s.dtype == DT_F32) return V == 8 ? fwd<float, 8>(g, s) : fwd<float, 1>(g, s);
  return V == 8 ? fwd<bf16, 8>(g, s) : fwd<bf16, 1>(g, s);
}

hipError_t launch_group_norm_bwd(const GroupNorm& g, hipStream_t s) {
  const int V = pieces(g, true);
  if (g.s.dtype == DT_F32) return V == 8 ? bwd<float, 8>(g, s) : bwd<float, 1>(g, s);
  return V == 8 ? bwd<bf16, 8>(g, s) : bwd<bf16, 1>(g, s);
}

}  // namespace sl
