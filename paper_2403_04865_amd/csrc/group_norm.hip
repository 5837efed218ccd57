// Group normalisation with its activation over channels-last tiles, forward and backward (gfx950).
//
// A unit is one tile's slice of whole groups.  Bound by memory traffic: forward x in, y out (and one byte of checkpoint), backward
// dy and x in, dx out; everything else is to keep a value from being read twice.
//   * One workgroup per unit.  Statistics of every thread's rows (count, mean, sum of squared distances, two rows at a time, merged), of the
//     groups out of these, then the result: the unit is read twice, the second time out of the caches, and rows that fit the
//     registers once.  The backward likewise: the two sums that dx needs of each group, then dx.
//   * Few large units are split over rows: partial statistics per channel (count, mean, sum of squared distances: merged, never a
//     difference of large sums), one small kernel for the groups, one pass for the result.
// Measured (bfloat16, us; in brackets the bytes that must move at the 5.16 TB/s of a copy): 1024 x 56 x 56 x 64 with SiLU: forward with
// checkpoint 259 (199), backward out of it 303 (199), a unit of 0.6 MB being read twice, 5 TB/s in all; 1024 x 28 x 28 x 128, ReLU and
// residual, backward 269 (199); split, 2 x 300 x 301 x 320 with GELU: 45 + 9 + 53 forward (79), 53 + 7 + 58 backward (56; GELU's slope twice).
// Keeping more of a unit (in LDS: a third of the second reading) gained 3 %, more workgroups per unit of the chip lost 15 %.
// A thread owns V neighbouring channels (16 bytes of bfloat16) and strides over rows.  All statistics and sums are float32; the
// gradients of gain and shift add the workgroups' sums in double, in a fixed order.
#include "act8_internal.h"
#include "lds_dma.h"

namespace sl {

namespace {

// V values of a row as they are in memory.
template <typename T, int V> struct Vec;
template <> struct Vec<bf16, 8> {
  u32x4 r;
  __device__ __forceinline__ void load(const bf16* p) { r = *reinterpret_cast<const u32x4*>(p); }
  __device__ __forceinline__ void load(__amdgpu_buffer_rsrc_t b, int v, int s) { r = __builtin_amdgcn_raw_buffer_load_b128(b, v, s, 0); }
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
  u32x4 lo, hi;
  __device__ __forceinline__ void load(const float* p) {
    lo = *reinterpret_cast<const u32x4*>(p); hi = *reinterpret_cast<const u32x4*>(p + 4);
  }
  __device__ __forceinline__ void load(__amdgpu_buffer_rsrc_t b, int v, int s) {
    lo = __builtin_amdgcn_raw_buffer_load_b128(b, v, s, 0);
    hi = __builtin_amdgcn_raw_buffer_load_b128(b, v + 16, s, 0);
  }
  __device__ __forceinline__ void zero() { lo = hi = u32x4{0, 0, 0, 0}; }
  __device__ __forceinline__ void get(float (&v)[8]) const {
#pragma unroll
    for (int e = 0; e < 4; ++e) { v[e] = __uint_as_float(lo[e]); v[4 + e] = __uint_as_float(hi[e]); }
  }
};
template <> struct Vec<bf16, 1> {
  unsigned short r;
  __device__ __forceinline__ void load(const bf16* p) { r = *reinterpret_cast<const unsigned short*>(p); }
  __device__ __forceinline__ void load(__amdgpu_buffer_rsrc_t b, int v, int s) { r = __builtin_amdgcn_raw_buffer_load_b16(b, v, s, 0); }
  __device__ __forceinline__ void zero() { r = 0; }
  __device__ __forceinline__ void get(float (&v)[1]) const { v[0] = __uint_as_float((unsigned)r << 16); }
};
template <> struct Vec<float, 1> {
  unsigned r;
  __device__ __forceinline__ void load(const float* p) { r = *reinterpret_cast<const unsigned*>(p); }
  __device__ __forceinline__ void load(__amdgpu_buffer_rsrc_t b, int v, int s) { r = __builtin_amdgcn_raw_buffer_load_b32(b, v, s, 0); }
  __device__ __forceinline__ void zero() { r = 0; }
  __device__ __forceinline__ void get(float (&v)[1]) const { v[0] = __uint_as_float(r); }
};
template <typename T, int V> __device__ __forceinline__ void less_of(const Vec<T, V>& b, const float (&m)[V], float (&v)[V]) {
  b.get(v);
#pragma unroll
  for (int e = 0; e < V; ++e) v[e] -= m[e];
}
__device__ __forceinline__ u32x4 rounded(const float (&v)[8]) {
  bf16x8 t;
#pragma unroll
  for (int e = 0; e < 8; ++e) t[e] = (bf16)v[e];
  return __builtin_bit_cast(u32x4, t);
}
__device__ __forceinline__ void store_vec(bf16* p, const float (&v)[8]) { *reinterpret_cast<u32x4*>(p) = rounded(v); }
__device__ __forceinline__ void store_vec(float* p, const float (&v)[8]) {
  *reinterpret_cast<f32x4*>(p) = f32x4{v[0], v[1], v[2], v[3]};
  *reinterpret_cast<f32x4*>(p + 4) = f32x4{v[4], v[5], v[6], v[7]};
}
template <typename T> __device__ __forceinline__ void store_vec(T* p, const float (&v)[1]) { *p = from_f<T>(v[0]); }
template <typename T> __device__ __forceinline__ void store_buf(__amdgpu_buffer_rsrc_t b, int o, int s, const float (&v)[8]) {
  if constexpr (sizeof(T) == 2) store16(rounded(v), b, o + s);
  else {
    u32x4 lo, hi;
#pragma unroll
    for (int e = 0; e < 4; ++e) { lo[e] = __float_as_uint(v[e]); hi[e] = __float_as_uint(v[4 + e]); }
    store16(lo, b, o + s);
    store16(hi, b, o + s + 16);
  }
}
template <typename T> __device__ __forceinline__ void store_buf(__amdgpu_buffer_rsrc_t b, int o, int s, const float (&v)[1]) {
  if constexpr (sizeof(T) == 2) __builtin_amdgcn_raw_buffer_store_b16(__builtin_bit_cast(unsigned short, (bf16)v[0]), b, o, s, 0);
  else __builtin_amdgcn_raw_buffer_store_b32(__float_as_uint(v[0]), b, o, s, 0);
}

// eight codes of a checkpoint and their scale byte, or (V = 1) one
template <int V> struct Vec8;
template <> struct Vec8<8> {
  u32x2 q; unsigned b;
  __device__ __forceinline__ void load(const A8& a, long long row, int c) {
    q = *reinterpret_cast<const u32x2*>(a.codes + row * a.ldc + c);
    b = a.scales[row * a.lds + (c >> 7)];
  }
  __device__ __forceinline__ void load(__amdgpu_buffer_rsrc_t c, int v, int s, __amdgpu_buffer_rsrc_t sc, int vs, int ss) {
    q = __builtin_amdgcn_raw_buffer_load_b64(c, v, s, 0);
    b = __builtin_amdgcn_raw_buffer_load_b8(sc, vs, ss, 0);
  }
  // the values less m: a code times its power is exact, so this rounds once, as a difference of the values does
  __device__ __forceinline__ void less(const float (&m)[8], float (&v)[8]) const {
    const float s = a8_scale(b);
    float t[4];
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      a8_value4(q[h], 1.f, t);
#pragma unroll
      for (int e = 0; e < 4; ++e) v[4 * h + e] = fmaf(t[e], s, -m[4 * h + e]);
    }
  }
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
  __device__ __forceinline__ void load(__amdgpu_buffer_rsrc_t c, int v, int s, __amdgpu_buffer_rsrc_t sc, int vs, int ss) {
    q = __builtin_amdgcn_raw_buffer_load_b8(c, v, s, 0);
    b = __builtin_amdgcn_raw_buffer_load_b8(sc, vs, ss, 0);
  }
  __device__ __forceinline__ void get(float (&v)[1]) const { v[0] = __builtin_amdgcn_cvt_f32_fp8((int)q, 0) * a8_scale(b); }
  __device__ __forceinline__ void less(const float (&m)[1], float (&v)[1]) const { get(v); v[0] -= m[0]; }
};

template <int V> __device__ __forceinline__ void less_of(const Vec8<V>& b, const float (&m)[V], float (&v)[V]) { b.less(m, v); }

// act: uniform, one branch for all V values
template <int V> __device__ __forceinline__ void act_vec(float (&u)[V], int act) {
  switch (act) {
    case SLIDE_ACT_RELU:
#pragma unroll
      for (int v = 0; v < V; ++v) u[v] = act_f<SLIDE_ACT_RELU>(u[v]);
      break;
    case SLIDE_ACT_SILU:
#pragma unroll
      for (int v = 0; v < V; ++v) u[v] = act_f<SLIDE_ACT_SILU>(u[v]);
      break;
    case SLIDE_ACT_GELU:
#pragma unroll
      for (int v = 0; v < V; ++v) u[v] = act_f<SLIDE_ACT_GELU>(u[v]);
      break;
    default: break;
  }
}

struct P {
  GroupNorm g;
  A8 x8;
  int S, slices, G, per, C, hw;   // channels of a slice, slices, groups, channels of a group
  long long n;
  int rows;                       // rows of a thread (unit kernels)
  int pack;                       // lanes of a block of the checkpoint that the forward writes; 0: it writes none
  int units_p;                    // workgroups per slice that share out the tiles (unit kernels)
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

// (count, mean, squared distances) of two disjoint sets, merged into the first
__device__ __forceinline__ void merge(float& n, float& m, float& q, float nb, float mb, float qb) {
  const float t = n + nb;
  if (t == 0.f) return;
  const float d = mb - m, f = nb / t;
  m = fmaf(d, f, m);
  q += qb + d * d * n * f;
  n = t;
}

// Sums over the rows of the workgroup: s[V] per thread -> ch[S] per channel of the slice.  red: TH V floats, red2: TH floats.  Ends with
// a barrier.
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

// Sums over each group of the slice of NS values s[i][V] per thread -> gs[i][groups].  A thread adds its channels of one group first: W
// neighbouring channels always are of one group (8, 4 or 2, dividing the group's channels or divided by them; else 1).  red: NS TH V
// floats.  Ends with a barrier.
constexpr int SMAX = 512;   // most channels of a unit's slice

template <int TH, int V, int NS>
__device__ __forceinline__ void group_sums(const float (&s)[NS][V], const Own<V>& o, int S, int per, float* red, float (*gs)[SMAX]) {
  const int gl = S / per;
  int slots = S;   // per row of threads
  auto put = [&](auto width) {
    constexpr int W = decltype(width)::value;
    slots = S / W;
    if (!o.on) return;
#pragma unroll
    for (int i = 0; i < NS; ++i)
#pragma unroll
      for (int h = 0; h < V / W; ++h) {
        float a = 0.f;
#pragma unroll
        for (int v = 0; v < W; ++v) a += s[i][h * W + v];
        red[i * TH * V + o.tr * slots + o.tc * (V / W) + h] = a;
      }
  };
  if (V == 8 && per % 8 == 0) put(std::integral_constant<int, V>{});
  else if (V == 8 && per % 4 == 0) put(std::integral_constant<int, V == 8 ? 4 : 1>{});
  else if (V == 8 && per % 2 == 0) put(std::integral_constant<int, V == 8 ? 2 : 1>{});
  else put(std::integral_constant<int, 1>{});
  __syncthreads();
  int L = 64;
  while (L > 1 && L * gl > TH) L >>= 1;
  const int sub = (int)threadIdx.x / L, lane = (int)threadIdx.x & (L - 1), sg = slots / gl, all = o.rpp * sg;
  for (int g = sub; g < gl; g += TH / L) {
    float a[NS];
#pragma unroll
    for (int i = 0; i < NS; ++i) a[i] = 0.f;
    for (int k = lane; k < all; k += L) {
      const int r = k / sg, at = r * slots + g * sg + (k - r * sg);
#pragma unroll
      for (int i = 0; i < NS; ++i) a[i] += red[i * TH * V + at];
    }
    for (int k = L >> 1; k > 0; k >>= 1)
#pragma unroll
      for (int i = 0; i < NS; ++i) a[i] += __shfl_xor(a[i], k, 64);
    if (lane == 0)
#pragma unroll
      for (int i = 0; i < NS; ++i) gs[i][g] = a[i];
  }
  __syncthreads();
}

// ---- a workgroup per unit ----------------------------------------------------------------------------------------------

constexpr int RG = 2;   // rows whose loads are in flight together, and whose statistics are formed together
// Rows are taken one after the other: interleaved by the compiler they took twice the registers (and spilled).
__device__ __forceinline__ void row_end() { __builtin_amdgcn_sched_barrier(0); }

// a tile's rows of S channels from p on; rows behind the last are outside, whatever is loaded from there is zero and nothing is stored
__device__ __forceinline__ __amdgpu_buffer_rsrc_t tile_buffer(const void* p, long long ld, int es, int hw, int S) {
  return dma_buffer(p, p ? ((hw - 1) * ld + S) * es : 0);
}

// V per-channel values of this thread
template <int V> __device__ __forceinline__ void mine(const float* ch, int c, float (&v)[V]) {
#pragma unroll
  for (int k = 0; k < V; ++k) v[k] = ch[c + k];
}

// KG: groups of RG rows of a thread that stay in registers
template <typename T, int V, int TH, int KG>
__global__ void __launch_bounds__(TH, 4) gn_fwd_k(P p) {
  __shared__ float red[TH * V], gs[1][SMAX], cm[SMAX], cg[SMAX], ca[SMAX], cb[SMAX];
  const GroupNorm& g = p.g;
  const Own<V> o(p.S, TH);
  const int j = blockIdx.x >> 3, slice = j % p.slices, first = (int)(blockIdx.x & 7) + 8 * (j / p.slices);
  if (first >= p.units_p) return;
  const int s0 = slice * p.S, tc = o.tc * V, at = o.on ? tc : 0, per = p.per, gl = p.S / per;
  const float count = (float)p.hw * (float)per;
  constexpr int es = sizeof(T);
  const int ldx = (int)g.ldx * es, ldy = (int)g.ldy * es, ldr = (int)g.ldr * es;
  const int vx = o.on ? o.tr * ldx + tc * es : DMA_ABSENT, vy = o.on ? o.tr * ldy + tc * es : DMA_ABSENT, vr = o.on ? o.tr * ldr + tc * es : DMA_ABSENT;
  for (int c = threadIdx.x; c < p.S; c += TH) { cg[c] = g.gamma[s0 + c]; cb[c] = g.beta[s0 + c]; }
  for (long long tile = first; tile < p.n; tile += p.units_p) {
    const long long r0 = tile * p.hw;
    const __amdgpu_buffer_rsrc_t xb = tile_buffer((const T*)g.x + r0 * g.ldx + s0, g.ldx, es, p.hw, p.S);
    const __amdgpu_buffer_rsrc_t cbuf = tile_buffer(p.pack ? p.x8.codes + r0 * p.x8.ldc + s0 : nullptr, p.x8.ldc, 1, p.hw, p.S);
    const __amdgpu_buffer_rsrc_t sbuf = tile_buffer(p.pack ? p.x8.scales + r0 * p.x8.lds + (s0 >> 7) : nullptr, p.x8.lds, 1, p.hw, (p.S + 127) >> 7);
    const int ldc = (int)p.x8.ldc, lds = (int)p.x8.lds;
    const int vc = o.on ? o.tr * ldc + tc : DMA_ABSENT, vs = o.on && (o.tc & (p.pack - 1)) == 0 ? o.tr * lds + (tc >> 7) : DMA_ABSENT;
    Vec<T, V> buf[KG][RG];
    auto load = [&](Vec<T, V> (&b)[RG], int e) __attribute__((always_inline)) {
#pragma unroll
      for (int k = 0; k < RG; ++k) b[k].load(xb, vx, (e + k) * o.rpp * ldx);
    };
    // the rows that are not kept, the next ones on their way while these are worked on (behind the last row: zeros)
    auto again = [&](auto f) __attribute__((always_inline)) {
      if (KG * RG >= p.rows) return;
      Vec<T, V> b[2][RG];
      load(b[0], KG * RG);
      for (int e = KG * RG; e < p.rows; e += 2 * RG) {
        load(b[1], e + RG);
        row_end();
        f(b[0], e);
        load(b[0], e + 2 * RG);
        row_end();
        if (e + RG < p.rows) f(b[1], e + RG);
      }
    };
    // ---- statistics of this thread's rows
    float n = 0.f, m[V], q[1][V], s[1][V];
#pragma unroll
    for (int v = 0; v < V; ++v) m[v] = q[0][v] = 0.f;
    auto stat = [&](const Vec<T, V> (&b)[RG], int e) __attribute__((always_inline)) {
      float l[V], d2[V];
#pragma unroll
      for (int v = 0; v < V; ++v) l[v] = d2[v] = 0.f;
#pragma unroll
      for (int k = 0; k < RG; ++k) {
        float t[V];
        b[k].get(t);
#pragma unroll
        for (int v = 0; v < V; ++v) l[v] += t[v];
        if (V == 8 && p.pack) {   // uniform
          if constexpr (V == 8) {
            const unsigned sc = a8_block_byte(t, p.pack);
            const float inv = a8_inverse(sc);
            u32x2 w;
            w[0] = a8_code4(t[0] * inv, t[1] * inv, t[2] * inv, t[3] * inv);
            w[1] = a8_code4(t[4] * inv, t[5] * inv, t[6] * inv, t[7] * inv);
            __builtin_amdgcn_raw_buffer_store_b64(w, cbuf, vc, (e + k) * o.rpp * ldc, 0);
            __builtin_amdgcn_raw_buffer_store_b8((unsigned char)sc, sbuf, vs, (e + k) * o.rpp * lds, 0);
          }
        }
      }
      // rows of these that exist; where all do (uniform) nothing is left out
      int have = 0;
#pragma unroll
      for (int k = 0; k < RG; ++k) have += o.on && o.tr + (e + k) * o.rpp < p.hw;
      const float nb = (float)have, inv = have ? 1.0f / nb : 0.f;
#pragma unroll
      for (int v = 0; v < V; ++v) l[v] *= inv;
      const bool whole = (e + RG) * o.rpp <= p.hw;
#pragma unroll
      for (int k = 0; k < RG; ++k) {
        float t[V];
        b[k].get(t);
        if (!whole && k >= have) continue;   // (a thread's rows exist up to some row)
#pragma unroll
        for (int v = 0; v < V; ++v) { const float d = t[v] - l[v]; d2[v] = fmaf(d, d, d2[v]); }
      }
      const float all = n + nb, f = all > 0.f ? nb / all : 0.f, nf = n * f;
#pragma unroll
      for (int v = 0; v < V; ++v) {
        const float d = l[v] - m[v];
        m[v] = fmaf(d, f, m[v]);
        q[0][v] += fmaf(d * d, nf, d2[v]);
      }
      n = all;
      row_end();
    };
#pragma unroll
    for (int h = 0; h < KG; ++h)
      if (h * RG < p.rows) load(buf[h], h * RG);
#pragma unroll
    for (int h = 0; h < KG; ++h)
      if (h * RG < p.rows) stat(buf[h], h * RG);
    again([&](const Vec<T, V> (&b)[RG], int e) __attribute__((always_inline)) { stat(b, e); });
    // ---- of the groups
#pragma unroll
    for (int v = 0; v < V; ++v) s[0][v] = n * m[v];
    group_sums<TH, V, 1>(s, o, p.S, per, red, gs);
    for (int c = threadIdx.x; c < p.S; c += TH) cm[c] = gs[0][c / per] / count;
    for (int k = threadIdx.x; k < gl; k += TH) g.mean[tile * p.G + slice * gl + k] = gs[0][k] / count;   // (more groups than threads: a channel each)
    __syncthreads();
    float mean[V];
    mine<V>(cm, at, mean);
#pragma unroll
    for (int v = 0; v < V; ++v) { const float d = m[v] - mean[v]; s[0][v] = fmaf(d * d, n, q[0][v]); }
    group_sums<TH, V, 1>(s, o, p.S, per, red, gs);
    for (int c = threadIdx.x; c < p.S; c += TH) ca[c] = cg[c] * (1.0f / sqrtf(gs[0][c / per] / count + g.s.eps));
    for (int k = threadIdx.x; k < gl; k += TH) g.rstd[tile * p.G + slice * gl + k] = 1.0f / sqrtf(gs[0][k] / count + g.s.eps);
    __syncthreads();
    // ---- the result
    const __amdgpu_buffer_rsrc_t yb = tile_buffer((T*)g.y + r0 * g.ldy + s0, g.ldy, es, p.hw, p.S);
    const __amdgpu_buffer_rsrc_t rb = tile_buffer(g.resid ? (const T*)g.resid + r0 * g.ldr + s0 : nullptr, g.ldr, es, p.hw, p.S);
    float a[V], b[V];
    mine<V>(ca, at, a);
    mine<V>(cb, at, b);
    auto apply = [&](const Vec<T, V> (&x)[RG], int e) __attribute__((always_inline)) {
      Vec<T, V> w[RG];
      if (g.resid) {
#pragma unroll
        for (int k = 0; k < RG; ++k) w[k].load(rb, vr, (e + k) * o.rpp * ldr);
      }
#pragma unroll
      for (int k = 0; k < RG; ++k) {
        float t[V], u[V];
        x[k].get(t);
#pragma unroll
        for (int v = 0; v < V; ++v) u[v] = fmaf(t[v] - mean[v], a[v], b[v]);
        if (g.resid) {
          w[k].get(t);
#pragma unroll
          for (int v = 0; v < V; ++v) u[v] += t[v];
        }
        act_vec<V>(u, g.s.act);
        store_buf<T>(yb, vy, (e + k) * o.rpp * ldy, u);
        row_end();
      }
    };
#pragma unroll
    for (int h = 0; h < KG; ++h)
      if (h * RG < p.rows) apply(buf[h], h * RG);
    again([&](const Vec<T, V> (&b)[RG], int e) __attribute__((always_inline)) { apply(b, e); });
    __syncthreads();   // (cm, ca, gs are written again by the next tile)
  }
}

// The third matrix that a backward reads: none, the residual, or (rectifiers only) what the forward put out, which says where it let
// values through.  Then du = dy where that is positive, and neither the sum nor its residual is formed.
enum Third { NONE, RESID, OUT };

// du = dy act'(u) of V values, u = (x - mean) (rstd gamma) + beta + residual.  A rectifier asks which side of zero u is on: where float32
// cannot tell, it is formed again in double (mean and rstd are what the forward stored).  The kernels of that branch are their own
// (RELU): in the others it would cost up to 50 registers (1024 tiles of 56 x 56 x 64, SiLU out of a checkpoint: 340 us with it, 310 without).
template <Third RES, bool RELU, int V, typename F>
__device__ __forceinline__ void du_vec(const float (&d)[V], const float (&dy)[V], const float (&rg)[V], const float (&bet)[V], const float (&res)[V],
                                       int act, float (&du)[V], F exactly) {
  if constexpr (RES == OUT) {
#pragma unroll
    for (int v = 0; v < V; ++v) du[v] = res[v] > 0.f ? dy[v] : 0.f * dy[v];
    return;
  }
  if (!RELU && act == SLIDE_ACT_NONE) {
#pragma unroll
    for (int v = 0; v < V; ++v) du[v] = dy[v];
    return;
  }
  float u[V];
#pragma unroll
  for (int v = 0; v < V; ++v) u[v] = fmaf(d[v], rg[v], bet[v]);
  if constexpr (RES != NONE) {
#pragma unroll
    for (int v = 0; v < V; ++v) u[v] += res[v];
  }
  if constexpr (RELU) {
    // u is off by less than 1e-6 of its parts' magnitudes; where it is as small as that, the first part is as large as the others
    bool near = false;
#pragma unroll
    for (int v = 0; v < V; ++v) near |= fabsf(u[v]) <= 2.1e-6f * (RES != NONE ? fabsf(bet[v]) + fabsf(res[v]) : fabsf(bet[v]));
    if (near) {
#pragma unroll
      for (int v = 0; v < V; ++v) { u[v] = exactly(v); __builtin_amdgcn_sched_barrier(0); }
    }
#pragma unroll
    for (int v = 0; v < V; ++v) du[v] = u[v] > 0.f ? dy[v] : 0.f * dy[v];
  } else if (act == SLIDE_ACT_SILU) {
#pragma unroll
    for (int v = 0; v < V; ++v) {   // s (1 + u (1 - s))
      const float s = sigmoid_f(u[v]);
      du[v] = dy[v] * fmaf(u[v] * s, 1.0f - s, s);
    }
  } else {
#pragma unroll
    for (int v = 0; v < V; ++v) {   // Phi(u) + u phi(u)
      float e;
      const float h = half_erfc(fminf(fabsf(u[v]), GELU_FAR), &e);
      du[v] = dy[v] * fmaf(u[v] * 0.39894228040143268f, e, u[v] < 0.f ? h : 1.0f - h);
    }
  }
}

// X8: the input is the checkpoint
template <typename T, int V, bool X8> struct Input { typedef Vec<T, V> type; };
template <typename T, int V> struct Input<T, V, true> { typedef Vec8<V> type; };
template <typename T, int V>
__device__ __forceinline__ void load_in(Vec<T, V>& b, const P& p, long long row, int c) { b.load((const T*)p.g.x + row * p.g.ldx + c); }
template <int V>
__device__ __forceinline__ void load_in(Vec8<V>& b, const P& p, long long row, int c) { b.load(p.x8, row, c); }

// sign of x's place before the activation, in double
__device__ __forceinline__ float side(double x, double mean, double rstd, double gam, double bet, double res) {
  const double u = (x - mean) * rstd * gam + bet + res;
  return u > 0.0 ? 1.f : u < 0.0 ? -1.f : (float)u;
}

template <typename T, int V, int TH, int KG, bool X8, Third RES, bool RELU>
__global__ void __launch_bounds__(TH, 2) gn_bwd_k(P p) {
  __shared__ float red[2 * TH * V], gs[2][SMAX], cm[SMAX], cr[SMAX], crg[SMAX], cbet[SMAX], red2[TH];
  const GroupNorm& g = p.g;
  const Own<V> o(p.S, TH);
  const int j = blockIdx.x >> 3, slice = j % p.slices, first = (int)(blockIdx.x & 7) + 8 * (j / p.slices);
  if (first >= p.units_p) return;
  const int s0 = slice * p.S, tc = o.tc * V, at = o.on ? tc : 0, per = p.per, act = g.s.act, gl = p.S / per;
  const float inv = 1.0f / ((float)p.hw * (float)per);
  constexpr int es = sizeof(T), esx = X8 ? 1 : es;
  const int ldx = X8 ? (int)p.x8.ldc : (int)g.ldx * es, lds = (int)p.x8.lds;
  const int ldd = (int)g.lddy * es, ldy = (int)g.ldy * es, ldr = (int)g.ldr * es, ldq = (int)g.lddr * es;
  auto lane_at = [&](int ld, int c) { return o.on ? o.tr * ld + c : DMA_ABSENT; };
  const int vx = lane_at(ldx, tc * esx), vs = lane_at(lds, (s0 + tc) / A8_BLOCK), vd = lane_at(ldd, tc * es), vy = lane_at(ldy, tc * es),
            vr = lane_at(ldr, tc * es), vq = lane_at(ldq, tc * es);
  float tg[V], tb[V];   // this thread's sums for the gain and the shift, over all of its tiles
#pragma unroll
  for (int v = 0; v < V; ++v) tg[v] = tb[v] = 0.f;
  for (int c = threadIdx.x; c < p.S; c += TH) cbet[c] = g.beta[s0 + c];
  for (long long tile = first; tile < p.n; tile += p.units_p) {
    const long long r0 = tile * p.hw;
    const __amdgpu_buffer_rsrc_t xb = X8 ? tile_buffer(p.x8.codes + r0 * p.x8.ldc + s0, p.x8.ldc, 1, p.hw, p.S)
                                         : tile_buffer((const T*)g.x + r0 * g.ldx + s0, g.ldx, es, p.hw, p.S);
    const __amdgpu_buffer_rsrc_t sb = tile_buffer(X8 ? p.x8.scales + r0 * p.x8.lds : nullptr, p.x8.lds, 1, p.hw, (p.C + 127) >> 7);
    const __amdgpu_buffer_rsrc_t db = tile_buffer((const T*)g.dy + r0 * g.lddy + s0, g.lddy, es, p.hw, p.S);
    const __amdgpu_buffer_rsrc_t rb = tile_buffer(RES != NONE ? (const T*)g.resid + r0 * g.ldr + s0 : nullptr, g.ldr, es, p.hw, p.S);
    typedef typename Input<T, V, X8>::type In;
    struct Rows { In x[RG]; Vec<T, V> d[RG], w[RES != NONE ? RG : 1]; } kept[KG];
    auto load = [&](Rows& b, int e) __attribute__((always_inline)) {
#pragma unroll
      for (int k = 0; k < RG; ++k) {
        const int row = (e + k) * o.rpp;
        if constexpr (X8) b.x[k].load(xb, vx, row * ldx, sb, vs, row * lds);
        else b.x[k].load(xb, vx, row * ldx);
        b.d[k].load(db, vd, row * ldd);
        if constexpr (RES != NONE) b.w[k].load(rb, vr, row * ldr);
      }
    };
#pragma unroll
    for (int h = 0; h < KG; ++h)
      if (h * RG < p.rows) load(kept[h], h * RG);
    for (int c = threadIdx.x; c < p.S; c += TH) {
      const long long k = tile * p.G + slice * gl + c / per;
      const float r = g.rstd[k];
      cm[c] = g.mean[k]; cr[c] = r; crg[c] = r * g.gamma[s0 + c];
    }
    __syncthreads();
    float m[V], rg[V], bet[V];
    mine<V>(cm, at, m);
    mine<V>(crg, at, rg);
    mine<V>(cbet, at, bet);
    // f(x - mean, du, row index) of RG rows
    auto take = [&](const Rows& b, int e, auto f) __attribute__((always_inline)) {
#pragma unroll
      for (int k = 0; k < RG; ++k) {
        float dy[V], res[V], d[V], du[V];
        less_of<>(b.x[k], m, d);
        b.d[k].get(dy);
        if constexpr (RES != NONE) b.w[k].get(res);
        du_vec<RES, RELU, V>(d, dy, rg, bet, res, act, du, [&](int v) __attribute__((always_inline)) {
          float x[V];
          b.x[k].get(x);
          return side(x[v], m[v], cr[at + v], g.gamma[s0 + at + v], bet[v], RES != NONE ? res[v] : 0.f);
        });
        f(d, du, e + k);
        row_end();
      }
    };
    auto each = [&](auto f) __attribute__((always_inline)) {
      Rows b[2];   // the next rows are on their way while these are worked on (behind the last row: zeros)
      const bool more = KG * RG < p.rows;
      if (more) load(b[0], KG * RG);
      row_end();
#pragma unroll
      for (int h = 0; h < KG; ++h)
        if (h * RG < p.rows) take(kept[h], h * RG, f);
      if (!more) return;
      for (int e = KG * RG; e < p.rows; e += 2 * RG) {
        load(b[1], e + RG);
        row_end();
        take(b[0], e, f);
        load(b[0], e + 2 * RG);
        row_end();
        if (e + RG < p.rows) take(b[1], e + RG, f);
      }
    };
    float s[V], q[V];
#pragma unroll
    for (int v = 0; v < V; ++v) s[v] = q[v] = 0.f;
    each([&](const float (&d)[V], const float (&du)[V], int) __attribute__((always_inline)) {   // (dy of a row that does not exist is zero)
#pragma unroll
      for (int v = 0; v < V; ++v) { s[v] += du[v]; q[v] = fmaf(du[v], d[v], q[v]); }
    });
    float r[V], w[2][V];
    mine<V>(cr, at, r);
#pragma unroll
    for (int v = 0; v < V; ++v) {
      tb[v] += s[v];
      tg[v] = fmaf(q[v], r[v], tg[v]);
      w[0][v] = s[v] * rg[v];           // of du gamma, times rstd
      w[1][v] = q[v] * rg[v] * r[v];    // of du gamma xhat, times rstd
    }
    group_sums<TH, V, 2>(w, o, p.S, per, red, gs);
    // dx = rstd (du gamma - mean of it - xhat mean of (du gamma xhat)) = du (rstd gamma) - k1 - (x - mean) k2
    float k1[V], k2[V];
#pragma unroll
    for (int v = 0; v < V; ++v) {
      const int gr = (at + v) / per;
      k1[v] = gs[0][gr] * inv;
      k2[v] = gs[1][gr] * inv * r[v];
    }
    const __amdgpu_buffer_rsrc_t yb = tile_buffer((T*)g.y + r0 * g.ldy + s0, g.ldy, es, p.hw, p.S);
    const __amdgpu_buffer_rsrc_t qb = tile_buffer(g.dresid ? (T*)g.dresid + r0 * g.lddr + s0 : nullptr, g.lddr, es, p.hw, p.S);
    each([&](const float (&d)[V], const float (&du)[V], int e) __attribute__((always_inline)) {
      if (g.dresid) store_buf<T>(qb, vq, e * o.rpp * ldq, du);
      float z[V];
#pragma unroll
      for (int v = 0; v < V; ++v) z[v] = fmaf(-d[v], k2[v], fmaf(du[v], rg[v], -k1[v]));
      store_buf<T>(yb, vy, e * o.rpp * ldy, z);
    });
    __syncthreads();   // (the arrays per channel are written again by the next tile)
  }
  channel_sums<TH, V>(tg, o, p.S, red, red2, cm);
  channel_sums<TH, V>(tb, o, p.S, red, red2, cr);
  for (int c = threadIdx.x; c < p.S; c += TH) {
    p.part[((long long)first * 2 + 0) * p.C + s0 + c] = cm[c];
    p.part[((long long)first * 2 + 1) * p.C + s0 + c] = cr[c];
  }
}

// dgamma, dbeta = (accumulate ? what is there : 0) + the partials [rows][2][C], added in double in a fixed order; 16 channels per workgroup
__global__ void __launch_bounds__(1024) gn_sum_k(const float* __restrict__ part, long long rows, int C, float* dgamma, float* dbeta,
                                                 int accumulate) {
  __shared__ double ra[64][17], rb[64][17];
  const int c = threadIdx.x & 15, q = threadIdx.x >> 4, ch = blockIdx.x * 16 + c;
  double a = 0.0, b = 0.0;
  if (ch < C) {
    const float* p = part + ch;
    long long r = q;
    for (; r + 192 < rows; r += 256) {   // eight loads in flight
      float u[4], v[4];
#pragma unroll
      for (int k = 0; k < 4; ++k) { u[k] = p[(r + 64 * k) * 2 * C]; v[k] = p[((r + 64 * k) * 2 + 1) * C]; }
#pragma unroll
      for (int k = 0; k < 4; ++k) { a += (double)u[k]; b += (double)v[k]; }
    }
    for (; r < rows; r += 64) { a += (double)p[r * 2 * C]; b += (double)p[(r * 2 + 1) * C]; }
  }
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

// row0: the chunk's first row, of the whole matrix.  Rows are counted within the chunk: a tile may have 2^31 - 1 of them, and a chunk's count with
// what a thread strides beyond it stays far below that.
struct Where { long long tile, row0; int slice, chunk, rows; };
__device__ __forceinline__ Where where(const P& p, long long unit) {
  Where w;
  w.slice = (int)(unit % p.slices);
  const long long k = unit / p.slices;
  w.chunk = (int)(k % p.chunks);
  w.tile = k / p.chunks;
  const int lo = w.chunk * p.rows_chunk;   // < hw
  w.rows = p.hw - lo < p.rows_chunk ? p.hw - lo : p.rows_chunk;
  w.row0 = w.tile * p.hw + lo;
  return w;
}

// Partial statistics of a chunk: part[tile * chunks + chunk][0 mean, 1 squared distances][C].
// A checkpoint may be written on the way (p.pack).  NARROW: all 2, 4 or 8 lanes of a row hold its only block of columns.  Else sixteen lanes hold a
// block; rows that are not whole sixteens are padded to them, and the lanes behind the last column go along with zeros (left out, they would cut the
// exchange of the block's maximum between the others).  Unpadded, a checkpoint leaves the order of the statistics' sums, and so their last
// bits, as they are without.
template <typename T, int V, bool NARROW>
__global__ void __launch_bounds__(ST) gn_stat_k(P p) {
  __shared__ float sn[ST], sm[ST * V], sq[ST * V];
  const GroupNorm& g = p.g;
  for (long long unit = blockIdx.x; unit < p.n * p.chunks * p.slices; unit += gridDim.x) {
    const Where w = where(p, unit);
    const int S = p.C - w.slice * p.S < p.S ? p.C - w.slice * p.S : p.S;   // the last slice may be short
    const Own<V> o(!NARROW && p.pack ? (S / V + 15) / 16 * 16 * V : S, ST);
    const bool have_cols = o.tc * V < S;
    const int c0 = w.slice * p.S + o.tc * V;
    const T* x = (const T*)g.x + w.row0 * g.ldx + c0;
    float n = 0.f, m[V], q[V];
#pragma unroll
    for (int v = 0; v < V; ++v) m[v] = q[v] = 0.f;
    if (o.on)
      for (int r = o.tr; r < w.rows; r += SE * o.rpp) {
        Vec<T, V> buf[SE];
        int have = 0;
#pragma unroll
        for (int e = 0; e < SE; ++e) {
          const int k = r + e * o.rpp;
          have += k < w.rows;
          if (k < w.rows && have_cols) buf[e].load(x + (long long)k * g.ldx);
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
          if constexpr (V == 8) {
            if (p.pack && r + e * o.rpp < w.rows) {   // (alike in the lanes of a row)
              const unsigned sc = a8_block_byte(t, NARROW ? p.pack : 16);
              const float inv = a8_inverse(sc);
              const long long row = w.row0 + r + e * o.rpp;
              u32x2 z;
              z[0] = a8_code4(t[0] * inv, t[1] * inv, t[2] * inv, t[3] * inv);
              z[1] = a8_code4(t[4] * inv, t[5] * inv, t[6] * inv, t[7] * inv);
              if (have_cols) *reinterpret_cast<u32x2*>(const_cast<uint8_t*>(p.x8.codes) + row * p.x8.ldc + c0) = z;
              if (have_cols && (o.tc & (NARROW ? p.pack - 1 : 15)) == 0) const_cast<uint8_t*>(p.x8.scales)[row * p.x8.lds + (c0 >> 7)] = (uint8_t)sc;
            }
          }
        }
#pragma unroll
        for (int v = 0; v < V; ++v) s[v] /= (float)have;
#pragma unroll
        for (int e = 0; e < SE; ++e) {
          if (r + e * o.rpp >= w.rows) continue;
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
    if (o.on && have_cols) {
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

constexpr int GT = 1024;   // threads that add up a group
__device__ __forceinline__ double block_sum(double v, double* red) {
#pragma unroll
  for (int k = 32; k > 0; k >>= 1) v += __shfl_xor(v, k, 64);
  __syncthreads();
  if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = v;
  __syncthreads();
  double s = 0.0;
#pragma unroll
  for (int k = 0; k < GT / 64; ++k) s += red[k];
  return s;
}

// mean and rstd of a group from the partials of its channels and chunks
__global__ void __launch_bounds__(GT) gn_stat_group_k(P p) {
  __shared__ double red[GT / 64];
  for (long long u = blockIdx.x; u < p.n * p.G; u += gridDim.x) {
    const long long tile = u / p.G;
    const int gr = (int)(u - tile * p.G);
    const float* part = p.part + tile * p.chunks * 2 * p.C + gr * p.per;
    const int all = p.chunks * p.per;
    double s = 0.0;
    for (int i = threadIdx.x; i < all; i += GT) {
      const int k = i / p.per, c = i - k * p.per;
      const int rows = p.hw - k * p.rows_chunk < p.rows_chunk ? p.hw - k * p.rows_chunk : p.rows_chunk;
      s += (double)rows * (double)part[(long long)k * 2 * p.C + c];
    }
    const double count = (double)p.hw * p.per, mean = block_sum(s, red) / count;
    double q = 0.0;
    for (int i = threadIdx.x; i < all; i += GT) {
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
    for (int r = o.tr; r < w.rows; r += o.rpp) {
      const long long row = w.row0 + r;
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
      act_vec<V>(u, g.s.act);
      store_vec((T*)g.y + row * g.ldy + c0, u);
    }
  }
}

// DX false: the chunk's sums of du xhat and du per channel -> part; true: dx (and dresidual) out of the groups' sums
template <typename T, int V, bool X8, bool DX, Third RES, bool RELU>
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
    float mean[V], rstd[V], rg[V], bet[V], s[V], q[V];
#pragma unroll
    for (int v = 0; v < V; ++v) { mean[v] = rstd[v] = rg[v] = bet[v] = s[v] = q[v] = 0.f; }
    if (o.on) {
      group_stats<V>(p, w.tile, c0, mean, rstd);
#pragma unroll
      for (int v = 0; v < V; ++v) {
        rg[v] = rstd[v] * g.gamma[c0 + v]; bet[v] = g.beta[c0 + v];
        if constexpr (DX) {   // dx = du (rstd gamma) - s - (x - mean) q
          const float* gsum = p.sums + (w.tile * p.G + (c0 + v) / p.per) * 2;
          q[v] = gsum[0] * inv * rstd[v] * rstd[v];   // of du gamma xhat
          s[v] = gsum[1] * inv * rstd[v];             // of du gamma
        }
      }
      for (int r = o.tr; r < w.rows; r += RG * o.rpp) {
        typename Input<T, V, X8>::type bx[RG];
        Vec<T, V> bd[RG], br[RG];
#pragma unroll
        for (int k = 0; k < RG; ++k) {   // (rows behind the last: the last one's values, left out below)
          const int at = r + k * o.rpp;
          const long long row = w.row0 + (at < w.rows ? at : w.rows - 1);
          load_in(bx[k], p, row, c0);
          bd[k].load((const T*)g.dy + row * g.lddy + c0);
          if constexpr (RES != NONE) br[k].load((const T*)g.resid + row * g.ldr + c0);
        }
#pragma unroll
        for (int k = 0; k < RG; ++k) {
          if (r + k * o.rpp >= w.rows) break;
          const long long row = w.row0 + r + k * o.rpp;
          float dy[V], res[V], d[V], du[V];
          less_of<>(bx[k], mean, d);
          bd[k].get(dy);
          if constexpr (RES != NONE) br[k].get(res);
          du_vec<RES, RELU, V>(d, dy, rg, bet, res, act, du, [&](int v) __attribute__((always_inline)) {
            float x[V];
            bx[k].get(x);
            return side(x[v], mean[v], rstd[v], g.gamma[c0 + v], bet[v], RES != NONE ? res[v] : 0.f);
          });
          if constexpr (DX) {
            if (g.dresid) store_vec((T*)g.dresid + row * g.lddr + c0, du);
#pragma unroll
            for (int v = 0; v < V; ++v) du[v] = fmaf(-d[v], q[v], fmaf(du[v], rg[v], -s[v]));
            store_vec((T*)g.y + row * g.ldy + c0, du);
          } else {
#pragma unroll
            for (int v = 0; v < V; ++v) { s[v] += du[v]; q[v] = fmaf(du[v], d[v], q[v]); }
          }
          row_end();
        }
      }
    }
    if constexpr (!DX) {
      float* out = p.part + (w.tile * p.chunks + w.chunk) * 2 * p.C + w.slice * p.S;
#pragma unroll
      for (int v = 0; v < V; ++v) q[v] *= rstd[v];
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
__global__ void __launch_bounds__(GT) gn_bwd_group_k(P p) {
  __shared__ double red[GT / 64];
  for (long long u = blockIdx.x; u < p.n * p.G; u += gridDim.x) {
    const long long tile = u / p.G;
    const int gr = (int)(u - tile * p.G);
    const float* part = p.part + tile * p.chunks * 2 * p.C + gr * p.per;
    double a = 0.0, b = 0.0;
    for (int i = threadIdx.x; i < p.chunks * p.per; i += GT) {
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

constexpr int WANT = 1024;              // workgroups of a split launch
constexpr int SPLIT_SMAX = 2048;
constexpr long long MOST_P = 4096;      // rows of partial sums that the unit kernels leave
constexpr long long MOST_WGS = 1 << 22; // workgroups of a unit launch, but for the rounding up to eight tiles (channels <= 65536: 64 tiles of slices at least)

int gcd(int a, int b) { while (b) { const int t = a % b; a = b; b = t; } return a; }

int pieces(const GroupNorm& g, bool bwd) {   // 8: every row can be read and written in pieces of eight channels
  const size_t es = elem_size(g.s.dtype);
  auto ok = [&](const void* q, long long ld) { return !q || (((uintptr_t)q & 15) == 0 && ld * es % 16 == 0); };
  bool v = g.s.channels % 8 == 0 && ok(g.y, g.ldy) && ok(g.resid, g.ldr) && ok(g.x, g.ldx);
  if (bwd) v = v && ok(g.dy, g.lddy) && ok(g.dresid, g.lddr);
  return v ? 8 : 1;
}

void split_plan(const slide_group_norm& s, int V, P* p) {
  const int most = ST * V < SPLIT_SMAX ? ST * V : SPLIT_SMAX;
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

size_t part_floats(const slide_group_norm& s) {
  P a{}, b{};
  split_plan(s, 8, &a);
  split_plan(s, 1, &b);
  const long long rows = s.n * (a.chunks > b.chunks ? a.chunks : b.chunks);
  return (size_t)rows * 2 * s.channels;
}

// A workgroup per unit: its slice, threads and rows.  False: the rows are split.
//   * The slice: whole groups, whole pieces of V, dividing the channels; the fewest channels that are 128 bytes of a row (narrower slices
//     fetch cache lines that other units want too) and, where there are units enough, PIECES pieces in all (a unit costs some
//     microseconds of barriers), or all of them.
//   * 256 threads up to sixteen rows of a thread, else 512.
//   * With fewer units than half the compute units (float32: three quarters) a longer unit is split instead (9 x 3136 x 512 float32, 144 units:
//     forward 46 us, split 37; backward 73 and 58; 130 x 3136 x 64, 260 units: 64 and 73, 119 and 113), and a float32 unit of 1.5 MB
//     (140 x 12544 x 64, units of 1.6 MB: 383 us and 327, 544 and 483; 1024: 2001 and 2030, 3233 and 3092; 256 x 6272 x 64, 0.8 MB: 266
//     and 295, 426 and 430; bfloat16, 500 x 12544 x 64, 1.6 MB: 475 and 539, 779 and 817; 256 x 25088 x 64, 3.2 MB: 480 and 530, 775 and 870).
constexpr int PIECES = 2048;
bool by_units(P* p, int V, int es, unsigned* grid, bool* small) {
  const slide_group_norm& s = p->g.s;
  const int base = p->per / gcd(p->per, V) * V;   // lcm
  if (base > SMAX || p->C % base) return false;
  long long ld = s.channels;
  for (long long q : {p->g.ldx, p->g.ldy, p->g.x8 ? p->x8.ldc : 0, p->g.x8 ? p->x8.lds : 0, p->g.resid ? p->g.ldr : 0,
                      p->g.dy ? p->g.lddy : 0, p->g.dresid ? p->g.lddr : 0})
    if (q > ld) ld = q;
  if ((s.hw + 4096) * ld * es > DMA_MAX) return false;   // 32-bit offsets, with rows behind the last
  p->S = 0;
  for (int k = 1; base * k <= SMAX && base * k <= p->C; ++k) {
    if ((p->C / base) % k) continue;
    const int S = base * k;
    if (S / V > 512) break;
    p->S = S;
    if ((long long)S * es >= 128 && (s.hw * (S / V) >= PIECES || s.n * (p->C / S) < 512)) break;
  }
  if (!p->S) return false;
  const int vpr = p->S / V;
  *small = vpr <= 256 && (s.hw + 256 / vpr - 1) / (256 / vpr) <= 16;
  const int rpp = (*small ? 256 : 512) / vpr;
  p->slices = p->C / p->S;
  p->rows = (int)((s.hw + rpp - 1) / rpp);
  if (s.n * p->slices < (es == 4 ? 192 : 128) && p->rows > 16) return false;
  if (es == 4 && s.hw * p->S * es >= 3 << 19) return false;
  // A launch may have 2^32 - 1 threads: with thousands of slices (a prime number of channels, each a group of its own) a workgroup takes more tiles
  const long long most_p = MOST_WGS / p->slices < MOST_P ? MOST_WGS / p->slices : MOST_P;
  p->units_p = (int)(s.n < most_p ? s.n : most_p);
  *grid = (unsigned)((p->units_p + 7) / 8 * 8 * p->slices);
  return true;
}

unsigned split_grid(const P& p) {
  const long long u = p.n * p.chunks * p.slices;
  return (unsigned)(u < (1 << 20) ? u : (1 << 20));
}
unsigned group_grid(const P& p) {
  const long long u = p.n * p.G;
  return (unsigned)(u < (1 << 20) ? u : (1 << 20));
}

// Groups of rows that stay in registers.  More of them (seven: a unit of 28 x 28 x 64 whole) cost more than they saved: one workgroup per
// compute unit then, whose loads, sums and stores wait for each other (1024 such tiles, backward: 299 us, 424 with seven groups).
constexpr int KEPT = 1;

template <typename T, int V>
hipError_t fwd_units(const P& p, unsigned grid, bool small, hipStream_t s) {
  if (small) gn_fwd_k<T, V, 256, KEPT><<<grid, 256, 0, s>>>(p);
  else gn_fwd_k<T, V, 512, KEPT><<<grid, 512, 0, s>>>(p);
  return hipGetLastError();
}

template <typename T, int V>
hipError_t fwd(const GroupNorm& g, hipStream_t s) {
  P p = base(g);
  unsigned grid;
  bool small;
  const bool units = by_units(&p, V, sizeof(T), &grid, &small);
  if (!units) split_plan(g.s, V, &p);
  // The checkpoint comes out of the same pass where 16 lanes (or the fewer of a narrow row) hold a block of its columns, and no byte behind
  // the last column is to be cleared.
  if (g.x8) {
    const int vpr = p.S / 8;
    if (V == 8 && p.C % A8_GRAIN == 0 && p.S == p.C && p.C < A8_BLOCK && (vpr & (vpr - 1)) == 0) p.pack = vpr;
    else if (V == 8 && p.C % A8_GRAIN == 0 && (!units || p.S % A8_BLOCK == 0)) p.pack = 16;
    else {
      const hipError_t e = launch_act8_pack(g.x, g.s.dtype, g.ldx, false, *g.x8, s);   // before y, which may be x, is written
      if (e != hipSuccess) return e;
    }
  }
  if (units) return fwd_units<T, V>(p, grid, small, s);
  p.part = g.work;
  if (V == 8 && p.pack && p.pack < 16) gn_stat_k<T, V, V == 8><<<split_grid(p), ST, 0, s>>>(p);
  else gn_stat_k<T, V, false><<<split_grid(p), ST, 0, s>>>(p);
  hipError_t err = hipGetLastError();
  if (err != hipSuccess) return err;
  gn_stat_group_k<<<group_grid(p), GT, 0, s>>>(p);
  err = hipGetLastError();
  if (err != hipSuccess) return err;
  gn_apply_k<T, V><<<split_grid(p), ST, 0, s>>>(p);
  return hipGetLastError();
}

template <typename T, int V, bool X8, Third RES, bool RELU>
hipError_t bwd_units(const P& p, unsigned grid, bool small, hipStream_t s) {
  if (small) gn_bwd_k<T, V, 256, KEPT, X8, RES, RELU><<<grid, 256, 0, s>>>(p);
  else gn_bwd_k<T, V, 512, KEPT, X8, RES, RELU><<<grid, 512, 0, s>>>(p);
  return hipGetLastError();
}

// the sums of the chunks, of the groups, then dx
template <typename T, int V, bool X8, Third RES, bool RELU>
hipError_t bwd_split(const P& p, hipStream_t s) {
  gn_bwd_split_k<T, V, X8, false, RES, RELU><<<split_grid(p), ST, 0, s>>>(p);
  hipError_t err = hipGetLastError();
  if (err != hipSuccess) return err;
  gn_bwd_group_k<<<group_grid(p), GT, 0, s>>>(p);
  err = hipGetLastError();
  if (err != hipSuccess) return err;
  gn_bwd_split_k<T, V, X8, true, RES, RELU><<<split_grid(p), ST, 0, s>>>(p);
  return hipGetLastError();
}

template <typename F> hipError_t either(bool b, F f) { return b ? f(std::true_type{}) : f(std::false_type{}); }

template <typename T, int V>
hipError_t bwd(const GroupNorm& g, hipStream_t s) {
  P p = base(g);
  unsigned grid;
  bool small;
  p.part = g.work;
  const bool units = by_units(&p, V, sizeof(T), &grid, &small);
  if (!units) {
    split_plan(g.s, V, &p);
    p.sums = g.work + part_floats(g.s);
  }
  auto run = [&](auto x8, auto third, auto relu) {
    constexpr bool X8 = decltype(x8)::value, RELU = decltype(relu)::value;
    constexpr Third RES = decltype(third)::value;
    return units ? bwd_units<T, V, X8, RES, RELU>(p, grid, small, s) : bwd_split<T, V, X8, RES, RELU>(p, s);
  };
  hipError_t err;
  if (g.out) {
    if constexpr (sizeof(T) == 2 && V == 8) err = run(std::true_type{}, std::integral_constant<Third, OUT>{}, std::true_type{});
    else return hipErrorInvalidValue;   // the convolutional encoder's rows are whole pieces
  } else {
    err = either(!g.x, [&](auto x8) {
      return either(g.s.act == SLIDE_ACT_RELU, [&](auto relu) {
        return g.resid ? run(x8, std::integral_constant<Third, RESID>{}, relu) : run(x8, std::integral_constant<Third, NONE>{}, relu);
      });
    });
  }
  if (err != hipSuccess) return err;
  gn_sum_k<<<(p.C + 15) / 16, 1024, 0, s>>>(p.part, units ? p.units_p : p.n * p.chunks, p.C, g.dgamma, g.dbeta, g.accumulate);
  return hipGetLastError();
}

}  // namespace

size_t group_norm_bytes(const slide_group_norm& s) {
  return ((part_floats(s) + (size_t)s.n * s.groups * 2) * 4 + 255) & ~(size_t)255;
}

hipError_t launch_group_norm_fwd(const GroupNorm& g, hipStream_t s) {
  const int V = pieces(g, false);
  if (g.s.dtype == DT_F32) return V == 8 ? fwd<float, 8>(g, s) : fwd<float, 1>(g, s);
  return V == 8 ? fwd<bf16, 8>(g, s) : fwd<bf16, 1>(g, s);
}

hipError_t launch_group_norm_bwd(const GroupNorm& given, hipStream_t s) {
  GroupNorm g = given;
  if (g.out) { g.resid = g.out; g.ldr = g.ldo; }   // read in the residual's place
  const int V = pieces(g, true);
  if (g.s.dtype == DT_F32) return V == 8 ? bwd<float, 8>(g, s) : bwd<float, 1>(g, s);
  return V == 8 ? bwd<bf16, 8>(g, s) : bwd<bf16, 1>(g, s);
}

}  // namespace sl
