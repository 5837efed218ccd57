// Norm of every query and key head and its rotation by the row's position, one pass forward and one backward (include/tokens.h).
//
//   r = (mean(x^2) + eps)^(-1/2),  h = x r,  n = h g,  y = R(pos) n          R turns pair p by pos[axis] * theta^(-j / n)
//   dn = R^T dy,  dg = sum dn h,  u = dn g,  dx = r (u - h mean(u h))
//
// Bound by the bytes: a value is read and written once.  A thread holds eight pairs of a head (16 values: two 16-byte loads in bfloat16), a
// head's threads are neighbours in a wavefront and sum by lane exchanges.  The angle depends on the row and the pair alone: a thread keeps its pairs and
// its row and goes over the heads, so sines are taken once for all of them.
// Angles: a pair's frequency in turns is a fraction of 2^64, so position times frequency modulo one turn is the low half of an
// integer product, without error at any position; its upper 32 bits are the angle.
#include <type_traits>

#include "tokens_internal.h"

namespace sl {

namespace {

typedef unsigned int u32x4 __attribute__((ext_vector_type(4)));
constexpr int ROPE_BLOCKS = 512;   // workgroups of the backward's queries, and of its keys, each of which leaves its part of the gains' gradients

__device__ __forceinline__ void load8(const float* p, float (&v)[8]) {
  const f32x4 a = *reinterpret_cast<const f32x4*>(p), b = *reinterpret_cast<const f32x4*>(p + 4);
#pragma unroll
  for (int i = 0; i < 4; ++i) { v[i] = a[i]; v[4 + i] = b[i]; }
}
__device__ __forceinline__ void load8(const bf16* p, float (&v)[8]) {
  const bf16x8 a = *reinterpret_cast<const bf16x8*>(p);
#pragma unroll
  for (int i = 0; i < 8; ++i) v[i] = (float)a[i];
}
__device__ __forceinline__ void store8(float* p, const float (&v)[8]) {
  *reinterpret_cast<f32x4*>(p) = f32x4{v[0], v[1], v[2], v[3]};
  *reinterpret_cast<f32x4*>(p + 4) = f32x4{v[4], v[5], v[6], v[7]};
}
__device__ __forceinline__ void store8(bf16* p, const float (&v)[8]) {
  bf16x8 a;
#pragma unroll
  for (int i = 0; i < 8; ++i) a[i] = (bf16)v[i];
  *reinterpret_cast<bf16x8*>(p) = a;
}

struct Pairs { float a[8], b[8]; };   // first and second columns of eight pairs
// the thread's columns of a head: `at` the first of them, the second eight `apart` behind
template <bool NEIGHBOURS, typename T>
__device__ __forceinline__ Pairs get_pairs(const T* p, int apart) {
  Pairs v;
  if (!NEIGHBOURS) {
    load8(p, v.a);
    load8(p + apart, v.b);
  } else {
    float x[8], y[8];
    load8(p, x);
    load8(p + apart, y);
#pragma unroll
    for (int i = 0; i < 4; ++i) { v.a[i] = x[2 * i]; v.b[i] = x[2 * i + 1]; v.a[4 + i] = y[2 * i]; v.b[4 + i] = y[2 * i + 1]; }
  }
  return v;
}
template <bool NEIGHBOURS, typename T>
__device__ __forceinline__ void put_pairs(T* p, int apart, const Pairs& v) {
  if (!NEIGHBOURS) {
    store8(p, v.a);
    store8(p + apart, v.b);
  } else {
    float x[8], y[8];
#pragma unroll
    for (int i = 0; i < 4; ++i) { x[2 * i] = v.a[i]; x[2 * i + 1] = v.b[i]; y[2 * i] = v.a[4 + i]; y[2 * i + 1] = v.b[4 + i]; }
    store8(p, x);
    store8(p + apart, y);
  }
}

// sine and cosine of `turn` / 2^32 of a turn: the nearest quarter turn and Taylor series of the rest, at most pi / 4 (next terms 2e-9, 2e-9)
__device__ __forceinline__ void sin_cos(unsigned turn, float* s, float* c) {
  const unsigned quarter = (turn + 0x20000000u) >> 30;
  const float t = (float)(int)(turn - (quarter << 30)) * 1.46291807926715968e-9f;   // 2 pi / 2^32
  const float w = t * t;
  const float sn = fmaf(t * w, fmaf(w, fmaf(w, fmaf(w, 1.f / 362880.f, -1.f / 5040.f), 1.f / 120.f), -1.f / 6.f), t);
  const float cs = fmaf(w, fmaf(w, fmaf(w, fmaf(w, fmaf(w, -1.f / 3628800.f, 1.f / 40320.f), -1.f / 720.f), 1.f / 24.f), -0.5f), 1.f);
  const float a = quarter & 1 ? cs : sn, b = quarter & 1 ? sn : cs;
  *s = quarter & 2 ? -a : a;
  *c = (quarter + 1) & 2 ? -b : b;
}
// the frequencies of as many pairs as a head's lanes hold: arguments of the kernel, of which a small call copies no more than it needs
template <int LANES> struct Freq { unsigned long long f[8 * LANES]; };
template <int LANES>
__device__ __forceinline__ void angles(const HeadRope& g, const Freq<LANES>& freq, long long row, int p0, float (&c)[8], float (&s)[8]) {
  const int* pos = g.pos + row * g.axes;
  const long long x0 = g.axes > 0 ? pos[0] : 0, x1 = g.axes > 1 ? pos[1] : 0, x2 = g.axes > 2 ? pos[2] : 0;
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const int p = p0 + i;
    const long long x = p < g.bound[0] ? x0 : p < g.bound[1] ? x1 : x2;   // frequencies behind the last axis' pairs are 0
    sin_cos((unsigned)((unsigned long long)x * freq.f[p] >> 32), &s[i], &c[i]);
  }
}

template <int LANES>
__device__ __forceinline__ float group_sum(float v) {
#pragma unroll
  for (int o = LANES / 2; o > 0; o >>= 1) v += __shfl_xor(v, o, 64);
  return v;
}
// 1 / sqrt(mean(x^2) + eps) of a head, in all of its lanes.  Squares past float32 are summed again in 64 bits.
template <int LANES>
__device__ __forceinline__ float inverse_rms(const Pairs& v, int dim, float eps) {
  float ss = 0.f;
#pragma unroll
  for (int i = 0; i < 8; ++i) ss = fmaf(v.a[i], v.a[i], fmaf(v.b[i], v.b[i], ss));
  ss = group_sum<LANES>(ss);
  if (ss == __builtin_huge_valf()) {   // alike in all lanes of a head
    double d = 0.0;
#pragma unroll
    for (int i = 0; i < 8; ++i) d += (double)v.a[i] * v.a[i] + (double)v.b[i] * v.b[i];
#pragma unroll
    for (int o = LANES / 2; o > 0; o >>= 1) d += __shfl_xor(d, o, 64);
    return (float)(1.0 / sqrt(d / dim + eps));
  }
  return 1.f / sqrtf(ss / (float)dim + eps);
}

// a thread's 16 values of a head as they lie in memory
template <typename T> struct Raw { u32x4 v[sizeof(T)]; };
template <typename T>
__device__ __forceinline__ Raw<T> get_raw(const T* p, int apart) {
  constexpr int H = sizeof(T) / 2;
  Raw<T> r;
#pragma unroll
  for (int i = 0; i < H; ++i) {
    r.v[i] = *reinterpret_cast<const u32x4*>(p + i * 4);
    r.v[H + i] = *reinterpret_cast<const u32x4*>(p + apart + i * 4);
  }
  return r;
}
template <bool NEIGHBOURS, typename T>
__device__ __forceinline__ Pairs pairs_of(const Raw<T>& r) {
  T e[16];
  __builtin_memcpy(e, &r, sizeof(r));
  Pairs v;
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    v.a[i] = to_f(e[NEIGHBOURS ? 2 * i : i]);
    v.b[i] = to_f(e[NEIGHBOURS ? 2 * i + 1 : 8 + i]);
  }
  return v;
}

// blockIdx.y: queries or keys.  A thread's row is item / slices; it goes over heads item % slices, + slices, ..., the next one's values on
// their way while it works.
template <typename T, int LANES, bool NEIGHBOURS, bool BACKWARD, bool NORM>
__device__ __forceinline__ void rope_side(const HeadRope& g, const Freq<LANES>& freq, bool key, int slices, long long items) {
  constexpr int PER = 256 / LANES;
  const int sub = threadIdx.x % LANES, p0 = sub * 8;
  const bool mine = sub * 16 < g.dim;                 // head widths that are no power of two leave lanes over
  const int first = mine ? (NEIGHBOURS ? 2 * p0 : p0) : 0, apart = NEIGHBOURS ? 8 : g.dim / 2;
  const int heads = key ? g.hk : g.hq, turns = (heads + slices - 1) / slices;
  const T* const xs = (const T*)(key ? g.k : g.q);
  const T* const ds = (const T*)(key ? g.dyk : g.dyq);
  T* const ys = (T*)(key ? g.yk : g.yq);
  const long long ldx = key ? g.ldk : g.ldq, ldd = key ? g.lddyk : g.lddyq, ldy = key ? g.ldyk : g.ldyq;
  Pairs w, sum;   // the gain, and this thread's part of its gradient
#pragma unroll
  for (int i = 0; i < 8; ++i) sum.a[i] = sum.b[i] = 0.f;
  if (NORM) w = get_pairs<NEIGHBOURS>((key ? g.gk : g.gq) + first, apart);

  for (long long base = blockIdx.x * (long long)PER; base < items; base += (long long)gridDim.x * PER) {   // alike in a workgroup
    const long long item = base + threadIdx.x / LANES;
    const bool there = item < items;
    const long long row = there ? item / slices : 0;
    const int slice = there ? (int)(item - row * slices) : 0;
    Raw<T> nx = {}, nd = {};
    auto ask = [&](int h) __attribute__((always_inline)) {
      if (there && mine && h < heads) {
        if (!BACKWARD || NORM) nx = get_raw(xs + row * ldx + (long long)h * g.dim + first, apart);
        if (BACKWARD) nd = get_raw(ds + row * ldd + (long long)h * g.dim + first, apart);
      }
    };
    ask(slice);
    float c[8], s[8];
    angles<LANES>(g, freq, row, mine ? p0 : 0, c, s);
    for (int t = 0; t < turns; ++t) {
      const int h = slice + t * slices;
      const bool work = there && mine && h < heads;
      Pairs x = pairs_of<NEIGHBOURS>(nx), d = pairs_of<NEIGHBOURS>(nd), y;
      ask(h + slices);
      if (NORM && !mine) {   // lanes left over count for nothing
#pragma unroll
        for (int i = 0; i < 8; ++i) x.a[i] = x.b[i] = d.a[i] = d.b[i] = 0.f;
      }
      if (!BACKWARD) {
        if (NORM) {
          const float r = inverse_rms<LANES>(x, g.dim, g.eps);
#pragma unroll
          for (int i = 0; i < 8; ++i) { x.a[i] *= r * w.a[i]; x.b[i] *= r * w.b[i]; }
        }
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          y.a[i] = fmaf(x.a[i], c[i], -x.b[i] * s[i]);
          y.b[i] = fmaf(x.b[i], c[i], x.a[i] * s[i]);
        }
      } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          y.a[i] = fmaf(d.a[i], c[i], d.b[i] * s[i]);
          y.b[i] = fmaf(d.b[i], c[i], -d.a[i] * s[i]);
        }
        if (NORM) {
          const float r = inverse_rms<LANES>(x, g.dim, g.eps);
          float dot = 0.f;
#pragma unroll
          for (int i = 0; i < 8; ++i) {
            x.a[i] *= r; x.b[i] *= r;
            const float da = y.a[i] * x.a[i], db = y.b[i] * x.b[i];
            if (work) { sum.a[i] += da; sum.b[i] += db; }
            dot = fmaf(da, w.a[i], fmaf(db, w.b[i], dot));
          }
          dot = group_sum<LANES>(dot) / (float)g.dim;
#pragma unroll
          for (int i = 0; i < 8; ++i) {
            y.a[i] = r * fmaf(y.a[i], w.a[i], -x.a[i] * dot);
            y.b[i] = r * fmaf(y.b[i], w.b[i], -x.b[i] * dot);
          }
        }
      }
      if (work) put_pairs<NEIGHBOURS>(ys + row * ldy + (long long)h * g.dim + first, apart, y);
    }
  }
  if (!BACKWARD || !NORM) return;
  // over the rows of a wavefront, then of the workgroup's four; work[queries, keys][workgroup][columns of a head]
  __shared__ float red[4][LANES][16];
#pragma unroll
  for (int i = 0; i < 16; ++i) {
    float v = i < 8 ? sum.a[i] : sum.b[i - 8];
#pragma unroll
    for (int o = LANES; o < 64; o <<= 1) v += __shfl_xor(v, o, 64);
    if ((threadIdx.x & 63) < LANES) red[threadIdx.x >> 6][sub][i] = v;
  }
  __syncthreads();
  for (int e = threadIdx.x; e < LANES * 16; e += 256) {
    const int l = e / 16, i = e % 16, pair = l * 8 + (i & 7), second = i >> 3;
    if (l * 16 >= g.dim) continue;
    const int col = NEIGHBOURS ? 2 * pair + second : pair + second * (g.dim / 2);
    g.work[((long long)key * gridDim.x + blockIdx.x) * g.dim + col] = (red[0][l][i] + red[1][l][i]) + (red[2][l][i] + red[3][l][i]);
  }
}
template <typename T, int LANES, bool NEIGHBOURS, bool BACKWARD>
__global__ void __launch_bounds__(256) head_rope_k(const HeadRope g, const Freq<LANES> freq, const int slices, const long long items) {
  const bool key = blockIdx.y == 1;
  if (key ? g.gk != nullptr : g.gq != nullptr) rope_side<T, LANES, NEIGHBOURS, BACKWARD, true>(g, freq, key, slices, items);
  else rope_side<T, LANES, NEIGHBOURS, BACKWARD, false>(g, freq, key, slices, items);
}

// gains' gradients: 4 columns a workgroup, 64 threads each; blockIdx.y: of the queries or of the keys
__global__ void __launch_bounds__(256) rope_gain_k(const float* __restrict__ work, int blocks, int dim, float* dgq, float* dgk, int accumulate) {
  float* const out = blockIdx.y ? dgk : dgq;
  if (!out) return;
  __shared__ float red[64][5];
  const int c = threadIdx.x & 3, part = threadIdx.x >> 2, col = blockIdx.x * 4 + c;
  const float* const at = work + (long long)blockIdx.y * blocks * dim + col;
  float v = 0.f;
#pragma unroll 8
  for (int b = part; b < blocks; b += 64) v += at[(long long)b * dim];
  red[part][c] = v;
  __syncthreads();
  if (threadIdx.x >= 4) return;
  v = 0.f;
#pragma unroll
  for (int i = 0; i < 64; ++i) v += red[i][threadIdx.x];
  out[col] = accumulate ? out[col] + v : v;
}

int lanes_of(int dim) { int l = 1; while (l * 16 < dim) l *= 2; return l; }
// Slices of a row's heads: all heads in one thread where the rows give a wavefront to each of the card's 1024 units that issue, else as many threads a
// row as do (7289 rows of 6 + 6 heads of 64: 8.1 us with half as many threads, 8.4, 11.1 with twice, 10.5 with four times)
int slices_of(long long rows, int heads, int lanes) {
  const long long want = 64 * 1024, have = rows * lanes, n = (want + have - 1) / have;
  return (int)(n > heads ? heads : n);
}
int slices_of(const HeadRope& g) { return slices_of(g.rows, g.hq > g.hk ? g.hq : g.hk, lanes_of(g.dim)); }

template <typename T, bool BACKWARD>
hipError_t run(const HeadRope& g, hipStream_t s) {
  const int lanes = lanes_of(g.dim), slices = slices_of(g), per = 256 / lanes;
  const long long items = g.rows * slices;
  long long blocks = (items + per - 1) / per;
  const long long most = BACKWARD ? ROPE_BLOCKS : 1 << 20;
  if (blocks > most) blocks = most;
  auto go = [&](auto l) {
    constexpr int L = decltype(l)::value;
    Freq<L> f;
    for (int i = 0; i < 8 * L; ++i) f.f[i] = g.freq[i];
    if (g.neighbours) head_rope_k<T, L, true, BACKWARD><<<dim3((unsigned)blocks, g.hk ? 2 : 1), 256, 0, s>>>(g, f, slices, items);
    else head_rope_k<T, L, false, BACKWARD><<<dim3((unsigned)blocks, g.hk ? 2 : 1), 256, 0, s>>>(g, f, slices, items);
  };
  switch (lanes) {
    case 1: go(std::integral_constant<int, 1>{}); break;
    case 2: go(std::integral_constant<int, 2>{}); break;
    case 4: go(std::integral_constant<int, 4>{}); break;
    case 8: go(std::integral_constant<int, 8>{}); break;
    default: go(std::integral_constant<int, 16>{}); break;
  }
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess || !BACKWARD || (!g.gq && !g.gk)) return e;
  rope_gain_k<<<dim3(g.dim / 4, g.hk ? 2 : 1), 256, 0, s>>>(g.work, (int)blocks, g.dim, g.gq ? g.dgq : nullptr, g.gk ? g.dgk : nullptr, g.accumulate);
  return hipGetLastError();
}

}  // namespace

size_t head_rope_work_bytes(const slide_head_rope& s) {
  const size_t n = (size_t)2 * ROPE_BLOCKS * s.head_dim * sizeof(float);
  return (n + 255) / 256 * 256;
}
hipError_t launch_head_rope_fwd(int dt, const HeadRope& g, hipStream_t s) { return dt == DT_F32 ? run<float, false>(g, s) : run<bf16, false>(g, s); }
hipError_t launch_head_rope_bwd(int dt, const HeadRope& g, hipStream_t s) { return dt == DT_F32 ? run<float, true>(g, s) : run<bf16, true>(g, s); }

}  // namespace sl
