// Device parts that the passes of the attention over packed slides share (tokens_attn_fwd / _dq / _dkv .hip).
//
// Every pass is a workgroup's 32 columns a wavefront against blocks of rows that pass through LDS.  Forward and dq: columns are queries, the heads that
// share a key head packed beside each other (column c of a slide is its query c / group, head c % group of the group), rows are keys.
// dk, dv: columns are keys, rows are such packed queries.  A block of scores is made transposed, rows down the registers of an
// accumulator and one column a lane, so a row statistic of the columns is a reduction inside a lane and one exchange between the halves of the
// wavefront, and the probabilities are in the layout in which the next product takes its second operand.
#pragma once
#include <type_traits>

#include "lds_dma.h"
#include "tokens_internal.h"

namespace sl {

typedef unsigned int u32x4 __attribute__((ext_vector_type(4)));

constexpr float TOK_NONE = -3e38f;   // below every score
constexpr int TOK_MEND_KEYS = 256;   // slides up to which four wavefronts mend the queries' gradients (tokens_attn_dq.hip)
constexpr float TOK_LOG2E = 1.4426950408889634f, TOK_LN2 = 0.69314718055994531f;

template <typename T> struct TokType;
template <> struct TokType<bf16>  { static constexpr int EPC = 8, KB = 64; };   // elements of 16 bytes, rows of a block in LDS
template <> struct TokType<float> { static constexpr int EPC = 4, KB = 32; };

template <typename T, int DP> constexpr int tok_ldr() { return DP + TokType<T>::EPC; }   // elements between rows in LDS: 16-byte reads of eight rows meet no bank twice

// Two wavefronts a SIMD where 256 registers hold what a wavefront keeps: their matrix instructions then take vector registers, without copies
template <typename T, int DP, int NW> constexpr int tok_waves() { return NW == 4 ? (DP <= 64 || sizeof(T) == 2 ? 2 : 1) : (DP <= 64 ? 2 : 1); }

// where the kernels for two heads at a time are built (what it takes of the call: tok_cut)
template <typename T, int DP, bool BIAS> constexpr bool tok_pairs() { return BIAS && DP == 64 && sizeof(T) == 2; }

// ---- who does what --------------------------------------------------------------------------------
// A pass is cut into units: `width` columns of a slide and key head against a block of KB rows.  They are numbered head by head, slide by slide,
// column tile by column tile, block by block (a slide with columns and without rows has one for each tile, so that its results are
// written), and every workgroup takes the same number of neighbouring ones, whatever the slides' lengths: no workgroup waits for the longest slide, and one
// query against 50000 keys keeps the card as busy as 8000 against each other.  Column tiles that end up with several workgroups
// leave partial results, which a second launch adds up in the order of the blocks.  (Before, a workgroup took a column tile, or every tile was
// split alike: 65 tiles of 12 heads on 256 units were 4 rounds for the work of 3.05; 8193 rows, 12 heads of 64: 557 us.)
__device__ __forceinline__ int tok_clamp(int v, int rows) { return v < 0 ? 0 : v > rows ? rows : v; }
struct TokSide { const int* start; int rows, group, per; };   // rows of slides, `group` columns (or rows) each, `per` of them a tile (block)
struct TokSpan { int lo, n; };                                // first row; packed columns (rows) of a slide
__device__ __forceinline__ TokSpan tok_span(const TokSide& s, int doc) {
  const int a = tok_clamp(s.start[doc], s.rows), b = tok_clamp(s.start[doc + 1], s.rows);
  return {a, b > a ? (b - a) * s.group : 0};
}
__device__ __forceinline__ int tok_parts(int n, int per) { return (int)(((long long)n + per - 1) / per); }
__device__ __forceinline__ long long tok_units(const TokSide& c, const TokSide& r, int doc) {
  const int tiles = tok_parts(tok_span(c, doc).n, c.per), blocks = tok_parts(tok_span(r, doc).n, r.per);
  return (long long)tiles * (blocks > 0 ? blocks : 1);
}
__device__ __forceinline__ long long tok_uniform(long long v) {
  return (long long)(unsigned)__builtin_amdgcn_readfirstlane((int)v) | (long long)__builtin_amdgcn_readfirstlane((int)(v >> 32)) << 32;
}
// The slides' first units: up to 64 slides a lane each, more in a table that a launch before has written ([docs + 1])
struct TokIndex {
  long long end, all;   // the lane's slide's last unit + 1 (docs <= 64); all units of a head
  const long long* table;
  int docs;
  __device__ __forceinline__ TokIndex(const TokSide& c, const TokSide& r, int n, const long long* t) : end(0), table(t), docs(n) {
    if (n > 64) {
      all = tok_uniform(t[n]);
      return;
    }
    const int lane = threadIdx.x & 63;
    end = lane < n ? tok_units(c, r, lane) : 0;
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
      const long long v = __shfl_up(end, o, 64);
      if (lane >= o) end += v;
    }
    all = tok_uniform(__shfl(end, 63, 64));
  }
  // the slide of unit u (below `all`), whose first unit goes to *first
  __device__ __forceinline__ int find(long long u, long long* first) const {
    const int lane = threadIdx.x & 63;
    if (docs <= 64) {
      const int l = __builtin_ctzll(__builtin_amdgcn_ballot_w64(end > u));
      const long long before = __shfl(end, l > 0 ? l - 1 : 0, 64);
      *first = l > 0 ? tok_uniform(before) : 0;
      return l;
    }
    int lo = 0, n = docs;   // candidates lo .. lo + n - 1: the last one that begins at u or before; n shrinks to n / 64 with every turn
    while (n > 1) {
      const int step = (n + 63) >> 6;
      const bool in = lane * step < n;
      const unsigned long long m = __builtin_amdgcn_ballot_w64(in && table[in ? lo + lane * step : 0] <= u);
      const int l = 63 - __builtin_clzll(m | 1);
      lo += l * step;
      n = n - l * step < step ? n - l * step : step;
    }
    *first = tok_uniform(table[lo]);
    return lo;
  }
};
// What a workgroup does of one column tile: rows' blocks a .. b - 1.  slot < 0: all of them; else the place of its partial results
struct TokSeg { int head, doc, tile, a, b, slot; TokSpan c, r; };
struct TokJoin { int pieces, head, doc, tile; };   // the tile that began in a workgroup and goes on in the next ones; pieces 0: none
// Neighbouring workgroups (dealt to the eight XCDs in turn) are made neighbours within an XCD: its L2 holds a head's rows
__device__ __forceinline__ int tok_block() { return (blockIdx.x & 7) * (gridDim.x >> 3) + (blockIdx.x >> 3); }
template <typename F>
__device__ __forceinline__ void tok_walk(const TokSide& c, const TokSide& r, int docs, int heads, const long long* table, TokJoin* joins, F f) {
  const TokIndex index(c, r, docs, table);
  const int me = tok_block(), blocks = gridDim.x;
  const long long all = index.all * heads;
  const long long per = (all + blocks - 1) / blocks;
  long long u = me * per;
  const long long end = u + per < all ? u + per : all;
  TokJoin join = {0, 0, 0, 0};
  while (u < end) {   // uniform
    TokSeg s;
    s.head = (int)(u / index.all);
    long long first;
    const long long v = u - s.head * index.all;
    s.doc = index.find(v, &first);
    s.c = tok_span(c, s.doc);
    s.r = tok_span(r, s.doc);
    s.c.lo = __builtin_amdgcn_readfirstlane(s.c.lo); s.c.n = __builtin_amdgcn_readfirstlane(s.c.n);
    s.r.lo = __builtin_amdgcn_readfirstlane(s.r.lo); s.r.n = __builtin_amdgcn_readfirstlane(s.r.n);
    const int n = tok_parts(s.r.n, r.per), rb = n > 0 ? n : 1;
    // never out of the matrices, whatever the starts are: those of a million slides that all begin and end anywhere have more units than 64 bits count
    if (s.head >= heads || v < first || (v - first) / rb * c.per >= s.c.n) break;
    s.tile = (int)((v - first) / rb);
    s.a = (int)((v - first) - (long long)s.tile * rb);
    s.b = end - u < rb - s.a ? s.a + (int)(end - u) : rb;
    s.slot = s.a == 0 && s.b == rb ? -1 : s.a > 0 ? me : blocks + me;
    if (s.a == 0 && s.b < rb) {
      const long long last = (u + rb - 1) / per;
      join = {(int)(last < blocks ? last : blocks - 1) - me + 1, s.head, s.doc, s.tile};
    }
    f(s);
    u += s.b - s.a;
  }
  if (threadIdx.x == 0) joins[me] = join;
}

// ---- blocks of rows into LDS ----------------------------------------------------------------------
__device__ __forceinline__ u32x4 tok_load16(__amdgpu_buffer_rsrc_t b, int voff) { return __builtin_amdgcn_raw_buffer_load_b128(b, voff, 0, 0); }

// A thread's pieces of a block of KB rows of `dim` columns: NTHR threads, 16 bytes each, rows one behind the other.  Columns from dim
// to DP and rows past the last are zeros (outside of the buffer).
template <typename T, int DP, int NTHR, int KB = TokType<T>::KB>
struct TokTile {
  static constexpr int EPC = TokType<T>::EPC, CH = DP / EPC, TOTAL = KB * CH, ITER = (TOTAL + NTHR - 1) / NTHR, LDR = tok_ldr<T, DP>();
  static_assert(TOTAL % NTHR == 0, "every thread has as many pieces");
  u32x4 v[ITER];
  int at[ITER];   // where the pieces are, from the block's first row on
  __device__ __forceinline__ TokTile() {}
  __device__ __forceinline__ TokTile(int ld, int dim) {
#pragma unroll
    for (int i = 0; i < ITER; ++i) {
      const int c = threadIdx.x + i * NTHR, row = c / CH, col = c % CH * EPC;
      at[i] = col < dim ? (row * ld + col) * (int)sizeof(T) : DMA_ABSENT;
    }
  }
  // rows 0 .. rows - 1 of p at ld
  __device__ __forceinline__ void load(const T* p, int rows, int ld, int dim) {
    const __amdgpu_buffer_rsrc_t b = dma_rows(p, rows < KB ? rows : KB, ld, dim);
#pragma unroll
    for (int i = 0; i < ITER; ++i) v[i] = tok_load16(b, at[i]);
  }
  // the same rows' columns of another head, with that tile's offsets
  __device__ __forceinline__ void load_as(const TokTile& o, const T* p, int rows, int ld, int dim) {
    const __amdgpu_buffer_rsrc_t b = dma_rows(p, rows < KB ? rows : KB, ld, dim);
#pragma unroll
    for (int i = 0; i < ITER; ++i) v[i] = tok_load16(b, o.at[i]);
  }
  // packed queries c0 .. c0 + KB - 1 of a slide with `cols` of them: p is its first query's first head of the group
  __device__ __forceinline__ void load_packed(const T* p, int c0, int cols, int ld, int dim, int group, unsigned magic) {
    if (group == 1) {   // uniform
      load(p + (long long)c0 * ld, cols - c0, ld, dim);
      return;
    }
    const int r0 = c0 / group, phase = c0 - r0 * group;
    const __amdgpu_buffer_rsrc_t b = dma_buffer(p + (long long)r0 * ld, DMA_MAX);
#pragma unroll
    for (int i = 0; i < ITER; ++i) {
      const int c = threadIdx.x + i * NTHR, row = c / CH, col = c % CH * EPC;
      const unsigned x = row + phase, r = x * magic >> 16, h = x - r * group;
      const int to = (int)((r * ld + h * dim + col) * sizeof(T));
      v[i] = tok_load16(b, col < dim && c0 + row < cols ? to : DMA_ABSENT);
    }
  }
  __device__ __forceinline__ void store(T* s) const {
#pragma unroll
    for (int i = 0; i < ITER; ++i) {
      const int c = threadIdx.x + i * NTHR, row = c / CH, col = c % CH * EPC;
      *reinterpret_cast<u32x4*>(s + row * LDR + col) = v[i];
    }
  }
};
// x / group for x < 64 + group as a product and a shift (group <= 128: the error x (group - 1) / (65536 group) is below 1 / group)
__device__ __forceinline__ unsigned tok_magic(int group) { return (65536u + group - 1) / group; }

// ---- products -------------------------------------------------------------------------------------
template <typename T, int DP> struct TokFrag { u32x4 v[DP / TokType<T>::EPC / 2]; };   // a column's DP values: the pieces 2 i + (lane / 32)
template <typename T, int DP>
__device__ __forceinline__ void tok_load_frag(TokFrag<T, DP>& f, const T* row, bool valid, int dim) {
  const int h2 = (threadIdx.x >> 5) & 1;
#pragma unroll
  for (int i = 0; i < DP / TokType<T>::EPC / 2; ++i) {
    const int col = (2 * i + h2) * TokType<T>::EPC;
    f.v[i] = u32x4{0, 0, 0, 0};
    if (valid && col < dim) f.v[i] = *reinterpret_cast<const u32x4*>(row + col);
  }
}
// Operands of a product out of LDS.
// rows j0 .. j0 + 31 of X, contraction over the DP columns
template <typename T, int DP> struct TokRows { u32x4 v[DP / TokType<T>::EPC / 2]; };
template <typename T, int DP>
__device__ __forceinline__ void tok_get(TokRows<T, DP>& x, const T* X, int j0) {
  const int li = threadIdx.x & 31, h2 = (threadIdx.x >> 5) & 1;
  const T* p = X + (j0 + li) * tok_ldr<T, DP>() + h2 * TokType<T>::EPC;
#pragma unroll
  for (int i = 0; i < DP / TokType<T>::EPC / 2; ++i) x.v[i] = *reinterpret_cast<const u32x4*>(p + 2 * i * TokType<T>::EPC);
}
// acc[rows][columns] += X f
template <typename T, int DP>
__device__ __forceinline__ void tok_mul(f32x16& acc, const TokRows<T, DP>& x, const TokFrag<T, DP>& f) {
#pragma unroll
  for (int i = 0; i < DP / TokType<T>::EPC / 2; ++i) {
    if constexpr (sizeof(T) == 2) {
      acc = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, x.v[i]), __builtin_bit_cast(bf16x8, f.v[i]), acc, 0, 0, 0);
    } else {
      const f32x4 fa = __builtin_bit_cast(f32x4, x.v[i]), fb = __builtin_bit_cast(f32x4, f.v[i]);
#pragma unroll
      for (int e = 0; e < 4; ++e) acc = __builtin_amdgcn_mfma_f32_32x32x2f32(fa[e], fb[e], acc, 0, 0, 0);
    }
  }
}
// the transpose of rows j0 .. j0 + 31 of X, contraction over the rows in the order in which an accumulator holds them
template <typename T, int DP> struct TokCols;
template <int DP> struct TokCols<bf16, DP> { bf16x8 v[2][DP / 32]; };
template <int DP> struct TokCols<float, DP> { const float* at; };   // read one by one at the products, whose 64 cycles cover it
template <int DP>
__device__ __forceinline__ void tok_get_t(TokCols<bf16, DP>& x, const bf16* X, int j0) {
  // LDS transpose reads: within 16 lanes, lane s addresses four columns of row s / 4 and receives column s of the four rows
  typedef short s16x4 __attribute__((ext_vector_type(4)));
  typedef short s16x8 __attribute__((ext_vector_type(8)));
  constexpr int LDR = tok_ldr<bf16, DP>();
  const int lane = threadIdx.x & 63, g = lane >> 4, s = lane & 15;
  const bf16* q = X + (j0 + 4 * (g >> 1) + (s >> 2)) * LDR + 16 * (g & 1) + (s & 3) * 4;
#pragma unroll
  for (int t = 0; t < 2; ++t)
#pragma unroll
    for (int d = 0; d < DP / 32; ++d) {
      const bf16* at = q + 16 * t * LDR + d * 32;
      const s16x4 a = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s16x4*)at);
      const s16x4 b = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s16x4*)(at + 8 * LDR));
      const s16x8 v = {a[0], a[1], a[2], a[3], b[0], b[1], b[2], b[3]};
      x.v[t][d] = __builtin_bit_cast(bf16x8, v);
    }
}
template <int DP>
__device__ __forceinline__ void tok_get_t(TokCols<float, DP>& x, const float* X, int j0) {
  x.at = X + (j0 + 4 * ((threadIdx.x >> 5) & 1)) * tok_ldr<float, DP>() + (threadIdx.x & 31);
}
// acc[DP][columns] += X^T p.  bfloat16: p is rounded to it (half a step, 2^-8 of each probability at most and of either sign, where the
// result's own rounding is as large); the matrix cores take no wider operand beside bfloat16.  EXACT: p goes in as two terms, which leaves 2^-16 of it,
// where that costs nothing: a wavefront that waits for memory.
template <int DP, bool EXACT>
__device__ __forceinline__ void tok_mul_t(f32x16 (&acc)[DP / 32], const TokCols<bf16, DP>& x, const f32x16& p) {
#pragma unroll
  for (int t = 0; t < 2; ++t) {
    bf16x8 b, rest;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      b[i] = (bf16)p[8 * t + i];
      if (EXACT) rest[i] = (bf16)(p[8 * t + i] - (float)b[i]);
    }
#pragma unroll
    for (int d = 0; d < DP / 32; ++d) {
      acc[d] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(x.v[t][d], b, acc[d], 0, 0, 0);
      if (EXACT) acc[d] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(x.v[t][d], rest, acc[d], 0, 0, 0);
    }
  }
}
template <int DP, bool>
__device__ __forceinline__ void tok_mul_t(f32x16 (&acc)[DP / 32], const TokCols<float, DP>& x, const f32x16& p) {
#pragma unroll
  for (int r = 0; r < 16; ++r)
#pragma unroll
    for (int d = 0; d < DP / 32; ++d)
      acc[d] = __builtin_amdgcn_mfma_f32_32x32x2f32(x.at[((r >> 2) * 8 + (r & 3)) * tok_ldr<float, DP>() + d * 32], p[r], acc[d], 0, 0, 0);
}
// row of a block of 32 that register r of this lane holds
__device__ __forceinline__ int tok_row(int r) { return (r >> 2) * 8 + ((threadIdx.x >> 5) & 1) * 4 + (r & 3); }
__device__ __forceinline__ f32x16 tok_zero() {
  f32x16 z;
#pragma unroll
  for (int r = 0; r < 16; ++r) z[r] = 0.f;
  return z;
}
template <int N>
__device__ __forceinline__ void tok_zero_all(f32x16 (&a)[N]) {
#pragma unroll
  for (int d = 0; d < N; ++d) a[d] = tok_zero();
}
// a column's DP results (down the registers) times f to `dim` elements at `row`
template <typename O, int N>
__device__ __forceinline__ void tok_store(const f32x16 (&a)[N], float f, O* row, int dim) {
  const int h2 = (threadIdx.x >> 5) & 1;
  typedef O O4 __attribute__((ext_vector_type(4)));
#pragma unroll
  for (int d = 0; d < N; ++d)
#pragma unroll
    for (int g = 0; g < 4; ++g) {
      const int col = d * 32 + g * 8 + h2 * 4;
      O4 v;
#pragma unroll
      for (int i = 0; i < 4; ++i) v[i] = (O)(a[d][g * 4 + i] * f);
      if (col < dim) *reinterpret_cast<O4*>(row + col) = v;
    }
}

// a value of the lane and of the other one of its column (lane ^ 32), without a way through LDS
__device__ __forceinline__ float tok_other_max(float v) {
  const auto x = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  return fmaxf(__uint_as_float(x[0]), __uint_as_float(x[1]));
}
__device__ __forceinline__ float tok_other_sum(float v) {
  const auto x = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  return __uint_as_float(x[0]) + __uint_as_float(x[1]);
}

// ---- scores ---------------------------------------------------------------------------------------
// A score is kept as z, a probability is 2^(ex z - ex max z): without a cap z = qk - slope / scale * d, so that the scale costs nothing beside
// the maximum; with one z = c2 tanh(c1 qk) - slope d, all in units of log2(e), and ex is 1.
struct TokScore { float c1, c2, ex, per_slope; };
// kernels without a cap, with one, and with one so large that bfloat16 takes float32's tanh too
enum TokCapped : int { TOK_UNCAPPED = 0, TOK_CAPPED = 1, TOK_CAPPED_FAR = 2 };
constexpr float TOK_CAP_NEAR = 64.f;
template <int CAP>
__device__ __forceinline__ TokScore tok_score_of(float scale, float cap) {
  return CAP ? TokScore{scale / cap, cap * TOK_LOG2E, 1.f, TOK_LOG2E} : TokScore{0.f, 0.f, scale * TOK_LOG2E, 1.f / scale};
}
// tanh(u) and a quarter of its derivative.  float32: e = exp(-2 |u|), (1 - e) / (1 + e) and e / (1 + e)^2, which lose nothing for large |u|; for small
// |u| 1 - e has e's rounding, 2^-25 of one, and the series is taken (next term 2^-27 of u at 1/4).
// bfloat16: r = 1 / (1 + exp(2 u)), 1 - 2 r and r (1 - r), four operations fewer.  However small u is, 1 - 2 r is off by up to six units of 2^-24 (those of
// the exponential, the sum and the reciprocal, twice), and a score by that times the cap: 1.3e-5 at a cap of 50, 2.3e-5 at most at TOK_CAP_NEAR, where
// a probability is rounded to 2^-8 of itself.  Beyond, that would count (a cap of 2^20: scores off by 0.1, of 2^25: all of them 0), and float32's form is
// taken (16 slides, 8 heads of 128: 147 us in the one, 168 in the other; 7 slides, 12 heads of 64, both directions: 211 and 270).
template <typename T, int CAP, bool SLOPE>
__device__ __forceinline__ float tok_cap(float qk, const TokScore& c, float* slope) {
  if constexpr (sizeof(T) == 2 && CAP == TOK_CAPPED) {
    const float r = __builtin_amdgcn_rcpf(1.f + __builtin_amdgcn_exp2f(qk * (c.c1 * (2.f * TOK_LOG2E))));
    if (SLOPE) *slope = fmaf(-r, r, r);
    return fmaf(r, -2.f * c.c2, c.c2);
  } else {
    const float u = qk * c.c1, a = fabsf(u);
    const float e = __builtin_amdgcn_exp2f(-2.f * TOK_LOG2E * a), r = __builtin_amdgcn_rcpf(1.f + e);
    if (SLOPE) *slope = e * r * r;
    const float w = u * u;
    const float series = a * fmaf(w, fmaf(w, fmaf(w, fmaf(w, 62.f / 2835.f, -17.f / 315.f), 2.f / 15.f), -1.f / 3.f), 1.f);
    return c.c2 * copysignf(a < 0.25f ? series : (1.f - e) * r, u);
  }
}
// slope: times c.per_slope
template <typename T, bool BIAS, int CAP, bool SLOPE>
__device__ __forceinline__ float tok_score(float qk, float d, float slope, const TokScore& c, float* dt) {
  const float z = CAP ? tok_cap<T, CAP, SLOPE>(qk, c, dt) : qk;
  return BIAS ? fmaf(-slope, d, z) : z;
}
// 2^(ex z - at)
template <int CAP>
__device__ __forceinline__ float tok_exp(float z, float at, const TokScore& c) {
  return __builtin_amdgcn_exp2f(CAP ? z - at : fmaf(z, c.ex, -at));
}
__device__ __forceinline__ float tok_dist(float ax, float ay, float bx, float by) {
  const float x = ax - bx, y = ay - by;
  return __builtin_amdgcn_sqrtf(fmaf(x, x, y * y));   // within an ulp
}

// Positions of a block's keys: 0 for keys without a place and behind the last.  Loaded a block ahead, like the tiles
struct TokPlace { float x, y; };
template <int KB>
__device__ __forceinline__ TokPlace tok_place(const float* pos, int lo, int k0, int n, int lead) {
  const int j = k0 + threadIdx.x;
  TokPlace p = {0.f, 0.f};
  if (threadIdx.x < KB && j < n && j >= lead) {
    const float2 v = *reinterpret_cast<const float2*>(pos + 2LL * (lo + j));
    p.x = v.x; p.y = v.y;
  }
  return p;
}

// Heads that a wavefront takes together where there is a bias, because the distances are then taken once for them: `heads` groups of NH, of
// `pack` heads beside each other in the columns; the n-th of a group's is `step` heads on, its key head `kv_step` on.
// One group a key head and all of its heads packed where NH is 1; half of them where 2 and they share a key head; two key heads else.
struct TokHeads { int heads, pack, step, kv_step; };
inline __host__ __device__ TokHeads tok_heads(const TokAttn& g, int nh) {
  if (nh == 1) return {g.hk, g.group, 0, 0};
  if (g.group == 1) return {g.hk / 2, 1, 1, 1};
  return {g.hk, g.group / 2, g.group / 2, 0};
}
// the sides of a pass: queries packed with the heads of a group, and keys
__device__ __forceinline__ TokSide tok_queries(const TokAttn& g, int per, int pack) { return {g.q_start, g.rows_q, pack, per}; }
__device__ __forceinline__ TokSide tok_keys(const TokAttn& g, int per) { return {g.k_start, g.rows_k, 1, per}; }

// Distances of a block's 32 rows from the columns, as scores lie: the differences of each coordinate are a product of two terms, (row, 1) (1, -column), in
// float32 on the matrix cores, which have nothing else to do while the vector unit works: one rounding, as the subtraction has.  px, py: the
// rows' coordinates in LDS; cx, cy: the column's.  (Read row by row they were 8 of 28 reads of 16 bytes a block, and 2 of 13 operations a score.)
template <typename T>
__device__ __forceinline__ void tok_dists(f32x16& d, const float* px, const float* py, int j0, float cx, float cy) {
  if constexpr (sizeof(T) == 4) {   // there the matrix cores are what is short
#pragma unroll
    for (int q4 = 0; q4 < 4; ++q4) {
      const f32x4 x = *reinterpret_cast<const f32x4*>(px + j0 + tok_row(q4 * 4)), y = *reinterpret_cast<const f32x4*>(py + j0 + tok_row(q4 * 4));
#pragma unroll
      for (int i = 0; i < 4; ++i) d[q4 * 4 + i] = tok_dist(x[i], y[i], cx, cy);
    }
    return;
  }
  const bool second = (threadIdx.x & 32) != 0;   // the term that this half of the wavefront holds
  const int row = j0 + (threadIdx.x & 31);
  const float ax = second ? 1.f : px[row], ay = second ? 1.f : py[row];
  const f32x16 x = __builtin_amdgcn_mfma_f32_32x32x2f32(ax, second ? -cx : 1.f, tok_zero(), 0, 0, 0);
  const f32x16 y = __builtin_amdgcn_mfma_f32_32x32x2f32(ay, second ? -cy : 1.f, tok_zero(), 0, 0, 0);
#pragma unroll
  for (int r = 0; r < 16; ++r) d[r] = __builtin_amdgcn_sqrtf(fmaf(x[r], x[r], y[r] * y[r]));   // within an ulp
}

// dispatch on the padded head width, bias and cap
template <typename T, typename F>
hipError_t tok_dispatch(const TokAttn& g, F f) {
  auto by_cap = [&](auto dp, auto bias) {
    if constexpr (sizeof(T) == 2) {
      if (g.cap > TOK_CAP_NEAR) return f(dp, bias, std::integral_constant<int, TOK_CAPPED_FAR>{});
    }
    return g.cap > 0.f ? f(dp, bias, std::integral_constant<int, TOK_CAPPED>{}) : f(dp, bias, std::integral_constant<int, TOK_UNCAPPED>{});
  };
  auto by_bias = [&](auto dp) { return g.slopes ? by_cap(dp, std::true_type{}) : by_cap(dp, std::false_type{}); };
  if (g.dim <= 32) return by_bias(std::integral_constant<int, 32>{});
  if (g.dim <= 64) return by_bias(std::integral_constant<int, 64>{});
  if (g.dim <= 96) return by_bias(std::integral_constant<int, 96>{});
  return by_bias(std::integral_constant<int, 128>{});
}

}  // namespace sl
