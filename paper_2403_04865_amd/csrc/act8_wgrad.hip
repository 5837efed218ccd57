// Weight gradient out of an 8-bit activation checkpoint (gfx950): dW[n][k] = sum_m dy[m][n] x8[m][k], db[n] = sum_m dy[m][n].
//
// A code times its power of two is exactly a bfloat16 (from 2^-133 on), so the checkpoint is decoded on its way into LDS and the products are the
// matrix cores' bfloat16 ones with float32 sums; float32 gradients go in as three bfloat16 terms of 2^48 times their value (split_f32.h), which
// are all of their bits, and blocks that come out infinite that way are taken again.  The contraction runs over the rows of both operands: 64-row slices lie in LDS as they are in memory and the fragments,
// eight consecutive rows of a column per lane, are read with the transposing LDS reads.
// The rows are split into slabs: a work item is (slab, output tile), writes its partial tile once, and a second kernel adds the slabs
// in a fixed order.
// Bound by what feeds the matrix cores, not by bytes: 403456 x 384 -> 1536 takes 545 us, 0.87 PFLOP/s (a library product of
// 8192 reaches 1.46; the bytes alone take 271 us); float32 1858 us, three products for one; 7289 x 384 -> 1152 26 and 40 us, 65536 x 1024 -> 1024
// 166 and 493.
#include "act8_internal.h"
#include "lds_dma.h"
#include "split_f32.h"

namespace sl {

namespace {

typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef short s16x8 __attribute__((ext_vector_type(8)));

constexpr int BX = 128, BK = 64, NW = 8, NTH = 64 * NW, WVN = 4;   // wavefronts: 2 x 4
constexpr int XCHUNKS = BX / 8 * BK / NTH;   // pieces of eight columns of dy per thread and step
constexpr int MAX_SLABS = 64;

struct Item {   // the kernel's view of one problem
  A8Wgrad g;
  int TX, TY, slabs;
  long long per;        // rows of a slab, a multiple of BK
  float *part, *cpart;  // [slabs][N][K], [slabs][N]; null with one slab
};

// MFMA operand from a row-major LDS slice S[row][col] (row stride LDW): lane l gets column c0 + l % 32 of rows
// k0 + 8 (l / 32) .. + 7
template <int LDW>
__device__ __forceinline__ bf16x8 frag_tr(const bf16* S, int c0, int k0, int lane) {
  const int g = lane >> 4, q = lane & 15;
  const bf16* p = S + (k0 + 8 * (g >> 1) + (q >> 2)) * LDW + c0 + 16 * (g & 1) + (q & 3) * 4;
  const s16x4 a = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s16x4*)p);
  const s16x4 b = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s16x4*)(p + 4 * LDW));
  const s16x8 r = {a[0], a[1], a[2], a[3], b[0], b[1], b[2], b[3]};
  return __builtin_bit_cast(bf16x8, r);
}

// 16 codes times their power of two, as two pieces of eight bfloat16 (the instruction is exact for every code under every scale)
__device__ __forceinline__ void decode16(const u32x4& q, float s, bf16x8 (&o)[2]) {
  typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
#pragma unroll
  for (int w = 0; w < 4; ++w) {
    const bf16x2 lo = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(q[w], s, false), hi = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(q[w], s, true);
    o[w >> 1][4 * (w & 1) + 0] = lo[0]; o[w >> 1][4 * (w & 1) + 1] = lo[1];
    o[w >> 1][4 * (w & 1) + 2] = hi[0]; o[w >> 1][4 * (w & 1) + 3] = hi[1];
  }
}

// YG: the tile is 128 rows of dW by 128 YG columns.  V: dy's rows can be read in 16-byte pieces.
template <typename T, int YG, bool V>
__global__ void __launch_bounds__(NTH) wgrad_k(Item it) {
  constexpr int TERMS = sizeof(T) == 2 ? 1 : 3;
  constexpr int BY = 128 * YG, LDW = TERMS * BX + BY + 32, STAGE = BK * LDW;
  constexpr int YCHUNKS = BY / 16 * BK / NTH;
  constexpr int WBN = BY / (32 * WVN);   // 32-column products of a wavefront; two of 32 rows
  __shared__ __attribute__((aligned(16))) bf16 ring0[STAGE], ring1[STAGE];
  __shared__ float scale[4][BK * YG];
  const A8Wgrad& g = it.g;
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int wm = wave / WVN, wn = wave % WVN;
  // work items in the order of the XCDs: a slab's tiles run on one, next to each other, and share its rows in that L2
  const int per_xcd = gridDim.x / 8;
  const int id = (blockIdx.x % 8) * per_xcd + blockIdx.x / 8;
  const int tiles = it.TX * it.TY;
  if (id >= tiles * it.slabs) return;
  const int slab = id / tiles, tile = id % tiles;
  const int x0 = tile / it.TY * BX, y0 = tile % it.TY * BY;
  const float up = TERMS > 1 ? split_up(slab) : 1.f;   // (slabs of either sign)
  const long long lo = slab * it.per;
  const int span = lo >= g.M ? 0 : (int)(g.M - lo < it.per ? g.M - lo : it.per);
  const int steps = (span + BK - 1) / BK;
  const int k16 = (g.K + A8_GRAIN - 1) / A8_GRAIN * A8_GRAIN;

  const int xr = tid >> 4, xc = (tid & 15) * 8;            // dy: rows xr + 32 i
  const int yr = tid / (BY / 16), yc = tid % (BY / 16) * 16;   // codes: rows yr + (NTH / (BY / 16)) j, one column of pieces
  constexpr int XR = NTH / 16, YR = NTH / (BY / 16);
  static_assert(YR * (BY / 16) == NTH || YG == 3, "loader split");
  const bool bias = g.db && y0 == 0;   // uniform
  struct Rows { T x[XCHUNKS][8]; u32x4 y[YCHUNKS]; } r0, r1;   // this thread's pieces of the rows of odd and of even steps
  // Buffers of one step's 64 rows, so that offsets stay small; rows that do not exist are outside of them: zeros.
  const int ldx = (int)(V ? g.lddy * (long long)sizeof(T) : 0), ldc = (int)g.x.ldc, lds = (int)g.x.lds;
  const int vx = V && x0 + xc < g.N ? xr * ldx + xc * (int)sizeof(T) : DMA_ABSENT;
  auto rows_left = [&](int step) { const int r = span - step * BK; return r < BK ? r : BK; };
  auto fetch_x = [&](Rows& R, int step) __attribute__((always_inline)) {
    const T* p = (const T*)g.dy + (lo + (long long)step * BK) * g.lddy + x0;
    const int left = rows_left(step);
    if constexpr (V) {
      const __amdgpu_buffer_rsrc_t b = dma_buffer(p, left > 0 ? (left - 1) * (long long)ldx + (g.N - x0) * (long long)sizeof(T) : 0);
#pragma unroll
      for (int i = 0; i < XCHUNKS; ++i)
#pragma unroll
        for (int h = 0; h < (int)sizeof(T) / 2; ++h)
          *reinterpret_cast<u32x4*>(&R.x[i][h * (16 / sizeof(T))]) = __builtin_amdgcn_raw_buffer_load_b128(b, vx + 16 * h, XR * i * ldx, 0);
    } else {
#pragma unroll
      for (int i = 0; i < XCHUNKS; ++i)
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          const int r = xr + XR * i;
          R.x[i][e] = r < left && x0 + xc + e < g.N ? p[r * g.lddy + xc + e] : (T)0.f;
        }
    }
  };
  auto piece = [&](int j, int* row, int* col) {   // with 24 pieces a row the threads do not stay in their column
    const int c = tid + NTH * j;
    *row = YG == 3 ? c / (BY / 16) : yr + YR * j;
    *col = YG == 3 ? c % (BY / 16) * 16 : yc;
  };
  auto fetch_y = [&](Rows& R, int step) __attribute__((always_inline)) {
    const long long row0 = lo + (long long)step * BK;
    const int left = rows_left(step);
    const __amdgpu_buffer_rsrc_t b = dma_buffer(g.x.codes + row0 * g.x.ldc + y0, left > 0 ? (left - 1) * (long long)ldc + k16 - y0 : 0);
#pragma unroll
    for (int j = 0; j < YCHUNKS; ++j) {
      int row, col;
      piece(j, &row, &col);
      R.y[j] = __builtin_amdgcn_raw_buffer_load_b128(b, y0 + col < k16 ? row * ldc + col : DMA_ABSENT, 0, 0);
    }
  };
  // The powers of a step's rows and blocks: one byte of memory by each of the first 64 YG threads, through LDS to the threads that decode
  // (as a byte load beside every piece of codes: 641 us for 403456 x 1536 -> 384, 518 without).
  const bool scaler = tid < BK * YG;
  auto fetch_s = [&](int step) __attribute__((always_inline)) {
    const int left = rows_left(step), row = tid / YG, blk = tid - row * YG;
    const __amdgpu_buffer_rsrc_t sb = dma_buffer(g.x.scales + (lo + (long long)step * BK) * g.x.lds + (y0 >> 7),
                                                 left > 0 ? (left - 1) * (long long)lds + ((k16 - y0 + 127) >> 7) : 0);
    return (unsigned)__builtin_amdgcn_raw_buffer_load_b8(sb, scaler && y0 + 128 * blk < k16 ? row * lds + blk : DMA_ABSENT, 0, 0);
  };
  auto put_s = [&](int step, unsigned b) __attribute__((always_inline)) {
    if (scaler) scale[step & 3][tid] = a8_scale(b);
  };
  auto stash_x = [&](const Rows& R, bf16* S, int i) __attribute__((always_inline)) {
    bf16* p = S + (xr + XR * i) * LDW + xc;
    float f[8];
    if constexpr (TERMS > 1) {
#pragma unroll
      for (int e = 0; e < 8; ++e) f[e] = to_f(R.x[i][e]) * up;
    }
#pragma unroll
    for (int t = 0; t < TERMS; ++t) {
      bf16x8 o;
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        if constexpr (TERMS == 1) o[e] = R.x[i][e];
        else {
          o[e] = (bf16)f[e];
          f[e] -= (float)o[e];   // (no number behind what rounds to an infinity: such blocks are taken again)
        }
      }
      *reinterpret_cast<bf16x8*>(p + t * BX) = o;
    }
  };
  auto stash_y = [&](const Rows& R, bf16* S, int step, int j) __attribute__((always_inline)) {
    int row, col;
    piece(j, &row, &col);
    bf16x8 o[2];
    decode16(R.y[j], scale[step & 3][row * YG + (col >> 7)], o);
    bf16* p = S + row * LDW + TERMS * BX + col;
    *reinterpret_cast<bf16x8*>(p) = o[0];
    *reinterpret_cast<bf16x8*>(p + 8) = o[1];
  };

  f32x16 acc[2][WBN];
#pragma unroll
  for (int i = 0; i < 2; ++i)
#pragma unroll
    for (int j = 0; j < WBN; ++j)
#pragma unroll
      for (int r = 0; r < 16; ++r) acc[i][j][r] = 0.f;

  struct Frags { bf16x8 x[TERMS][2], y[WBN]; };
  auto read = [&](Frags& f, const bf16* S, int k) __attribute__((always_inline)) {   // 16 rows of the stage
#pragma unroll
    for (int j = 0; j < WBN; ++j) f.y[j] = frag_tr<LDW>(S, TERMS * BX + (wn * WBN + j) * 32, k, lane);
#pragma unroll
    for (int t = 0; t < TERMS; ++t)
#pragma unroll
      for (int i = 0; i < 2; ++i) f.x[t][i] = frag_tr<LDW>(S, t * BX + (wm * 2 + i) * 32, k, lane);
  };
  // Bias gradient out of the fragments, whose lanes hold eight rows of a column: four two-term sums a fragment, and the four wavefronts that
  // read the same ones take a slice each (as additions of what a thread loads, or as products with ones: 100 to 150 us of the 690 of
  // 403456 x 384 -> 1536).
  float cs[2] = {0.f, 0.f};
  auto multiply = [&](const Frags& f, int q) __attribute__((always_inline)) {   // q: slice
    if (bias && wn == q) {   // uniform
      typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
      const bf16x2 one = {(bf16)1.f, (bf16)1.f};
#pragma unroll
      for (int t = 0; t < TERMS; ++t)
#pragma unroll
        for (int i = 0; i < 2; ++i)
#pragma unroll
          for (int e = 0; e < 8; e += 2) cs[i] = __builtin_amdgcn_fdot2_f32_bf16(bf16x2{f.x[t][i][e], f.x[t][i][e + 1]}, one, cs[i], false);
    }
#pragma unroll
    for (int t = 0; t < TERMS; ++t)
#pragma unroll
      for (int i = 0; i < 2; ++i)
#pragma unroll
        for (int j = 0; j < WBN; ++j) acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(f.x[t][i], f.y[j], acc[i][j], 0, 0, 0);
    __builtin_amdgcn_sched_barrier(0);
  };
  // A step multiplies out of one stage, writes what was fetched two steps ago to the other and fetches the rows two steps after
  // those, and the decoding and the LDS writes lie between the products of the slices.  The fragments are read a slice
  // ahead; the barrier (it waits for LDS, not for the loads) stands before the last slice's products, so that the next step's first
  // fragments come under these.
  Frags fa, fb;
  unsigned s0 = 0, s1 = 0;   // scales of the next even and odd step but one
  auto step = [&](int s, const bf16* S, bf16* N, Rows& R, unsigned& sr) __attribute__((always_inline)) {
    const bool more = s + 1 < steps;   // uniform
    read(fb, S, 16);
    if (more) {
#pragma unroll
      for (int i = 0; i < XCHUNKS; ++i) stash_x(R, N, i);
    }
    fetch_x(R, s + 3);
    put_s(s + 2, sr);
    sr = fetch_s(s + 4);
    multiply(fa, 0);
    read(fa, S, 32);
    if (more) {
#pragma unroll
      for (int j = 0; j < YCHUNKS; ++j) stash_y(R, N, s + 1, j);
    }
    fetch_y(R, s + 3);
    multiply(fb, 1);
    read(fb, S, 48);
    multiply(fa, 2);
    step_barrier();
    if (more) read(fa, N, 0);
    multiply(fb, 3);
  };
  if (steps > 0) {
    fetch_x(r1, 0);
    fetch_y(r1, 0);
    const unsigned first = fetch_s(0), second = fetch_s(1);
    s0 = fetch_s(2);
    s1 = fetch_s(3);
    fetch_x(r0, 1);
    fetch_y(r0, 1);
    put_s(0, first);
    put_s(1, second);
    __syncthreads();
#pragma unroll
    for (int i = 0; i < XCHUNKS; ++i) stash_x(r1, ring0, i);
#pragma unroll
    for (int j = 0; j < YCHUNKS; ++j) stash_y(r1, ring0, 0, j);
    fetch_x(r1, 2);
    fetch_y(r1, 2);
  }
  __syncthreads();
  if (steps > 0) read(fa, ring0, 0);
  for (int s = 0; s < steps; s += 2) {
    step(s, ring0, ring1, r0, s0);
    if (s + 1 < steps) step(s + 1, ring1, ring0, r1, s1);
  }

  // Float32: back from 2^48.  A block with a result that is not finite (a gradient of 2^80 or more, a result as large, an infinity, a NaN) is taken
  // again from memory, in sums of double: 403456 x 384 -> 1536 with one NaN in it 106 ms, 2 without.
  if constexpr (TERMS > 1) {
    if (not_finite(acc)) {   // of this wavefront
#pragma unroll
      for (int i = 0; i < 2; ++i)
#pragma unroll
        for (int j = 0; j < WBN; ++j) {
          const int n0 = x0 + (wm * 2 + i) * 32 + 4 * (lane >> 5), k0 = y0 + (wn * WBN + j) * 32 + (lane & 31), k = k0 < g.K ? k0 : g.K - 1;
          const long long n_last = g.N - 1;   // (what is not there: the last one again; it is not stored)
          double a[16];
#pragma unroll
          for (int r = 0; r < 16; ++r) a[r] = 0.0;
#pragma unroll 4
          for (int m = 0; m < span; ++m) {
            const T* d = (const T*)g.dy + (lo + m) * g.lddy;
            const double v = __builtin_amdgcn_cvt_f32_fp8(g.x.codes[(lo + m) * g.x.ldc + k], 0) * a8_scale(g.x.scales[(lo + m) * g.x.lds + (k >> 7)]);
            float t[16];
#pragma unroll
            for (int r = 0; r < 16; ++r) {
              const long long n = n0 + 8 * (r >> 2) + (r & 3);
              t[r] = to_f(d[n < n_last ? n : n_last]);
            }
#pragma unroll
            for (int r = 0; r < 16; ++r) a[r] = fma((double)t[r], v, a[r]);
          }
#pragma unroll
          for (int r = 0; r < 16; ++r) acc[i][j][r] = (float)a[r];
        }
    } else scale_down(acc, up);
  }

  // lane: column l % 32, rows 8 (r / 4) + 4 (l / 32) + r % 4
  const bool direct = it.slabs == 1;
  float* out = direct ? g.dW : it.part + (long long)slab * g.N * g.K;
  const long long ldo = direct ? g.lddw : g.K;
#pragma unroll
  for (int i = 0; i < 2; ++i)
#pragma unroll
    for (int j = 0; j < WBN; ++j) {
      const int k = y0 + (wn * WBN + j) * 32 + (lane & 31);
#pragma unroll
      for (int r = 0; r < 16; ++r) {
        const int n = x0 + (wm * 2 + i) * 32 + 8 * (r >> 2) + 4 * (lane >> 5) + (r & 3);
        if (n < g.N && k < g.K) {
          float* p = out + n * ldo + k;
          *p = direct && g.accumulate ? *p + acc[i][j][r] : acc[i][j][r];
        }
      }
    }
  // bias gradient: the four wavefronts' slices, in order
  if (bias) {
    __syncthreads();
    float* red = reinterpret_cast<float*>(ring0);   // [4][128]
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const float v = cs[i] + __shfl_xor(cs[i], 32, 64);
      if (lane < 32) red[wn * BX + (wm * 2 + i) * 32 + lane] = v;
    }
    __syncthreads();
    if (tid < BX && x0 + tid < g.N) {
      float v = (red[tid] + red[BX + tid]) + (red[2 * BX + tid] + red[3 * BX + tid]);
      if constexpr (TERMS > 1) {
        if (a8_mag(v) || v == 0.f) v *= 1.0f / SPLIT_UP / SPLIT_UP * up;
        else {   // not finite: as above
          double a = 0.0;
#pragma unroll 1
          for (int m = 0; m < span; ++m) a += to_f(((const T*)g.dy)[(lo + m) * g.lddy + x0 + tid]);
          v = (float)a;
        }
      }
      if (direct) g.db[x0 + tid] = g.accumulate ? g.db[x0 + tid] + v : v;
      else it.cpart[(long long)slab * g.N + x0 + tid] = v;
    }
  }
}

// dW = (accumulate ? dW : 0) + the slabs' partials, in order; db likewise (the entries behind the last of dW)
__global__ void __launch_bounds__(256) wgrad_sum_k(Item it) {
  const A8Wgrad& g = it.g;
  const long long nk = (long long)g.N * g.K, all = nk + (g.db ? g.N : 0);
  for (long long i = (long long)blockIdx.x * 256 + threadIdx.x; i < all; i += (long long)gridDim.x * 256) {
    const bool w = i < nk;
    const long long stride = w ? nk : g.N;
    const float* p = w ? it.part + i : it.cpart + (i - nk);
    float v = 0.f;
    for (int s = 0; s < it.slabs; ++s) v += p[s * stride];
    float* o = w ? g.dW + i / g.K * g.lddw + i % g.K : g.db + (i - nk);
    *o = g.accumulate ? *o + v : v;
  }
}

// Tile width (128 yg columns) and slabs that a model of the time says are the fastest.  Its parts were measured (microseconds): a step of a
// workgroup 0.85, 1.3, 1.65 (yg 1, 2, 3; float32 1.6), 1.45 where two workgroups of yg 1 share a compute unit; launches and prologue 4;
// a second kernel 5, and a slab's partial out and back at 6 MB a microsecond.  It finds 7289 x 384 -> 1152: yg 1, 8 slabs, 28 us (yg 3:
// 30 at best); 403456 x 384 -> 1536: yg 3, 21 slabs, 545 us (yg 1: 661); 65536 x 1024 -> 1024: yg 2, 8 slabs, 181 us.
void plan(long long M, int N, int K, bool f32, Item* it, int* width) {
  const long long steps = (M + BK - 1) / BK;
  double best = 1e300;
  for (int yg = 1; yg <= (f32 ? 1 : 3); ++yg) {
    const int TX = (N + BX - 1) / BX, TY = (int)((K + 128LL * yg - 1) / (128 * yg));
    const long long tiles = (long long)TX * TY, slots = yg == 1 && !f32 ? 512 : 256;
    for (int s = 1; s <= MAX_SLABS && (s == 1 || steps / s >= 2); ++s) {
      const long long wgs = tiles * s, rounds = (wgs + slots - 1) / slots;
      const double t = f32 ? 1.6 : yg == 1 ? (wgs > 256 ? 1.45 : 0.85) : yg == 2 ? 1.3 : 1.65;
      const double cost = (double)rounds * (double)((steps + s - 1) / s) * t + 4 + (s > 1 ? 5 + (double)s * N * K * 8e-6 / 6.0 : 0.0);
      if (cost < best) { best = cost; it->slabs = s; it->TX = TX; it->TY = TY; *width = yg; }
    }
  }
  it->per = (steps + it->slabs - 1) / it->slabs * BK;
}

template <typename T, bool V>
hipError_t run(const Item& it, int yg, hipStream_t s) {
  const unsigned grid = (unsigned)((it.TX * it.TY * it.slabs + 7) / 8 * 8);
  if (sizeof(T) == 4) wgrad_k<T, 1, V><<<grid, NTH, 0, s>>>(it);
  else if (yg == 1) wgrad_k<T, 1, V><<<grid, NTH, 0, s>>>(it);
  else if (yg == 2) wgrad_k<T, sizeof(T) == 4 ? 1 : 2, V><<<grid, NTH, 0, s>>>(it);
  else wgrad_k<T, sizeof(T) == 4 ? 1 : 3, V><<<grid, NTH, 0, s>>>(it);
  return hipGetLastError();
}

size_t part_bytes(const Item& it, int N, int K) {
  return it.slabs == 1 ? 0 : (((size_t)it.slabs * N * K * 4 + 255) & ~(size_t)255) + (size_t)it.slabs * N * 4;
}

}  // namespace

size_t act8_wgrad_bytes(long long M, int N, int K) {
  Item a{}, b{};
  int yg;
  plan(M, N, K, false, &a, &yg);
  plan(M, N, K, true, &b, &yg);
  const size_t x = part_bytes(a, N, K), y = part_bytes(b, N, K);
  return ((x > y ? x : y) + 256 + 255) & ~(size_t)255;
}

hipError_t launch_act8_wgrad(const A8Wgrad& g, hipStream_t s) {
  int yg;
  Item it{};
  it.g = g;
  plan(g.M, g.N, g.K, g.dt == DT_F32, &it, &yg);
  it.part = g.work;
  it.cpart = g.work + (((size_t)it.slabs * g.N * g.K * 4 + 255) & ~(size_t)255) / 4;
  const size_t es = elem_size(g.dt);
  // whole 16-byte pieces of eight columns, 32-bit offsets within 64 rows
  const bool v = ((uintptr_t)g.dy & 15) == 0 && (g.lddy * es) % 16 == 0 && g.N % 8 == 0 && g.lddy <= (1 << 22);
  hipError_t e;
  if (g.dt == DT_F32) e = v ? run<float, true>(it, yg, s) : run<float, false>(it, yg, s);
  else e = v ? run<bf16, true>(it, yg, s) : run<bf16, false>(it, yg, s);
  if (e != hipSuccess || it.slabs == 1) return e;
  const long long all = (long long)g.N * g.K + (g.db ? g.N : 0), blocks = (all + 255) / 256;
  wgrad_sum_k<<<(unsigned)(blocks < 4096 ? blocks : 4096), 256, 0, s>>>(it);
  return hipGetLastError();
}

}  // namespace sl
