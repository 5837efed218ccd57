// Weight gradient out of an 8-bit activation checkpoint (gfx950): dW[n][k] = sum_m dy[m][n] x8[m][k], db[n] = sum_m dy[m][n].
//
// A code times its power of two is exactly a bfloat16, so the checkpoint is decoded on its way into LDS and the products are the
// matrix cores' bfloat16 ones with float32 sums; float32 gradients go in as three bfloat16 terms (split_f32.h), which are
// all of their bits.  The contraction runs over the rows of both operands: 64-row slices lie in LDS as they are in memory and the fragments,
// eight consecutive rows of a column per lane, are read with the transposing LDS reads.
// The rows are split into slabs: a work item is (slab, output tile), writes its partial tile once, and a second kernel adds the slabs
// in a fixed order.
#include "act8_internal.h"

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

// 16 codes times their power of two, as two pieces of eight bfloat16: exact
__device__ __forceinline__ void decode16(const u32x4& q, float s, bf16x8 (&o)[2]) {
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    float v[4], w[4];
    a8_value4(q[2 * h], s, v);
    a8_value4(q[2 * h + 1], s, w);
#pragma unroll
    for (int e = 0; e < 4; ++e) { o[h][e] = (bf16)v[e]; o[h][4 + e] = (bf16)w[e]; }
  }
}

// eight values of dy in float32
struct Eight { float v[8]; };

// YG: the tile is 128 rows of dW by 128 YG columns.  V: dy's rows can be read in 16-byte pieces.
template <typename T, int YG, bool V>
__global__ void __launch_bounds__(NTH) wgrad_k(Item it) {
  constexpr int TERMS = sizeof(T) == 2 ? 1 : 3;
  constexpr int BY = 128 * YG, LDW = TERMS * BX + BY + 32, STAGE = BK * LDW;
  constexpr int YCHUNKS = BY / 16 * BK / NTH;
  constexpr int WBN = BY / (32 * WVN);   // 32-column products of a wavefront; two of 32 rows
  __shared__ __attribute__((aligned(16))) bf16 ring[2][STAGE];
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
  const long long lo = slab * it.per;
  const int span = lo >= g.M ? 0 : (int)(g.M - lo < it.per ? g.M - lo : it.per);
  const int steps = (span + BK - 1) / BK;
  const int k16 = (g.K + A8_GRAIN - 1) / A8_GRAIN * A8_GRAIN;

  const int xr = tid >> 4, xc = (tid & 15) * 8;            // dy: rows xr + 32 i
  const T* const xb = (const T*)g.dy + lo * g.lddy + x0 + xc;
  T rx[XCHUNKS][8];
  u32x4 ry[YCHUNKS];
  float rs[YCHUNKS];
  auto fetch = [&](int step) {
#pragma unroll
    for (int i = 0; i < XCHUNKS; ++i) {
      const int r = step * BK + xr + (NTH / 16) * i;
      const T* p = xb + (long long)r * g.lddy;
      if (V && r < span && x0 + xc + 8 <= g.N) {
        typedef T vec __attribute__((ext_vector_type(16 / sizeof(T))));
#pragma unroll
        for (int h = 0; h < (int)sizeof(T) / 2; ++h)
          *reinterpret_cast<vec*>(&rx[i][h * (16 / sizeof(T))]) = *reinterpret_cast<const vec*>(p + h * (16 / sizeof(T)));
      } else {
#pragma unroll
        for (int e = 0; e < 8; ++e) rx[i][e] = r < span && x0 + xc + e < g.N ? p[e] : (T)0.f;
      }
    }
#pragma unroll
    for (int j = 0; j < YCHUNKS; ++j) {
      const int c = tid + NTH * j, r = step * BK + c / (BY / 16), col = y0 + c % (BY / 16) * 16;
      const bool have = r < span && col < k16;
      const u32x4 z = {0, 0, 0, 0};
      ry[j] = have ? *reinterpret_cast<const u32x4*>(g.x.codes + (lo + r) * g.x.ldc + col) : z;
      rs[j] = have ? a8_scale(g.x.scales[(lo + r) * g.x.lds + (col >> 7)]) : 0.f;
    }
  };
  float cs[8];
#pragma unroll
  for (int e = 0; e < 8; ++e) cs[e] = 0.f;
  auto stash = [&](int st) {
    bf16* S = ring[st];
#pragma unroll
    for (int i = 0; i < XCHUNKS; ++i) {
      bf16* p = S + (xr + (NTH / 16) * i) * LDW + xc;
      float f[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) { f[e] = to_f(rx[i][e]); cs[e] += f[e]; }
#pragma unroll
      for (int t = 0; t < TERMS; ++t) {
        bf16x8 o;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          o[e] = (bf16)f[e];
          // (what rounds to an infinity, or is none, has no further terms)
          if constexpr (TERMS > 1) f[e] = a8_mag((float)o[e]) ? f[e] - (float)o[e] : 0.f;
        }
        *reinterpret_cast<bf16x8*>(p + t * BX) = o;
      }
    }
#pragma unroll
    for (int j = 0; j < YCHUNKS; ++j) {
      const int c = tid + NTH * j;
      bf16x8 o[2];
      decode16(ry[j], rs[j], o);
      bf16* p = S + c / (BY / 16) * LDW + TERMS * BX + c % (BY / 16) * 16;
      *reinterpret_cast<bf16x8*>(p) = o[0];
      *reinterpret_cast<bf16x8*>(p + 8) = o[1];
    }
  };

  f32x16 acc[2][WBN];
#pragma unroll
  for (int i = 0; i < 2; ++i)
#pragma unroll
    for (int j = 0; j < WBN; ++j)
#pragma unroll
      for (int r = 0; r < 16; ++r) acc[i][j][r] = 0.f;

  if (steps > 0) {
    fetch(0);
    stash(0);
  }
  __syncthreads();
  for (int s = 0; s < steps; ++s) {
    const bool more = s + 1 < steps;   // uniform
    if (more) fetch(s + 1);
    const bf16* S = ring[s & 1];
#pragma unroll
    for (int k = 0; k < BK; k += 16) {
      bf16x8 fy[WBN];
#pragma unroll
      for (int j = 0; j < WBN; ++j) fy[j] = frag_tr<LDW>(S, TERMS * BX + (wn * WBN + j) * 32, k, lane);
#pragma unroll
      for (int t = 0; t < TERMS; ++t)
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          const bf16x8 fx = frag_tr<LDW>(S, t * BX + (wm * 2 + i) * 32, k, lane);
#pragma unroll
          for (int j = 0; j < WBN; ++j) acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(fx, fy[j], acc[i][j], 0, 0, 0);
        }
    }
    if (more) stash((s + 1) & 1);
    __syncthreads();
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
  // bias gradient: the tiles of the first columns add the rows their threads loaded
  if (g.db && y0 == 0) {
    __syncthreads();
    float* red = reinterpret_cast<float*>(ring[0]);   // [32 threads][128 columns]
#pragma unroll
    for (int e = 0; e < 8; ++e) red[xr * BX + xc + e] = cs[e];
    __syncthreads();
    if (tid < BX && x0 + tid < g.N) {
      float v = 0.f;
      for (int r = 0; r < NTH / 16; ++r) v += red[r * BX + tid];
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

int tile_groups(int K) {   // 128-column groups of a tile: the fewest columns beyond K, then the widest
  int best = 1;
  long long waste = 1LL << 60;
  for (int yg = 1; yg <= 3; ++yg) {
    const long long cols = (long long)(K + 128 * yg - 1) / (128 * yg) * 128 * yg;
    if (cols <= waste) { waste = cols; best = yg; }
  }
  return best;
}

void plan(long long M, int N, int K, int yg, Item* it) {
  it->TX = (N + BX - 1) / BX;
  it->TY = (K + 128 * yg - 1) / (128 * yg);
  const long long tiles = (long long)it->TX * it->TY, steps = (M + BK - 1) / BK;
  // slabs: the fewest rounds of 256 workgroups; a slab has eight steps at least, and costs its partial's way out and back
  double best = 1e300;
  it->slabs = 1;
  for (int s = 1; s <= MAX_SLABS && (s == 1 || steps / s >= 8); ++s) {
    const double rounds = (double)((tiles * s + 255) / 256);
    const double cost = rounds * (double)((steps + s - 1) / s + 4) + (s > 1 ? s * (double)N * K * 8e-6 / 2.0 : 0.0);
    if (cost < best) { best = cost; it->slabs = s; }
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
  plan(M, N, K, tile_groups(K), &a);
  plan(M, N, K, 1, &b);   // float32 gradients
  const size_t x = part_bytes(a, N, K), y = part_bytes(b, N, K);
  return ((x > y ? x : y) + 256 + 255) & ~(size_t)255;
}

hipError_t launch_act8_wgrad(const A8Wgrad& g, hipStream_t s) {
  const int yg = g.dt == DT_F32 ? 1 : tile_groups(g.K);
  Item it{};
  it.g = g;
  plan(g.M, g.N, g.K, yg, &it);
  it.part = g.work;
  it.cpart = g.work + (((size_t)it.slabs * g.N * g.K * 4 + 255) & ~(size_t)255) / 4;
  const size_t es = elem_size(g.dt);
  const bool v = ((uintptr_t)g.dy & 15) == 0 && (g.lddy * es) % 16 == 0;
  hipError_t e;
  if (g.dt == DT_F32) e = v ? run<float, true>(it, yg, s) : run<float, false>(it, yg, s);
  else e = v ? run<bf16, true>(it, yg, s) : run<bf16, false>(it, yg, s);
  if (e != hipSuccess || it.slabs == 1) return e;
  const long long all = (long long)g.N * g.K + (g.db ? g.N : 0), blocks = (all + 255) / 256;
  wgrad_sum_k<<<(unsigned)(blocks < 4096 ? blocks : 4096), 256, 0, s>>>(it);
  return hipGetLastError();
}

}  // namespace sl
