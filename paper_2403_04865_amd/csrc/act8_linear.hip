// Linear layers on 8-bit activations and weights (gfx950): y = act(x8 w8^T + bias) + residual.
//
// Both operands are e4m3 codes [rows][k] with a power of two per row and 128 columns, which is what the matrix cores' scaled
// instruction takes: one 16 x 16 x 128 product per block, the power of each operand row in a register beside it (the instruction has a
// power for every 32 columns; a lane holds 32 columns of one row, so the block's byte is given to all four).  Nothing is
// decoded, and the 128s are added in the float32 accumulator.
//   * Inside an instruction eight neighbouring products are aligned to the largest of them and cut off 13 bits below it; the sums of
//     the eights keep 24 bits (measured with single pairs of operands).  Results were 1.6e-5 (normal operands) to 8e-5 (operands over
//     four decades) off, against 2e-3 for the rounding to bfloat16 that follows.  Where y is float32 the codes are decoded into
//     bfloat16 instead (exact from 2^-133 on: code times a power of two) and multiplied by 16 x 16 x 32 instructions, at half the rate, whose
//     sums are as exact as float32 ones (1e-7; on positive operands 1e-8 low to 3e-8 high).  Decoding twice per tile takes most of that path's time:
//     7289 x 384 -> 1152 37 us, 403456 x 384 -> 1536 1600, 8192 x 4096 -> 4096 544 (0.5 PFLOP/s).
//   * The first operand is w: a lane then holds four consecutive output columns of one row.  Rows of w are dealt to the 16 rows of
//     two neighbouring products so that the two give a lane eight consecutive columns: 16-byte stores, 64 bytes in a row.
#include "act8_internal.h"
#include "lds_dma.h"

namespace sl {

namespace {

typedef int i32x8 __attribute__((ext_vector_type(8)));
typedef int i32x4 __attribute__((ext_vector_type(4)));

typedef i32x8 Codes;   // 32 codes of a lane
__device__ __forceinline__ Codes codes_of(const uint8_t* lo, const uint8_t* hi) {   // two pieces of 16
  return __builtin_shufflevector(*reinterpret_cast<const i32x4*>(lo), *reinterpret_cast<const i32x4*>(hi), 0, 1, 2, 3, 4, 5, 6, 7);
}
__device__ __forceinline__ f32x4 mfma_f8(const Codes& a, int sa, const Codes& b, int sb, f32x4 c) {
  return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(a, b, c, 0, 0, 0, sa, 0, sb);
}
// the same with byte `at` (known when compiled, behind the unrolling) of both scale registers
__device__ __forceinline__ f32x4 mfma_f8_at(int at, const Codes& a, int sa, const Codes& b, int sb, f32x4 c) {
  switch (at) {
    case 0: return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(a, b, c, 0, 0, 0, sa, 0, sb);
    case 1: return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(a, b, c, 0, 0, 1, sa, 1, sb);
    case 2: return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(a, b, c, 0, 0, 2, sa, 2, sb);
    default: return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(a, b, c, 0, 0, 3, sa, 3, sb);
  }
}
// eight codes -> bfloat16 values times s; exact
__device__ __forceinline__ bf16x8 decode8(int q0, int q1, float s) {
  float v[4], w[4];
  a8_value4((unsigned)q0, s, v);
  a8_value4((unsigned)q1, s, w);
  bf16x8 r;
#pragma unroll
  for (int e = 0; e < 4; ++e) { r[e] = (bf16)v[e]; r[4 + e] = (bf16)w[e]; }
  return r;
}
// a lane's 32 codes as the operands of four products of 32 columns
struct Terms { bf16x8 t[4]; };
__device__ __forceinline__ Terms decode(const Codes& c, float s) {
  return Terms{{decode8(c[0], c[1], s), decode8(c[2], c[3], s), decode8(c[4], c[5], s), decode8(c[6], c[7], s)}};
}
__device__ __forceinline__ f32x4 mfma_b16(const Terms& a, const Terms& b, f32x4 c) {
#pragma unroll
  for (int j = 0; j < 4; ++j) c = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a.t[j], b.t[j], c, 0, 0, 0);
  return c;
}

__device__ __forceinline__ Codes load_codes(const uint8_t* p, int k, int k16) {   // zeros from k16 on
  const i32x4 z = {0, 0, 0, 0};
  const i32x4 lo = k < k16 ? *reinterpret_cast<const i32x4*>(p + k) : z, hi = k + 16 < k16 ? *reinterpret_cast<const i32x4*>(p + k + 16) : z;
  return __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
}

// ---- few rows -------------------------------------------------------------------------------------------------------
// A workgroup takes 16 output columns and 16 MT rows; its wavefronts share out the blocks of k and their partial products are added in
// LDS, in a fixed order.  PACK: x comes as it is and every workgroup makes the codes it multiplies for itself, the first one
// leaves them as the checkpoint: one launch instead of two (1 x 4096 -> 4096: 12.2 us a call with a launch for the packing, 8.5 so).
constexpr int SW = 8;   // wavefronts

// 32 values of row `x` from column k on (zeros from K on)
template <typename T> struct Raw {
  static constexpr int E = 16 / sizeof(T);
  typedef T vec16 __attribute__((ext_vector_type(E)));
  vec16 q[32 / E];
  __device__ __forceinline__ void load(const T* x, int k, int K, bool vec) {
    if (vec && K % A8_BLOCK == 0 && k < K) {   // (k < K in all lanes of a block)
#pragma unroll
      for (int h = 0; h < 32 / E; ++h) q[h] = *reinterpret_cast<const vec16*>(x + k + h * E);
    } else if (vec && K % E == 0) {
#pragma unroll
      for (int h = 0; h < 32 / E; ++h) {
        q[h] = vec16{};
        if (k + h * E < K) q[h] = *reinterpret_cast<const vec16*>(x + k + h * E);
      }
    } else {
#pragma unroll
      for (int h = 0; h < 32 / E; ++h)
#pragma unroll
        for (int e = 0; e < E; ++e) q[h][e] = k + h * E + e < K ? x[k + h * E + e] : (T)0.f;
    }
  }
};
// ... -> codes and the scale byte of their block, which the four lanes that differ in bits 4 and 5 hold together
template <typename T>
__device__ __forceinline__ Codes pack32(const Raw<T>& w, int* byte) {
  float v[32];
#pragma unroll
  for (int e = 0; e < 32; ++e) v[e] = to_f(w.q[e / Raw<T>::E][e % Raw<T>::E]);
  auto most = [](float m) { m = fmaxf(m, __shfl_xor(m, 16, 64)); return fmaxf(m, __shfl_xor(m, 32, 64)); };
  float m = 0.f;
#pragma unroll
  for (int e = 0; e < 32; ++e) m = fmaxf(m, fabsf(v[e]));   // (drops NaN)
  m = most(m);
  if (m == __builtin_huge_valf()) {   // alike in the four lanes; the other lanes of the wavefront take no part in their exchange
    m = 0.f;
#pragma unroll
    for (int e = 0; e < 32; ++e) m = fmaxf(m, __uint_as_float(a8_mag(v[e])));
    m = most(m);
  }
  const unsigned b = a8_scale_byte(__float_as_uint(m));
  const float s = a8_inverse(b);
  Codes c;
#pragma unroll
  for (int j = 0; j < 8; ++j) c[j] = (int)a8_code4(v[4 * j] * s, v[4 * j + 1] * s, v[4 * j + 2] * s, v[4 * j + 3] * s);
  *byte = (int)b;
  return c;
}

// what pack32 gave, as the checkpoint
__device__ __forceinline__ void leave32(const Codes& c, int byte, uint8_t* row, uint8_t* scale, int k, int k16) {
  if (k < k16) *reinterpret_cast<i32x4*>(row + k) = __builtin_shufflevector(c, c, 0, 1, 2, 3);
  if (k + 16 < k16) *reinterpret_cast<i32x4*>(row + k + 16) = __builtin_shufflevector(c, c, 4, 5, 6, 7);
  if ((k & (A8_BLOCK - 1)) == 0) *scale = (uint8_t)byte;
}

template <int MT, int ACT, typename T, bool PACK>
__global__ void __launch_bounds__(64 * SW) linear_few_k(A8Linear g, bool vec) {
  constexpr bool F8 = sizeof(T) == 2;
  constexpr int U = MT == 1 ? 4 : MT == 2 ? 2 : 1;   // blocks whose loads are in flight together
  __shared__ float red[SW][MT * 256];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, r = lane & 15, kg = (lane >> 4) * 32;
  const int n0 = blockIdx.x * 16;
  const long long m0 = (long long)blockIdx.y * 16 * MT;
  const int nb = (g.K + A8_BLOCK - 1) / A8_BLOCK, k16 = (g.K + A8_GRAIN - 1) / A8_GRAIN * A8_GRAIN;
  const int n = n0 + r < g.N ? n0 + r : g.N - 1;
  const uint8_t *wp = g.w.codes + n * g.w.ldc, *ws = g.w.scales + n * g.w.lds;
  const uint8_t *xp[MT], *xs[MT];
  long long mr[MT];
#pragma unroll
  for (int i = 0; i < MT; ++i) {
    mr[i] = m0 + 16 * i + r < g.M ? m0 + 16 * i + r : g.M - 1;
    xp[i] = g.x.codes + mr[i] * g.x.ldc; xs[i] = g.x.scales + mr[i] * g.x.lds;
  }
  f32x4 acc[MT];
#pragma unroll
  for (int i = 0; i < MT; ++i) acc[i] = f32x4{0.f, 0.f, 0.f, 0.f};
  for (int b0 = wave; b0 < nb; b0 += SW * U) {
    Codes cw[U], cx[U][MT];
    int sw[U], sx[U][MT];
#pragma unroll
    for (int u = 0; u < U; ++u) {   // (a block that does not exist is all zeros, under any scale)
      const int b = b0 + u * SW, k = b * A8_BLOCK + kg, at = b < nb ? b : nb - 1;
      cw[u] = load_codes(wp, k, k16);
      sw[u] = ws[at];
      if constexpr (!PACK) {
#pragma unroll
        for (int i = 0; i < MT; ++i) { cx[u][i] = load_codes(xp[i], k, k16); sx[u][i] = xs[i][at]; }
      }
    }
    if constexpr (PACK) {
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const int b = b0 + u * SW, k = b * A8_BLOCK + kg;
#pragma unroll
        for (int i = 0; i < MT; ++i) {
          if (b >= nb) { cx[u][i] = Codes{}; sx[u][i] = 127; continue; }   // uniform
          Raw<T> raw;
          raw.load((const T*)g.xin + mr[i] * g.ldxin, k, g.K, vec);
          cx[u][i] = pack32(raw, &sx[u][i]);
          if (blockIdx.x == 0 && m0 + 16 * i + r < g.M)   // this lane's codes are the checkpoint's
            leave32(cx[u][i], sx[u][i], const_cast<uint8_t*>(xp[i]), const_cast<uint8_t*>(xs[i]) + b, k, k16);
        }
      }
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
      Terms tw;
      if constexpr (!F8) tw = decode(cw[u], a8_scale(sw[u]));
#pragma unroll
      for (int i = 0; i < MT; ++i) {
        if constexpr (F8) acc[i] = mfma_f8(cw[u], sw[u], cx[u][i], sx[u][i], acc[i]);
        else acc[i] = mfma_b16(tw, decode(cx[u][i], a8_scale(sx[u][i])), acc[i]);
      }
    }
  }
  // lane: columns 4 (lane / 16) .. + 3 of row lane % 16
#pragma unroll
  for (int i = 0; i < MT; ++i)
    *reinterpret_cast<f32x4*>(&red[wave][i * 256 + r * 16 + (lane >> 4) * 4]) = acc[i];
  __syncthreads();
  for (int o = threadIdx.x; o < MT * 256; o += 64 * SW) {
    const long long m = m0 + (o >> 4);
    const int c = n0 + (o & 15);
    if (m >= g.M || c >= g.N) continue;
    float v = 0.f;
#pragma unroll
    for (int w = 0; w < SW; ++w) v += red[w][o];
    if (g.bias) v += g.bias[c];
    v = act_f<ACT>(v);
    if (g.resid) v += to_f(((const T*)g.resid)[m * g.ldr + c]);
    ((T*)g.y)[m * g.ldy + c] = from_f<T>(v);
  }
}

template <int ACT, typename T>
hipError_t few(const A8Linear& g, hipStream_t s) {
  const int mt = g.M <= 16 ? 1 : g.M <= 32 ? 2 : 4;
  const bool vec = ((uintptr_t)g.xin & 15) == 0 && g.ldxin * sizeof(T) % 16 == 0;
  A8Linear p = g;
  // grid.y is limited to 65535: the rows go in pieces
  const long long most = 16LL * mt * 65535;
  for (long long m = 0; m < g.M; m += most) {
    p.M = g.M - m < most ? g.M - m : most;
    p.x.codes = g.x.codes + m * g.x.ldc; p.x.scales = g.x.scales + m * g.x.lds;
    p.y = (T*)g.y + m * g.ldy;
    if (g.xin) p.xin = (const T*)g.xin + m * g.ldxin;
    if (g.resid) p.resid = (const T*)g.resid + m * g.ldr;
    const dim3 grid((g.N + 15) / 16, (unsigned)((p.M + 16 * mt - 1) / (16 * mt)));
    auto go = [&](auto pack) {
      constexpr bool PACK = decltype(pack)::value;
      if (mt == 1) linear_few_k<1, ACT, T, PACK><<<grid, 64 * SW, 0, s>>>(p, vec);
      else if (mt == 2) linear_few_k<2, ACT, T, PACK><<<grid, 64 * SW, 0, s>>>(p, vec);
      else linear_few_k<4, ACT, T, PACK><<<grid, 64 * SW, 0, s>>>(p, vec);
    };
    if (g.xin) go(std::true_type{});
    else go(std::false_type{});
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  return hipSuccess;
}

// ---- tiles ------------------------------------------------------------------------------------------------------------
// A workgroup takes BM rows of x by BN rows of w, a wavefront 16 FM of x by 64 of w; 128 columns per step, brought straight into LDS
// one step ahead, in two stages.  A row of a stage is eight 16-byte pieces; piece c lies in place c ^ (3 bits of the row), chosen so
// that eight neighbouring lanes of a fragment read find their pieces in eight different places (no bank conflicts).
constexpr int STEP = A8_BLOCK;
constexpr int CHUNK = 32, SROW = CHUNK + 4;   // blocks whose scales lie in LDS together; bytes between rows of them there

__device__ __forceinline__ int turn_x(int row) { return row & 7; }
// rows of w are dealt to fragments so that neighbouring lanes have rows 0 1 2 3, 8 9 10 11
__device__ __forceinline__ int turn_w(int row) { return (row & 3) | ((row >> 1) & 4); }

// A wavefront's 16 FM rows of 64 columns: bias, activation, residual and the way out.  A lane has row r of each 16 and columns
// 32 p + 8 kg .. + 7.  They go through a patch of LDS, 16 rows at a time, and leave in whole rows of 64 columns: written as the
// lanes have them, 64 bytes of a row at a time, every half cache line was fetched from memory first (403456 x 1536 -> 384: 561 us, 373
// so).  A residual comes the same way in.  Buffer instructions: what lies behind the last row or column is left out without a branch.
struct Store {
  void* y; long long ldy;            // the wavefront's first value
  const void* res; long long ldr;    // may be null
  int have, left;                    // rows and columns that exist from there on
  bool vec;                          // 16-byte pieces of y and the residual are aligned
  bool stream;                       // y is larger than what the caches would keep of it
};
// What is written past this many bytes of y has left the 256 MB of last-level cache before anybody reads it: stores with the
// streaming hint (403456 x 384 -> 1536: 422 -> 327 us; 200000 x 512: 111 -> 96; 134 MB of output: no difference)
constexpr long long STREAM_BYTES = 160 << 20;
template <typename T> constexpr int patch_row() { return 64 * (int)sizeof(T) + 16; }   // bytes between rows of a patch (no bank conflicts)

template <typename T>
__device__ __forceinline__ __amdgpu_buffer_rsrc_t out_buffer(const void* p, long long ld, const Store& o) {
  return dma_buffer(p, o.have > 0 && o.left > 0 ? ((o.have - 1) * ld + (o.left < 64 ? o.left : 64)) * (long long)sizeof(T) : 0);
}

template <int FM, int ACT, typename T>
__device__ __forceinline__ void store_tile(const f32x4 (&acc)[4][FM], const f32x4 (&bias)[2][2], uint8_t* patch, int lane, const Store& o) {
  constexpr int E = 16 / sizeof(T), PROW = patch_row<T>(), LR = 64 / E, RP = 64 / LR, NH = 16 / RP;   // lanes of a row, rows at a time
  typedef T vec16 __attribute__((ext_vector_type(E)));
  const int r = lane & 15, kg = lane >> 4, orow = lane / LR, oc = lane % LR * E;
  const bool fast = o.vec && (o.left >= 64 || o.left % E == 0);   // uniform
  const __amdgpu_buffer_rsrc_t yb = out_buffer<T>(o.y, o.ldy, o), rb = out_buffer<T>(o.res, o.res ? o.ldr : 0, o);
  const int yo = oc < o.left ? (orow * (int)o.ldy + oc) * (int)sizeof(T) : DMA_ABSENT, ro = oc < o.left ? (orow * (int)o.ldr + oc) * (int)sizeof(T) : DMA_ABSENT;
  uint8_t* const out = patch + orow * PROW + oc * sizeof(T);
  u32x4 q[NH];
  auto fetch = [&](int i) {
#pragma unroll
    for (int h = 0; h < NH; ++h) q[h] = __builtin_amdgcn_raw_buffer_load_b128(rb, ro, (i * 16 + h * RP) * (int)o.ldr * (int)sizeof(T), 0);
  };
  if (o.res && fast) fetch(0);
#pragma unroll
  for (int i = 0; i < FM; ++i) {
    if (o.res) {   // uniform
      if (fast) {
#pragma unroll
        for (int h = 0; h < NH; ++h) *reinterpret_cast<u32x4*>(out + h * RP * PROW) = q[h];
        if (i + 1 < FM) fetch(i + 1);
      } else {
#pragma unroll 1
        for (int k = lane; k < 16 * 64; k += 64) {
          const int row = k >> 6, c = k & 63;
          if (i * 16 + row < o.have && c < o.left)
            *reinterpret_cast<T*>(patch + row * PROW + c * sizeof(T)) = ((const T*)o.res)[(i * 16 + row) * o.ldr + c];
        }
      }
      __builtin_amdgcn_wave_barrier();   // the patch is this wavefront's own; its LDS accesses are in order
    }
#pragma unroll
    for (int p = 0; p < 2; ++p)
#pragma unroll
      for (int h = 0; h < 8 / E; ++h) {
        vec16* at = reinterpret_cast<vec16*>(patch + r * PROW + (32 * p + 8 * kg + h * E) * sizeof(T));
        float v[E];
#pragma unroll
        for (int e = 0; e < E; ++e) {
          const int k = h * E + e;
          v[e] = act_f<ACT>(acc[2 * p + (k >> 2)][i][k & 3] + bias[p][k >> 2][k & 3]);
        }
        if (o.res) {
          const vec16 z = *at;
#pragma unroll
          for (int e = 0; e < E; ++e) v[e] += to_f(z[e]);
        }
        vec16 w;
#pragma unroll
        for (int e = 0; e < E; ++e) w[e] = from_f<T>(v[e]);
        *at = w;
      }
    __builtin_amdgcn_wave_barrier();
    if (fast) {
#pragma unroll
      for (int h = 0; h < NH; ++h) {
        const u32x4 w = *reinterpret_cast<const u32x4*>(out + h * RP * PROW);
        const int at = (i * 16 + h * RP) * (int)o.ldy * (int)sizeof(T);
        if (o.stream) store16<2>(w, yb, yo + at);
        else store16(w, yb, yo + at);
      }
    } else {
#pragma unroll 1
      for (int k = lane; k < 16 * 64; k += 64) {
        const int row = k >> 6, c = k & 63;
        if (i * 16 + row < o.have && c < o.left)
          ((T*)o.y)[(i * 16 + row) * o.ldy + c] = *reinterpret_cast<const T*>(patch + row * PROW + c * sizeof(T));
      }
    }
    __builtin_amdgcn_wave_barrier();
  }
}

template <int BM, int BN, int FM, int ACT, typename T>
__global__ void __launch_bounds__(64 * (BM / (16 * FM)) * (BN / 64)) linear_tile_k(A8Linear g, int TM, int TN, bool vec, bool stream) {
  constexpr bool F8 = sizeof(T) == 2;
  constexpr int WM = BM / (16 * FM), NW = WM * (BN / 64);
  constexpr int XI = BM / 8 / NW, WI = BN / 8 / NW;   // kilobytes that a wavefront loads per step
  static_assert(XI * 8 * NW == BM && WI * 8 * NW == BN, "loads are dealt evenly");
  __shared__ __attribute__((aligned(16))) uint8_t ring0[(BM + BN) * STEP], ring1[(BM + BN) * STEP], sc[(BM + BN) * SROW];
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int wm = wave % WM, wn = wave / WM, r = lane & 15, kg = lane >> 4;
  // consecutive tiles of the same rows of x run on one XCD and share them in its L2
  const int j = blockIdx.x >> 3, tm = (int)(blockIdx.x & 7) + 8 * (j / TN), tn = j % TN;
  if (tm >= TM) return;
  const long long m0 = (long long)tm * BM;
  const int n0 = tn * BN;
  const int rows = g.M - m0 < BM ? (int)(g.M - m0) : BM, cols = g.N - n0 < BN ? g.N - n0 : BN;
  const int k16 = (g.K + A8_GRAIN - 1) / A8_GRAIN * A8_GRAIN, steps = (g.K + STEP - 1) / STEP;
  const int ldx = (int)g.x.ldc, ldw = (int)g.w.ldc;
  const __amdgpu_buffer_rsrc_t xb = dma_buffer(g.x.codes + m0 * g.x.ldc, (long long)(rows - 1) * ldx + k16);
  const __amdgpu_buffer_rsrc_t wb = dma_buffer(g.w.codes + n0 * g.w.ldc, (long long)(cols - 1) * ldw + k16);

  // load i of this wavefront brings rows 8 (wave XI + i) .. + 7 of x: lane's row 8 (..) + lane / 8, place lane % 8
  int xo[XI], wo[WI], wc[WI];
  const int xc = 16 * ((lane & 7) ^ (lane >> 3));
#pragma unroll
  for (int i = 0; i < XI; ++i) xo[i] = (8 * (wave * XI + i) + (lane >> 3)) * ldx + xc;
#pragma unroll
  for (int i = 0; i < WI; ++i) {
    const int row = 8 * (wave * WI + i) + (lane >> 3);
    wc[i] = 16 * ((lane & 7) ^ turn_w(row));
    wo[i] = row * ldw + wc[i];
  }
  auto fetch = [&](uint8_t* st, int k0) {
#pragma unroll
    for (int i = 0; i < XI; ++i)
      dma16(xb, st + (wave * XI + i) * 1024, k0 + xc < k16 ? xo[i] : DMA_ABSENT, k0);
#pragma unroll
    for (int i = 0; i < WI; ++i)
      dma16(wb, st + BM * STEP + (wave * WI + i) * 1024, k0 + wc[i] < k16 ? wo[i] : DMA_ABSENT, k0);
  };

  // Scale bytes of up to CHUNK blocks of every row of the tile go to LDS together (rows behind the last one: any byte, what they give is
  // not stored), and from there four blocks of a row per register.  As single bytes out of memory, a dozen loads of 16 rows per
  // wavefront and step, they cost as much as the products (8192 x 4096 x 4096: 253 us, 125 without them).
  auto stage_scales = [&](int b0) {
    const int nb = steps - b0 < CHUNK ? steps - b0 : CHUNK;
    auto rows_of = [&](const uint8_t* p, long long ld, int have, uint8_t* to) {
      if (((uintptr_t)p & 3) == 0 && (ld & 3) == 0) {   // uniform
        const int nd = (nb + 3) / 4;
        for (int i = tid; i < have * nd; i += 64 * NW) {
          const int row = i / nd, d = 4 * (i - row * nd);
          const uint8_t* from = p + row * ld + d;
          if (d + 4 <= nb) *reinterpret_cast<unsigned*>(to + row * SROW + d) = *reinterpret_cast<const unsigned*>(from);
          else
            for (int e = 0; d + e < nb; ++e) to[row * SROW + d + e] = from[e];
        }
      } else {
        for (int i = tid; i < have * nb; i += 64 * NW) {
          const int row = i / nb, d = i - row * nb;
          to[row * SROW + d] = p[row * ld + d];
        }
      }
    };
    rows_of(g.x.scales + m0 * g.x.lds + b0, g.x.lds, rows, sc);
    rows_of(g.w.scales + (long long)n0 * g.w.lds + b0, g.w.lds, cols, sc + BM * SROW);
  };
  int sx[FM], sw[4];
  auto scales = [&](int b) {   // b: block within the chunk
    if ((b & 3) == 0) {
#pragma unroll
      for (int i = 0; i < FM; ++i) sx[i] = *reinterpret_cast<const int*>(sc + ((wm * FM + i) * 16 + r) * SROW + b);
#pragma unroll
      for (int f = 0; f < 4; ++f)
        sw[f] = *reinterpret_cast<const int*>(sc + (BM + wn * 64 + (f >> 1) * 32 + 8 * (r >> 2) + 4 * (f & 1) + (r & 3)) * SROW + b);
    } else {
#pragma unroll
      for (int i = 0; i < FM; ++i) sx[i] = (int)((unsigned)sx[i] >> 8);
#pragma unroll
      for (int f = 0; f < 4; ++f) sw[f] = (int)((unsigned)sw[f] >> 8);
    }
  };

  f32x4 acc[4][FM];
#pragma unroll
  for (int f = 0; f < 4; ++f)
#pragma unroll
    for (int i = 0; i < FM; ++i) acc[f][i] = f32x4{0.f, 0.f, 0.f, 0.f};

  auto take = [&](const uint8_t* st, int row, int turn) {
    const uint8_t* p = st + row * STEP;
    return codes_of(p + 16 * ((2 * kg) ^ turn), p + 16 * ((2 * kg + 1) ^ turn));
  };
  auto multiply = [&](const uint8_t* st) {
    Codes cw[4];
    Terms tw[F8 ? 1 : 4];
#pragma unroll
    for (int f = 0; f < 4; ++f) {
      const int row = wn * 64 + (f >> 1) * 32 + 8 * (r >> 2) + 4 * (f & 1) + (r & 3);
      cw[f] = take(st + BM * STEP, row, turn_w(row));
      if constexpr (!F8) tw[f] = decode(cw[f], a8_scale(sw[f] & 0xff));
    }
#pragma unroll
    for (int i = 0; i < FM; ++i) {
      const int row = (wm * FM + i) * 16 + r;
      const Codes cx = take(st, row, turn_x(row));
      if constexpr (F8) {
#pragma unroll
        for (int f = 0; f < 4; ++f) acc[f][i] = mfma_f8(cw[f], sw[f], cx, sx[i], acc[f][i]);
      } else {
        const Terms tx = decode(cx, a8_scale(sx[i] & 0xff));
#pragma unroll
        for (int f = 0; f < 4; ++f) acc[f][i] = mfma_b16(tw[f], tx, acc[f][i]);
      }
    }
  };
  auto step = [&](int s, const uint8_t* st, uint8_t* other) {
    __syncthreads();   // this stage's loads are done, the other one's readers too
    if (s > 0 && (s & (CHUNK - 1)) == 0) { stage_scales(s); __syncthreads(); }
    if (s + 1 < steps) fetch(other, (s + 1) * STEP);
    scales(s & (CHUNK - 1));
    multiply(st);
  };
  fetch(ring0, 0);
  stage_scales(0);
  for (int s = 0; s < steps; s += 2) {
    step(s, ring0, ring1);
    if (s + 1 < steps) step(s + 1, ring1, ring0);
  }

  __syncthreads();   // every wavefront has left the stages
  const int nw = n0 + wn * 64, nl = nw + 8 * kg, row0 = wm * FM * 16;
  f32x4 bias[2][2];
#pragma unroll
  for (int p = 0; p < 2; ++p)
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const int n = nl + 32 * p + e;
      bias[p][e >> 2][e & 3] = g.bias ? g.bias[n < g.N ? n : g.N - 1] : 0.f;
    }
  const Store o{(T*)g.y + (m0 + row0) * g.ldy + nw, g.ldy, g.resid ? (const T*)g.resid + (m0 + row0) * g.ldr + nw : nullptr, g.ldr,
                rows - row0, g.N - nw, vec, stream};
  store_tile<FM, ACT, T>(acc, bias, ring0 + wave * 16 * patch_row<T>(), lane, o);
}

template <int BM, int BN, int FM, int ACT, typename T>
hipError_t tiles(const A8Linear& g, hipStream_t s) {
  const int TM = (int)((g.M + BM - 1) / BM), TN = (g.N + BN - 1) / BN;
  auto ok = [&](const void* p, long long ld) { return !p || (((uintptr_t)p & 15) == 0 && ld * sizeof(T) % 16 == 0); };
  const long long grid = (long long)(TM + 7) / 8 * 8 * TN;
  linear_tile_k<BM, BN, FM, ACT, T><<<(unsigned)grid, 64 * (BM / (16 * FM)) * (BN / 64), 0, s>>>(
      g, TM, TN, ok(g.y, g.ldy) && ok(g.resid, g.ldr), g.M * g.N * (long long)sizeof(T) >= STREAM_BYTES);
  return hipGetLastError();
}

// ---- many rows, short contraction ------------------------------------------------------------------------------------
// With K <= 384 a wavefront holds all of its rows of x, 16 FM of them, in registers (KB blocks of 128), and w streams past in stages of
// 64 rows, one stage ahead, shared by the workgroup's wavefronts.  Next to a tile of the kernel above, which starts, loads three steps
// and stores: x is read once, nothing drains between tiles, and the epilogue of one wavefront runs under the products of the others
// (403456 x 384 -> 1536 without an activation, plain stores on all sides: 422 us, 487 by tiles of 256, 637 by tiles of 128; from K = 512 on
// the tiles of 256 were the faster ones).  With streaming stores 327 us, 4.3 TB/s; with GELU 500 to 590: its 24 vector operations a value are
// 370 us of the vector units' time.
constexpr int RN = 64, RCOLS = 1024;   // rows of w per stage; most columns of y of a workgroup

constexpr int RWAVES = 4;              // two such workgroups per compute unit
template <int KB> constexpr int rows_fm() { return KB <= 2 ? 4 : 3; }   // what fits 256 registers

template <int KB, int ACT, bool PACK>
__global__ void __launch_bounds__(64 * RWAVES, 2) linear_rows_k(A8Linear g, int TM, int TN, int ncols, bool vec, bool stream, bool xvec) {
  constexpr int FM = rows_fm<KB>(), NW = RWAVES, STAGE = RN * KB * STEP, LOADS = RN / 8 * KB / NW;
  static_assert(LOADS * NW * 8 == RN * KB, "loads are dealt evenly");
  __shared__ __attribute__((aligned(16))) uint8_t ring0[STAGE], ring1[STAGE], wsc[RCOLS * 4], patch[NW][16 * patch_row<bf16>()];
  __shared__ __attribute__((aligned(16))) float bia[RCOLS];
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), r = lane & 15, kg = lane >> 4;
  const int j = blockIdx.x >> 3, tm = (int)(blockIdx.x & 7) + 8 * (j / TN), tn = j % TN;   // column pieces of the same rows on one XCD
  if (tm >= TM) return;
  const long long m0 = (long long)tm * (16 * FM * NW) + wave * (16 * FM);
  const int n0 = tn * ncols, cols = g.N - n0 < ncols ? g.N - n0 : ncols, stages = (cols + RN - 1) / RN;
  const int k16 = (g.K + A8_GRAIN - 1) / A8_GRAIN * A8_GRAIN;
  const int ldw = (int)g.w.ldc;

  int wo[LOADS], wk[LOADS];   // load i: eight rows of one block; offset in memory, column
#pragma unroll
  for (int i = 0; i < LOADS; ++i) {
    const int q = wave * LOADS + i, b = q >> 3, row = 8 * (q & 7) + (lane >> 3);
    wk[i] = b * STEP + 16 * ((lane & 7) ^ turn_w(row));
    wo[i] = row * ldw + wk[i];
  }
  auto fetch = [&](uint8_t* st, int s) {
    const int n = n0 + s * RN, left = cols - s * RN < RN ? cols - s * RN : RN;
    const __amdgpu_buffer_rsrc_t wb = dma_buffer(g.w.codes + (long long)n * g.w.ldc, (long long)(left - 1) * ldw + k16);
#pragma unroll
    for (int i = 0; i < LOADS; ++i) dma16(wb, st + (wave * LOADS + i) * 1024, wk[i] < k16 ? wo[i] : DMA_ABSENT, 0);
  };
  fetch(ring0, 0);
  for (int c = tid; c < cols; c += 64 * NW) {
    const uint8_t* p = g.w.scales + (long long)(n0 + c) * g.w.lds;
#pragma unroll
    for (int b = 0; b < KB; ++b) wsc[c * 4 + b] = p[b];
    bia[c] = g.bias ? g.bias[n0 + c] : 0.f;
  }

  // this wavefront's rows (behind the last: the last one again, nothing of it is stored)
  Codes x[FM][KB];
  unsigned sx[FM];   // a byte per block
  auto row_of = [&](int i) { return m0 + 16 * i + r < g.M ? m0 + 16 * i + r : g.M - 1; };
  if constexpr (PACK) {
    Raw<bf16> raw[FM][KB];   // all of them on their way before the first is looked at
#pragma unroll
    for (int i = 0; i < FM; ++i)
#pragma unroll
      for (int b = 0; b < KB; ++b) raw[i][b].load((const bf16*)g.xin + row_of(i) * g.ldxin, b * A8_BLOCK + 32 * kg, g.K, xvec);
    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
    for (int i = 0; i < FM; ++i) {
      const bool leave = tn == 0 && m0 + 16 * i + r < g.M;
      uint8_t* const to = const_cast<uint8_t*>(g.x.codes) + row_of(i) * g.x.ldc;
      uint8_t* const scale = const_cast<uint8_t*>(g.x.scales) + row_of(i) * g.x.lds;
      sx[i] = 0;
#pragma unroll
      for (int b = 0; b < KB; ++b) {
        int byte;
        x[i][b] = pack32(raw[i][b], &byte);
        sx[i] |= (unsigned)byte << (8 * b);
        if (leave) leave32(x[i][b], byte, to, scale + b, b * A8_BLOCK + 32 * kg, k16);
      }
    }
  } else {
#pragma unroll
    for (int i = 0; i < FM; ++i) {
      const uint8_t *p = g.x.codes + row_of(i) * g.x.ldc, *q = g.x.scales + row_of(i) * g.x.lds;
#pragma unroll
      for (int b = 0; b < KB; ++b) x[i][b] = load_codes(p, b * A8_BLOCK + 32 * kg, k16);
      sx[i] = 0;
#pragma unroll
      for (int b = 0; b < KB; ++b) sx[i] |= (unsigned)q[b] << (8 * b);
    }
  }

  const int have = (int)(g.M - m0 < 16 * FM ? g.M - m0 : 16 * FM);   // may be negative
  // where a lane's two pieces of fragment 0 lie: row 8 (r / 4) + r % 4 (fragment f: 32 (f / 2) + 4 (f % 2) rows on, the same turn)
  const int wrow = 8 * (r >> 2) + (r & 3), wlo = wrow * STEP + 16 * ((2 * kg) ^ turn_w(wrow)), whi = wrow * STEP + 16 * ((2 * kg + 1) ^ turn_w(wrow));
  auto step = [&](int s, const uint8_t* st, uint8_t* other) {
    __syncthreads();   // this stage's loads are done, the other one's readers too
    if (s + 1 < stages) fetch(other, s + 1);
    f32x4 acc[4][FM];
    unsigned sw[4];
#pragma unroll
    for (int f = 0; f < 4; ++f) {
      const int row = (f >> 1) * 32 + 8 * (r >> 2) + 4 * (f & 1) + (r & 3);
      sw[f] = *reinterpret_cast<const unsigned*>(wsc + (s * RN + row) * 4);
#pragma unroll
      for (int i = 0; i < FM; ++i) acc[f][i] = f32x4{0.f, 0.f, 0.f, 0.f};
    }
    // Fragments of w two ahead of their products; the fences keep the compiler from fetching all of them first (it spilled).
    auto frag = [&](int q) {   // q: fragment q % 4 of block q / 4
      const uint8_t* p = st + (q >> 2) * RN * STEP + ((q >> 1) & 1) * 32 * STEP + (q & 1) * 4 * STEP;
      return codes_of(p + wlo, p + whi);
    };
    Codes cw[3];
    cw[0] = frag(0);
    cw[1] = frag(1);
#pragma unroll
    for (int q = 0; q < 4 * KB; ++q) {
      const int f = q & 3, b = q >> 2;
      if (q + 2 < 4 * KB) cw[(q + 2) % 3] = frag(q + 2);
#pragma unroll
      for (int i = 0; i < FM; ++i) acc[f][i] = mfma_f8_at(b, cw[q % 3], (int)sw[f], x[i][b], (int)sx[i], acc[f][i]);
      __builtin_amdgcn_sched_barrier(0);
    }
    // (keeps the products here: sunk into the branches of the epilogue, they left all their operands waiting in registers)
#pragma unroll
    for (int f = 0; f < 4; ++f)
#pragma unroll
      for (int i = 0; i < FM; ++i) asm volatile("" : "+v"(acc[f][i]));
    const int c0 = s * RN;
    f32x4 bi[2][2];
#pragma unroll
    for (int p = 0; p < 2; ++p)
#pragma unroll
      for (int h = 0; h < 2; ++h) bi[p][h] = *reinterpret_cast<const f32x4*>(bia + c0 + 32 * p + 8 * kg + 4 * h);
    const Store o{(bf16*)g.y + m0 * g.ldy + n0 + c0, g.ldy, g.resid ? (const bf16*)g.resid + m0 * g.ldr + n0 + c0 : nullptr, g.ldr,
                  have, cols - c0, vec, stream};
    store_tile<FM, ACT, bf16>(acc, bi, patch[wave], lane, o);
  };
  for (int s = 0; s < stages; s += 2) {
    step(s, ring0, ring1);
    if (s + 1 < stages) step(s + 1, ring1, ring0);
  }
}

template <int KB, int ACT>
hipError_t rows_kb(const A8Linear& g, hipStream_t s) {
  constexpr int BM = 16 * rows_fm<KB>() * RWAVES, SLOTS = 512;
  const long long TM = (g.M + BM - 1) / BM;
  // columns of a workgroup: eight rounds of the chip's workgroups where there is work for them, whole stages, at most RCOLS
  const int st = (g.N + RN - 1) / RN;
  long long tn = (8LL * SLOTS + TM - 1) / TM;
  if (tn > st) tn = st;
  const int least = (st + RCOLS / RN - 1) / (RCOLS / RN);
  if (tn < least || g.xin) tn = least;   // (x is packed again for every piece of columns)
  const int per = (int)((st + tn - 1) / tn), TN = (st + per - 1) / per;
  auto ok = [&](const void* p, long long ld) { return !p || (((uintptr_t)p & 15) == 0 && ld % 8 == 0); };
  const unsigned grid = (unsigned)((TM + 7) / 8 * 8 * TN);
  const bool vec = ok(g.y, g.ldy) && ok(g.resid, g.ldr), stream = g.M * g.N * 2 >= STREAM_BYTES;
  if (g.xin) linear_rows_k<KB, ACT, true><<<grid, 64 * RWAVES, 0, s>>>(g, (int)TM, TN, per * RN, vec, stream, ok(g.xin, g.ldxin));
  else linear_rows_k<KB, ACT, false><<<grid, 64 * RWAVES, 0, s>>>(g, (int)TM, TN, per * RN, vec, stream, false);
  return hipGetLastError();
}

template <int ACT>
hipError_t rows(const A8Linear& g, hipStream_t s) {
  if (g.K <= A8_BLOCK) return rows_kb<1, ACT>(g, s);
  if (g.K <= 2 * A8_BLOCK) return rows_kb<2, ACT>(g, s);
  return rows_kb<3, ACT>(g, s);
}

template <int ACT, typename T>
hipError_t run(const A8Linear& given, hipStream_t s) {
  A8Linear g = given;
  const long long t128 = ((g.M + 127) / 128) * ((g.N + 127) / 128);
  // 32-bit offsets within a tile's rows; the launch's threads within 2^32
  const bool near = g.x.ldc <= (1 << 22) && g.w.ldc <= (1 << 22) && g.ldy <= (1 << 21) && g.ldr <= (1 << 21) && t128 < (1 << 22);
  const bool fewer = !near || g.M <= 64 || t128 < 64;
  // Who packs x (two launches otherwise).  The few-rows kernel, every workgroup for itself, up to 16 rows; beyond, where its workgroups are there
  // at once, x comes in 16-byte pieces and a wavefront has one block of 128 bfloat16 columns, or two of up to 32 rows (with the packing before and
  // so: 64 x 384 -> 384 9.5 and 7.0 us, 64 x 1024 9.3 and 8.2, 64 x 1280 9.5 and 10.4, 32 x 2048 9.4 and 8.3, 17 x 4096 10.6 and 11.9; 400 x 384
  // -> 384 9.2 and 6.9, 1152 9.4 and 9.8; 256 x 1024 -> 1152
  // 10.6 and 13.2; 64 x 333 8.9 and 14; float32, 64 x 384 -> 384 8.8 and 7.0, 64 x 1024 8.8 and 12).  The rows kernel (bfloat16) where every compute unit has rows and no row is
  // packed twice: from 32768 rows on, up to 384 columns (40000 x 384 -> 64, 256, 384, 768: 21.6, 23.8, 33.7, 35.7 us with the packing before,
  // 14.3, 20.7, 24.4, 35.5 so; 120000: 47.8, 52, 74, 102 and 32, 44, 53, 75; 403456: 157, 169, 189, 260 and 116, 152, 180, 250; 16384 x 384 -> 256
  // 15.3 and 17.8; 403456 x 384 -> 1152 323 and 368).  Without packing it wants several stages of w per workgroup (16384 x 384 -> 384: 13.7 us,
  // 10.2 by tiles of 128; 7289 x 384 -> 1152: 13.1, 14.6 and by tiles of 256 12.6).
  const int nb = (g.K + A8_BLOCK - 1) / A8_BLOCK;
  const bool pieces = ((uintptr_t)g.xin & 15) == 0 && g.ldxin * sizeof(T) % 16 == 0 && g.K * sizeof(T) % 16 == 0;
  bool rows_k = false, packs = fewer && (g.M <= 16 || (pieces && nb * (int)sizeof(T) <= (g.M <= 32 ? 4 * SW : 2 * SW) &&
                                                       (g.N + 15LL) / 16 * ((g.M + 63) / 64) <= 256));
  if constexpr (sizeof(T) == 2) {
    const bool ok = !fewer && g.K <= 3 * A8_BLOCK;
    packs = packs || (ok && g.M >= (1 << 15) && g.N <= 384);
    rows_k = ok && ((g.xin && packs) || g.M * g.N >= (1LL << 25));
  }
  if (g.xin && !packs) {
    const slide_act8 o{const_cast<uint8_t*>(g.x.codes), g.x.ldc, const_cast<uint8_t*>(g.x.scales), g.x.lds, g.M, g.K};
    const hipError_t e = launch_act8_pack(g.xin, g.dt, g.ldxin, false, o, s);
    if (e != hipSuccess) return e;
    g.xin = nullptr;
  }
  if (fewer) return few<ACT, T>(g, s);
  if constexpr (sizeof(T) == 2) {
    if (rows_k) return rows<ACT>(g, s);
    // Tiles of 256 or of 128, by rounds of an XCD's workgroups: it takes every eighth row of tiles, 32 large or 64 small tiles at once.  A round of
    // the large ones takes 54 to 60 us with K = 4096, one of the small ones 42, the last, which is rarely full, ten less (x packed before, 128
    // and 256, rounds in brackets: 6000 x 1152 39.7 [1] and 55.0 us [1]; 7289 64.2 [2] and 55.9 [1]; 14000 78.0 [2] and 110 [2]; 20000 112 [3] and
    // 112 [2]; 28000 151 [4] and 165 [3]; 2304 x 4096 66.5 [2] and 56.8 [1]; 6000 125 [3] and 118 [2]; 33000 x 384 73.0 [2] and 108 [2]; 50000 102
    // [3] and 111 [2].  Shorter ones likewise: 7289 x 256 -> 1152 12.7 and 11.5; 14000 15.3 and 20.2; 28000 26.4 and 28.8; 403456 x 1536 -> 384
    // 368 [19] and 350 [13]; 600 x 512 -> 20000 25.5 [3] and 37.4 [3]).
    auto rounds = [&](int b, int at_once) { return (((g.M + b - 1) / b + 7) / 8 * ((g.N + b - 1) / b) + at_once - 1) / at_once; };
    if (54 * rounds(256, 32) <= 42 * rounds(128, 64) - 10) return tiles<256, 256, 8, ACT, T>(g, s);
  }
  return tiles<128, 128, 4, ACT, T>(g, s);
}

template <typename T>
hipError_t by_act(const A8Linear& g, hipStream_t s) {
  switch (g.act) {
    case SLIDE_ACT_RELU: return run<SLIDE_ACT_RELU, T>(g, s);
    case SLIDE_ACT_SILU: return run<SLIDE_ACT_SILU, T>(g, s);
    case SLIDE_ACT_GELU: return run<SLIDE_ACT_GELU, T>(g, s);
    default: return run<SLIDE_ACT_NONE, T>(g, s);
  }
}

}  // namespace

hipError_t launch_act8_linear(const A8Linear& g, hipStream_t s) {
  return g.dt == DT_F32 ? by_act<float>(g, s) : by_act<bf16>(g, s);
}

}  // namespace sl
