// Linear layers on 8-bit activations and weights (gfx950): y = act(x8 w8^T + bias) + residual.
//
// Both operands are e4m3 codes [rows][k] with a power of two per row and 128 columns, which is what the matrix cores' scaled
// instruction takes: one 16 x 16 x 128 product per block, the power of each operand row in a register beside it (the instruction has a
// power for every 32 columns; a lane holds 32 columns of one row, so the block's byte is given to all four).  Nothing is
// decoded, and the 128s are added in the float32 accumulator.
//   * Inside an instruction eight neighbouring products are aligned to the largest of them and cut off 13 bits below it; the sums of
//     the eights keep 24 bits (measured with single pairs of operands).  Results were 1.6e-5 (normal operands) to 8e-5 (operands over
//     four decades) off, against 2e-3 for the rounding to bfloat16 that follows.  Where y is float32 the codes are decoded into
//     bfloat16 instead (exact: code times a power of two) and multiplied by 16 x 16 x 32 instructions, at half the rate, whose
//     sums are as exact as float32 ones (1e-7).
//   * The first operand is w: a lane then holds four consecutive output columns of one row.  Rows of w are dealt to the 16 rows of
//     two neighbouring products so that the two give a lane eight consecutive columns: 16-byte stores, 64 bytes in a row.
#include "act8_internal.h"
#include "lds_dma.h"

namespace sl {

namespace {

typedef int i32x8 __attribute__((ext_vector_type(8)));
typedef int i32x4 __attribute__((ext_vector_type(4)));

// 32 codes of a lane
struct Codes { i32x4 lo, hi; };

__device__ __forceinline__ i32x8 whole(const Codes& c) {
  return __builtin_shufflevector(c.lo, c.hi, 0, 1, 2, 3, 4, 5, 6, 7);
}
__device__ __forceinline__ f32x4 mfma_f8(const Codes& a, int sa, const Codes& b, int sb, f32x4 c) {
  return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(whole(a), whole(b), c, 0, 0, 0, sa, 0, sb);
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
  return Terms{{decode8(c.lo[0], c.lo[1], s), decode8(c.lo[2], c.lo[3], s), decode8(c.hi[0], c.hi[1], s), decode8(c.hi[2], c.hi[3], s)}};
}
__device__ __forceinline__ f32x4 mfma_b16(const Terms& a, const Terms& b, f32x4 c) {
#pragma unroll
  for (int j = 0; j < 4; ++j) c = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a.t[j], b.t[j], c, 0, 0, 0);
  return c;
}

__device__ __forceinline__ Codes load_codes(const uint8_t* p, int k, int k16) {
  Codes c;
  const i32x4 z = {0, 0, 0, 0};
  c.lo = k < k16 ? *reinterpret_cast<const i32x4*>(p + k) : z;
  c.hi = k + 16 < k16 ? *reinterpret_cast<const i32x4*>(p + k + 16) : z;
  return c;
}

// ---- few rows -------------------------------------------------------------------------------------------------------
// A workgroup takes 16 output columns and 16 MT rows; its wavefronts share out the blocks of k and their partial products are added in
// LDS, in a fixed order.
constexpr int SW = 8;   // wavefronts

template <int MT, int ACT, typename T>
__global__ void __launch_bounds__(64 * SW) linear_few_k(A8Linear g) {
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
#pragma unroll
  for (int i = 0; i < MT; ++i) {
    const long long m = m0 + 16 * i + r < g.M ? m0 + 16 * i + r : g.M - 1;
    xp[i] = g.x.codes + m * g.x.ldc; xs[i] = g.x.scales + m * g.x.lds;
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
#pragma unroll
      for (int i = 0; i < MT; ++i) { cx[u][i] = load_codes(xp[i], k, k16); sx[u][i] = xs[i][at]; }
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
  A8Linear p = g;
  // grid.y is limited to 65535: the rows go in pieces
  const long long most = 16LL * mt * 65535;
  for (long long m = 0; m < g.M; m += most) {
    p.M = g.M - m < most ? g.M - m : most;
    p.x.codes = g.x.codes + m * g.x.ldc; p.x.scales = g.x.scales + m * g.x.lds;
    p.y = (T*)g.y + m * g.ldy;
    if (g.resid) p.resid = (const T*)g.resid + m * g.ldr;
    const dim3 grid((g.N + 15) / 16, (unsigned)((p.M + 16 * mt - 1) / (16 * mt)));
    if (mt == 1) linear_few_k<1, ACT, T><<<grid, 64 * SW, 0, s>>>(p);
    else if (mt == 2) linear_few_k<2, ACT, T><<<grid, 64 * SW, 0, s>>>(p);
    else linear_few_k<4, ACT, T><<<grid, 64 * SW, 0, s>>>(p);
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

__device__ __forceinline__ int turn_x(int row) { return row & 7; }
// rows of w are dealt to fragments so that neighbouring lanes have rows 0 1 2 3, 8 9 10 11
__device__ __forceinline__ int turn_w(int row) { return (row & 3) | ((row >> 1) & 4); }

template <int BM, int BN, int FM, int ACT, typename T>
__global__ void __launch_bounds__(64 * (BM / (16 * FM)) * (BN / 64)) linear_tile_k(A8Linear g, int TM, int TN, bool vec) {
  constexpr bool F8 = sizeof(T) == 2;
  constexpr int WM = BM / (16 * FM), NW = WM * (BN / 64);
  constexpr int XI = BM / 8 / NW, WI = BN / 8 / NW;   // kilobytes that a wavefront loads per step
  static_assert(XI * 8 * NW == BM && WI * 8 * NW == BN, "loads are dealt evenly");
  __shared__ __attribute__((aligned(16))) uint8_t ring0[(BM + BN) * STEP], ring1[(BM + BN) * STEP];
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

  // scale bytes of this lane's operand rows (rows behind the last are read as the last one's; what they give is not stored)
  const uint8_t *xs[FM], *ws[4];
#pragma unroll
  for (int i = 0; i < FM; ++i) {
    const int row = (wm * FM + i) * 16 + r;
    xs[i] = g.x.scales + (m0 + (row < rows ? row : rows - 1)) * g.x.lds;
  }
#pragma unroll
  for (int f = 0; f < 4; ++f) {
    const int row = wn * 64 + (f >> 1) * 32 + 8 * (r >> 2) + 4 * (f & 1) + (r & 3);
    ws[f] = g.w.scales + (long long)(n0 + (row < cols ? row : cols - 1)) * g.w.lds;
  }
  int sx[FM], sw[4], nx[FM], nw[4];
  auto scales = [&](int b) {
#pragma unroll
    for (int i = 0; i < FM; ++i) nx[i] = xs[i][b];
#pragma unroll
    for (int f = 0; f < 4; ++f) nw[f] = ws[f][b];
  };

  f32x4 acc[4][FM];
#pragma unroll
  for (int f = 0; f < 4; ++f)
#pragma unroll
    for (int i = 0; i < FM; ++i) acc[f][i] = f32x4{0.f, 0.f, 0.f, 0.f};

  auto take = [&](const uint8_t* st, int row, int turn) {
    Codes c;
    const uint8_t* p = st + row * STEP;
    c.lo = *reinterpret_cast<const i32x4*>(p + 16 * ((2 * kg) ^ turn));
    c.hi = *reinterpret_cast<const i32x4*>(p + 16 * ((2 * kg + 1) ^ turn));
    return c;
  };
  auto multiply = [&](const uint8_t* st) {
    Codes cw[4];
    Terms tw[F8 ? 1 : 4];
#pragma unroll
    for (int f = 0; f < 4; ++f) {
      const int row = wn * 64 + (f >> 1) * 32 + 8 * (r >> 2) + 4 * (f & 1) + (r & 3);
      cw[f] = take(st + BM * STEP, row, turn_w(row));
      if constexpr (!F8) tw[f] = decode(cw[f], a8_scale(sw[f]));
    }
#pragma unroll
    for (int i = 0; i < FM; ++i) {
      const int row = (wm * FM + i) * 16 + r;
      const Codes cx = take(st, row, turn_x(row));
      if constexpr (F8) {
#pragma unroll
        for (int f = 0; f < 4; ++f) acc[f][i] = mfma_f8(cw[f], sw[f], cx, sx[i], acc[f][i]);
      } else {
        const Terms tx = decode(cx, a8_scale(sx[i]));
#pragma unroll
        for (int f = 0; f < 4; ++f) acc[f][i] = mfma_b16(tw[f], tx, acc[f][i]);
      }
    }
  };
  auto step = [&](int s, const uint8_t* st, uint8_t* other) {
    __syncthreads();   // this stage's loads are done, the other one's readers too
#pragma unroll
    for (int i = 0; i < FM; ++i) sx[i] = nx[i];
#pragma unroll
    for (int f = 0; f < 4; ++f) sw[f] = nw[f];
    if (s + 1 < steps) { fetch(other, (s + 1) * STEP); scales(s + 1); }
    multiply(st);
  };
  fetch(ring0, 0);
  scales(0);
  for (int s = 0; s < steps; s += 2) {
    step(s, ring0, ring1);
    if (s + 1 < steps) step(s + 1, ring1, ring0);
  }

  // lane: row r of each 16, columns 32 p + 8 kg .. + 7 of the wavefront's 64
#pragma unroll
  for (int p = 0; p < 2; ++p) {
    const int n = n0 + wn * 64 + p * 32 + 8 * kg;
    float bias[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) bias[e] = g.bias && n + e < g.N ? g.bias[n + e] : 0.f;
    const bool whole8 = vec && n + 8 <= g.N;
#pragma unroll
    for (int i = 0; i < FM; ++i) {
      const int row = (wm * FM + i) * 16 + r;
      if (row >= rows) continue;
      T* y = (T*)g.y + (m0 + row) * g.ldy + n;
      const T* res = g.resid ? (const T*)g.resid + (m0 + row) * g.ldr + n : nullptr;
      float v[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) v[e] = act_f<ACT>(acc[2 * p + (e >> 2)][i][e & 3] + bias[e]);
      if (whole8) {
        typedef T vec8 __attribute__((ext_vector_type(16 / sizeof(T))));
        constexpr int E = 16 / sizeof(T);
#pragma unroll
        for (int h = 0; h < 8 / E; ++h) {
          vec8 o;
          if (res) {
            const vec8 q = *reinterpret_cast<const vec8*>(res + h * E);
#pragma unroll
            for (int e = 0; e < E; ++e) v[h * E + e] += to_f(q[e]);
          }
#pragma unroll
          for (int e = 0; e < E; ++e) o[e] = from_f<T>(v[h * E + e]);
          *reinterpret_cast<vec8*>(y + h * E) = o;
        }
      } else {
#pragma unroll
        for (int e = 0; e < 8; ++e)
          if (n + e < g.N) y[e] = from_f<T>(v[e] + (res ? to_f(res[e]) : 0.f));
      }
    }
  }
}

template <int BM, int BN, int FM, int ACT, typename T>
hipError_t tiles(const A8Linear& g, hipStream_t s) {
  const int TM = (int)((g.M + BM - 1) / BM), TN = (g.N + BN - 1) / BN;
  auto ok = [&](const void* p, long long ld) { return !p || (((uintptr_t)p & 15) == 0 && ld * sizeof(T) % 16 == 0); };
  const long long grid = (long long)(TM + 7) / 8 * 8 * TN;
  linear_tile_k<BM, BN, FM, ACT, T><<<(unsigned)grid, 64 * (BM / (16 * FM)) * (BN / 64), 0, s>>>(
      g, TM, TN, ok(g.y, g.ldy) && ok(g.resid, g.ldr));
  return hipGetLastError();
}

template <int ACT, typename T>
hipError_t run(const A8Linear& g, hipStream_t s) {
  const long long t128 = ((g.M + 127) / 128) * ((g.N + 127) / 128), t256 = ((g.M + 255) / 256) * ((g.N + 255) / 256);
  // 32-bit offsets within a tile's rows; the launch's threads within 2^32
  const bool near = g.x.ldc <= (1 << 22) && g.w.ldc <= (1 << 22) && t128 < (1 << 23);
  if (!near || g.M <= 64 || t128 < 64) return few<ACT, T>(g, s);
  if constexpr (sizeof(T) == 2)
    if (t256 >= 192 && g.K >= 768) return tiles<256, 256, 8, ACT, T>(g, s);
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
