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

template <int ACT, typename T>
hipError_t run(const A8Linear& g, hipStream_t s) {
  return few<ACT, T>(g, s);
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
