// Internal declarations of the layers on 8-bit activations (include/act8.h; gfx950 only).
#pragma once
#include "../../include/act8.h"
#include <type_traits>

#include "slide_internal.h"

namespace sl {

constexpr int A8_BLOCK = 128;          // columns that share a scale
constexpr int A8_GRAIN = 16;           // a row's codes are zero up to the next multiple of this
constexpr long long A8_MAX_ROWS = (1LL << 31) - 1, A8_MAX_COLS = (1LL << 24) - 1;

typedef unsigned int u32x2 __attribute__((ext_vector_type(2)));
typedef unsigned int u32x4 __attribute__((ext_vector_type(4)));
typedef float f32x2 __attribute__((ext_vector_type(2)));

// The scale byte of a block from the bits of its largest finite magnitude: the magnitude is m 2^E with 1 <= m < 2, 448 is
// 1.75 * 2^8, so the power is E - 8, one more where m > 1.75; not below 2^-127, and 1 for a block of zeros.
__device__ __forceinline__ unsigned a8_scale_byte(unsigned amax_bits) {
  int b = (int)(amax_bits >> 23) - 8 + ((amax_bits & 0x7fffffu) > 0x600000u);
  b = b > 0 ? b : 0;
  return amax_bits ? (unsigned)b : 127u;
}
// 2^(127 - byte): what a value is multiplied with before it is rounded to a code (byte <= 247: never subnormal)
__device__ __forceinline__ float a8_inverse(unsigned byte) { return __uint_as_float((254u - byte) << 23); }
// 2^(byte - 127); byte 0 is a subnormal number, byte 255 (no scale) a NaN
__device__ __forceinline__ float a8_scale(unsigned byte) {
  return __uint_as_float(byte == 0 ? 0x00400000u : byte == 255 ? 0x7fc00000u : byte << 23);
}
// magnitude bits of a value for the block's maximum: what is not finite does not count
__device__ __forceinline__ unsigned a8_mag(float v) {
  const unsigned a = __float_as_uint(v) & 0x7fffffffu;
  return a < 0x7f800000u ? a : 0u;
}
// the largest of a magnitude over neighbouring groups of `lanes` lanes (1, 2, 4, 8 or 16; uniform), in every lane of them
__device__ __forceinline__ float a8_group_max(float v, int lanes) {
  auto step = [&](auto ctrl) {
    v = fmaxf(v, __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(v), decltype(ctrl)::value, 0xf, 0xf, false)));
  };
  if (lanes > 1) step(std::integral_constant<int, 0xb1>{});    // lane ^ 1
  if (lanes > 2) step(std::integral_constant<int, 0x4e>{});    // lane ^ 2
  if (lanes > 4) step(std::integral_constant<int, 0x141>{});   // 7 - lane within eight: the other four, which are all alike
  if (lanes > 8) step(std::integral_constant<int, 0x140>{});   // 15 - lane within sixteen
  return v;
}
// scale byte of the block that `lanes` neighbouring lanes hold, eight values each.  The maximum drops NaN by itself; where an infinity is
// among the values it is taken again over the finite ones.
__device__ __forceinline__ unsigned a8_block_byte(const float (&v)[8], int lanes) {
  float m = 0.f;
#pragma unroll
  for (int e = 0; e < 8; ++e) m = fmaxf(m, fabsf(v[e]));
  m = a8_group_max(m, lanes);
  if (m == __builtin_huge_valf()) {   // alike in all lanes of a block
    m = 0.f;
#pragma unroll
    for (int e = 0; e < 8; ++e) m = fmaxf(m, __uint_as_float(a8_mag(v[e])));
    m = a8_group_max(m, lanes);
  }
  return a8_scale_byte(__float_as_uint(m));
}
// four values -> four codes: nearest, ties to even; what is not finite becomes a NaN
__device__ __forceinline__ unsigned a8_code4(float a, float b, float c, float d) {
  int r = __builtin_amdgcn_cvt_pk_fp8_f32(a, b, 0, false);
  return (unsigned)__builtin_amdgcn_cvt_pk_fp8_f32(c, d, r, true);
}
// four codes -> their values times s
__device__ __forceinline__ void a8_value4(unsigned q, float s, float (&v)[4]) {
  const f32x2 lo = __builtin_amdgcn_cvt_pk_f32_fp8((int)q, false), hi = __builtin_amdgcn_cvt_pk_f32_fp8((int)q, true);
  v[0] = lo[0] * s; v[1] = lo[1] * s; v[2] = hi[0] * s; v[3] = hi[1] * s;
}

// act(u).  GELU: with h = erfc(|u| / sqrt 2) / 2, u Phi(u) = max(u, 0) - |u| h for either sign, no difference of nearly equal numbers;
// h by the same rational approximation as erf_exp (7.1.26 of Abramowitz & Stegun, error 7.5e-8 in h), the factors folded into its
// constants.  Behind GELU_FAR h is below the smallest float, so the argument may stop there (an infinity stays one).
constexpr float GELU_FAR = 16.f;
__device__ __forceinline__ float half_erfc(float x, float* e_out) {   // 0 <= x <= GELU_FAR; e_out: exp(-x^2 / 2)
  const float t = __builtin_amdgcn_rcpf(__builtin_fmaf(0.3275911f * 0.70710678118654752f, x, 1.0f));
  const float e = __builtin_amdgcn_exp2f(x * x * -0.72134752044448170f);
  *e_out = e;
  return (((((0.5f * 1.061405429f) * t - 0.5f * 1.453152027f) * t + 0.5f * 1.421413741f) * t - 0.5f * 0.284496736f) * t + 0.5f * 0.254829592f) * t * e;
}
__device__ __forceinline__ float sigmoid_f(float u) {
  return __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(u * -1.4426950408889634f));
}
template <int ACT> __device__ __forceinline__ float act_f(float u) {
  if constexpr (ACT == SLIDE_ACT_RELU) return u < 0.f ? 0.f : u;      // a NaN stays one
  if constexpr (ACT == SLIDE_ACT_SILU) return u * sigmoid_f(u);
  if constexpr (ACT == SLIDE_ACT_GELU) {
    float e;
    const float x = fminf(fabsf(u), GELU_FAR), h = half_erfc(x, &e);
    return __builtin_fmaf(-x, h, u < 0.f ? 0.f : u);   // a NaN stays one
  }
  return u;
}

// A matrix [rows][cols] in 8 bits as the kernels see it.
struct A8 { const uint8_t* codes; long long ldc; const uint8_t* scales; long long lds; };
inline A8 a8_view(const slide_act8& a) { return A8{a.codes, a.ldc, a.scales, a.lds}; }

hipError_t launch_act8_pack(const void* x, int dt, long long ldx, bool transpose, const slide_act8& out, hipStream_t s);
hipError_t launch_act8_unpack(const slide_act8& a, void* y, int dt, long long ldy, hipStream_t s);

struct A8Linear {
  const void* xin; long long ldxin;   // x to be packed into `x` (shares no memory with y), or null: packed before
  A8 x, w;
  long long M; int N, K;
  const float* bias;
  int act, dt;
  const void* resid; long long ldr;
  void* y; long long ldy;
};
hipError_t launch_act8_linear(const A8Linear& g, hipStream_t s);

struct A8Wgrad {
  const void* dy; int dt; long long lddy;
  A8 x;
  long long M; int N, K;
  float* dW; long long lddw;
  float* db;
  int accumulate;
  float* work;
};
size_t act8_wgrad_bytes(long long M, int N, int K);
hipError_t launch_act8_wgrad(const A8Wgrad& g, hipStream_t s);

struct GroupNorm {
  slide_group_norm s;
  const void* x; long long ldx;       // bwd: null = from x8
  const float *gamma, *beta;
  const void* resid; long long ldr;
  const void* out; long long ldo;     // bwd of a rectifier from x8, bfloat16: what the forward put out (resid is not read then), or null
  void* y; long long ldy;             // bwd: dx
  const slide_act8* x8;               // fwd: written (may be null); bwd: read where x is null
  float *mean, *rstd;
  const void* dy; long long lddy;
  void* dresid; long long lddr;
  float *dgamma, *dbeta;
  int accumulate;
  float* work;
};
size_t group_norm_bytes(const slide_group_norm& s);
hipError_t launch_group_norm_fwd(const GroupNorm& g, hipStream_t s);
hipError_t launch_group_norm_bwd(const GroupNorm& g, hipStream_t s);

}  // namespace sl
