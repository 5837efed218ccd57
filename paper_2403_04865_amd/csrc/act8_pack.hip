// Activations to 8 bits and back (gfx950).
//
// Pack: 16 lanes take a block of 128 columns of one row, 8 columns each: largest finite magnitude over the 16 (within
// a DPP row), the block's power of two, one exact multiplication and one rounding per value.  One pass, 16-byte loads, 8-byte
// stores; bound by memory: es + 1 + 1/128 bytes a value (es: 2 or 4).  403456 x 384 of bfloat16: 92 us there, 75 us back, 5.1 and
// 6.3 TB/s (the way back finds codes in the last-level cache).  The transpose (weights, once per update) reads 64 bytes of a row at a
// time: 1536 x 384 5.5 us (5.5 untransposed), 4096 x 4096 20 (10), 403456 x 384 212 (84).
#include "act8_internal.h"

namespace sl {

namespace {

template <typename T> __device__ __forceinline__ void load8(const T* p, float (&v)[8]);
template <> __device__ __forceinline__ void load8<bf16>(const bf16* p, float (&v)[8]) {
  const u32x4 t = *reinterpret_cast<const u32x4*>(p);
#pragma unroll
  for (int w = 0; w < 4; ++w) {
    v[2 * w] = __uint_as_float(t[w] << 16);
    v[2 * w + 1] = __uint_as_float(t[w] & 0xffff0000u);
  }
}
template <> __device__ __forceinline__ void load8<float>(const float* p, float (&v)[8]) {
  const f32x4 lo = *reinterpret_cast<const f32x4*>(p), hi = *reinterpret_cast<const f32x4*>(p + 4);
#pragma unroll
  for (int e = 0; e < 4; ++e) { v[e] = lo[e]; v[4 + e] = hi[e]; }
}

// 8 values of a lane (zeros behind the last column) -> codes and, by lane 0 of the 16, the scale
__device__ __forceinline__ void put8(const float (&v)[8], uint8_t* codes, uint8_t* scale, bool store, bool first) {
  const unsigned b = a8_block_byte(v, 16);
  const float s = a8_inverse(b);
  u32x2 q;
  q[0] = a8_code4(v[0] * s, v[1] * s, v[2] * s, v[3] * s);
  q[1] = a8_code4(v[4] * s, v[5] * s, v[6] * s, v[7] * s);
  if (store) *reinterpret_cast<u32x2*>(codes) = q;
  if (first) *scale = (uint8_t)b;
}

// V: x's rows can be read in 16-byte pieces
template <typename T, bool V>
__global__ void __launch_bounds__(256) pack_k(const T* __restrict__ x, long long ldx, long long rows, int cols, int nb,
                                              uint8_t* __restrict__ codes, long long ldc, uint8_t* __restrict__ scales, long long lds) {
  const int lane16 = threadIdx.x & 15;
  const long long items = rows * nb, step = (long long)gridDim.x * 16;
  for (long long it = (long long)blockIdx.x * 16 + (threadIdx.x >> 4); it < items; it += step) {
    long long r; int b;
    if (items <= 0xffffffffLL) { const unsigned q = (unsigned)it / (unsigned)nb; r = q; b = (int)((unsigned)it - q * (unsigned)nb); }
    else { r = it / nb; b = (int)(it - r * nb); }
    const int c0 = b * A8_BLOCK + lane16 * 8;
    float v[8];
    const T* p = x + r * ldx + c0;
    if (V && c0 + 8 <= cols) load8(p, v);
    else {
#pragma unroll
      for (int e = 0; e < 8; ++e) v[e] = c0 + e < cols ? to_f(p[e]) : 0.f;
    }
    put8(v, codes + r * ldc + c0, scales + r * lds + b, c0 < (cols + A8_GRAIN - 1) / A8_GRAIN * A8_GRAIN, lane16 == 0);
  }
}

// The transpose: out row r is column r of x.  A workgroup takes a block of 128 rows of x and 32 of its columns through LDS.
template <typename T>
__global__ void __launch_bounds__(256) pack_t_k(const T* __restrict__ x, long long ldx, long long rows, int cols, int nb,
                                                uint8_t* __restrict__ codes, long long ldc, uint8_t* __restrict__ scales, long long lds) {
  __shared__ float t[A8_BLOCK][33];
  const long long rb = (rows + 31) / 32, items = rb * nb;
  for (long long it = blockIdx.x; it < items; it += gridDim.x) {
    const int b = (int)(it / rb), c0 = b * A8_BLOCK;   // columns of the result = rows of x
    const long long r0 = (it - b * rb) * 32;           // rows of the result
    for (int i = threadIdx.x >> 5; i < A8_BLOCK; i += 8) {
      const long long r = r0 + (threadIdx.x & 31);
      t[i][threadIdx.x & 31] = r < rows && c0 + i < cols ? to_f(x[(c0 + i) * ldx + r]) : 0.f;
    }
    __syncthreads();
    const int lane16 = threadIdx.x & 15;
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const int rr = (threadIdx.x >> 4) + 16 * h, cc = c0 + lane16 * 8;
      float v[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) v[e] = t[lane16 * 8 + e][rr];
      const bool have = r0 + rr < rows;
      put8(v, codes + (r0 + rr) * ldc + cc, scales + (r0 + rr) * lds + b,
           have && cc < (cols + A8_GRAIN - 1) / A8_GRAIN * A8_GRAIN, have && lane16 == 0);
    }
    __syncthreads();
  }
}

// V: y's rows can be written in 16-byte pieces.  A lane takes 16 columns.
template <typename T, bool V>
__global__ void __launch_bounds__(256) unpack_k(const uint8_t* __restrict__ codes, long long ldc, const uint8_t* __restrict__ scales,
                                                long long lds, long long rows, int cols, int pieces, T* __restrict__ y, long long ldy) {
  const long long items = rows * pieces, step = (long long)gridDim.x * 256;
  for (long long it = (long long)blockIdx.x * 256 + threadIdx.x; it < items; it += step) {
    long long r; int b;
    if (items <= 0xffffffffLL) { const unsigned q = (unsigned)it / (unsigned)pieces; r = q; b = (int)((unsigned)it - q * (unsigned)pieces); }
    else { r = it / pieces; b = (int)(it - r * pieces); }
    const int c0 = b * 16;
    const u32x4 q = *reinterpret_cast<const u32x4*>(codes + r * ldc + c0);
    const float s = a8_scale(scales[r * lds + (c0 >> 7)]);
    float v[16];
#pragma unroll
    for (int w = 0; w < 4; ++w) {
      float t[4];
      a8_value4(q[w], s, t);
#pragma unroll
      for (int e = 0; e < 4; ++e) v[4 * w + e] = t[e];
    }
    T* p = y + r * ldy + c0;
    if (V && c0 + 16 <= cols) {
      constexpr int E = 16 / sizeof(T);
      typedef T vec __attribute__((ext_vector_type(E)));
#pragma unroll
      for (int h = 0; h < 16 / E; ++h) {
        vec o;
#pragma unroll
        for (int e = 0; e < E; ++e) o[e] = from_f<T>(v[h * E + e]);
        *reinterpret_cast<vec*>(p + h * E) = o;
      }
    } else {
#pragma unroll
      for (int e = 0; e < 16; ++e)
        if (c0 + e < cols) p[e] = from_f<T>(v[e]);
    }
  }
}

int grid_for(long long items, int per) {
  const long long g = (items + per - 1) / per;
  return (int)(g < (1 << 20) ? g : (1 << 20));
}

template <typename T>
hipError_t pack_t(const T* x, long long ldx, bool transpose, const slide_act8& o, hipStream_t s) {
  const int cols = (int)o.cols, nb = (cols + A8_BLOCK - 1) / A8_BLOCK;
  if (transpose) {
    const int grid = grid_for((o.rows + 31) / 32 * nb, 1);
    pack_t_k<T><<<grid, 256, 0, s>>>(x, ldx, o.rows, cols, nb, o.codes, o.ldc, o.scales, o.lds);
    return hipGetLastError();
  }
  const bool v = ((uintptr_t)x & 15) == 0 && (ldx * sizeof(T)) % 16 == 0;
  const int grid = grid_for(o.rows * nb, 16);
  if (v) pack_k<T, true><<<grid, 256, 0, s>>>(x, ldx, o.rows, cols, nb, o.codes, o.ldc, o.scales, o.lds);
  else pack_k<T, false><<<grid, 256, 0, s>>>(x, ldx, o.rows, cols, nb, o.codes, o.ldc, o.scales, o.lds);
  return hipGetLastError();
}

template <typename T>
hipError_t unpack_t(const slide_act8& a, T* y, long long ldy, hipStream_t s) {
  const int cols = (int)a.cols, pieces = (cols + 15) / 16;
  const bool v = ((uintptr_t)y & 15) == 0 && (ldy * sizeof(T)) % 16 == 0;
  const int grid = grid_for(a.rows * pieces, 256);
  if (v) unpack_k<T, true><<<grid, 256, 0, s>>>(a.codes, a.ldc, a.scales, a.lds, a.rows, cols, pieces, y, ldy);
  else unpack_k<T, false><<<grid, 256, 0, s>>>(a.codes, a.ldc, a.scales, a.lds, a.rows, cols, pieces, y, ldy);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_act8_pack(const void* x, int dt, long long ldx, bool transpose, const slide_act8& out, hipStream_t s) {
  return dt == DT_F32 ? pack_t((const float*)x, ldx, transpose, out, s) : pack_t((const bf16*)x, ldx, transpose, out, s);
}
hipError_t launch_act8_unpack(const slide_act8& a, void* y, int dt, long long ldy, hipStream_t s) {
  return dt == DT_F32 ? unpack_t(a, (float*)y, ldy, s) : unpack_t(a, (bf16*)y, ldy, s);
}

}  // namespace sl
