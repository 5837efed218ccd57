// Attention over packed slides, backward: dout . o of every row, and the gradient of the queries (layout: tokens_attn.h).
#include "tokens_attn.h"

namespace sl {

namespace {

// delta[head][row] = dout . o in float32: a group of eight lanes a row and head
template <typename T>
__global__ void __launch_bounds__(256) tok_delta_k(const TokAttn g) {
  constexpr int EPC = TokType<T>::EPC;
  const long long item = blockIdx.x * 32LL + (threadIdx.x >> 3);
  const int part = threadIdx.x & 7;
  if (item >= (long long)g.rows_q * g.hq) return;
  const long long row = item / g.hq;
  const int head = (int)(item % g.hq);
  if (row < tok_clamp(g.q_start[0], g.rows_q) || row >= tok_clamp(g.q_start[g.docs], g.rows_q)) return;
  const T* a = (const T*)g.dout + row * g.lddo + head * g.dim;
  const T* b = (const T*)g.o_in + row * g.ldo + head * g.dim;
  float sum = 0.f;
  for (int c = part * EPC; c < g.dim; c += 8 * EPC) {
    const u32x4 va = *reinterpret_cast<const u32x4*>(a + c), vb = *reinterpret_cast<const u32x4*>(b + c);
    T ea[EPC], eb[EPC];
    __builtin_memcpy(ea, &va, 16);
    __builtin_memcpy(eb, &vb, 16);
#pragma unroll
    for (int i = 0; i < EPC; ++i) sum = fmaf(to_f(ea[i]), to_f(eb[i]), sum);
  }
#pragma unroll
  for (int o = 4; o > 0; o >>= 1) sum += __shfl_xor(sum, o, 64);
  if (part == 0) g.delta[head * (long long)g.rows_q + row] = sum;
}

template <typename T, int DP, int NW, bool BIAS, bool CAP>
__global__ void __launch_bounds__(NW * 64, (tok_waves<T, DP, NW>())) tok_dq_k(const TokAttn g, const int slots) {
  constexpr int KB = TokType<T>::KB, LDR = tok_ldr<T, DP>(), NB = KB / 32, W = NW * 32;
  __shared__ __attribute__((aligned(16))) T Ks[KB * LDR], Vs[KB * LDR];
  __shared__ __attribute__((aligned(16))) float px[KB], py[KB];
  TokWork w;
  if (!tok_work(slots, g.splits, g.hk, &w)) return;
  const TokDoc doc = tok_find(g.q_start, g.docs, g.rows_q, g.group, W, w.slot);
  if (doc.doc < 0) return;
  const int cols = (doc.hi - doc.lo) * g.group;
  if ((long long)doc.tile * W >= cols) return;
  const int klo = tok_clamp(g.k_start[doc.doc], g.rows_k), khi = tok_clamp(g.k_start[doc.doc + 1], g.rows_k), nk = khi > klo ? khi - klo : 0;

  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int c = doc.tile * W + wave * 32 + (lane & 31);
  const bool valid = c < cols;
  const int qi = valid ? c / g.group : 0, head = w.head * g.group + (valid ? c - qi * g.group : 0);
  const long long qrow = doc.lo + qi;
  TokFrag<T, DP> fq, fo;
  tok_load_frag<T, DP>(fq, (const T*)g.q + qrow * g.ldq + head * g.dim, valid, g.dim);
  tok_load_frag<T, DP>(fo, (const T*)g.dout + qrow * g.lddo + head * g.dim, valid, g.dim);
  // a column that is not there: infinite, so its probabilities are zero
  const float lse = valid ? g.lse[(long long)head * g.rows_q + qrow] * TOK_LOG2E : INFINITY;
  const float delta = valid ? g.delta[(long long)head * g.rows_q + qrow] : 0.f;
  const TokScore sc = tok_score_of<CAP>(g.scale, g.cap);
  float qx = 0.f, qy = 0.f, slope = 0.f;
  if (BIAS && valid && qi >= g.lead_q) {
    qx = g.pos_q[2 * qrow]; qy = g.pos_q[2 * qrow + 1];
    slope = g.slopes[head] * sc.per_slope;
  }

  const int tiles = (nk + KB - 1) / KB, per = (tiles + g.splits - 1) / g.splits;
  const int t0 = w.split * per, t1 = t0 + per < tiles ? t0 + per : tiles;
  const T* const kp = (const T*)g.k + (long long)klo * g.ldk + w.head * g.dim;
  const T* const vp = (const T*)g.v + (long long)klo * g.ldv + w.head * g.dim;
  TokTile<T, DP, NW * 64> kt, vt;
  f32x16 dq[DP / 32];
  tok_zero_all(dq);
  if (t0 < t1) {
    kt.load(kp + (long long)t0 * KB * g.ldk, nk - t0 * KB, g.ldk, g.dim);
    vt.load(vp + (long long)t0 * KB * g.ldv, nk - t0 * KB, g.ldv, g.dim);
  }
#pragma unroll 1
  for (int t = t0; t < t1; ++t) {
    const int k0 = t * KB;
    __syncthreads();
    kt.store(Ks);
    vt.store(Vs);
    if (BIAS) tok_put_places<KB>(px, py, g.pos_k, klo, k0, nk, g.lead_k);
    __syncthreads();
    if (t + 1 < t1) {
      kt.load(kp + (long long)(k0 + KB) * g.ldk, nk - k0 - KB, g.ldk, g.dim);
      vt.load(vp + (long long)(k0 + KB) * g.ldv, nk - k0 - KB, g.ldv, g.dim);
    }
    auto block = [&](auto edge, int b) __attribute__((always_inline)) {
      constexpr bool EDGE = decltype(edge)::value;
      f32x16 s = tok_zero(), dp = tok_zero();
      tok_mul<T, DP>(s, Ks, b * 32, fq);
      tok_mul<T, DP>(dp, Vs, b * 32, fo);
#pragma unroll
      for (int q4 = 0; q4 < 4; ++q4) {
        const int r0 = b * 32 + tok_row(q4 * 4);
        f32x4 kx, ky;
        if (BIAS) {
          kx = *reinterpret_cast<const f32x4*>(px + r0);
          ky = *reinterpret_cast<const f32x4*>(py + r0);
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const int r = q4 * 4 + i;
          float d = BIAS ? tok_dist(qx, qy, kx[i], ky[i]) : 0.f, dt = 1.f;
          if (EDGE && BIAS && k0 + r0 + i < g.lead_k) d = 0.f;
          const float z = tok_score<T, BIAS, CAP, true>(s[r], d, slope, sc, &dt);
          float ds = tok_exp<CAP>(z, lse, sc) * (dp[r] - delta);
          if (CAP) ds *= dt;
          if (EDGE && k0 + r0 + i >= nk) ds = 0.f;   // there K is zeros, but a probability may be no number
          s[r] = ds;
        }
      }
      tok_mul_t<T, DP>(dq, Ks, b * 32, s);
    };
    const bool edge = (BIAS && k0 < g.lead_k) || k0 + KB > nk;   // uniform
#pragma unroll
    for (int b = 0; b < NB; ++b) {
      if (edge) block(std::true_type{}, b);
      else block(std::false_type{}, b);
    }
  }
  if (!valid) return;
  const float f = CAP ? 4.f * g.scale : g.scale;   // scores' gradients carry a quarter of the cap's derivative
  if (g.splits > 1) tok_store(dq, f, g.part + ((w.split * (long long)g.rows_q + qrow) * g.hq + head) * g.dim, g.dim);
  else tok_store(dq, f, (T*)g.dq + qrow * g.lddq + head * g.dim, g.dim);
}

template <typename T>
__global__ void __launch_bounds__(256) tok_sum_k(const float* __restrict__ part, int splits, int rows, int cols, const int* __restrict__ start,
                                                 int docs, T* __restrict__ out, int ld) {
  const long long at = (blockIdx.x * 256LL + threadIdx.x) * 4;
  const long long row = at / cols;
  const int col = (int)(at - row * cols);
  if (row < tok_clamp(start[0], rows) || row >= tok_clamp(start[docs], rows)) return;
  f32x4 a = {0.f, 0.f, 0.f, 0.f};
  const long long stride = (long long)rows * cols;
  for (int z = 0; z < splits; ++z) a += *reinterpret_cast<const f32x4*>(part + z * stride + at);
  typedef T T4 __attribute__((ext_vector_type(4)));
  T4 v;
#pragma unroll
  for (int i = 0; i < 4; ++i) v[i] = from_f<T>(a[i]);
  *reinterpret_cast<T4*>(out + row * ld + col) = v;
}

template <typename T>
hipError_t run_dq(const TokAttn& g, TokCut c, hipStream_t s) {
  return tok_dispatch<T>(g, [&](auto dp, auto bias, auto cap) {
    constexpr int DP = decltype(dp)::value;
    constexpr bool BIAS = decltype(bias)::value, CAP = decltype(cap)::value;
    if (c.waves == 4) tok_dq_k<T, DP, 4, BIAS, CAP><<<tok_grid(c, g.hk), 256, 0, s>>>(g, c.slots);
    else tok_dq_k<T, DP, 1, BIAS, CAP><<<tok_grid(c, g.hk), 64, 0, s>>>(g, c.slots);
    return hipGetLastError();
  });
}

}  // namespace

hipError_t launch_tok_delta(int dt, const TokAttn& g, hipStream_t s) {
  const unsigned blocks = (unsigned)(((long long)g.rows_q * g.hq + 31) / 32);
  if (dt == DT_F32) tok_delta_k<float><<<blocks, 256, 0, s>>>(g);
  else tok_delta_k<bf16><<<blocks, 256, 0, s>>>(g);
  return hipGetLastError();
}

hipError_t launch_tok_dq(int dt, const TokAttn& g, TokCut c, hipStream_t s) { return dt == DT_F32 ? run_dq<float>(g, c, s) : run_dq<bf16>(g, c, s); }

hipError_t launch_tok_sum(int dt, const float* part, int splits, int rows, int cols, const int* start, int docs, void* out, int ld, hipStream_t s) {
  const unsigned blocks = (unsigned)(((long long)rows * cols / 4 + 255) / 256);
  if (dt == DT_F32) tok_sum_k<float><<<blocks, 256, 0, s>>>(part, splits, rows, cols, start, docs, (float*)out, ld);
  else tok_sum_k<bf16><<<blocks, 256, 0, s>>>(part, splits, rows, cols, start, docs, (bf16*)out, ld);
  return hipGetLastError();
}

}  // namespace sl
