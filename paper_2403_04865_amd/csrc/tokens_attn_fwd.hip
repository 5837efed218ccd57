// Attention over packed slides, forward: one pass over the keys with a running maximum and sum (layout: tokens_attn.h).
#include "tokens_attn.h"

namespace sl {

namespace {

template <typename T, int DP, int NW, bool BIAS, bool CAP>
__global__ void __launch_bounds__(NW * 64, (tok_waves<T, DP, NW>())) tok_fwd_k(const TokAttn g, const int slots) {
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
  TokFrag<T, DP> fq;
  tok_load_frag<T, DP>(fq, (const T*)g.q + qrow * g.ldq + head * g.dim, valid, g.dim);
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
  f32x16 o[DP / 32];
  tok_zero_all(o);
  float m = -INFINITY, l = 0.f;
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
    f32x16 s[NB];
#pragma unroll
    for (int b = 0; b < NB; ++b) {
      s[b] = tok_zero();
      tok_mul<T, DP>(s[b], Ks, b * 32, fq);
    }
    // the first and the last blocks hold keys without a place and keys that are not there: a copy of the loop of their own
    auto scores = [&](auto edge) __attribute__((always_inline)) {
      constexpr bool EDGE = decltype(edge)::value;
#pragma unroll
      for (int b = 0; b < NB; ++b)
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
            float d = BIAS ? tok_dist(qx, qy, kx[i], ky[i]) : 0.f;
            if (EDGE && BIAS && k0 + r0 + i < g.lead_k) d = 0.f;
            float z = tok_score<T, BIAS, CAP, false>(s[b][q4 * 4 + i], d, slope, sc, nullptr);
            if (EDGE && k0 + r0 + i >= nk) z = -INFINITY;
            s[b][q4 * 4 + i] = z;
          }
        }
    };
    if ((BIAS && k0 < g.lead_k) || k0 + KB > nk) scores(std::true_type{});   // uniform
    else scores(std::false_type{});
    float mn = m;
#pragma unroll
    for (int b = 0; b < NB; ++b)
#pragma unroll
      for (int r = 0; r < 16; ++r) mn = fmaxf(mn, s[b][r]);
    mn = fmaxf(mn, __shfl_xor(mn, 32, 64));
    const float ms = mn == -INFINITY ? 0.f : mn * sc.ex;
    const float resc = tok_exp<CAP>(m, ms, sc);   // 0 at the first block
    m = mn;
    float ls = 0.f;
#pragma unroll
    for (int b = 0; b < NB; ++b)
#pragma unroll
      for (int r = 0; r < 16; ++r) {
        s[b][r] = tok_exp<CAP>(s[b][r], ms, sc);
        ls += s[b][r];
      }
    l = fmaf(l, resc, ls);
    if (__builtin_amdgcn_ballot_w64(resc != 1.f) != 0) {   // uniform: after the first blocks the maximum rarely moves
#pragma unroll
      for (int d = 0; d < DP / 32; ++d)
#pragma unroll
        for (int r = 0; r < 16; ++r) o[d][r] *= resc;
    }
#pragma unroll
    for (int b = 0; b < NB; ++b) tok_mul_t<T, DP>(o, Vs, b * 32, s[b]);
  }
  l += __shfl_xor(l, 32, 64);
  m *= sc.ex;
  if (!valid) return;
  const bool none = t0 >= t1;
  if (g.splits > 1) {
    const long long at = (w.split * (long long)g.rows_q + qrow) * g.hq + head;
    if (lane < 32) *reinterpret_cast<float2*>(g.part2 + 2 * at) = float2{none ? -INFINITY : m, none ? 0.f : l};
    if (!none) tok_store(o, 1.f, g.part + at * g.dim, g.dim);
    return;
  }
  const bool nothing = l == 0.f;   // no keys, or none within reach of a bias that is infinite
  tok_store(o, nothing ? 0.f : 1.f / l, (T*)g.o + qrow * g.ldo + head * g.dim, g.dim);
  if (lane < 32) g.lse[(long long)head * g.rows_q + qrow] = nothing ? -INFINITY : (m + __builtin_amdgcn_logf(l)) * TOK_LN2;
}

// The ranges' results of a query and head joined, a wavefront each
template <typename T>
__global__ void __launch_bounds__(256) tok_join_k(const TokAttn g) {
  const long long item = blockIdx.x * 4LL + (threadIdx.x >> 6);
  const int lane = threadIdx.x & 63;
  const int first = tok_clamp(g.q_start[0], g.rows_q), end = tok_clamp(g.q_start[g.docs], g.rows_q);
  const long long row = item / g.hq;
  const int head = (int)(item % g.hq);
  if (row < first || row >= end) return;
  const float2* ml = reinterpret_cast<const float2*>(g.part2);
  const long long stride = (long long)g.rows_q * g.hq;
  float m = -INFINITY, l = 0.f;
  for (int z = lane; z < g.splits; z += 64) {
    const float2 p = ml[z * stride + item];
    const float n = fmaxf(m, p.x), ns = n == -INFINITY ? 0.f : n;
    l = l * __builtin_amdgcn_exp2f(m - ns) + p.y * __builtin_amdgcn_exp2f(p.x - ns);
    m = n;
  }
  const float all = wave_max(m), alls = all == -INFINITY ? 0.f : all;
  l = wave_sum(l * __builtin_amdgcn_exp2f(m - alls));
  const bool none = l == 0.f;
  const float inv = none ? 0.f : 1.f / l;
  for (int d = lane; d < g.dim; d += 64) {
    float o = 0.f;
    for (int z = 0; z < g.splits; ++z) {
      const float2 p = ml[z * stride + item];
      if (p.y != 0.f) o = fmaf(g.part[(z * stride + item) * g.dim + d], __builtin_amdgcn_exp2f(p.x - alls), o);   // ranges without keys wrote no sums
    }
    ((T*)g.o)[row * g.ldo + head * g.dim + d] = from_f<T>(o * inv);
  }
  if (lane == 0) g.lse[head * (long long)g.rows_q + row] = none ? -INFINITY : (all + __builtin_amdgcn_logf(l)) * TOK_LN2;
}

template <typename T>
hipError_t run_fwd(const TokAttn& g, TokCut c, hipStream_t s) {
  const hipError_t e = tok_dispatch<T>(g, [&](auto dp, auto bias, auto cap) {
    constexpr int DP = decltype(dp)::value;
    constexpr bool BIAS = decltype(bias)::value, CAP = decltype(cap)::value;
    if (c.waves == 4) tok_fwd_k<T, DP, 4, BIAS, CAP><<<tok_grid(c, g.hk), 256, 0, s>>>(g, c.slots);
    else tok_fwd_k<T, DP, 1, BIAS, CAP><<<tok_grid(c, g.hk), 64, 0, s>>>(g, c.slots);
    return hipGetLastError();
  });
  if (e != hipSuccess || c.splits == 1) return e;
  tok_join_k<T><<<(unsigned)(((long long)g.rows_q * g.hq + 3) / 4), 256, 0, s>>>(g);
  return hipGetLastError();
}

}  // namespace

// Few columns a slide leave three of four wavefronts idle: a wavefront a workgroup then.  Rows are split over as many workgroups as give the card's
// 256 units two of four wavefronts, or eight of one, but not below four blocks of rows each.
TokCut tok_cut(long long cols, long long other, int docs, int heads, int dt, int dim) {
  TokCut c;
  c.waves = cols <= 32LL * docs ? 1 : 4;
  const int width = 32 * c.waves;
  c.slots = (int)(cols / width + docs);
  const long long filled = (cols / width > docs ? cols / width : docs) * heads;
  const long long wanted = c.waves == 1 ? 2048 : 512, kb = dt == DT_F32 ? 32 : 64;
  long long n = filled >= wanted / 2 ? 1 : (wanted + filled - 1) / filled;
  const long long most = (other / kb + 3) / 4;
  n = n < most ? n : most;
  c.splits = (int)(n < 1 ? 1 : n > 128 ? 128 : n);
  return c;
}

hipError_t launch_tok_fwd(int dt, const TokAttn& g, TokCut c, hipStream_t s) { return dt == DT_F32 ? run_fwd<float>(g, c, s) : run_fwd<bf16>(g, c, s); }

}  // namespace sl
