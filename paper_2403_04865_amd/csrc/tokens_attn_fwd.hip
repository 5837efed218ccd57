// Attention over packed slides, forward: one pass over the keys with a running maximum and sum (layout: tokens_attn.h).
#include "tokens_attn.h"

namespace sl {

namespace {

template <typename T, int DP, int NW, bool BIAS, bool CAP>
__global__ void __launch_bounds__(NW * 64, (tok_waves<T, DP, NW>())) tok_fwd_k(const TokAttn g) {
  constexpr int KB = TokType<T>::KB, LDR = tok_ldr<T, DP>(), NB = KB / 32, W = NW * 32;
  __shared__ __attribute__((aligned(16))) T Ks[KB * LDR], Vs[KB * LDR];
  __shared__ __attribute__((aligned(16))) float px[KB], py[KB];
  const TokScore sc = tok_score_of<CAP>(g.scale, g.cap);
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  tok_walk(tok_queries(g, W), tok_keys(g, KB), g.docs, g.hk, g.table, (TokJoin*)g.joins, [&](const TokSeg& w) __attribute__((always_inline)) {
    const int cols = w.c.n, nk = w.r.n, klo = w.r.lo;
    const int c = w.tile * W + wave * 32 + (lane & 31);
    const bool valid = c < cols, idle = w.tile * W + wave * 32 >= cols;
    const int qi = valid ? c / g.group : 0, head = w.head * g.group + (valid ? c - qi * g.group : 0);
    const long long qrow = w.c.lo + qi;
    TokFrag<T, DP> fq;
    tok_load_frag<T, DP>(fq, (const T*)g.q + qrow * g.ldq + head * g.dim, valid, g.dim);
    float qx = 0.f, qy = 0.f, slope = 0.f;
    if (BIAS && valid && qi >= g.lead_q) {
      qx = g.pos_q[2 * qrow]; qy = g.pos_q[2 * qrow + 1];
      slope = g.slopes[head] * sc.per_slope;
    }
    const T* const kp = (const T*)g.k + (long long)klo * g.ldk + w.head * g.dim;
    const T* const vp = (const T*)g.v + (long long)klo * g.ldv + w.head * g.dim;
    TokTile<T, DP, NW * 64> kt, vt;
    f32x16 o[DP / 32];
    tok_zero_all(o);
    float m = -INFINITY, l = 0.f;
    if (nk > 0) {
      kt.load(kp + (long long)w.a * KB * g.ldk, nk - w.a * KB, g.ldk, g.dim);
      vt.load(vp + (long long)w.a * KB * g.ldv, nk - w.a * KB, g.ldv, g.dim);
#pragma unroll 1
      for (int t = w.a; t < w.b; ++t) {
        const int k0 = t * KB;
        __syncthreads();
        kt.store(Ks);
        vt.store(Vs);
        if (BIAS) tok_put_places<KB>(px, py, g.pos_k, klo, k0, nk, g.lead_k);
        __syncthreads();
        if (t + 1 < w.b) {
          kt.load(kp + (long long)(k0 + KB) * g.ldk, nk - k0 - KB, g.ldk, g.dim);
          vt.load(vp + (long long)(k0 + KB) * g.ldv, nk - k0 - KB, g.ldv, g.dim);
        }
        if (idle) continue;   // uniform in a wavefront: none of its columns is there
        f32x16 s[NB];
#pragma unroll
        for (int b = 0; b < NB; ++b) {
          s[b] = tok_zero();
          tok_mul<T, DP>(s[b], Ks, b * 32, fq);
        }
        // the first and the last blocks hold keys without a place and keys that are not there: a copy of the code of their own
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
        mn = tok_other_max(mn);
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
    }
    l = tok_other_sum(l);
    m *= sc.ex;
    if (!valid) return;
    if (w.slot >= 0) {
      const long long at = (long long)w.slot * W + wave * 32 + (lane & 31);
      if (lane < 32) *reinterpret_cast<float2*>(g.part2 + 2 * at) = float2{m, l};
      tok_store(o, 1.f, g.part + at * g.dim, g.dim);
      return;
    }
    const bool nothing = l == 0.f;   // no keys, or none within reach of a bias that is infinite
    tok_store(o, nothing ? 0.f : 1.f / l, (T*)g.o + qrow * g.ldo + head * g.dim, g.dim);
    if (lane < 32) g.lse[(long long)head * g.rows_q + qrow] = nothing ? -INFINITY : (m + __builtin_amdgcn_logf(l)) * TOK_LN2;
  });
}

template <typename T>
hipError_t run_fwd(const TokAttn& g, TokCut c, hipStream_t s) {
  return tok_dispatch<T>(g, [&](auto dp, auto bias, auto cap) {
    constexpr int DP = decltype(dp)::value;
    constexpr bool BIAS = decltype(bias)::value, CAP = decltype(cap)::value;
    if (c.waves == 4) tok_fwd_k<T, DP, 4, BIAS, CAP><<<c.blocks, 256, 0, s>>>(g);
    else tok_fwd_k<T, DP, 1, BIAS, CAP><<<c.blocks, 64, 0, s>>>(g);
    return hipGetLastError();
  });
}

}  // namespace

hipError_t launch_tok_fwd(int dt, const TokAttn& g, TokCut c, hipStream_t s) { return dt == DT_F32 ? run_fwd<float>(g, c, s) : run_fwd<bf16>(g, c, s); }

}  // namespace sl
