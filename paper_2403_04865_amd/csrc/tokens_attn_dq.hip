// Attention over packed slides, backward: the gradient of the queries, and dout . o of every row for the keys' pass (layout: tokens_attn.h).
#include "tokens_attn.h"

namespace sl {

namespace {

// sum of the products of two columns, over the lane and the other one of its column
template <typename T, int DP>
__device__ __forceinline__ float tok_dot(const TokFrag<T, DP>& a, const TokFrag<T, DP>& b) {
  constexpr int EPC = TokType<T>::EPC;
  float sum = 0.f;
#pragma unroll
  for (int i = 0; i < DP / EPC / 2; ++i) {
    T ea[EPC], eb[EPC];
    __builtin_memcpy(ea, &a.v[i], 16);
    __builtin_memcpy(eb, &b.v[i], 16);
#pragma unroll
    for (int e = 0; e < EPC; ++e) sum = fmaf(to_f(ea[e]), to_f(eb[e]), sum);
  }
  return tok_other_sum(sum);
}

// dS = P (dP - delta) with delta = dout . o = sum P dP.  Out of an o that has been rounded to bfloat16 delta is some e short, and every dS of the row off by
// P e.  The sum of a row's P (dP - delta) is that e (P sums to one), so it is known when the row has been passed: the keys' pass gets the right delta.  Mending: this
// pass takes e times sum P k off, for another product.  Where few keys count, dP - delta is small beside both and e decides (slides of 2 rows: gradients of the
// queries 3.7e-3 off, 2.4e-3 mended; of 100 rows, head of 32, strong bias: 3.4e-3 and 2.4e-3); in slides of more than TOK_MEND_KEYS keys it is 2e-4 to 6e-4 beside the 2.4e-3
// of the roundings to bfloat16 where a row's probabilities spread (a bias of 1 a place of a grid: gradients of the queries 2.7e-3 off), and the product not worth its time (8193 rows, 6 heads
// of 64, both directions: 731 us without e, 764 with e for the keys, 860 with the product too); a head whose bias leaves a long slide's rows one or two keys (4 a place) has
// 8e-3.  So it goes by the slide's keys, in a copy of the loop.  A single wavefront mends always.  float32 needs neither.
// Bound by the vector and matrix units in turn: 51 and 31 % of the time there, two wavefronts a SIMD that do not hide all of each other's waits.
template <typename T, int DP, int NW, bool BIAS, int CAP>
__global__ void __launch_bounds__(NW * 64, DP <= 64 && NW == 4 ? 2 : 1) tok_dq_k(const TokAttn g) {
  constexpr int KB = DP == 128 ? 32 : TokType<T>::KB, LDR = tok_ldr<T, DP>(), NB = KB / 32, W = NW * 32;
  __shared__ __attribute__((aligned(16))) T Ks[KB * LDR], Vs[KB * LDR];
  __shared__ __attribute__((aligned(16))) float px[KB], py[KB];
  const TokScore sc = tok_score_of<CAP>(g.scale, g.cap);
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  tok_walk(tok_queries(g, W, g.group), tok_keys(g, KB), g.docs, g.hk, g.table, (TokJoin*)g.joins, [&](const TokSeg& w) __attribute__((always_inline)) {
    const int cols = w.c.n, nk = w.r.n, klo = w.r.lo;
    const int c = w.tile * W + wave * 32 + (lane & 31);
    const bool valid = c < cols, idle = w.tile * W + wave * 32 >= cols;
    const int qi = valid ? c / g.group : 0, head = w.head * g.group + (valid ? c - qi * g.group : 0);
    const long long qrow = w.c.lo + qi;
    TokFrag<T, DP> fq, fo;
    tok_load_frag<T, DP>(fq, (const T*)g.q + qrow * g.ldq + head * g.dim, valid, g.dim);
    tok_load_frag<T, DP>(fo, (const T*)g.dout + qrow * g.lddo + head * g.dim, valid, g.dim);
    // a column that is not there: infinite, so its probabilities are zero
    const float lse = valid ? g.lse[(long long)head * g.rows_q + qrow] * TOK_LOG2E : INFINITY;
    float delta;   // dout . o, also for the keys' pass (where a tile is shared, its join adds e)
    {
      TokFrag<T, DP> f;
      tok_load_frag<T, DP>(f, (const T*)g.o_in + qrow * g.ldo + head * g.dim, valid, g.dim);
      delta = tok_dot<T, DP>(fo, f);
      if (valid && w.a == 0 && lane < 32) g.delta[(long long)head * g.rows_q + qrow] = delta;
    }
    float qx = 0.f, qy = 0.f, slope = 0.f;
    if (BIAS && valid && qi >= g.lead_q) {
      qx = g.pos_q[2 * qrow]; qy = g.pos_q[2 * qrow + 1];
      slope = g.slopes[head] * sc.per_slope;
    }
    const T* const kp = (const T*)g.k + (long long)klo * g.ldk + w.head * g.dim;
    const T* const vp = (const T*)g.v + (long long)klo * g.ldv + w.head * g.dim;
    TokTile<T, DP, NW * 64, KB> kt(g.ldk, g.dim), vt(g.ldv, g.dim);
    TokPlace place = {0.f, 0.f};
    constexpr bool ERR = sizeof(T) == 2;
    auto pass = [&](auto mend) __attribute__((always_inline)) {
      constexpr bool MEND = decltype(mend)::value;
      f32x16 dq[DP / 32], pk[MEND ? DP / 32 : 1];
      tok_zero_all(dq);
      tok_zero_all(pk);
      float e = 0.f;   // sum of P (dP - delta)
      if (nk > 0) {
        kt.load(kp + (long long)w.a * KB * g.ldk, nk - w.a * KB, g.ldk, g.dim);
        vt.load(vp + (long long)w.a * KB * g.ldv, nk - w.a * KB, g.ldv, g.dim);
        if (BIAS) place = tok_place<KB>(g.pos_k, klo, w.a * KB, nk, g.lead_k);
#pragma unroll 1
        for (int t = w.a; t < w.b; ++t) {
          const int k0 = t * KB;
          __syncthreads();
          kt.store(Ks);
          vt.store(Vs);
          if (BIAS && threadIdx.x < KB) { px[threadIdx.x] = place.x; py[threadIdx.x] = place.y; }
          __syncthreads();
          if (t + 1 < w.b) {
            kt.load(kp + (long long)(k0 + KB) * g.ldk, nk - k0 - KB, g.ldk, g.dim);
            vt.load(vp + (long long)(k0 + KB) * g.ldv, nk - k0 - KB, g.ldv, g.dim);
            if (BIAS) place = tok_place<KB>(g.pos_k, klo, k0 + KB, nk, g.lead_k);
          }
          if (idle) continue;   // uniform in a wavefront: none of its columns is there
          // the first and the last blocks hold keys without a place and keys that are not there: a copy of the code of their own
          auto block = [&](auto edge, int b) __attribute__((always_inline)) {
            constexpr bool EDGE = decltype(edge)::value;
            f32x16 s = tok_zero(), dp = tok_zero(), dist, p;
            if (BIAS) tok_dists<T>(dist, px, py, b * 32, qx, qy);
            TokRows<T, DP> kr, vr;
            TokCols<T, DP> kc;
            tok_get<T, DP>(kr, Ks, b * 32);
            tok_get<T, DP>(vr, Vs, b * 32);
            tok_mul<T, DP>(s, kr, fq);
            tok_mul<T, DP>(dp, vr, fo);
#pragma unroll
            for (int q4 = 0; q4 < 4; ++q4) {
              const int r0 = b * 32 + tok_row(q4 * 4);
#pragma unroll
              for (int i = 0; i < 4; ++i) {
                const int r = q4 * 4 + i;
                float d = BIAS ? dist[r] : 0.f, dt = 1.f;
                if (EDGE && BIAS && k0 + r0 + i < g.lead_k) d = 0.f;
                const float z = tok_score<T, BIAS, CAP, true>(s[r], d, slope, sc, &dt);
                p[r] = tok_exp<CAP>(z, lse, sc);
                if (EDGE && k0 + r0 + i >= nk) p[r] = 0.f;   // there K is zeros, but a probability may be no number
                float ds = p[r] * (dp[r] - delta);
                if (ERR) e += ds;
                if (CAP) {
                  ds *= dt;
                  if (MEND) p[r] *= dt;
                }
                s[r] = ds;
              }
            }
            tok_get_t(kc, Ks, b * 32);
            tok_mul_t<DP, NW == 1>(dq, kc, s);
            if constexpr (MEND) tok_mul_t<DP, false>(pk, kc, p);
          };
          const bool edge = (BIAS && k0 < g.lead_k) || k0 + KB > nk;   // uniform
#pragma unroll
          for (int b = 0; b < NB; ++b) {
            // short slides' blocks are edges mostly, and with both copies four wavefronts run out of registers (256 slides of 197 rows, both directions: 269 us, 251 without)
            if ((MEND && NW == 4) || edge) block(std::true_type{}, b);
            else block(std::false_type{}, b);
          }
        }
      }
      if (ERR) e = tok_other_sum(e);
      if (!valid) return;
      const float f = CAP ? 4.f * g.scale : g.scale;   // scores' gradients carry a quarter of the cap's derivative
      if (w.slot >= 0) {
        const long long at = (long long)w.slot * W + wave * 32 + (lane & 31);
        tok_store(dq, f, g.part + at * g.dim, g.dim);
        if constexpr (MEND) tok_store(pk, f, g.part2 + at * g.dim, g.dim);
        if (ERR && lane < 32) g.part3[at] = e;
        return;
      }
      if constexpr (MEND) {
#pragma unroll
        for (int d = 0; d < DP / 32; ++d)
#pragma unroll
          for (int r = 0; r < 16; ++r) dq[d][r] = fmaf(-e, pk[d][r], dq[d][r]);
      }
      if (ERR && lane < 32) g.delta[(long long)head * g.rows_q + qrow] = delta + e;
      tok_store(dq, f, (T*)g.dq + qrow * g.lddq + head * g.dim, g.dim);
    };
    if constexpr (!ERR) pass(std::false_type{});
    else if constexpr (NW == 1) pass(std::true_type{});
    else if (nk <= TOK_MEND_KEYS) pass(std::true_type{});   // uniform
    else pass(std::false_type{});
  });
}

template <typename T>
hipError_t run_dq(const TokAttn& g, TokCut c, hipStream_t s) {
  return tok_dispatch<T>(g, [&](auto dp, auto bias, auto cap) {
    constexpr int DP = decltype(dp)::value;
    constexpr bool BIAS = decltype(bias)::value;
    constexpr int CAP = decltype(cap)::value;
    if (c.waves == 4) tok_dq_k<T, DP, 4, BIAS, CAP><<<c.blocks, 256, 0, s>>>(g);
    else tok_dq_k<T, DP, 1, BIAS, CAP><<<c.blocks, 64, 0, s>>>(g);
    return hipGetLastError();
  });
}

}  // namespace

hipError_t launch_tok_dq(int dt, const TokAttn& g, TokCut c, hipStream_t s) { return dt == DT_F32 ? run_dq<float>(g, c, s) : run_dq<bf16>(g, c, s); }

}  // namespace sl
