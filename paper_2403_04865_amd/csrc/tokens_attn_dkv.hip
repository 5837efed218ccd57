// Attention over packed slides, backward: the gradients of keys and values (layout: tokens_attn.h).  Columns are keys; the queries of all heads
// that share them pass by, so the sum over a group's heads is part of the products.
#include "tokens_attn.h"

namespace sl {

namespace {

// Four products a score beside one root and one exponential: vector and matrix units are busy 43 and 36 % of the time (8193 rows, 6 heads of 64, with a
// bias: 290 us, 0.71 PFLOP/s), with two wavefronts a SIMD; a third has no registers.
template <typename T, int DP, int NW, bool BIAS, int CAP>
__global__ void __launch_bounds__(NW * 64, DP <= 64 && NW == 4 ? 2 : 1) tok_dkv_k(const TokAttn g) {
  constexpr int KB = TokType<T>::KB, LDR = tok_ldr<T, DP>(), NB = KB / 32, W = NW * 32;
  __shared__ __attribute__((aligned(16))) T Qs[KB * LDR], Os[KB * LDR];
  __shared__ __attribute__((aligned(16))) float px[KB], py[KB], ps[KB], pl[KB], pd[KB];
  const TokScore sc = tok_score_of<CAP>(g.scale, g.cap);
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const unsigned magic = tok_magic(g.group);
  tok_walk(tok_keys(g, W), tok_queries(g, KB, g.group), g.docs, g.hk, g.table, (TokJoin*)g.joins, [&](const TokSeg& w) __attribute__((always_inline)) {
    const int cols = w.r.n, nk = w.c.n, qlo = w.r.lo;
    const int j = w.tile * W + wave * 32 + (lane & 31);
    const bool valid = j < nk, idle = w.tile * W + wave * 32 >= nk;
    const long long krow = w.c.lo + (valid ? j : 0);
    TokFrag<T, DP> fk, fv;
    tok_load_frag<T, DP>(fk, (const T*)g.k + krow * g.ldk + w.head * g.dim, valid, g.dim);
    tok_load_frag<T, DP>(fv, (const T*)g.v + krow * g.ldv + w.head * g.dim, valid, g.dim);
    const bool placed = BIAS && valid && j >= g.lead_k;
    float kx = 0.f, ky = 0.f;
    if (placed) { kx = g.pos_k[2 * krow]; ky = g.pos_k[2 * krow + 1]; }
    const T* const qp = (const T*)g.q + (long long)qlo * g.ldq + w.head * g.group * g.dim;
    const T* const op = (const T*)g.dout + (long long)qlo * g.lddo + w.head * g.group * g.dim;
    TokTile<T, DP, NW * 64> qt(g.ldq, g.dim), ot(g.lddo, g.dim);
    // what belongs to a block's queries, loaded a block ahead like the tiles.  A query that is not there: probabilities of zero
    struct Row { float x, y, slope, lse, delta; };
    auto row_of = [&](int c0) __attribute__((always_inline)) {
      Row r = {0.f, 0.f, 0.f, INFINITY, 0.f};
      const int c = c0 + threadIdx.x;
      if (threadIdx.x < KB && c < cols) {
        const int qi = c / g.group, head = w.head * g.group + (c - qi * g.group);
        const long long row = qlo + qi;
        r.lse = g.lse[(long long)head * g.rows_q + row] * TOK_LOG2E;
        r.delta = -g.delta[(long long)head * g.rows_q + row];
        if (BIAS && qi >= g.lead_q) {
          const float2 p = *reinterpret_cast<const float2*>(g.pos_q + 2 * row);
          r.x = p.x; r.y = p.y;
          r.slope = g.slopes[head] * sc.per_slope;
        }
      }
      return r;
    };
    f32x16 dk[DP / 32], dv[DP / 32];
    tok_zero_all(dk);
    tok_zero_all(dv);
    // keys without a place are among the first tiles' only, whose loop is a copy of its own
    auto pass = [&](auto lead) __attribute__((always_inline)) {
      constexpr bool LEADS = decltype(lead)::value;
      qt.load_packed(qp, w.a * KB, cols, g.ldq, g.dim, g.group, magic);
      ot.load_packed(op, w.a * KB, cols, g.lddo, g.dim, g.group, magic);
      Row row = row_of(w.a * KB);
#pragma unroll 1
      for (int t = w.a; t < w.b; ++t) {
        const int c0 = t * KB;
        __syncthreads();
        qt.store(Qs);
        ot.store(Os);
        if (threadIdx.x < KB) {
          if (BIAS) { px[threadIdx.x] = row.x; py[threadIdx.x] = row.y; ps[threadIdx.x] = row.slope; }
          pl[threadIdx.x] = row.lse;
          pd[threadIdx.x] = row.delta;
        }
        __syncthreads();
        if (t + 1 < w.b) {
          qt.load_packed(qp, c0 + KB, cols, g.ldq, g.dim, g.group, magic);
          ot.load_packed(op, c0 + KB, cols, g.lddo, g.dim, g.group, magic);
          row = row_of(c0 + KB);
        }
        if (idle) continue;   // uniform in a wavefront: none of its columns is there
#pragma unroll
        for (int b = 0; b < NB; ++b) {
          f32x16 s = tok_zero(), dp, p, dist;
          if (BIAS) tok_dists<T>(dist, px, py, b * 32, kx, ky);
#pragma unroll
          for (int q4 = 0; q4 < 4; ++q4) {   // the product starts from -delta
            const f32x4 d = *reinterpret_cast<const f32x4*>(pd + b * 32 + tok_row(q4 * 4));
#pragma unroll
            for (int i = 0; i < 4; ++i) dp[q4 * 4 + i] = d[i];
          }
          TokRows<T, DP> qr, dr;
          TokCols<T, DP> qc, dc;
          tok_get<T, DP>(qr, Qs, b * 32);
          tok_get<T, DP>(dr, Os, b * 32);
          tok_mul<T, DP>(s, qr, fk);
          tok_mul<T, DP>(dp, dr, fv);
#pragma unroll
          for (int q4 = 0; q4 < 4; ++q4) {
            const int r0 = b * 32 + tok_row(q4 * 4);
            f32x4 slope;
            if (BIAS) slope = *reinterpret_cast<const f32x4*>(ps + r0);
            const f32x4 lse = *reinterpret_cast<const f32x4*>(pl + r0);
#pragma unroll
            for (int i = 0; i < 4; ++i) {
              const int r = q4 * 4 + i;
              float d = BIAS ? dist[r] : 0.f, dt = 1.f;
              if (LEADS && !placed) d = 0.f;
              const float z = tok_score<T, BIAS, CAP, true>(s[r], d, BIAS ? slope[i] : 0.f, sc, &dt);
              p[r] = tok_exp<CAP>(z, lse[i], sc);
              float ds = p[r] * dp[r];
              if (CAP) ds *= dt;
              s[r] = ds;
            }
          }
          tok_get_t(dc, Os, b * 32);
          tok_mul_t<DP, NW == 1>(dv, dc, p);
          tok_get_t(qc, Qs, b * 32);
          tok_mul_t<DP, NW == 1>(dk, qc, s);
        }
      }
    };
    if (cols > 0) {
      if constexpr (BIAS) {
        if (w.tile * W < g.lead_k) pass(std::true_type{});   // uniform
        else pass(std::false_type{});
      } else {
        pass(std::false_type{});
      }
    }
    if (!valid) return;
    const float f = CAP ? 4.f * g.scale : g.scale;   // scores' gradients carry a quarter of the cap's derivative
    if (w.slot >= 0) {
      const long long at = ((long long)w.slot * W + wave * 32 + (lane & 31)) * g.dim;
      tok_store(dk, f, g.part + at, g.dim);
      tok_store(dv, 1.f, g.part2 + at, g.dim);
    } else {
      tok_store(dk, f, (T*)g.dk + krow * g.lddk + w.head * g.dim, g.dim);
      tok_store(dv, 1.f, (T*)g.dv + krow * g.lddv + w.head * g.dim, g.dim);
    }
  });
}

template <typename T>
hipError_t run_dkv(const TokAttn& g, TokCut c, hipStream_t s) {
  return tok_dispatch<T>(g, [&](auto dp, auto bias, auto cap) {
    constexpr int DP = decltype(dp)::value;
    constexpr bool BIAS = decltype(bias)::value;
    constexpr int CAP = decltype(cap)::value;
    if (c.waves == 4) tok_dkv_k<T, DP, 4, BIAS, CAP><<<c.blocks, 256, 0, s>>>(g);
    else tok_dkv_k<T, DP, 1, BIAS, CAP><<<c.blocks, 64, 0, s>>>(g);
    return hipGetLastError();
  });
}

}  // namespace

hipError_t launch_tok_dkv(int dt, const TokAttn& g, TokCut c, hipStream_t s) { return dt == DT_F32 ? run_dkv<float>(g, c, s) : run_dkv<bf16>(g, c, s); }

}  // namespace sl
