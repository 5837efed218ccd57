// Attention over packed slides, forward: one pass over the keys with a running maximum and sum (layout: tokens_attn.h).
#include "tokens_attn.h"

namespace sl {

namespace {

// Bound by the vector unit where there is a bias or a cap: of the 14 issue slots' time of a score with a bias its distance takes 6.4 (four operations and a
// root), which two heads share where a wavefront has the registers (8193 rows, 12 heads of 64: 470 -> 426 us).
template <typename T, int DP, int NW, int NH, bool BIAS, int CAP>
__global__ void __launch_bounds__(NW * 64, (tok_waves<T, DP, NW>())) tok_fwd_k(const TokAttn g) {
  // differences of coordinates on the matrix cores (tok_dists) for one head and four wavefronts: 16 slides, capped scores, 8 heads of 128 156 -> 152 us; with two
  // heads, which share them, 383 -> 389, and with one wavefront, which waits for its loads, 38 -> 49
  constexpr bool DISTS = BIAS && NH == 1 && NW == 4 && sizeof(T) == 2;
  constexpr int KB = NH == 2 || DP == 128 ? 32 : TokType<T>::KB, LDR = tok_ldr<T, DP>(), NB = KB / 32, W = NW * 32;
  __shared__ __attribute__((aligned(16))) T Ks[NH][KB * LDR], Vs[NH][KB * LDR];
  __shared__ __attribute__((aligned(16))) float px[KB], py[KB];
  const TokScore sc = tok_score_of<CAP>(g.scale, g.cap);
  const TokHeads hs = tok_heads(g, NH);
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  tok_walk(tok_queries(g, W, hs.pack), tok_keys(g, KB), g.docs, hs.heads, g.table, (TokJoin*)g.joins, [&](const TokSeg& w) __attribute__((always_inline)) {
    const int cols = w.c.n, nk = w.r.n, klo = w.r.lo;
    const int c = w.tile * W + wave * 32 + (lane & 31);
    const bool valid = c < cols, idle = w.tile * W + wave * 32 >= cols;
    const int kv = NH == 1 ? w.head : w.head * (hs.kv_step + 1);   // the group's first key head
    const int qi = valid ? c / hs.pack : 0, head = kv * g.group + (valid ? c - qi * hs.pack : 0);
    const long long qrow = w.c.lo + qi;
    TokFrag<T, DP> fq[NH];
    float qx = 0.f, qy = 0.f, slope[NH];
#pragma unroll
    for (int n = 0; n < NH; ++n) {
      tok_load_frag<T, DP>(fq[n], (const T*)g.q + qrow * g.ldq + (head + n * hs.step) * g.dim, valid, g.dim);
      slope[n] = BIAS && valid && qi >= g.lead_q ? g.slopes[head + n * hs.step] * sc.per_slope : 0.f;
    }
    if (BIAS && valid && qi >= g.lead_q) { qx = g.pos_q[2 * qrow]; qy = g.pos_q[2 * qrow + 1]; }
    const T* const kp = (const T*)g.k + (long long)klo * g.ldk + kv * g.dim;
    const T* const vp = (const T*)g.v + (long long)klo * g.ldv + kv * g.dim;
    const int apart = hs.kv_step * g.dim;   // 0: both heads read the first's
    TokTile<T, DP, NW * 64, KB> kt[NH] = {TokTile<T, DP, NW * 64, KB>(g.ldk, g.dim)}, vt[NH] = {TokTile<T, DP, NW * 64, KB>(g.ldv, g.dim)};
    TokPlace place = {0.f, 0.f};
    f32x16 o[NH][DP / 32];
    float top[NH], l[NH];   // what exponents are taken relative to, and their sum
#pragma unroll
    for (int n = 0; n < NH; ++n) {
      tok_zero_all(o[n]);
      top[n] = TOK_NONE;
      l[n] = 0.f;
    }
    auto fetch = [&](int k0) __attribute__((always_inline)) {
      kt[0].load(kp + (long long)k0 * g.ldk, nk - k0, g.ldk, g.dim);
      vt[0].load(vp + (long long)k0 * g.ldv, nk - k0, g.ldv, g.dim);
      if (NH == 2 && apart) {   // uniform
        kt[NH - 1].load_as(kt[0], kp + (long long)k0 * g.ldk + apart, nk - k0, g.ldk, g.dim);
        vt[NH - 1].load_as(vt[0], vp + (long long)k0 * g.ldv + apart, nk - k0, g.ldv, g.dim);
      }
      if (BIAS) place = tok_place<KB>(g.pos_k, klo, k0, nk, g.lead_k);
    };
    if (nk > 0) {
      fetch(w.a * KB);
#pragma unroll 1
      for (int t = w.a; t < w.b; ++t) {
        const int k0 = t * KB;
        __syncthreads();
        kt[0].store(Ks[0]);
        vt[0].store(Vs[0]);
        if (NH == 2 && apart) {
          kt[NH - 1].store(Ks[NH - 1]);
          vt[NH - 1].store(Vs[NH - 1]);
        }
        if (BIAS && threadIdx.x < KB) { px[threadIdx.x] = place.x; py[threadIdx.x] = place.y; }
        __syncthreads();
        if (t + 1 < w.b) fetch(k0 + KB);
        if (idle) continue;   // uniform in a wavefront: none of its columns is there
        const int second = NH == 2 && apart ? 1 : 0;
        f32x16 s[NH][NB];
#pragma unroll
        for (int n = 0; n < NH; ++n)
#pragma unroll
          for (int b = 0; b < NB; ++b) {
            TokRows<T, DP> kr;
            tok_get<T, DP>(kr, Ks[n * second], b * 32);
            s[n][b] = tok_zero();
            tok_mul<T, DP>(s[n][b], kr, fq[n]);
          }
        f32x16 dist[NB];
        if (DISTS) {
#pragma unroll
          for (int b = 0; b < NB; ++b) tok_dists<T>(dist[b], px, py, b * 32, qx, qy);
        }
        float mn[NH];
#pragma unroll
        for (int n = 0; n < NH; ++n) mn[n] = -INFINITY;
        // the first and the last blocks hold keys without a place and keys that are not there: a copy of the code of their own
        auto scores = [&](auto edge) __attribute__((always_inline)) {
          constexpr bool EDGE = decltype(edge)::value;
#pragma unroll
          for (int b = 0; b < NB; ++b)
#pragma unroll
            for (int q4 = 0; q4 < 4; ++q4) {
              const int r0 = b * 32 + tok_row(q4 * 4);
              f32x4 kx, ky;
              if (BIAS && !DISTS) {
                kx = *reinterpret_cast<const f32x4*>(px + r0);
                ky = *reinterpret_cast<const f32x4*>(py + r0);
              }
#pragma unroll
              for (int i = 0; i < 4; ++i) {
                float d = DISTS ? dist[b][q4 * 4 + i] : BIAS ? tok_dist(qx, qy, kx[i], ky[i]) : 0.f;
                if (EDGE && BIAS && k0 + r0 + i < g.lead_k) d = 0.f;
#pragma unroll
                for (int n = 0; n < NH; ++n) {
                  float z = tok_score<T, BIAS, CAP, false>(s[n][b][q4 * 4 + i], d, slope[n], sc, nullptr);
                  if (EDGE && k0 + r0 + i >= nk) z = -INFINITY;
                  s[n][b][q4 * 4 + i] = z;
                  mn[n] = fmaxf(mn[n], z);
                }
              }
            }
        };
        if ((BIAS && k0 < g.lead_k) || k0 + KB > nk) scores(std::true_type{});   // uniform
        else scores(std::false_type{});
#pragma unroll
        for (int n = 0; n < NH; ++n) {
          // The reference is a maximum of before and moves when a score is 2^8 above it: sums keep their relative precision either way.  A branch for the
          // lanes, not for the wavefront: behind a uniform one the compiler keeps the sums in two places and copies them every time.
          const float mx = tok_other_max(mn[n]) * sc.ex;
          if (mx > top[n] + 8.f) {
            const float resc = __builtin_amdgcn_exp2f(top[n] - mx);   // 0 at the first block
            top[n] = mx;
            l[n] *= resc;
#pragma unroll
            for (int d = 0; d < DP / 32; ++d)
#pragma unroll
              for (int r = 0; r < 16; ++r) o[n][d][r] *= resc;
          }
#pragma unroll
          for (int b = 0; b < NB; ++b)
#pragma unroll
            for (int r = 0; r < 16; ++r) {
              s[n][b][r] = tok_exp<CAP>(s[n][b][r], top[n], sc);
              l[n] += s[n][b][r];
            }
#pragma unroll
          for (int b = 0; b < NB; ++b) {
            TokCols<T, DP> vc;
            tok_get_t(vc, Vs[n * second], b * 32);
            tok_mul_t<DP, NW == 1>(o[n], vc, s[n][b]);
          }
        }
      }
    }
#pragma unroll
    for (int n = 0; n < NH; ++n) {
      l[n] = tok_other_sum(l[n]);
      if (!valid) continue;
      const int h = head + n * hs.step;
      if (w.slot >= 0) {
        const long long at = ((long long)w.slot * NH + n) * W + wave * 32 + (lane & 31);
        if (lane < 32) *reinterpret_cast<float2*>(g.part2 + 2 * at) = float2{top[n], l[n]};
        tok_store(o[n], 1.f, g.part + at * g.dim, g.dim);
        continue;
      }
      const bool nothing = l[n] == 0.f;   // no keys, or none within reach of a bias that is infinite
      tok_store(o[n], nothing ? 0.f : 1.f / l[n], (T*)g.o + qrow * g.ldo + h * g.dim, g.dim);
      if (lane < 32) g.lse[(long long)h * g.rows_q + qrow] = nothing ? -INFINITY : (top[n] + __builtin_amdgcn_logf(l[n])) * TOK_LN2;
    }
  });
}

template <typename T>
hipError_t run_fwd(const TokAttn& g, TokCut c, hipStream_t s) {
  return tok_dispatch<T>(g, [&](auto dp, auto bias, auto cap) {
    constexpr int DP = decltype(dp)::value;
    constexpr bool BIAS = decltype(bias)::value;
    constexpr int CAP = decltype(cap)::value;
    if constexpr (tok_pairs<T, DP, BIAS>()) {
      if (c.heads == 2) {
        tok_fwd_k<T, DP, 4, 2, BIAS, CAP><<<c.blocks, 256, 0, s>>>(g);
        return hipGetLastError();
      }
    }
    if (c.waves == 4) tok_fwd_k<T, DP, 4, 1, BIAS, CAP><<<c.blocks, 256, 0, s>>>(g);
    else tok_fwd_k<T, DP, 1, 1, BIAS, CAP><<<c.blocks, 64, 0, s>>>(g);
    return hipGetLastError();
  });
}

}  // namespace

hipError_t launch_tok_fwd(int dt, const TokAttn& g, TokCut c, hipStream_t s) { return dt == DT_F32 ? run_fwd<float>(g, c, s) : run_fwd<bf16>(g, c, s); }

}  // namespace sl
