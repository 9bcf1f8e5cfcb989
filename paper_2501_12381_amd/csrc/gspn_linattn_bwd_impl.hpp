// Linear attention, backward: one workgroup walks one piece of one head from its
// last chunk to its first, with the gradient dM of the state behind the chunk in
// registers, and reads the state S before each chunk (linattn_state_kernel, mode 1):
//
//   Z_ts = scale e^{G_t-G_s} (do_t.v_s),  P_ts = scale e^{G_t-G_s} (q_t.k_s),  s <= t
//   dq_t = sum_s Z_ts k_s + scale e^{G_t} S do_t
//   dk_s = sum_t Z_ts q_t + e^{G_C-G_s} dM v_s
//   dv_s = sum_t P_ts do_t + e^{G_C-G_s} dM^T k_s
//   dM  <- e^{G_C} dM + sum_t scale e^{G_t} q_t do_t^T
//   da_r = sum_{s<r<=t} W_ts + sum_{t>=r} u_t + sum_{s<r} w_s + e^{G_C} <S, dM>
//     W_ts = P_ts (do_t.v_s), u_t = q_t . (second term of dq_t), w_s = k_s . (second term of dk_s)
//
// The decay's gradient is formed from the pairs that a token's decay lies
// between, chunk by chunk; the shorter formula, q.dq - k.dk summed from the end,
// adds up the rounding of every later token.
//
// Two kinds of waves: VP/32 own 32 columns of v each (P, dv, dM), KP/32 own 32
// columns of k each (Z, dq, dk, W).  P, Z and dM (rounded to the element type) pass
// through LDS.  What bounds it: bytes (q, k, v, do and a state in, dq, dk, dv out),
// then the LDS reads of the operands.
#pragma once

#include "gspn_linattn_fwd_impl.hpp"

namespace gspn {
namespace la {

template <typename T, int KP, int VP> struct BwdLds {
  static constexpr int C = Elem<T>::kChunk, kPad = Elem<T>::kPad;
  static constexpr int KS = KP + kPad, VS = VP + kPad, PS = C + kPad, MS = KP + kPad, NB = KP / 32;
  __align__(16) T q[C * KS], k[C * KS], v[C * VS], g[C * VS], p[C * PS], z[C * PS];
  __align__(16) T m[VP * MS];  // dM^T: [column of v][column of k]
  Decays<C> dec;
  float u[NB][C], w[NB][C];    // per wave's columns of k
  float row[2][C], col[2][C];  // sums of W: row[s tile][t], col[t tile][s]
  float x[NB];
};

// sum over the 32 lanes of a half, in every lane
__device__ __forceinline__ float half_sum(float v) {
#pragma unroll
  for (int k = 1; k < 32; k <<= 1) v += __shfl_xor(v, k);
  return v;
}

template <typename T, int KP, int VP>
__global__ void __launch_bounds__(2 * (KP + VP)) linattn_bwd_kernel(BwdArgs A) {
  using E = Elem<T>;
  using Lds = BwdLds<T, KP, VP>;
  constexpr int C = E::kChunk, NC = C / 32, kTiles = NC * (NC + 1) / 2;
  constexpr int NA = VP / 32, NB = KP / 32, NT = 64 * (NA + NB);
  constexpr int KS = Lds::KS, VS = Lds::VS, PS = Lds::PS, MS = Lds::MS;
  extern __shared__ __align__(16) unsigned char lds_raw[];
  Lds& s = *reinterpret_cast<Lds*>(lds_raw);

  const Geom& g = A.g;
  const int tid = threadIdx.x, wave = tid >> 6, lane = tid & 63, h = lane >> 5, l = lane & 31;
  const int head = blockIdx.x % g.H, pi = blockIdx.x / g.H;
  const Piece pc = find_piece(g, pi);
  const int64_t slot = (int64_t)pi * g.H + head;
  if (pc.len < 0 || pc.seq >= g.N) {
    if (!A.per_token && tid == 0) A.da_piece[slot] = 0.f;
    if (pc.len <= 0) return;
  }
  const int64_t row0 = pc.batch * g.T + pc.t0, kt = (int64_t)g.H * g.Dk, vt = (int64_t)g.H * g.Dv;
  T *dq = reinterpret_cast<T*>(A.dq) + row0 * kt + head * g.Dk, *dk = reinterpret_cast<T*>(A.dk) + row0 * kt + head * g.Dk;
  float *dq32 = A.dq32 ? A.dq32 + row0 * kt + head * g.Dk : nullptr,
        *dk32 = A.dk32 ? A.dk32 + row0 * kt + head * g.Dk : nullptr;
  T* dv = reinterpret_cast<T*>(A.dv) + row0 * vt + head * g.Dv;
  T* da = reinterpret_cast<T*>(A.da) + row0 * g.H + head;
  if (pc.seq >= g.N) {  // tokens of no sequence
    for (int i = tid; i < pc.len * g.Dk; i += NT) {
      const int64_t at = (i / g.Dk) * kt + i % g.Dk;
      if (dq32) dq32[at] = dk32[at] = 0.f;
      else dq[at] = dk[at] = from_f<T>(0.f);
    }
    for (int i = tid; i < pc.len * g.Dv; i += NT) dv[(i / g.Dv) * vt + i % g.Dv] = from_f<T>(0.f);
    if (A.per_token)
      for (int i = tid; i < pc.len; i += NT) da[(int64_t)i * g.H] = from_f<T>(0.f);
    return;
  }
  const int hk = head / (g.H / g.Hk);
  const bool va = wave < NA;               // this wave owns columns of v (else of k)
  const int c0 = 32 * (va ? wave : wave - NA), wb = wave - NA;
  const int64_t sidx = ((int64_t)pc.seq * g.H + head) * g.Dk * g.Dv;
  const T *q = head_rows<T>(A.q, pc, hk), *k = head_rows<T>(A.k, pc, hk), *v = head_rows<T>(A.v, pc, head),
          *dout = head_rows<T>(A.dout, pc, head);
  const T* a = reinterpret_cast<const T*>(A.a) + head + (A.per_token ? row0 * g.H : (int64_t)0);
  const int64_t at = A.per_token ? g.H : 0;

  Stage<T, KP, NT> rq, rk;
  Stage<T, VP, NT> rv, rg;
  double ra = 0.0;
  const auto load = [&](int t) {
    const int rows = pc.len - t;
    rq.load(q + t * A.q.st, A.q.st, rows, g.Dk, A.q.vec, tid);
    rk.load(k + t * A.k.st, A.k.st, rows, g.Dk, A.k.vec, tid);
    rv.load(v + t * A.v.st, A.v.st, rows, g.Dv, A.v.vec, tid);
    rg.load(dout + t * A.dout.st, A.dout.st, rows, g.Dv, A.dout.vec, tid);
    if (wave == 0 && lane < C) ra = load_decay(a + t * at, at, lane, rows);
  };
  const int n = (pc.len + C - 1) / C;
  const auto stage = [&] {
    rq.store(s.q, tid);
    rk.store(s.k, tid);
    rv.store(s.v, tid);
    rg.store(s.g, tid);
    if (wave == 0) chunk_decays(s.dec, ra, A.scale, lane);
  };
  if (n > 0) load((n - 1) * C);
  // the two kinds of waves run loops of their own (the registers of the one are
  // then not kept through the other's code), with the same barriers
  if (va) {
    f32x16 M[KP / 32];
    if (pc.last) state_read<KP>(M, A.dsf ? A.dsf + sidx : nullptr, g.Dk, g.Dv, g.Dv, 1, c0 + l, h);
    else state_read_regs<KP>(M, A.end + slot * (KP * VP), wave, lane);
    float da_sum = 0.f;  // wave 0, with one decay for the head
    for (int c = n - 1; c >= 0; --c) {
      const int t0 = c * C;
      stage();
#pragma unroll
      for (int m = 0; m < KP / 32; ++m)
#pragma unroll
        for (int r = 0; r < 16; r += 4) {
          float x[4] = {M[m][r], M[m][r + 1], M[m][r + 2], M[m][r + 3]};
          E::store4(s.m + (c0 + l) * MS + 32 * m + acc_row(r, h), x);
        }
      lds_barrier();
      if (c > 0) load(t0 - C);
      // P[t][s]
      for (int tile = wave; tile < kTiles; tile += NA) {
        int st, tt;
        pair_of(tile, st, tt);
        const f32x16 raw = pair_tile<T, KP>(s.k, s.q, KS, st, tt, lane);
        const int t = 32 * tt + l;
        const float hi = s.dec.hi[t], lo = s.dec.lo[t];
#pragma unroll
        for (int r = 0; r < 16; r += 4) {
          const int ss = 32 * st + acc_row(r, h);
          float x[4];
#pragma unroll
          for (int j = 0; j < 4; ++j)
            x[j] = ss + j <= t ? raw[r + j] * (A.scale * decay_between(s.dec, ss + j, hi, lo)) : 0.f;
          E::store4(s.p + t * PS + ss, x);
        }
      }
      // dv^T = dM^T k^T e^{G_C - G_s}
      f32x16 acc[NC];
#pragma unroll
      for (int ts = 0; ts < NC; ++ts) acc[ts] = f32x16{};
#pragma unroll
      for (int kk = 0; kk < KP / 16; ++kk) {
        const auto mf = acc_frag<T>(M[kk >> 1], kk & 1);
#pragma unroll
        for (int ts = 0; ts < NC; ++ts) E::mma(acc[ts], mf, row_frag_acc(s.k, KS, 32 * ts + l, 16 * kk, h));
      }
#pragma unroll
      for (int ts = 0; ts < NC; ++ts) acc[ts] *= s.dec.kf[32 * ts + l];
      lds_barrier();
      // + do^T P
#pragma unroll
      for (int k0 = 0; k0 < C; k0 += 16) {
        const auto gf = col_frag(s.g, VS, k0, c0, lane);
#pragma unroll
        for (int ts = 0; ts <= k0 / 32; ++ts) E::mma(acc[ts], gf, col_frag(s.p, PS, k0, 32 * ts, lane));
      }
#pragma unroll
      for (int ts = 0; ts < NC; ++ts) {
        const int t = t0 + 32 * ts + l;
        if (t < pc.len) {
#pragma unroll
          for (int r = 0; r < 16; r += 4) {
            const int cc = c0 + acc_row(r, h);
            float x[4] = {acc[ts][r], acc[ts][r + 1], acc[ts][r + 2], acc[ts][r + 3]};
            put4(dv + t * vt + cc, x, g.Dv - cc, A.dvvec);
          }
        }
      }
      state_add<T, KP>(M, s.q, KS, s.g, VS, c0, s.dec.qf, s.dec.tot, lane);
      lds_barrier();
      if (wave == 0) {
        // da_r: suffix sums of row - col + u, prefix sums of w, and the product of the two states
        float f = 0.f, w = 0.f, x = 0.f;
#pragma unroll
        for (int b = 0; b < NB; ++b) x += s.x[b];
        if (lane < C) {
#pragma unroll
          for (int b = 0; b < NB; ++b) {
            f += s.u[b][lane];
            w += s.w[b][lane];
          }
          float d = s.row[0][lane] - s.col[NC - 1][lane];
          if (NC == 2) d += lane < 32 ? -s.col[0][lane] : s.row[1][lane];
          f += d;
        }
        const float own = w;
#pragma unroll
        for (int i = 1; i < 64; i <<= 1) {
          const float fo = __shfl_down(f, i), wo = __shfl_up(w, i);
          if (lane + i < 64) f += fo;
          if (lane >= i) w += wo;
        }
        const float r = f + (w - own) + s.dec.tot * x;
        if (lane < C && t0 + lane < pc.len) {
          if (A.per_token) da[(int64_t)(t0 + lane) * g.H] = from_f<T>(r);
          else da_sum += r;
        }
      }
    }
    if (pc.first && A.ds0) state_write<KP>(M, A.ds0 + sidx, g.Dk, g.Dv, g.Dv, 1, c0 + l, h);
    if (!A.per_token && wave == 0) {
      da_sum = half_sum(da_sum);
      da_sum += __shfl_xor(da_sum, 32);
      if (lane == 0) A.da_piece[slot] = da_sum;
    }
  } else {
    for (int c = n - 1; c >= 0; --c) {
      const int t0 = c * C;
      stage();
      lds_barrier();
      if (c > 0) load(t0 - C);
      // do.v of this wave's pairs, and Z[t][s]
      constexpr int kMine = (kTiles + NB - 1) / NB;
      f32x16 raw[kMine];
#pragma unroll
      for (int i = 0; i < kMine; ++i) {
        const int tile = wb + i * NB;
        if (tile >= kTiles) continue;
        int st, tt;
        pair_of(tile, st, tt);
        raw[i] = pair_tile<T, VP>(s.v, s.g, VS, st, tt, lane);
        const int t = 32 * tt + l;
        const float hi = s.dec.hi[t], lo = s.dec.lo[t];
#pragma unroll
        for (int r = 0; r < 16; r += 4) {
          const int ss = 32 * st + acc_row(r, h);
          float x[4];
#pragma unroll
          for (int j = 0; j < 4; ++j)
            x[j] = ss + j <= t ? raw[i][r + j] * (A.scale * decay_between(s.dec, ss + j, hi, lo)) : 0.f;
          E::store4(s.z + t * PS + ss, x);
        }
      }
      // the terms through the states: dq^T = S do^T scale e^{G_t}, dk^T = dM v^T e^{G_C - G_s}
      f32x16 aq[NC], ak[NC];
#pragma unroll
      for (int i = 0; i < NC; ++i) aq[i] = ak[i] = f32x16{};
      const T* chunk = reinterpret_cast<const T*>(A.chunks) +
                       (((int64_t)pi * (g.L / C) + c) * g.H + head) * (KP * VP) + (wb * (VP / 16) * 64 + lane) * 8;
      float dot = 0.f;
#pragma unroll
      for (int kk = 0; kk < VP / 16; ++kk) {
        const auto sf = *reinterpret_cast<const typename E::Frag*>(chunk + kk * 512);
        const auto mf = col_frag_acc(s.m, MS, 16 * kk, c0, lane);
        float x[8], y[8];
        E::get(sf, x);
        E::get(mf, y);
#pragma unroll
        for (int j = 0; j < 8; ++j) dot = __builtin_fmaf(x[j], y[j], dot);
#pragma unroll
        for (int i = 0; i < NC; ++i) {
          E::mma(aq[i], sf, row_frag_acc(s.g, VS, 32 * i + l, 16 * kk, h));
          E::mma(ak[i], mf, row_frag_acc(s.v, VS, 32 * i + l, 16 * kk, h));
        }
      }
      dot = half_sum(dot);
      dot += __shfl_xor(dot, 32);
      if (lane == 0) s.x[wb] = dot;
#pragma unroll
      for (int i = 0; i < NC; ++i) {
        const int t = 32 * i + l;
        aq[i] *= s.dec.qf[t];
        ak[i] *= s.dec.kf[t];
        float u = 0.f, w = 0.f;
#pragma unroll
        for (int r = 0; r < 16; r += 4) {
          float x[4], y[4];
          E::load4(s.q + t * KS + c0 + acc_row(r, h), x);
          E::load4(s.k + t * KS + c0 + acc_row(r, h), y);
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            u = __builtin_fmaf(x[j], aq[i][r + j], u);
            w = __builtin_fmaf(y[j], ak[i][r + j], w);
          }
        }
        u += __shfl_xor(u, 32);
        w += __shfl_xor(w, 32);
        if (h == 0) {
          s.u[wb][t] = u;
          s.w[wb][t] = w;
        }
      }
      lds_barrier();
      // W = P (do.v): sums over s and over t
#pragma unroll
      for (int i = 0; i < kMine; ++i) {
        const int tile = wb + i * NB;
        if (tile >= kTiles) continue;
        int st, tt;
        pair_of(tile, st, tt);
        const int t = 32 * tt + l;
        float rs = 0.f;
#pragma unroll
        for (int r = 0; r < 16; r += 4) {
          const int ss = 32 * st + acc_row(r, h);
          float x[4];
          E::load4(s.p + t * PS + ss, x);
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            const float wv = x[j] * raw[i][r + j];
            rs += wv;
            const float cs = half_sum(wv);
            if (l == 0) s.col[tt][ss + j] = cs;
          }
        }
        rs += __shfl_xor(rs, 32);
        if (h == 0) s.row[st][t] = rs;
      }
      // + k^T Z^T, + q^T Z
#pragma unroll
      for (int k0 = 0; k0 < C; k0 += 16) {
        const auto kf = col_frag(s.k, KS, k0, c0, lane), qf = col_frag(s.q, KS, k0, c0, lane);
#pragma unroll
        for (int i = 0; i < NC; ++i) {
          if (i >= k0 / 32) E::mma(aq[i], kf, row_frag(s.z, PS, 32 * i + l, k0, h));
          if (i <= k0 / 32) E::mma(ak[i], qf, col_frag(s.z, PS, k0, 32 * i, lane));
        }
      }
#pragma unroll
      for (int i = 0; i < NC; ++i) {
        const int t = t0 + 32 * i + l;
        if (t < pc.len) {
#pragma unroll
          for (int r = 0; r < 16; r += 4) {
            const int cc = c0 + acc_row(r, h);
            float x[4] = {aq[i][r], aq[i][r + 1], aq[i][r + 2], aq[i][r + 3]};
            float y[4] = {ak[i][r], ak[i][r + 1], ak[i][r + 2], ak[i][r + 3]};
            if (dq32) {
              put4(dq32 + t * kt + cc, x, g.Dk - cc, A.dkvec);
              put4(dk32 + t * kt + cc, y, g.Dk - cc, A.dkvec);
            } else {
              put4(dq + t * kt + cc, x, g.Dk - cc, A.dkvec);
              put4(dk + t * kt + cc, y, g.Dk - cc, A.dkvec);
            }
          }
        }
      }
      lds_barrier();
    }
  }
}

template <typename T, int KP, int VP> hipError_t linattn_bwd_launch(const BwdArgs& a) {
  constexpr int bytes = sizeof(BwdLds<T, KP, VP>);
  static_assert(bytes <= 160 * 1024, "");
  const hipError_t e = hipFuncSetAttribute(reinterpret_cast<const void*>(&linattn_bwd_kernel<T, KP, VP>),
                                           hipFuncAttributeMaxDynamicSharedMemorySize, bytes);
  if (e != hipSuccess) return e;
  hipLaunchKernelGGL((linattn_bwd_kernel<T, KP, VP>), dim3((unsigned)((int64_t)a.g.pieces * a.g.H)),
                     dim3(2 * (KP + VP)), bytes, (hipStream_t)a.stream, a);
  return hipGetLastError();
}

template <typename T> hipError_t linattn_bwd_t(const BwdArgs& a) {
  const bool kw = a.g.Dk > 64, vw = a.g.Dv > 64;
  if (kw && vw) return linattn_bwd_launch<T, 128, 128>(a);
  if (kw) return linattn_bwd_launch<T, 128, 64>(a);
  if (vw) return linattn_bwd_launch<T, 64, 128>(a);
  return linattn_bwd_launch<T, 64, 64>(a);
}

}  // namespace la
}  // namespace gspn
