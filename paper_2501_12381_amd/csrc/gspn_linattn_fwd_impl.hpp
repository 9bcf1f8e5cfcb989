// Linear attention, forward: one workgroup walks one piece of one head.
//
// What bounds it: the bytes of q, k, v and o (each is moved once; a chunk of 64
// tokens of 128 values takes 64 KB and about 300 matrix instructions on each of the
// four SIMDs' waves, a third of the time its bytes need at the card's rate).
// Split: wave w owns columns 32w..32w+31 of v, o and the state, so the state
// never leaves its registers: a 32 x 32 result tile is, register for register,
// an operand of the next product (row_frag_acc gives the other operand the same
// depth order).  Only the C x C products q.k are shared, through LDS.
#pragma once

#include "gspn_linattn_common.hpp"

namespace gspn {
namespace la {

// raw[s][t] tile (s tile st, t tile tt): sum over the depth of a_s . b_t
template <typename T, int DP>
__device__ __forceinline__ f32x16 pair_tile(const T* a, const T* b, int stride, int st, int tt, int lane) {
  const int h = lane >> 5, l = lane & 31;
  f32x16 acc = {};
#pragma unroll
  for (int k0 = 0; k0 < DP; k0 += 16)
    Elem<T>::mma(acc, row_frag(a, stride, 32 * st + l, k0, h), row_frag(b, stride, 32 * tt + l, k0, h));
  return acc;
}

// index of the tile'th pair of 32-token tiles with s <= t
__device__ __forceinline__ void pair_of(int tile, int& st, int& tt) {
  tt = (tile + 1) >> 1;   // 0: (0, 0), 1: (0, 1), 2: (1, 1)
  st = tile >> 1;
}

// state += sum_t x_t (f_t y_t)^T over a chunk: x's rows (tiles of 32 along XP)
// against this wave's 32 columns of y, whose values are scaled in fp32 and given
// to the product in parts that keep their 24 bits (a single bf16 rounding would
// cost the fp32 state its precision)
template <typename T, int XP>
__device__ __forceinline__ void state_add(f32x16* S, const T* x, int xstride, const T* y, int ystride, int ycol,
                                          const float* f, float tot, int lane) {
  constexpr int C = Elem<T>::kChunk, NP = Elem<T>::kParts;
  const int h = lane >> 5;
#pragma unroll
  for (int m = 0; m < XP / 32; ++m) S[m] *= tot;
#pragma unroll
  for (int k0 = 0; k0 < C; k0 += 16) {
    float v[8];
    Elem<T>::get(col_frag(y, ystride, k0, ycol, lane), v);
#pragma unroll
    for (int j = 0; j < 8; ++j) v[j] *= f[k0 + 8 * h + j];
    typename Elem<T>::Frag p[NP];
    Elem<T>::split(v, p);
#pragma unroll
    for (int m = 0; m < XP / 32; ++m) {
      const auto xf = col_frag(x, xstride, k0, 32 * m, lane);
#pragma unroll
      for (int i = NP - 1; i >= 0; --i) Elem<T>::mma(S[m], xf, p[i]);
    }
  }
}

// S from / to (x, y)-strided fp32 memory, or zero
template <int XP>
__device__ __forceinline__ void state_read(f32x16* S, const float* s, int Dx, int Dy, int sx, int sy, int y, int h) {
#pragma unroll
  for (int m = 0; m < XP / 32; ++m)
#pragma unroll
    for (int r = 0; r < 16; ++r) {
      const int x = 32 * m + acc_row(r, h);
      S[m][r] = s && x < Dx && y < Dy ? s[x * sx + y * sy] : 0.f;
    }
}
template <int XP>
__device__ __forceinline__ void state_write(const f32x16* S, float* s, int Dx, int Dy, int sx, int sy, int y, int h) {
#pragma unroll
  for (int m = 0; m < XP / 32; ++m)
#pragma unroll
    for (int r = 0; r < 16; ++r) {
      const int x = 32 * m + acc_row(r, h);
      if (x < Dx && y < Dy) s[x * sx + y * sy] = S[m][r];
    }
}
// register order: register after register, 64 lanes each
template <int XP> __device__ __forceinline__ void state_read_regs(f32x16* S, const float* s, int wave, int lane) {
#pragma unroll
  for (int m = 0; m < XP / 32; ++m)
#pragma unroll
    for (int r = 0; r < 16; ++r) S[m][r] = s[((wave * (XP / 32) + m) * 16 + r) * 64 + lane];
}
template <int XP> __device__ __forceinline__ void state_write_regs(const f32x16* S, float* s, int wave, int lane) {
#pragma unroll
  for (int m = 0; m < XP / 32; ++m)
#pragma unroll
    for (int r = 0; r < 16; ++r) s[((wave * (XP / 32) + m) * 16 + r) * 64 + lane] = S[m][r];
}

template <typename T> __device__ __forceinline__ const T* head_rows(const Rows& r, const Piece& pc, int head) {
  return reinterpret_cast<const T*>(r.p) + pc.batch * r.sb + (int64_t)pc.t0 * r.st + (int64_t)head * r.sh;
}

// the first `left` of four values of a row; vec: `left` is 4 or nothing, p is aligned to the four
template <typename T> __device__ __forceinline__ void put4(T* p, const float* x, int left, int vec) {
  if (vec) {
    if (left > 0) Elem<T>::store4(p, x);
  } else {
#pragma unroll
    for (int j = 0; j < 4; ++j)
      if (j < left) p[j] = from_f<T>(x[j]);
  }
}

template <typename T, int KP, int VP> __global__ void __launch_bounds__(2 * VP, 2) linattn_fwd_kernel(FwdArgs A) {
  constexpr int C = Elem<T>::kChunk, NT = 2 * VP, NW = VP / 32, PS = C + Elem<T>::kPad;
  constexpr int KS = KP + Elem<T>::kPad, VS = VP + Elem<T>::kPad;
  constexpr int NC = C / 32, kTiles = NC * (NC + 1) / 2;
  __shared__ __align__(16) T sq[C * KS], sk[C * KS], sv[C * VS], sp[C * PS];
  __shared__ Decays<C> dec;

  const Geom& g = A.g;
  const int tid = threadIdx.x, wave = tid >> 6, lane = tid & 63, h = lane >> 5, l = lane & 31;
  const int head = blockIdx.x % g.H, pi = blockIdx.x / g.H;
  const Piece pc = find_piece(g, pi);
  if (pc.len < 0) return;
  T* o = reinterpret_cast<T*>(A.o) + ((pc.batch * g.T + pc.t0) * g.H + head) * (int64_t)g.Dv;
  const int64_t ot = (int64_t)g.H * g.Dv;
  if (pc.seq >= g.N) {  // tokens of no sequence
    for (int i = tid; i < pc.len * g.Dv; i += NT) o[(i / g.Dv) * ot + i % g.Dv] = from_f<T>(0.f);
    return;
  }
  const int hk = head / (g.H / g.Hk), y = 32 * wave + l;
  f32x16 S[KP / 32];
  const int64_t sidx = ((int64_t)pc.seq * g.H + head) * g.Dk * g.Dv;
  if (pc.first) state_read<KP>(S, A.s0 ? A.s0 + sidx : nullptr, g.Dk, g.Dv, g.Dv, 1, y, h);
  else state_read_regs<KP>(S, A.start + ((int64_t)pi * g.H + head) * (KP * VP), wave, lane);

  const T *q = head_rows<T>(A.q, pc, hk), *k = head_rows<T>(A.k, pc, hk), *v = head_rows<T>(A.v, pc, head);
  const T* a = reinterpret_cast<const T*>(A.a) + head +
               (A.per_token ? (pc.batch * g.T + pc.t0) * (int64_t)g.H : (int64_t)0);
  const int64_t at = A.per_token ? g.H : 0;

  Stage<T, KP, NT> rq, rk;
  Stage<T, VP, NT> rv;
  double ra = 0.0;
  const auto load = [&](int t) {
    const int rows = pc.len - t;
    rq.load(q + t * A.q.st, A.q.st, rows, g.Dk, A.q.vec, tid);
    rk.load(k + t * A.k.st, A.k.st, rows, g.Dk, A.k.vec, tid);
    rv.load(v + t * A.v.st, A.v.st, rows, g.Dv, A.v.vec, tid);
    if (wave == 0 && lane < C) ra = load_decay(a + t * at, at, lane, rows);
  };
  if (pc.len > 0) load(0);
  for (int t0 = 0; t0 < pc.len; t0 += C) {
    rq.store(sq, tid);
    rk.store(sk, tid);
    rv.store(sv, tid);
    if (wave == 0) chunk_decays(dec, ra, A.scale, lane);
    lds_barrier();
    if (t0 + C < pc.len) load(t0 + C);

    // (q.k) decay, transposed: lane = t, registers = s, so that four
    // neighbouring s are one store of P[t][s]
    for (int tile = wave; tile < kTiles; tile += NW) {
      int st, tt;
      pair_of(tile, st, tt);
      const f32x16 raw = pair_tile<T, KP>(sk, sq, KS, st, tt, lane);
      const int t = 32 * tt + l;
      const float hi = dec.hi[t], lo = dec.lo[t];
#pragma unroll
      for (int r = 0; r < 16; r += 4) {
        const int s = 32 * st + acc_row(r, h);
        float p[4];
#pragma unroll
        for (int j = 0; j < 4; ++j)
          p[j] = s + j <= t ? raw[r + j] * (A.scale * decay_between(dec, s + j, hi, lo)) : 0.f;
        Elem<T>::store4(sp + t * PS + s, p);
      }
    }
    // o^T = S^T q^T: rows of v's columns, lane = t
    f32x16 acc[NC];
#pragma unroll
    for (int tt = 0; tt < NC; ++tt) acc[tt] = f32x16{};
#pragma unroll
    for (int kk = 0; kk < KP / 16; ++kk) {
      const auto sf = acc_frag<T>(S[kk >> 1], kk & 1);
#pragma unroll
      for (int tt = 0; tt < NC; ++tt) Elem<T>::mma(acc[tt], sf, row_frag_acc(sq, KS, 32 * tt + l, 16 * kk, h));
    }
#pragma unroll
    for (int tt = 0; tt < NC; ++tt) acc[tt] *= dec.qf[32 * tt + l];
    lds_barrier();
    // + v^T P^T
#pragma unroll
    for (int k0 = 0; k0 < C; k0 += 16) {
      const auto vf = col_frag(sv, VS, k0, 32 * wave, lane);
#pragma unroll
      for (int tt = k0 / 32; tt < NC; ++tt) Elem<T>::mma(acc[tt], vf, row_frag(sp, PS, 32 * tt + l, k0, h));
    }
#pragma unroll
    for (int tt = 0; tt < NC; ++tt) {
      const int t = t0 + 32 * tt + l;
      if (t < pc.len) {
#pragma unroll
        for (int r = 0; r < 16; r += 4) {
          const int c = 32 * wave + acc_row(r, h);
          float x[4] = {acc[tt][r], acc[tt][r + 1], acc[tt][r + 2], acc[tt][r + 3]};
          put4(o + t * ot + c, x, g.Dv - c, A.ovec);
        }
      }
    }
    state_add<T, KP>(S, sk, KS, sv, VS, 32 * wave, dec.kf, dec.tot, lane);
    lds_barrier();
  }
  if (pc.last && A.sf) state_write<KP>(S, A.sf + sidx, g.Dk, g.Dv, g.Dv, 1, y, h);
}

template <typename T> hipError_t linattn_fwd_t(const FwdArgs& a) {
  const dim3 grid((unsigned)((int64_t)a.g.pieces * a.g.H));
  const hipStream_t st = (hipStream_t)a.stream;
  const bool kw = a.g.Dk > 64, vw = a.g.Dv > 64;
  if (kw && vw) hipLaunchKernelGGL((linattn_fwd_kernel<T, 128, 128>), grid, dim3(256), 0, st, a);
  else if (kw) hipLaunchKernelGGL((linattn_fwd_kernel<T, 128, 64>), grid, dim3(128), 0, st, a);
  else if (vw) hipLaunchKernelGGL((linattn_fwd_kernel<T, 64, 128>), grid, dim3(256), 0, st, a);
  else hipLaunchKernelGGL((linattn_fwd_kernel<T, 64, 64>), grid, dim3(128), 0, st, a);
  return hipGetLastError();
}

}  // namespace la
}  // namespace gspn
