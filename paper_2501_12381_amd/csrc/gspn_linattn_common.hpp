// Linear attention with a decay for each head: what its kernels share.
//
//   S_t = e^{a_t} S_{t-1} + k_t v_t^T          (S: Dk x Dv, fp32)
//   o_t = scale q_t S_t
//
// A sequence is walked in chunks of C tokens.  With G_t the sum of a over the
// chunk's tokens up to t, S the state before the chunk and G_C the whole sum,
//
//   o_t = scale (e^{G_t} q_t S + sum_{s<=t} e^{G_t-G_s} (q_t.k_s) v_s)
//   S  <- e^{G_C} S + sum_s e^{G_C-G_s} k_s v_s^T
//
// which is products of small matrices: matrix instructions of 32 x 32 tiles
// (16 deep in bf16, 2 deep in fp32), with the state in the registers of the
// workgroup that walks the sequence.  Sequences are cut into pieces where there
// are too few of them to fill the card: each piece's own state is formed first,
// the pieces of a sequence are joined, and each is walked from its start state.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "gspn_device.hpp"
#include "gspn_linattn.hpp"

namespace gspn {
namespace la {

typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x4 __attribute__((ext_vector_type(4)));
typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef __attribute__((address_space(3))) s16x4 lds_s16x4;

// ---------------------------------------------------------------------------
// element types: chunk length, LDS row padding, matrix products
// ---------------------------------------------------------------------------
// A fragment is the 8 values a lane gives to one product step of depth 16: lane
// l holds line l % 32 of its operand and, with h = l / 32, the depths 8h..8h+7.
// Any order of the depths serves as long as both operands have the same one.
template <typename T> struct Elem;

template <> struct Elem<bf16> {
  static constexpr int kChunk = 64;
  static constexpr int kVec = 8;   // elements of a 16-byte load
  static constexpr int kPad = 8;   // LDS rows are 16 bytes longer: 16 rows cover all 64 banks
  // an fp32 value as sums of bf16 ones: three carry all of its 24 bits
  static constexpr int kParts = 3;
  struct Frag {
    bf16x8 v;
  };
  static __device__ __forceinline__ void set(Frag& f, const float* x) {
#pragma unroll
    for (int j = 0; j < 8; ++j) f.v[j] = (bf16)x[j];
  }
  static __device__ __forceinline__ void get(const Frag& f, float* x) {
#pragma unroll
    for (int j = 0; j < 8; ++j) x[j] = (float)f.v[j];
  }
  // x = sum of the parts, each the rounding of what the ones before left
  static __device__ __forceinline__ void split(const float* x, Frag* f) {
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      float r = x[j];
#pragma unroll
      for (int p = 0; p < kParts; ++p) {
        const bf16 b = (bf16)r;
        f[p].v[j] = b;
        r -= (float)b;
      }
    }
  }
  static __device__ __forceinline__ void mma(f32x16& c, const Frag& a, const Frag& b) {
    c = __builtin_amdgcn_mfma_f32_32x32x16_bf16(a.v, b.v, c, 0, 0, 0);
  }
  // 8 consecutive values at p (16-byte aligned) / two runs of 4
  static __device__ __forceinline__ Frag row(const bf16* p) { return {*reinterpret_cast<const bf16x8*>(p)}; }
  static __device__ __forceinline__ Frag row2(const bf16* p, const bf16* q) {
    const bf16x4 a = *reinterpret_cast<const bf16x4*>(p), b = *reinterpret_cast<const bf16x4*>(q);
    return {__builtin_shufflevector(a, b, 0, 1, 2, 3, 4, 5, 6, 7)};
  }
  // 8 values down a column of an LDS tile: rows r0..r0+3 and r1..r1+3 (both
  // the lane's own), columns c0..c0+31, column l % 32 for this lane.  The
  // transposing read hands lane i of 16 the values of column i from four rows,
  // when lane i addresses four values of row i / 4, columns 4 (i % 4).
  static __device__ __forceinline__ Frag col(const bf16* tile, int stride, int r0, int r1, int c0, int lane) {
    const int i = lane & 15;
    const bf16* p = tile + (r0 + (i >> 2)) * stride + c0 + (lane & 16) + 4 * (i & 3);
    const bf16* q = tile + (r1 + (i >> 2)) * stride + c0 + (lane & 16) + 4 * (i & 3);
    const bf16x4 a = __builtin_bit_cast(bf16x4, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)p));
    const bf16x4 b = __builtin_bit_cast(bf16x4, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)q));
    return {__builtin_shufflevector(a, b, 0, 1, 2, 3, 4, 5, 6, 7)};
  }
  static __device__ __forceinline__ void store4(bf16* p, const float* x) {
    uint2 w;
    w.x = pack_bf2(x[0], x[1]);
    w.y = pack_bf2(x[2], x[3]);
    *reinterpret_cast<uint2*>(p) = w;
  }
  static __device__ __forceinline__ void load4(const bf16* p, float* x) {
    const bf16x4 v = *reinterpret_cast<const bf16x4*>(p);
#pragma unroll
    for (int j = 0; j < 4; ++j) x[j] = (float)v[j];
  }
};

template <> struct Elem<float> {
  // half the tokens: the products within a chunk cost as much as those with the
  // state at 64, and the fp32 matrix rate is a sixteenth of bf16's
  static constexpr int kChunk = 32;
  static constexpr int kVec = 4;
  static constexpr int kPad = 4;
  static constexpr int kParts = 1;
  struct Frag {
    float v[8];
  };
  static __device__ __forceinline__ void set(Frag& f, const float* x) {
#pragma unroll
    for (int j = 0; j < 8; ++j) f.v[j] = x[j];
  }
  static __device__ __forceinline__ void get(const Frag& f, float* x) {
#pragma unroll
    for (int j = 0; j < 8; ++j) x[j] = f.v[j];
  }
  static __device__ __forceinline__ void split(const float* x, Frag* f) { set(f[0], x); }
  static __device__ __forceinline__ void mma(f32x16& c, const Frag& a, const Frag& b) {
#pragma unroll
    for (int j = 0; j < 8; ++j) c = __builtin_amdgcn_mfma_f32_32x32x2f32(a.v[j], b.v[j], c, 0, 0, 0);
  }
  static __device__ __forceinline__ Frag row2(const float* p, const float* q) {
    const float4 a = *reinterpret_cast<const float4*>(p), b = *reinterpret_cast<const float4*>(q);
    return {{a.x, a.y, a.z, a.w, b.x, b.y, b.z, b.w}};
  }
  static __device__ __forceinline__ Frag row(const float* p) { return row2(p, p + 4); }
  static __device__ __forceinline__ Frag col(const float* tile, int stride, int r0, int r1, int c0, int lane) {
    Frag f;
    const float* p = tile + c0 + (lane & 31);
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      f.v[j] = p[(r0 + j) * stride];
      f.v[4 + j] = p[(r1 + j) * stride];
    }
    return f;
  }
  static __device__ __forceinline__ void store4(float* p, const float* x) {
    *reinterpret_cast<float4*>(p) = make_float4(x[0], x[1], x[2], x[3]);
  }
  static __device__ __forceinline__ void load4(const float* p, float* x) {
    const float4 v = *reinterpret_cast<const float4*>(p);
    x[0] = v.x; x[1] = v.y; x[2] = v.z; x[3] = v.w;
  }
};

// Depth orders of a fragment in block k0 of 16: natural (8h..8h+7), and the one
// in which the registers of a 32 x 32 result hold its rows: register r of half h
// is row 8 (r/4) + 4h + r%4, so registers 0-7 are rows 4h..4h+3, 8+4h..8+4h+3.
template <typename T>
__device__ __forceinline__ typename Elem<T>::Frag row_frag(const T* tile, int stride, int row, int k0, int h) {
  return Elem<T>::row(tile + row * stride + k0 + 8 * h);
}
template <typename T>
__device__ __forceinline__ typename Elem<T>::Frag row_frag_acc(const T* tile, int stride, int row, int k0, int h) {
  const T* p = tile + row * stride + k0 + 4 * h;
  return Elem<T>::row2(p, p + 8);
}
template <typename T>
__device__ __forceinline__ typename Elem<T>::Frag col_frag(const T* tile, int stride, int k0, int c0, int lane) {
  const int r = k0 + 8 * (lane >> 5);
  return Elem<T>::col(tile, stride, r, r + 4, c0, lane);
}
template <typename T>
__device__ __forceinline__ typename Elem<T>::Frag col_frag_acc(const T* tile, int stride, int k0, int c0, int lane) {
  const int r = k0 + 4 * (lane >> 5);
  return Elem<T>::col(tile, stride, r, r + 8, c0, lane);
}
__device__ __forceinline__ int acc_row(int r, int h) { return 8 * (r >> 2) + 4 * h + (r & 3); }

// the fragment that 8 registers (kk even: 0-7, odd: 8-15) of a result tile are
template <typename T> __device__ __forceinline__ typename Elem<T>::Frag acc_frag(const f32x16& s, int odd) {
  float x[8];
#pragma unroll
  for (int j = 0; j < 8; ++j) x[j] = s[8 * odd + j];
  typename Elem<T>::Frag f;
  Elem<T>::set(f, x);
  return f;
}

__device__ __forceinline__ float exp2_hw(float x) { return __builtin_amdgcn_exp2f(x); }
// 2^x of a 64-bit x: the hardware's power of the nearest float, corrected by what
// that rounding left out
__device__ __forceinline__ float exp2_wide(double x) {
  const float hi = (float)x;
  return exp2_hw(hi) * __builtin_fmaf((float)(x - (double)hi), 0.6931472f, 1.f);
}

// LDS barrier: global loads and stores stay in flight
__device__ __forceinline__ void lds_barrier() {
  asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
  __builtin_amdgcn_s_barrier();
  asm volatile("" ::: "memory");
}

// ---------------------------------------------------------------------------
// pieces
// ---------------------------------------------------------------------------
// Batched sequences are cut at multiples of L tokens; piece i is piece i % P of
// sequence i / P.  Packed ones are cut where the packed axis passes a multiple of
// L: block b of the axis and sequence n meet in piece b + n, an index that no
// other pair has.  Indexes without such a pair have len < 0.  Behind the
// last sequence the rest of the packed axis is sequence N, whose outputs are 0.
struct Piece {
  int seq;         // sequence (its states), or N: tokens of no sequence
  int64_t batch;   // row of the tensors
  int t0, len;     // tokens t0 .. t0 + len - 1 of that row
  bool first, last;
};

__device__ __forceinline__ int cu_at(const Geom& g, int n) {
  // positions out of order or out of range stay inside the tensors
  const int v = n > g.N ? g.T : g.cu[n];
  return v < 0 ? 0 : (v > g.T ? g.T : v);
}

__device__ __forceinline__ Piece find_piece(const Geom& g, int i) {
  Piece p;
  if (!g.cu) {
    p.seq = i / g.P;
    p.batch = p.seq;
    const int b = i - p.seq * g.P;
    p.t0 = b * g.L;
    p.len = min(g.L, g.T - p.t0);
    p.first = b == 0;
    p.last = b == g.P - 1;
    return p;
  }
  int lo = 0, hi = g.N;  // the largest n with cu[n] / L + n <= i (cu[0] is taken as 0)
  while (lo < hi) {
    const int n = (lo + hi + 1) >> 1;
    if (cu_at(g, n) / g.L + n <= i) lo = n;
    else hi = n - 1;
  }
  const int n = lo, b = i - n;
  const int s = n == 0 ? 0 : cu_at(g, n), e = max(n == 0 ? 0 : s, cu_at(g, n + 1));
  const int b0 = s / g.L, b1 = max(b0, (e - 1) / g.L);
  p.seq = n;
  p.batch = 0;
  p.first = b == b0;
  p.last = b == b1;
  p.t0 = max(s, b * g.L);
  p.len = b < b0 || b > b1 ? -1 : max(0, min(e, (b + 1) * g.L) - p.t0);
  return p;
}

// ---------------------------------------------------------------------------
// staging: a chunk's rows from global memory to registers to LDS
// ---------------------------------------------------------------------------
// C rows of D <= DP values; rows past `rows` and columns past D are zero.
template <typename T, int DP, int NT> struct Stage {
  static constexpr int C = Elem<T>::kChunk, V = Elem<T>::kVec;
  static constexpr int kStride = DP + Elem<T>::kPad;
  static constexpr int kRowVecs = DP / V;
  static constexpr int kPer = (C * kRowVecs + NT - 1) / NT;
  static constexpr bool kExact = C * kRowVecs % NT == 0;
  uint4 r[kPer];

  __device__ __forceinline__ void load(const T* __restrict__ base, int64_t tstride, int rows, int D, bool vec,
                                       int tid) {
#pragma unroll
    for (int i = 0; i < kPer; ++i) {
      const int p = tid + i * NT, row = p / kRowVecs, c = (p % kRowVecs) * V;
      uint4 x = make_uint4(0, 0, 0, 0);
      if ((kExact || row < C) && row < rows && c < D) {
        const T* s = base + row * tstride + c;
        if (vec) {
          x = *reinterpret_cast<const uint4*>(s);
        } else {  // rows that are not whole 16-byte vectors
          T e[V];
#pragma unroll
          for (int j = 0; j < V; ++j) e[j] = c + j < D ? s[j] : (T)0.f;
          x = __builtin_bit_cast(uint4, e);
        }
      }
      r[i] = x;
    }
  }
  __device__ __forceinline__ void store(T* tile, int tid) const {
#pragma unroll
    for (int i = 0; i < kPer; ++i) {
      const int p = tid + i * NT, row = p / kRowVecs, c = (p % kRowVecs) * V;
      if (kExact || row < C) *reinterpret_cast<uint4*>(tile + row * kStride + c) = r[i];
    }
  }
};

// ---------------------------------------------------------------------------
// a chunk's decays
// ---------------------------------------------------------------------------
// G_t in powers of two, summed in 64 bits and held as two floats, so that
// differences keep their digits behind a token whose decay is a reset (-inf,
// taken as 2^-150: zero in fp32).
template <int C> struct Decays {
  float hi[C], lo[C];  // G_t
  float qf[C];         // scale e^{G_t}
  float kf[C];         // e^{G_C - G_t}
  float tot;           // e^{G_C}
  float pad[3];
};

template <typename T>
__device__ __forceinline__ double load_decay(const T* __restrict__ a, int64_t stride, int t, int rows) {
  if (t >= rows) return 0.0;
  const double g = (double)to_f(a[t * stride]) * 1.4426950408889634;
  return g < -150.0 ? -150.0 : g;
}

// one wave; g: lane t's own term (0 past the chunk).  Returns G_C.
template <int C> __device__ __forceinline__ double chunk_decays(Decays<C>& d, double g, float scale, int lane) {
#pragma unroll
  for (int k = 1; k < C; k <<= 1) {
    const double o = __shfl_up(g, k);
    if (lane >= k) g += o;
  }
  const double all = __shfl(g, C - 1);
  if (lane < C) {
    const float hi = (float)g;
    d.hi[lane] = hi;
    d.lo[lane] = (float)(g - (double)hi);
    d.qf[lane] = scale * exp2_wide(g);
    d.kf[lane] = exp2_wide(all - g);
  }
  if (lane == 0) d.tot = exp2_wide(all);
  return all;
}

// e^{G_t - G_s} for s <= t, 0 above
template <int C> __device__ __forceinline__ float decay_between(const Decays<C>& d, int s, float hi_t, float lo_t) {
  return exp2_hw((hi_t - d.hi[s]) + (lo_t - d.lo[s]));
}

}  // namespace la
}  // namespace gspn
