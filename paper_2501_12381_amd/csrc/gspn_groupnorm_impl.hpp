// Group norm with an activation on channels-last maps, x (B, L, C):
//
//   xh = (x - mean) rstd over the L x C/G values of a group, z = xh w + b, y = act(z)
//   dz = dy act'(z), db = sum dz, dw = sum dz xh
//   dx = rstd (dz w - S1 - xh S2),  S1 = mean(dz w), S2 = mean(dz w xh)  over the group
//
// Statistics are sums in fp32 of x - p and (x - p)^2, p the group's first value:
// maps whose mean is large against their spread keep their digits, and partial
// sums of parts of L add up.  Every sum has one order: results repeat bit for bit.
#pragma once

#include "gspn_device.hpp"
#include "gspn_groupnorm.hpp"

namespace gspn {
namespace gn {

template <typename T, int V> __device__ __forceinline__ void load_v(const T* p, float* x) {
  if constexpr (V == 1) {
    x[0] = to_f(p[0]);
  } else {
    union {
      uint4 r;
      T e[V];
    } u;
    u.r = *reinterpret_cast<const uint4*>(p);
#pragma unroll
    for (int j = 0; j < V; ++j) x[j] = to_f(u.e[j]);
  }
}
template <typename T, int V> __device__ __forceinline__ void store_v(T* p, const float* x) {
  if constexpr (V == 1) {
    p[0] = from_f<T>(x[0]);
  } else {
    union {
      uint4 r;
      T e[V];
    } u;
#pragma unroll
    for (int j = 0; j < V; ++j) u.e[j] = from_f<T>(x[j]);
    *reinterpret_cast<uint4*>(p) = u.r;
  }
}

__device__ __forceinline__ float sigmoid_f(float z) { return __builtin_amdgcn_rcpf(1.f + __expf(-z)); }

__device__ __forceinline__ float act_f(float z, int act) {
  if (act == 1) return z * sigmoid_f(z);
  if (act == 2) return 0.5f * z * (1.f + erff(z * 0.70710678f));
  return z;
}
__device__ __forceinline__ float act_slope(float z, int act) {
  if (act == 1) {
    const float g = sigmoid_f(z);
    return g * (1.f + z * (1.f - g));
  }
  if (act == 2) return 0.5f * (1.f + erff(z * 0.70710678f)) + z * 0.39894228f * __expf(-0.5f * z * z);
  return 1.f;
}

__device__ __forceinline__ float wave_sum(float v) {
#pragma unroll
  for (int k = 1; k < 64; k <<= 1) v += __shfl_xor(v, k);
  return v;
}

// mean and 1 / sqrt(var + eps) from the sums of x - p and (x - p)^2 over m values
__device__ __forceinline__ void finish_stats(float p, float s, float q, float inv_m, float eps, float& mean,
                                             float& rstd) {
  const float d = s * inv_m;
  mean = p + d;
  const float var = q * inv_m - d * d;
  rstd = rsqrtf((var > 0.f || var != var ? var : 0.f) + eps);
}

template <typename T> __device__ __forceinline__ float param(const void* p, int c, float none) {
  return p ? to_f(reinterpret_cast<const T*>(p)[c]) : none;
}

// ---------------------------------------------------------------------------
// slabs that a wave holds: K loads of V values a lane, one launch
// ---------------------------------------------------------------------------
// Value e of a slab is channel e % cpg of row e / cpg; neighbouring waves take
// neighbouring groups, so that together they read whole rows.
template <typename T, int V, int K> __global__ void __launch_bounds__(256) gn_wave_fwd_kernel(Args A) {
  const int lane = threadIdx.x & 63;
  const int64_t i = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
  if (i >= A.B * A.G) return;
  const int64_t b = i / A.G;
  const int gi = (int)(i - b * A.G), cpg = A.C / A.G, m = (int)A.L * cpg;
  const T* x = reinterpret_cast<const T*>(A.x) + b * A.L * A.C + gi * cpg;
  T* y = reinterpret_cast<T*>(A.y) + b * A.L * A.C + gi * cpg;
  float v[K][V];
  const float p = to_f(x[0]);
  float s = 0.f, q = 0.f;
#pragma unroll
  for (int k = 0; k < K; ++k) {
    const int e = (k * 64 + lane) * V;
    if (e < m) load_v<T, V>(x + (int64_t)(e / cpg) * A.C + e % cpg, v[k]);
    else
#pragma unroll
      for (int j = 0; j < V; ++j) v[k][j] = p;
  }
#pragma unroll
  for (int k = 0; k < K; ++k)
#pragma unroll
    for (int j = 0; j < V; ++j) s += v[k][j] - p;
  s = wave_sum(s);
  const float inv_m = 1.f / (float)m, mean = p + s * inv_m;
  // the values are here: the squares go around the mean itself
#pragma unroll
  for (int k = 0; k < K; ++k)
#pragma unroll
    for (int j = 0; j < V; ++j) {
      const float d = v[k][j] - mean;
      q += (k * 64 + lane) * V < m ? d * d : 0.f;
    }
  q = wave_sum(q);
  const float rstd = rsqrtf(q * inv_m + A.eps);
  if (lane == 0) {
    A.mean[i] = mean;
    A.rstd[i] = rstd;
  }
#pragma unroll
  for (int k = 0; k < K; ++k) {
    const int e = (k * 64 + lane) * V;
    if (e < m) {
      const int c = e % cpg;
      float w[V], o[V];
#pragma unroll
      for (int j = 0; j < V; ++j) w[j] = param<T>(A.weight, gi * cpg + c + j, 1.f);
#pragma unroll
      for (int j = 0; j < V; ++j)
        o[j] = act_f(__builtin_fmaf((v[k][j] - mean) * rstd, w[j], param<T>(A.bias, gi * cpg + c + j, 0.f)), A.act);
      store_v<T, V>(y + (int64_t)(e / cpg) * A.C + c, o);
    }
  }
}

// backward; `rows` batch entries a wave, sums over them to ws[part][2][C]
template <typename T, int V, int K> __global__ void __launch_bounds__(256) gn_wave_bwd_kernel(Args A, int rows) {
  extern __shared__ float lds[];  // a wave's dw and db of every value of the slab
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int64_t i = (int64_t)blockIdx.x * 4 + wave, parts = (A.B + rows - 1) / rows;
  const int cpg = A.C / A.G, m = (int)A.L * cpg;
  const int64_t part = i / A.G;
  const int gi = (int)(i - part * A.G);
  const bool on = part < parts;
  float aw[K][V], ab[K][V], w[K][V], bias[K][V];
#pragma unroll
  for (int k = 0; k < K; ++k) {
    const int e = (k * 64 + lane) * V, c = gi * cpg + e % cpg;
#pragma unroll
    for (int j = 0; j < V; ++j) {
      aw[k][j] = ab[k][j] = 0.f;
      w[k][j] = on && e < m ? param<T>(A.weight, c + j, 1.f) : 0.f;
      bias[k][j] = on && e < m && A.act ? param<T>(A.bias, c + j, 0.f) : 0.f;
    }
  }
  const float inv_m = 1.f / (float)m;
  if (on)
    for (int64_t b = part * rows; b < min(A.B, (part + 1) * rows); ++b) {
      const int64_t base = b * A.L * A.C + gi * cpg;
      const T *x = reinterpret_cast<const T*>(A.x) + base, *dy = reinterpret_cast<const T*>(A.dy) + base;
      T* dx = reinterpret_cast<T*>(A.dx) + base;
      const float mean = A.mean[b * A.G + gi], rstd = A.rstd[b * A.G + gi];
      float xh[K][V], dz[K][V], s1 = 0.f, s2 = 0.f;
#pragma unroll
      for (int k = 0; k < K; ++k) {
        const int e = (k * 64 + lane) * V;
        if (e < m) {
          const int64_t at = (int64_t)(e / cpg) * A.C + e % cpg;
          load_v<T, V>(x + at, xh[k]);
          load_v<T, V>(dy + at, dz[k]);
        } else {
#pragma unroll
          for (int j = 0; j < V; ++j) {
            xh[k][j] = mean;
            dz[k][j] = 0.f;
          }
        }
      }
#pragma unroll
      for (int k = 0; k < K; ++k)
#pragma unroll
        for (int j = 0; j < V; ++j) {
          xh[k][j] = (xh[k][j] - mean) * rstd;
          if (A.act) dz[k][j] *= act_slope(__builtin_fmaf(xh[k][j], w[k][j], bias[k][j]), A.act);
          ab[k][j] += dz[k][j];
          aw[k][j] = __builtin_fmaf(dz[k][j], xh[k][j], aw[k][j]);
          const float d = dz[k][j] * w[k][j];
          s1 += d;
          s2 = __builtin_fmaf(d, xh[k][j], s2);
        }
      s1 = wave_sum(s1) * inv_m;
      s2 = wave_sum(s2) * inv_m;
#pragma unroll
      for (int k = 0; k < K; ++k) {
        const int e = (k * 64 + lane) * V;
        if (e < m) {
          float o[V];
#pragma unroll
          for (int j = 0; j < V; ++j) o[j] = rstd * (dz[k][j] * w[k][j] - s1 - xh[k][j] * s2);
          store_v<T, V>(dx + (int64_t)(e / cpg) * A.C + e % cpg, o);
        }
      }
    }
  // sums over the L rows of the slab, channel by channel
  float* out = reinterpret_cast<float*>(A.ws) + part * 2 * A.C + gi * cpg;
  if (A.L == 1) {
#pragma unroll
    for (int k = 0; k < K; ++k) {
      const int e = (k * 64 + lane) * V;
#pragma unroll
      for (int j = 0; j < V; ++j)
        if (on && e < m) {
          out[e + j] = aw[k][j];
          out[A.C + e + j] = ab[k][j];
        }
    }
    return;
  }
  float* sw = lds + wave * 2 * m;
#pragma unroll
  for (int k = 0; k < K; ++k) {
    const int e = (k * 64 + lane) * V;
#pragma unroll
    for (int j = 0; j < V; ++j)
      if (e < m) {
        sw[e + j] = aw[k][j];
        sw[m + e + j] = ab[k][j];
      }
  }
  __syncthreads();
  if (on)
    for (int c = lane; c < 2 * cpg; c += 64) {
      const float* p = sw + (c < cpg ? c : m + c - cpg);
      float t = 0.f;
      for (int r = 0; r < (int)A.L; ++r) t += p[r * cpg];
      out[c < cpg ? c : A.C + c - cpg] = t;
    }
}

// dw, db: sums of `parts` partial sums ws[part][2][C]
template <typename T> __global__ void __launch_bounds__(256) gn_param_kernel(Args A, int64_t parts) {
  __shared__ float red[2][256];
  const int tx = threadIdx.x & 31, ty = threadIdx.x >> 5, c = blockIdx.x * 32 + tx;
  float w = 0.f, b = 0.f;
  if (c < A.C)
    for (int64_t p = ty; p < parts; p += 8) {
      const float* s = reinterpret_cast<const float*>(A.ws) + p * 2 * A.C + c;
      w += s[0];
      b += s[A.C];
    }
  red[0][threadIdx.x] = w;
  red[1][threadIdx.x] = b;
  __syncthreads();
  if (ty == 0 && c < A.C) {
#pragma unroll
    for (int i = 1; i < 8; ++i) {
      w += red[0][i * 32 + tx];
      b += red[1][i * 32 + tx];
    }
    if (A.dweight) reinterpret_cast<T*>(A.dweight)[c] = from_f<T>(w);
    if (A.dbias) reinterpret_cast<T*>(A.dbias)[c] = from_f<T>(b);
  }
}

// ---------------------------------------------------------------------------
// larger slabs: parts of the L axis
// ---------------------------------------------------------------------------
// A workgroup of 256 takes rows [r0, r1) of a batch entry, all channels: TX
// threads side by side on the channels (V each), 256 / TX rows at a time.
struct Tile {
  int nvec, TX, TY, tx, ty;
  bool on;
  int64_t r0, r1;
};
template <int V> __device__ __forceinline__ Tile make_tile(const Args& A, int split, int splits) {
  Tile t;
  t.nvec = A.C / V;
  t.TX = min(t.nvec, 256);
  t.TY = 256 / t.TX;
  t.ty = threadIdx.x / t.TX;
  t.tx = threadIdx.x - t.ty * t.TX;
  t.on = t.ty < t.TY;
  t.r0 = A.L * split / splits;
  t.r1 = A.L * (split + 1) / splits;
  return t;
}

// parts of the sums: part[b][split][g] = sums of x - p, (x - p)^2
template <typename T, int V> __global__ void __launch_bounds__(256) gn_stats_kernel(Args A, int splits) {
  extern __shared__ float red[];  // [TY][C][2]
  const int split = blockIdx.x % splits;
  const int64_t b = blockIdx.x / splits;
  const Tile t = make_tile<V>(A, split, splits);
  const int cpg = A.C / A.G;
  const T* x = reinterpret_cast<const T*>(A.x) + b * A.L * A.C;
  if (t.on)
    for (int cv = t.tx; cv < t.nvec; cv += t.TX) {
      float p[V], s[V], q[V];
#pragma unroll
      for (int j = 0; j < V; ++j) {
        p[j] = to_f(x[(cv * V + j) / cpg * cpg]);
        s[j] = q[j] = 0.f;
      }
#pragma unroll 4
      for (int64_t r = t.r0 + t.ty; r < t.r1; r += t.TY) {
        float v[V];
        load_v<T, V>(x + r * A.C + cv * V, v);
#pragma unroll
        for (int j = 0; j < V; ++j) {
          const float d = v[j] - p[j];
          s[j] += d;
          q[j] = __builtin_fmaf(d, d, q[j]);
        }
      }
#pragma unroll
      for (int j = 0; j < V; ++j) {
        red[((int64_t)t.ty * A.C + cv * V + j) * 2] = s[j];
        red[((int64_t)t.ty * A.C + cv * V + j) * 2 + 1] = q[j];
      }
    }
  __syncthreads();
  const int lane = threadIdx.x & 63;
  float* part = reinterpret_cast<float*>(A.ws) + (int64_t)blockIdx.x * A.G * 2;
  for (int g = threadIdx.x >> 6; g < A.G; g += 4) {
    float s = 0.f, q = 0.f;
    for (int i = lane; i < cpg * t.TY; i += 64) {
      const int at = (i / cpg * A.C + g * cpg + i % cpg) * 2;
      s += red[at];
      q += red[at + 1];
    }
    s = wave_sum(s);
    q = wave_sum(q);
    if (lane == 0) {
      part[g * 2] = s;
      part[g * 2 + 1] = q;
    }
  }
}

template <typename T, int V> __global__ void __launch_bounds__(256) gn_apply_kernel(Args A, int splits) {
  extern __shared__ float st[];  // [G] mean, [G] rstd
  const int split = blockIdx.x % splits;
  const int64_t b = blockIdx.x / splits;
  const Tile t = make_tile<V>(A, split, splits);
  const int cpg = A.C / A.G, lane = threadIdx.x & 63;
  const T* x = reinterpret_cast<const T*>(A.x) + b * A.L * A.C;
  T* y = reinterpret_cast<T*>(A.y) + b * A.L * A.C;
  const float inv_m = 1.f / ((float)A.L * (float)cpg);
  const float* part = reinterpret_cast<const float*>(A.ws) + b * splits * A.G * 2;
  for (int g = threadIdx.x >> 6; g < A.G; g += 4) {
    float s = 0.f, q = 0.f;
    for (int i = lane; i < splits; i += 64) {
      s += part[((int64_t)i * A.G + g) * 2];
      q += part[((int64_t)i * A.G + g) * 2 + 1];
    }
    s = wave_sum(s);
    q = wave_sum(q);
    float mean, rstd;
    finish_stats(to_f(x[g * cpg]), s, q, inv_m, A.eps, mean, rstd);
    if (lane == 0) {
      st[g] = mean;
      st[A.G + g] = rstd;
      if (split == 0) {
        A.mean[b * A.G + g] = mean;
        A.rstd[b * A.G + g] = rstd;
      }
    }
  }
  __syncthreads();
  if (!t.on) return;
  for (int cv = t.tx; cv < t.nvec; cv += t.TX) {
    float mu[V], a[V], c[V];
#pragma unroll
    for (int j = 0; j < V; ++j) {
      const int ch = cv * V + j, g = ch / cpg;
      mu[j] = st[g];
      a[j] = st[A.G + g] * param<T>(A.weight, ch, 1.f);
      c[j] = param<T>(A.bias, ch, 0.f);
    }
#pragma unroll 4
    for (int64_t r = t.r0 + t.ty; r < t.r1; r += t.TY) {
      float v[V];
      load_v<T, V>(x + r * A.C + cv * V, v);
#pragma unroll
      for (int j = 0; j < V; ++j) v[j] = act_f(__builtin_fmaf(v[j] - mu[j], a[j], c[j]), A.act);
      store_v<T, V>(y + r * A.C + cv * V, v);
    }
  }
}

// backward, first launch: part[b][split][2][C] = sums over the rows of dz xh, dz
template <typename T, int V> __global__ void __launch_bounds__(256) gn_bwd_sums_kernel(Args A, int splits) {
  extern __shared__ float red[];  // [TY][C][2]
  const int split = blockIdx.x % splits;
  const int64_t b = blockIdx.x / splits;
  const Tile t = make_tile<V>(A, split, splits);
  const int cpg = A.C / A.G;
  const T *x = reinterpret_cast<const T*>(A.x) + b * A.L * A.C, *dy = reinterpret_cast<const T*>(A.dy) + b * A.L * A.C;
  if (t.on)
    for (int cv = t.tx; cv < t.nvec; cv += t.TX) {
      float mu[V], rs[V], w[V], c[V], aw[V], ab[V];
#pragma unroll
      for (int j = 0; j < V; ++j) {
        const int ch = cv * V + j;
        mu[j] = A.mean[b * A.G + ch / cpg];
        rs[j] = A.rstd[b * A.G + ch / cpg];
        w[j] = param<T>(A.weight, ch, 1.f);
        c[j] = param<T>(A.bias, ch, 0.f);
        aw[j] = ab[j] = 0.f;
      }
#pragma unroll 2
      for (int64_t r = t.r0 + t.ty; r < t.r1; r += t.TY) {
        float v[V], d[V];
        load_v<T, V>(x + r * A.C + cv * V, v);
        load_v<T, V>(dy + r * A.C + cv * V, d);
#pragma unroll
        for (int j = 0; j < V; ++j) {
          const float xh = (v[j] - mu[j]) * rs[j];
          if (A.act) d[j] *= act_slope(__builtin_fmaf(xh, w[j], c[j]), A.act);
          ab[j] += d[j];
          aw[j] = __builtin_fmaf(d[j], xh, aw[j]);
        }
      }
#pragma unroll
      for (int j = 0; j < V; ++j) {
        red[((int64_t)t.ty * A.C + cv * V + j) * 2] = aw[j];
        red[((int64_t)t.ty * A.C + cv * V + j) * 2 + 1] = ab[j];
      }
    }
  __syncthreads();
  float* part = reinterpret_cast<float*>(A.ws) + (int64_t)blockIdx.x * 2 * A.C;
  for (int c = threadIdx.x; c < A.C; c += 256) {
    float w = 0.f, d = 0.f;
    for (int y = 0; y < t.TY; ++y) {
      w += red[((int64_t)y * A.C + c) * 2];
      d += red[((int64_t)y * A.C + c) * 2 + 1];
    }
    part[c] = w;
    part[A.C + c] = d;
  }
}

// second launch, one workgroup a (batch entry, group): S1, S2 to sums[b][g][2] and
// the channel sums of the entry to its first split's place
template <typename T> __global__ void __launch_bounds__(256) gn_bwd_group_kernel(Args A, int splits, float* sums) {
  __shared__ float red[2][4];
  const int g = blockIdx.x % A.G;
  const int64_t b = blockIdx.x / A.G;
  const int cpg = A.C / A.G;
  float* part = reinterpret_cast<float*>(A.ws) + b * splits * 2 * A.C + g * cpg;
  float s1 = 0.f, s2 = 0.f;
  for (int c = threadIdx.x; c < cpg; c += 256) {
    float w = 0.f, d = 0.f;
    for (int i = 0; i < splits; ++i) {
      w += part[(int64_t)i * 2 * A.C + c];
      d += part[(int64_t)i * 2 * A.C + A.C + c];
    }
    part[c] = w;
    part[A.C + c] = d;
    const float wt = param<T>(A.weight, g * cpg + c, 1.f);
    s1 = __builtin_fmaf(d, wt, s1);
    s2 = __builtin_fmaf(w, wt, s2);
  }
  s1 = wave_sum(s1);
  s2 = wave_sum(s2);
  if ((threadIdx.x & 63) == 0) {
    red[0][threadIdx.x >> 6] = s1;
    red[1][threadIdx.x >> 6] = s2;
  }
  __syncthreads();
  if (threadIdx.x == 0) {
    const float inv_m = 1.f / ((float)A.L * (float)cpg);
    sums[(b * A.G + g) * 2] = (red[0][0] + red[0][1] + red[0][2] + red[0][3]) * inv_m;
    sums[(b * A.G + g) * 2 + 1] = (red[1][0] + red[1][1] + red[1][2] + red[1][3]) * inv_m;
  }
}

// third launch: dx, and dw, db from the entries' channel sums
template <typename T, int V>
__global__ void __launch_bounds__(256) gn_bwd_dx_kernel(Args A, int splits, const float* sums) {
  const int split = blockIdx.x % splits;
  const int64_t b = blockIdx.x / splits;
  const Tile t = make_tile<V>(A, split, splits);
  const int cpg = A.C / A.G;
  for (int64_t c = (int64_t)blockIdx.x * 256 + threadIdx.x; c < A.C; c += (int64_t)gridDim.x * 256) {
    float w = 0.f, d = 0.f;
    for (int64_t i = 0; i < A.B; ++i) {
      const float* p = reinterpret_cast<const float*>(A.ws) + i * splits * 2 * A.C + c;
      w += p[0];
      d += p[A.C];
    }
    if (A.dweight) reinterpret_cast<T*>(A.dweight)[c] = from_f<T>(w);
    if (A.dbias) reinterpret_cast<T*>(A.dbias)[c] = from_f<T>(d);
  }
  if (!t.on) return;
  const T *x = reinterpret_cast<const T*>(A.x) + b * A.L * A.C, *dy = reinterpret_cast<const T*>(A.dy) + b * A.L * A.C;
  T* dx = reinterpret_cast<T*>(A.dx) + b * A.L * A.C;
  for (int cv = t.tx; cv < t.nvec; cv += t.TX) {
    float mu[V], rs[V], w[V], c[V], s1[V], s2[V];
#pragma unroll
    for (int j = 0; j < V; ++j) {
      const int ch = cv * V + j;
      const int64_t g = b * A.G + ch / cpg;
      mu[j] = A.mean[g];
      rs[j] = A.rstd[g];
      w[j] = param<T>(A.weight, ch, 1.f);
      c[j] = param<T>(A.bias, ch, 0.f);
      s1[j] = sums[g * 2];
      s2[j] = sums[g * 2 + 1];
    }
#pragma unroll 2
    for (int64_t r = t.r0 + t.ty; r < t.r1; r += t.TY) {
      float v[V], d[V];
      load_v<T, V>(x + r * A.C + cv * V, v);
      load_v<T, V>(dy + r * A.C + cv * V, d);
#pragma unroll
      for (int j = 0; j < V; ++j) {
        const float xh = (v[j] - mu[j]) * rs[j];
        if (A.act) d[j] *= act_slope(__builtin_fmaf(xh, w[j], c[j]), A.act);
        v[j] = rs[j] * (d[j] * w[j] - s1[j] - xh * s2[j]);
      }
      store_v<T, V>(dx + r * A.C + cv * V, v);
    }
  }
}

// ---------------------------------------------------------------------------
// launches
// ---------------------------------------------------------------------------
template <typename T, int V> hipError_t fwd_wave(const Args& a, const Plan& p) {
  const dim3 grid((unsigned)((a.B * a.G + 3) / 4));
  const hipStream_t st = (hipStream_t)a.stream;
  switch (p.K) {
    case 1: hipLaunchKernelGGL((gn_wave_fwd_kernel<T, V, 1>), grid, dim3(256), 0, st, a); break;
    case 2: hipLaunchKernelGGL((gn_wave_fwd_kernel<T, V, 2>), grid, dim3(256), 0, st, a); break;
    case 4: hipLaunchKernelGGL((gn_wave_fwd_kernel<T, V, 4>), grid, dim3(256), 0, st, a); break;
    case 8: hipLaunchKernelGGL((gn_wave_fwd_kernel<T, V, 8>), grid, dim3(256), 0, st, a); break;
    default:
      if constexpr (V == 1) hipLaunchKernelGGL((gn_wave_fwd_kernel<T, V, 16>), grid, dim3(256), 0, st, a);
  }
  return hipGetLastError();
}

template <typename T, int V> hipError_t fwd_split(const Args& a, const Plan& p) {
  const int nvec = a.C / V, TX = nvec < 256 ? nvec : 256, TY = 256 / TX;
  const dim3 grid((unsigned)(a.B * p.splits));
  const hipStream_t st = (hipStream_t)a.stream;
  hipLaunchKernelGGL((gn_stats_kernel<T, V>), grid, dim3(256), (size_t)TY * a.C * 8, st, a, p.splits);
  hipLaunchKernelGGL((gn_apply_kernel<T, V>), grid, dim3(256), (size_t)a.G * 8, st, a, p.splits);
  return hipGetLastError();
}

template <typename T, int V> hipError_t bwd_wave(const Args& a, const Plan& p) {
  const int64_t parts = (a.B + p.rows - 1) / p.rows;
  const dim3 grid((unsigned)((parts * a.G + 3) / 4));
  const hipStream_t st = (hipStream_t)a.stream;
  const size_t lds = a.L == 1 ? 0 : (size_t)4 * 2 * a.L * (a.C / a.G) * 4;
  switch (p.K) {
    case 1: hipLaunchKernelGGL((gn_wave_bwd_kernel<T, V, 1>), grid, dim3(256), lds, st, a, p.rows); break;
    case 2: hipLaunchKernelGGL((gn_wave_bwd_kernel<T, V, 2>), grid, dim3(256), lds, st, a, p.rows); break;
    case 4: hipLaunchKernelGGL((gn_wave_bwd_kernel<T, V, 4>), grid, dim3(256), lds, st, a, p.rows); break;
    default:
      if constexpr (V == 1) {
        if (p.K == 8) hipLaunchKernelGGL((gn_wave_bwd_kernel<T, V, 8>), grid, dim3(256), lds, st, a, p.rows);
        else hipLaunchKernelGGL((gn_wave_bwd_kernel<T, V, 16>), grid, dim3(256), lds, st, a, p.rows);
      }
  }
  hipLaunchKernelGGL(gn_param_kernel<T>, dim3((a.C + 31) / 32), dim3(256), 0, st, a, parts);
  return hipGetLastError();
}

template <typename T, int V> hipError_t bwd_split(const Args& a, const Plan& p) {
  const int nvec = a.C / V, TX = nvec < 256 ? nvec : 256, TY = 256 / TX;
  const dim3 grid((unsigned)(a.B * p.splits));
  const hipStream_t st = (hipStream_t)a.stream;
  float* sums = reinterpret_cast<float*>(a.ws) + a.B * p.splits * 2 * a.C;
  hipLaunchKernelGGL((gn_bwd_sums_kernel<T, V>), grid, dim3(256), (size_t)TY * a.C * 8, st, a, p.splits);
  hipLaunchKernelGGL((gn_bwd_group_kernel<T>), dim3((unsigned)(a.B * a.G)), dim3(256), 0, st, a, p.splits, sums);
  hipLaunchKernelGGL((gn_bwd_dx_kernel<T, V>), grid, dim3(256), 0, st, a, p.splits, sums);
  return hipGetLastError();
}

template <typename T> hipError_t fwd_t(const Args& a) {
  constexpr int F = 16 / sizeof(T);
  const Plan p = make_plan(a.B, a.L, a.C, a.G, sizeof(T) == 4 ? 0 : 1, a.vec, false);
  if (p.wave) return p.V == 1 ? fwd_wave<T, 1>(a, p) : fwd_wave<T, F>(a, p);
  return p.V == 1 ? fwd_split<T, 1>(a, p) : fwd_split<T, F>(a, p);
}
template <typename T> hipError_t bwd_t(const Args& a) {
  constexpr int F = 16 / sizeof(T);
  const Plan p = make_plan(a.B, a.L, a.C, a.G, sizeof(T) == 4 ? 0 : 1, a.vec, true);
  if (p.wave) return p.V == 1 ? bwd_wave<T, 1>(a, p) : bwd_wave<T, F>(a, p);
  return p.V == 1 ? bwd_split<T, 1>(a, p) : bwd_split<T, F>(a, p);
}

}  // namespace gn
}  // namespace gspn
