// Launch interface of the group-norm kernels (gspn_groupnorm_*.hip).
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

namespace gspn {
namespace gn {

// x (B, L, C), groups of C / G channels
struct Args {
  const void* x;
  const void* weight;  // (C) or null: ones
  const void* bias;    // (C) or null: zeros
  float eps;
  int act;             // 0 none, 1 silu, 2 gelu
  int64_t B, L;
  int C, G;
  float *mean, *rstd;  // (B, G)
  // forward
  void* y;
  // backward
  const void* dy;
  void *dx, *dweight, *dbias;
  void* ws;
  int vec;             // x, y (dy, dx) start on 16 bytes
  void* stream;
};

size_t fwd_workspace(int64_t B, int64_t L, int C, int G, int dtype);
size_t bwd_workspace(int64_t B, int64_t L, int C, int G, int dtype);
hipError_t fwd_f32(const Args& a);
hipError_t fwd_bf16(const Args& a);
hipError_t bwd_f32(const Args& a);
hipError_t bwd_bf16(const Args& a);

constexpr int kMaxC = 8192;

// ---- how a problem is cut (host; the workspace sizes go by it) ----------------
// Slabs (one group of one batch entry) that a wave holds in its registers take
// one launch; larger ones are summed in splits of the L axis and normalised by a
// second launch.
struct Plan {
  bool wave;       // a wave holds a slab
  int V, K;        // elements of a load, loads a lane
  int rows;        // wave: batch entries a wave takes (backward: for one partial sum)
  int splits;      // else: parts of L
};

inline Plan make_plan(int64_t B, int64_t L, int C, int G, int dtype, int vec, bool bwd) {
  Plan p{};
  const int cpg = C / G, full = dtype == 0 ? 4 : 8;
  const int64_t m = L * cpg;
  const int V = vec && cpg % full == 0 ? full : 1;
  const int64_t per = (m / V + 63) / 64;  // loads a lane
  const int most = V == 1 ? 16 : (bwd ? 4 : 8);
  if (per <= most) {
    p.wave = true;
    p.V = V;
    p.K = 1;
    while (p.K < per) p.K *= 2;
    p.rows = 1;
    // backward: the sums over the batch are kept in registers over several
    // entries, which leaves fewer partial sums; enough waves stay to fill the card
    if (bwd)
      while (p.rows < 64 && B * G / (p.rows * 2) >= 4096) p.rows *= 2;
    return p;
  }
  p.V = vec && C % full == 0 ? full : 1;
  // four workgroups a compute unit, at least 16 rows each
  int64_t s = (1024 + B - 1) / B;
  const int64_t most_s = (L + 15) / 16;
  if (s > most_s) s = most_s;
  if (s > 256) s = 256;
  p.splits = (int)(s < 1 ? 1 : s);
  return p;
}

}  // namespace gn
}  // namespace gspn
