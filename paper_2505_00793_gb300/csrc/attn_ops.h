// Operators on packed token rows (the entry points mf_qk_rope_* and mf_attn_* of ops_capi.cu,
// which checks the arguments; kernels in rope_ops.cu and attn_tc.cu).
#pragma once

#include <cuda_bf16.h>
#include <cuda_runtime.h>
#include <stdint.h>

#include "../../include/mixflow.h"

namespace mf {

// Sequences of a packed batch: rows 0 .. rows-1; start [n+1] on the device, or null for
// sequences of len rows each.
struct SeqRows {
  const int* start = nullptr;
  int n = 0, len = 0, rows = 0;
};

// Blocks of a head-norm launch (two per SM), which bounds its partial sums.
constexpr int kRopeMaxBlocks = 2 * 152;

struct RopeParams {
  SeqRows seq;
  int Hq = 0, Hkv = 0, Hc = 0, D = 0;   // query, key and converted heads of D elements
  int R = 0;                            // rotated elements
  bool half = true;                     // pairs (j, j + R/2), else (2j, 2j + 1)
  float eps = 0.f, mscale = 1.f;
  const void *x = nullptr, *xd = nullptr;
  void *y = nullptr, *yd = nullptr;
  const void *dy = nullptr, *dyd = nullptr;
  void *dx = nullptr, *dxd = nullptr;
  int64_t ldx = 0, ldy = 0, lddy = 0, lddx = 0;
  const float *gq = nullptr, *gk = nullptr, *gqd = nullptr, *gkd = nullptr;
  float *dgq = nullptr, *dgk = nullptr, *dgqd = nullptr, *dgkd = nullptr;
  float* part = nullptr;                // [blocks][2 or 4][D] partial gain gradients
  const int* pos = nullptr;
  int* status = nullptr;
  // set by qk_rope: lanes a head takes, vector access; heads of a part of a row, the parts, units of
  // work a row is split into and the parts of each; a warp's next unit; shared memory
  int lanes = 1;
  bool vec = false;
  int hc = 1, parts = 1, splits = 1, run = 1;
  int step_row = 0, step_split = 0;
  int stage_bytes = 0, ring_bytes = 0;
  uint64_t phase[64];                   // 2^-64 turns a position, per rotated pair
};
// Whether r describes rotary positions of heads of D elements.
bool rope_desc_ok(const mf_rope_desc& r, int D);
cudaError_t qk_rope(RopeParams p, bool bwd, bool x_bf16, bool y_bf16, cudaStream_t s);

struct AttnParams {
  SeqRows seq;
  int Hq = 0, Hkv = 0, D = 0;
  float scale = 1.f;
  const __nv_bfloat16 *q = nullptr, *k = nullptr, *v = nullptr;
  const __nv_bfloat16 *qd = nullptr, *kd = nullptr, *vd = nullptr;
  __nv_bfloat16 *o = nullptr, *od = nullptr;
  const __nv_bfloat16 *d_o = nullptr, *d_od = nullptr;
  __nv_bfloat16 *dq = nullptr, *dk = nullptr, *dv = nullptr;
  __nv_bfloat16 *dqd = nullptr, *dkd = nullptr, *dvd = nullptr;
  int64_t ldq = 0, ldk = 0, ldv = 0, ldo = 0, lddo = 0, lddq = 0, lddk = 0, lddv = 0;
  float *lse = nullptr, *rbar = nullptr;     // [Hq][rows]
  float *Dr = nullptr, *Drd = nullptr;       // backward: D = rowsum(dO O) and its tangent
  int* status = nullptr;
};
// Both passes (attn_tc.cu): heads of up to 128 columns, 64 with tangents.
cudaError_t attn_tc_fwd(const AttnParams& p, bool dual, cudaStream_t s);
cudaError_t attn_tc_bwd(const AttnParams& p, bool dual, cudaStream_t s);

}  // namespace mf
