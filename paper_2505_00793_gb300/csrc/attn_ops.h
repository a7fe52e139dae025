// Operators on packed token rows (the entry points mf_qk_rope_*, mf_attn_*, mf_attn_window_* and
// mf_embed_* of ops_capi.cu, which checks the arguments; kernels in rope_ops.cu, attn_tc_impl.cuh
// and embed_ops.cu).
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
  // attn_window_*: rows of a window (fewer than seq.rows), first rows of a sequence that stay
  // visible, sums of those rows' gradients
  int window = 0, sinks = 0;
  float* part = nullptr;
};
// Both passes (attn_tc.cu, kernels in attn_tc_impl.cuh): heads of up to 128 columns, 64 with tangents.
cudaError_t attn_tc_fwd(const AttnParams& p, bool dual, cudaStream_t s);
cudaError_t attn_tc_bwd(const AttnParams& p, bool dual, cudaStream_t s);
// The same with a window (attn_tc_window.cu).
cudaError_t attn_window_fwd(const AttnParams& p, bool dual, cudaStream_t s);
cudaError_t attn_window_bwd(const AttnParams& p, bool dual, cudaStream_t s);
constexpr int kMaxSinks = 128;               // a tile of key rows
// Query rows of a chunk that one CTA of the backward pass takes for a sequence's sinks.
inline int window_chunk(int window) { return window > 512 ? 1024 : 512; }
// Floats of AttnParams::part.
inline int64_t window_part(int64_t rows, int Hkv, int D, int window, int sinks, bool dual) {
  const int64_t chunk = window_chunk(window), chunks = (rows + chunk - 1) / chunk;
  return sinks > 0 && chunks > 1 ? 2 * chunks * Hkv * (dual ? 4 : 2) * sinks * (D > 64 ? 128 : 64) : 0;
}


struct EmbedParams {
  SeqRows seq;                               // rows of tokens: those before the last sequence's end
  int vocab = 0, dim = 0;
  float scale = 1.f;
  const int* ids = nullptr;
  const void *E = nullptr, *Ed = nullptr;
  void *y = nullptr, *yd = nullptr;
  const void *dy = nullptr, *dyd = nullptr;
  float *dE = nullptr, *dEd = nullptr;
  int64_t ldE = 0, ldy = 0, lddy = 0, lddE = 0;
};
// How the gradient of a table is summed (embed_ops.cu).
struct EmbedPlan {
  int blocks = 0, shared = 0;                // one launch of so many blocks a part, their shared memory
  uint32_t by = 0;                           // (2^32 / blocks, rounded up); or:
  int bits = 0, passes = 0;                  // of a digit; of the sort
  int tile = 0, tiles = 0;                   // tokens of a block of the sort, blocks
  bool cluster = false;                      // the sort is one cluster's
  int slabs = 0, parts = 0;                  // of 128 columns; warps of a range
  int per = 0, groups = 0;                   // steps of a range, a warp's; blocks along the ranges
  int64_t list = 0, hist = 0, ends = 0, part = 0, bytes = 0;   // offsets into the workspace
};
EmbedPlan embed_plan(int64_t rows, int64_t vocab, int64_t dim, bool dual);
cudaError_t embed_fwd(const EmbedParams& p, bool e_bf16, bool y_bf16, cudaStream_t s);
cudaError_t embed_bwd(const EmbedParams& p, bool y_bf16, void* work, cudaStream_t s);

}  // namespace mf
