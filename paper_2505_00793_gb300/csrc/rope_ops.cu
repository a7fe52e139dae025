// Head norms with rotary positions (mf_qk_rope_fwd / mf_qk_rope_bwd): one pass from the rows
// of the fused q | k | v projection to the attention's operands, and back, each with its
// forward tangent.  Per head x with gain g and position p:
//   r = (mean x^2 + eps)^-1/2,  y = g x r,  z = R(p) y
//   r' = -r^3 mean(x x'),       y' = g' x r + g (x' r + x r'),  z' = R(p) y'
// and backward, with dy = R(p)^T dz, a = g dy, m = mean(x a):
//   dx  = r a - r^3 m x,   dg = sum dy x r
//   dx' = r' a + r a' - (3 r^2 r' m + r^3 m') x - r^3 m x',
//         a' = g' dy + g dy',  m' = mean(x' a + x a'),  dg' = sum dy' x r + dy (x' r + x r')
//
// Layout: a warp walks the heads of one row.  A head is cut into units of eight elements, one
// unit a lane, so that both elements of every rotated pair are in one lane: in the half layout
// a rotated unit is four elements of the first half and their four partners, else eight
// neighbours.  A lane keeps its unit for every head of the row, so each pair's cos and sin are
// computed once a row, in registers, and no table is read.  A head takes the next power of two
// of lanes, and the sums over a head are shuffles.
#include "attn_ops.h"
#include "device_math.cuh"
#include "launch.cuh"
#include "packed_rows.cuh"

namespace mf {
namespace {

constexpr int kRopeThreads = 256;
constexpr int kRopeWarps = kRopeThreads / 32;

// cos and sin of pos * phase, phase in units of 2^-64 turns: the product modulo 2^64 is the
// angle modulo a turn, exactly, so a far position loses nothing.  The nearest quarter turn is
// taken off before the angle becomes a float.
__device__ __forceinline__ void turn_cos_sin(int pos, uint64_t phase, float& c, float& s) {
  const uint64_t ph = static_cast<uint64_t>(static_cast<int64_t>(pos)) * phase;
  const uint32_t quad = static_cast<uint32_t>((ph + (1ull << 61)) >> 62);
  const int64_t rest = static_cast<int64_t>(ph - (static_cast<uint64_t>(quad) << 62));
  float cs, sn;
  sincospif(__ll2float_rn(rest) * 1.0842021724855044e-19f, &sn, &cs);   // 2^-63: half turns
  const float x = (quad & 1) ? sn : cs, y = (quad & 1) ? cs : sn;
  c = (quad == 1 || quad == 2) ? -x : x;
  s = (quad & 2) ? -y : y;
}

// A lane's unit of a head: four pairs (a, b) of elements.
struct Unit {
  int oa, ob;      // first element of a and of b (vector form)
  int u;           // rotated units: first pair is 4 u; others: place 8 u behind the rotated part
  bool on, rot, mix;   // in use; rotated; a and b alternate in memory
};

__device__ __forceinline__ Unit make_unit(const RopeParams& p, int lane) {
  Unit t;
  const int u = lane & (p.lanes - 1);
  const int nrot = (p.R / 2 + 3) / 4;
  t.rot = u < nrot;
  t.u = t.rot ? u : u - nrot;
  t.on = t.rot || p.R + 8 * t.u < p.D;
  t.mix = t.rot && !p.half;
  t.oa = t.rot ? (p.half ? 4 * t.u : 8 * t.u) : p.R + 8 * t.u;
  t.ob = t.rot && p.half ? p.R / 2 + 4 * t.u : t.oa + 4;
  return t;
}

// Element of pair e's a (b = 0) or b (b = 1), or -1 where the head has none.
__device__ __forceinline__ int unit_elem(const RopeParams& p, const Unit& t, int b, int e) {
  if (!t.on) return -1;
  if (t.rot) {
    const int q = 4 * t.u + e;
    if (q >= p.R / 2) return -1;
    return p.half ? (b ? p.R / 2 + q : q) : 2 * q + b;
  }
  const int i = p.R + 8 * t.u + 4 * b + e;
  return i < p.D ? i : -1;
}

__device__ __forceinline__ void load4(const float* s, float (&v)[4]) {
  const float4 f = *reinterpret_cast<const float4*>(s);
  v[0] = f.x; v[1] = f.y; v[2] = f.z; v[3] = f.w;
}
__device__ __forceinline__ void load4(const __nv_bfloat16* s, float (&v)[4]) {
  const uint2 w = *reinterpret_cast<const uint2*>(s);
  v[0] = __uint_as_float(w.x << 16); v[1] = __uint_as_float(w.x & 0xffff0000u);
  v[2] = __uint_as_float(w.y << 16); v[3] = __uint_as_float(w.y & 0xffff0000u);
}
__device__ __forceinline__ void store4(float* d, const float (&v)[4]) {
  *reinterpret_cast<float4*>(d) = make_float4(v[0], v[1], v[2], v[3]);
}
__device__ __forceinline__ void store4(__nv_bfloat16* d, const float (&v)[4]) {
  const __nv_bfloat162 lo = __floats2bfloat162_rn(v[0], v[1]), hi = __floats2bfloat162_rn(v[2], v[3]);
  *reinterpret_cast<uint2*>(d) = make_uint2(*reinterpret_cast<const uint32_t*>(&lo),
                                            *reinterpret_cast<const uint32_t*>(&hi));
}
__device__ __forceinline__ float as_f(float x) { return x; }
__device__ __forceinline__ float as_f(__nv_bfloat16 x) { return __bfloat162float(x); }

// A unit's pairs from and to one head.  Rotated parts of whole eights move as vectors (p.vec),
// others element by element.
template <typename T>
__device__ __forceinline__ void load_unit(const RopeParams& p, const Unit& t, bool on, const T* h,
                                          float (&a)[4], float (&b)[4]) {
#pragma unroll
  for (int e = 0; e < 4; ++e) a[e] = b[e] = 0.f;
  if (!on) return;
  if (p.vec) {
    load4(h + t.oa, a);
    load4(h + t.ob, b);
    if (t.mix) {
      const float a1 = a[1], a3 = a[3], b0 = b[0], b2 = b[2];
      a[1] = a[2]; a[2] = b0; a[3] = b2;
      b[2] = b[1]; b[0] = a1; b[1] = a3;
    }
  } else {
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const int i = unit_elem(p, t, 0, e), j = unit_elem(p, t, 1, e);
      if (i >= 0) a[e] = as_f(h[i]);
      if (j >= 0) b[e] = as_f(h[j]);
    }
  }
}
template <typename T>
__device__ __forceinline__ void store_unit(const RopeParams& p, const Unit& t, bool on, T* h,
                                           const float (&a)[4], const float (&b)[4]) {
  if (!on) return;
  if (p.vec) {
    if (t.mix) {
      const float lo[4] = {a[0], b[0], a[1], b[1]}, hi[4] = {a[2], b[2], a[3], b[3]};
      store4(h + t.oa, lo);
      store4(h + t.ob, hi);
    } else {
      store4(h + t.oa, a);
      store4(h + t.ob, b);
    }
  } else {
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const int i = unit_elem(p, t, 0, e), j = unit_elem(p, t, 1, e);
      if (i >= 0) h[i] = to_t<T>(a[e]);
      if (j >= 0) h[j] = to_t<T>(b[e]);
    }
  }
}

__device__ __forceinline__ void rotate4(float (&a)[4], float (&b)[4], const float (&c)[4],
                                        const float (&s)[4]) {
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    const float x = a[e], y = b[e];
    a[e] = x * c[e] - y * s[e];
    b[e] = y * c[e] + x * s[e];
  }
}

// Sum over the lanes of a head (every lane of the warp takes part).
__device__ __forceinline__ float head_sum(float v, int lanes) {
  for (int o = lanes >> 1; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
  return v;
}

// The rows and heads of one warp: row by row, or, when there are few rows, parts of a row.
struct Walk {
  int64_t item, items, step;
  int per, iters;
};
__device__ __forceinline__ Walk make_walk(const RopeParams& p) {
  Walk w;
  const int hpw = 32 / p.lanes;
  w.iters = (p.Hq + p.Hkv + p.Hc + hpw - 1) / hpw;
  w.per = (w.iters + p.chunks - 1) / p.chunks;
  w.item = static_cast<int64_t>(blockIdx.x) * kRopeWarps + (threadIdx.x >> 5);
  w.step = static_cast<int64_t>(gridDim.x) * kRopeWarps;
  w.items = static_cast<int64_t>(seq_total(p.seq)) * p.chunks;
  return w;
}

// cos and sin (times mscale) of a lane's pairs at a row.
__device__ __forceinline__ void row_turns(const RopeParams& p, const Unit& t, int row,
                                          float (&c)[4], float (&s)[4]) {
  const int pos = p.pos ? p.pos[row] : row - seq_begin(p.seq, row);
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    c[e] = 1.f;
    s[e] = 0.f;
    const int q = 4 * t.u + e;
    if (t.rot && q < p.R / 2) {
      turn_cos_sin(pos, p.phase[q], c[e], s[e]);
      c[e] *= p.mscale;
      s[e] *= p.mscale;
    }
  }
}

template <typename Tx, typename Ty, bool DUAL, bool NORM>
__global__ void __launch_bounds__(kRopeThreads)
    qk_rope_fwd_kernel(const __grid_constant__ RopeParams p) {
  pdl_entry();
  const int lane = threadIdx.x & 31;
  const Unit t = make_unit(p, lane);
  const int sub = lane / p.lanes, hpw = 32 / p.lanes;
  const int Hn = p.Hq + p.Hkv, H = Hn + p.Hc;
  const float invD = 1.f / static_cast<float>(p.D);
  Walk w = make_walk(p);
  for (; w.item < w.items; w.item += w.step) {
    const int row = static_cast<int>(w.item / p.chunks);
    const int i0 = static_cast<int>(w.item % p.chunks) * w.per;
    const int i1 = min(w.iters, i0 + w.per);
    float c[4], s[4];
    row_turns(p, t, row, c, s);
    const Tx* x = static_cast<const Tx*>(p.x) + row * p.ldx;
    const Tx* xd = DUAL ? static_cast<const Tx*>(p.xd) + row * p.ldx : nullptr;
    Ty* y = static_cast<Ty*>(p.y) + row * p.ldy;
    Ty* yd = DUAL ? static_cast<Ty*>(p.yd) + row * p.ldy : nullptr;
    for (int i = i0; i < i1; ++i) {
      const int h = i * hpw + sub;
      const bool on = t.on && h < H;
      float a[4], b[4], ad[4], bd[4];
      load_unit(p, t, on, x + h * p.D, a, b);
      if (DUAL) load_unit(p, t, on, xd + h * p.D, ad, bd);
      if (NORM) {
        float s2 = 0.f, s1 = 0.f;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          s2 += a[e] * a[e] + b[e] * b[e];
          if (DUAL) s1 += a[e] * ad[e] + b[e] * bd[e];
        }
        s2 = head_sum(s2, p.lanes);
        if (DUAL) s1 = head_sum(s1, p.lanes);
        if (h < Hn) {
          const float r = rsqrtf(s2 * invD + p.eps);
          const float rd = DUAL ? -r * r * r * s1 * invD : 0.f;
          float ga[4], gb[4];
          load_unit(p, t, on, h < p.Hq ? p.gq : p.gk, ga, gb);
          float da[4] = {0.f, 0.f, 0.f, 0.f}, db[4] = {0.f, 0.f, 0.f, 0.f};
          if (DUAL && p.gqd) load_unit(p, t, on, h < p.Hq ? p.gqd : p.gkd, da, db);
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const float na = a[e] * r, nb = b[e] * r;
            if (DUAL) {
              ad[e] = da[e] * na + ga[e] * (ad[e] * r + a[e] * rd);
              bd[e] = db[e] * nb + gb[e] * (bd[e] * r + b[e] * rd);
            }
            a[e] = ga[e] * na;
            b[e] = gb[e] * nb;
          }
        }
      }
      if (h < Hn && t.rot) {
        rotate4(a, b, c, s);
        if (DUAL) rotate4(ad, bd, c, s);
      }
      store_unit(p, t, on, y + h * p.D, a, b);
      if (DUAL) store_unit(p, t, on, yd + h * p.D, ad, bd);
    }
  }
}

// Accumulators of the gain gradients: dgq, dgk and, with tangents, dgq', dgk'.
template <typename Tx, typename Ty, bool DUAL, bool NORM>
__global__ void __launch_bounds__(kRopeThreads)
    qk_rope_bwd_kernel(const __grid_constant__ RopeParams p) {
  pdl_entry();
  constexpr int NA = DUAL ? 4 : 2;
  __shared__ float sums[NORM ? kRopeWarps : 1][NORM ? NA * 128 : 1];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const Unit t = make_unit(p, lane);
  const int sub = lane / p.lanes, hpw = 32 / p.lanes;
  const int Hn = p.Hq + p.Hkv, H = Hn + p.Hc;
  const float invD = 1.f / static_cast<float>(p.D);
  float acc[NORM ? NA : 1][8];
#pragma unroll
  for (int i = 0; i < (NORM ? NA : 1); ++i)
#pragma unroll
    for (int e = 0; e < 8; ++e) acc[i][e] = 0.f;
  Walk w = make_walk(p);
  for (; w.item < w.items; w.item += w.step) {
    const int row = static_cast<int>(w.item / p.chunks);
    const int i0 = static_cast<int>(w.item % p.chunks) * w.per;
    const int i1 = min(w.iters, i0 + w.per);
    float c[4], s[4];
    row_turns(p, t, row, c, s);
#pragma unroll
    for (int e = 0; e < 4; ++e) s[e] = -s[e];   // the transposed rotation
    const Ty* dy = static_cast<const Ty*>(p.dy) + row * p.lddy;
    const Ty* dyd = DUAL ? static_cast<const Ty*>(p.dyd) + row * p.lddy : nullptr;
    Ty* dx = static_cast<Ty*>(p.dx) + row * p.lddx;
    Ty* dxd = DUAL ? static_cast<Ty*>(p.dxd) + row * p.lddx : nullptr;
    const Tx* x = NORM ? static_cast<const Tx*>(p.x) + row * p.ldx : nullptr;
    const Tx* xd = NORM && DUAL ? static_cast<const Tx*>(p.xd) + row * p.ldx : nullptr;
    for (int i = i0; i < i1; ++i) {
      const int h = i * hpw + sub;
      const bool on = t.on && h < H, normed = NORM && h < Hn;
      float a[4], b[4], ad[4], bd[4];
      load_unit(p, t, on, dy + h * p.D, a, b);
      if (DUAL) load_unit(p, t, on, dyd + h * p.D, ad, bd);
      if (h < Hn && t.rot) {
        rotate4(a, b, c, s);
        if (DUAL) rotate4(ad, bd, c, s);
      }
      if (NORM) {
        float xa[4], xb[4], xad[4], xbd[4];
        load_unit(p, t, on && normed, x + h * p.D, xa, xb);
        if (DUAL) load_unit(p, t, on && normed, xd + h * p.D, xad, xbd);
        float ga[4], gb[4];
        float da[4] = {0.f, 0.f, 0.f, 0.f}, db[4] = {0.f, 0.f, 0.f, 0.f};
        load_unit(p, t, on && normed, h < p.Hq ? p.gq : p.gk, ga, gb);
        if (DUAL && p.gqd) load_unit(p, t, on && normed, h < p.Hq ? p.gqd : p.gkd, da, db);
        float s2 = 0.f, s1 = 0.f, m = 0.f, md = 0.f;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const float ua = ga[e] * a[e], ub = gb[e] * b[e];
          s2 += xa[e] * xa[e] + xb[e] * xb[e];
          m += xa[e] * ua + xb[e] * ub;
          if (DUAL) {
            s1 += xa[e] * xad[e] + xb[e] * xbd[e];
            md += xad[e] * ua + xbd[e] * ub;
            md += xa[e] * (da[e] * a[e] + ga[e] * ad[e]) + xb[e] * (db[e] * b[e] + gb[e] * bd[e]);
          }
        }
        s2 = head_sum(s2, p.lanes);
        m = head_sum(m, p.lanes) * invD;
        if (DUAL) {
          s1 = head_sum(s1, p.lanes);
          md = head_sum(md, p.lanes) * invD;
        }
        if (normed) {
          const float r = rsqrtf(s2 * invD + p.eps);
          const float r3 = r * r * r;
          const float rd = DUAL ? -r3 * s1 * invD : 0.f;
          const float k0 = r3 * m, k1 = 3.f * r * r * rd * m + r3 * md;
          const bool isq = h < p.Hq;
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const float ca = a[e], cb = b[e], na = xa[e] * r, nb = xb[e] * r;
            const float wa = ca * na, wb = cb * nb;
            acc[0][e] += isq ? wa : 0.f;
            acc[0][4 + e] += isq ? wb : 0.f;
            acc[NORM ? 1 : 0][e] += isq ? 0.f : wa;
            acc[NORM ? 1 : 0][4 + e] += isq ? 0.f : wb;
            a[e] = r * ga[e] * ca - k0 * xa[e];
            b[e] = r * gb[e] * cb - k0 * xb[e];
            if (DUAL) {
              const float va = ad[e] * na + ca * (xad[e] * r + xa[e] * rd);
              const float vb = bd[e] * nb + cb * (xbd[e] * r + xb[e] * rd);
              acc[NORM ? NA - 2 : 0][e] += isq ? va : 0.f;
              acc[NORM ? NA - 2 : 0][4 + e] += isq ? vb : 0.f;
              acc[NORM ? NA - 1 : 0][e] += isq ? 0.f : va;
              acc[NORM ? NA - 1 : 0][4 + e] += isq ? 0.f : vb;
              ad[e] = rd * ga[e] * ca + r * (da[e] * ca + ga[e] * ad[e]) - k1 * xa[e] - k0 * xad[e];
              bd[e] = rd * gb[e] * cb + r * (db[e] * cb + gb[e] * bd[e]) - k1 * xb[e] - k0 * xbd[e];
            }
          }
        }
      }
      store_unit(p, t, on, dx + h * p.D, a, b);
      if (DUAL) store_unit(p, t, on, dxd + h * p.D, ad, bd);
    }
  }
  if (NORM) {
    // lanes of the same unit, then the block's warps, in a fixed order
#pragma unroll
    for (int k = 0; k < NA; ++k)
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        float v = acc[k][e];
        for (int o = p.lanes; o < 32; o <<= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
        const int i = unit_elem(p, t, e >> 2, e & 3);
        if (lane < p.lanes && i >= 0) sums[warp][k * p.D + i] = v;
      }
    __syncthreads();
    float* part = p.part + static_cast<int64_t>(blockIdx.x) * NA * p.D;
    for (int i = threadIdx.x; i < NA * p.D; i += kRopeThreads) {
      float v = 0.f;
#pragma unroll
      for (int j = 0; j < kRopeWarps; ++j) v += sums[j][i];
      part[i] = v;
    }
  }
}

// Sum of the blocks' partial gain gradients in a fixed order: 32 columns a block, eight
// threads a column.
__global__ void __launch_bounds__(256)
    rope_gain_final_kernel(int nblk, int D, int NA, const float* __restrict__ part,
                           float* __restrict__ d0, float* __restrict__ d1, float* __restrict__ d2,
                           float* __restrict__ d3) {
  pdl_entry();
  __shared__ float s[8][33];
  const int col = blockIdx.x * 32 + (threadIdx.x & 31), ty = threadIdx.x >> 5;
  float v = 0.f;
  if (col < NA * D)
    for (int j = ty; j < nblk; j += 8) v += part[static_cast<int64_t>(j) * NA * D + col];
  s[ty][threadIdx.x & 31] = v;
  __syncthreads();
  if (ty == 0 && col < NA * D) {
    float sum = 0.f;
#pragma unroll
    for (int j = 0; j < 8; ++j) sum += s[j][threadIdx.x];
    const int k = col / D;
    (k == 0 ? d0 : k == 1 ? d1 : k == 2 ? d2 : d3)[col % D] = sum;
  }
}

template <typename Tx, typename Ty>
cudaError_t launch_rope(const RopeParams& p, bool bwd, bool dual, bool norm, int grid,
                        cudaStream_t s) {
  const dim3 g(grid), b(kRopeThreads);
  if (bwd) {
    if (dual) return norm ? launch_k(qk_rope_bwd_kernel<Tx, Ty, true, true>, g, b, 0, s, p)
                          : launch_k(qk_rope_bwd_kernel<Tx, Ty, true, false>, g, b, 0, s, p);
    return norm ? launch_k(qk_rope_bwd_kernel<Tx, Ty, false, true>, g, b, 0, s, p)
                : launch_k(qk_rope_bwd_kernel<Tx, Ty, false, false>, g, b, 0, s, p);
  }
  if (dual) return norm ? launch_k(qk_rope_fwd_kernel<Tx, Ty, true, true>, g, b, 0, s, p)
                        : launch_k(qk_rope_fwd_kernel<Tx, Ty, true, false>, g, b, 0, s, p);
  return norm ? launch_k(qk_rope_fwd_kernel<Tx, Ty, false, true>, g, b, 0, s, p)
              : launch_k(qk_rope_fwd_kernel<Tx, Ty, false, false>, g, b, 0, s, p);
}

}  // namespace

cudaError_t qk_rope(RopeParams p, bool bwd, bool x_bf16, bool y_bf16, cudaStream_t s) {
  const bool norm = p.gq != nullptr, dual = bwd ? p.dyd != nullptr : p.xd != nullptr;
  const int units = (p.R / 2 + 3) / 4 + (p.D - p.R + 7) / 8;
  p.lanes = 1;
  while (p.lanes < units) p.lanes *= 2;
  p.vec = p.R % 8 == 0;
  const int hpw = 32 / p.lanes, iters = (p.Hq + p.Hkv + p.Hc + hpw - 1) / hpw;
  // a warp a row once the rows fill the GPU's warps; below that, rows are cut into parts of
  // their heads
  const int64_t warps = static_cast<int64_t>(kRopeMaxBlocks) * kRopeWarps;
  p.chunks = 1;
  while (p.chunks < iters && p.seq.rows * static_cast<int64_t>(p.chunks) * 2 <= warps) p.chunks *= 2;
  const int64_t blocks = (static_cast<int64_t>(p.seq.rows) * p.chunks + kRopeWarps - 1) / kRopeWarps;
  const int grid = static_cast<int>(blocks < kRopeMaxBlocks ? blocks : kRopeMaxBlocks);
  cudaError_t e =
      !x_bf16 && !y_bf16 ? launch_rope<float, float>(p, bwd, dual, norm, grid, s)
      : !x_bf16          ? launch_rope<float, __nv_bfloat16>(p, bwd, dual, norm, grid, s)
                         : launch_rope<__nv_bfloat16, __nv_bfloat16>(p, bwd, dual, norm, grid, s);
  if (e != cudaSuccess || !bwd || !norm) return e;
  const int NA = dual ? 4 : 2;
  return launch_k(rope_gain_final_kernel, dim3((NA * p.D + 31) / 32), dim3(256), 0, s, grid, p.D,
                  NA, static_cast<const float*>(p.part), p.dgq, p.dgk, p.dgqd, p.dgkd);
}

}  // namespace mf
