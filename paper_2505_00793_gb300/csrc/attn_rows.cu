// Attention on packed token rows, a warp per row: the plainest form of the formulas in
// mixflow.h, exact for every mask (only a row's own keys are ever read) and every head width.
// A lane owns four elements of a head; a key or query row costs two loads and a warp sum.
#include "attn_ops.h"
#include "device_math.cuh"
#include "launch.cuh"
#include "packed_rows.cuh"

namespace mf {
namespace {

constexpr int kWarps = 8;

struct F4 { float v[4]; };
__device__ __forceinline__ F4 zero4() { return F4{{0.f, 0.f, 0.f, 0.f}}; }
// Elements 4 lane .. 4 lane + 3 of a head.
__device__ __forceinline__ F4 row4(const __nv_bfloat16* p, int D, int lane) {
  F4 r = zero4();
  if (4 * lane < D) {
    const uint2 w = *reinterpret_cast<const uint2*>(p + 4 * lane);
    r.v[0] = __uint_as_float(w.x << 16); r.v[1] = __uint_as_float(w.x & 0xffff0000u);
    r.v[2] = __uint_as_float(w.y << 16); r.v[3] = __uint_as_float(w.y & 0xffff0000u);
  }
  return r;
}
__device__ __forceinline__ void put4(__nv_bfloat16* p, int D, int lane, const F4& a, float f) {
  if (4 * lane < D) {
#pragma unroll
    for (int e = 0; e < 4; ++e) p[4 * lane + e] = __float2bfloat16_rn(a.v[e] * f);
  }
}
__device__ __forceinline__ float dot4(const F4& a, const F4& b) {
  float s = a.v[0] * b.v[0] + a.v[1] * b.v[1] + a.v[2] * b.v[2] + a.v[3] * b.v[3];
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) s += __shfl_xor_sync(0xffffffffu, s, o);
  return s;
}
__device__ __forceinline__ void fma4(F4& a, float f, const F4& b) {
#pragma unroll
  for (int e = 0; e < 4; ++e) a.v[e] += f * b.v[e];
}
__device__ __forceinline__ void mul4(F4& a, float f) {
#pragma unroll
  for (int e = 0; e < 4; ++e) a.v[e] *= f;
}

template <bool DUAL>
__global__ void __launch_bounds__(32 * kWarps) rows_fwd_kernel(const AttnParams p) {
  pdl_entry();
  const int64_t id = static_cast<int64_t>(blockIdx.x) * kWarps + (threadIdx.x >> 5);
  const int lane = threadIdx.x & 31, h = static_cast<int>(id % p.Hq);
  const int q = static_cast<int>(id / p.Hq);
  if (q >= seq_total(p.seq)) return;
  const int hk = h / (p.Hq / p.Hkv), D = p.D, lo = seq_begin(p.seq, q);
  const F4 Q = row4(p.q + q * p.ldq + h * D, D, lane);
  const F4 Qd = DUAL ? row4(p.qd + q * p.ldq + h * D, D, lane) : zero4();
  F4 o = zero4(), od = zero4();
  float m = -INFINITY, l = 0.f, rs = 0.f;
  for (int j = lo; j <= q; ++j) {
    const F4 K = row4(p.k + j * p.ldk + hk * D, D, lane), V = row4(p.v + j * p.ldv + hk * D, D, lane);
    const float s = p.scale * dot4(Q, K);
    if (s > m) {
      const float f = expf(m - s);
      m = s;
      l *= f; rs *= f;
      mul4(o, f); mul4(od, f);
    }
    const float e = expf(s - m);
    l += e;
    fma4(o, e, V);
    if (DUAL) {
      const F4 Kd = row4(p.kd + j * p.ldk + hk * D, D, lane), Vd = row4(p.vd + j * p.ldv + hk * D, D, lane);
      const float sd = p.scale * (dot4(Qd, K) + dot4(Q, Kd));
      rs += e * sd;
      fma4(od, e * sd, V);
      fma4(od, e, Vd);
    }
  }
  const float inv = 1.f / l, rb = rs * inv;
  mul4(o, inv);
  put4(p.o + q * p.ldo + h * D, D, lane, o, 1.f);
  if (DUAL) {
    mul4(od, inv);
    fma4(od, -rb, o);
    put4(p.od + q * p.ldo + h * D, D, lane, od, 1.f);
  }
  if (lane == 0) {
    p.lse[static_cast<int64_t>(h) * p.seq.rows + q] = m + logf(l);
    if (DUAL) p.rbar[static_cast<int64_t>(h) * p.seq.rows + q] = rb;
  }
}

// P, dS (and tangents) of one pair from its row's statistics.
struct Pair { float pr, ds, pd, dsd; };
template <bool DUAL>
__device__ __forceinline__ Pair pair_of(const AttnParams& p, const F4& Q, const F4& Qd, const F4& K,
                                        const F4& Kd, const F4& V, const F4& Vd, const F4& O,
                                        const F4& Od, float lse, float rb, float Dr, float Drd) {
  Pair r;
  r.pr = expf(p.scale * dot4(Q, K) - lse);
  const float x = dot4(O, V) - Dr;
  r.ds = r.pr * x;
  if (DUAL) {
    r.pd = r.pr * (p.scale * (dot4(Qd, K) + dot4(Q, Kd)) - rb);
    r.dsd = r.pd * x + r.pr * (dot4(Od, V) + dot4(O, Vd) - Drd);
  }
  return r;
}

template <bool DUAL>
__global__ void __launch_bounds__(32 * kWarps) rows_bwd_q_kernel(const AttnParams p) {
  pdl_entry();
  const int64_t id = static_cast<int64_t>(blockIdx.x) * kWarps + (threadIdx.x >> 5);
  const int lane = threadIdx.x & 31, h = static_cast<int>(id % p.Hq);
  const int q = static_cast<int>(id / p.Hq);
  if (q >= seq_total(p.seq)) return;
  const int hk = h / (p.Hq / p.Hkv), D = p.D, lo = seq_begin(p.seq, q);
  const int64_t st = static_cast<int64_t>(h) * p.seq.rows + q;
  const F4 Q = row4(p.q + q * p.ldq + h * D, D, lane), dO = row4(p.d_o + q * p.lddo + h * D, D, lane);
  const F4 O = row4(p.o + q * p.ldo + h * D, D, lane);
  const float Dr = dot4(dO, O), lse = p.lse[st];
  F4 Qd = zero4(), dOd = zero4();
  float Drd = 0.f, rb = 0.f;
  if (DUAL) {
    Qd = row4(p.qd + q * p.ldq + h * D, D, lane);
    dOd = row4(p.d_od + q * p.lddo + h * D, D, lane);
    Drd = dot4(dOd, O) + dot4(dO, row4(p.od + q * p.ldo + h * D, D, lane));
    rb = p.rbar[st];
  }
  if (lane == 0) {
    p.Dr[st] = Dr;
    if (DUAL) p.Drd[st] = Drd;
  }
  F4 dq = zero4(), dqd = zero4();
  for (int j = lo; j <= q; ++j) {
    const F4 K = row4(p.k + j * p.ldk + hk * D, D, lane), V = row4(p.v + j * p.ldv + hk * D, D, lane);
    const F4 Kd = DUAL ? row4(p.kd + j * p.ldk + hk * D, D, lane) : zero4();
    const F4 Vd = DUAL ? row4(p.vd + j * p.ldv + hk * D, D, lane) : zero4();
    const Pair r = pair_of<DUAL>(p, Q, Qd, K, Kd, V, Vd, dO, dOd, lse, rb, Dr, Drd);
    fma4(dq, r.ds, K);
    if (DUAL) {
      fma4(dqd, r.dsd, K);
      fma4(dqd, r.ds, Kd);
    }
  }
  put4(p.dq + q * p.lddq + h * D, D, lane, dq, p.scale);
  if (DUAL) put4(p.dqd + q * p.lddq + h * D, D, lane, dqd, p.scale);
}

template <bool DUAL>
__global__ void __launch_bounds__(32 * kWarps) rows_bwd_kv_kernel(const AttnParams p) {
  pdl_entry();
  const int64_t id = static_cast<int64_t>(blockIdx.x) * kWarps + (threadIdx.x >> 5);
  const int lane = threadIdx.x & 31, hk = static_cast<int>(id % p.Hkv);
  const int j = static_cast<int>(id / p.Hkv);
  if (j >= seq_total(p.seq)) return;
  const int G = p.Hq / p.Hkv, D = p.D, hi = seq_end(p.seq, j);
  const F4 K = row4(p.k + j * p.ldk + hk * D, D, lane), V = row4(p.v + j * p.ldv + hk * D, D, lane);
  const F4 Kd = DUAL ? row4(p.kd + j * p.ldk + hk * D, D, lane) : zero4();
  const F4 Vd = DUAL ? row4(p.vd + j * p.ldv + hk * D, D, lane) : zero4();
  F4 dk = zero4(), dv = zero4(), dkd = zero4(), dvd = zero4();
  for (int h = hk * G; h < (hk + 1) * G; ++h) {
    for (int q = j; q < hi; ++q) {
      const int64_t st = static_cast<int64_t>(h) * p.seq.rows + q;
      const F4 Q = row4(p.q + q * p.ldq + h * D, D, lane), dO = row4(p.d_o + q * p.lddo + h * D, D, lane);
      const F4 Qd = DUAL ? row4(p.qd + q * p.ldq + h * D, D, lane) : zero4();
      const F4 dOd = DUAL ? row4(p.d_od + q * p.lddo + h * D, D, lane) : zero4();
      const Pair r = pair_of<DUAL>(p, Q, Qd, K, Kd, V, Vd, dO, dOd, p.lse[st],
                                   DUAL ? p.rbar[st] : 0.f, p.Dr[st], DUAL ? p.Drd[st] : 0.f);
      fma4(dv, r.pr, dO);
      fma4(dk, r.ds, Q);
      if (DUAL) {
        fma4(dvd, r.pd, dO); fma4(dvd, r.pr, dOd);
        fma4(dkd, r.dsd, Q); fma4(dkd, r.ds, Qd);
      }
    }
  }
  put4(p.dv + j * p.lddv + hk * D, D, lane, dv, 1.f);
  put4(p.dk + j * p.lddk + hk * D, D, lane, dk, p.scale);
  if (DUAL) {
    put4(p.dvd + j * p.lddv + hk * D, D, lane, dvd, 1.f);
    put4(p.dkd + j * p.lddk + hk * D, D, lane, dkd, p.scale);
  }
}

dim3 warp_grid(int64_t rows) { return dim3(static_cast<unsigned>((rows + kWarps - 1) / kWarps)); }

}  // namespace

cudaError_t attn_rows_fwd(const AttnParams& p, bool dual, cudaStream_t s) {
  const dim3 g = warp_grid(static_cast<int64_t>(p.seq.rows) * p.Hq), b(32 * kWarps);
  return dual ? launch_k(rows_fwd_kernel<true>, g, b, 0, s, p)
              : launch_k(rows_fwd_kernel<false>, g, b, 0, s, p);
}

cudaError_t attn_rows_bwd(const AttnParams& p, bool dual, cudaStream_t s) {
  const dim3 gq = warp_grid(static_cast<int64_t>(p.seq.rows) * p.Hq), b(32 * kWarps);
  const dim3 gk = warp_grid(static_cast<int64_t>(p.seq.rows) * p.Hkv);
  cudaError_t e = dual ? launch_k(rows_bwd_q_kernel<true>, gq, b, 0, s, p)
                       : launch_k(rows_bwd_q_kernel<false>, gq, b, 0, s, p);
  if (e != cudaSuccess) return e;
  return dual ? launch_k(rows_bwd_kv_kernel<true>, gk, b, 0, s, p)
              : launch_k(rows_bwd_kv_kernel<false>, gk, b, 0, s, p);
}

}  // namespace mf
