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
// Layout.  A head is cut into units of eight elements, one a lane, so that both elements of every
// rotated pair are in one lane: in the half layout a rotated unit is four elements of the first
// half and their four partners, else eight neighbours.  A head takes the next power of two of
// lanes, and sums over a head are shuffles.
//
// What bounds the forward pass is memory.  Every warp reads ahead of its arithmetic by itself: it
// copies parts of rows into a ring of its own in shared memory (bulk copies), so that
// what is in flight does not depend on registers, and meets no other warp.  Plain loads left the
// memory idle two thirds of the time; a ring for a whole block cost more in barriers than the heads
// in arithmetic.  The cos and sin of a row's position are computed a pair a lane and kept in
// registers for all its heads.  Measured: 16 + 16 + 16 heads of 64 with tangents, 8192 rows,
// float32 to bf16, 302 MB in 50 us (6.1 TB/s, 89 % of a plain copy); 8 + 2 + 2 heads of 128,
// 40001 rows of bf16, 246 MB in 41 us (6.0 TB/s).
// What bounds the backward pass with norms is arithmetic whose latency 16 warps an SM do not cover
// (issue slots 57 % busy): 16 + 4 + 4 heads of 64 with tangents, 8192 rows, 185 MB in 53 us; 12 +
// 3 + 3 heads of 80 (10 of 16 lanes in use), 5003 rows of float32, 82 MB in 31 us.  A third block
// an SM spilled: 34 us for the last.
#include "attn_ops.h"
#include "device_math.cuh"
#include "launch.cuh"
#include "packed_rows.cuh"
#include "pair_math.cuh"

namespace mf {
namespace {

constexpr int kRopeWarps = 8;
constexpr int kRopeThreads = 32 * kRopeWarps;
// A warp's ring: stages, and bytes of one at most.  Heads of 64 with tangents, 8192 rows: forward
// 49.8 us with three stages of 4 KB (eight heads), 55.9 with two of 6 KB, 55.1 with four of 3 KB;
// backward 53.5 with two of 6 KB (eight heads), 56.9 and 58.9 with two and three of 4 KB.
constexpr int kFwdStages = 3, kFwdStage = 4 * 1024;
constexpr int kBwdStages = 2, kBwdStage = 6 * 1024;
constexpr int kRopeRing = kRopeWarps * (12 * 1024 + 512);          // of a block, two an SM
static_assert(kFwdStages * kFwdStage == 12 * 1024 && kBwdStages * kBwdStage == 12 * 1024);

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

// A lane's unit of a head: four pairs of elements.
struct Unit {
  int oa, ob;      // first elements of its two fours (vector form)
  int u;           // rotated units: first pair is 4 u; others: place 8 u behind the rotated part
  bool on, rot;    // in use; rotated
};

__device__ __forceinline__ Unit make_unit(const RopeParams& p, int lane) {
  Unit t;
  const int u = lane & (p.lanes - 1);
  const int nrot = (p.R / 2 + 3) / 4;
  t.rot = u < nrot;
  t.u = t.rot ? u : u - nrot;
  t.on = t.rot || p.R + 8 * t.u < p.D;
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

__device__ __forceinline__ void load4(const float* s, uint64_t& a, uint64_t& b) {
  const float4 f = *reinterpret_cast<const float4*>(s);
  a = pair(f.x, f.y);
  b = pair(f.z, f.w);
}
__device__ __forceinline__ void load4(const __nv_bfloat16* s, uint64_t& a, uint64_t& b) {
  const uint2 w = *reinterpret_cast<const uint2*>(s);
  a = pair(__uint_as_float(w.x << 16), __uint_as_float(w.x & 0xffff0000u));
  b = pair(__uint_as_float(w.y << 16), __uint_as_float(w.y & 0xffff0000u));
}
__device__ __forceinline__ void store4(float* d, uint64_t a, uint64_t b) {
  const float2 x = halves(a), y = halves(b);
  *reinterpret_cast<float4*>(d) = make_float4(x.x, x.y, y.x, y.y);
}
__device__ __forceinline__ void store4(__nv_bfloat16* d, uint64_t a, uint64_t b) {
  const float2 x = halves(a), y = halves(b);
  const __nv_bfloat162 lo = __floats2bfloat162_rn(x.x, x.y), hi = __floats2bfloat162_rn(y.x, y.y);
  *reinterpret_cast<uint2*>(d) = make_uint2(*reinterpret_cast<const uint32_t*>(&lo),
                                            *reinterpret_cast<const uint32_t*>(&hi));
}
__device__ __forceinline__ float as_f(float x) { return x; }
__device__ __forceinline__ float as_f(__nv_bfloat16 x) { return __bfloat162float(x); }

// A unit's eight elements from and to one head as four pairs, in memory order: v[0], v[1] from oa
// on, v[2], v[3] from ob on.  Units of whole eights move as vectors (VEC), others element by
// element, then in pair order (element e of the pair in v[e / 2], its partner in v[2 + e / 2]).
template <bool VEC, typename T>
__device__ __forceinline__ void load_unit(const RopeParams& p, const Unit& t, bool on, const T* h,
                                          uint64_t (&v)[4]) {
  if (VEC) {
    if (on) {
      load4(h + t.oa, v[0], v[1]);
      load4(h + t.ob, v[2], v[3]);
    }
  } else {
    float f[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const int i = unit_elem(p, t, e >> 2, e & 3);
      f[e] = on && i >= 0 ? as_f(h[i]) : 0.f;
    }
#pragma unroll
    for (int e = 0; e < 4; ++e) v[e] = pair(f[2 * e], f[2 * e + 1]);
  }
}
template <bool VEC, typename T>
__device__ __forceinline__ void store_unit(const RopeParams& p, const Unit& t, T* h,
                                           const uint64_t (&v)[4]) {
  if (VEC) {
    store4(h + t.oa, v[0], v[1]);
    store4(h + t.ob, v[2], v[3]);
  } else {
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const float2 f = halves(v[e]);
      const int i = unit_elem(p, t, e >> 1, 2 * (e & 1)), j = unit_elem(p, t, e >> 1, 2 * (e & 1) + 1);
      if (i >= 0) h[i] = to_t<T>(f.x);
      if (j >= 0) h[j] = to_t<T>(f.y);
    }
  }
}

// cos and sin of a lane's four pairs at the current row (sin negated for the transposed turn).
struct Turns {
  uint64_t c[2], s[2];
};
// Turns a unit's pairs: elements of v[0], v[1] with those of v[2], v[3], or neighbours where the
// interleaved layout moves as vectors.
template <bool VEC>
__device__ __forceinline__ void rotate(const RopeParams& p, uint64_t (&v)[4], const Turns& t) {
  const uint64_t neg = pair(-1.f, -1.f);
  if (!VEC || p.half) {
#pragma unroll
    for (int e = 0; e < 2; ++e) {
      const uint64_t x = v[e], y = v[2 + e];
      v[e] = fma2(mul2(y, t.s[e]), neg, mul2(x, t.c[e]));
      v[2 + e] = fma2(y, t.c[e], mul2(x, t.s[e]));
    }
  } else {
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const float2 x = halves(v[e]), c2 = halves(t.c[e >> 1]), s2 = halves(t.s[e >> 1]);
      const float c = e & 1 ? c2.y : c2.x, s = e & 1 ? s2.y : s2.x;
      v[e] = pair(x.x * c - x.y * s, x.y * c + x.x * s);
    }
  }
}

__device__ __forceinline__ float sum2(uint64_t a) {
  const float2 f = halves(a);
  return f.x + f.y;
}
// Sum over the lanes of a head (every lane of the warp takes part).
__device__ __forceinline__ float head_sum(float v, int lanes) {
  for (int o = lanes >> 1; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
  return v;
}

// ---- a warp's ring ----------------------------------------------------------------------------
__device__ __forceinline__ uint32_t saddr(const void* p) {
  return static_cast<uint32_t>(__cvta_generic_to_shared(p));
}
__device__ __forceinline__ bool try_phase(uint32_t bar, uint32_t parity) {
  uint32_t ok;
  asm volatile(
      "{\n\t.reg .pred p, q;\n\t"
      "mbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2;\n\t"
      "vote.sync.all.pred q, p, 0xffffffff;\n\t"
      "selp.u32 %0, 1, 0, q;\n\t}"
      : "=r"(ok)
      : "r"(bar), "r"(parity)
      : "memory");
  return ok != 0;
}
// A warp's bounded wait (2 s at 2 GHz).
__device__ __forceinline__ bool phase_wait(uint32_t bar, uint32_t parity, int* status) {
  if (try_phase(bar, parity)) return true;
  const long long t0 = clock64();
  while (!try_phase(bar, parity)) {
    if (__any_sync(0xffffffffu, clock64() - t0 > 4000000000LL)) {
      if (status) atomicMax(status, DEV_TIMEOUT);
      return false;
    }
  }
  return true;
}

struct RowBuf {
  const char* base;     // row 0, head 0
  int64_t ld;           // bytes a row
  int esize, heads;     // element size, heads that are needed
};

// This warp's parts of rows in order.  A unit of work is a row, or a run of `run` parts of one when
// there are fewer rows than warps; part c holds heads c hc .. c hc + hc - 1.
struct Cursor {
  int64_t left;         // units still to come, this one included
  int row, first, c;    // row, first part of its run, current part
};
__device__ __forceinline__ Cursor first_part(const RopeParams& p, int total) {
  const int64_t units = static_cast<int64_t>(total) * p.splits;
  const int64_t g = static_cast<int64_t>(blockIdx.x) * kRopeWarps + (threadIdx.x >> 5);
  const int64_t all = static_cast<int64_t>(gridDim.x) * kRopeWarps;
  Cursor k;
  k.left = units > g ? (units - g + all - 1) / all : 0;
  k.row = static_cast<int>(g / p.splits);
  k.first = k.c = static_cast<int>(g % p.splits) * p.run;
  return k;
}
// The next part; true when it is in another unit.
__device__ __forceinline__ bool next_part(const RopeParams& p, Cursor& k) {
  if (++k.c < min(k.first + p.run, p.parts)) return false;
  --k.left;
  k.row += p.step_row;
  k.first += p.step_split * p.run;
  if (k.first >= p.splits * p.run) {
    k.first -= p.splits * p.run;
    ++k.row;
  }
  k.c = k.first;
  return true;
}

// The warp's ring and what it works with.
template <int NARR, int STAGES>
struct Reader {
  const RopeParams& p;
  RowBuf buf[NARR];
  char* ring;            // its stages, then cos and sin tables
  uint32_t bars;         // a barrier a stage
  int lane, H, st, got;
  uint32_t ph;
  Cursor ahead;          // next part to be copied
  int issued;

  __device__ __forceinline__ Reader(const RopeParams& p_, char* ring_, uint32_t bars_, int total)
      : p(p_), ring(ring_), bars(bars_), lane(threadIdx.x & 31), H(p_.Hq + p_.Hkv + p_.Hc), st(0),
        got(0), ph(0), ahead(first_part(p_, total)), issued(0) {}
  // Copies the next part into stage s (whose old contents every lane has read).
  __device__ __forceinline__ void issue(int s) {
    if (ahead.left <= 0) return;
    const int h0 = ahead.c * p.hc, h1 = min(h0 + p.hc, H);
    if (lane == 0) {
      const uint32_t bar = bars + 8 * s;
      int n[NARR], bytes = 0;
#pragma unroll
      for (int k = 0; k < NARR; ++k) {
        n[k] = max(min(h1, buf[k].heads) - h0, 0) * p.D * buf[k].esize;
        bytes += n[k];
      }
      asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;" ::"r"(bar), "r"(bytes)
                   : "memory");
      uint32_t at = saddr(ring) + s * p.stage_bytes;
#pragma unroll
      for (int k = 0; k < NARR; ++k) {
        const char* src = buf[k].base + ahead.row * buf[k].ld + static_cast<int64_t>(h0) * p.D * buf[k].esize;
        if (n[k] > 0)
          asm volatile(
              "cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];" ::"r"(at),
              "l"(src), "r"(n[k]), "r"(bar)
              : "memory");
        at += p.hc * p.D * buf[k].esize;
      }
    }
    __syncwarp();
    ++issued;
    next_part(p, ahead);
  }
  // Waits for the next stage.
  __device__ __forceinline__ bool next() { return phase_wait(bars + 8 * st, ph, p.status); }
  __device__ __forceinline__ const char* stage() const { return ring + st * p.stage_bytes; }
  // Gives the stage back and copies on.
  __device__ __forceinline__ void done() {
    __syncwarp();
    ++got;
    issue(st);
    if (++st == STAGES) {
      st = 0;
      ph ^= 1;
    }
  }
  // Given up: what was issued still has to land.
  __device__ __forceinline__ void drain() {
    for (; got < issued; ++got) {
      const long long t0 = clock64();
      while (!try_phase(bars + 8 * st, ph) && clock64() - t0 < 4000000000LL) {
      }
      if (++st == STAGES) {
        st = 0;
        ph ^= 1;
      }
    }
  }
};

// Positions of a warp's next 32 units, one a lane.
struct Positions {
  int pos, have;
};
__device__ __forceinline__ int next_pos(const RopeParams& p, Positions& s, const Cursor& k, int total) {
  if (s.have == 0) {
    const int lane = threadIdx.x & 31;
    const int64_t all = static_cast<int64_t>(gridDim.x) * kRopeWarps;
    const int64_t unit = static_cast<int64_t>(k.row) * p.splits + k.first / p.run + lane * all;
    const int row = static_cast<int>(min(unit / p.splits, static_cast<int64_t>(total) - 1));
    s.pos = p.pos ? p.pos[row] : row - seq_begin(p.seq, row);
    s.have = 32;
  }
  const int r = __shfl_sync(0xffffffffu, s.pos, 32 - s.have);
  --s.have;
  return r;
}

// cos and sin at a position: a pair a lane, handed round through the warp's table.
__device__ __forceinline__ Turns make_turns(const RopeParams& p, const Unit& t, int pos, float* tab,
                                            float sign) {
  const int lane = threadIdx.x & 31, pairs = (p.R / 2 + 3) / 4 * 4;
  __syncwarp();
  for (int q = lane; q < pairs; q += 32) {
    float c = 1.f, s = 0.f;
    if (q < p.R / 2) {
      turn_cos_sin(pos, p.phase[q], c, s);
      c *= p.mscale;
      s *= p.mscale * sign;
    }
    tab[q] = c;
    tab[64 + q] = s;
  }
  __syncwarp();
  Turns r{};
  if (t.rot) {
    load4(tab + 4 * t.u, r.c[0], r.c[1]);
    load4(tab + 64 + 4 * t.u, r.s[0], r.s[1]);
  }
  return r;
}

// Shared memory of a block: every warp's ring, barriers, and the gains [gq | gk | gq' | gk'][D].
struct RopeShared {
  uint64_t bars[kRopeWarps][kFwdStages];
  float gains[4][128];
};
__device__ __forceinline__ void rope_start(const RopeParams& p, RopeShared& sh) {
  if (threadIdx.x < kRopeWarps * kFwdStages) {
    asm volatile("mbarrier.init.shared::cta.b64 [%0], 1;" ::"r"(saddr(&sh.bars[0][0]) + 8 * threadIdx.x));
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  pdl_entry();
  if (p.gq)
    for (int i = threadIdx.x; i < 4 * p.D; i += kRopeThreads) {
      const int k = i / p.D, e = i % p.D;
      const float* g = k == 0 ? p.gq : k == 1 ? p.gk : k == 2 ? p.gqd : p.gkd;
      sh.gains[k][e] = g ? g[e] : 0.f;
    }
  __syncthreads();
}
constexpr int kTurnBytes = 2 * 64 * static_cast<int>(sizeof(float));
__device__ __forceinline__ int warp_bytes(const RopeParams& p, int stages) {
  return stages * p.stage_bytes + kTurnBytes;
}

template <typename Tx, typename Ty, bool DUAL, bool NORM, bool VEC>
__device__ __forceinline__ void fwd_rows(const RopeParams& p, char* ring, RopeShared& sh) {
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int H = p.Hq + p.Hkv + p.Hc, Hn = p.Hq + p.Hkv, total = seq_total(p.seq);
  constexpr int STAGES = kFwdStages;
  Reader<DUAL ? 2 : 1, STAGES> rd(p, ring + warp * warp_bytes(p, STAGES), saddr(sh.bars[warp]), total);
  rd.buf[0] = {static_cast<const char*>(p.x), p.ldx * static_cast<int>(sizeof(Tx)), sizeof(Tx), H};
  if constexpr (DUAL) rd.buf[1] = {static_cast<const char*>(p.xd), rd.buf[0].ld, sizeof(Tx), H};
#pragma unroll
  for (int s = 0; s < STAGES; ++s) rd.issue(s);
  float* tab = reinterpret_cast<float*>(rd.ring + STAGES * p.stage_bytes);
  const Unit t = make_unit(p, lane);
  const int sub = lane / p.lanes, hpw = 32 / p.lanes, half = p.hc * p.D;
  const float invD = 1.f / static_cast<float>(p.D);
  Positions ps{0, 0};
  Turns turns{};
  bool fresh = true;
  for (Cursor k = first_part(p, total); k.left > 0; fresh = next_part(p, k)) {
    if (fresh) turns = make_turns(p, t, next_pos(p, ps, k, total), tab, 1.f);
    if (!rd.next()) break;
    const Tx* sx = reinterpret_cast<const Tx*>(rd.stage());
    const int h0 = k.c * p.hc, n = min(p.hc, H - h0);
    Ty* y = static_cast<Ty*>(p.y) + k.row * p.ldy + static_cast<int64_t>(h0) * p.D;
    Ty* yd = DUAL ? static_cast<Ty*>(p.yd) + k.row * p.ldy + static_cast<int64_t>(h0) * p.D : nullptr;
    for (int hl = sub; hl - sub < n; hl += hpw) {
      const bool on = t.on && hl < n;
      const int e0 = hl * p.D, h = h0 + hl;
      uint64_t v[4] = {}, d[4] = {};
      load_unit<VEC>(p, t, on, sx + e0, v);
      if (DUAL) load_unit<VEC>(p, t, on, sx + half + e0, d);
      if (NORM) {
        uint64_t q2 = 0, q1 = 0;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          q2 = fma2(v[e], v[e], q2);
          if (DUAL) q1 = fma2(v[e], d[e], q1);
        }
        const float s2 = head_sum(sum2(q2), p.lanes), s1 = DUAL ? head_sum(sum2(q1), p.lanes) : 0.f;
        if (on && h < Hn) {
          const float r = rsqrtf(s2 * invD + p.eps);
          const float rt = DUAL ? -r * r * r * s1 * invD : 0.f;
          const uint64_t r2 = pair(r, r), rt2 = pair(rt, rt);
          const int gi = h < p.Hq ? 0 : 1;
          uint64_t g[4], gd[4];
          load_unit<VEC>(p, t, true, sh.gains[gi], g);
          if (DUAL) load_unit<VEC>(p, t, true, sh.gains[2 + gi], gd);
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const uint64_t nv = mul2(v[e], r2);
            if (DUAL) d[e] = fma2(gd[e], nv, mul2(g[e], fma2(d[e], r2, mul2(v[e], rt2))));
            v[e] = mul2(g[e], nv);
          }
        }
      }
      if (on) {
        if (h < Hn && t.rot) {
          rotate<VEC>(p, v, turns);
          if (DUAL) rotate<VEC>(p, d, turns);
        }
        store_unit<VEC>(p, t, y + e0, v);
        if (DUAL) store_unit<VEC>(p, t, yd + e0, d);
      }
    }
    rd.done();
  }
  rd.drain();
}

template <typename Tx, typename Ty, bool DUAL, bool NORM>
__global__ void __launch_bounds__(kRopeThreads, 2)
    qk_rope_fwd_kernel(const __grid_constant__ RopeParams p) {
  extern __shared__ __align__(128) char ring[];
  __shared__ __align__(16) RopeShared sh;
  rope_start(p, sh);
  if (p.vec) fwd_rows<Tx, Ty, DUAL, NORM, true>(p, ring, sh);
  else fwd_rows<Tx, Ty, DUAL, NORM, false>(p, ring, sh);
}

// acc: dgq, dgk and, with tangents, dgq', dgk' of this lane's elements.
template <typename Tx, typename Ty, bool DUAL, bool NORM, bool VEC, int NACC>
__device__ __forceinline__ void bwd_rows(const RopeParams& p, char* ring, RopeShared& sh,
                                         uint64_t (&acc)[NACC][4]) {
  constexpr int NARR = (DUAL ? 2 : 1) * (NORM ? 2 : 1);
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int H = p.Hq + p.Hkv + p.Hc, Hn = p.Hq + p.Hkv, total = seq_total(p.seq);
  constexpr int STAGES = kBwdStages;
  Reader<NARR, STAGES> rd(p, ring + warp * warp_bytes(p, STAGES), saddr(sh.bars[warp]), total);
  const RowBuf dy{static_cast<const char*>(p.dy), p.lddy * static_cast<int>(sizeof(Ty)), sizeof(Ty), H};
  const RowBuf xb{static_cast<const char*>(p.x), p.ldx * static_cast<int>(sizeof(Tx)), sizeof(Tx), Hn};
  rd.buf[0] = dy;
  if constexpr (DUAL) rd.buf[1] = {static_cast<const char*>(p.dyd), dy.ld, sizeof(Ty), H};
  if constexpr (NORM) rd.buf[DUAL ? 2 : 1] = xb;
  if constexpr (NORM && DUAL) rd.buf[3] = {static_cast<const char*>(p.xd), xb.ld, sizeof(Tx), Hn};
#pragma unroll
  for (int s = 0; s < STAGES; ++s) rd.issue(s);
  float* tab = reinterpret_cast<float*>(rd.ring + STAGES * p.stage_bytes);
  const Unit t = make_unit(p, lane);
  const int sub = lane / p.lanes, hpw = 32 / p.lanes, half = p.hc * p.D;
  const float invD = 1.f / static_cast<float>(p.D);
  Positions ps{0, 0};
  Turns turns{};
  bool fresh = true;
  for (Cursor k = first_part(p, total); k.left > 0; fresh = next_part(p, k)) {
    if (fresh) turns = make_turns(p, t, next_pos(p, ps, k, total), tab, -1.f);   // transposed
    if (!rd.next()) break;
    const Ty* sdy = reinterpret_cast<const Ty*>(rd.stage());
    const Tx* sx = reinterpret_cast<const Tx*>(sdy + (DUAL ? 2 : 1) * half);
    const int h0 = k.c * p.hc, n = min(p.hc, H - h0);
    Ty* dx = static_cast<Ty*>(p.dx) + k.row * p.lddx + static_cast<int64_t>(h0) * p.D;
    Ty* dxd = DUAL ? static_cast<Ty*>(p.dxd) + k.row * p.lddx + static_cast<int64_t>(h0) * p.D : nullptr;
    for (int hl = sub; hl - sub < n; hl += hpw) {
      const bool on = t.on && hl < n;
      const int e0 = hl * p.D, h = h0 + hl;
      const bool normed = NORM && on && h < Hn;
      uint64_t v[4] = {}, d[4] = {};
      load_unit<VEC>(p, t, on, sdy + e0, v);
      if (DUAL) load_unit<VEC>(p, t, on, sdy + half + e0, d);
      if (on && h < Hn && t.rot) {
        rotate<VEC>(p, v, turns);
        if (DUAL) rotate<VEC>(p, d, turns);
      }
      if (NORM) {
        uint64_t x[4] = {}, xd[4] = {};
        load_unit<VEC>(p, t, normed, sx + e0, x);
        if (DUAL) load_unit<VEC>(p, t, normed, sx + half + e0, xd);
        const int gi = h < p.Hq ? 0 : 1;
        uint64_t q2 = 0, q1 = 0, qm = 0, qd = 0;
        {
          uint64_t g[4] = {}, gd[4] = {};
          load_unit<VEC>(p, t, normed, sh.gains[gi], g);
          if (DUAL) load_unit<VEC>(p, t, normed, sh.gains[2 + gi], gd);
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const uint64_t a = mul2(g[e], v[e]);
            q2 = fma2(x[e], x[e], q2);
            qm = fma2(x[e], a, qm);
            if (DUAL) {
              q1 = fma2(x[e], xd[e], q1);
              qd = fma2(xd[e], a, qd);
              qd = fma2(x[e], fma2(gd[e], v[e], mul2(g[e], d[e])), qd);
            }
          }
        }
        const float s2 = head_sum(sum2(q2), p.lanes), m = head_sum(sum2(qm), p.lanes) * invD;
        const float s1 = DUAL ? head_sum(sum2(q1), p.lanes) : 0.f;
        const float md = DUAL ? head_sum(sum2(qd), p.lanes) * invD : 0.f;
        if (normed) {
          const float r = rsqrtf(s2 * invD + p.eps), r3 = r * r * r;
          const float rt = DUAL ? -r3 * s1 * invD : 0.f;
          const float k0 = -r3 * m, k1 = -3.f * r * r * rt * m - r3 * md;
          const uint64_t r2 = pair(r, r), rt2 = pair(rt, rt), k02 = pair(k0, k0), k12 = pair(k1, k1);
          // the gains are read again rather than kept across the sums: registers
          asm volatile("" ::: "memory");
          uint64_t g[4], gd[4];
          load_unit<VEC>(p, t, true, sh.gains[gi], g);
          if (DUAL) load_unit<VEC>(p, t, true, sh.gains[2 + gi], gd);
          // query and key heads' sums apart: a NaN of the one does not reach the other
          const bool query = h < p.Hq;
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const uint64_t dyv = v[e], nv = mul2(x[e], r2), gw = mul2(dyv, nv), a = mul2(g[e], dyv);
            acc[0][e] = add2(query ? gw : 0, acc[0][e]);
            acc[NORM ? 1 : 0][e] = add2(query ? 0 : gw, acc[NORM ? 1 : 0][e]);
            v[e] = fma2(r2, a, mul2(k02, x[e]));
            if (DUAL) {
              const uint64_t gt = fma2(d[e], nv, mul2(dyv, fma2(xd[e], r2, mul2(x[e], rt2))));
              constexpr int iq = NACC - 2 > 0 ? NACC - 2 : 0;
              acc[iq][e] = add2(query ? gt : 0, acc[iq][e]);
              acc[NACC - 1][e] = add2(query ? 0 : gt, acc[NACC - 1][e]);
              const uint64_t b = fma2(gd[e], dyv, mul2(g[e], d[e]));
              d[e] = fma2(rt2, a, fma2(r2, b, fma2(k12, x[e], mul2(k02, xd[e]))));
            }
          }
        }
      }
      if (on) {
        store_unit<VEC>(p, t, dx + e0, v);
        if (DUAL) store_unit<VEC>(p, t, dxd + e0, d);
      }
    }
    rd.done();
  }
  rd.drain();
}

template <typename Tx, typename Ty, bool DUAL, bool NORM>
__global__ void __launch_bounds__(kRopeThreads, 2)
    qk_rope_bwd_kernel(const __grid_constant__ RopeParams p) {
  constexpr int NA = DUAL ? 4 : 2;
  extern __shared__ __align__(128) char ring[];
  __shared__ __align__(16) RopeShared sh;
  rope_start(p, sh);
  uint64_t acc[NORM ? NA : 1][4] = {};
  if (p.vec) bwd_rows<Tx, Ty, DUAL, NORM, true>(p, ring, sh, acc);
  else bwd_rows<Tx, Ty, DUAL, NORM, false>(p, ring, sh, acc);
  if (NORM) {
    // lanes of the same unit, then the block's warps, in a fixed order; the rings are free
    __syncthreads();
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const Unit t = make_unit(p, lane);
    float* sums = reinterpret_cast<float*>(ring);
#pragma unroll
    for (int k = 0; k < NA; ++k)
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const float2 f = halves(acc[NORM ? k : 0][e >> 1]);
        float v = e & 1 ? f.y : f.x;
        for (int o = p.lanes; o < 32; o <<= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
        // vector units are in memory order, others in pair order
        const int i = !p.vec ? unit_elem(p, t, e >> 2, e & 3) : t.on ? (e < 4 ? t.oa + e : t.ob + e - 4) : -1;
        if (lane < p.lanes && i >= 0) sums[(warp * NA + k) * p.D + i] = v;
      }
    __syncthreads();
    float* part = p.part + static_cast<int64_t>(blockIdx.x) * NA * p.D;
    for (int i = threadIdx.x; i < NA * p.D; i += kRopeThreads) {
      float v = 0.f;
      for (int j = 0; j < kRopeWarps; ++j) v += sums[j * NA * p.D + i];
      part[i] = v;
    }
  }
}

// Sum of the blocks' partial gain gradients in a fixed order: 32 columns a block, 32 threads a
// column, their sums by halves.
__global__ void __launch_bounds__(1024)
    rope_gain_final_kernel(int nblk, int D, int NA, const float* __restrict__ part,
                           float* __restrict__ d0, float* __restrict__ d1, float* __restrict__ d2,
                           float* __restrict__ d3) {
  pdl_entry();
  __shared__ float s[32][33];
  const int tx = threadIdx.x & 31, ty = threadIdx.x >> 5;
  const int col = blockIdx.x * 32 + tx;
  float v = 0.f;
  if (col < NA * D) {
#pragma unroll 4
    for (int j = ty; j < nblk; j += 32) v += part[static_cast<int64_t>(j) * NA * D + col];
  }
  s[ty][tx] = v;
  __syncthreads();
  // warp ty adds up column ty of the block
  float sum = s[tx][ty];
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
  const int c = blockIdx.x * 32 + ty;
  if (tx == 0 && c < NA * D) {
    const int k = c / D;
    (k == 0 ? d0 : k == 1 ? d1 : k == 2 ? d2 : d3)[c % D] = sum;
  }
}

template <auto kernel>
cudaError_t launch_ring(const RopeParams& p, int grid, cudaStream_t s) {
  static PerDeviceOnce once;
  const cudaError_t e = once.run([](int&) {
    return cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, kRopeRing);
  });
  if (e != cudaSuccess) return e;
  return launch_k(kernel, dim3(grid), dim3(kRopeThreads), p.ring_bytes, s, p);
}

template <typename Tx, typename Ty, bool BWD>
cudaError_t launch_rope(const RopeParams& p, bool dual, bool norm, int grid, cudaStream_t s) {
  if constexpr (BWD) {
    if (dual) return norm ? launch_ring<qk_rope_bwd_kernel<Tx, Ty, true, true>>(p, grid, s)
                          : launch_ring<qk_rope_bwd_kernel<Tx, Ty, true, false>>(p, grid, s);
    return norm ? launch_ring<qk_rope_bwd_kernel<Tx, Ty, false, true>>(p, grid, s)
                : launch_ring<qk_rope_bwd_kernel<Tx, Ty, false, false>>(p, grid, s);
  } else {
    if (dual) return norm ? launch_ring<qk_rope_fwd_kernel<Tx, Ty, true, true>>(p, grid, s)
                          : launch_ring<qk_rope_fwd_kernel<Tx, Ty, true, false>>(p, grid, s);
    return norm ? launch_ring<qk_rope_fwd_kernel<Tx, Ty, false, true>>(p, grid, s)
                : launch_ring<qk_rope_fwd_kernel<Tx, Ty, false, false>>(p, grid, s);
  }
}

template <bool BWD>
cudaError_t launch_types(const RopeParams& p, bool x_bf16, bool y_bf16, bool dual, bool norm, int grid,
                         cudaStream_t s) {
  return !x_bf16 && !y_bf16 ? launch_rope<float, float, BWD>(p, dual, norm, grid, s)
         : !x_bf16          ? launch_rope<float, __nv_bfloat16, BWD>(p, dual, norm, grid, s)
                            : launch_rope<__nv_bfloat16, __nv_bfloat16, BWD>(p, dual, norm, grid, s);
}

}  // namespace

cudaError_t qk_rope(RopeParams p, bool bwd, bool x_bf16, bool y_bf16, cudaStream_t s) {
  const bool norm = p.gq != nullptr, dual = bwd ? p.dyd != nullptr : p.xd != nullptr;
  const int lanes_units = (p.R / 2 + 3) / 4 + (p.D - p.R + 7) / 8;
  p.lanes = 1;
  while (p.lanes < lanes_units) p.lanes *= 2;
  p.vec = p.R % 8 == 0;
  // heads of a part: what fills a stage, whole warps of them
  const int two = dual ? 2 : 1, xs = x_bf16 ? 2 : 4, ys = y_bf16 ? 2 : 4;
  const int head = p.D * two * (bwd ? ys + (norm ? xs : 0) : xs);     // bytes, at most 2 KB
  const int H = p.Hq + p.Hkv + p.Hc, hpw = 32 / p.lanes;
  int hc = (bwd ? kBwdStage : kFwdStage) / head;
  if (hc > hpw) hc -= hc % hpw;
  p.hc = hc < H ? hc : H;
  p.parts = (H + p.hc - 1) / p.hc;
  p.stage_bytes = (p.hc * head + 127) / 128 * 128;
  // a warp a row; with fewer than eight rows a warp, runs of a row's parts, so that the last round
  // of units is a small part of all
  const int64_t warps = static_cast<int64_t>(kRopeMaxBlocks) * kRopeWarps;
  const int64_t want = (8 * warps + p.seq.rows - 1) / p.seq.rows;
  p.splits = want < p.parts ? static_cast<int>(want) : p.parts;
  p.run = (p.parts + p.splits - 1) / p.splits;
  p.splits = (p.parts + p.run - 1) / p.run;
  const int64_t blocks = (static_cast<int64_t>(p.seq.rows) * p.splits + kRopeWarps - 1) / kRopeWarps;
  const int grid = static_cast<int>(blocks < kRopeMaxBlocks ? blocks : kRopeMaxBlocks);
  p.step_row = grid * kRopeWarps / p.splits;
  p.step_split = grid * kRopeWarps % p.splits;
  const int NA = dual ? 4 : 2;
  const int rings = kRopeWarps * ((bwd ? kBwdStages : kFwdStages) * p.stage_bytes + kTurnBytes);
  const int sums = bwd && norm ? kRopeWarps * NA * p.D * static_cast<int>(sizeof(float)) : 0;
  p.ring_bytes = rings > sums ? rings : sums;
  const cudaError_t e = bwd ? launch_types<true>(p, x_bf16, y_bf16, dual, norm, grid, s)
                            : launch_types<false>(p, x_bf16, y_bf16, dual, norm, grid, s);
  if (e != cudaSuccess || !bwd || !norm) return e;
  return launch_k(rope_gain_final_kernel, dim3((NA * p.D + 31) / 32), dim3(1024), 0, s, grid, p.D,
                  NA, static_cast<const float*>(p.part), p.dgq, p.dgk, p.dgqd, p.dgkd);
}

}  // namespace mf
