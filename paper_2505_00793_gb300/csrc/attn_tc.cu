// Causal attention with grouped heads over packed sequences on the 5th-generation tensor cores
// (tcgen05 + TMEM + TMA), with its forward tangent and its backward pass: the kernels behind
// mf_attn_fwd and mf_attn_bwd.  Formulas in mixflow.h.
//
// Tiles run along the packed row axis, 128 rows each, whatever sequences they hold: row r of a
// tile attends to rows lo(r) .. r, lo(r) the first row of its sequence, so a tile walks the
// other side from its first row's lo to its own end and nothing is padded, however short the
// sequences are.  The grid depends on the number of rows alone, and a captured call serves
// any lengths.  Only tiles on the diagonal or across a sequence's border compare positions
// ("mixed" tiles).
//
// Softmax operands stay in TMEM.  The warps that read a tile's scores S (TMEM) write P as bf16
// over the same columns, and P is the A operand of the next product from there: no shared
// memory is moved for it, and the products of one CTA, issued by one thread in order, need no
// barrier between reading P and overwriting it with the next scores.
//
// Values of masked places: a product with a zero of P still meets them (0 * inf = NaN).  In
// mixed tiles the warp that issues the products first looks over the rows that P or dS will
// multiply, puts zeros in place of what is not finite and notes those rows; rows that attend to
// a noted one get NaN, others are as if it was not there.
//
// Every wait is bounded (2 s), as in flash_tc.cu.
#include "attn_ops.h"
#include "attn_tc_util.cuh"
#include "packed_rows.cuh"

namespace mf {
namespace {

constexpr int TR = 128;                       // rows of a CTA's own tile (MMA M)
constexpr int ATOM64 = 64 * 128, ATOM128 = 128 * 128;   // bytes of [64 or 128 rows][64] bf16
constexpr float LOG2E = 1.44269504088896341f, LN2 = 0.693147180559945309f;

// MN-major operand of 64-column boxes of 128-byte rows, `box` bytes apart.
__device__ __forceinline__ uint64_t sdesc_mn(uint32_t saddr, int box) {
  return (sdesc_mn_sw128(saddr) & ~(0x3FFFull << 16)) | (static_cast<uint64_t>(box >> 4) << 16);
}

// D[tmem] (+)= A[tmem] B, A bf16: lane = row, two consecutive K elements a column.
__device__ __forceinline__ void mma_ts(uint32_t d, uint32_t a, uint64_t bd, uint32_t idesc,
                                       uint32_t acc) {
  asm volatile(
      "{\n\t.reg .pred p;\n\t"
      "setp.ne.b32 p, %4, 0;\n\t"
      "tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n\t}" ::"r"(d),
      "r"(a), "l"(bd), "r"(idesc), "r"(acc));
}

__device__ __forceinline__ void tmem_st8(uint32_t t, const uint32_t* v) {
  asm volatile("tcgen05.st.sync.aligned.32x32b.x8.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8};" ::"r"(t),
               "r"(v[0]), "r"(v[1]), "r"(v[2]), "r"(v[3]), "r"(v[4]), "r"(v[5]), "r"(v[6]), "r"(v[7])
               : "memory");
}
__device__ __forceinline__ void tmem_st16u(uint32_t t, const uint32_t* v) {
  asm volatile(
      "tcgen05.st.sync.aligned.32x32b.x16.b32 [%0], "
      "{%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16};" ::"r"(t),
      "r"(v[0]), "r"(v[1]), "r"(v[2]), "r"(v[3]), "r"(v[4]), "r"(v[5]), "r"(v[6]), "r"(v[7]),
      "r"(v[8]), "r"(v[9]), "r"(v[10]), "r"(v[11]), "r"(v[12]), "r"(v[13]), "r"(v[14]), "r"(v[15])
      : "memory");
}
__device__ __forceinline__ void tmem_wait_st() {
  asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory");
}
__device__ __forceinline__ float ex2(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}

// ---- sequences of a tile's rows -------------------------------------------------------------
// Borders inside the tile as a bit per row (a sequence starts there), the start of the first
// row's sequence and the end of the last row's.
struct SeqTile {
  int lo0, hi1;
  uint32_t bits[4];
};

// Row count of the batch that belongs to sequences is read by every thread; the table is filled
// by all threads of the block between two barriers.
__device__ __forceinline__ void seq_tile_init(const SeqRows& s, int row0, SeqTile& t) {
  if (threadIdx.x < 4) t.bits[threadIdx.x] = 0;
  if (threadIdx.x == 4) t.lo0 = s.start ? 0 : row0 - row0 % s.len;
  if (threadIdx.x == 5) t.hi1 = s.start ? s.rows : (row0 + TR - 1) - (row0 + TR - 1) % s.len + s.len;
}
__device__ __forceinline__ void seq_tile_fill(const SeqRows& s, int row0, SeqTile& t, int threads) {
  if (!s.start) {
    const int p = threadIdx.x;
    if (p > 0 && p < TR && (row0 + p) % s.len == 0) atomicOr(&t.bits[p >> 5], 1u << (p & 31));
    return;
  }
  // long tables: from the first row's sequence on
  const int first = s.n > 2048 ? seq_find(s, row0) : 0;
  for (int i = first + static_cast<int>(threadIdx.x); i <= s.n; i += threads) {
    const int v = s.start[i];
    if (v <= row0) {
      atomicMax(&t.lo0, v);
    } else if (v - row0 < TR) {
      atomicOr(&t.bits[(v - row0) >> 5], 1u << ((v - row0) & 31));
    } else {
      atomicMin(&t.hi1, v);
      break;
    }
  }
}
// First row of row0 + r's sequence, and the row behind its last.
__device__ __forceinline__ int tile_lo(const SeqTile& t, int row0, int r) {
  int w = r >> 5;
  uint32_t m = t.bits[w] & (0xffffffffu >> (31 - (r & 31)));
  while (!m && w > 0) m = t.bits[--w];
  return m ? row0 + w * 32 + 31 - __clz(m) : t.lo0;
}
__device__ __forceinline__ int tile_hi(const SeqTile& t, int row0, int r) {
  int w = r >> 5;
  uint32_t m = (r & 31) == 31 ? 0u : t.bits[w] & (0xffffffffu << ((r & 31) + 1));
  while (!m && w < 3) m = t.bits[++w];
  return m ? row0 + w * 32 + __ffs(m) - 1 : t.hi1;
}

// ---- non-finite values of a mixed tile --------------------------------------------------------
// A warp looks over `atoms` blocks of `rows` 128-byte rows of bf16, zeroes what is not finite
// and sets the bit of its row in bad[].  0 * x is zero for every finite x and NaN otherwise, so
// one multiply-add a pair tells whether there is anything to do.
__device__ __forceinline__ void scrub(uint8_t* base, int rows, int atoms, uint32_t* bad, int lane) {
  if (lane < 4) bad[lane] = 0;
  const __nv_bfloat162 z = __float2bfloat162_rn(0.f);
  __nv_bfloat162 acc = z;
  const uint4* p = reinterpret_cast<const uint4*>(base);
  const int n = rows * atoms * 8;
#pragma unroll 8
  for (int i = lane; i < n; i += 32) {
    const uint4 w = p[i];
    acc = __hfma2(*reinterpret_cast<const __nv_bfloat162*>(&w.x), z, acc);
    acc = __hfma2(*reinterpret_cast<const __nv_bfloat162*>(&w.y), z, acc);
    acc = __hfma2(*reinterpret_cast<const __nv_bfloat162*>(&w.z), z, acc);
    acc = __hfma2(*reinterpret_cast<const __nv_bfloat162*>(&w.w), z, acc);
  }
  const bool clean = __low2float(acc) == 0.f && __high2float(acc) == 0.f;
  __syncwarp();
  if (!__all_sync(0xffffffffu, clean)) {
    for (int i = lane; i < n; i += 32) {
      uint4 w = p[i];
      uint32_t* u = reinterpret_cast<uint32_t*>(&w);
      bool hit = false;
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        if ((u[k] & 0x7f80u) == 0x7f80u) { u[k] &= 0xffff0000u; hit = true; }
        if ((u[k] & 0x7f800000u) == 0x7f800000u) { u[k] &= 0xffffu; hit = true; }
      }
      if (hit) {
        reinterpret_cast<uint4*>(base)[i] = w;
        const int row = (i >> 3) % rows;
        atomicOr(&bad[row >> 5], 1u << (row & 31));
      }
    }
    fence_async_smem();
  }
  __syncwarp();
}

// ---- forward ------------------------------------------------------------------------------------
// One CTA per (query head, 128 rows): warp 0 loads (Q once, then key tiles into a ring of K and a
// ring of V), warp 1 owns TMEM, looks over mixed V tiles and issues the products, warps 2..5 hold
// a row a thread.  The tangent shares the operands: Q [K | K']^T -> [S | Q K'^T], then Q' K^T
// into S'; P [V | V'] -> [O | T], then (P (*) S') V into T; o' = T / l - rbar o.
template <bool DUAL, int HDP>
struct FwdCfg {
  static constexpr int NA = HDP / 64;                      // 64-column atoms of a head
  static constexpr int TK = DUAL ? 64 : 128;               // keys a tile
  static constexpr int NT = DUAL ? 2 : 1;
  static constexpr int Q_B = NT * NA * ATOM128;
  static constexpr int KATOM = TK * 128;
  static constexpr int TILE_B = NT * NA * KATOM;           // K (K') or V (V') of a tile
  static constexpr int STAGES = HDP == 128 ? 1 : 2;
  static constexpr int SMEM = Q_B + 2 * STAGES * TILE_B + 1024;
  static constexpr int THREADS = 192;
  static constexpr int CTAS = 2;
  static constexpr uint32_t TMEM_COLS = 256;
  static constexpr uint32_t C_S = 0, C_SD = 64, C_O = 128, C_T = 192;
};

struct TcParams2 {
  SeqRows seq;
  int Hq, Hkv, D, tiles;
  float c2, scale;                // scale log2 e, scale
  int64_t ldo, lddo, lddq, lddk, lddv;
  const __nv_bfloat16 *o, *od, *d_o, *d_od;
  __nv_bfloat16 *ow, *owd, *dq, *dk, *dv, *dqd, *dkd, *dvd;
  float *lse, *rbar, *Dr, *Drd;
  int* status;
};

// Columns c0 .. c0+15 of a row of a head of D columns, as bf16.
__device__ __forceinline__ void put16(__nv_bfloat16* row, int c0, int D, const float* v) {
#pragma unroll
  for (int h = 0; h < 2; ++h)
    if (c0 + 8 * h < D)
      *reinterpret_cast<uint4*>(row + c0 + 8 * h) =
          make_uint4(pack_bf16x2(v[8 * h], v[8 * h + 1]), pack_bf16x2(v[8 * h + 2], v[8 * h + 3]),
                     pack_bf16x2(v[8 * h + 4], v[8 * h + 5]), pack_bf16x2(v[8 * h + 6], v[8 * h + 7]));
}

template <bool DUAL, int HDP>
__global__ void __launch_bounds__(FwdCfg<DUAL, HDP>::THREADS, FwdCfg<DUAL, HDP>::CTAS)
    attn_tc_fwd_kernel(const __grid_constant__ CUtensorMap tmQ, const __grid_constant__ CUtensorMap tmK,
                       const __grid_constant__ CUtensorMap tmV, const __grid_constant__ CUtensorMap tmQd,
                       const __grid_constant__ CUtensorMap tmKd, const __grid_constant__ CUtensorMap tmVd,
                       const __grid_constant__ TcParams2 p) {
  using C = FwdCfg<DUAL, HDP>;
  constexpr int TK = C::TK, NA = C::NA;
  extern __shared__ __align__(1024) uint8_t smem_raw[];
  __shared__ __align__(8) uint64_t q_full, s_full, p_full, drain;
  __shared__ __align__(8) uint64_t k_full[C::STAGES], k_empty[C::STAGES];
  __shared__ __align__(8) uint64_t v_full[C::STAGES], v_empty[C::STAGES], v_clean[C::STAGES];
  __shared__ uint32_t bad[C::STAGES][4];
  __shared__ SeqTile st_rows;
  __shared__ uint32_t tmem_slot;
  __shared__ int abort_flag;

  uint8_t* smem = reinterpret_cast<uint8_t*>(
      (reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~static_cast<uintptr_t>(1023));
  uint8_t* sQ = smem;
  uint8_t* sK = smem + C::Q_B;
  uint8_t* sV = sK + C::STAGES * C::TILE_B;
  // heads fastest (a group's heads share K and V), the last rows first (the longest walks of a
  // long sequence)
  const int h = static_cast<int>(blockIdx.x % p.Hq);
  const int row0 = (p.tiles - 1 - static_cast<int>(blockIdx.x / p.Hq)) * TR;
  const int hk = h / (p.Hq / p.Hkv);
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;

  pdl_entry();
  const int nvalid = min(seq_total(p.seq) - row0, TR);
  if (nvalid <= 0) return;
  seq_tile_init(p.seq, row0, st_rows);
  if (threadIdx.x == 0) {
    mbar_init(&q_full, 1);
    mbar_init(&s_full, 1);
    mbar_init(&p_full, 4);
    mbar_init(&drain, 1);
    for (int i = 0; i < C::STAGES; ++i) {
      mbar_init(&k_full[i], 1);
      mbar_init(&k_empty[i], 1);
      mbar_init(&v_full[i], 1);
      mbar_init(&v_empty[i], 1);
      mbar_init(&v_clean[i], 1);
    }
    abort_flag = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  if (warp == 1) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(
                     smem_u32(&tmem_slot)),
                 "r"(C::TMEM_COLS));
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;");
  }
  __syncthreads();
  seq_tile_fill(p.seq, row0, st_rows, C::THREADS);
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tb = tmem_slot;
  volatile int* abort = &abort_flag;
  const int k0 = tile_lo(st_rows, row0, 0), lo1 = tile_lo(st_rows, row0, nvalid - 1);
  const int nkt = (row0 + nvalid - k0 + TK - 1) / TK;
  // whether some row does not attend to the whole of key tile j
  auto mixed = [&](int j) { return k0 + j * TK + TK - 1 > row0 || k0 + j * TK < lo1; };

  if (warp == 0) {
    if (elect_one()) {
      // ---- TMA producer ---------------------------------------------------------------------
      mbar_expect_tx(&q_full, C::Q_B);
#pragma unroll
      for (int a = 0; a < NA; ++a) {
        tma_load_3d(sQ + a * ATOM128, &tmQ, &q_full, 64 * a, row0, h);
        if (DUAL) tma_load_3d(sQ + (NA + a) * ATOM128, &tmQd, &q_full, 64 * a, row0, h);
      }
      int nk = 0, nv = 0;
      for (int j = 0; j < nkt; ++j) {
        const int st = j % C::STAGES;
        const uint32_t ph = ((j / C::STAGES) & 1) ^ 1;
        const int kr = k0 + j * TK;
        if (!fwait(&k_empty[st], ph, p.status, abort)) break;
        mbar_expect_tx(&k_full[st], C::TILE_B);
        uint8_t* b = sK + st * C::TILE_B;
#pragma unroll
        for (int a = 0; a < NA; ++a) {
          tma_load_3d(b + a * C::KATOM, &tmK, &k_full[st], 64 * a, kr, hk);
          if (DUAL) tma_load_3d(b + (NA + a) * C::KATOM, &tmKd, &k_full[st], 64 * a, kr, hk);
        }
        ++nk;
        if (!fwait(&v_empty[st], ph, p.status, abort)) break;
        mbar_expect_tx(&v_full[st], C::TILE_B);
        b = sV + st * C::TILE_B;
#pragma unroll
        for (int a = 0; a < NA; ++a) {
          tma_load_3d(b + a * C::KATOM, &tmV, &v_full[st], 64 * a, kr, hk);
          if (DUAL) tma_load_3d(b + (NA + a) * C::KATOM, &tmVd, &v_full[st], 64 * a, kr, hk);
        }
        ++nv;
      }
      mbar_wait(&q_full, 0, p.status, FTC_WAIT_NS);
      drain_loads(k_full, nk, C::STAGES, p.status);
      drain_loads(v_full, nv, C::STAGES, p.status);
    }
    __syncwarp();
  } else if (warp == 1) {
    // ---- products -------------------------------------------------------------------------------
    constexpr uint32_t idS = idesc_bf16(TR, TK), idS2 = idesc_bf16(TR, 2 * TK);
    constexpr uint32_t idO = idesc_bf16(TR, HDP) | (1u << 16), idO2 = idesc_bf16(TR, 2 * HDP) | (1u << 16);
    const uint64_t dQ = sdesc_sw128(smem_u32(sQ)), dQd = dQ + (NA * ATOM128 >> 4);
    const uint64_t dKs = sdesc_sw128(smem_u32(sK)), mVs = sdesc_mn(smem_u32(sV), C::KATOM);
    constexpr uint64_t ST = C::TILE_B >> 4;
    auto scores = [&](int j) -> bool {
      const int st = j % C::STAGES;
      if (!wwait(&k_full[st], (j / C::STAGES) & 1, p.status, abort)) return false;
      tc_fence_after();
      if (elect_one()) {
        const uint64_t dK = dKs + st * ST;
#pragma unroll
        for (int kk = 0; kk < HDP / 16; ++kk) {
          const uint64_t qo = (kk >> 2) * (ATOM128 >> 4) + 2 * (kk & 3);
          const uint64_t ko = (kk >> 2) * (C::KATOM >> 4) + 2 * (kk & 3);
          mma_bf16(tb + C::C_S, dQ + qo, dK + ko, DUAL ? idS2 : idS, kk > 0);
        }
        if (DUAL) {
#pragma unroll
          for (int kk = 0; kk < HDP / 16; ++kk)
            mma_bf16(tb + C::C_SD, dQd + 2 * kk, dK + 2 * kk, idS, 1);
        }
        mma_commit(&s_full);
        mma_commit(&k_empty[st]);
      }
      __syncwarp();
      return true;
    };
    bool ok = wwait(&q_full, 0, p.status, abort) && scores(0);
    for (int j = 0; ok && j < nkt; ++j) {
      const int st = j % C::STAGES;
      const uint32_t ph = (j / C::STAGES) & 1;
      if (mixed(j)) {
        if (!wwait(&v_full[st], ph, p.status, abort)) break;
        scrub(sV + st * C::TILE_B, TK, C::NT * NA, bad[st], lane);
      }
      if (lane == 0) mbar_arrive_local(&v_clean[st]);
      __syncwarp();
      if (!wwait(&v_full[st], ph, p.status, abort)) break;
      if (!wwait(&p_full, j & 1, p.status, abort)) break;
      tc_fence_after();
      if (elect_one()) {
        const uint64_t mV = mVs + st * ST;
#pragma unroll
        for (int kk = 0; kk < TK / 16; ++kk) {
          const uint32_t acc = (j > 0 || kk > 0) ? 1u : 0u;
          // keys 64.. of a tile sit 64 columns on, where their scores were
          const uint32_t pc = (kk >> 2) * 64 + 8 * (kk & 3);
          if (DUAL) {
            mma_ts(tb + C::C_O, tb + C::C_S + pc, mV + 128 * kk, idO2, acc);
            mma_ts(tb + C::C_T, tb + C::C_SD + pc, mV + 128 * kk, idO, 1);
          } else {
            mma_ts(tb + C::C_O, tb + C::C_S + pc, mV + 128 * kk, idO, acc);
          }
        }
        mma_commit(&v_empty[st]);
      }
      __syncwarp();
      if (j + 1 < nkt && !scores(j + 1)) break;
    }
    // every product issued here has completed before the rows are read and TMEM is released
    if (elect_one()) mma_commit(&drain);
    __syncwarp();
    mbar_wait(&drain, 0, p.status, FTC_WAIT_NS);
  } else {
    // ---- rows: thread r owns row row0 + r (TMEM lane r) ------------------------------------------
    const int q4 = warp & 3;
    const int r = q4 * 32 + lane;
    const uint32_t lane_base = tb + (static_cast<uint32_t>(q4 * 32) << 16);
    const int lo = tile_lo(st_rows, row0, r);
    float m2 = -INFINITY, l = 0.f, rs = 0.f;
    bool ok = true;
    for (int j = 0; j < nkt; ++j) {
      const int st = j % C::STAGES;
      const bool mx_tile = mixed(j);
      if (!wwait(&s_full, j & 1, p.status, abort)) { ok = false; break; }
      uint32_t badw[TK / 32];
      bool any_bad = false;
      if (mx_tile) {
        if (!wwait(&v_clean[st], (j / C::STAGES) & 1, p.status, abort)) { ok = false; break; }
#pragma unroll
        for (int i = 0; i < TK / 32; ++i) { badw[i] = bad[st][i]; any_bad |= badw[i] != 0; }
      }
      tc_fence_after();
      // keys a .. b of this tile are the row's own
      const int a = lo - (k0 + j * TK), b = row0 + r - (k0 + j * TK);
      float sv[64];
      auto own = [&](int i) { return i >= a && i <= b; };
      auto tile_max = [&](int c0, float mx) {
        tmem_ld32_nowait(lane_base + C::C_S + c0, sv);
        tmem_ld32_nowait(lane_base + C::C_S + c0 + 32, sv + 32);
        tmem_wait_ld();
        if (mx_tile) {
#pragma unroll
          for (int i = 0; i < 64; ++i)
            if (own(c0 + i)) mx = fmaxf(mx, sv[i]);
        } else {
          float y0 = mx, y1 = sv[0];
#pragma unroll
          for (int i = 0; i < 64; i += 4) {
            y0 = fmaxf(fmaxf(y0, sv[i]), sv[i + 1]);
            y1 = fmaxf(fmaxf(y1, sv[i + 2]), sv[i + 3]);
          }
          mx = fmaxf(y0, y1);
        }
        return mx;
      };
      float mx = -INFINITY;
#pragma unroll
      for (int c0 = 0; c0 < TK; c0 += 64) mx = tile_max(c0, mx);
      const float t2 = mx * p.c2;
      float f = 1.f;
      if (t2 > m2 + TAU) {
        f = ex2(m2 - t2);
        m2 = t2;
      }
      l *= f;
      rs *= f;
      if (j > 0 && __any_sync(0xffffffffu, f != 1.f)) {
        // scores j were issued behind the products of tile j - 1, which are done
#pragma unroll 1
        for (int c0 = 0; c0 < HDP * C::NT; c0 += 16) {
          float v[16];
          tmem_ld16(lane_base + C::C_O + c0, v);
#pragma unroll
          for (int i = 0; i < 16; ++i) v[i] *= f;
          tmem_st16(lane_base + C::C_O + c0, v);
        }
      }
      const float base = m2 == -INFINITY ? 0.f : m2;     // no key of the row so far: P = 0
      const uint64_t c2p = pair(p.c2, p.c2), nm = pair(-base, -base);
      uint64_t l2 = 0, r2 = 0;
      auto probs = [&](int c0, auto masked) {
        constexpr bool MASK = decltype(masked)::value;
#pragma unroll
        for (int g = 0; g < 2; ++g) {
          uint32_t pk[16], psk[16];
          float sd[32];
          if (DUAL) {
            tmem_ld32_nowait(lane_base + C::C_SD + c0 + 32 * g, sd);
            tmem_wait_ld();
          }
#pragma unroll
          for (int i = 0; i < 32; i += 2) {
            const int e = 32 * g + i;
            const float2 x = halves(fma2(pair(sv[e], sv[e + 1]), c2p, nm));
            float p0 = ex2(x.x), p1 = ex2(x.y);
            const bool o0 = !MASK || own(c0 + e), o1 = !MASK || own(c0 + e + 1);
            if (!o0) p0 = 0.f;
            if (!o1) p1 = 0.f;
            const uint64_t pp = pair(p0, p1);
            l2 = add2(l2, pp);
            pk[i / 2] = pack_bf16x2(p0, p1);
            if (DUAL) {
              float2 ps = halves(mul2(pp, pair(sd[i], sd[i + 1])));
              if (!o0) ps.x = 0.f;      // the tangent's score may be anything there
              if (!o1) ps.y = 0.f;
              r2 = add2(r2, pair(ps.x, ps.y));
              psk[i / 2] = pack_bf16x2(ps.x * p.scale, ps.y * p.scale);
            }
            if (MASK && any_bad) {
              const uint32_t w = badw[(c0 + e) >> 5] >> (e & 31);
              const uint32_t nan2 = (o0 && (w & 1) ? 0x7fffu : 0u) | (o1 && (w & 2) ? 0x7fff0000u : 0u);
              pk[i / 2] |= nan2;
              if (DUAL) psk[i / 2] |= nan2;
            }
          }
          tmem_st16u(lane_base + C::C_S + c0 + 16 * g, pk);
          if (DUAL) tmem_st16u(lane_base + C::C_SD + c0 + 16 * g, psk);
        }
      };
#pragma unroll
      for (int c0 = TK - 64; c0 >= 0; c0 -= 64) {
        if (c0 != TK - 64) {   // the last 64 keys' scores are still in registers
          tmem_ld32_nowait(lane_base + C::C_S + c0, sv);
          tmem_ld32_nowait(lane_base + C::C_S + c0 + 32, sv + 32);
          tmem_wait_ld();
        }
        if (mx_tile) probs(c0, std::true_type{});
        else probs(c0, std::false_type{});
      }
      const float2 lh = halves(l2), rh = halves(r2);
      l += lh.x + lh.y;
      rs += rh.x + rh.y;
      tmem_wait_st();
      tc_fence_before();
      __syncwarp();
      if (lane == 0) mbar_arrive_local(&p_full);
    }
    if (ok && wwait(&drain, 0, p.status, abort) && !*abort) {
      tc_fence_after();
      const float inv = 1.f / l;
      const float rb = DUAL ? rs * p.scale * inv : 0.f;
      const int64_t row = row0 + r;
      const bool on = r < nvalid;
      __nv_bfloat16* orow = p.ow + row * p.ldo + h * p.D;
      __nv_bfloat16* drow = DUAL ? p.owd + row * p.ldo + h * p.D : nullptr;
#pragma unroll 1
      for (int c0 = 0; c0 < HDP; c0 += 16) {
        if (c0 >= p.D) break;
        float o[16], t[16];
        tmem_ld16(lane_base + C::C_O + c0, o);
        if (DUAL) tmem_ld16(lane_base + C::C_T + c0, t);
#pragma unroll
        for (int i = 0; i < 16; ++i) {
          o[i] *= inv;
          if (DUAL) t[i] = t[i] * inv - rb * o[i];
        }
        if (on) put16(orow, c0, p.D, o);
        if (DUAL && on) put16(drow, c0, p.D, t);
      }
      if (on) {
        const int64_t si = static_cast<int64_t>(h) * p.seq.rows + row;
        p.lse[si] = (m2 + log2f(l)) * LN2;
        if (DUAL) p.rbar[si] = rb;
      }
    }
    tc_fence_before();
  }
  __syncthreads();
  if (warp == 1) {
    tc_fence_after();
    asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tb),
                 "r"(C::TMEM_COLS));
  }
}

// Heads of row buffer t as a tensor map {columns of a head, rows, heads}, boxes of 64 columns.
bool head_map(CUtensorMap* m, const __nv_bfloat16* t, int D, int rows, int64_t ld, int heads, int box) {
  if (!t) {
    memset(m, 0, sizeof(*m));
    return true;
  }
  return make_head_map(m, t, D, rows, ld, heads, box);
}

TcParams2 tc_params(const AttnParams& a) {
  TcParams2 p;
  memset(&p, 0, sizeof(p));
  p.seq = a.seq;
  p.Hq = a.Hq; p.Hkv = a.Hkv; p.D = a.D;
  p.tiles = (a.seq.rows + TR - 1) / TR;
  p.scale = a.scale;
  p.c2 = a.scale * LOG2E;
  p.ldo = a.ldo; p.lddo = a.lddo; p.lddq = a.lddq; p.lddk = a.lddk; p.lddv = a.lddv;
  p.o = a.o; p.od = a.od; p.d_o = a.d_o; p.d_od = a.d_od;
  p.ow = a.o; p.owd = a.od;
  p.dq = a.dq; p.dk = a.dk; p.dv = a.dv; p.dqd = a.dqd; p.dkd = a.dkd; p.dvd = a.dvd;
  p.lse = a.lse; p.rbar = a.rbar; p.Dr = a.Dr; p.Drd = a.Drd;
  p.status = a.status;
  return p;
}

template <bool DUAL, int HDP>
cudaError_t launch_fwd(const AttnParams& a, cudaStream_t s) {
  using C = FwdCfg<DUAL, HDP>;
  CUtensorMap q, k, v, qd, kd, vd;
  const int N = a.seq.rows;
  if (!head_map(&q, a.q, a.D, N, a.ldq, a.Hq, TR) || !head_map(&k, a.k, a.D, N, a.ldk, a.Hkv, C::TK) ||
      !head_map(&v, a.v, a.D, N, a.ldv, a.Hkv, C::TK) ||
      !head_map(&qd, DUAL ? a.qd : nullptr, a.D, N, a.ldq, a.Hq, TR) ||
      !head_map(&kd, DUAL ? a.kd : nullptr, a.D, N, a.ldk, a.Hkv, C::TK) ||
      !head_map(&vd, DUAL ? a.vd : nullptr, a.D, N, a.ldv, a.Hkv, C::TK))
    return cudaErrorInvalidValue;
  static PerDeviceOnce once;
  cudaError_t e = once.run([](int&) {
    return cudaFuncSetAttribute(attn_tc_fwd_kernel<DUAL, HDP>,
                                cudaFuncAttributeMaxDynamicSharedMemorySize, C::SMEM);
  });
  if (e != cudaSuccess) return e;
  const TcParams2 p = tc_params(a);
  const int64_t grid = static_cast<int64_t>(p.tiles) * a.Hq;
  if (grid > INT32_MAX) return cudaErrorInvalidValue;
  return launch_k(attn_tc_fwd_kernel<DUAL, HDP>, dim3(static_cast<unsigned>(grid)), dim3(C::THREADS),
                  C::SMEM, s, q, k, v, qd, kd, vd, p);
}

}  // namespace

cudaError_t attn_tc_fwd(const AttnParams& a, bool dual, cudaStream_t s) {
  if (dual) return launch_fwd<true, 64>(a, s);
  return a.D <= 64 ? launch_fwd<false, 64>(a, s) : launch_fwd<false, 128>(a, s);
}

}  // namespace mf
