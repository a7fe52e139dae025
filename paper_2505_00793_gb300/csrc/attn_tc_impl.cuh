// Causal attention with grouped heads over packed sequences on the 5th-generation tensor cores
// (tcgen05 + TMEM + TMA), with its forward tangent and its backward pass: the kernels behind
// mf_attn_fwd and mf_attn_bwd, and with a window (WIN) mf_attn_window_*.  Formulas in mixflow.h.
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
// Rounded to bf16 are the outputs and, as operands of the tensor cores next to bf16 rows, P,
// P (*) (S' - c), P', dS and dS', each by 2^-8 of its value at most: the tensor cores take both operands
// of a product in one 16-bit type, and the rows are bf16.  Scores, maxima, sums, lse, rbar, D and
// every accumulator are float32; D comes from the rounded o, D' from o and o'.  Off from 64 bits, in
// relative L2 (an output's own rounding alone is 0.0017; independent rows of unit variance):
//   1024 tokens             o 0.0020, o' 0.0022, dv, dv' 0.0023, dq, dk, dq', dk' 0.0025
//   2 tokens                dq, dk 0.0038, dq', dk' 0.0042 (8 tokens 0.0031): dP - D is a difference of
//                           near values, and D carries o's rounding
//   scores of std 3, 8      o' 0.0030, 0.0039 (with a window 0.0025), dq .. dk' up to 0.0038, 0.0058
//   keys with 3, 10 of a unit vector in common    dq, dq' 0.0088, 0.029, all else as above: the roundings
//                           of dS and D leave sum dS = 0 off by 2^-9 of its terms, times what the keys share
//
// Values of masked places: a product with a zero of P still meets them (0 * inf = NaN).  So a
// CTA whose results are all finite is done; one that finds a NaN or an infinity in them walks its
// tiles a second time, carefully: in mixed tiles the rows that P or dS will multiply are looked
// over first, what is not finite in them becomes zero, and rows that do attend to such a row get
// NaN, in their tangents alone where only tangents were not finite.  Others come out as if it was
// not there, bit for bit, and a call without such values pays for a check of its results.
//
// Every wait is bounded (2 s), as in flash_tc.cu.
#pragma once

#include <limits.h>

#include "attn_ops.h"
#include "attn_tc_util.cuh"
#include "packed_rows.cuh"

namespace mf {
namespace {

constexpr int TR = 128;                       // rows of a CTA's own tile (MMA M)
constexpr int ATOM128 = 128 * 128;            // bytes of [128 rows][64] bf16
constexpr float LOG2E = 1.44269504088896341f, LN2 = 0.693147180559945309f;

// Shared-memory operands as the low words of their matrix descriptors (start address >> 4 and
// leading byte offset >> 4; the high word is the same for all: 128-byte swizzle, 8-row groups of
// 1024 bytes).  A byte offset moves a low word by offset >> 4.  Kept as 32-bit words: with 64-bit
// descriptors moved by a ring's stage, nvcc 13.0 built products of the wrong columns.
constexpr uint32_t DESC_HI = 0x40004040u;
__device__ __forceinline__ uint32_t kdesc(uint32_t saddr) {        // K-major
  return ((saddr & 0x3FFFFu) >> 4) | (1u << 16);
}
__device__ __forceinline__ uint32_t ndesc(uint32_t saddr, int box) {   // MN-major: 64-column boxes
  return ((saddr & 0x3FFFFu) >> 4) | (static_cast<uint32_t>(box >> 4) << 16);
}
__device__ __forceinline__ uint64_t desc(uint32_t lo) {
  uint64_t d;
  asm("mov.b64 %0, {%1, %2};" : "=l"(d) : "r"(lo), "r"(DESC_HI));
  return d;
}
__device__ __forceinline__ void mma_ss(uint32_t d, uint32_t a, uint32_t b, uint32_t idesc,
                                       uint32_t acc) {
  mma_bf16(d, desc(a), desc(b), idesc, acc);
}

// D[tmem] (+)= A[tmem] B, A bf16: lane = row, two consecutive K elements a column.
__device__ __forceinline__ void mma_ts(uint32_t d, uint32_t a, uint32_t b, uint32_t idesc,
                                       uint32_t acc) {
  asm volatile(
      "{\n\t.reg .pred p;\n\t"
      "setp.ne.b32 p, %4, 0;\n\t"
      "tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n\t}" ::"r"(d),
      "r"(a), "l"(desc(b)), "r"(idesc), "r"(acc));
}

__device__ __forceinline__ void tmem_st8(uint32_t t, const uint32_t* v) {
  asm volatile("tcgen05.st.sync.aligned.32x32b.x8.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8};" ::"r"(t),
               "r"(v[0]), "r"(v[1]), "r"(v[2]), "r"(v[3]), "r"(v[4]), "r"(v[5]), "r"(v[6]), "r"(v[7])
               : "memory");
}
__device__ __forceinline__ void tmem_wait_st() {
  asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory");
}
__device__ __forceinline__ float4 ld_cluster4(uint32_t addr) {
  float4 v;
  asm volatile("ld.shared::cluster.v4.f32 {%0,%1,%2,%3}, [%4];"
               : "=f"(v.x), "=f"(v.y), "=f"(v.z), "=f"(v.w) : "r"(addr) : "memory");
  return v;
}
// The cluster's last barrier: what was read of other CTAs has arrived, and nothing is published
// (a releasing arrive would wait for the rows just written to be acknowledged).
__device__ __forceinline__ void cluster_leave() {
  asm volatile("barrier.cluster.arrive.relaxed.aligned;\n\t"
               "barrier.cluster.wait.aligned;" ::: "memory");
}
__device__ __forceinline__ float ex2(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}

// Barriers are shared-memory addresses.  Waits are bounded by the SM's clock: 2 s at 2 GHz.
constexpr long long WAIT_CLOCKS = 4000000000LL;
__device__ __forceinline__ void bar_init(uint32_t bar, uint32_t count) {
  asm volatile("mbarrier.init.shared::cta.b64 [%0], %1;" ::"r"(bar), "r"(count));
}
__device__ __forceinline__ void bar_arrive(uint32_t bar) {
  asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" ::"r"(bar) : "memory");
}
// One vote of a warp on whether the phase is complete.
__device__ __forceinline__ bool warp_try(uint32_t bar, uint32_t parity) {
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
// A warp's bounded wait: all of it goes on, or none.
__device__ __forceinline__ bool rwait(uint32_t bar, uint32_t parity, int* status,
                                      volatile int* abort) {
  if (warp_try(bar, parity)) return true;
  const long long t0 = clock64();
  while (!warp_try(bar, parity)) {
    if (__any_sync(0xffffffffu, *abort != 0)) return false;
    if (__any_sync(0xffffffffu, clock64() - t0 > WAIT_CLOCKS)) {
      if (status) atomicMax(status, DEV_TIMEOUT);
      *abort = 1;
      return false;
    }
  }
  return true;
}
// The same for one thread.
__device__ __forceinline__ bool twait(uint32_t bar, uint32_t parity, int* status,
                                      volatile int* abort) {
  if (mbar_try_wait_addr(bar, parity)) return true;
  const long long t0 = clock64();
  while (!mbar_try_wait_addr(bar, parity)) {
    if (*abort) return false;
    if (clock64() - t0 > WAIT_CLOCKS) {
      if (status) atomicMax(status, DEV_TIMEOUT);
      *abort = 1;
      return false;
    }
  }
  return true;
}
// Waits for the loads that were issued, `n` of them round a ring: nothing may still arrive when
// the CTA ends, given up or not.
__device__ __forceinline__ void drain_ring(uint32_t full, int n, int stages, int* status) {
  for (int j = n - stages > 0 ? n - stages : 0; j < n; ++j)
    if (!mbar_wait_addr(full + 8 * (j % stages), (j / stages) & 1, status, FTC_WAIT_NS)) return;
}

// Zero while everything added so far was finite, else NaN (0 x is NaN for a NaN or an infinity).
__device__ __forceinline__ void add_check(float& z, float x) { z = fmaf(x, 0.f, z); }

// ---- sequences of a tile's rows -------------------------------------------------------------
// Borders inside the tile as a bit per row (a sequence starts there), the start of the first
// row's sequence and the end of the last row's.
struct SeqTile {
  int lo0, hi1;
  uint32_t bits[4];
};

// The table is filled by the first `threads` of the block: each reads its first start (SeqLoad) before
// their first barrier, so that the reads of the prologue are in flight together.
struct SeqLoad {
  int first, v;
};
__device__ __forceinline__ SeqLoad seq_tile_load(const SeqRows& s, int row0) {
  SeqLoad l{0, 0};
  if (!s.start) return l;
  if (s.n > 2048) l.first = seq_find(s, row0);   // long tables: from the first row's sequence on
  const int i = l.first + static_cast<int>(threadIdx.x);
  if (i <= s.n) l.v = s.start[i];
  return l;
}
__device__ __forceinline__ void seq_tile_init(const SeqRows& s, int row0, SeqTile& t) {
  const int e = static_cast<int>(threadIdx.x) - 64;
  if (e >= 0 && e < 4) t.bits[e] = 0;
  if (e == 4) t.lo0 = s.start ? 0 : row0 - row0 % s.len;
  if (e == 5) t.hi1 = s.start ? s.rows : (row0 + TR - 1) - (row0 + TR - 1) % s.len + s.len;
}
__device__ __forceinline__ void seq_tile_fill(const SeqRows& s, int row0, SeqTile& t, int threads,
                                              const SeqLoad& l) {
  if (!s.start) {
    for (int p = threadIdx.x; p < TR; p += threads)
      if (p > 0 && (row0 + p) % s.len == 0) atomicOr(&t.bits[p >> 5], 1u << (p & 31));
    return;
  }
  int v = l.v;
  for (int i = l.first + static_cast<int>(threadIdx.x); i <= s.n;) {
    if (v <= row0) {
      atomicMax(&t.lo0, v);
    } else if (v - row0 < TR) {
      atomicOr(&t.bits[(v - row0) >> 5], 1u << ((v - row0) & 31));
    } else {
      atomicMin(&t.hi1, v);
      break;
    }
    i += threads;
    if (i <= s.n) v = s.start[i];
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

// Bits lo .. hi of a word of 32 columns.
__device__ __forceinline__ uint32_t col_bits(int lo, int hi) {
  lo = max(lo, 0);
  hi = min(hi, 31);
  return lo > hi ? 0u : (0xffffffffu << lo) & (0xffffffffu >> (31 - hi));
}
// Bits of the 32 keys from kb on that row attends to with a window: itself, the window - 1 rows
// before it and the first `sinks` rows of its sequence, which begins at lo.
__device__ __forceinline__ uint32_t window_bits(int lo, int row, int window, int sinks, int kb) {
  uint32_t w = col_bits(max(lo, row - window + 1) - kb, row - kb);
  if (sinks > 0) w |= col_bits(lo - kb, min(lo + sinks - 1, row) - kb);
  return w;
}
// bf16 pair with NaN in the halves whose bits of w are set.
__device__ __forceinline__ uint32_t nan_pair(uint32_t w) {
  return (w & 1 ? 0x7fffu : 0u) | (w & 2 ? 0x7fff0000u : 0u);
}

// ---- non-finite values of a mixed tile --------------------------------------------------------
// A warp looks over `atoms` blocks of `rows` 128-byte rows of bf16, zeroes what is not finite
// and sets the bit of its row in bad[].  0 * x is zero for every finite x and NaN otherwise, so
// one multiply-add a pair tells whether there is anything to do.
__device__ __forceinline__ void scrub_part(uint8_t* base, int rows, int atoms, uint32_t* bad, int lane) {
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

// An operand's rows, and behind them its tangent's, which have bits of their own.
template <bool DUAL>
__device__ __forceinline__ void scrub(uint8_t* base, int rows, int atoms, uint32_t (*bad)[4], int lane) {
  scrub_part(base, rows, atoms, bad[0], lane);
  if (DUAL) scrub_part(base + rows * atoms * 128, rows, atoms, bad[1], lane);
}

// ---- forward ------------------------------------------------------------------------------------
// One CTA per (query head, 128 rows): warp 0 loads (Q once, then key tiles into a ring of K and a
// ring of V), warp 1 owns TMEM, looks over mixed V tiles and issues the products, warps 2..5 hold
// the rows, a thread each (two threads a row, which have to agree on its maximum, took longer).
// The tangent shares the operands: Q [K | K']^T -> [S | Q K'^T], then Q' K^T into S';
// P [V | V'] -> [O | T], then (P (*) (S' - c)) V into T; o' = T / l - (rbar - c) o.  c is a mean of
// the row's S' by P, over its first tiles and again where its maximum moves by TAU or a key outweighs what came
// before: what all of a row's S' have in common (keys or their tangents with a common part) cancels in o', and
// rounded to bf16 as part of P (*) S' it would leave 2^-9 of itself.  With keys of 10 of a unit vector in common o' was off by
// 0.012 in relative L2, with 30 by 0.035; now 0.0022.  By P, since a sequence's first keys may outweigh
// the rest: with the plain mean of the first whole tile such rows, whose other S' differed by 4 and 30, had o'
// off by 0.010 and 0.095, dq' (through D') by 0.08 and 0.17; now 0.0024 and 0.016.  Scores of std 1, 2, 3 and 8
// take 342, 348, 384 and 446 us against 335, 337, 389 and 492 with that (16 heads over 4, one sequence of 8192;
// 16384 rows in four, window 1000: 229, 277, 289 and 293 against 231, 307, 319 and 336).
// What bounds it: at 128 columns the products (8 heads over one, 16384 rows: 342 to 366 us, 1.50 to 1.60 PF/s
// of causal work; the tensor pipe busy 67 % of the cycles with scores read 32 columns at a time); at 64
// the chain scores - maximum -
// exponentials - product of each CTA, which two or three CTAs an SM fill by turns (16 heads, 16384
// rows: 0.94 PF/s; 16 heads with tangents, eight sequences of 1024: 79 us, pipe 36 %).  Taking the
// exponentials against the last tile's maximum, so that they need not wait for this one's, cost
// registers and was up to 17 % slower.
// TKEYS keys a tile: 64 where the tangents leave no TMEM for more, and where many CTAs are to be
// had: tiles of 64 let three of them, not two, fill each other's waits on an SM (launch_fwd).
// With a window, whose walks are all as long, four CTAs of 64 keys a tile hide one another's ends better, for
// fewer registers: 16 heads over 4, 32768 rows, windows of 32, 1024, 4096, 8192 and 24000 84, 207, 539, 932 and
// 1885 us against 90, 225, 592, 1026 and 2076 with three; 8192 rows, windows of 128, 1024, 3000 and 8191 33, 59,
// 115 and 158 against 35, 66, 111 and 162; without one 16 heads over 4, 8192 rows 191 (a training step)
// against 181.  (Few CTAs and a long window: attn_window_fwd.)
template <bool DUAL, int HDP, int TKEYS, bool WIN>
struct FwdCfg {
  static constexpr int NA = HDP / 64;                      // 64-column atoms of a head
  static constexpr int TK = TKEYS;
  static constexpr int NT = DUAL ? 2 : 1;
  static constexpr int Q_B = NT * NA * ATOM128;
  static constexpr int KATOM = TK * 128;
  static constexpr int TILE_B = NT * NA * KATOM;           // K (K') or V (V') of a tile
  static constexpr int STAGES = HDP == 128 ? 1 : 2;
  static constexpr int SMEM = Q_B + 2 * STAGES * TILE_B + 1024;
  static constexpr int EW = 4;                             // row warps: a thread a row
  static constexpr int THREADS = 64 + 32 * EW;
  static constexpr bool SMALL = TK * NT + HDP * NT <= 128;
  static constexpr int CTAS = SMALL ? (WIN ? 4 : 3) : 2;
  static constexpr uint32_t TMEM_COLS = SMALL ? 128 : 256;
  static constexpr uint32_t C_S = 0, C_SD = 64, C_O = NT * TK, C_T = 192;
};

struct TcParams2 {
  SeqRows seq;
  int D, tiles, Hkv;
  int G;                          // query heads of a group
  int share, Gs;                  // key-row kernel: CTAs that share a group, query heads of each
  float c2, scale;                // scale log2 e, scale
  int64_t ldo, lddo, lddq, lddk, lddv;
  const __nv_bfloat16 *o, *od, *d_o, *d_od;
  __nv_bfloat16 *ow, *owd, *dq, *dk, *dv, *dqd, *dkd, *dvd;
  float *lse, *rbar, *Dr, *Drd;
  int* status;
  int window, sinks;              // a row's own keys (WIN)
  int chunk, chunks;              // key-row kernel: rows of a chunk, chunks
  float* part;                    // sums of sink rows, [2 chunks][Hkv][sums][sinks][HDP]
};

// Tile of this CTA: grid y, continued along z.
constexpr int GRID_Y = 65535;
__device__ __forceinline__ int tile_index() {
  return static_cast<int>(blockIdx.y) + GRID_Y * static_cast<int>(blockIdx.z);
}

// Results leave through shared memory, so that global rows are written whole: a tile of 128
// rows of W bf16, 16-byte chunk c of row r at place c ^ (r & 7).
template <int W>
__device__ __forceinline__ void stage16(uint8_t* buf, int r, int c0, const float* v) {
#pragma unroll
  for (int h = 0; h < 2; ++h)
    *reinterpret_cast<uint4*>(buf + r * (2 * W) + (((c0 / 8 + h) ^ (r & 7)) << 4)) =
        make_uint4(pack_bf16x2(v[8 * h], v[8 * h + 1]), pack_bf16x2(v[8 * h + 2], v[8 * h + 3]),
                   pack_bf16x2(v[8 * h + 4], v[8 * h + 5]), pack_bf16x2(v[8 * h + 6], v[8 * h + 7]));
}
// By THREADS threads, each a chunk of every RS-th row.
template <int W, int THREADS>
__device__ __forceinline__ void stage_out(const uint8_t* buf, int nvalid, int D, __nv_bfloat16* dst,
                                          int64_t ld, int t) {
  constexpr int RS = THREADS / (W / 8);
  static_assert(RS % 8 == 0 && TR % RS == 0, "a thread's chunk has one place in all its rows");
  const int c = t % (W / 8), r0 = t / (W / 8);
  if (8 * c >= D) return;
  const uint8_t* from = buf + r0 * (2 * W) + ((c ^ (r0 & 7)) << 4);
  dst += r0 * ld + 8 * c;
#pragma unroll 1
  for (int r = r0; r < nvalid; r += RS, from += RS * 2 * W, dst += RS * ld)
    *reinterpret_cast<uint4*>(dst) = *reinterpret_cast<const uint4*>(from);
}

// With a window (WIN) row i of a sequence that begins at lo attends to the rows j of it with j <= i and
// i - j < window or j - lo < sinks: the same sums over fewer pairs.  A tile of 128 rows walks window + 127
// keys, and 128 at most of sinks before them, so that its ends, some 6000 cycles of a forward CTA (set-up and
// first scores 4000, results 2200) beside 1900 a tile, weigh more than without one.  Of the products
// that the pairs need, at 1888 TF/s: 16 heads of 64 over 4, 32768 rows, window 1024 203 us forward (72: 669
// TF/s); window 512, 16384 rows 292 us forward and backward (45); 16 heads of 128 over 2, 24577 rows,
// window 1000 935 us (305).  Issue slots are half used, the tensor pipe 30 %: the chain of a tile
// bounds it, and four CTAs an SM fill what three left.  Tried, and no faster: products and exponentials of
// no more sinks than there are, columns that no row of a warp attends to left out of masked tiles, two
// buffers of scores, the next CTA's rows fetched into L2.
//
// The key tiles that a tile of query rows walks: from the first row's sequence on (k0), or, with
// a window, from the first row's window on, ahead of them the sinks of its sequence where they lie
// before that window.  (Other sequences of the tile begin inside it, and so do their sinks.)
template <bool WIN, int T>
struct KeyWalk {
  int k0, kw, ns, tiles;          // kw: where the window's tiles begin; ns tiles of sinks
  __device__ __forceinline__ KeyWalk(const TcParams2& p, int row0, int nvalid, int first) {
    k0 = kw = first;
    ns = 0;
    if constexpr (WIN) {
      kw = max(k0, row0 - p.window + 1);
      ns = (min(p.sinks, kw - k0) + T - 1) / T;
    }
    tiles = ns + (row0 + nvalid - kw + T - 1) / T;
  }
  // first key of tile j
  __device__ __forceinline__ int row(int j) const {
    if constexpr (WIN) return j < ns ? k0 + j * T : kw + (j - ns) * T;
    return k0 + j * T;
  }
  // whether some row does not attend to the whole of tile j; lo1: first row of the last row's sequence
  __device__ __forceinline__ bool mixed(int j, int row0, int nvalid, int lo1, int window) const {
    const int kb = row(j);
    if constexpr (WIN)
      return j < ns || kb + T - 1 > row0 || kb < max(lo1, row0 + nvalid - window);
    return kb + T - 1 > row0 || kb < lo1;
  }
  // A row's own keys of tile j, 32 from kb on.
  __device__ __forceinline__ uint32_t bits(int j, int lo, int row, const TcParams2& p, int kb) const {
    if constexpr (WIN) {
      const uint32_t w = window_bits(lo, row, p.window, p.sinks, kb);
      return j < ns ? w & col_bits(0, kw - 1 - kb) : w;
    }
    return col_bits(lo - kb, row - kb);
  }
  // A row's first whole tile, where its first one holds keys of others (with a window: the first
  // that begins inside it).
  __device__ __forceinline__ int first_whole(int lo, int row, int window) const {
    if constexpr (WIN) return ns + (max(lo, row - window + 1) - kw + T - 1) / T;
    return (lo - k0) % T ? (lo - k0) / T + 1 : -1;
  }
};

template <bool DUAL, int HDP, int TKEYS, bool WIN>
__global__ void __launch_bounds__(FwdCfg<DUAL, HDP, TKEYS, WIN>::THREADS, FwdCfg<DUAL, HDP, TKEYS, WIN>::CTAS)
    attn_tc_fwd_kernel(const __grid_constant__ CUtensorMap tmQ, const __grid_constant__ CUtensorMap tmK,
                       const __grid_constant__ CUtensorMap tmV, const __grid_constant__ CUtensorMap tmQd,
                       const __grid_constant__ CUtensorMap tmKd, const __grid_constant__ CUtensorMap tmVd,
                       const __grid_constant__ TcParams2 p) {
  using C = FwdCfg<DUAL, HDP, TKEYS, WIN>;
  constexpr int TK = C::TK, NA = C::NA;
  extern __shared__ __align__(1024) uint8_t smem_raw[];
  // barriers, as byte offsets in a set; one set per walk
  constexpr uint32_t B_Q_FULL = 0, B_S_FULL = 8, B_P_FULL = 16, B_DRAIN = 24;
  constexpr uint32_t B_K_FULL = 32 + 0 * C::STAGES, B_K_EMPTY = 32 + 8 * C::STAGES,
      B_V_FULL = 32 + 16 * C::STAGES, B_V_EMPTY = 32 + 24 * C::STAGES,
      B_V_CLEAN = 32 + 32 * C::STAGES;
  constexpr int NBARS = 4 + 5 * C::STAGES;
  __shared__ __align__(8) uint64_t bars[2][NBARS];
  __shared__ uint32_t bad[C::STAGES][2][4];    // rows of V, of V'
  __shared__ SeqTile st_rows;
  __shared__ uint32_t tmem_slot;
  __shared__ int abort_flag, redo_flag;

  uint8_t* smem = reinterpret_cast<uint8_t*>(
      (reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~static_cast<uintptr_t>(1023));
  uint8_t* sQ = smem;
  uint8_t* sK = smem + C::Q_B;
  uint8_t* sV = sK + C::STAGES * C::TILE_B;
  // heads fastest (a group's heads share K and V), the last rows first (the longest walks of a
  // long sequence)
  const int h = static_cast<int>(blockIdx.x), tile = tile_index();
  if (tile >= p.tiles) return;
  const int row0 = (p.tiles - 1 - tile) * TR;
  const int hk = h / p.G;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  auto load_rows = [&](uint32_t bar) {
    mbar_expect_tx_addr(bar, C::Q_B);
#pragma unroll
    for (int a = 0; a < NA; ++a) {
      tma_load_at<false>(smem_u32(sQ + a * ATOM128), &tmQ, bar, 64 * a, row0, h);
      if (DUAL) tma_load_at<false>(smem_u32(sQ + (NA + a) * ATOM128), &tmQd, bar, 64 * a, row0, h);
    }
  };

  pdl_entry();
  const SeqLoad sl = seq_tile_load(p.seq, row0);
  const int nvalid = min(seq_total(p.seq) - row0, TR);
  if (nvalid <= 0) return;
  seq_tile_init(p.seq, row0, st_rows);
  // a barrier a thread; the first thread's own is the one that its loads complete
  if (threadIdx.x < 2 * NBARS) {
    const uint32_t b = threadIdx.x % NBARS;
    bar_init(smem_u32(&bars[0][0]) + 8 * threadIdx.x, 8 * b == B_P_FULL ? C::EW : 1);
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  if (threadIdx.x == 0) {
    abort_flag = redo_flag = 0;
    load_rows(smem_u32(&bars[0][0]) + B_Q_FULL);   // the rows' own operands need nothing of the sequences
  }
  if (warp == 1) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(
                     smem_u32(&tmem_slot)),
                 "r"(C::TMEM_COLS));
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;");
  }
  __syncthreads();
  seq_tile_fill(p.seq, row0, st_rows, C::THREADS, sl);
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tb = tmem_slot;
  volatile int* abort = &abort_flag;
  const int k0 = tile_lo(st_rows, row0, 0), lo1 = tile_lo(st_rows, row0, nvalid - 1);
  const KeyWalk<WIN, TK> kw(p, row0, nvalid, k0);
  const int nkt = kw.tiles;
  // whether some row does not attend to the whole of key tile j
  auto mixed = [&](int j) { return kw.mixed(j, row0, nvalid, lo1, p.window); };

  for (int walk = 0;; ++walk) {
  const bool careful = walk > 0;
  const uint32_t bb = smem_u32(&bars[walk][0]);
  if (warp == 0) {
    if (elect_one()) {
      // ---- TMA producer ---------------------------------------------------------------------
      if (walk) load_rows(bb + B_Q_FULL);
      int nk = 0, nv = 0;
      for (int j = 0; j < nkt; ++j) {
        const int st = j % C::STAGES;
        const uint32_t ph = ((j / C::STAGES) & 1) ^ 1;
        const int kr = kw.row(j);
        if (!twait(bb + B_K_EMPTY + 8 * st, ph, p.status, abort)) break;
        mbar_expect_tx_addr(bb + B_K_FULL + 8 * st, C::TILE_B);
        uint8_t* b = sK + st * C::TILE_B;
#pragma unroll
        for (int a = 0; a < NA; ++a) {
          tma_load_at<false>(smem_u32(b + a * C::KATOM), &tmK, bb + B_K_FULL + 8 * st, 64 * a, kr, hk);
          if (DUAL) tma_load_at<false>(smem_u32(b + (NA + a) * C::KATOM), &tmKd, bb + B_K_FULL + 8 * st, 64 * a, kr, hk);
        }
        ++nk;
        if (!twait(bb + B_V_EMPTY + 8 * st, ph, p.status, abort)) break;
        mbar_expect_tx_addr(bb + B_V_FULL + 8 * st, C::TILE_B);
        b = sV + st * C::TILE_B;
#pragma unroll
        for (int a = 0; a < NA; ++a) {
          tma_load_at<false>(smem_u32(b + a * C::KATOM), &tmV, bb + B_V_FULL + 8 * st, 64 * a, kr, hk);
          if (DUAL) tma_load_at<false>(smem_u32(b + (NA + a) * C::KATOM), &tmVd, bb + B_V_FULL + 8 * st, 64 * a, kr, hk);
        }
        ++nv;
      }
      mbar_wait_addr(bb + B_Q_FULL, 0, p.status, FTC_WAIT_NS);
      drain_ring(bb + B_K_FULL, nk, C::STAGES, p.status);
      drain_ring(bb + B_V_FULL, nv, C::STAGES, p.status);
    }
    __syncwarp();
  } else if (warp == 1) {
    // ---- products -------------------------------------------------------------------------------
    constexpr uint32_t idS = idesc_bf16(TR, TK), idS2 = idesc_bf16(TR, 2 * TK);
    constexpr uint32_t idO = idesc_bf16(TR, HDP) | (1u << 16), idO2 = idesc_bf16(TR, 2 * HDP) | (1u << 16);
    const uint32_t dQ = kdesc(smem_u32(sQ)), dQd = dQ + (NA * ATOM128 >> 4);
    const uint32_t dKs = kdesc(smem_u32(sK)), mVs = ndesc(smem_u32(sV), C::KATOM);
    constexpr uint32_t ST = C::TILE_B >> 4;
    auto scores = [&](int j) -> bool {
      const int st = j % C::STAGES;
      if (!rwait(bb + B_K_FULL + 8 * st, (j / C::STAGES) & 1, p.status, abort)) return false;
      tc_fence_after();
      if (elect_one()) {
        const uint32_t dK = dKs + st * ST;
#pragma unroll
        for (int kk = 0; kk < HDP / 16; ++kk) {
          const uint32_t qo = (kk >> 2) * (ATOM128 >> 4) + 2 * (kk & 3);
          const uint32_t ko = (kk >> 2) * (C::KATOM >> 4) + 2 * (kk & 3);
          mma_ss(tb + C::C_S, dQ + qo, dK + ko, DUAL ? idS2 : idS, kk > 0);
        }
        if (DUAL) {
#pragma unroll
          for (int kk = 0; kk < HDP / 16; ++kk)
            mma_ss(tb + C::C_SD, dQd + 2 * kk, dK + 2 * kk, idS, 1);
        }
        mma_commit_addr(bb + B_S_FULL);
        mma_commit_addr(bb + B_K_EMPTY + 8 * st);
      }
      __syncwarp();
      return true;
    };
    bool ok = rwait(bb + B_Q_FULL, 0, p.status, abort) && scores(0);
    for (int j = 0; ok && j < nkt; ++j) {
      const int st = j % C::STAGES;
      const uint32_t ph = (j / C::STAGES) & 1;
      if (careful) {
        if (!rwait(bb + B_V_FULL + 8 * st, ph, p.status, abort)) break;
        if (lane < 8) bad[st][lane >> 2][lane & 3] = 0;
        __syncwarp();
        if (mixed(j)) scrub<DUAL>(sV + st * C::TILE_B, TK, NA, bad[st], lane);
        if (lane == 0) bar_arrive(bb + B_V_CLEAN + 8 * st);
        __syncwarp();
      }
      if (!rwait(bb + B_V_FULL + 8 * st, ph, p.status, abort)) break;
      if (!rwait(bb + B_P_FULL, j & 1, p.status, abort)) break;
      tc_fence_after();
      if (elect_one()) {
        const uint32_t mV = mVs + st * ST;
#pragma unroll
        for (int kk = 0; kk < TK / 16; ++kk) {
          const uint32_t acc = (j > 0 || kk > 0) ? 1u : 0u;
          // each 32 keys' P begins where their scores did
          const uint32_t pc = (kk >> 1) * 32 + 8 * (kk & 1);
          if (DUAL) {
            mma_ts(tb + C::C_O, tb + C::C_S + pc, mV + 128 * kk, idO2, acc);
            mma_ts(tb + C::C_T, tb + C::C_SD + pc, mV + 128 * kk, idO, 1);
          } else {
            mma_ts(tb + C::C_O, tb + C::C_S + pc, mV + 128 * kk, idO, acc);
          }
        }
        mma_commit_addr(bb + B_V_EMPTY + 8 * st);
      }
      __syncwarp();
      if (j + 1 < nkt && !scores(j + 1)) break;
    }
    // every product issued here has completed before the rows are read and TMEM is released
    if (elect_one()) mma_commit_addr(bb + B_DRAIN);
    __syncwarp();
    mbar_wait_addr(bb + B_DRAIN, 0, p.status, FTC_WAIT_NS);
  } else {
    // ---- rows: thread r owns row row0 + r (TMEM lane r) ----------------------------------------------
    const int q4 = warp & 3;
    const int r = q4 * 32 + lane;
    const uint32_t lanes = tb + (static_cast<uint32_t>(q4 * 32) << 16);
    const uint32_t aS = lanes + C::C_S, aSd = lanes + C::C_SD;
    const int lo = tile_lo(st_rows, row0, r);
    const uint64_t c2p = pair(p.c2, p.c2), scp = pair(p.scale, p.scale);
    float m2 = -INFINITY, l = 0.f, rs = 0.f;    // rs: sum P (S' - cen)
    float cen = 0.f;
    // a row's first whole tile, where its first one holds the end of another sequence
    const int j1 = kw.first_whole(lo, row0 + r, p.window);
    bool ok = true, hit = false, hitd = false;   // the row attends to a noted row of V, of V'
    for (int j = 0; j < nkt; ++j) {
      const int st = j % C::STAGES;
      const bool mx_tile = mixed(j);
      if (!rwait(bb + B_S_FULL, j & 1, p.status, abort)) { ok = false; break; }
      uint32_t own[TK / 32];      // the row's own keys of the tile
      if (mx_tile) {
        if (careful && !rwait(bb + B_V_CLEAN + 8 * st, (j / C::STAGES) & 1, p.status, abort)) {
          ok = false;
          break;
        }
        const int kb = kw.row(j);
#pragma unroll
        for (int c = 0; c < TK / 32; ++c) {
          own[c] = kw.bits(j, lo, row0 + r, p, kb + 32 * c);
          if (careful) {
            hit |= (own[c] & bad[st][0][c]) != 0;
            hitd |= DUAL && (own[c] & bad[st][1][c]) != 0;
          }
        }
      }
      tc_fence_after();
      // mixed tiles have code of their own: selects in the common one would be issued for every
      // element, taken or not
      // Scores come in groups of 16 columns, the next one while one is looked at; with tangents two
      // together, between whose parts there is enough to do (81 us for 79 otherwise, 16 heads, eight
      // sequences of 1024).
      constexpr int GROUPS = TK / 16;
      float sv[2][16], mx = -INFINITY;
      auto load_group = [&](int g) { tmem_ld16_nowait(aS + 16 * g, sv[g & 1]); };
      auto load_pair = [&](int g) {
        tmem_ld32_nowait(aS + 16 * g, sv[0]);
        tmem_wait_ld();
      };
      auto mask_group = [&](int g) {
#pragma unroll
        for (int i = 0; i < 16; ++i) sv[g & 1][i] = own[g >> 1] >> (16 * (g & 1) + i) & 1 ? sv[g & 1][i] : -INFINITY;
      };
      auto find_max = [&](auto masked) {
        if (!DUAL) {
          load_group(0);
          tmem_wait_ld();
        }
#pragma unroll
        for (int g = 0; g < GROUPS; ++g) {
          if (DUAL && g % 2 == 0) load_pair(g);
          if (!DUAL && g + 1 < GROUPS) load_group(g + 1);
          if constexpr (decltype(masked)::value) mask_group(g);
          const float* v = sv[g & 1];
          float y0 = mx, y1 = v[0];
#pragma unroll
          for (int i = 0; i < 16; i += 4) {
            y0 = fmaxf(fmaxf(y0, v[i]), v[i + 1]);
            y1 = fmaxf(fmaxf(y1, v[i + 2]), v[i + 3]);
          }
          mx = fmaxf(y0, y1);
          if (!DUAL && g + 1 < GROUPS) tmem_wait_ld();
        }
      };
      if (mx_tile) find_max(std::true_type{});
      else find_max(std::false_type{});
      const float t2 = mx * p.c2;
      float f = 1.f;
      // also where one key outweighs all before, with a window, or eight times all before.  Scores of std 1, 2, 3
      // and 8 in 16384 rows, window 1000 took 234, 285, 299 and 305 us with that and 233, 281, 287 and 301
      // without; 8192 rows, no window 342, 348, 384 and 446 against 338, 344, 376 and 432, and outweighed once
      // 341, 356, 409 and 468.
      bool again = DUAL && (j == j1 || ex2(t2 - m2 - (WIN ? 0.f : 3.f)) > l);
      if (t2 > m2 + TAU) {
        f = ex2(m2 - t2);
        m2 = t2;
        again = true;
      }
      l *= f;
      rs *= f;
      const float base = m2 == -INFINITY ? 0.f : m2;     // no key of the row so far: P = 0
      if (__any_sync(0xffffffffu, again)) {
        float dc = 0.f;
        if (DUAL) {
          // The mean with the weights P over all keys so far: rbar itself, if no more come or none that
          // weigh.
          float wl = 0.f, ws = 0.f;
          const uint64_t nmb = pair(-base, -base);
          auto mean = [&](auto masked) {
            constexpr bool MASK = decltype(masked)::value;
            uint64_t wl2 = 0, ws2 = 0;
            // (four groups in a row: with a window 282 us a training step against 279, 16 heads over 4, 8192
            // rows, window 257; without one the other way round, 336 against 342, one sequence of 8192)
#pragma unroll(WIN ? 2 : 4)
            for (int c0 = 0; c0 < TK; c0 += 16) {
              float x[16], y[16];
              tmem_ld16_nowait(aS + c0, x);
              tmem_ld16_nowait(aSd + c0, y);
              tmem_wait_ld();
              const uint32_t w = MASK ? (c0 < 32 ? own[0] : own[TK / 32 - 1]) >> (c0 & 16) : 0u;
#pragma unroll
              for (int i = 0; i < 16; i += 2) {
                const float2 e = halves(fma2(pair(x[i], x[i + 1]), c2p, nmb));
                float p0 = ex2(e.x), p1 = ex2(e.y);
                if (MASK) {
                  p0 = w >> i & 1 ? p0 : 0.f;
                  p1 = w >> (i + 1) & 1 ? p1 : 0.f;
                  y[i] = w >> i & 1 ? y[i] : 0.f;
                  y[i + 1] = w >> (i + 1) & 1 ? y[i + 1] : 0.f;
                }
                const uint64_t pp = pair(p0, p1);
                wl2 = add2(wl2, pp);
                ws2 = fma2(pp, pair(y[i], y[i + 1]), ws2);
              }
            }
            const float2 a = halves(wl2), b = halves(ws2);
            wl = a.x + a.y;
            ws = b.x + b.y;
          };
          if (!mx_tile) mean(std::false_type{});
          else mean(std::true_type{});
          if (again && m2 != -INFINITY) {
            dc = __fdividef(fmaf(cen, wl, -p.scale * ws) - rs, l + wl);
            rs = fmaf(dc, l, rs);
            cen -= dc;
          }
        }
        if (j > 0) {
          // scores j were issued behind the products of tile j - 1, which are done
#pragma unroll 1
          for (int c0 = 0; c0 < HDP; c0 += 16) {
            float v[16], t[16];
            tmem_ld16_nowait(lanes + C::C_O + c0, v);
            if (DUAL) tmem_ld16_nowait(lanes + C::C_T + c0, t);
            tmem_wait_ld();
#pragma unroll
            for (int i = 0; i < 16; ++i) {
              v[i] *= f;
              if (DUAL) t[i] = fmaf(dc, v[i], t[i] * f);
            }
            tmem_st16(lanes + C::C_O + c0, v);
            if (DUAL) tmem_st16(lanes + C::C_T + c0, t);
          }
        }
      }
      const uint64_t nm = pair(-base, -base), nc = pair(-cen, -cen);
      uint64_t l2 = 0, r2 = 0;
      auto probs = [&](auto masked) {
        constexpr bool MASK = decltype(masked)::value;
        // from the last 32 columns on, whose scores are still here (masked, too)
        auto group = [](int k) { return 2 * (TK / 32 - 1 - k / 2) + (k & 1); };
#pragma unroll
        for (int k = 0; k < GROUPS; ++k) {
          const int g = group(k), b = g & 1;
          float sd[16];
          if (DUAL && k > 1 && b == 0) load_pair(g);
          if (!DUAL && k > 0 && k + 1 < GROUPS) load_group(group(k + 1));
          if (DUAL) tmem_ld16(aSd + 16 * g, sd);
          if (MASK && k > 1) mask_group(g);
          if (DUAL && MASK) {   // the tangent of a masked score may be anything
#pragma unroll
            for (int i = 0; i < 16; ++i) sd[i] = own[g >> 1] >> (16 * b + i) & 1 ? sd[i] : 0.f;
          }
          uint32_t pk[8], psk[8];
#pragma unroll
          for (int i = 0; i < 16; i += 2) {
            const float2 x = halves(fma2(pair(sv[b][i], sv[b][i + 1]), c2p, nm));
            const float p0 = ex2(x.x), p1 = ex2(x.y);
            const uint64_t pp = pair(p0, p1);
            l2 = add2(l2, pp);
            pk[i / 2] = pack_bf16x2(p0, p1);
            if (DUAL) {
              const uint64_t ps = mul2(pp, fma2(pair(sd[i], sd[i + 1]), scp, nc));
              r2 = add2(r2, ps);
              psk[i / 2] = pack2(ps);
            }
          }
          if (!DUAL && k > 0 && k + 1 < GROUPS) tmem_wait_ld();
          // each 32 keys' P begins where their scores did
          tmem_st8(aS + 32 * (g >> 1) + 8 * b, pk);
          if (DUAL) tmem_st8(aSd + 32 * (g >> 1) + 8 * b, psk);
        }
      };
      if (mx_tile) probs(std::true_type{});
      else probs(std::false_type{});
      const float2 lh = halves(l2), rh = halves(r2);
      l += lh.x + lh.y;
      rs += rh.x + rh.y;
      tmem_wait_st();
      tc_fence_before();
      __syncwarp();
      if (lane == 0) bar_arrive(bb + B_P_FULL);
    }
    if (ok && rwait(bb + B_DRAIN, 0, p.status, abort) && !*abort) {
      tc_fence_after();
      const float inv = hit ? NAN : 1.f / l, invd = hitd ? NAN : inv;
      const float rc = DUAL ? rs / l : 0.f;     // rbar - cen
      float z = 0.f;
#pragma unroll 1
      for (int c = 0; c < HDP; c += 16) {
        float o[16], t[16];
        tmem_ld16_nowait(lanes + C::C_O + c, o);
        if (DUAL) tmem_ld16_nowait(lanes + C::C_T + c, t);
        tmem_wait_ld();
#pragma unroll
        for (int i = 0; i < 16; ++i) {
          o[i] *= inv;
          if (DUAL) t[i] = t[i] * invd - rc * o[i];
        }
#pragma unroll
        for (int i = 0; i < 16; ++i) {
          add_check(z, o[i]);
          if (DUAL) add_check(z, t[i]);
        }
        stage16<HDP>(smem, r, c, o);
        if (DUAL) stage16<HDP>(smem + TR * HDP * 2, r, c, t);
      }
      if (r < nvalid && z != 0.f) redo_flag = 1;
      if (r < nvalid) {
        const int64_t si = static_cast<int64_t>(h) * p.seq.rows + row0 + r;
        p.lse[si] = (m2 + log2f(l)) * LN2;
        if (DUAL) p.rbar[si] = cen + rc;
      }
    } else {
      ok = false;
    }
    // rows are staged over the operands, which every product has read; a warp without a result
    // writes none (the status says so)
    asm volatile("bar.sync 5, %0;" ::"n"(C::EW * 32) : "memory");
    if (ok) {
      const int64_t at = static_cast<int64_t>(row0) * p.ldo + h * p.D;
      stage_out<HDP, C::EW * 32>(smem, nvalid, p.D, p.ow + at, p.ldo, threadIdx.x - 64);
      if (DUAL)
        stage_out<HDP, C::EW * 32>(smem + TR * HDP * 2, nvalid, p.D, p.owd + at, p.ldo, threadIdx.x - 64);
    }
    tc_fence_before();
    fence_async_smem();
  }
  __syncthreads();
  tc_fence_after();
  // NaN is what z != 0 sees; a careful walk's result stands
  if (careful || !redo_flag || *abort) break;
  }
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

dim3 tile_grid(int x, int tiles) {
  return dim3(static_cast<unsigned>(x), static_cast<unsigned>(tiles < GRID_Y ? tiles : GRID_Y),
              static_cast<unsigned>((tiles + GRID_Y - 1) / GRID_Y));
}

TcParams2 tc_params(const AttnParams& a) {
  TcParams2 p;
  memset(&p, 0, sizeof(p));
  p.seq = a.seq;
  p.D = a.D;
  p.tiles = (a.seq.rows + TR - 1) / TR;
  p.Hkv = a.Hkv;
  p.G = a.Hq / a.Hkv;
  p.scale = a.scale;
  p.c2 = a.scale * LOG2E;
  p.ldo = a.ldo; p.lddo = a.lddo; p.lddq = a.lddq; p.lddk = a.lddk; p.lddv = a.lddv;
  p.o = a.o; p.od = a.od; p.d_o = a.d_o; p.d_od = a.d_od;
  p.ow = a.o; p.owd = a.od;
  p.dq = a.dq; p.dk = a.dk; p.dv = a.dv; p.dqd = a.dqd; p.dkd = a.dkd; p.dvd = a.dvd;
  p.lse = a.lse; p.rbar = a.rbar; p.Dr = a.Dr; p.Drd = a.Drd;
  p.status = a.status;
  p.window = a.window;
  p.sinks = a.sinks;
  return p;
}

template <bool DUAL, int HDP, int TKEYS, bool WIN>
cudaError_t launch_fwd(const AttnParams& a, cudaStream_t s) {
  using C = FwdCfg<DUAL, HDP, TKEYS, WIN>;
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
    return cudaFuncSetAttribute(attn_tc_fwd_kernel<DUAL, HDP, TKEYS, WIN>,
                                cudaFuncAttributeMaxDynamicSharedMemorySize, C::SMEM);
  });
  if (e != cudaSuccess) return e;
  const TcParams2 p = tc_params(a);
  return launch_k(attn_tc_fwd_kernel<DUAL, HDP, TKEYS, WIN>, tile_grid(a.Hq, p.tiles), dim3(C::THREADS),
                  C::SMEM, s, q, k, v, qd, kd, vd, p);
}

// ---- backward -------------------------------------------------------------------------------------
// Two kernels, so that every sum keeps a fixed order: attn_tc_bwd_q_kernel, one CTA per (query
// head, 128 query rows), walks key tiles for dQ (and computes D = rowsum(dO O) on its way), and
// attn_tc_bwd_kv_kernel, one CTA per (key/value head, 128 key rows), walks the query tiles of its
// group's heads for dK and dV.  Both recompute the scores.
//
// Key-row kernel, per query tile (scores transposed: key rows are TMEM lanes):
//   S^T = K Q^T,  S'^T = K' Q^T + K Q'^T,  dP^T = V dO^T,  dP'^T = V' dO^T + V dO'^T
//   P^T = exp(S^T - lse), P'^T = P^T (S'^T - rbar)       over S^T, S'^T as bf16
//   dV += P^T dO,  dV' += P'^T dO + P^T dO'
//   dS^T = P^T (dP^T - D),  dS'^T = P'^T (dP^T - D) + P^T (dP'^T - D')   over dP^T, dP'^T
//   dK += dS^T Q,  dK' += dS'^T Q + dS^T Q'
// The products run in the order  dV(i) S(i+1) | dK(i) dP(i+1):  while the row warps turn dP(i)
// into dS(i), the tensor cores work on dV(i) and S(i+1); while they turn S(i+1) into P(i+1), on
// dK(i) and dP(i+1).
// What bounds them (per SM): at 128 columns the seven products of a tile pair (query rows 1.04 us
// a pair of 128 by 128, key rows 1.43, 0.80 and 1.07 at the tensor cores' clocked rate); with
// tangents 0.98 and 1.32 us a pair of 128 by 64 (0.60, 0.80); at 64 columns without, the row
// warps' arithmetic and issue.  A CTA adds 6 us that nothing hides where one has the SM: its first
// loads 1.1, first scores 2 to 4, results 1.2 (query rows); 1.2, 1.5, 3 to 5 (key rows).  A
// single pass would need five products but add dQ up by atomics, in an order of the moment.
// Query-row kernel, per key tile:  dS as above, untransposed, over dP;  dQ += dS K,
// dQ' += dS' K + dS K'.  dP has two buffers, so that S(j+1) and dP(j+1) run while the row warps
// work on tile j.
// Position in a ring of N stages: the stage and the parity of its phase.
template <int N>
struct Ring {
  int st = 0;
  uint32_t ph = 0;
  __device__ __forceinline__ void next() {
    if (++st == N) {
      st = 0;
      ph ^= 1;
    }
  }
};

template <bool DUAL, int HDP>
struct BwdCfg {
  static constexpr int NA = HDP / 64;
  static constexpr int BT = HDP == 128 ? 128 : 64;         // streamed rows a tile
  static constexpr int NT = DUAL ? 2 : 1;
  static constexpr int CTAS = DUAL || HDP == 128 ? 1 : 2;
  static constexpr int EW = 8;                             // row warps
  static constexpr int THREADS = 96 + 32 * EW;             // loads, products, look-over, rows
  static constexpr int CW = BT * 4 / EW;                   // columns of a row thread
  static constexpr int OWN = (CW + 31) / 32;               // words of a bit a column
  static constexpr int OW = HDP * 4 / EW;                  // accumulator columns it brings out
  static constexpr int RES1 = NT * NA * ATOM128;           // K (K') or V (V'); Q (Q') or dO (dO')
  static constexpr int BATOM = BT * 128;
  static constexpr int TILE_B = NT * NA * BATOM;           // one streamed operand with its tangent
  // two rings: X is read to the end of a tile (Q, or K), Y only by its first products (dO, or V),
  // so X needs a stage more to be loaded ahead
  static constexpr int XS = HDP == 128 ? 3 : 5, YS = HDP == 128 ? 2 : 4;
  static constexpr int NSTAT = DUAL ? 4 : 2;               // -lse log2 e, -D (-rbar, -D')
  static constexpr int STAT_F = NSTAT * BT;
  static constexpr int OPND_B = 2 * RES1 + XS * TILE_B + YS * TILE_B;
  // the widest buffers leave no room to round their base up: it begins on a 1024-byte boundary
  // (the declared alignment), which the kernels check
  static constexpr int SLACK = HDP == 128 ? 0 : 1024;
  static constexpr int SMEM_Q = OPND_B + SLACK;
  static constexpr int SMEM_KV = OPND_B + 2 * STAT_F * 4 + SLACK;
  static_assert(SMEM_KV + 1024 <= 227 * 1024 && SMEM_Q + 2048 <= 227 * 1024, "a CTA's shared memory");
  // TMEM: S (S'), dP (dP'), then the accumulators, tangents behind their primal
  static constexpr uint32_t C_S = 0, C_SD = BT, C_DP = NT * BT, C_DPD = C_DP + BT;
  static constexpr uint32_t C_A = 2 * NT * BT;             // dV (dV')
  static constexpr uint32_t C_B = C_A + NT * HDP;          // dK (dK')
  static constexpr uint32_t COLS = C_B + NT * HDP;         // 256 or 512, all of it
  // query-row kernel: two buffers of dP (dP') behind each other, then dQ (dQ')
  static constexpr uint32_t DP_STEP = NT * BT, C_Q = 3 * NT * BT;
  static_assert((COLS == 256 || COLS == 512) && C_Q + NT * HDP == COLS, "TMEM columns");
};

// ---- sinks and the query rows that attend to them ------------------------------------------------
// With a window a key row has the query rows up to its window's end, but a sink has all of its
// sequence: walked by the CTA of its tile, it would hold up the whole launch.  So query rows are cut
// into chunks of p.chunk rows.  A sink's own tile takes the chunk that its sequence begins in; of
// every later chunk, in which one sequence at most has begun before it, a CTA of its own takes the
// rows that attend to that sequence's sinks from behind their windows.  The sums stay float32 and
// are added up in the order of the chunks (sink_sum_kernel).
// The row behind the last of a sequence's rows start .. end - 1 that its sinks' own tile takes.
__device__ __forceinline__ int near_end(const TcParams2& p, int start, int end) {
  const int base = start - start % p.chunk;
  return end - base > p.chunk ? base + p.chunk : end;
}
// Whether other chunks have sums of its sinks.
__device__ __forceinline__ bool has_far(const TcParams2& p, int start, int end) {
  return end - start > p.window && end - (start - start % p.chunk) > p.chunk;
}
// Sum k of `sums` of a sequence's sink `place`: slot c holds the tile's own of the sequence that
// begins in chunk c, slot chunks + c those of chunk c.
__device__ __forceinline__ int64_t part_at(const TcParams2& p, int sums, int hdp, int slot, int hk, int k,
                                           int place) {
  return (((static_cast<int64_t>(slot) * p.Hkv + hk) * sums + k) * p.sinks + place) * hdp;
}

// dK, dV (and tangents) of the sinks of the sequence that begins in chunk y and reaches behind it:
// CTAs of a key/value head, a thread four columns of a sink's sum.
constexpr int SINK_THREADS = 128;
template <bool DUAL, int HDP>
__global__ void __launch_bounds__(SINK_THREADS) sink_sum_kernel(const __grid_constant__ TcParams2 p) {
  constexpr int SUMS = DUAL ? 4 : 2, CH = HDP / 4;
  pdl_entry();
  const int hk = static_cast<int>(blockIdx.x) % p.Hkv, c0 = tile_index();
  if (c0 >= p.chunks - 1) return;
  const int row = (c0 + 1) * p.chunk;            // below seq.rows: there is a chunk behind c0
  if (row >= seq_total(p.seq)) return;
  const int start = seq_begin(p.seq, row), end = seq_end(p.seq, row);
  if (start / p.chunk != c0 || !has_far(p, start, end)) return;
  // start + window < end, so neither overflows
  const int first = max(c0 + 1, (start + p.window) / p.chunk), last = (end - 1) / p.chunk;
  const int i = static_cast<int>(blockIdx.x) / p.Hkv * SINK_THREADS + static_cast<int>(threadIdx.x);
  const int c = i % CH, place = i / CH % p.sinks, k = i / CH / p.sinks;
  if (k >= SUMS || 4 * c >= p.D || place >= end - start) return;
  float4 x = *reinterpret_cast<const float4*>(p.part + part_at(p, SUMS, HDP, c0, hk, k, place) + 4 * c);
#pragma unroll 8
  for (int j = first; j <= last; ++j) {
    const float4 v = *reinterpret_cast<const float4*>(p.part + part_at(p, SUMS, HDP, p.chunks + j, hk, k, place) + 4 * c);
    x = make_float4(x.x + v.x, x.y + v.y, x.z + v.z, x.w + v.w);
  }
  const bool isv = k < SUMS / 2;
  const float f = isv ? 1.f : p.scale;
  __nv_bfloat16* dst = k == 0 ? p.dv : !DUAL ? p.dk : k == 1 ? p.dvd : k == 2 ? p.dk : p.dkd;
  *reinterpret_cast<uint2*>(dst + (static_cast<int64_t>(start) + place) * (isv ? p.lddv : p.lddk) + hk * p.D + 4 * c) =
      make_uint2(pack_bf16x2(x.x * f, x.y * f), pack_bf16x2(x.z * f, x.w * f));
}

// The row warps' barrier.
template <int EW>
__device__ __forceinline__ void row_bar() {
  asm volatile("bar.sync 1, %0;" ::"n"(EW * 32) : "memory");
}

// D = rowsum(dO (*) O) of the tile's rows, and its tangent rowsum(dO' (*) O + dO (*) O'), by the
// row warps: the lanes of a row read its 16-byte chunks side by side.  ALL: every row's reads in flight
// together.
template <bool DUAL, int HDP, int EW, bool ALL>
__device__ __forceinline__ void row_dots(const TcParams2& p, int row0, int nvalid, int h, int w,
                                         int lane, float2* out) {
  constexpr int LPR = HDP / 8, STEP = EW * (32 / LPR);
  auto f8 = [](const uint4& w4, float (&v)[8]) {
    const uint32_t u[4] = {w4.x, w4.y, w4.z, w4.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      v[2 * i] = __uint_as_float(u[i] << 16);
      v[2 * i + 1] = __uint_as_float(u[i] & 0xffff0000u);
    }
  };
  const int c = 8 * (lane % LPR);
  constexpr int IT = TR / STEP, NB = ALL ? IT : DUAL || IT > 4 ? IT / 2 : IT;   // rows read together
#pragma unroll
  for (int i0 = 0; i0 < IT; i0 += NB) {
    uint4 x[NB][DUAL ? 4 : 2];
#pragma unroll
    for (int i = 0; i < NB; ++i) {
      const int r = w * (32 / LPR) + lane / LPR + (i0 + i) * STEP;
      const bool on = r < nvalid && c < p.D;
      const int64_t oo = (static_cast<int64_t>(row0) + r) * p.ldo + h * p.D + c;
      const int64_t og = (static_cast<int64_t>(row0) + r) * p.lddo + h * p.D + c;
      const uint4 z = make_uint4(0, 0, 0, 0);
      x[i][0] = on ? *reinterpret_cast<const uint4*>(p.o + oo) : z;
      x[i][1] = on ? *reinterpret_cast<const uint4*>(p.d_o + og) : z;
      if (DUAL) {
        x[i][DUAL ? 2 : 0] = on ? *reinterpret_cast<const uint4*>(p.od + oo) : z;
        x[i][DUAL ? 3 : 0] = on ? *reinterpret_cast<const uint4*>(p.d_od + og) : z;
      }
    }
#pragma unroll
    for (int i = 0; i < NB; ++i) {
      float o[8], g[8], od[8], gd[8], s = 0.f, sd = 0.f;
      f8(x[i][0], o);
      f8(x[i][1], g);
      if (DUAL) {
        f8(x[i][DUAL ? 2 : 0], od);
        f8(x[i][DUAL ? 3 : 0], gd);
      }
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        s += o[e] * g[e];
        if (DUAL) sd += o[e] * gd[e] + od[e] * g[e];
      }
#pragma unroll
      for (int k = LPR / 2; k > 0; k >>= 1) {
        s += __shfl_xor_sync(0xffffffffu, s, k);
        if (DUAL) sd += __shfl_xor_sync(0xffffffffu, sd, k);
      }
      if (lane % LPR == 0) out[w * (32 / LPR) + lane / LPR + (i0 + i) * STEP] = make_float2(s, sd);
    }
  }
}

template <bool DUAL, int HDP, bool WIN>
__global__ void __launch_bounds__(BwdCfg<DUAL, HDP>::THREADS, BwdCfg<DUAL, HDP>::CTAS)
    attn_tc_bwd_kv_kernel(const __grid_constant__ CUtensorMap tmK, const __grid_constant__ CUtensorMap tmV,
                          const __grid_constant__ CUtensorMap tmKd, const __grid_constant__ CUtensorMap tmVd,
                          const __grid_constant__ CUtensorMap tmQ, const __grid_constant__ CUtensorMap tmO,
                          const __grid_constant__ CUtensorMap tmQd, const __grid_constant__ CUtensorMap tmOd,
                          const __grid_constant__ TcParams2 p) {
  using C = BwdCfg<DUAL, HDP>;
  constexpr int NA = C::NA, BT = C::BT, CW = C::CW;
  extern __shared__ __align__(1024) uint8_t smem_raw[];
  // barriers, as byte offsets in a set; one set per walk
  constexpr uint32_t B_RES_FULL = 0, B_S_FULL = 8, B_DP_FULL = 16, B_P_FULL = 24, B_DS_FULL = 32,
                     B_DRAIN = 40, B_CLEAN = 48, B_READ = 64;
  constexpr uint32_t B_X_FULL = 80, B_X_EMPTY = B_X_FULL + 8 * C::XS, B_Y_FULL = B_X_EMPTY + 8 * C::XS,
                     B_Y_EMPTY = B_Y_FULL + 8 * C::YS;
  constexpr int NBARS = 10 + 2 * C::XS + 2 * C::YS;
  __shared__ __align__(8) uint64_t bars[2][NBARS];
  __shared__ uint32_t bad[2][2][4];            // rows of Q and dO, of Q' and dO'
  __shared__ SeqTile st_rows;
  __shared__ uint32_t tmem_slot;
  __shared__ int abort_flag, redo_flag;

  uint8_t* smem = reinterpret_cast<uint8_t*>(
      (reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~static_cast<uintptr_t>(1023));
  uint8_t* sRes = smem;                        // K (K'), V (V')
  uint8_t* sX = smem + 2 * C::RES1;            // Q (Q')
  uint8_t* sY = sX + C::XS * C::TILE_B;        // dO (dO')
  float* sStat = reinterpret_cast<float*>(sY + C::YS * C::TILE_B);   // two tiles' statistics
  if (C::SLACK == 0 && smem != smem_raw) {     // the whole grid alike, before any barrier
    if (threadIdx.x == 0 && p.status) atomicMax(p.status, DEV_SMEM_BASE);
    return;
  }
  // a cluster shares the query heads of a group; heads fastest; the first rows of a long
  // sequence (the longest walks) come first
  int rank, hk;
  asm("mov.u32 %0, %%cluster_ctarank;" : "=r"(rank));
  asm("mov.u32 %0, %%clusterid.x;" : "=r"(hk));
  const int tile = tile_index();
  // with sinks the last CTAs take a chunk of query rows each, all others a tile of key rows (first, the
  // shorter chunks filled less of the last round: 325 us a training step against 316, 16 heads over 4,
  // 16384 rows, window 512; 973 against 966 with 16 heads of 128 over 2, 24577 rows, window 1000)
  const int nfar = WIN && p.sinks > 0 ? p.chunks - 1 : 0;
  const int far = WIN && tile >= p.tiles ? tile - p.tiles + 1 : 0;
  if (WIN ? far > nfar : tile >= p.tiles) return;
  const int trow0 = WIN && far ? far * p.chunk : tile * TR;   // the tile whose sequences are looked up
  const int G = p.Gs, h0 = (hk * p.share + rank) * G;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  int row0 = trow0;
  auto load_rows = [&](uint32_t bar) {
    mbar_expect_tx_addr(bar, 2 * C::RES1);
#pragma unroll
    for (int a = 0; a < NA; ++a) {
      tma_load_at<false>(smem_u32(sRes + a * ATOM128), &tmK, bar, 64 * a, row0, hk);
      tma_load_at<false>(smem_u32(sRes + C::RES1 + a * ATOM128), &tmV, bar, 64 * a, row0, hk);
      if (DUAL) {
        tma_load_at<false>(smem_u32(sRes + (NA + a) * ATOM128), &tmKd, bar, 64 * a, row0, hk);
        tma_load_at<false>(smem_u32(sRes + C::RES1 + (NA + a) * ATOM128), &tmVd, bar, 64 * a, row0, hk);
      }
    }
  };

  pdl_entry();
  const SeqLoad sl = seq_tile_load(p.seq, trow0);
  int nvalid = min(seq_total(p.seq) - trow0, TR);
  if (nvalid <= 0) return;
  seq_tile_init(p.seq, trow0, st_rows);
  // a barrier a thread; the first thread's own is the one that its loads complete
  if (threadIdx.x < 2 * NBARS) {
    const uint32_t b = threadIdx.x % NBARS;
    bar_init(smem_u32(&bars[0][0]) + 8 * threadIdx.x, 8 * b == B_P_FULL || 8 * b == B_DS_FULL ? C::EW : 1);
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  if (threadIdx.x == 0) {
    abort_flag = redo_flag = 0;
    // the rows' own operands need nothing of the sequences
    if (!WIN || !far) load_rows(smem_u32(&bars[0][0]) + B_RES_FULL);
  }
  if (warp == 1) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(
                     smem_u32(&tmem_slot)),
                 "r"(C::COLS));
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;");
  }
  __syncthreads();
  seq_tile_fill(p.seq, trow0, st_rows, C::THREADS, sl);
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tb = tmem_slot;
  volatile int* abort = &abort_flag;
  // The key rows row0 .. row0 + nvalid - 1 walk the query rows q0 .. q1 - 1; a tile of those from
  // qa to qb attends to all of them.
  const int hi0 = tile_hi(st_rows, trow0, 0);
  int q0 = row0, q1 = tile_hi(st_rows, trow0, nvalid - 1), qa = row0 + nvalid - 1, qb = hi0;
  if constexpr (WIN) {
    if (far) {
      // the sinks of the chunk's first row's sequence, with the chunk's rows behind their windows
      row0 = tile_lo(st_rows, trow0, 0);
      nvalid = min(p.sinks, hi0 - row0);
      q1 = qb = min(hi0, trow0 + min(p.chunk, p.seq.rows - trow0));
      q0 = max(trow0, row0 + min(p.window, p.seq.rows - row0));
      qa = max(q0, row0 + nvalid - 1 + min(p.window, p.seq.rows - row0));
      if (row0 == trow0 || q0 >= q1) {               // the whole cluster alike
        if (warp == 1)
          asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tb), "r"(C::COLS));
        return;
      }
      if (threadIdx.x == 0) load_rows(smem_u32(&bars[0][0]) + B_RES_FULL);
    } else {
      const int lo1 = tile_lo(st_rows, row0, nvalid - 1);
      const int hi1 = q1, last = row0 + nvalid - 1;
      q1 = last + min(p.window, hi1 - last);
      if (lo1 + p.sinks > row0) q1 = max(q1, near_end(p, lo1, hi1));
      qb = row0 + min(p.window, hi0 - row0);
    }
  }
  const bool alone = p.share == 1;
  // Whether row q's sums leave as float32, for sink_sum_kernel: sinks that other CTAs have sums of too, as
  // slot and place (-1: no).  Looked up once a row: for each sum, with divisions, it took 7 us of a CTA's 68
  // (heads of 128).
  auto sink_slot = [&](int q) {
    if (!WIN || p.sinks == 0 || q >= nvalid) return -1;
    if (far) return (p.chunks + far) << 7 | q;
    const int start = tile_lo(st_rows, row0, q), place = row0 + q - start;
    return place < p.sinks && has_far(p, start, tile_hi(st_rows, row0, q)) ? start / p.chunk << 7 | place : -1;
  };
  const int nqt = (q1 - q0 + BT - 1) / BT;          // query tiles of a head
  const int ntile = nqt * G;
  // whether some key row is not attended to by the whole of query tile t
  auto mixed = [&](int t) { return q0 + t * BT < qa || q0 + t * BT + BT > qb; };

  for (int walk = 0;; ++walk) {
  const bool careful = walk > 0;
  const uint32_t bb = smem_u32(&bars[walk][0]);
  if (warp == 0) {
    if (elect_one()) {
      if (walk) load_rows(bb + B_RES_FULL);
      // ---- TMA producer ---------------------------------------------------------------------------
      int n = 0, t = 0, h = h0;
      Ring<C::XS> x;
      Ring<C::YS> y;
      for (; n < ntile; ++n) {
        const int qr = q0 + t * BT;
        if (!twait(bb + B_X_EMPTY + 8 * x.st, x.ph ^ 1, p.status, abort)) break;
        // both or neither: the waits at the end count them together
        if (!twait(bb + B_Y_EMPTY + 8 * y.st, y.ph ^ 1, p.status, abort)) break;
        uint32_t b = smem_u32(sX + x.st * C::TILE_B), bar = bb + B_X_FULL + 8 * x.st;
        mbar_expect_tx_addr(bar, C::TILE_B);
#pragma unroll
        for (int a = 0; a < NA; ++a) {
          tma_load_at<false>(b + a * C::BATOM, &tmQ, bar, 64 * a, qr, h);
          if (DUAL) tma_load_at<false>(b + (NA + a) * C::BATOM, &tmQd, bar, 64 * a, qr, h);
        }
        b = smem_u32(sY + y.st * C::TILE_B);
        bar = bb + B_Y_FULL + 8 * y.st;
        mbar_expect_tx_addr(bar, C::TILE_B);
#pragma unroll
        for (int a = 0; a < NA; ++a) {
          tma_load_at<false>(b + a * C::BATOM, &tmO, bar, 64 * a, qr, h);
          if (DUAL) tma_load_at<false>(b + (NA + a) * C::BATOM, &tmOd, bar, 64 * a, qr, h);
        }
        x.next();
        y.next();
        if (++t == nqt) { t = 0; ++h; }
      }
      mbar_wait_addr(bb + B_RES_FULL, 0, p.status, FTC_WAIT_NS);
      drain_ring(bb + B_X_FULL, n, C::XS, p.status);
      drain_ring(bb + B_Y_FULL, n, C::YS, p.status);
    }
    __syncwarp();
  } else if (warp == 2) {
    // ---- look-over: row statistics (negated, read a tile ahead) and mixed tiles ----------------------
    float v[C::NSTAT][BT / 32];
    auto read = [&](int t, int h) {
      const int64_t base = static_cast<int64_t>(h) * p.seq.rows;
#pragma unroll
      for (int e = 0; e < BT / 32; ++e) {
        const int row = q0 + t * BT + 32 * e + lane;
        const bool in = row < p.seq.rows;
        v[0][e] = in ? p.lse[base + row] * -LOG2E : 0.f;
        v[1][e] = in ? -p.Dr[base + row] : 0.f;
        if (DUAL) {
          v[2][e] = in ? -p.rbar[base + row] : 0.f;
          v[3][e] = in ? -p.Drd[base + row] : 0.f;
        }
      }
    };
    int t = 0, h = h0;
    read(0, h0);
    Ring<C::XS> x;
    Ring<C::YS> y;
    for (int i = 0; i < ntile; ++i) {
      const int sl = i & 1;
      const bool mx = mixed(t);
      // the row warps are done with the tile before the last one
      if (!rwait(bb + B_READ + 8 * sl, ((i >> 1) & 1) ^ 1, p.status, abort)) break;
      float* sst = sStat + sl * C::STAT_F;
#pragma unroll
      for (int k = 0; k < C::NSTAT; ++k)
#pragma unroll
        for (int e = 0; e < BT / 32; ++e) sst[k * BT + 32 * e + lane] = v[k][e];
      if (++t == nqt) { t = 0; ++h; }
      if (i + 1 < ntile) read(t, h);
      if (careful) {
        if (!rwait(bb + B_X_FULL + 8 * x.st, x.ph, p.status, abort)) break;
        if (!rwait(bb + B_Y_FULL + 8 * y.st, y.ph, p.status, abort)) break;
        if (mx) {
          if (lane < 8) bad[sl][lane >> 2][lane & 3] = 0;
          __syncwarp();
          scrub<DUAL>(sX + x.st * C::TILE_B, BT, NA, bad[sl], lane);
          scrub<DUAL>(sY + y.st * C::TILE_B, BT, NA, bad[sl], lane);
        }
        x.next();
        y.next();
      }
      __syncwarp();
      if (lane == 0) bar_arrive(bb + B_CLEAN + 8 * sl);
    }
  } else if (warp == 1) {
    // ---- products ------------------------------------------------------------------------------------
    constexpr uint32_t idS = idesc_bf16(TR, BT), idS2 = idesc_bf16(TR, 2 * BT);
    constexpr uint32_t idA = idesc_bf16(TR, HDP) | (1u << 16), idA2 = idesc_bf16(TR, 2 * HDP) | (1u << 16);
    const uint32_t dK = kdesc(smem_u32(sRes)), dV = dK + (C::RES1 >> 4);
    constexpr uint32_t RD = NA * ATOM128 >> 4;            // a resident operand's tangent
    const uint32_t kX = kdesc(smem_u32(sX)), mX = ndesc(smem_u32(sX), C::BATOM);
    const uint32_t kY = kdesc(smem_u32(sY)), mY = ndesc(smem_u32(sY), C::BATOM);
    constexpr uint32_t ST = C::TILE_B >> 4;
    // X Y^T into column c (and the tangent's next to it)
    auto score = [&](uint32_t x, uint32_t y, uint32_t c) {
#pragma unroll
      for (int kk = 0; kk < HDP / 16; ++kk)
        mma_ss(tb + c, x + (kk >> 2) * (ATOM128 >> 4) + 2 * (kk & 3),
                 y + (kk >> 2) * (C::BATOM >> 4) + 2 * (kk & 3), DUAL ? idS2 : idS, kk > 0);
      if (DUAL) {
#pragma unroll
        for (int kk = 0; kk < HDP / 16; ++kk)
          mma_ss(tb + c + BT, x + RD + 2 * kk, y + 2 * kk, idS, 1);
      }
    };
    // acc += A^T-rows (TMEM columns a, tangent a + BT) times streamed rows y
    auto accum = [&](uint32_t c, uint32_t a, uint32_t y, bool first) {
#pragma unroll
      for (int kk = 0; kk < BT / 16; ++kk) {
        // the two threads of a row keep their halves apart
        const uint32_t ac = a + (kk / (CW / 16)) * CW + (kk % (CW / 16)) * 8;
        const uint32_t acc = (!first || kk > 0) ? 1u : 0u;
        mma_ts(tb + c, tb + ac, y + 128 * kk, DUAL ? idA2 : idA, acc);
        if (DUAL) mma_ts(tb + c + HDP, tb + ac + BT, y + 128 * kk, idA, 1);
      }
    };
    Ring<C::XS> x, xd;      // of the tile whose scores are next, and of the one being added up
    Ring<C::YS> y, yd;
    // S of tile i, and dP
    auto s_scores = [&](int i) -> bool {
      if (careful && !rwait(bb + B_CLEAN + 8 * (i & 1), (i >> 1) & 1, p.status, abort)) return false;
      if (!rwait(bb + B_X_FULL + 8 * x.st, x.ph, p.status, abort)) return false;
      tc_fence_after();
      if (elect_one()) {
        score(dK, kX + x.st * ST, C::C_S);
        mma_commit_addr(bb + B_S_FULL);
      }
      __syncwarp();
      x.next();
      return true;
    };
    auto p_scores = [&]() -> bool {
      if (!rwait(bb + B_Y_FULL + 8 * y.st, y.ph, p.status, abort)) return false;
      tc_fence_after();
      if (elect_one()) {
        score(dV, kY + y.st * ST, C::C_DP);
        mma_commit_addr(bb + B_DP_FULL);
      }
      __syncwarp();
      y.next();
      return true;
    };
    bool ok = rwait(bb + B_RES_FULL, 0, p.status, abort) && s_scores(0) && p_scores();
    for (int i = 0; ok && i < ntile; ++i) {
      const bool more = i + 1 < ntile;
      if (!rwait(bb + B_P_FULL, i & 1, p.status, abort)) break;
      tc_fence_after();
      if (elect_one()) {
        accum(C::C_A, C::C_S, mY + yd.st * ST, i == 0);
        mma_commit_addr(bb + B_Y_EMPTY + 8 * yd.st);
      }
      __syncwarp();
      yd.next();
      if (more && !s_scores(i + 1)) break;
      if (!rwait(bb + B_DS_FULL, i & 1, p.status, abort)) break;
      tc_fence_after();
      if (elect_one()) {
        accum(C::C_B, C::C_DP, mX + xd.st * ST, i == 0);
        mma_commit_addr(bb + B_X_EMPTY + 8 * xd.st);
        bar_arrive(bb + B_READ + 8 * (i & 1));
      }
      __syncwarp();
      xd.next();
      if (more && !p_scores()) break;
    }
    if (elect_one()) mma_commit_addr(bb + B_DRAIN);
    __syncwarp();
    mbar_wait_addr(bb + B_DRAIN, 0, p.status, FTC_WAIT_NS);
  } else {
    // ---- rows: key row r (TMEM lane r), query columns cb .. cb + CW - 1 ---------------------------------
    const int q4 = warp & 3;
    const int r = q4 * 32 + lane;
    const int part = (warp - 3) >> 2, cb = part * CW;
    const uint32_t lane_base = tb + (static_cast<uint32_t>(q4 * 32) << 16) + cb;
    // the row behind its sequence's last; the sign bit marks a sequence's first row, which attends
    // to one key, itself
    // (with a window of one and no sinks all rows do)
    int lo = row0 + r, hi;
    if (WIN && far) {
      lo = max(q0, lo + min(p.window, q1 - lo));
      hi = q1;
    } else {
      const int start = tile_lo(st_rows, row0, r);
      hi = tile_hi(st_rows, row0, r);
      const bool lone = start == lo || (WIN && p.window == 1 && p.sinks == 0);
      if constexpr (WIN) {
        const int end = hi;
        hi = lo + min(p.window, end - lo);
        if (lo - start < p.sinks) hi = max(hi, near_end(p, start, end));
      }
      hi |= lone ? INT_MIN : 0;
    }
    const uint64_t c2p = pair(p.c2, p.c2), sc = pair(p.scale, p.scale);
    bool ok = true;
    int t = 0;
    for (int i = 0; i < ntile; ++i) {
      const int sl = i & 1;
      const bool mx = mixed(t);
      // columns a .. b - 1 (of the tile) attend to this key
      const int a = lo - (q0 + t * BT), b = (hi & INT_MAX) - (q0 + t * BT);
      if (++t == nqt) t = 0;
      // the statistics
      if (!rwait(bb + B_CLEAN + 8 * sl, (i >> 1) & 1, p.status, abort)) { ok = false; break; }
      // the row's own columns, the noted ones of them, those noted in the tangents too
      uint32_t own[C::OWN], bads[C::OWN] = {}, badd[C::OWN] = {};
      if (mx) {
#pragma unroll
        for (int w = 0; w < C::OWN; ++w) {
          own[w] = col_bits(a - cb - 32 * w, b - 1 - cb - 32 * w);
          if (careful) {
            bads[w] = own[w] & (bad[sl][0][(cb >> 5) + w] >> (cb & 31));
            badd[w] = bads[w] | (DUAL ? own[w] & (bad[sl][1][(cb >> 5) + w] >> (cb & 31)) : 0u);
          }
        }
      }
      const float4* stat = reinterpret_cast<const float4*>(sStat + sl * C::STAT_F + cb);
      if (!rwait(bb + B_S_FULL, i & 1, p.status, abort)) { ok = false; break; }
      tc_fence_after();
      float pr[CW], pd[DUAL ? CW : 1];
      auto probs = [&](auto masked) {
        constexpr bool MASK = decltype(masked)::value;
#pragma unroll
        for (int c0 = 0; c0 < CW; c0 += 16) {
          float sv[16], sd[16];
          uint32_t pk[8], pdk[8];
          tmem_ld16_nowait(lane_base + C::C_S + c0, sv);
          if (DUAL) tmem_ld16_nowait(lane_base + C::C_SD + c0, sd);
          tmem_wait_ld();
#pragma unroll
          for (int e = 0; e < 16; e += 4) {
            const float4 l4 = stat[(c0 + e) / 4];
            const uint64_t lv[2] = {pair(l4.x, l4.y), pair(l4.z, l4.w)};
            float4 r4 = make_float4(0.f, 0.f, 0.f, 0.f);
            if (DUAL) r4 = stat[2 * (BT / 4) + (c0 + e) / 4];
            const uint64_t rv[2] = {pair(r4.x, r4.y), pair(r4.z, r4.w)};
#pragma unroll
            for (int u = 0; u < 2; ++u) {
              const int f = e + 2 * u, c = c0 + f;
              const float2 x = halves(fma2(pair(sv[f], sv[f + 1]), c2p, lv[u]));
              float p0 = ex2(x.x), p1 = ex2(x.y);
              const bool o0 = !MASK || (own[c >> 5] >> (c & 31) & 1);
              const bool o1 = !MASK || (own[c >> 5] >> (c & 31) & 2);
              if (!o0) p0 = 0.f;
              if (!o1) p1 = 0.f;
              pr[c] = p0;
              pr[c + 1] = p1;
              pk[f / 2] = pack_bf16x2(p0, p1);
              if (DUAL) {
                float2 y = halves(mul2(pair(p0, p1),
                                       fma2(pair(sd[f], sd[f + 1]), sc, rv[u])));
                if (!o0) y.x = 0.f;
                if (!o1) y.y = 0.f;
                pd[c] = y.x;
                pd[DUAL ? c + 1 : 0] = y.y;
                pdk[f / 2] = pack_bf16x2(y.x, y.y);
              }
            }
          }
          if (MASK && badd[c0 >> 5]) {
#pragma unroll
            for (int k = 0; k < 8; ++k) {
              pk[k] |= nan_pair(bads[c0 >> 5] >> ((c0 & 31) + 2 * k));
              if (DUAL) pdk[k] |= nan_pair(badd[c0 >> 5] >> ((c0 & 31) + 2 * k));
            }
          }
          tmem_st8(lane_base + C::C_S + c0 / 2, pk);
          if (DUAL) tmem_st8(lane_base + C::C_SD + c0 / 2, pdk);
        }
      };
      if (mx) probs(std::true_type{});
      else probs(std::false_type{});
      tmem_wait_st();
      tc_fence_before();
      __syncwarp();
      if (lane == 0) bar_arrive(bb + B_P_FULL);
      if (!rwait(bb + B_DP_FULL, i & 1, p.status, abort)) { ok = false; break; }
      tc_fence_after();
      auto scores = [&](auto masked) {
        constexpr bool MASK = decltype(masked)::value;
#pragma unroll
        for (int c0 = 0; c0 < CW; c0 += 16) {
          float dp[16], dd[16];
          uint32_t sk[8], sdk[8];
          tmem_ld16_nowait(lane_base + C::C_DP + c0, dp);
          if (DUAL) tmem_ld16_nowait(lane_base + C::C_DPD + c0, dd);
          tmem_wait_ld();
#pragma unroll
          for (int e = 0; e < 16; e += 4) {
            const float4 d4 = stat[BT / 4 + (c0 + e) / 4];
            const uint64_t dv[2] = {pair(d4.x, d4.y), pair(d4.z, d4.w)};
            float4 g4 = make_float4(0.f, 0.f, 0.f, 0.f);
            if (DUAL) g4 = stat[3 * (BT / 4) + (c0 + e) / 4];
            const uint64_t gv[2] = {pair(g4.x, g4.y), pair(g4.z, g4.w)};
#pragma unroll
            for (int u = 0; u < 2; ++u) {
              const int f = e + 2 * u, c = c0 + f;
              const uint64_t pp = pair(pr[c], pr[c + 1]);
              const uint64_t x = add2(dv[u], pair(dp[f], dp[f + 1]));
              float2 s = halves(mul2(pp, x));
              const bool o0 = !MASK || (own[c >> 5] >> (c & 31) & 1);
              const bool o1 = !MASK || (own[c >> 5] >> (c & 31) & 2);
              if (!o0) s.x = 0.f;
              if (!o1) s.y = 0.f;
              sk[f / 2] = pack_bf16x2(s.x, s.y);
              if (DUAL) {
                const uint64_t y = add2(gv[u], pair(dd[f], dd[f + 1]));
                float2 z = halves(fma2(pair(pd[c], pd[DUAL ? c + 1 : 0]), x, mul2(pp, y)));
                if (!o0) z.x = 0.f;
                if (!o1) z.y = 0.f;
                sdk[f / 2] = pack_bf16x2(z.x, z.y);
              }
            }
          }
          if (MASK && badd[c0 >> 5]) {
#pragma unroll
            for (int k = 0; k < 8; ++k) {
              sk[k] |= nan_pair(bads[c0 >> 5] >> ((c0 & 31) + 2 * k));
              if (DUAL) sdk[k] |= nan_pair(badd[c0 >> 5] >> ((c0 & 31) + 2 * k));
            }
          }
          tmem_st8(lane_base + C::C_DP + c0 / 2, sk);
          if (DUAL) tmem_st8(lane_base + C::C_DPD + c0 / 2, sdk);
        }
      };
      if (mx) {
        // a row with one key has P = 1 and dS = dS' = 0, of which dP - D, two sums of the same
        // terms, would leave their rounding
#pragma unroll
        for (int w = 0; w < C::OWN; ++w)
          if (hi < 0) own[w] &= ~col_bits(a - cb - 32 * w, a - cb - 32 * w);
        scores(std::true_type{});
      } else {
        scores(std::false_type{});
      }
      tmem_wait_st();
      tc_fence_before();
      __syncwarp();
      if (lane == 0) bar_arrive(bb + B_DS_FULL);
    }
    // Accumulators to shared memory, over the operands, which every product has read: the results' rows where
    // this CTA has all of their sums, else a tile of float32 rows each, 16-byte chunk c of row r at place
    // c ^ (r & 7).  (Always float32, the way out took 9 to 12 thousand cycles of a CTA's 21 to 120, results
    // four.)
    if (ok && rwait(bb + B_DRAIN, 0, p.status, abort) && !*abort) {
      tc_fence_after();
      const uint32_t acc = tb + (static_cast<uint32_t>(q4 * 32) << 16) + part * C::OW;
      const int at = WIN && alone ? sink_slot(r) : -1;
      float z = 0.f;
      // rolled up where two CTAs share the SM: code that runs once a CTA is not in the instruction cache when it
      // is wanted (16 heads over 4, 16384 rows, window 512 301 us a training step against 292; heads of 128 894
      // against 888 the other way round)
#pragma unroll(C::CTAS == 1 ? 4 : 1)
      for (int k = 0; k < 2 * C::NT; ++k)
#pragma unroll(C::CTAS == 1 ? 8 : 1)
        for (int c0 = 0; c0 < C::OW; c0 += 16) {
          float v[16];
          tmem_ld16(acc + C::C_A + k * HDP + c0, v);
#pragma unroll
          for (int e = 0; e < 16; ++e) add_check(z, v[e]);
          float* to = reinterpret_cast<float*>(smem + (k * TR + r) * (4 * HDP));
          int sw = r & 7;
          if (alone) {
            if (at < 0) {
              // dV (dV') as they are, dK (dK') with the scale of the scores
              const float f = k < C::NT ? 1.f : p.scale;
#pragma unroll
              for (int e = 0; e < 16; ++e) v[e] *= f;
              stage16<HDP>(smem + k * TR * HDP * 2, r, part * C::OW + c0, v);
              continue;
            }
            to = p.part + part_at(p, 2 * C::NT, HDP, at >> 7, hk, k, at & 127);
            sw = 0;
          }
#pragma unroll
          for (int e = 0; e < 16; e += 4)
            *reinterpret_cast<float4*>(to + 4 * (((part * C::OW + c0 + e) / 4) ^ sw)) =
                make_float4(v[e], v[e + 1], v[e + 2], v[e + 3]);
        }
      if (r < nvalid && z != 0.f) redo_flag = 1;
    }
    tc_fence_before();
    fence_async_smem();
  }
  __syncthreads();
  tc_fence_after();
  if (careful || !redo_flag || *abort) break;
  }
  if (alone) {
    // rows whose sums have left as float32 are written again by sink_sum_kernel
    if (warp >= 3 && !*abort && !(WIN && far)) {
#pragma unroll 1
      for (int k = 0; k < 2 * C::NT; ++k) {
        const int64_t ld = k < C::NT ? p.lddv : p.lddk;
        __nv_bfloat16* dst = k == 0 ? p.dv : !DUAL ? p.dk : k == 1 ? p.dvd : k == 2 ? p.dk : p.dkd;
        stage_out<HDP, C::EW * 32>(smem + k * TR * HDP * 2, nvalid, p.D, dst + row0 * ld + hk * p.D, ld,
                                   static_cast<int>(threadIdx.x) - 96);
      }
    }
    if (warp == 1) {
      asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tb),
                   "r"(C::COLS));
    }
    return;
  }
  int* sink_of = reinterpret_cast<int*>(smem + 2 * C::NT * TR * 4 * HDP);
  static_assert(2 * C::NT * TR * 4 * HDP + TR * 4 <= C::OPND_B, "behind the accumulators");
  if constexpr (WIN) {
    const int q = static_cast<int>(threadIdx.x) - 96;
    if (p.sinks > 0 && q >= 0 && q < TR && !*abort) sink_of[q] = sink_slot(q);
  }
  // The cluster's sums, rank by rank in order, each CTA its part of the rows; the second barrier
  // keeps a CTA's shared memory until the others have read it.  Short code counts here: it runs once
  // a CTA, and unrolled eight ranks wide it took 4.5 us of a CTA's 45 (16 heads of 64 over 4, two
  // CTAs a cluster, tangents), as much as the reads themselves.
  cluster_sync_all();
  if (warp >= 3 && !*abort) {
    const int rows = (TR + p.share - 1) / p.share;
    const int r0 = rank * rows, nr = min(min(r0 + rows, TR), nvalid) - r0;
    // A lane has four columns of one sum, so that a warp reads whole rows, and every RS-th row,
    // NI of them together.
    constexpr int CH = HDP / 4, RS = 32 * C::EW / (2 * C::NT * CH), NI = WIN ? (C::CTAS == 1 ? 8 : 4) : 2;
    static_assert(RS * 2 * C::NT * CH == 32 * C::EW, "every thread its columns");
    const int t = static_cast<int>(threadIdx.x) - 96, c = t % CH, k = t / CH % (2 * C::NT);
    const int end = r0 + nr;
    // dV (dV') as they are, dK (dK') with the scale of the scores
    const bool isv = k < C::NT;
    const float f = isv ? 1.f : p.scale;
    const int64_t ld = isv ? p.lddv : p.lddk;
    __nv_bfloat16* dst = (k == 0 ? p.dv : !DUAL ? p.dk : k == 1 ? p.dvd : k == 2 ? p.dk : p.dkd) +
                         row0 * ld + hk * p.D + 4 * c;
    const uint32_t own = smem_u32(smem) + k * TR * (4 * HDP);
#pragma unroll 1
    for (int r = r0 + t / (2 * C::NT * CH); r < end; r += NI * RS) {
      float4 x[NI];
#pragma unroll 1
      for (int j = 0; j < p.share; ++j) {
        const uint32_t from = j == rank ? own : dsmem_addr(own, j);
        float4 v[NI];
#pragma unroll
        for (int u = 0; u < NI; ++u) {
          const int q = (r + u * RS) & (TR - 1);
          v[u] = ld_cluster4(from + q * (4 * HDP) + ((c ^ (q & 7)) << 4));
        }
#pragma unroll
        for (int u = 0; u < NI; ++u)
          x[u] = j == 0 ? v[u] : make_float4(x[u].x + v[u].x, x[u].y + v[u].y, x[u].z + v[u].z, x[u].w + v[u].w);
      }
      uint32_t rows_left = (1u << NI) - 1;
      if (WIN && p.sinks > 0) {
#pragma unroll
        for (int u = 0; u < NI; ++u) {
          const int at = r + u * RS < end ? sink_of[(r + u * RS) & (TR - 1)] : -1;
          if (at < 0) continue;
          *reinterpret_cast<float4*>(p.part + part_at(p, 2 * C::NT, HDP, at >> 7, hk, k, at & 127) + 4 * c) = x[u];
          rows_left &= ~(1u << u);
        }
      }
      if (4 * c < p.D) {
#pragma unroll
        for (int u = 0; u < NI; ++u)
          if ((rows_left >> u & 1) && r + u * RS < end)
            *reinterpret_cast<uint2*>(dst + (r + u * RS) * ld) =
                make_uint2(pack_bf16x2(x[u].x * f, x[u].y * f), pack_bf16x2(x[u].z * f, x[u].w * f));
      }
    }
  }
  cluster_leave();
  if (warp == 1) {
    asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tb),
                 "r"(C::COLS));
  }
}

template <bool DUAL, int HDP, bool WIN>
__global__ void __launch_bounds__(BwdCfg<DUAL, HDP>::THREADS, BwdCfg<DUAL, HDP>::CTAS)
    attn_tc_bwd_q_kernel(const __grid_constant__ CUtensorMap tmQ, const __grid_constant__ CUtensorMap tmO,
                         const __grid_constant__ CUtensorMap tmQd, const __grid_constant__ CUtensorMap tmOd,
                         const __grid_constant__ CUtensorMap tmK, const __grid_constant__ CUtensorMap tmV,
                         const __grid_constant__ CUtensorMap tmKd, const __grid_constant__ CUtensorMap tmVd,
                         const __grid_constant__ TcParams2 p) {
  using C = BwdCfg<DUAL, HDP>;
  constexpr int NA = C::NA, BT = C::BT, CW = C::CW;
  extern __shared__ __align__(1024) uint8_t smem_raw[];
  // barriers, as byte offsets in a set; one set per walk
  constexpr uint32_t B_RES_FULL = 0, B_S_FULL = 8, B_S_FREE = 16, B_DRAIN = 24;
  // one for each buffer of dP: the next tile's phase may be complete before somebody has come to
  // wait for this one's, and a barrier tells only two phases apart
  constexpr uint32_t B_DP_FULL = 32, B_DS_FULL = 48;
  constexpr uint32_t B_X_FULL = 64, B_X_EMPTY = B_X_FULL + 8 * C::XS, B_CLEAN = B_X_EMPTY + 8 * C::XS,
                     B_Y_FULL = B_CLEAN + 8 * C::XS, B_Y_EMPTY = B_Y_FULL + 8 * C::YS;
  constexpr int NBARS = 8 + 3 * C::XS + 2 * C::YS;
  __shared__ __align__(8) uint64_t bars[2][NBARS];
  __shared__ uint32_t bad[C::XS][2][4];        // rows of K, of K'
  __shared__ float2 sD[TR];
  __shared__ SeqTile st_rows;
  __shared__ uint32_t tmem_slot;
  __shared__ int abort_flag, redo_flag;

  uint8_t* smem = reinterpret_cast<uint8_t*>(
      (reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~static_cast<uintptr_t>(1023));
  uint8_t* sRes = smem;                        // Q (Q'), dO (dO')
  uint8_t* sX = smem + 2 * C::RES1;            // K (K')
  uint8_t* sY = sX + C::XS * C::TILE_B;        // V (V')
  if (C::SLACK == 0 && smem != smem_raw) {     // the whole grid alike, before any barrier
    if (threadIdx.x == 0 && p.status) atomicMax(p.status, DEV_SMEM_BASE);
    return;
  }
  const int h = static_cast<int>(blockIdx.x), tile = tile_index();
  if (tile >= p.tiles) return;
  const int row0 = (p.tiles - 1 - tile) * TR;
  const int hk = h / p.G;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  auto load_rows = [&](uint32_t bar) {
    mbar_expect_tx_addr(bar, 2 * C::RES1);
#pragma unroll
    for (int a = 0; a < NA; ++a) {
      tma_load_at<false>(smem_u32(sRes + a * ATOM128), &tmQ, bar, 64 * a, row0, h);
      tma_load_at<false>(smem_u32(sRes + C::RES1 + a * ATOM128), &tmO, bar, 64 * a, row0, h);
      if (DUAL) {
        tma_load_at<false>(smem_u32(sRes + (NA + a) * ATOM128), &tmQd, bar, 64 * a, row0, h);
        tma_load_at<false>(smem_u32(sRes + C::RES1 + (NA + a) * ATOM128), &tmOd, bar, 64 * a, row0, h);
      }
    }
  };

  pdl_entry();
  const int nvalid = min(seq_total(p.seq) - row0, TR);
  if (nvalid <= 0) return;
  // The first three warps set up and look the sequences up, while the row warps sum D of the rows and read
  // their statistics: behind one another these took 4 us of a CTA's 17 (heads of 128, window 1000).
  float lse = 0.f, rbar = 0.f;
  if (warp < 3) {
    const SeqLoad sl = seq_tile_load(p.seq, row0);
    seq_tile_init(p.seq, row0, st_rows);
    // a barrier a thread; the first thread's own is the one that its loads complete
    static_assert(2 * NBARS <= 96, "a thread a barrier");
    if (threadIdx.x < 2 * NBARS) {
      const uint32_t b = threadIdx.x % NBARS;
      bar_init(smem_u32(&bars[0][0]) + 8 * threadIdx.x, 8 * b == B_S_FREE || (8 * b & ~8u) == B_DS_FULL ? C::EW : 1);
      asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (threadIdx.x == 0) {
      abort_flag = redo_flag = 0;
      load_rows(smem_u32(&bars[0][0]) + B_RES_FULL);   // the rows' own operands need nothing of the sequences
    }
    if (warp == 1) {
      asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(
                       smem_u32(&tmem_slot)),
                   "r"(C::COLS));
      asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;");
    }
    asm volatile("bar.sync 2, 96;" ::: "memory");
    seq_tile_fill(p.seq, row0, st_rows, 96, sl);
    tc_fence_before();
    asm volatile("bar.sync 2, 96;" ::: "memory");
    asm volatile("bar.arrive 3, %0;" ::"n"(C::THREADS) : "memory");
  } else {
    const int64_t r = (warp & 3) * 32 + lane, si = static_cast<int64_t>(h) * p.seq.rows + row0 + r;
    if (r < nvalid) {
      lse = p.lse[si];
      if (DUAL) rbar = p.rbar[si];
    }
    // D of the rows, a row's chunks of 16 bytes in neighbouring lanes
    row_dots<DUAL, HDP, C::EW, C::CTAS == 1>(p, row0, nvalid, h, warp - 3, lane, sD);
    asm volatile("bar.sync 3, %0;" ::"n"(C::THREADS) : "memory");
  }
  tc_fence_after();
  const uint32_t tb = tmem_slot;
  volatile int* abort = &abort_flag;
  const int k0 = tile_lo(st_rows, row0, 0), lo1 = tile_lo(st_rows, row0, nvalid - 1);
  const KeyWalk<WIN, BT> kw(p, row0, nvalid, k0);
  const int nkt = kw.tiles;
  auto mixed = [&](int j) { return kw.mixed(j, row0, nvalid, lo1, p.window); };

  for (int walk = 0;; ++walk) {
  const bool careful = walk > 0;
  const uint32_t bb = smem_u32(&bars[walk][0]);
  if (warp == 0) {
    if (elect_one()) {
      if (walk) load_rows(bb + B_RES_FULL);
      // ---- TMA producer ---------------------------------------------------------------------------
      int n = 0;
      Ring<C::XS> x;
      Ring<C::YS> y;
      for (; n < nkt; ++n) {
        const int kr = kw.row(n);
        if (!twait(bb + B_X_EMPTY + 8 * x.st, x.ph ^ 1, p.status, abort)) break;
        // both or neither: the waits at the end count them together
        if (!twait(bb + B_Y_EMPTY + 8 * y.st, y.ph ^ 1, p.status, abort)) break;
        uint32_t b = smem_u32(sX + x.st * C::TILE_B), bar = bb + B_X_FULL + 8 * x.st;
        mbar_expect_tx_addr(bar, C::TILE_B);
#pragma unroll
        for (int a = 0; a < NA; ++a) {
          tma_load_at<false>(b + a * C::BATOM, &tmK, bar, 64 * a, kr, hk);
          if (DUAL) tma_load_at<false>(b + (NA + a) * C::BATOM, &tmKd, bar, 64 * a, kr, hk);
        }
        b = smem_u32(sY + y.st * C::TILE_B);
        bar = bb + B_Y_FULL + 8 * y.st;
        mbar_expect_tx_addr(bar, C::TILE_B);
#pragma unroll
        for (int a = 0; a < NA; ++a) {
          tma_load_at<false>(b + a * C::BATOM, &tmV, bar, 64 * a, kr, hk);
          if (DUAL) tma_load_at<false>(b + (NA + a) * C::BATOM, &tmVd, bar, 64 * a, kr, hk);
        }
        x.next();
        y.next();
      }
      mbar_wait_addr(bb + B_RES_FULL, 0, p.status, FTC_WAIT_NS);
      drain_ring(bb + B_X_FULL, n, C::XS, p.status);
      drain_ring(bb + B_Y_FULL, n, C::YS, p.status);
    }
    __syncwarp();
  } else if (warp == 2) {
    // ---- look-over of mixed tiles: K (K') multiplies dS; V (V') only meets dO, whose product with a
    // masked key is dropped
    Ring<C::XS> x;
    for (int j = 0; careful && j < nkt; ++j) {
      if (!rwait(bb + B_X_FULL + 8 * x.st, x.ph, p.status, abort)) break;
      if (lane < 8) bad[x.st][lane >> 2][lane & 3] = 0;
      __syncwarp();
      if (mixed(j)) scrub<DUAL>(sX + x.st * C::TILE_B, BT, NA, bad[x.st], lane);
      if (lane == 0) bar_arrive(bb + B_CLEAN + 8 * x.st);
      x.next();
    }
  } else if (warp == 1) {
    // ---- products ------------------------------------------------------------------------------------
    constexpr uint32_t idS = idesc_bf16(TR, BT), idS2 = idesc_bf16(TR, 2 * BT);
    constexpr uint32_t idA = idesc_bf16(TR, HDP) | (1u << 16), idA2 = idesc_bf16(TR, 2 * HDP) | (1u << 16);
    const uint32_t dQ = kdesc(smem_u32(sRes)), dO = dQ + (C::RES1 >> 4);
    constexpr uint32_t RD = NA * ATOM128 >> 4;
    const uint32_t kX = kdesc(smem_u32(sX)), mX = ndesc(smem_u32(sX), C::BATOM);
    const uint32_t kY = kdesc(smem_u32(sY));
    constexpr uint32_t ST = C::TILE_B >> 4;
    auto score = [&](uint32_t x, uint32_t y, uint32_t c) {
#pragma unroll
      for (int kk = 0; kk < HDP / 16; ++kk)
        mma_ss(tb + c, x + (kk >> 2) * (ATOM128 >> 4) + 2 * (kk & 3),
                 y + (kk >> 2) * (C::BATOM >> 4) + 2 * (kk & 3), DUAL ? idS2 : idS, kk > 0);
      if (DUAL) {
#pragma unroll
        for (int kk = 0; kk < HDP / 16; ++kk)
          mma_ss(tb + c + BT, x + RD + 2 * kk, y + 2 * kk, idS, 1);
      }
    };
    Ring<C::XS> x, xd;      // of the tile whose scores are next, and of the one being added up
    Ring<C::YS> y;
    // the scores of tile j, ahead of its dP: S waits until the row warps have read the last one
    auto scores = [&](int j) -> bool {
      if (!rwait(bb + (careful ? B_CLEAN : B_X_FULL) + 8 * x.st, x.ph, p.status, abort)) return false;
      if (j > 0 && !rwait(bb + B_S_FREE, (j - 1) & 1, p.status, abort)) return false;
      tc_fence_after();
      if (elect_one()) {
        score(dQ, kX + x.st * ST, C::C_S);
        mma_commit_addr(bb + B_S_FULL);
      }
      __syncwarp();
      if (!rwait(bb + B_Y_FULL + 8 * y.st, y.ph, p.status, abort)) return false;
      tc_fence_after();
      if (elect_one()) {
        // buffer j & 1 held dS of tile j - 2, whose product has been issued
        score(dO, kY + y.st * ST, C::C_DP + (j & 1) * C::DP_STEP);
        mma_commit_addr(bb + B_DP_FULL + 8 * (j & 1));
        mma_commit_addr(bb + B_Y_EMPTY + 8 * y.st);
      }
      __syncwarp();
      x.next();
      y.next();
      return true;
    };
    bool ok = rwait(bb + B_RES_FULL, 0, p.status, abort) && scores(0);
    for (int j = 0; ok && j < nkt; ++j) {
      if (j + 1 < nkt && !scores(j + 1)) break;
      if (!rwait(bb + B_DS_FULL + 8 * (j & 1), (j >> 1) & 1, p.status, abort)) break;
      tc_fence_after();
      if (elect_one()) {
        const uint32_t mK = mX + xd.st * ST;
        const uint32_t a = tb + C::C_DP + (j & 1) * C::DP_STEP;
#pragma unroll
        for (int kk = 0; kk < BT / 16; ++kk) {
          const uint32_t ac = a + (kk / (CW / 16)) * CW + (kk % (CW / 16)) * 8;
          const uint32_t acc = (j > 0 || kk > 0) ? 1u : 0u;
          mma_ts(tb + C::C_Q, ac, mK + 128 * kk, DUAL ? idA2 : idA, acc);
          if (DUAL) mma_ts(tb + C::C_Q + HDP, ac + BT, mK + 128 * kk, idA, 1);
        }
        mma_commit_addr(bb + B_X_EMPTY + 8 * xd.st);
      }
      __syncwarp();
      xd.next();
    }
    if (elect_one()) mma_commit_addr(bb + B_DRAIN);
    __syncwarp();
    mbar_wait_addr(bb + B_DRAIN, 0, p.status, FTC_WAIT_NS);
  } else {
    // ---- rows: query row r (TMEM lane r), key columns cb .. cb + CW - 1 ---------------------------------
    const int q4 = warp & 3;
    const int r = q4 * 32 + lane;
    const int part = (warp - 3) >> 2, cb = part * CW;
    const uint32_t lane_base = tb + (static_cast<uint32_t>(q4 * 32) << 16) + cb;
    const int lo = tile_lo(st_rows, row0, r);
    // attends to one key, itself
    const bool lone = lo == row0 + r || (WIN && p.window == 1 && p.sinks == 0);
    const int64_t row = row0 + r, si = static_cast<int64_t>(h) * p.seq.rows + row;
    const bool on = r < nvalid;
    const float Dv = sD[r].x, Dd = sD[r].y;
    if (on && part == 0) {
      p.Dr[si] = Dv;
      if (DUAL) p.Drd[si] = Dd;
    }
    const float lse2 = lse * LOG2E, rb = rbar;
    const uint64_t c2p = pair(p.c2, p.c2), nl = pair(-lse2, -lse2), nD = pair(-Dv, -Dv);
    const uint64_t nr = pair(-rb, -rb), nDd = pair(-Dd, -Dd), sc = pair(p.scale, p.scale);
    bool ok = true;
    Ring<C::XS> x;
    for (int j = 0; j < nkt; ++j, x.next()) {
      const bool mx = mixed(j);
      uint32_t own[C::OWN], bads[C::OWN] = {}, badd[C::OWN] = {};   // as in the key-row kernel
      if (mx) {
        if (careful && !rwait(bb + B_CLEAN + 8 * x.st, x.ph, p.status, abort)) {
          ok = false;
          break;
        }
#pragma unroll
        for (int w = 0; w < C::OWN; ++w) {
          own[w] = kw.bits(j, lo, row0 + r, p, kw.row(j) + cb + 32 * w);
          if (careful) {
            bads[w] = own[w] & (bad[x.st][0][(cb >> 5) + w] >> (cb & 31));
            badd[w] = bads[w] | (DUAL ? own[w] & (bad[x.st][1][(cb >> 5) + w] >> (cb & 31)) : 0u);
          }
        }
      }
      if (!rwait(bb + B_S_FULL, j & 1, p.status, abort)) { ok = false; break; }
      tc_fence_after();
      float pr[CW], pd[DUAL ? CW : 1];
      auto probs = [&](auto masked) {
        constexpr bool MASK = decltype(masked)::value;
#pragma unroll
        for (int c0 = 0; c0 < CW; c0 += 16) {
          float sv[16], sd[16];
          tmem_ld16_nowait(lane_base + C::C_S + c0, sv);
          if (DUAL) tmem_ld16_nowait(lane_base + C::C_SD + c0, sd);
          tmem_wait_ld();
#pragma unroll
          for (int f = 0; f < 16; f += 2) {
            const int c = c0 + f;
            const float2 x = halves(fma2(pair(sv[f], sv[f + 1]), c2p, nl));
            pr[c] = ex2(x.x);
            pr[c + 1] = ex2(x.y);
            if (MASK && !(own[c >> 5] >> (c & 31) & 1)) pr[c] = 0.f;
            if (MASK && !(own[c >> 5] >> (c & 31) & 2)) pr[c + 1] = 0.f;
            if (DUAL) {
              const float2 y = halves(mul2(pair(pr[c], pr[c + 1]), fma2(pair(sd[f], sd[f + 1]), sc, nr)));
              pd[c] = y.x;
              pd[DUAL ? c + 1 : 0] = y.y;
            }
          }
        }
      };
      if (mx) probs(std::true_type{});
      else probs(std::false_type{});
      tc_fence_before();
      __syncwarp();
      if (lane == 0) bar_arrive(bb + B_S_FREE);
      if (!rwait(bb + B_DP_FULL + 8 * (j & 1), (j >> 1) & 1, p.status, abort)) { ok = false; break; }
      tc_fence_after();
      const uint32_t aP = lane_base + C::C_DP + (j & 1) * C::DP_STEP;
      auto scores = [&](auto masked) {
        constexpr bool MASK = decltype(masked)::value;
#pragma unroll
        for (int c0 = 0; c0 < CW; c0 += 16) {
          float dp[16], dd[16];
          uint32_t sk[8], sdk[8];
          tmem_ld16_nowait(aP + c0, dp);
          if (DUAL) tmem_ld16_nowait(aP + BT + c0, dd);
          tmem_wait_ld();
#pragma unroll
          for (int f = 0; f < 16; f += 2) {
            const int c = c0 + f;
            const uint64_t pp = pair(pr[c], pr[c + 1]);
            const uint64_t x = add2(pair(dp[f], dp[f + 1]), nD);
            float2 s = halves(mul2(pp, x));
            const bool o0 = !MASK || (own[c >> 5] >> (c & 31) & 1);
            const bool o1 = !MASK || (own[c >> 5] >> (c & 31) & 2);
            if (!o0) s.x = 0.f;
            if (!o1) s.y = 0.f;
            sk[f / 2] = pack_bf16x2(s.x, s.y);
            if (DUAL) {
              const uint64_t y = add2(pair(dd[f], dd[f + 1]), nDd);
              float2 z = halves(fma2(pair(pd[c], pd[DUAL ? c + 1 : 0]), x, mul2(pp, y)));
              if (!o0) z.x = 0.f;
              if (!o1) z.y = 0.f;
              sdk[f / 2] = pack_bf16x2(z.x, z.y);
            }
          }
          if (MASK && badd[c0 >> 5]) {
#pragma unroll
            for (int k = 0; k < 8; ++k) {
              sk[k] |= nan_pair(bads[c0 >> 5] >> ((c0 & 31) + 2 * k));
              if (DUAL) sdk[k] |= nan_pair(badd[c0 >> 5] >> ((c0 & 31) + 2 * k));
            }
          }
          tmem_st8(aP + c0 / 2, sk);
          if (DUAL) tmem_st8(aP + BT + c0 / 2, sdk);
        }
      };
      if (mx) {
#pragma unroll
        for (int w = 0; w < C::OWN; ++w) own[w] = lone ? 0u : own[w];    // dS = 0, as above
        scores(std::true_type{});
      } else {
        scores(std::false_type{});
      }
      tmem_wait_st();
      tc_fence_before();
      __syncwarp();
      if (lane == 0) bar_arrive(bb + B_DS_FULL + 8 * (j & 1));
    }
    if (ok && rwait(bb + B_DRAIN, 0, p.status, abort) && !*abort) {
      tc_fence_after();
      const uint32_t acc = tb + (static_cast<uint32_t>(q4 * 32) << 16) + part * C::OW;
      float z = 0.f;
#pragma unroll(C::CTAS == 1 ? 4 : 1)
      for (int k = 0; k < C::NT; ++k)
#pragma unroll(C::CTAS == 1 ? 8 : 1)
        for (int c0 = 0; c0 < C::OW; c0 += 16) {
          float v[16];
          tmem_ld16(acc + C::C_Q + k * HDP + c0, v);
#pragma unroll
          for (int e = 0; e < 16; ++e) {
            v[e] *= p.scale;
            add_check(z, v[e]);
          }
          stage16<HDP>(smem + k * TR * HDP * 2, r, part * C::OW + c0, v);
        }
      if (on && z != 0.f) redo_flag = 1;
    } else {
      ok = false;
    }
    row_bar<C::EW>();
    if (ok) {
      const int64_t at = static_cast<int64_t>(row0) * p.lddq + h * p.D;
      stage_out<HDP, C::EW * 32>(smem, nvalid, p.D, p.dq + at, p.lddq, threadIdx.x - 96);
      if (DUAL)
        stage_out<HDP, C::EW * 32>(smem + TR * HDP * 2, nvalid, p.D, p.dqd + at, p.lddq, threadIdx.x - 96);
    }
    tc_fence_before();
    fence_async_smem();
  }
  __syncthreads();
  tc_fence_after();
  if (careful || !redo_flag || *abort) break;
  }
  if (warp == 1) {
    asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tb),
                 "r"(C::COLS));
  }
}

// CTAs of a cluster that share the query heads of a group in the key-row kernel: the fewest
// (dividing the group, at most 8) that fill the GPU's places three times over.  A backward pass with
// one CTA a group, these, and as many as divide it: 8 heads of 64 over one, 512 rows 78, 28 and 28 us;
// 16 over 4 with tangents, 8192 rows 252, 236 and 264; 32 over 8, 16384 rows in sequences of 256 212,
// 212 and 292; 16 of 128 over 4, 12289 rows 669, 569 and 635.
// With a window below 2048 all walks are as long, and the fewest that fill the places once do (a fill of one):
// 16 heads over 4, 8192 rows, windows of 128, 512, 1024 and 2048 86, 127, 176 and 268 us backward against 98 to
// 143, 190 and 274 with a fill of three, with tangents 147, 246, 375 and 606 against 174, 270, 387 and 543; 16
// heads of 128 over 2, 24576 rows, window 1024 657 against 641, with sinks 685 against 711; a training step with
// four CTAs a group, 16384 rows, window 512 357 against 316.  Longer windows walk like none: windows of 2048,
// 4096 and 8192 in 16384 rows 535, 907 and 1563 against 530, 843 and 1397, in four sequences with 16 heads
// over 2 498, 618 and 612 against 446, 528 and 528 (504 without a window).
int kv_share(int group, int64_t ctas, int per_sm, int fill) {
  int best = 1;
  for (int n = 1; n <= 8 && n <= group; ++n) {
    if (group % n) continue;
    best = n;
    if (ctas * n >= static_cast<int64_t>(fill) * 152 * per_sm) break;
  }
  return best;
}

template <bool DUAL, int HDP, bool WIN>
cudaError_t launch_bwd(const AttnParams& a, cudaStream_t s) {
  using C = BwdCfg<DUAL, HDP>;
  const int N = a.seq.rows;
  // {q, dO} and {k, v} with their tangents, as 128-row and as streamed boxes
  CUtensorMap qr[4], qs[4], kr[4], ks[4];
  const __nv_bfloat16* qo[4] = {a.q, a.d_o, DUAL ? a.qd : nullptr, DUAL ? a.d_od : nullptr};
  const __nv_bfloat16* kv[4] = {a.k, a.v, DUAL ? a.kd : nullptr, DUAL ? a.vd : nullptr};
  for (int i = 0; i < 4; ++i) {
    const int64_t lq = i & 1 ? a.lddo : a.ldq, lk = i & 1 ? a.ldv : a.ldk;
    if (!head_map(&qr[i], qo[i], a.D, N, lq, a.Hq, TR) || !head_map(&kr[i], kv[i], a.D, N, lk, a.Hkv, TR))
      return cudaErrorInvalidValue;
    qs[i] = qr[i];
    ks[i] = kr[i];
    if (C::BT != TR && (!head_map(&qs[i], qo[i], a.D, N, lq, a.Hq, C::BT) ||
                        !head_map(&ks[i], kv[i], a.D, N, lk, a.Hkv, C::BT)))
      return cudaErrorInvalidValue;
  }
  static PerDeviceOnce once;
  cudaError_t e = once.run([](int&) {
    cudaError_t r = cudaFuncSetAttribute(attn_tc_bwd_kv_kernel<DUAL, HDP, WIN>,
                                         cudaFuncAttributeMaxDynamicSharedMemorySize, C::SMEM_KV);
    if (r != cudaSuccess) return r;
    return cudaFuncSetAttribute(attn_tc_bwd_q_kernel<DUAL, HDP, WIN>,
                                cudaFuncAttributeMaxDynamicSharedMemorySize, C::SMEM_Q);
  });
  if (e != cudaSuccess) return e;
  TcParams2 p = tc_params(a);
  p.share = kv_share(p.G, static_cast<int64_t>(p.tiles) * a.Hkv, C::CTAS, WIN && a.window < 2048 ? 1 : 3);
  p.Gs = p.G / p.share;
  e = launch_k(attn_tc_bwd_q_kernel<DUAL, HDP, WIN>, tile_grid(a.Hq, p.tiles), dim3(C::THREADS),
               C::SMEM_Q, s, qr[0], qr[1], qr[2], qr[3], ks[0], ks[1], ks[2], ks[3], p);
  if (e != cudaSuccess) return e;
  int nfar = 0;
  if constexpr (WIN) {
    p.chunk = window_chunk(a.window);
    p.chunks = (N - 1) / p.chunk + 1;              // N + chunk may pass 2^31 - 1
    p.part = a.part;
    nfar = a.sinks > 0 ? p.chunks - 1 : 0;
  }
  e = launch_cluster(attn_tc_bwd_kv_kernel<DUAL, HDP, WIN>, tile_grid(a.Hkv * p.share, p.tiles + nfar), p.share,
                     C::THREADS, C::SMEM_KV, s, kr[0], kr[1], kr[2], kr[3], qs[0], qs[1], qs[2], qs[3], p);
  if constexpr (WIN) {
    if (e == cudaSuccess && nfar > 0)
      e = launch_k(sink_sum_kernel<DUAL, HDP>,
                   tile_grid(a.Hkv * (((DUAL ? 4 : 2) * a.sinks * (HDP / 4) + SINK_THREADS - 1) / SINK_THREADS), nfar),
                   dim3(SINK_THREADS), 0, s, p);
  }
  return e;
}

}  // namespace
}  // namespace mf
