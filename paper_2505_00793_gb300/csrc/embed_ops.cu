// Embedding lookup with scaling on packed token rows (mf_embed_fwd) and the gradient of the table
// (mf_embed_bwd), each with its tangent:
//   y_r = s E[id_r],  y'_r = s E'[id_r]          (zeros where id_r is no row of the table)
//   dE_v = s sum_{r: id_r = v} dy_r,  dE'_v = s sum_{r: id_r = v} dy'_r
// Sums are float32, in an order that depends on the ids and the sizes alone.
//
// Memory bounds both.  The backward pass writes every row of the table, of which most may occur
// nowhere, and reads every token's row once.  Tokens are sorted by id (radix sort, stable, so that
// an id's tokens stay in their order), and the list of tokens and the list of table rows are merged
// into one path of "add a token's row" and "write a table's row", cut into ranges of equal length:
// however the ids are spread, every warp moves the same bytes.  A few tokens take one launch instead
// (embed_plan), in which a block has the table rows that it owns and all of their tokens.
//
// Measured (of 6.75 TB/s, a plain copy): 8192 tokens, 32768 ids, two tables of 1024 columns, float32: lookup
// 94 MB in 18 us (78 %), gradient 335 MB in 72 us (69 %), of which the sort takes 10, the sums 57 (87 %)
// and the rows that blocks share 4; 131071 tokens, 50001 ids, 768 columns of bf16 355 MB in 96 us (55 %):
// 23, 65 and 8.  4096 tokens, 8192 ids, 512 columns take one launch, 21 MB in 12 us, latencies.  Zeros
// written by blocks beside the sort, and sums of the ids that occur alone, took longer (87 us in the
// first): writes by themselves come at 4.5 TB/s, among reads at 6.
#include "attn_ops.h"
#include "internal.h"
#include "launch.cuh"
#include "packed_rows.cuh"

#include <limits.h>

namespace mf {
namespace {

constexpr unsigned ALL = 0xffffffffu;

// Four columns of a row as they lie in memory, n of them there (n >= 4: all), and their values.
// Apart, so that several loads are in flight before the first value is needed.
template <typename T>
struct Four;
template <>
struct Four<float> {
  float4 w;
  __device__ __forceinline__ void zero() { w = make_float4(0.f, 0.f, 0.f, 0.f); }
  __device__ __forceinline__ void load(const float* p, int n) {
    if (n >= 4) w = *reinterpret_cast<const float4*>(p);
    else w = make_float4(p[0], n > 1 ? p[1] : 0.f, n > 2 ? p[2] : 0.f, 0.f);
  }
  __device__ __forceinline__ float4 get() const { return w; }
};
template <>
struct Four<__nv_bfloat16> {
  uint2 w;
  __device__ __forceinline__ void zero() { w = make_uint2(0, 0); }
  __device__ __forceinline__ void load(const __nv_bfloat16* p, int n) {
    if (n >= 4) {
      w = *reinterpret_cast<const uint2*>(p);
    } else {
      const uint16_t* u = reinterpret_cast<const uint16_t*>(p);
      w = make_uint2(u[0] | (n > 1 ? static_cast<uint32_t>(u[1]) << 16 : 0u), n > 2 ? u[2] : 0u);
    }
  }
  __device__ __forceinline__ float4 get() const {
    return make_float4(__uint_as_float(w.x << 16), __uint_as_float(w.x & 0xffff0000u), __uint_as_float(w.y << 16),
                       __uint_as_float(w.y & 0xffff0000u));
  }
};
__device__ __forceinline__ void store4(float* p, int n, const float4& v) {
  if (n >= 4) {
    *reinterpret_cast<float4*>(p) = v;
    return;
  }
  p[0] = v.x;
  if (n > 1) p[1] = v.y;
  if (n > 2) p[2] = v.z;
}
__device__ __forceinline__ void store4(__nv_bfloat16* p, int n, const float4& v) {
  const __nv_bfloat162 a = __floats2bfloat162_rn(v.x, v.y), b = __floats2bfloat162_rn(v.z, v.w);
  if (n >= 4) {
    *reinterpret_cast<uint2*>(p) =
        make_uint2(*reinterpret_cast<const uint32_t*>(&a), *reinterpret_cast<const uint32_t*>(&b));
    return;
  }
  p[0] = a.x;
  if (n > 1) p[1] = a.y;
  if (n > 2) p[2] = b.x;
}
__device__ __forceinline__ float4 zero4() { return make_float4(0.f, 0.f, 0.f, 0.f); }
__device__ __forceinline__ void add4(float4& a, const float4& b) {
  a.x += b.x; a.y += b.y; a.z += b.z; a.w += b.w;
}
__device__ __forceinline__ float4 times4(const float4& a, float s) {
  return make_float4(a.x * s, a.y * s, a.z * s, a.w * s);
}

// ---- lookup ------------------------------------------------------------------------------------
constexpr int LOOK_THREADS = 256, LOOK_ITEMS = 4;

// A block takes `rows` rows, its threads four columns of a row each, LOOK_ITEMS of them in flight.
template <typename TE, typename TY>
__global__ void __launch_bounds__(LOOK_THREADS)
    embed_fwd_kernel(const __grid_constant__ EmbedParams p, int rows, int units) {
  pdl_entry();
  const int total = seq_total(p.seq);
  const int64_t first = static_cast<int64_t>(blockIdx.x) * rows;
  if (first >= total) return;
  const int r0 = static_cast<int>(first), n = min(rows, total - r0) * units;
  const bool tangent = blockIdx.y > 0;
  const TE* E = static_cast<const TE*>(tangent ? p.Ed : p.E);
  TY* y = static_cast<TY*>(tangent ? p.yd : p.y);
  for (int i0 = threadIdx.x; i0 < n; i0 += LOOK_ITEMS * LOOK_THREADS) {
    Four<TE> x[LOOK_ITEMS];
    int row[LOOK_ITEMS], col[LOOK_ITEMS];
#pragma unroll
    for (int k = 0; k < LOOK_ITEMS; ++k) {
      const int i = i0 + k * LOOK_THREADS;
      row[k] = i / units;
      col[k] = 4 * (i - row[k] * units);
      row[k] += r0;
      x[k].zero();
      if (i < n) {
        const int id = p.ids[row[k]];
        if (id >= 0 && id < p.vocab) x[k].load(E + id * p.ldE + col[k], p.dim - col[k]);
      }
    }
#pragma unroll
    for (int k = 0; k < LOOK_ITEMS; ++k)
      if (i0 + k * LOOK_THREADS < n)
        store4(y + row[k] * p.ldy + col[k], p.dim - col[k], times4(x[k].get(), p.scale));
  }
}

// ---- tokens sorted by id --------------------------------------------------------------------------
// Least significant digit first, digits of up to nine bits, each pass stable.  A block takes a tile of
// tokens, a warp neighbours of it.  A token goes behind all tokens of smaller digits, those of its digit
// in the tiles before, those in its tile's warps before, and those in its warp before.
constexpr int DIGITS = 512, SORT_THREADS = 512, SORT_WARPS = SORT_THREADS / 32;
constexpr int SORT_ROUNDS = 8, SORT_SUB = SORT_ROUNDS * SORT_THREADS;    // tokens of a thread, of a block at a time
constexpr int CLUSTER_TILES = 8, MAX_TILES = 64;
static_assert(SORT_THREADS == DIGITS, "a thread a digit");

struct SortShared {
  uint16_t cnt[SORT_WARPS][DIGITS];   // tokens of a warp with a digit; those of the warps before
  int base[DIGITS], wtot[SORT_WARPS];
};

// A token's key: its id, behind all of the table where it has none.
__device__ __forceinline__ int token_key(const EmbedParams& p, int row, int total) {
  const int id = p.ids[row];          // before it is known whether it counts: one wait less
  return row < total && id >= 0 && id < p.vocab ? id : p.vocab;
}

// Inclusive sum over a warp.
__device__ __forceinline__ int warp_sum_scan(int v, int lane) {
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const int x = __shfl_up_sync(ALL, v, o);
    if (lane >= o) v += x;
  }
  return v;
}

// Lanes of the warp whose d agrees in its lowest `bits`, nine at most.  (match.any takes longer the more values there
// are: 1500 cycles more a round of 32 warps.)
__device__ __forceinline__ unsigned peers_of(int d, int bits) {
  unsigned peers = ALL;
#pragma unroll
  for (int b = 0; b < 9; ++b) {
    const bool one = d >> b & 1;
    const unsigned set = __ballot_sync(ALL, one);
    peers &= b >= bits ? ALL : one ? set : ~set;
  }
  return peers;
}

// Ranks of a thread's tokens (x negative: none) among those of their digit in their warp, and in cnt those
// of the warps before; returns the tile's tokens of digit threadIdx.x.
__device__ __forceinline__ int rank_tokens(const int2 (&x)[SORT_ROUNDS], int (&rank)[SORT_ROUNDS], int rounds, int shift,
                                           int bits, SortShared& sh) {
  const int t = threadIdx.x, lane = t & 31, w = t >> 5, mask = (1 << bits) - 1;
  for (int i = t; i < SORT_WARPS * DIGITS / 8; i += SORT_THREADS)
    reinterpret_cast<uint4*>(&sh.cnt[0][0])[i] = make_uint4(0, 0, 0, 0);
  __syncthreads();
#pragma unroll
  for (int k = 0; k < SORT_ROUNDS; ++k) {
    if (k >= rounds) break;
    const bool in = x[k].x >= 0;
    const int d = (x[k].x >> shift) & mask;
    const unsigned peers = peers_of(d, bits) & __ballot_sync(ALL, in);
    const int old = in ? sh.cnt[w][d] : 0;
    __syncwarp();
    if (in && lane == __ffs(peers) - 1) sh.cnt[w][d] = static_cast<uint16_t>(old + __popc(peers));
    __syncwarp();
    rank[k] = old + __popc(peers & ((1u << lane) - 1));
  }
  __syncthreads();
  int run = 0;
#pragma unroll
  for (int k = 0; k < SORT_WARPS; ++k) {
    const int c = sh.cnt[k][t];
    sh.cnt[k][t] = static_cast<uint16_t>(run);
    run += c;
  }
  return run;
}

// Tokens of digits smaller than threadIdx.x, from those of each.
__device__ __forceinline__ int smaller_digits(int tokens, SortShared& sh) {
  const int t = threadIdx.x, lane = t & 31, w = t >> 5;
  const int inc = warp_sum_scan(tokens, lane);
  if (lane == 31) sh.wtot[w] = inc;
  __syncthreads();
  int ahead = inc - tokens;
#pragma unroll
  for (int k = 0; k < SORT_WARPS; ++k) ahead += k < w ? sh.wtot[k] : 0;
  return ahead;
}

// Up to 32768 tokens: one cluster, whose CTAs keep their tiles in shared memory and store tokens into one
// another's.
struct ClusterShared {
  SortShared s;
  int hist[2][DIGITS];                // of the tile, by pass
  int2 token[2][SORT_SUB];
};

__device__ __forceinline__ void cluster_barrier() {
  asm volatile("barrier.cluster.arrive.release.aligned;\n\t"
               "barrier.cluster.wait.acquire.aligned;" ::: "memory");
}
// This address in the shared memory of the cluster's CTA `rank`.
__device__ __forceinline__ uint32_t in_cta(const void* at, int rank) {
  uint32_t a;
  asm("mapa.shared::cluster.u32 %0, %1, %2;"
      : "=r"(a)
      : "r"(static_cast<uint32_t>(__cvta_generic_to_shared(at))), "r"(rank));
  return a;
}

__global__ void __launch_bounds__(SORT_THREADS)
    token_cluster_kernel(const __grid_constant__ EmbedParams p, const __grid_constant__ EmbedPlan m, int2* list) {
  extern __shared__ __align__(16) uint8_t raw[];
  ClusterShared& sh = *reinterpret_cast<ClusterShared*>(raw);
  pdl_entry();
  const int t = threadIdx.x, lane = t & 31, w = t >> 5, tile = blockIdx.x;
  const int total = seq_total(p.seq), first = tile * m.tile, n = min(m.tile, p.seq.rows - first);
  const int rounds = m.tile / SORT_THREADS, mask = (1 << m.bits) - 1;
  int2 x[SORT_ROUNDS];
  int rank[SORT_ROUNDS];
#pragma unroll
  for (int k = 0; k < SORT_ROUNDS; ++k) {
    const int i = (w * rounds + k) * 32 + lane;
    x[k] = k < rounds && i < n ? make_int2(token_key(p, first + i, total), first + i) : make_int2(-1, 0);
  }
  for (int pass = 0; pass < m.passes; ++pass) {
    const int shift = pass * m.bits;
    const bool last = pass + 1 == m.passes;
    if (pass > 0) {
#pragma unroll
      for (int k = 0; k < SORT_ROUNDS; ++k) {
        const int i = (w * rounds + k) * 32 + lane;
        if (k < rounds && i < n) x[k] = sh.token[pass & 1][i];
      }
    }
    sh.hist[pass & 1][t] = rank_tokens(x, rank, rounds, shift, m.bits, sh.s);
    cluster_barrier();
    int before = 0, all = 0, c[CLUSTER_TILES];
#pragma unroll
    for (int k = 0; k < CLUSTER_TILES; ++k)
      asm volatile("ld.shared::cluster.u32 %0, [%1];" : "=r"(c[k]) : "r"(in_cta(&sh.hist[pass & 1][t], min(k, m.tiles - 1))));
#pragma unroll
    for (int k = 0; k < CLUSTER_TILES; ++k) {
      all += k < m.tiles ? c[k] : 0;
      before += k < tile ? c[k] : 0;
    }
    sh.s.base[t] = before + smaller_digits(all, sh.s);
    __syncthreads();
#pragma unroll
    for (int k = 0; k < SORT_ROUNDS; ++k) {
      if (k >= rounds) break;
      if (x[k].x < 0) continue;
      const int d = (x[k].x >> shift) & mask, at = sh.s.base[d] + sh.s.cnt[w][d] + rank[k];
      if (last) {
        list[at] = x[k];
      } else {
        const int cta = at / m.tile;
        asm volatile("st.shared::cluster.v2.u32 [%0], {%1, %2};" ::"r"(
                         in_cta(&sh.token[(pass + 1) & 1][at - cta * m.tile], cta)),
                     "r"(x[k].x), "r"(x[k].y)
                     : "memory");
      }
    }
    // tokens have arrived, and a histogram has been read before its buffer is written again or its CTA ends
    cluster_barrier();
  }
}

// More tokens: a launch for the first digit's table hist[tile][digit], and one a pass, which fills the next
// digit's table.
__global__ void __launch_bounds__(SORT_THREADS)
    token_hist_kernel(const __grid_constant__ EmbedParams p, const __grid_constant__ EmbedPlan m, int* hist) {
  __shared__ int cnt[DIGITS];
  pdl_entry();
  const int t = threadIdx.x, lane = t & 31, tile = blockIdx.x, total = seq_total(p.seq);
  cnt[t] = 0;
  for (int k = 1; k < m.passes; ++k) hist[(k * m.tiles + tile) * DIGITS + t] = 0;
  __syncthreads();
  const int64_t a = static_cast<int64_t>(tile) * m.tile;
  const int end = static_cast<int>(min(static_cast<int64_t>(p.seq.rows), a + m.tile));
  // a tile holds tokens, and the token behind its last step may lie behind 2^31 - 1
  for (int i0 = static_cast<int>(a);; i0 += SORT_SUB) {
    int d[SORT_ROUNDS];
#pragma unroll
    for (int k = 0; k < SORT_ROUNDS; ++k) {
      const int i = i0 + k * SORT_THREADS + t;
      d[k] = i < end ? token_key(p, i, total) & ((1 << m.bits) - 1) : -1;
    }
#pragma unroll
    for (int k = 0; k < SORT_ROUNDS; ++k) {
      if (i0 + k * SORT_THREADS >= end) break;
      const unsigned peers = peers_of(d[k], m.bits) & __ballot_sync(ALL, d[k] >= 0);
      if (d[k] >= 0 && lane == __ffs(peers) - 1) atomicAdd(&cnt[d[k]], __popc(peers));
    }
    if (end - i0 <= SORT_SUB) break;
  }
  __syncthreads();
  hist[tile * DIGITS + t] = cnt[t];
}

__global__ void __launch_bounds__(SORT_THREADS)
    token_sort_kernel(const __grid_constant__ EmbedParams p, const __grid_constant__ EmbedPlan m, int pass,
                      const int2* from, int2* to, int* hist) {
  __shared__ __align__(16) SortShared sh;
  pdl_entry();
  const int t = threadIdx.x, lane = t & 31, w = t >> 5, tile = blockIdx.x, total = seq_total(p.seq);
  const int shift = pass * m.bits, mask = (1 << m.bits) - 1;
  const int* h = hist + pass * m.tiles * DIGITS + t;
  int* next = pass + 1 < m.passes ? hist + (pass + 1) * m.tiles * DIGITS : nullptr;
  const int64_t a = static_cast<int64_t>(tile) * m.tile;
  const int end = static_cast<int>(min(static_cast<int64_t>(p.seq.rows), a + m.tile));
  const int rounds = min(m.tile / SORT_THREADS, SORT_ROUNDS);
  int tile_bits = 0;
  while ((m.tiles - 1) >> tile_bits) ++tile_bits;
  int2 x[SORT_ROUNDS];
  int rank[SORT_ROUNDS];
  auto load = [&](int s0) {
#pragma unroll
    for (int k = 0; k < SORT_ROUNDS; ++k) {
      const int i = s0 + (w * rounds + k) * 32 + lane;
      x[k] = make_int2(-1, 0);
      if (k < rounds && i < end) x[k] = pass == 0 ? make_int2(token_key(p, i, total), i) : from[i];
    }
  };
  load(static_cast<int>(a));
  int before = 0, all = 0;
#pragma unroll 16
  for (int k = 0; k < m.tiles; ++k) {
    const int c = h[k * DIGITS];
    all += c;
    before += k < tile ? c : 0;
  }
  int base = before + smaller_digits(all, sh);
  for (int s0 = static_cast<int>(a);; s0 += rounds * SORT_THREADS) {
    if (s0 > a) load(s0);
    const int mine = rank_tokens(x, rank, rounds, shift, m.bits, sh);
    sh.base[t] = base;
    base += mine;
    __syncthreads();
#pragma unroll
    for (int k = 0; k < SORT_ROUNDS; ++k) {
      if (k >= rounds) break;
      const bool in = x[k].x >= 0;
      int to_tile = 0, d = 0;
      if (in) {
        d = (x[k].x >> shift) & mask;
        const int at = sh.base[d] + sh.cnt[w][d] + rank[k];
        to[at] = x[k];
        to_tile = at / m.tile;
      }
      if (next) {
        d = (x[k].x >> (shift + m.bits)) & mask;
        const unsigned peers = peers_of(d, m.bits) & peers_of(to_tile, tile_bits) & __ballot_sync(ALL, in);
        if (in && lane == __ffs(peers) - 1) atomicAdd(&next[to_tile * DIGITS + d], __popc(peers));
      }
    }
    if (end - s0 <= rounds * SORT_THREADS) break;
    __syncthreads();                  // base and cnt are written again
  }
}

// ---- sums ---------------------------------------------------------------------------------------
// The path: step by step the next token of the list, if it belongs to table row v, is added to v's
// sum, else row v is written and v + 1 is next.  Token i of key k is taken at step i + k, so the
// state at a step is found by a search.  A warp takes NV slabs of 128 columns of a range of `per`
// steps.  A border of two ranges that cuts an id's tokens moves ahead of them, if there are fewer than 32
// of them before it; else both sides' sums are added up at the end: those of a block's ranges by the
// block, and where a block's own border cuts, through the workspace by embed_join_kernel.
// Four warps a block: 131071 tokens, 50001 ids, 768 columns of bf16 96 us; eight 104, two 98, sixteen 105.
constexpr int SUM_WARPS = 4, SLAB = 128;
constexpr int64_t SUM_HELD = 152 * 24;             // warps that the GPU holds

struct PathState {
  int i, v;              // tokens taken, rows written
  bool cut;              // inside a row's tokens
};

// Both ends of a range, by the halves of a warp: tokens taken before step d of this half.  key(i) is token i's.
template <typename Key>
__device__ __forceinline__ int path_search(const Key& key, int N, int64_t d, int lane) {
  int lo = 0, hi = N;
  const int l = lane & 15, sh = lane & 16;
  while (__any_sync(ALL, lo < hi)) {
    const int step = (hi - lo + 17) / 17;
    const int64_t x = lo + static_cast<int64_t>(l + 1) * step - 1;
    const bool ahead = x < hi && x + key(x) < d;
    const int c = __popc((__ballot_sync(ALL, ahead) >> sh) & 0xffffu);
    const int64_t top = lo + static_cast<int64_t>(c + 1) * step - 1;
    hi = static_cast<int>(min(static_cast<int64_t>(hi), top));
    lo = lo + c * step;
  }
  return lo;
}
template <typename Key>
__device__ __forceinline__ PathState path_state(const Key& key, int64_t d, int i, int V, int lane) {
  PathState s{i, static_cast<int>(d - i), false};
  if (s.v >= V) {
    s.v = V;
    return s;
  }
  const int j = i - 1 - lane;
  const unsigned mine = __ballot_sync(ALL, j >= 0 && key(j) == s.v);
  s.cut = mine == ALL;
  if (!s.cut) s.i -= __ffs(~mine) - 1;
  return s;
}

// Bytes of a row that are asked for together count: 256 bytes at a time of rows in any order come at
// 4.4 TB/s.  So a lane has four columns of NV neighbouring slabs.
template <typename TY, int NV>
__global__ void __launch_bounds__(32 * SUM_WARPS)
    embed_sum_kernel(const __grid_constant__ EmbedParams p, const __grid_constant__ EmbedPlan m, const int2* list,
                     int* headv, int* tailv, float* part) {
  __shared__ float4 heads[SUM_WARPS][NV][32], tails[SUM_WARPS][NV][32];
  __shared__ int head_row[SUM_WARPS], tail_row[1 + SUM_WARPS];  // -1: none; the first, of the block's own start
  constexpr int FLIGHT = 32 / sizeof(TY);      // loads in flight: 128 bytes a lane
  constexpr int AHEAD = FLIGHT / NV;
  pdl_entry();
  const int lane = threadIdx.x & 31;
  // a block's warps take neighbouring ranges of the same columns
  const int w = threadIdx.x >> 5;
  const int64_t group = blockIdx.x / m.parts, range = group * SUM_WARPS + w;
  const int part_of = static_cast<int>(blockIdx.x - group * m.parts);   // tangents' behind the primal ones
  const int half = m.parts / (p.dEd ? 2 : 1);
  const bool tangent = part_of >= half;
  const int slab = (tangent ? part_of - half : part_of) * NV;    // first of NV
  const int col = slab * SLAB + 4 * lane, cols = p.dim - col;
  const TY* dy = static_cast<const TY*>(tangent ? p.dyd : p.dy) + col;
  float* dE = (tangent ? p.dEd : p.dE) + col;
  const int V = p.vocab, N = p.seq.rows;
  // ranges behind the last are empty
  const int64_t steps = static_cast<int64_t>(N) + V, d0 = min(range * m.per, steps), d1 = min(d0 + m.per, steps);
  auto key_of = [&](int64_t i) { return list[i].x; };
  const int at = path_search(key_of, N, lane < 16 ? d0 : d1, lane);
  const PathState a = path_state(key_of, d0, __shfl_sync(ALL, at, 0), V, lane);
  const PathState b = path_state(key_of, d1, __shfl_sync(ALL, at, 16), V, lane);
  float4 acc[NV];
  auto zero = [&]() {
#pragma unroll
    for (int q = 0; q < NV; ++q) acc[q] = zero4();
  };
  zero();
  int v = a.v;
  bool head = a.cut;
  auto row_sum = [&](float f) {
    float* row = dE + v * p.lddE;
#pragma unroll
    for (int q = 0; q < NV; ++q)
      if (cols > q * SLAB) store4(row + q * SLAB, cols - q * SLAB, times4(acc[q], f));
  };
  auto write_to = [&](int to) {
    if (v >= to) return;
    if (head) {
#pragma unroll
      for (int q = 0; q < NV; ++q) heads[w][q][lane] = acc[q];
    } else {
      row_sum(p.scale);
    }
    head = false;
    zero();
    ++v;
#pragma unroll 2
    for (; v < to; ++v) row_sum(0.f);
  };
  auto entry = [&](int j) { return j + lane < b.i ? list[j + lane] : make_int2(V, 0); };
  int2 next = entry(a.i);
  for (int j = a.i; j < b.i; j += 32) {
    const int2 kp = next;
    next = entry(j + 32);
#pragma unroll 1
    for (int u0 = 0; u0 < 32 && j + u0 < b.i; u0 += AHEAD) {
      Four<TY> x[AHEAD][NV];
#pragma unroll
      for (int u = 0; u < AHEAD; ++u) {
        const int key = __shfl_sync(ALL, kp.x, u0 + u), row = __shfl_sync(ALL, kp.y, u0 + u);
        const TY* from = dy + row * p.lddy;
#pragma unroll
        for (int q = 0; q < NV; ++q) {
          x[u][q].zero();
          if (key < V && cols > q * SLAB) x[u][q].load(from + q * SLAB, cols - q * SLAB);
        }
      }
#pragma unroll
      for (int u = 0; u < AHEAD; ++u) {
        const int key = __shfl_sync(ALL, kp.x, u0 + u);
        if (key < V) {         // those without a table row come last
          write_to(key);
#pragma unroll
          for (int q = 0; q < NV; ++q) add4(acc[q], x[u][q].get());
        }
      }
    }
  }
  write_to(b.v);
#pragma unroll
  for (int q = 0; q < NV; ++q) tails[w][q][lane] = acc[q];       // of the row that the end cuts
  if (lane == 0) {
    head_row[w] = a.cut && b.v > a.v ? a.v : -1;
    tail_row[1 + w] = b.cut ? b.v : -1;
    if (w == 0) tail_row[0] = a.cut ? a.v : -1;
  }
  __syncthreads();
  // Range by range, a slab a warp: `open` is the sum of the row that the last end has cut.  It began before
  // the block as long as no range has written a row.
  if (w >= NV || slab + w >= m.slabs) return;
  const int64_t step = static_cast<int64_t>(m.slabs) * (p.dEd ? 2 : 1) * SLAB;
  // the block's own ends: head, and behind it tail, of all slabs, the tangents' behind
  float* mine = part + 2 * group * step + static_cast<int64_t>((tangent ? m.slabs : 0) + slab + w) * SLAB + 4 * lane;
  int before = -1;
  bool ours = false;                  // the open row's tokens begin in the block
  float4 open = zero4();
#pragma unroll 1
  for (int k = 0; k < SUM_WARPS; ++k) {
    const int hr = head_row[k], tr = tail_row[1 + k];
    if (hr >= 0) {
      add4(open, heads[k][w][lane]);
      if (ours) {
        if (cols > w * SLAB) store4(dE + hr * p.lddE + w * SLAB, cols - w * SLAB, times4(open, p.scale));
      } else {
        *reinterpret_cast<float4*>(mine) = open;
        before = hr;
      }
    }
    if (tr < 0) continue;
    if (hr >= 0 || tail_row[k] != tr) {       // else the range lies inside the row
      open = zero4();
      ours = true;
    }
    add4(open, tails[k][w][lane]);
  }
  const int last = tail_row[SUM_WARPS];
  if (last >= 0) *reinterpret_cast<float4*>(mine + step) = open;
  if (part_of == 0 && w == 0 && lane == 0) {
    headv[group] = before;
    tailv[group] = last;
  }
}

// Few tokens: one launch.  Block b of n owns the table's rows b, b + n, b + 2n, ... (the smallest ids are the
// most frequent) in 128 columns.  It looks all ids over for its rows, sorts what it finds in shared
// memory, and walks the path of its own tokens and rows, a range a warp.
constexpr int NEAR_WARPS = 16, NEAR_THREADS = 32 * NEAR_WARPS;
constexpr int NEAR_TOKENS = 6144, NEAR_OWN = 8192;             // and rows of a block, at most
constexpr int NEAR_EACH = 1024;                                // tokens a row of the table, at most
constexpr int NEAR_BITS = 13, NEAR_IDS = NEAR_TOKENS / NEAR_THREADS;
// Tokens of a warp's part of the ids.
__host__ __device__ constexpr int near_part(int rows) { return (rows + NEAR_THREADS - 1) / NEAR_THREADS * 32; }

constexpr int NEAR_SHARED = (2 * NEAR_TOKENS + NEAR_OWN) * 4;  // bytes, at most

template <typename TY>
__global__ void __launch_bounds__(NEAR_THREADS, 2)
    embed_near_kernel(const __grid_constant__ EmbedParams p, const __grid_constant__ EmbedPlan m) {
  constexpr int AHEAD = 8;
  constexpr uint32_t AT = (1u << NEAR_BITS) - 1;        // a token: its row's place in the block, and its own place
  extern __shared__ uint32_t near_raw[];
  __shared__ float4 heads[NEAR_WARPS][32], tails[NEAR_WARPS][32];
  __shared__ int head_row[NEAR_WARPS], tail_row[1 + NEAR_WARPS], wtot[NEAR_WARPS], found[NEAR_WARPS];
  pdl_entry();
  const int t = threadIdx.x, lane = t & 31, w = t >> 5, total = seq_total(p.seq);
  const int b = blockIdx.x / m.parts, n = m.blocks, slab = blockIdx.x - b * m.parts;
  const bool tangent = slab >= m.slabs;
  const int col = (tangent ? slab - m.slabs : slab) * SLAB + 4 * lane, cols = p.dim - col;
  const TY* dy = static_cast<const TY*>(tangent ? p.dyd : p.dy) + col;
  float* dE = (tangent ? p.dEd : p.dE) + b * p.lddE + col;
  const int64_t ld = n * p.lddE;                // from one row of the block to the next
  const int R = (p.vocab - b + n - 1) / n, S = near_part(p.seq.rows);
  uint32_t* raw = near_raw;                     // as they are found, by warps
  uint32_t* list = raw + NEAR_WARPS * S;        // side by side
  int* start = reinterpret_cast<int*>(list + NEAR_WARPS * S);    // tokens of a row; where they begin
  int id[NEAR_IDS];
#pragma unroll
  for (int k = 0; k < NEAR_IDS; ++k) {
    const int i = w * S + 32 * k + lane;
    id[k] = 32 * k < S && i < total ? p.ids[i] : -1;
  }
  for (int i = t; i < R; i += NEAR_THREADS) start[i] = 0;
  __syncthreads();
  int mine = 0;
#pragma unroll
  for (int k = 0; k < NEAR_IDS; ++k) {
    const int r = m.by ? __umulhi(id[k], m.by) : id[k];      // id / n
    const bool hit = id[k] >= 0 && id[k] < p.vocab && id[k] - r * n == b;
    const unsigned hits = __ballot_sync(ALL, hit);
    if (hit) {
      raw[w * S + mine + __popc(hits & ((1u << lane) - 1))] = static_cast<uint32_t>(r) << NEAR_BITS | (w * S + 32 * k + lane);
      atomicAdd(&start[r], 1);
    }
    mine += __popc(hits);
  }
  if (lane == 0) found[w] = mine;
  __syncthreads();
  // where rows' tokens begin: a thread sums neighbouring rows
  const int chunk = (R + NEAR_THREADS - 1) / NEAR_THREADS, c0 = min(t * chunk, R), c1 = min(c0 + chunk, R);
  int sum = 0;
  for (int i = c0; i < c1; ++i) sum += start[i];
  const int inc = warp_sum_scan(sum, lane);
  if (lane == 31) wtot[w] = inc;
  __syncthreads();
  int at = inc - sum, T = 0;
  for (int k = 0; k < NEAR_WARPS; ++k) {
    at += k < w ? wtot[k] : 0;
    T += found[k];
  }
  for (int i = c0; i < c1; ++i) {
    const int c = start[i];
    start[i] = at;
    at += c;
  }
  __syncthreads();
  // found tokens side by side, in their order, which one warp keeps as it sorts them
  int ahead = 0;
  for (int k = 0; k < w; ++k) ahead += found[k];
  for (int i = lane; i < mine; i += 32) list[ahead + i] = raw[w * S + i];
  __syncthreads();
  uint32_t* sorted = raw;
  if (w == 0)
    for (int j = 0; j < T; j += 32) {
      const bool in = j + lane < T;
      const uint32_t e = in ? list[j + lane] : ALL;
      const unsigned peers = __match_any_sync(ALL, e >> NEAR_BITS);
      const int old = in ? start[e >> NEAR_BITS] : 0, before = __popc(peers & ((1u << lane) - 1));
      __syncwarp();
      if (in && before == 0) start[e >> NEAR_BITS] = old + __popc(peers);
      if (in) sorted[old + before] = e;
      __syncwarp();
    }
  __syncthreads();

  const int steps = T + R, per = (steps + NEAR_WARPS - 1) / NEAR_WARPS;
  const int d0 = min(w * per, steps), d1 = min(d0 + per, steps);
  auto key_of = [&](int64_t i) { return static_cast<int>(sorted[i] >> NEAR_BITS); };
  const int ends = path_search(key_of, T, lane < 16 ? d0 : d1, lane);
  // all cuts stay where they are: the block joins them, and ranges are short
  auto state = [&](int d, int i) {
    PathState s{i, min(d - i, R), false};
    s.cut = s.v < R && i > 0 && key_of(i - 1) == s.v;
    return s;
  };
  const PathState a = state(d0, __shfl_sync(ALL, ends, 0)), z = state(d1, __shfl_sync(ALL, ends, 16));
  float4 acc = zero4();
  int v = a.v;
  bool head = a.cut;
  auto write_to = [&](int to) {
    if (v >= to) return;
    if (head) heads[w][lane] = acc;
    else if (cols > 0) store4(dE + v * ld, cols, times4(acc, p.scale));
    head = false;
    acc = zero4();
    ++v;
#pragma unroll 4
    for (; v < to; ++v)
      if (cols > 0) store4(dE + v * ld, cols, acc);
  };
  for (int j = a.i; j < z.i; j += 32) {
    const uint32_t kp = j + lane < z.i ? sorted[j + lane] : 0u;
#pragma unroll 1
    for (int u0 = 0; u0 < 32 && j + u0 < z.i; u0 += AHEAD) {
      Four<TY> x[AHEAD];
#pragma unroll
      for (int u = 0; u < AHEAD; ++u) {
        const uint32_t e = __shfl_sync(ALL, kp, u0 + u);
        x[u].zero();
        if (j + u0 + u < z.i && cols > 0) x[u].load(dy + static_cast<int64_t>(e & AT) * p.lddy, cols);
      }
#pragma unroll
      for (int u = 0; u < AHEAD; ++u) {
        const uint32_t e = __shfl_sync(ALL, kp, u0 + u);
        if (j + u0 + u < z.i) {
          write_to(static_cast<int>(e >> NEAR_BITS));
          add4(acc, x[u].get());
        }
      }
    }
  }
  write_to(z.v);
  tails[w][lane] = acc;
  if (lane == 0) {
    head_row[w] = a.cut && z.v > a.v ? a.v : -1;
    tail_row[1 + w] = z.cut ? z.v : -1;
    if (w == 0) tail_row[0] = -1;
  }
  __syncthreads();
  if (w > 0) return;
  float4 open = zero4();                        // as in embed_sum_kernel, of rows that all begin here
#pragma unroll 1
  for (int k = 0; k < NEAR_WARPS; ++k) {
    const int hr = head_row[k], tr = tail_row[1 + k];
    if (hr >= 0) {
      add4(open, heads[k][lane]);
      if (cols > 0) store4(dE + hr * ld, cols, times4(open, p.scale));
    }
    if (tr < 0) continue;
    if (hr >= 0 || tail_row[k] != tr) open = zero4();
    add4(open, tails[k][lane]);
  }
}

// Rows whose tokens lie in several blocks' ranges: the sums at the ends of the blocks before the one that
// writes the row, and that one's own, in their order.  A warp adds up to 31 such sums; more, the
// block's warps, neighbours each.
constexpr int JOIN_WARPS = 16;

__global__ void __launch_bounds__(32 * JOIN_WARPS)
    embed_join_kernel(const __grid_constant__ EmbedParams p, const __grid_constant__ EmbedPlan m, const int* headv, const int* tailv,
                      const float* part) {
  __shared__ int2 found[32 * JOIN_WARPS];
  __shared__ int count[JOIN_WARPS];
  __shared__ bool longer[32 * JOIN_WARPS];
  __shared__ float4 sums[JOIN_WARPS][32];
  pdl_entry();
  const int t = threadIdx.x, lane = t & 31, w = t >> 5;
  const int slab = blockIdx.y;
  const bool tangent = slab >= m.slabs;
  const int col = (tangent ? slab - m.slabs : slab) * SLAB + 4 * lane, cols = p.dim - col;
  float* dE = (tangent ? p.dEd : p.dE) + col;
  const int64_t step = static_cast<int64_t>(gridDim.y) * SLAB;
  const float* sum = part + static_cast<int64_t>(slab) * SLAB + 4 * lane;   // of group r: + 2 r step, its tail + step
  auto tail_sums = [&](int a, int b) {
    float4 acc = zero4();
#pragma unroll 16
    for (int k = a; k < b; ++k) add4(acc, *reinterpret_cast<const float4*>(sum + (2 * static_cast<int64_t>(k) + 1) * step));
    return acc;
  };
  auto write = [&](int group, int row, float4 acc) {
    add4(acc, *reinterpret_cast<const float4*>(sum + 2 * static_cast<int64_t>(group) * step));
    if (cols > 0) store4(dE + row * p.lddE, cols, times4(acc, p.scale));
  };
  for (int64_t r0 = blockIdx.x; r0 < m.groups; r0 += static_cast<int64_t>(32 * JOIN_WARPS) * gridDim.x) {
    const int64_t r = r0 + static_cast<int64_t>(t) * gridDim.x;
    const int v = r < m.groups ? headv[r] : -1;
    const unsigned hits = __ballot_sync(ALL, v >= 0);
    if (lane == 0) count[w] = __popc(hits);
    __syncthreads();
    int n = 0, at = 0;
    for (int k = 0; k < JOIN_WARPS; ++k) {
      at += k < w ? count[k] : 0;
      n += count[k];
    }
    if (v >= 0) found[at + __popc(hits & ((1u << lane) - 1))] = make_int2(static_cast<int>(r), v);
    __syncthreads();
    for (int e = w; e < n; e += JOIN_WARPS) {
      const int group = found[e].x, row = found[e].y, q = group - 1 - lane;
      const unsigned same = __ballot_sync(ALL, q >= 0 && tailv[max(q, 0)] == row);
      if (lane == 0) longer[e] = same == ALL;
      if (same != ALL) write(group, row, tail_sums(group - __ffs(~same) + 1, group));
    }
    __syncthreads();
    for (int e = 0; e < n; ++e) {
      if (!longer[e]) continue;
      const int group = found[e].x, row = found[e].y;
      int tails = 0;
      for (;;) {
        const int q = group - 1 - tails - t;
        const unsigned same = __ballot_sync(ALL, q >= 0 && tailv[max(q, 0)] == row);
        if (lane == 0) count[w] = same == ALL ? 32 : __ffs(~same) - 1;
        __syncthreads();
        int more = 0;
        for (int k = 0; k < JOIN_WARPS && more == 32 * k; ++k) more += count[k];
        __syncthreads();
        tails += more;
        if (more < 32 * JOIN_WARPS) break;
      }
      const int first = group - tails;
      float4 acc = tail_sums(first + static_cast<int>(static_cast<int64_t>(tails) * w / JOIN_WARPS),
                             first + static_cast<int>(static_cast<int64_t>(tails) * (w + 1) / JOIN_WARPS));
      sums[w][lane] = acc;
      __syncthreads();
      if (w == 0) {
        for (int k = 1; k < JOIN_WARPS; ++k) add4(acc, sums[k][lane]);
        write(group, row, acc);
      }
      __syncthreads();
    }
    __syncthreads();                      // found and count are written again
  }
}

int64_t up(int64_t x, int64_t to) { return (x + to - 1) / to * to; }

}  // namespace

EmbedPlan embed_plan(int64_t rows, int64_t vocab, int64_t dim, bool dual) {
  EmbedPlan m;
  m.slabs = static_cast<int>((dim + SLAB - 1) / SLAB);
  m.parts = m.slabs * (dual ? 2 : 1);
  // Up to 6144 tokens one launch of two blocks an SM, of 64 steps at least, if a block's rows fit: 4096 of 8192
  // ids, 512 columns of bf16 16 us against 28 (6144 tokens 18 against 30), 1000 of them 12 against 24;
  // of 600000 ids, 128 columns 57 to 66 against 71 to 73; two tables of 32768 by 1024 59 to 70 against 67 to
  // 73.  It takes longer, and the sort is taken, where a row has many tokens, as a block takes them all:
  // 1000 tokens of one id 20 us against 20, 2000 33 against 22, 6144 82 to 90 against 22 to 30, and of four
  // ids 41 against 30 (4096 31 against 30); and where slabs leave a part fewer than four blocks, which fill
  // the places badly: 4096 tokens of 8000 ids, 8192 columns (four) 76 to 86 against 77 to 79, with tangents
  // (two) 141 to 162 against 123, 20000 columns (one) 203 to 272 against 145.  (What the ids are is not known
  // here: 4096 of 50001, a third of them one, take 30 against 29.)
  const int64_t held = 2 * 152 / m.parts, some = (rows + vocab + 63) / 64;
  const int64_t blocks = held < some ? held : some;
  if (held >= 4 && rows <= NEAR_TOKENS && rows <= NEAR_EACH * vocab && (vocab + blocks - 1) / blocks <= NEAR_OWN) {
    const int64_t own = (vocab + blocks - 1) / blocks;
    m.blocks = static_cast<int>(blocks);
    // id / blocks as the upper half of a product: exact below 2^32 / blocks, and there are 304 blocks of 8192
    // ids at most
    m.by = blocks > 1 ? static_cast<uint32_t>(((int64_t{1} << 32) + blocks - 1) / blocks) : 0;
    m.shared = static_cast<int>((2 * NEAR_WARPS * near_part(static_cast<int>(rows)) + own) * sizeof(uint32_t));
    m.bytes = 16;                                       // no workspace
    return m;
  }
  int key = 1;
  while (key < 31 && (vocab >> key) > 0) ++key;          // keys 0 .. vocab
  m.passes = (key + 8) / 9;
  m.bits = (key + m.passes - 1) / m.passes;
  m.cluster = rows <= CLUSTER_TILES * SORT_SUB;
  const int64_t most = m.cluster ? CLUSTER_TILES : MAX_TILES;
  int64_t tile = up((rows + most - 1) / most, SORT_THREADS);
  if (tile > SORT_SUB) tile = up(tile, SORT_SUB);
  m.tile = static_cast<int>(tile);
  m.tiles = rows > 0 ? static_cast<int>((rows + tile - 1) / tile) : 0;
  const int64_t slabs = static_cast<int64_t>(m.slabs) * (dual ? 2 : 1), steps = rows + vocab;
  // Short ranges leave warps for all of the GPU and spread what is slow, but each costs a search.  64 steps
  // against 48, 96 and 128: 8192 tokens, 32768 ids, two tables of 1024 columns 72 us against 71, 78 and 85;
  // 131071 tokens, 50001 ids, 768 columns 96 against 101, 112 and 109.
  m.per = steps * slabs >= 2 * 64 * SUM_HELD ? 64 : 32;
  m.groups = static_cast<int>((steps + m.per * SUM_WARPS - 1) / (m.per * SUM_WARPS));
  m.list = 0;
  m.hist = up(2 * rows * static_cast<int64_t>(sizeof(int2)), 16);
  m.ends = m.hist + static_cast<int64_t>(m.passes) * m.tiles * DIGITS * sizeof(int);
  m.part = m.ends + up(2 * static_cast<int64_t>(m.groups) * sizeof(int), 16);
  m.bytes = m.part + 2 * static_cast<int64_t>(m.groups) * slabs * SLAB * sizeof(float);
  return m;
}

cudaError_t embed_fwd(const EmbedParams& p, bool e_bf16, bool y_bf16, cudaStream_t s) {
  const int units = (p.dim + 3) / 4;
  const int rows = units >= LOOK_THREADS * LOOK_ITEMS ? 1 : LOOK_THREADS * LOOK_ITEMS / units;
  const dim3 grid(static_cast<unsigned>((p.seq.rows - 1) / rows + 1), p.Ed ? 2 : 1);
  auto run = [&](auto kernel) { return launch_k(kernel, grid, dim3(LOOK_THREADS), 0, s, p, rows, units); };
  if (e_bf16)
    return y_bf16 ? run(embed_fwd_kernel<__nv_bfloat16, __nv_bfloat16>) : run(embed_fwd_kernel<__nv_bfloat16, float>);
  return y_bf16 ? run(embed_fwd_kernel<float, __nv_bfloat16>) : run(embed_fwd_kernel<float, float>);
}

cudaError_t embed_bwd(const EmbedParams& p, bool y_bf16, void* work, cudaStream_t s) {
  const bool dual = p.dEd != nullptr;
  EmbedPlan m = embed_plan(p.seq.rows, p.vocab, p.dim, dual);
  if (m.blocks) {
    auto near = [&](auto kernel, PerDeviceOnce& once) {
      const cudaError_t r = once.run([&](int&) {
        return cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, NEAR_SHARED);
      });
      if (r != cudaSuccess) return r;
      return launch_k(kernel, dim3(static_cast<unsigned>(m.blocks * m.parts)), dim3(NEAR_THREADS), m.shared, s, p, m);
    };
    static PerDeviceOnce once[2];
    return y_bf16 ? near(embed_near_kernel<__nv_bfloat16>, once[1]) : near(embed_near_kernel<float>, once[0]);
  }
  char* base = static_cast<char*>(work);
  int2* lists[2] = {reinterpret_cast<int2*>(base + m.list), reinterpret_cast<int2*>(base + m.list) + p.seq.rows};
  int* hist = reinterpret_cast<int*>(base + m.hist);
  int* headv = reinterpret_cast<int*>(base + m.ends);
  int* tailv = headv + m.groups;
  float* part = reinterpret_cast<float*>(base + m.part);
  cudaError_t e = cudaSuccess;
  if (m.tiles && m.cluster) {
    static PerDeviceOnce once;
    e = once.run([](int&) {
      return cudaFuncSetAttribute(token_cluster_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, sizeof(ClusterShared));
    });
    if (e == cudaSuccess)
      e = launch_cluster(token_cluster_kernel, dim3(m.tiles), m.tiles, SORT_THREADS, sizeof(ClusterShared), s, p, m,
                         lists[(m.passes - 1) & 1]);
  } else if (m.tiles) {
    e = launch_k(token_hist_kernel, dim3(m.tiles), dim3(SORT_THREADS), 0, s, p, m, hist);
    for (int k = 0; k < m.passes && e == cudaSuccess; ++k)
      e = launch_k(token_sort_kernel, dim3(m.tiles), dim3(SORT_THREADS), 0, s, p, m, k,
                   static_cast<const int2*>(lists[(k + 1) & 1]), lists[k & 1], hist);
  }
  if (e != cudaSuccess) return e;
  const int2* list = lists[(m.passes - 1) & 1];
  // Two slabs a warp for rows of bf16, where that leaves two rounds of warps: 131071 tokens, 50001 ids, 768
  // columns 96 us against 115, three 99; float32 rows gain nothing (83 us against 75 in the case of 1024).
  const int slabs = m.slabs * (dual ? 2 : 1);
  const int64_t warps = (static_cast<int64_t>(p.seq.rows) + p.vocab) / m.per * slabs;
  const int wide = y_bf16 && m.slabs > 1 && warps >= 4 * SUM_HELD ? 2 : 1;
  m.parts = (m.slabs + wide - 1) / wide * (dual ? 2 : 1);
  const int64_t blocks = static_cast<int64_t>(m.groups) * m.parts;
  if (blocks > INT_MAX) return cudaErrorInvalidValue;
  auto sum = [&](auto kernel) {
    return launch_k(kernel, dim3(static_cast<unsigned>(blocks)), dim3(32 * SUM_WARPS), 0, s, p, m, list, headv, tailv,
                    part);
  };
  e = !y_bf16 ? sum(embed_sum_kernel<float, 1>)
      : wide == 2 ? sum(embed_sum_kernel<__nv_bfloat16, 2>) : sum(embed_sum_kernel<__nv_bfloat16, 1>);
  if (e != cudaSuccess || m.groups < 2 || p.seq.rows < 32) return e;   // no border has 32 tokens of a row before it
  const int most = 2 * 152 / slabs;
  const int x = most < 1 ? 1 : most < m.groups ? most : m.groups;
  return launch_k(embed_join_kernel, dim3(static_cast<unsigned>(x), static_cast<unsigned>(slabs)),
                  dim3(32 * JOIN_WARPS), 0, s, p, m, headv, tailv, part);
}

}  // namespace mf
