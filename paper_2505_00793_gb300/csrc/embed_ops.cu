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
// however the ids are spread, every warp moves the same bytes.
#include "attn_ops.h"
#include "launch.cuh"
#include "packed_rows.cuh"

#include <limits.h>

namespace mf {
namespace {

constexpr unsigned ALL = 0xffffffffu;

// Four columns of a row, n of them there (n >= 4: all).
__device__ __forceinline__ float4 load4(const float* p, int n) {
  if (n >= 4) return *reinterpret_cast<const float4*>(p);
  return make_float4(p[0], n > 1 ? p[1] : 0.f, n > 2 ? p[2] : 0.f, 0.f);
}
__device__ __forceinline__ float4 load4(const __nv_bfloat16* p, int n) {
  if (n >= 4) {
    const uint2 w = *reinterpret_cast<const uint2*>(p);
    return make_float4(__uint_as_float(w.x << 16), __uint_as_float(w.x & 0xffff0000u),
                       __uint_as_float(w.y << 16), __uint_as_float(w.y & 0xffff0000u));
  }
  return make_float4(__bfloat162float(p[0]), n > 1 ? __bfloat162float(p[1]) : 0.f,
                     n > 2 ? __bfloat162float(p[2]) : 0.f, 0.f);
}
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
    float4 x[LOOK_ITEMS];
    int row[LOOK_ITEMS], col[LOOK_ITEMS];
#pragma unroll
    for (int k = 0; k < LOOK_ITEMS; ++k) {
      const int i = i0 + k * LOOK_THREADS;
      row[k] = i / units;
      col[k] = 4 * (i - row[k] * units);
      row[k] += r0;
      x[k] = zero4();
      if (i < n) {
        const int id = p.ids[row[k]];
        if (id >= 0 && id < p.vocab) x[k] = load4(E + id * p.ldE + col[k], p.dim - col[k]);
      }
    }
#pragma unroll
    for (int k = 0; k < LOOK_ITEMS; ++k)
      if (i0 + k * LOOK_THREADS < n)
        store4(y + row[k] * p.ldy + col[k], p.dim - col[k], times4(x[k], p.scale));
  }
}

// ---- tokens sorted by id --------------------------------------------------------------------------
// Least significant digit first, digits of up to nine bits, each pass stable.  A block takes a tile
// of tokens; hist[pass][tile][digit] says how many of a tile's tokens have a digit.  The first
// pass's table comes from the ids, each later one's from the pass before it, which knows where its
// tokens go.
constexpr int DIGITS = 512, SORT_THREADS = 1024, SORT_WARPS = SORT_THREADS / 32;
constexpr int SORT_ROUNDS = 4, SORT_SUB = SORT_THREADS * SORT_ROUNDS;
constexpr int MAX_TILES = 64;

// A token's key: its id, behind all of the table where it has none.
__device__ __forceinline__ int token_key(const EmbedParams& p, int row, int total) {
  if (row >= total) return p.vocab;
  const int id = p.ids[row];
  return id >= 0 && id < p.vocab ? id : p.vocab;
}

__global__ void __launch_bounds__(SORT_THREADS)
    token_hist_kernel(const __grid_constant__ EmbedParams p, const __grid_constant__ EmbedPlan m, int* hist) {
  __shared__ int cnt[DIGITS];
  pdl_entry();
  const int t = threadIdx.x, tile = blockIdx.x, lane = t & 31;
  const int total = seq_total(p.seq);
  if (t < DIGITS) {
    cnt[t] = 0;
    for (int k = 1; k < m.passes; ++k) hist[(k * m.tiles + tile) * DIGITS + t] = 0;
  }
  __syncthreads();
  const int64_t a = static_cast<int64_t>(tile) * m.tile;
  const int n = static_cast<int>(min(static_cast<int64_t>(m.tile), p.seq.rows - a));
  for (int i0 = 0; i0 < n; i0 += SORT_THREADS) {
    const int i = i0 + t;
    const int d = i < n ? token_key(p, static_cast<int>(a) + i, total) & ((1 << m.bits) - 1) : -1;
    const unsigned peers = __match_any_sync(ALL, d);
    if (d >= 0 && lane == __ffs(peers) - 1) atomicAdd(&cnt[d], __popc(peers));
  }
  __syncthreads();
  if (t < DIGITS) hist[tile * DIGITS + t] = cnt[t];
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

template <bool FIRST>
__global__ void __launch_bounds__(SORT_THREADS)
    token_sort_kernel(const __grid_constant__ EmbedParams p, const __grid_constant__ EmbedPlan m, int pass,
                      const int2* from, int2* to, int* hist) {
  __shared__ __align__(16) uint16_t cnt[SORT_WARPS][DIGITS];   // tokens of a warp with a digit; those before them
  __shared__ int base[DIGITS], half[2][DIGITS], wtot[DIGITS / 32];
  pdl_entry();
  const int t = threadIdx.x, tile = blockIdx.x, lane = t & 31, w = t >> 5;
  const int total = seq_total(p.seq), N = p.seq.rows;
  const int shift = pass * m.bits, mask = (1 << m.bits) - 1;
  const int* h = hist + pass * m.tiles * DIGITS;
  int* next = pass + 1 < m.passes ? hist + (pass + 1) * m.tiles * DIGITS : nullptr;

  // where this tile's tokens of a digit begin: behind all smaller digits and the tiles before
  {
    const int d = t % DIGITS, part = t / DIGITS;
    int before = 0, all = 0;
#pragma unroll 16
    for (int k = part; k < m.tiles; k += 2) {
      const int c = h[k * DIGITS + d];
      all += c;
      before += k < tile ? c : 0;
    }
    half[part][d] = all;
    if (part == 1) base[d] = before;
    __syncthreads();
    int sum = 0, inc = 0;
    if (t < DIGITS) {
      sum = half[0][d] + half[1][d];
      inc = warp_sum_scan(sum, lane);
      if (lane == 31) wtot[w] = inc;
    }
    __syncthreads();
    if (t < DIGITS) {
      int ahead = 0;
      for (int k = 0; k < w; ++k) ahead += wtot[k];
      base[d] += before + ahead + inc - sum;
    }
  }
  const int64_t a = static_cast<int64_t>(tile) * m.tile;
  const int end = static_cast<int>(min(static_cast<int64_t>(N), a + m.tile));
  for (int s0 = static_cast<int>(a); s0 < end; s0 += SORT_SUB) {
    for (int i = t; i < SORT_WARPS * DIGITS / 8; i += SORT_THREADS)
      reinterpret_cast<uint4*>(&cnt[0][0])[i] = make_uint4(0, 0, 0, 0);
    int2 x[SORT_ROUNDS];
    int rank[SORT_ROUNDS];
#pragma unroll
    for (int k = 0; k < SORT_ROUNDS; ++k) {
      const int i = s0 + (w * SORT_ROUNDS + k) * 32 + lane;     // a warp's tokens are neighbours
      x[k] = make_int2(-1, i);
      if (i < end) x[k] = FIRST ? make_int2(token_key(p, i, total), i) : from[i];
    }
    __syncthreads();
#pragma unroll
    for (int k = 0; k < SORT_ROUNDS; ++k) {
      const bool in = x[k].x >= 0;
      const int d = in ? (x[k].x >> shift) & mask : -1;
      const unsigned peers = __match_any_sync(ALL, d);
      const int old = in ? cnt[w][d] : 0;
      __syncwarp();
      if (in && lane == __ffs(peers) - 1) cnt[w][d] = static_cast<uint16_t>(old + __popc(peers));
      __syncwarp();
      rank[k] = old + __popc(peers & ((1u << lane) - 1));
    }
    __syncthreads();
    int run = 0;
    if (t < DIGITS)
#pragma unroll 8
      for (int k = 0; k < SORT_WARPS; ++k) {
        const int c = cnt[k][t];
        cnt[k][t] = static_cast<uint16_t>(run);
        run += c;
      }
    __syncthreads();
#pragma unroll
    for (int k = 0; k < SORT_ROUNDS; ++k) {
      const bool in = x[k].x >= 0;
      int at = 0, slot = -1;
      if (in) {
        const int d = (x[k].x >> shift) & mask;
        at = base[d] + cnt[w][d] + rank[k];
        to[at] = x[k];
        if (next) slot = at / m.tile * DIGITS + ((x[k].x >> (shift + m.bits)) & mask);
      }
      if (next) {
        const unsigned peers = __match_any_sync(ALL, slot);
        if (in && lane == __ffs(peers) - 1) atomicAdd(&next[slot], __popc(peers));
      }
    }
    __syncthreads();
    if (t < DIGITS) base[t] += run;
    // base and cnt are written again behind the next barrier only
  }
}

// ---- sums ---------------------------------------------------------------------------------------
// The path: step by step the next token of the list, if it belongs to table row v, is added to v's
// sum, else row v is written and v + 1 is next.  Token i of key k is taken at step i + k, so the
// state at a step is found by a search.  A warp takes 128 columns of a range of `per` steps.  A
// border of two ranges that cuts an id's tokens moves ahead of them, if there are fewer than 32
// of them before it; else both sides' sums go to the workspace, and embed_join_kernel adds them up.
constexpr int SUM_WARPS = 8, SLAB = 128, AHEAD = 8;

struct PathState {
  int i, v;              // tokens taken, rows written
  bool cut;              // inside a row's tokens
};

// Both ends of a range, by the halves of a warp: tokens taken before step d of this half.
__device__ __forceinline__ int path_search(const int2* list, int N, int64_t d, int lane) {
  int lo = 0, hi = N;
  const int l = lane & 15, sh = lane & 16;
  while (__any_sync(ALL, lo < hi)) {
    const int step = (hi - lo + 17) / 17;
    const int64_t x = lo + static_cast<int64_t>(l + 1) * step - 1;
    const bool ahead = x < hi && x + list[x].x < d;
    const int c = __popc((__ballot_sync(ALL, ahead) >> sh) & 0xffffu);
    const int64_t top = lo + static_cast<int64_t>(c + 1) * step - 1;
    hi = static_cast<int>(min(static_cast<int64_t>(hi), top));
    lo = lo + c * step;
  }
  return lo;
}
__device__ __forceinline__ PathState path_state(const int2* list, int64_t d, int i, int V, int lane) {
  PathState s{i, static_cast<int>(d - i), false};
  if (s.v >= V) {
    s.v = V;
    return s;
  }
  const int j = i - 1 - lane;
  const unsigned mine = __ballot_sync(ALL, j >= 0 && list[j].x == s.v);
  s.cut = mine == ALL;
  if (!s.cut) s.i -= __ffs(~mine) - 1;
  return s;
}

template <typename TY>
__global__ void __launch_bounds__(32 * SUM_WARPS)
    embed_sum_kernel(const __grid_constant__ EmbedParams p, const __grid_constant__ EmbedPlan m, int parts,
                     const int2* list, int* headv, int* tailv, float* part) {
  pdl_entry();
  const int lane = threadIdx.x & 31;
  const int64_t g = static_cast<int64_t>(blockIdx.x) * SUM_WARPS + (threadIdx.x >> 5);
  const int64_t range = g / parts;
  if (range >= m.ranges) return;
  const int slab = static_cast<int>(g - range * parts);          // tangents' behind the primal ones
  const bool tangent = slab >= m.slabs;
  const int col = (tangent ? slab - m.slabs : slab) * SLAB + 4 * lane, cols = p.dim - col;
  const TY* dy = static_cast<const TY*>(tangent ? p.dyd : p.dy) + col;
  float* dE = (tangent ? p.dEd : p.dE) + col;
  const int V = p.vocab, N = p.seq.rows;
  const int64_t d0 = range * m.per, d1 = min(d0 + m.per, static_cast<int64_t>(N) + V);
  const int at = path_search(list, N, lane < 16 ? d0 : d1, lane);
  const PathState a = path_state(list, d0, __shfl_sync(ALL, at, 0), V, lane);
  const PathState b = path_state(list, d1, __shfl_sync(ALL, at, 16), V, lane);
  float* mine = part + ((2 * range) * parts + slab) * SLAB + 4 * lane;    // head, and behind it tail
  const int64_t step = static_cast<int64_t>(parts) * SLAB;
  if (slab == 0 && lane == 0) {
    headv[range] = a.cut && b.v > a.v ? a.v : -1;
    tailv[range] = b.cut ? b.v : -1;
  }
  float4 acc = zero4();
  int v = a.v;
  bool head = a.cut;
  auto write_to = [&](int to) {
    if (v >= to) return;
    if (head) *reinterpret_cast<float4*>(mine) = acc;
    else if (cols > 0) store4(dE + v * p.lddE, cols, times4(acc, p.scale));
    head = false;
    acc = zero4();
    ++v;
#pragma unroll 4
    for (; v < to; ++v)
      if (cols > 0) store4(dE + v * p.lddE, cols, acc);
  };
  for (int j = a.i; j < b.i; j += 32) {
    int2 kp = make_int2(V, 0);
    if (j + lane < b.i) kp = list[j + lane];
    for (int u0 = 0; u0 < 32 && j + u0 < b.i; u0 += AHEAD) {
      float4 x[AHEAD];
#pragma unroll
      for (int u = 0; u < AHEAD; ++u) {
        const int key = __shfl_sync(ALL, kp.x, u0 + u), row = __shfl_sync(ALL, kp.y, u0 + u);
        x[u] = key < V && cols > 0 ? load4(dy + row * p.lddy, cols) : zero4();
      }
#pragma unroll
      for (int u = 0; u < AHEAD; ++u) {
        const int key = __shfl_sync(ALL, kp.x, u0 + u);
        if (key < V) {         // those without a table row come last
          write_to(key);
          add4(acc, x[u]);
        }
      }
    }
  }
  write_to(b.v);
  if (b.cut) *reinterpret_cast<float4*>(mine + step) = acc;
}

// Rows whose tokens lie in several ranges: the sums at the ends of the ranges before the one that
// writes the row, and that one's own, in their order: eight groups of threads add neighbours.
constexpr int JOIN_GROUPS = 8;

__global__ void __launch_bounds__(32 * JOIN_GROUPS)
    embed_join_kernel(const __grid_constant__ EmbedParams p, const __grid_constant__ EmbedPlan m, int parts,
                      const int* headv, const int* tailv, const float* part) {
  __shared__ int2 found[32 * JOIN_GROUPS];
  __shared__ int count[JOIN_GROUPS];
  __shared__ float4 sums[JOIN_GROUPS][32];
  pdl_entry();
  const int t = threadIdx.x, lane = t & 31, w = t >> 5;
  const int slab = blockIdx.y;
  const bool tangent = slab >= m.slabs;
  const int col = (tangent ? slab - m.slabs : slab) * SLAB + 4 * lane, cols = p.dim - col;
  float* dE = (tangent ? p.dEd : p.dE) + col;
  const int64_t step = static_cast<int64_t>(parts) * SLAB;
  const float* sum = part + static_cast<int64_t>(slab) * SLAB + 4 * lane;   // of range r: + 2 r step, its tail + step
  for (int64_t r0 = blockIdx.x; r0 < m.ranges; r0 += static_cast<int64_t>(32 * JOIN_GROUPS) * gridDim.x) {
    const int64_t r = r0 + static_cast<int64_t>(t) * gridDim.x;
    const int v = r < m.ranges ? headv[r] : -1;
    const unsigned hits = __ballot_sync(ALL, v >= 0);
    __syncthreads();                      // the last batch has been read
    if (lane == 0) count[w] = __popc(hits);
    __syncthreads();
    int n = 0, at = 0;
    for (int k = 0; k < JOIN_GROUPS; ++k) {
      at += k < w ? count[k] : 0;
      n += count[k];
    }
    if (v >= 0) found[at + __popc(hits & ((1u << lane) - 1))] = make_int2(static_cast<int>(r), v);
    __syncthreads();
    for (int e = 0; e < n; ++e) {
      const int range = found[e].x, row = found[e].y;
      int tails = 0;
      for (;;) {
        const int q = range - 1 - tails - lane;
        const unsigned same = __ballot_sync(ALL, q >= 0 && tailv[q] == row);
        tails += same == ALL ? 32 : __ffs(~same) - 1;
        if (same != ALL) break;
      }
      const int a = static_cast<int>(static_cast<int64_t>(tails) * w / JOIN_GROUPS);
      const int b = static_cast<int>(static_cast<int64_t>(tails) * (w + 1) / JOIN_GROUPS);
      const float* from = sum + (2 * static_cast<int64_t>(range - tails) + 1) * step;
      float4 acc = zero4();
#pragma unroll 8
      for (int k = a; k < b; ++k) add4(acc, *reinterpret_cast<const float4*>(from + 2 * k * step));
      sums[w][lane] = acc;
      __syncthreads();
      if (w == 0) {
        for (int k = 1; k < JOIN_GROUPS; ++k) add4(acc, sums[k][lane]);
        add4(acc, *reinterpret_cast<const float4*>(sum + 2 * static_cast<int64_t>(range) * step));
        if (cols > 0) store4(dE + row * p.lddE, cols, times4(acc, p.scale));
      }
      __syncthreads();
    }
  }
}

int64_t up(int64_t x, int64_t to) { return (x + to - 1) / to * to; }

}  // namespace

EmbedPlan embed_plan(int64_t rows, int64_t vocab, int64_t dim, bool dual) {
  EmbedPlan m;
  int key = 1;
  while (key < 31 && (vocab >> key) > 0) ++key;          // keys 0 .. vocab
  m.passes = (key + 8) / 9;
  m.bits = (key + m.passes - 1) / m.passes;
  m.tile = static_cast<int>(up((rows + MAX_TILES - 1) / MAX_TILES, SORT_SUB));
  m.tiles = m.tile ? static_cast<int>((rows + m.tile - 1) / m.tile) : 0;
  m.slabs = static_cast<int>((dim + SLAB - 1) / SLAB);
  const int64_t parts = static_cast<int64_t>(m.slabs) * (dual ? 2 : 1), steps = rows + vocab;
  // two ranges for every warp that the GPU holds, of 32 to 512 steps
  int64_t per = (steps * parts + 2 * 152 * 32 - 1) / (2 * 152 * 32);
  per = per < 32 ? 32 : per > 512 ? 512 : per;
  m.per = static_cast<int>(per);
  m.ranges = static_cast<int>((steps + per - 1) / per);
  m.list = 0;
  m.hist = up(2 * rows * static_cast<int64_t>(sizeof(int2)), 16);
  m.flags = m.hist + static_cast<int64_t>(m.passes) * m.tiles * DIGITS * sizeof(int);
  m.part = m.flags + up(2 * static_cast<int64_t>(m.ranges) * sizeof(int), 16);
  m.bytes = m.part + 2 * static_cast<int64_t>(m.ranges) * parts * SLAB * sizeof(float);
  return m;
}

cudaError_t embed_fwd(const EmbedParams& p, bool e_bf16, bool y_bf16, cudaStream_t s) {
  const int units = (p.dim + 3) / 4;
  const int rows = units >= LOOK_THREADS * LOOK_ITEMS ? 1 : LOOK_THREADS * LOOK_ITEMS / units;
  const dim3 grid(static_cast<unsigned>((p.seq.rows + rows - 1) / rows), p.Ed ? 2 : 1);
  auto run = [&](auto kernel) { return launch_k(kernel, grid, dim3(LOOK_THREADS), 0, s, p, rows, units); };
  if (e_bf16)
    return y_bf16 ? run(embed_fwd_kernel<__nv_bfloat16, __nv_bfloat16>) : run(embed_fwd_kernel<__nv_bfloat16, float>);
  return y_bf16 ? run(embed_fwd_kernel<float, __nv_bfloat16>) : run(embed_fwd_kernel<float, float>);
}

cudaError_t embed_bwd(const EmbedParams& p, bool y_bf16, void* work, cudaStream_t s) {
  const bool dual = p.dEd != nullptr;
  const EmbedPlan m = embed_plan(p.seq.rows, p.vocab, p.dim, dual);
  char* base = static_cast<char*>(work);
  int2* lists[2] = {reinterpret_cast<int2*>(base + m.list), reinterpret_cast<int2*>(base + m.list) + p.seq.rows};
  int* hist = reinterpret_cast<int*>(base + m.hist);
  int* headv = reinterpret_cast<int*>(base + m.flags);
  int* tailv = headv + m.ranges;
  float* part = reinterpret_cast<float*>(base + m.part);
  const int parts = m.slabs * (dual ? 2 : 1);
  const unsigned tiles = static_cast<unsigned>(m.tiles);
  cudaError_t e = cudaSuccess;
  if (tiles) e = launch_k(token_hist_kernel, dim3(tiles), dim3(SORT_THREADS), 0, s, p, m, hist);
  for (int k = 0; tiles && k < m.passes && e == cudaSuccess; ++k) {
    const int2* from = lists[(k + 1) & 1];
    e = k == 0 ? launch_k(token_sort_kernel<true>, dim3(tiles), dim3(SORT_THREADS), 0, s, p, m, k, from, lists[0], hist)
               : launch_k(token_sort_kernel<false>, dim3(tiles), dim3(SORT_THREADS), 0, s, p, m, k, from,
                          lists[k & 1], hist);
  }
  if (e != cudaSuccess) return e;
  const int2* list = lists[(m.passes - 1) & 1];
  const int64_t blocks = (static_cast<int64_t>(m.ranges) * parts + SUM_WARPS - 1) / SUM_WARPS;
  if (blocks > INT_MAX) return cudaErrorInvalidValue;
  auto sum = [&](auto kernel) {
    return launch_k(kernel, dim3(static_cast<unsigned>(blocks)), dim3(32 * SUM_WARPS), 0, s, p, m, parts, list, headv,
                    tailv, part);
  };
  e = y_bf16 ? sum(embed_sum_kernel<__nv_bfloat16>) : sum(embed_sum_kernel<float>);
  if (e != cudaSuccess || p.seq.rows < 32) return e;       // no border has 32 tokens of a row before it
  const int wide = 4 * 152 / parts;
  const int x = wide < 1 ? 1 : wide < m.ranges ? wide : m.ranges;
  return launch_k(embed_join_kernel, dim3(static_cast<unsigned>(x), static_cast<unsigned>(parts)),
                  dim3(32 * JOIN_GROUPS), 0, s, p, m, parts, headv, tailv, part);
}

}  // namespace mf
