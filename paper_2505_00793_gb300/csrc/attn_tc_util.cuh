// Device helpers of the tcgen05 attention kernels (flash_tc.cu, attn_tc.cu): TMEM access by
// rows, arithmetic on pairs of float32, bounded waits.
#pragma once

#include "pair_math.cuh"
#include "tc_gemm_impl.cuh"

namespace mf {
namespace {

// A row's reference maximum moves only when a tile exceeds it by more than this.
constexpr float TAU = 8.f;
constexpr long long FTC_WAIT_NS = 2000000000LL;   // bounded waits: 2 s

__device__ __forceinline__ void tmem_st16(uint32_t taddr, const float (&v)[16]) {
  asm volatile(
      "tcgen05.st.sync.aligned.32x32b.x16.b32 [%0], "
      "{%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16};" ::"r"(taddr),
      "r"(__float_as_uint(v[0])), "r"(__float_as_uint(v[1])), "r"(__float_as_uint(v[2])),
      "r"(__float_as_uint(v[3])), "r"(__float_as_uint(v[4])), "r"(__float_as_uint(v[5])),
      "r"(__float_as_uint(v[6])), "r"(__float_as_uint(v[7])), "r"(__float_as_uint(v[8])),
      "r"(__float_as_uint(v[9])), "r"(__float_as_uint(v[10])), "r"(__float_as_uint(v[11])),
      "r"(__float_as_uint(v[12])), "r"(__float_as_uint(v[13])), "r"(__float_as_uint(v[14])),
      "r"(__float_as_uint(v[15]))
      : "memory");
  asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory");
}

// 32 consecutive TMEM columns of this thread's lane, without waiting (tmem_wait_ld after a
// batch of loads).
__device__ __forceinline__ void tmem_ld32_nowait(uint32_t taddr, float* v) {
  uint32_t r[32];
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x32.b32 "
      "{%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,"
      "%16,%17,%18,%19,%20,%21,%22,%23,%24,%25,%26,%27,%28,%29,%30,%31}, [%32];"
      : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]),
        "=r"(r[7]), "=r"(r[8]), "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]),
        "=r"(r[13]), "=r"(r[14]), "=r"(r[15]), "=r"(r[16]), "=r"(r[17]), "=r"(r[18]),
        "=r"(r[19]), "=r"(r[20]), "=r"(r[21]), "=r"(r[22]), "=r"(r[23]), "=r"(r[24]),
        "=r"(r[25]), "=r"(r[26]), "=r"(r[27]), "=r"(r[28]), "=r"(r[29]), "=r"(r[30]),
        "=r"(r[31])
      : "r"(taddr));
#pragma unroll
  for (int i = 0; i < 32; ++i) v[i] = __uint_as_float(r[i]);
}
// e^x of a pair as 2^(x log2 e) on the exponential unit (subnormal results become zero).
__device__ __forceinline__ float2 exp_pair(uint64_t x) {
  float2 t = halves(mul2(x, pair(1.44269504f, 1.44269504f)));
  asm("ex2.approx.ftz.f32 %0, %0;" : "+f"(t.x));
  asm("ex2.approx.ftz.f32 %0, %0;" : "+f"(t.y));
  return t;
}
__device__ __forceinline__ uint32_t pack2(uint64_t a) {
  const float2 v = halves(a);
  return pack_bf16x2(v.x, v.y);
}

__device__ __forceinline__ void mbar_arrive_local(uint64_t* bar) {
  asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" ::"r"(smem_u32(bar)) : "memory");
}

__device__ __forceinline__ void fence_async_smem() {
  asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
}

// Bounded wait that gives up at once when another role of the CTA has given up.
__device__ __forceinline__ bool fwait(uint64_t* bar, uint32_t parity, int* status,
                                      volatile int* abort) {
  if (*abort) return false;
  if (mbar_try_wait(bar, parity)) return true;
  const long long t0 = global_ns();
  while (true) {
    if (mbar_try_wait(bar, parity)) return true;
    if (*abort) return false;
    if (global_ns() - t0 > FTC_WAIT_NS) {
      if (status) atomicMax(status, DEV_TIMEOUT);
      *abort = 1;
      return false;
    }
  }
}

// Byte offset of (row r, 16-byte chunk ch) in a K-major [128][64] bf16 atom, 128-byte swizzle.
__device__ __forceinline__ uint32_t swz(int r, int ch) {
  return static_cast<uint32_t>(r * 128 + ((ch ^ (r & 7)) << 4));
}


// Warp-uniform bounded wait: every lane polls, and the warp proceeds only if all lanes saw
// the phase complete (the TMEM loads after it are warp-collective).
__device__ __forceinline__ bool wwait(uint64_t* bar, uint32_t parity, int* status,
                                      volatile int* abort) {
  const bool ok = fwait(bar, parity, status, abort);
  return __all_sync(0xffffffffu, ok);
}

}  // namespace
}  // namespace mf
