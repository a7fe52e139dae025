// Causal attention over whole sequences (mf_attn_*): kernels in attn_tc_impl.cuh.
#include "attn_tc_impl.cuh"

namespace mf {

cudaError_t attn_tc_bwd(const AttnParams& a, bool dual, cudaStream_t s) {
  if (dual) return launch_bwd<true, 64, false>(a, s);
  return a.D <= 64 ? launch_bwd<false, 64, false>(a, s) : launch_bwd<false, 128, false>(a, s);
}

cudaError_t attn_tc_fwd(const AttnParams& a, bool dual, cudaStream_t s) {
  if (dual) return launch_fwd<true, 64, 64, false>(a, s);
  if (a.D > 64) return launch_fwd<false, 128, 128, false>(a, s);
  // From two rounds of three CTAs an SM on, tiles of 64 keys, whatever the sequences' lengths and the
  // heads' width: 16 heads of 64, 8192 rows in sequences of 16, 128, 1024 and 4096 take 20, 19, 40 and
  // 90 us against 24, 23, 43 and 99 with tiles of 128 and two CTAs; heads of 32 the same; 32 heads in
  // 16384 rows 70, 64, 128 and 332 against 89, 82, 148 and 352.  With fewer CTAs a walk's own
  // length counts, and it has twice as many steps: 4096 rows (512 CTAs) in sequences of 128, 1024 and
  // 4096 take 13, 24 and 60 us against 13, 26 and 56.
  const int64_t ctas = static_cast<int64_t>((a.seq.rows + TR - 1) / TR) * a.Hq;
  return ctas >= 2 * 3 * 152 ? launch_fwd<false, 64, 64, false>(a, s) : launch_fwd<false, 64, 128, false>(a, s);
}

}  // namespace mf
