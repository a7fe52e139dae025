// Causal attention with a sliding window and a few first rows of a sequence that stay visible
// (mf_attn_window_*): kernels in attn_tc_impl.cuh.
#include "attn_tc_impl.cuh"

namespace mf {

cudaError_t attn_window_bwd(const AttnParams& a, bool dual, cudaStream_t s) {
  if (dual) return launch_bwd<true, 64, true>(a, s);
  return a.D <= 64 ? launch_bwd<false, 64, true>(a, s) : launch_bwd<false, 128, true>(a, s);
}

cudaError_t attn_window_fwd(const AttnParams& a, bool dual, cudaStream_t s) {
  if (dual) return launch_fwd<true, 64, 64, true>(a, s);
  return a.D > 64 ? launch_fwd<false, 128, 128, true>(a, s) : launch_fwd<false, 64, 64, true>(a, s);
}

}  // namespace mf
