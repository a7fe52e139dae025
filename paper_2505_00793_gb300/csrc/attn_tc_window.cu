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
  if (a.D > 64) return launch_fwd<false, 128, 128, true>(a, s);
  // Where all CTAs have a place at two an SM and the window is long, a walk's own length counts, as without a
  // window: tiles of 128 keys.  2048 rows, 16 heads of 64, windows of 256, 512, 1024 and 2047 take 16, 20, 23
  // and 29 us against 18, 23, 27 and 37 with four CTAs of 64 keys; 4096 rows, 8 heads, windows of 1024 and
  // 4095 26 and 45 against 29 and 61; 32768 rows, one head, window 8192 94 against 127.  Other ways round from
  // there on: 3000 rows, 16 heads, windows of 512, 1024 and 2048 29, 33 and 41 against 25, 31 and 43; 4096
  // rows, 16 heads 31, 41 and 51 against 27, 35 and 47.
  const int64_t ctas = static_cast<int64_t>((a.seq.rows + TR - 1) / TR) * a.Hq;
  return ctas <= 2 * 152 && a.window >= 512 ? launch_fwd<false, 64, 128, true>(a, s)
                                            : launch_fwd<false, 64, 64, true>(a, s);
}

}  // namespace mf
