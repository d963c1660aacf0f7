// The bf16 split attention (decode_mfma_kernel.hpp) for caches in pages and for trees of drafted tokens.
//
// Maxima, sums and accumulators are fp32.  Rounded to bf16, as in the kernels of rows back to back: the absorbed query (an operand of the
// matrix cores that every tile reads; in fp32 the scores would take four times the products), the probabilities (the same), and a split's
// accumulators, normalised by nothing yet, on their way to the merge (half of its bytes).  Together 3e-3 of a result's norm; a plain form
// with scores and probabilities in fp32 has 1.7e-3.
//
// us, pages of 64 rows in any order / the same rows back to back by the kernels without a map: 13B 25 % 16 x 8192 182 / 176, 7B 25 %
// 1 x 32768 48.5 / 47.0, 4 x 20 queries of 4096 177 / 166, 4 x 5 68.8 / 65.9; the page's size and order make 1 % at most.
#include "decode_mfma_kernel.hpp"

namespace ekv {

hipError_t launch_attn_mapped(const AttnMfmaParams& prm, const DecodeArgs& a, hipStream_t stream) {
  AttnMfmaMappedParams p;
  static_cast<AttnMfmaParams&>(p) = prm;
  p.map = a.map;
  return dispatch_attn<true>(p, a, stream);
}

}  // namespace ekv
