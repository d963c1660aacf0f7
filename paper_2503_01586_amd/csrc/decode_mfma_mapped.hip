// The bf16 split attention (decode_mfma_kernel.hpp) for caches in pages and for trees of drafted tokens.
#include "decode_mfma_kernel.hpp"

namespace ekv {

hipError_t launch_attn_mapped(const AttnMfmaParams& prm, const DecodeArgs& a, hipStream_t stream) {
  AttnMfmaMappedParams p;
  static_cast<AttnMfmaParams&>(p) = prm;
  p.map = a.map;
  return dispatch_attn<true>(p, a, stream);
}

}  // namespace ekv
