// The bf16 split attention's dispatch, and its kernels (decode_mfma_kernel.hpp) for caches whose rows lie back to back.
#include "decode_mfma_kernel.hpp"

namespace ekv {

// does the tile set of (waves, slice width) hold its LDS layout with elite rows of 2r values?
template <int NW, int DC_W>
static bool layout_fits(int two_r) {
  return two_r == 8 ? AttnMfmaLayout<NW, DC_W, 8>::kFits
       : two_r == 16 ? AttnMfmaLayout<NW, DC_W, 16>::kFits
       : two_r == 32 ? AttnMfmaLayout<NW, DC_W, 32>::kFits
       : two_r == 64 ? AttnMfmaLayout<NW, DC_W, 64>::kFits : false;
}

static void shape_of(int d_c, int* nw, int* dcw) {
  *nw = 0; *dcw = 0;
#define X(DC, NWV, DCW) if (d_c == DC) { *nw = NWV; *dcw = DCW; }
  EKV_ATTN_SHAPES(X)
#undef X
}
static int slice_width(int d_c) { int nw, w; shape_of(d_c, &nw, &w); return w; }
int decode_mfma_slice_width(int d_c) { return slice_width(d_c); }

// work-groups of the attention kernel that run side by side on a compute unit: as many as its launch bounds ask for, and
// two where a work-group has two waves for its four SIMDs
int decode_mfma_groups_per_cu(const elitekv_dims& d) {
  int g = 1;
  const int two_r = 2 * d.r;
#define X(DC, NWV, DCW)                                                                         \
  if (d.d_c == DC)                                                                              \
    g = two_r == 8 ? AttnMfmaLayout<NWV, DCW, 8>::kGroupsPerCu                                  \
      : two_r == 16 ? AttnMfmaLayout<NWV, DCW, 16>::kGroupsPerCu                                \
      : two_r == 32 ? AttnMfmaLayout<NWV, DCW, 32>::kGroupsPerCu                                \
      : two_r == 64 ? AttnMfmaLayout<NWV, DCW, 64>::kGroupsPerCu : 1;
  EKV_ATTN_SHAPES(X)
#undef X
  int nw, w;
  shape_of(d.d_c, &nw, &w);
  return nw == 2 ? 2 : g;
}

bool decode_mfma_supported(const elitekv_dims& d, int d_ck) {
  if (d.dtype != ELITEKV_BF16) return false;
  if ((d.head_dim != 128 && d.head_dim != 64) || (d.head_dim - 2 * d.r) % 8) return false;
  const int two_r = 2 * d.r;
  if (two_r != 8 && two_r != 16 && two_r != 32 && two_r != 64) return false;   // r = 4, 8, 16, 32 elite chunks per head
  const int w = slice_width(d.d_c);
  if (w == 0) return false;
  bool fits = false;                                      // 2r = 32 and 64 with the widest rows do not fit the LDS
#define X(DC, NWV, DCW) if (d.d_c == DC) fits = layout_fits<NWV, DCW>(two_r);
  EKV_ATTN_SHAPES(X)
#undef X
  if (!fits) return false;
  if (d_ck > 0 && w > 256) return false;    // the one-wave-per-SIMD instantiations are compiled for the joint latent only
  // separated latents with 64 elite values per head, or 32 beside 224-column slices: the compiled code parks query
  // registers in AGPRs right behind their loads (before they have landed), so these shapes take the generic kernels
  if (d_ck > 0 && (two_r == 64 || (two_r == 32 && w == 224))) return false;
  // separated latents: whole wave slices on either side of the boundary
  // (and the value part a whole number of the merge kernels' 64-column chunks)
  return d_ck == 0 || (d_ck > 0 && d_ck < d.d_c && d_ck % w == 0 && (d.d_c - d_ck) % 64 == 0);
}

hipError_t launch_decode_mfma(const DecodeArgs& a, const DecodePlan& p, hipStream_t stream) {
  const elitekv_dims& d = a.dims;
  float* qe = (float*)(a.ws + p.off_qe);
  bf16_t* qt = (bf16_t*)(a.ws + p.off_qt);
  AttnMfmaParams prm;
  prm.ke_plane = (const bf16_t*)a.ke_plane; prm.c_plane = (const bf16_t*)a.c_plane;
  prm.qe = qe; prm.qt = qt; prm.seq_len = a.seq_len;
  prm.part_m = (float*)(a.ws + p.off_m); prm.part_l = (float*)(a.ws + p.off_l);
  prm.part_u = (bf16_t*)(a.ws + p.off_u);
  prm.n_h = d.n_heads; prm.d_c = d.d_c; prm.n_splits = p.n_splits; prm.chunk = p.chunk;
  prm.head_groups = p.head_groups; prm.max_seq_len = a.max_seq_len;
  prm.batch_stride_rows = a.batch_stride_rows; prm.plane_rows = a.plane_rows;
  prm.batch = (int)a.B;
  const bool rows_to_xcds = a.B >= 8 && a.B % 8 == 0 && a.q_per_seq == 1;
  prm.pair_map = p.head_groups == 2 ? (rows_to_xcds ? 3 : 1) : rows_to_xcds && p.head_groups == 1 ? 2 : 0;
  prm.reader_run = prm.reader_turns = 0;
  // (two readers gain nothing: 1 x 2 queries of 32768 tokens 74.3 against 78.0 us, 16 x 2 of 4096 at 7B 12.5 % 75.2 / 77.8)
  if (a.q_per_seq > 1 && a.q_per_seq * p.head_groups > 2 && (int64_t)p.n_splits * a.B * p.head_groups < (1 << 30)) {
    prm.pair_map = 4;
    const int all = (int)(p.n_splits * a.B * p.head_groups);
    prm.reader_run = reader_run(a.q_per_seq * p.head_groups, all);
    prm.reader_turns = reader_turns(all, prm.reader_run);
  }
  prm.d_q = p.d_q; prm.d_u = p.d_u; prm.q_per_seq = a.q_per_seq; prm.q_slice = slice_width(d.d_c);
  prm.n_part = p.n_part; prm.fresh = p.fresh;
  // fr_slot is read (through the scalar cache) by every work-group of every launch; outside a fused step it points
  // at the first bytes of the workspace (the elite queries: at least 32 bytes per batch row) and the value is ignored
  prm.fr_partial = nullptr; prm.fr_sincos = nullptr; prm.fr_slot = (const int64_t*)(a.ws + p.off_qe); prm.fr_ks = 0; prm.fr_stride = 0;
  prm.fr_ke_out = nullptr; prm.fr_c_out = nullptr;
  prm.chunk_counters = (int*)(a.ws + p.off_cnt);
  if (p.fresh) {
    prm.fr_partial = (const float*)(a.ws + p.off_apart); prm.fr_sincos = (const float2*)(a.ws + p.off_sincos);
    prm.fr_slot = a.fr_slot; prm.fr_ks = p.fr_ks; prm.fr_stride = p.fr_stride;
    prm.fr_ke_out = (bf16_t*)a.fr_ke_out; prm.fr_c_out = (bf16_t*)a.fr_c_out;
  }

  hipError_t e = hipSuccess;
  if (a.stages & 1) e = launch_qprep_rows(a, p, qe, qt, stream);
  if (e != hipSuccess) return e;
  if (!(a.stages & 2)) return (a.stages & 4) ? launch_merge_up(a, p, stream) : hipSuccess;

  e = !a.mapped ? dispatch_attn<false>(prm, a, stream)
    : p.pairs   ? launch_attn_pairs(prm, a, stream)
                : launch_attn_mapped(prm, a, stream);
  if (e != hipSuccess) return e;
  return (a.stages & 4) ? launch_merge_up(a, p, stream) : hipSuccess;
}

}  // namespace ekv
