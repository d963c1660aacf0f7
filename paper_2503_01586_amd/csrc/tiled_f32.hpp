// What the kernels in fp32 arithmetic share (tiled_f32.hip, tiled_seen.hip).
#pragma once
#include "common.hpp"
#include "launch.hpp"

namespace ekv {

typedef __attribute__((ext_vector_type(4))) float tf_f32x4;

__device__ __forceinline__ tf_f32x4 ld4(const float* p) { return *reinterpret_cast<const tf_f32x4*>(p); }
__device__ __forceinline__ tf_f32x4 ld4(const bf16_t* p) {
  const uint2 v = *reinterpret_cast<const uint2*>(p);
  tf_f32x4 r;
  r[0] = __uint_as_float(v.x << 16); r[1] = __uint_as_float(v.x & 0xffff0000u);
  r[2] = __uint_as_float(v.y << 16); r[3] = __uint_as_float(v.y & 0xffff0000u);
  return r;
}

// split attention: tiles of kTtTok cached tokens, kTtWaves waves a work-group, up to 8 kTtKeRegs elite values a head requested ahead
constexpr int kTtTok = 16, kTtWaves = 8, kTtKeRegs = 4, kTtComputeUnits = 256;
// up-projection: output columns of a work-group
constexpr int kTuCols = 32;

// Rows in pages or behind a tree's mask, and from kTsManyRows rows on the products around the attention on the matrix cores
// (tiled_seen.hip): the vector units' kernels read the weights once per four rows.  Trees of n nodes behind 200 tokens, us, vector /
// matrix: 7B 25 % 4: 39.4 / 41.9, 8: 44.7 / 47.3, 12: 58.0 / 52.2, 24: 81.1 / 63.9, 64: 164.7 / 111.9; 7B 12.5 % 8: 32.2 / 33.1,
// 12: 38.8 / 35.4, 64: 104.1 / 68.9.
constexpr int kTsManyRows = 9;
hipError_t launch_attn_seen_tiled(const DecodeArgs& a, const DecodePlan& p, const float* qe, const float* qt, float* pm, float* pl,
                                  float* pu, hipStream_t stream);
hipError_t launch_qprep_many_tiled(const DecodeArgs& a, const DecodePlan& p, float* qe, float* qt, hipStream_t stream);
hipError_t launch_upproj_many_tiled(const DecodeArgs& a, const DecodePlan& p, const float* ubar, hipStream_t stream);

}  // namespace ekv
