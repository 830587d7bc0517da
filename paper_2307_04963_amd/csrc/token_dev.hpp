// Device helpers of the token operators: sums and maxima over a wave's
// lanes, element loads and stores of either type.
#pragma once

#include "conv_dev.hpp"
#include "tokens.hpp"

namespace dycl {
namespace k {

typedef float f32x4 __attribute__((ext_vector_type(4)));

// 16 bytes at any element's alignment: the hardware takes them in one access
typedef uint32_t bits128 __attribute__((ext_vector_type(4), aligned(2)));

__device__ __forceinline__ uint4 load16(const void* p) { return __builtin_bit_cast(uint4, *static_cast<const bits128*>(p)); }
__device__ __forceinline__ void store16(void* p, const uint4& v) { *static_cast<bits128*>(p) = __builtin_bit_cast(bits128, v); }

// lane i of every 16 receives v of lane (i + R) % 16
template <int R>
__device__ __forceinline__ float rotate16(float v) {
  return __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, v), 0x120 + R, 0xf, 0xf, false));
}

__device__ __forceinline__ float lane_value(float v, int lane) {
  return __builtin_bit_cast(float, __builtin_amdgcn_readlane(__builtin_bit_cast(int, v), lane));
}

// the sum over each 16 lanes, in all of them
__device__ __forceinline__ float sum16(float v) {
  v += rotate16<8>(v);
  v += rotate16<4>(v);
  v += rotate16<2>(v);
  v += rotate16<1>(v);
  return v;
}

__device__ __forceinline__ float wave_sum(float v) {
  v = sum16(v);
  return (lane_value(v, 0) + lane_value(v, 16)) + (lane_value(v, 32) + lane_value(v, 48));
}

// inclusive prefix sum over the lanes
__device__ __forceinline__ int scan_lanes(int v) {
  v += __builtin_amdgcn_update_dpp(0, v, 0x111, 0xf, 0xf, false);     // row_shr 1, 2, 4, 8
  v += __builtin_amdgcn_update_dpp(0, v, 0x112, 0xf, 0xf, false);
  v += __builtin_amdgcn_update_dpp(0, v, 0x114, 0xf, 0xf, false);
  v += __builtin_amdgcn_update_dpp(0, v, 0x118, 0xf, 0xf, false);
  v += __builtin_amdgcn_update_dpp(0, v, 0x142, 0xa, 0xf, false);     // row_bcast 15 into rows 1 and 3
  v += __builtin_amdgcn_update_dpp(0, v, 0x143, 0xc, 0xf, false);     // row_bcast 31 into rows 2 and 3
  return v;
}

__device__ __forceinline__ float sigmoid_fast(float v) { return __builtin_amdgcn_rcpf(1.0f + __expf(-v)); }

__device__ __forceinline__ float token_act(float v, int act) {
  if (act == TACT_RELU) return v < 0.f ? 0.f : v;   // (NaN stays NaN)
  if (act == TACT_GELU) return gelu_f32(v);
  if (act == TACT_SILU) return v * sigmoid_fast(v);
  return v;
}

}  // namespace k
}  // namespace dycl
