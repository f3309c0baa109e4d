// The 8-bit format of include/aeris_fp8.h in registers: blocks of 128 columns, held by 16 neighbouring
// lanes of eight columns each, and their power-of-two scale.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "aeris_fp8.h"
#include "winattn_common.hpp"

namespace aeris {

constexpr int kBlockLanes = 16;                     // lanes of a block, eight columns each
constexpr uint32_t kNotFinite = 0x7f800000u;        // magnitudes from here on are infinite or NaN
constexpr unsigned char kScaleOne = 127;

__host__ __device__ inline int scale_pitch(int cols) { return (cols + 511) / 512 * 4; }

// Largest of x over the 16 lanes of a row of lanes.  Every lane of the wave takes part.
__device__ __forceinline__ uint32_t block_max(uint32_t x) {
  auto turned = [&](auto by) __attribute__((always_inline)) {
    constexpr int kRowRotate = 0x120 + decltype(by)::value;
    const uint32_t y = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, kRowRotate, 0xf, 0xf, false);
    x = x > y ? x : y;
  };
  turned(Const<8>{});
  turned(Const<4>{});
  turned(Const<2>{});
  turned(Const<1>{});
  return x;
}

// Largest magnitude of eight values as its bits, which order as the values do; `finite`: of the finite ones.
__device__ __forceinline__ uint32_t most8(const float (&v)[8], bool finite) {
  uint32_t m = 0;
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const uint32_t a = __float_as_uint(v[i]) & 0x7fffffffu;
    m = finite && a >= kNotFinite ? m : m > a ? m : a;
  }
  return m;
}

// Scale byte of a block whose largest finite magnitude has the bits `most`: 2^(b - 127) is the smallest power
// of two >= 2^-126 with most <= 448 * 2^(b - 127) = 7/4 * 2^(b - 119).  A mantissa above 7/4 carries.
__device__ __forceinline__ uint32_t scale_byte(uint32_t most) {
  const int b = (int)((most + 0x1fffffu) >> 23) - 8;
  return (uint32_t)(b > 1 ? b : 1);
}
__device__ __forceinline__ float scale_value(uint32_t byte) { return __uint_as_float(byte << 23); }

// Four values over a scale as e4m3, one rounding to nearest even; what is not finite becomes NaN.
typedef short i16x2 __attribute__((ext_vector_type(2)));
__device__ __forceinline__ uint32_t pack4_e4m3(float a, float b, float c, float d, float scale) {
  i16x2 q = {0, 0};
  q = __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(q, a, b, scale, false);
  q = __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(q, c, d, scale, true);
  return __builtin_bit_cast(uint32_t, q);
}
// The same of four bf16 values, two per register.
__device__ __forceinline__ uint32_t pack4_e4m3(uint32_t ab, uint32_t cd, float scale) {
  i16x2 q = {0, 0};
  q = __builtin_amdgcn_cvt_scalef32_pk_fp8_bf16(q, __builtin_bit_cast(bf16x2, ab), scale, false);
  q = __builtin_amdgcn_cvt_scalef32_pk_fp8_bf16(q, __builtin_bit_cast(bf16x2, cd), scale, true);
  return __builtin_bit_cast(uint32_t, q);
}

// Quantises a block per 16 lanes; lanes without columns pass zeros.  Every lane of the wave takes part.
// Returns the scale byte.  That only finite values count is worked out where a wave meets one that is not.
__device__ __forceinline__ uint32_t quantize_block(const float (&v)[8], u32x2& q) {
  uint32_t most = block_max(most8(v, false));
  if (__builtin_expect(__any(most >= kNotFinite), 0)) most = block_max(most8(v, true));
  const uint32_t byte = scale_byte(most);
  const float scale = scale_value(byte);
  q = u32x2{pack4_e4m3(v[0], v[1], v[2], v[3], scale), pack4_e4m3(v[4], v[5], v[6], v[7], scale)};
  return byte;
}

// Scale of block `block` of a row of `blocks`, by the 16 lanes that hold it; those behind the row's last
// block store what fills the row of scales up.
__device__ __forceinline__ void store_scale(unsigned char* row, int block, int blocks, int pitch, uint32_t byte,
                                            int lane) {
  const int at = block + (lane & (kBlockLanes - 1));
  if (at == block) row[at] = (unsigned char)byte;
  else if (block == blocks - 1 && at < pitch) row[at] = kScaleOne;
}

}  // namespace aeris
