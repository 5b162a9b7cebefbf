// What the quantisers and the 8-bit products share.
#pragma once
#include "common.h"

namespace symi {

typedef int intx8 __attribute__((ext_vector_type(8)));
typedef int intx4_ __attribute__((ext_vector_type(4)));
typedef float floatx4_ __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x8_ __attribute__((ext_vector_type(8)));

constexpr int QB = 128;               // values that share a power

// |x| as an integer, which orders as the value does; 0 for what is not finite
__device__ __forceinline__ int size_of(float x) {
  const int u = __float_as_int(x) & 0x7fffffff;
  return u < 0x7f800000 ? u : 0;
}
// s of a block whose largest |x| has these bits: 448 = 1.75 * 2^8, so the exponent counts one more from 1.75 on
__device__ __forceinline__ int scale_of(int most) { return max(((most + 0x1fffff) >> 23) - 8, 0); }
__device__ __forceinline__ float inverse_of(int s) { return __int_as_float((254 - s) << 23); }      // 2^(127 - s), s <= 247
__device__ __forceinline__ float power_of(int s) { return __int_as_float(s > 0 ? s << 23 : 1 << 22); }   // 2^(s - 127)

// x 2^(127 - s) to e4m3, to nearest even; not finite: NaN
__device__ __forceinline__ uint32_t codes4(float a, float b, float c, float d, float inv) {
  const float x[4] = {a, b, c, d};
  float y[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) y[i] = size_of(x[i]) || (__float_as_int(x[i]) & 0x7fffffff) == 0 ? x[i] * inv : NAN;
  int w = __builtin_amdgcn_cvt_pk_fp8_f32(y[0], y[1], 0, false);
  w = __builtin_amdgcn_cvt_pk_fp8_f32(y[2], y[3], w, true);
  return (uint32_t)w;
}

struct Product8 {
  const uint8_t *Aq, *As, *Wq, *Ws;
  const int32_t* slot_offsets;
  const int32_t* map;   // [0]: tiles, then {first row, slot + 2^16 (rows - 1)} of each
  void* Y;              // product: [rows, R]
  uint16_t *UV, *H;     // experts' first product, or nullptr
  uint8_t *Hq, *Hs;
  int R, p8, sp;        // R: rows of a slot's weight (f in the experts' first product: gate and up rows each)
  int hp8, hsp;         // pitches of Hq, Hs
  int slots;
};

__device__ __forceinline__ float sigmoid8(float u) { return __builtin_amdgcn_rcpf(1.f + __builtin_amdgcn_exp2f(-1.4426950408889634f * u)); }

// gemm8.hip: many rows; the map's tiles have 256 or 128 (fp32 contexts: 128)
void launch_gemm8(const symi_ctx* ctx, const Product8& p, int rows, bool expert, hipStream_t st);

}  // namespace symi
