// The FP8 block quantiser's arithmetic, shared by the quantisers and the grouped
// GEMM's quantising epilogue: for a block with m = max |x| >= 2^-100,
//   enc = fl(448 / m), dec = fl(1 / enc), code = E4M3_RNE(clamp(fl(x enc), +-448));
// a smaller block takes enc = dec = 1 (its codes are zeros).  A NaN keeps its place as
// the code 0x7F or 0xFF; an infinity gives dec = inf, so that the whole block stands
// for NaN.
#pragma once
#include "common.h"

namespace qdb {

using namespace qd;

constexpr int FB = 128;                // elements of a block along K

__device__ __forceinline__ void fb_scale(float m, float &enc, float &dec) {
  enc = m >= kZeroAmax ? 448.0f / m : 1.0f;
  dec = 1.0f / enc;
}
// Four codes, element 0 in the low byte.  |x| <= m, so x enc is at most 448 (1 + 2^-23) before
// its rounding, which the conversion takes to 448: the clamp of the definition needs no
// instruction.
__device__ __forceinline__ uint32_t fb_codes4(float a, float b, float c, float d, float enc) {
  int w = 0;
  w = __builtin_amdgcn_cvt_pk_fp8_f32(a * enc, b * enc, w, false);
  w = __builtin_amdgcn_cvt_pk_fp8_f32(c * enc, d * enc, w, true);
  return (uint32_t)w;
}

// max over the 16 lanes of a row (lanes 16 i .. 16 i + 15), in every lane of it
__device__ __forceinline__ float row16_max(float m) {
  m = fmaxf(m, __int_as_float(__builtin_amdgcn_mov_dpp(__float_as_int(m), 0xB1, 0xF, 0xF, false)));
  m = fmaxf(m, __int_as_float(__builtin_amdgcn_mov_dpp(__float_as_int(m), 0x4E, 0xF, 0xF, false)));
  m = fmaxf(m, __int_as_float(__builtin_amdgcn_mov_dpp(__float_as_int(m), 0x124, 0xF, 0xF, false)));
  m = fmaxf(m, __int_as_float(__builtin_amdgcn_mov_dpp(__float_as_int(m), 0x128, 0xF, 0xF, false)));
  return m;
}

// eight consecutive elements
template <typename T>
struct Eight;
template <>
struct Eight<uint16_t> {
  uint4 q;
  __device__ __forceinline__ void load(const uint16_t *p) { q = *reinterpret_cast<const uint4 *>(p); }
  __device__ __forceinline__ void zero() { q = make_uint4(0, 0, 0, 0); }
  __device__ __forceinline__ float at(int j) const {
    const uint32_t w = j < 2 ? q.x : j < 4 ? q.y : j < 6 ? q.z : q.w;
    return __uint_as_float(j & 1 ? w & 0xFFFF0000u : w << 16);
  }
};
template <>
struct Eight<float> {
  float4 q[2];
  __device__ __forceinline__ void load(const float *p) {
    q[0] = reinterpret_cast<const float4 *>(p)[0];
    q[1] = reinterpret_cast<const float4 *>(p)[1];
  }
  __device__ __forceinline__ void zero() { q[0] = q[1] = make_float4(0.f, 0.f, 0.f, 0.f); }
  __device__ __forceinline__ float at(int j) const {
    const float4 &f = q[j >> 2];
    return (j & 3) == 0 ? f.x : (j & 3) == 1 ? f.y : (j & 3) == 2 ? f.z : f.w;
  }
};
template <typename T>
__device__ __forceinline__ float eight_amax(const Eight<T> &v) {
  float m = 0.0f;
#pragma unroll
  for (int j = 0; j < 8; ++j) m = fmaxf(m, fabsf(v.at(j)));
  return m;
}
template <typename T>
__device__ __forceinline__ uint2 eight_codes(const Eight<T> &v, float enc) {
  return make_uint2(fb_codes4(v.at(0), v.at(1), v.at(2), v.at(3), enc),
                    fb_codes4(v.at(4), v.at(5), v.at(6), v.at(7), enc));
}

// One workgroup's part of the 1 x 128 quantiser: a row of each 16 lanes (from
// rb * blockDim.x / 16 on) x four blocks (from 4 cb on), so that the scales of a block are
// stored side by side.  Rows from `live` on are left alone.
template <typename T>
__device__ __forceinline__ void fb_quantize_act_body(int64_t rb, int cb, const T *__restrict__ x,
                                                     int64_t rows, int64_t live, int64_t cols,
                                                     int64_t ld,
                                                     uint8_t *__restrict__ codes,
                                                     float *__restrict__ scales) {
  constexpr int NB = 4;
  const int l = threadIdx.x & 15;
  const int64_t r = rb * (blockDim.x >> 4) + (threadIdx.x >> 4);
  if (r >= live) return;                 // whole rows of 16 lanes
  const int nkb = (int)((cols + FB - 1) / FB);
  const int b0 = cb * NB;
  Eight<T> v[NB];
#pragma unroll
  for (int b = 0; b < NB; ++b) {
    const int64_t c = (int64_t)(b0 + b) * FB + 8 * l;
    if (c < cols) v[b].load(x + r * ld + c);
    else v[b].zero();
  }
#pragma unroll
  for (int b = 0; b < NB; ++b) {
    if (b0 + b >= nkb) break;
    float enc, dec;
    fb_scale(row16_max(eight_amax(v[b])), enc, dec);
    const int64_t c = (int64_t)(b0 + b) * FB + 8 * l;
    if (c < cols) *reinterpret_cast<uint2 *>(codes + r * cols + c) = eight_codes(v[b], enc);
    if (l == 0) scales[(int64_t)(b0 + b) * rows + r] = dec;
  }
}

}  // namespace qdb
