// Operands and arithmetic that the two kernels of the FP8 block GEMM share.
#pragma once
#include <atomic>

#include "fp8_block_dev.h"

namespace qdb {

typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));

struct BlkArgs {
  const uint8_t *a;            // [a_rows][K]
  const float *a_scales;       // [KB][a_rows]
  int64_t a_rows;
  const int32_t *row_token;
  const int32_t *offsets;
  int E;
  int64_t rows;
  const uint8_t *w;            // [E][N][K]
  const float *w_scales;       // [E][NB][KB]
  int N, K;
  void *out;                   // bf16 [rows][N or N / 2], or FP8 codes [rows][N / 2]
  float *out_scales;           // [N / 256 rounded up][rows]
};

static __device__ const uint4 bk_zero = {0, 0, 0, 0};

// eight codes (two words) times the power of two of sc, exact in bf16
__device__ __forceinline__ bf16x8 dec8b(uint32_t lo, uint32_t hi, float sc) {
  const bf16x2 a = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8((int)lo, sc, false);
  const bf16x2 b = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8((int)lo, sc, true);
  const bf16x2 c = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8((int)hi, sc, false);
  const bf16x2 d = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8((int)hi, sc, true);
  return bf16x8{a[0], a[1], b[0], b[1], c[0], c[1], d[0], d[1]};
}
// the mantissa of a scale with its sign, of size in [1, 2); NaN of a scale that is not finite
__device__ __forceinline__ float bk_mant(float v) {
  const uint32_t b = __float_as_uint(v);
  const float m = __uint_as_float((b & 0x807FFFFFu) | 0x3F800000u);
  return (b & 0x7F800000u) == 0x7F800000u ? __uint_as_float(0x7FC00000u) : m;
}
__device__ __forceinline__ float bk_swiglu(float g, float u) {
  const float ex = __builtin_amdgcn_exp2f(-g * 1.4426950408889634f);
  return g * __builtin_amdgcn_rcpf(1.0f + ex) * u;
}
__device__ __forceinline__ uint32_t bf16_pair(float a, float b) {
  typedef __bf16 b2 __attribute__((ext_vector_type(2)));
  typedef float f2 __attribute__((ext_vector_type(2)));
  return __builtin_bit_cast(uint32_t, __builtin_convertvector(f2{a, b}, b2));
}
// The upper half of a against the lower half of b: with a and b the words of columns
// 4 h .. and 16 + 4 h .. (h the lane's half) the two results are, for the lower lanes,
// the words of columns 0 and 4, for the upper ones of 16 and 20.
struct Pair32 { uint32_t x, y; };
__device__ __forceinline__ Pair32 swap32(uint32_t a, uint32_t b) {
  const auto r = __builtin_amdgcn_permlane32_swap(a, b, false, false);
  return {r[0], r[1]};
}
// The same between sixteens: lanes 16 .. 31 (48 .. 63) of a against lanes 0 .. 15 (32 .. 47) of b.
__device__ __forceinline__ Pair32 swap16(uint32_t a, uint32_t b) {
  const auto r = __builtin_amdgcn_permlane16_swap(a, b, false, false);
  return {r[0], r[1]};
}

// Weight row of row tb of a run of 32-row fragments that starts at output column c0 (0 past
// the last: never stored); SwiGLU: a fragment is 16 gate rows and the 16 up rows of the
// same columns.
template <bool GLU>
__device__ __forceinline__ int bk_wrow(int tb, int c0, int N) {
  if (GLU) {
    const int I = N >> 1, c = c0 + 16 * (tb >> 5) + (tb & 15);
    return c < I ? c + (tb & 16 ? I : 0) : 0;
  }
  return c0 + tb < N ? c0 + tb : 0;
}

// More than 64 KB of dynamic LDS for a kernel, once on each device (done: a bit a device).
inline void blk_allow_lds(const void *kern, int bytes, std::atomic<uint64_t> &done) {
  int dev = -1;
  if (hipGetDevice(&dev) != hipSuccess) return;
  const uint64_t bit = dev >= 0 && dev < 64 ? 1ull << dev : 0;
  if (bit && (done.load(std::memory_order_relaxed) & bit)) return;
  if (hipFuncSetAttribute(kern, hipFuncAttributeMaxDynamicSharedMemorySize, bytes) == hipSuccess)
    done.fetch_or(bit, std::memory_order_relaxed);
}

// gemm_block_few.hip: the rows of a tile of its kernel for a call of these sizes (0: the
// large kernel takes it), and the launch (h: f32 [rows][N / 2] of workspace with
// QD_EPI_SWIGLU_FP8; codes false: h is left there, not quantised), and the product without an
// epilogue of rows that are quantised from such an h.
int blk_few_rows(int64_t rows, int E, int64_t N, int64_t K, int epilogue);
void launch_blk_few(const BlkArgs &p, int epilogue, float *h, bool codes, hipStream_t s);
void launch_blk_few_h(const BlkArgs &p, const float *h, hipStream_t s);

}  // namespace qdb
