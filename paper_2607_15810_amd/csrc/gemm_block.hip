// Grouped GEMM over FP8 operands with block scales:
//   v[r][n] = sum_kb sa[kb][src(r)] sw[e][n / 128][kb] sum_{k in block kb} a[src(r)][k] w[e][n][k]
// with its epilogues: bf16, SwiGLU in bf16, SwiGLU quantised to FP8 with 1 x 128 scales.
//
// A block's 128 products go through two v_mfma_scale_f32_32x32x64_f8f6f4 with unit
// scales into a partial sum, which one multiply-add per element folds into the f32
// total with the product of the two scales.  The weights are the instruction's first
// operand, so a lane holds one activation row: its row scale is one register, the
// weight scale is uniform, and four consecutive columns of a row leave a lane together.
#include "fp8_block_dev.h"
#include "lds_dma.h"
#include "tile_sched.h"

namespace {

using namespace qdb;
using namespace qdl;

typedef int v8i __attribute__((ext_vector_type(8)));
typedef float f32x16 __attribute__((ext_vector_type(16)));

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

constexpr int BK_EMAX = 1024;

__device__ __forceinline__ f32x16 mfma_f8(v8i a, v8i b, f32x16 c) {
  return __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(a, b, c, 0, 0, 0, 127, 0, 127);
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

// 32 rows of an expert x 256 weight rows (SwiGLU: 128 gate rows and the matching up
// rows), four waves of two 32 x 32 fragments, operands straight from memory.
template <int EPI>
__global__ __launch_bounds__(256) void gemm_block_kernel(BlkArgs p, int ntn) {
  __shared__ int sh_w[4], sh_t[4];
  __shared__ float sh_m[4][32];
  const int tid = threadIdx.x, lane = tid & 63, w = (int)uni((uint32_t)tid >> 6);
  const qdt::Tile tl = qdt::find_tile<32>(p.offsets, p.E, p.rows, ntn, sh_w, sh_t);
  if (tl.e < 0) return;
  const int N = p.N, K = p.K, KB = (K + FB - 1) / FB, NB = (N + FB - 1) / FB;
  const int c = lane & 31, h = lane >> 5;
  constexpr bool GLU = EPI != QD_EPI_NONE;
  const int I = GLU ? N >> 1 : N;
  int64_t src = tl.row0 + (c < tl.nrows ? c : 0);
  if (p.row_token) src = p.row_token[src];
  const uint8_t *pa = p.a + src * K;
  const uint8_t *pw[2];
  const float *ws[2];
  int col0[2];
#pragma unroll
  for (int j = 0; j < 2; ++j) {
    col0[j] = GLU ? tl.nt * 128 + 32 * w : tl.nt * 256 + 64 * w + 32 * j;
    const int wr = (GLU && j == 1 ? I : 0);
    const int n = wr + (col0[j] + c < I ? col0[j] + c : 0);
    pw[j] = p.w + ((int64_t)tl.e * N + n) * K;
    const int nb = col0[j] < I ? (wr + col0[j]) / FB : 0;
    ws[j] = p.w_scales + ((int64_t)tl.e * NB + nb) * KB;
  }
  auto piece = [&](const uint8_t *q, int k) __attribute__((always_inline)) -> uint4 {
    return k < K ? *reinterpret_cast<const uint4 *>(q + k) : make_uint4(0, 0, 0, 0);
  };
  struct Two { uint4 x, y; };
  f32x16 acc[2];
#pragma unroll
  for (int j = 0; j < 2; ++j)
#pragma unroll
    for (int q = 0; q < 16; ++q) acc[j][q] = 0.0f;
  for (int kb = 0; kb < KB; ++kb) {
    const float sa = p.a_scales[(int64_t)kb * p.a_rows + src];
    v8i a[2];
#pragma unroll
    for (int st = 0; st < 2; ++st) {
      const int k = kb * FB + 64 * st + 32 * h;
      a[st] = __builtin_bit_cast(v8i, Two{piece(pa, k), piece(pa, k + 16)});
    }
#pragma unroll
    for (int j = 0; j < 2; ++j) {
      f32x16 part;
#pragma unroll
      for (int q = 0; q < 16; ++q) part[q] = 0.0f;
#pragma unroll
      for (int st = 0; st < 2; ++st) {
        const int k = kb * FB + 64 * st + 32 * h;
        part = mfma_f8(__builtin_bit_cast(v8i, Two{piece(pw[j], k), piece(pw[j], k + 16)}), a[st], part);
      }
      const float s = sa * ws[j][kb];
#pragma unroll
      for (int q = 0; q < 16; ++q) acc[j][q] = __builtin_fmaf(part[q], s, acc[j][q]);
    }
  }
  // element q of a fragment: column 8 (q / 4) + 4 h + q % 4 of row c
  const int64_t row = tl.row0 + c;
  const bool in_row = c < tl.nrows;
  if constexpr (!GLU) {
#pragma unroll
    for (int j = 0; j < 2; ++j)
#pragma unroll
      for (int q = 0; q < 16; q += 4) {
        const int n = col0[j] + 2 * q + 4 * h;
        if (in_row && n < N)
          *reinterpret_cast<uint2 *>(static_cast<uint16_t *>(p.out) + row * N + n) = make_uint2(
              bf16_pair(acc[j][q], acc[j][q + 1]), bf16_pair(acc[j][q + 2], acc[j][q + 3]));
      }
  } else {
    float v[16];
#pragma unroll
    for (int q = 0; q < 16; ++q) v[q] = bk_swiglu(acc[0][q], acc[1][q]);
    if constexpr (EPI == QD_EPI_SWIGLU) {
#pragma unroll
      for (int q = 0; q < 16; q += 4) {
        const int n = col0[0] + 2 * q + 4 * h;
        if (in_row && n < I)
          *reinterpret_cast<uint2 *>(static_cast<uint16_t *>(p.out) + row * I + n) =
              make_uint2(bf16_pair(v[q], v[q + 1]), bf16_pair(v[q + 2], v[q + 3]));
      }
    } else {
      float m = 0.0f;
#pragma unroll
      for (int q = 0; q < 16; ++q)
        if (col0[0] < I) m = fmaxf(m, fabsf(v[q]));
      m = fmaxf(m, __shfl_xor(m, 32, 64));
      if (h == 0) sh_m[w][c] = m;
      __syncthreads();
      m = fmaxf(fmaxf(sh_m[0][c], sh_m[1][c]), fmaxf(sh_m[2][c], sh_m[3][c]));
      float enc, dec;
      fb_scale(m, enc, dec);
      if (in_row && w == 0 && h == 0) p.out_scales[(int64_t)tl.nt * p.rows + row] = dec;
#pragma unroll
      for (int q = 0; q < 16; q += 4) {
        const int n = col0[0] + 2 * q + 4 * h;
        if (in_row && n < I)
          *reinterpret_cast<uint32_t *>(static_cast<uint8_t *>(p.out) + row * I + n) =
              fb_codes4(v[q], v[q + 1], v[q + 2], v[q + 3], enc);
      }
    }
  }
}

}  // namespace

extern "C" qd_status moe_fp8_block_grouped_gemm(
    const uint8_t *a_codes, const float *a_scales, int64_t a_rows, const int32_t *row_token,
    const int32_t *expert_offsets, int32_t E, int64_t rows, const uint8_t *w_codes,
    const float *w_scales, int64_t N, int64_t K, int32_t epilogue, void *out, float *out_scales,
    void *stream) {
  if (epilogue != QD_EPI_NONE && epilogue != QD_EPI_SWIGLU && epilogue != QD_EPI_SWIGLU_FP8)
    return QD_ERR_DTYPE;
  if (E < 1 || rows < 0 || a_rows < 0 || N <= 0 || K <= 0 || K % 16 != 0) return QD_ERR_SHAPE;
  if (epilogue == QD_EPI_NONE ? N % 8 != 0 : N % 64 != 0) return QD_ERR_SHAPE;
  if (!expert_offsets && E != 1) return QD_ERR_SHAPE;
  if (!row_token && rows > a_rows) return QD_ERR_SHAPE;
  if (!w_codes || !w_scales) return QD_ERR_NULL;
  if (rows > 0 && (!a_codes || !a_scales || !out)) return QD_ERR_NULL;
  if (rows > 0 && epilogue == QD_EPI_SWIGLU_FP8 && !out_scales) return QD_ERR_NULL;
  if (!qdh::aligned16(a_codes) || !qdh::aligned16(a_scales) || !qdh::aligned16(w_codes) ||
      !qdh::aligned16(w_scales) || !qdh::aligned16(out) || !qdh::aligned16(out_scales) ||
      ((uintptr_t)row_token & 3u) || ((uintptr_t)expert_offsets & 3u))
    return QD_ERR_ALIGN;
  const int64_t lim = 1LL << 32;
  if (E > BK_EMAX || rows > 0x7fffffffLL || a_rows > 0x7fffffffLL || N > 0x3fffffffLL ||
      K > 0x3fffffffLL || (a_rows > rows ? a_rows : rows) + 1 > lim / K || N > (lim - 1) / K)
    return QD_ERR_UNSUPPORTED;
  if (qdh::fault_injected()) return QD_ERR_HIP;
  if (rows == 0) return QD_OK;
  BlkArgs p{a_codes, a_scales, a_rows, row_token, expert_offsets, E, rows, w_codes, w_scales,
            (int)N, (int)K, out, out_scales};
  const int ntn = (int)((N + 255) / 256);
  const int64_t g = qdt::tile_grid(rows, E, 32, ntn);
  if (g > 0x7fffffffLL) return QD_ERR_UNSUPPORTED;
  hipStream_t s = qdh::S(stream);
  const dim3 grid((unsigned)g), block(256);
  if (epilogue == QD_EPI_NONE)
    hipLaunchKernelGGL(gemm_block_kernel<QD_EPI_NONE>, grid, block, 0, s, p, ntn);
  else if (epilogue == QD_EPI_SWIGLU)
    hipLaunchKernelGGL(gemm_block_kernel<QD_EPI_SWIGLU>, grid, block, 0, s, p, ntn);
  else
    hipLaunchKernelGGL(gemm_block_kernel<QD_EPI_SWIGLU_FP8>, grid, block, 0, s, p, ntn);
  return qdh::check_launch();
}
