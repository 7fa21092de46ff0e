// FP8 (E4M3) with fine-grained scales: one float32 scale per 128 elements of a row
// (activations) or per 128 x 128 block (weights).  The arithmetic is in
// fp8_block_dev.h.
//
// Both quantisers are bound by HBM: an activation element is read once (2 B, kept in
// registers between the block's maximum and its codes) and written as 1 + 4/128 B; a
// weight element likewise, with one more byte for the transposed copy, which goes
// through LDS.  5001 x 4096 activations 14.8 us with the launch (62 MB, 4.2 TB/s; a copy of
// that size 4.9), 64 experts of 1536 x 2048 weights with the transposed copy 154 us (805 MB,
// 5.2 TB/s).
#include "gemm_block.h"

namespace {

using namespace qdb;

template <typename T>
__global__ __launch_bounds__(256) void fp8_block_act_kernel(const T *__restrict__ x, int64_t rows,
                                                            int64_t cols, int64_t ld,
                                                            uint8_t *__restrict__ codes,
                                                            float *__restrict__ scales) {
  fb_quantize_act_body<T>(blockIdx.x, blockIdx.y, x, rows, rows, cols, ld, codes, scales);
}

// One workgroup per 128 x 128 block: thread (row group tid / 16, lane tid % 16) keeps
// eight elements of eight rows.  The transposed copy: codes as rows of 33 dwords in
// LDS (two lanes a bank at most), 16 rows x 4 columns a thread back, turned by byte
// permutes, so that eight lanes store a line of the transposed matrix.
template <typename T, bool TR>
__global__ __launch_bounds__(256) void fp8_block_weight_kernel(
    const T *__restrict__ w, int64_t N, int64_t K, int nnb, int nkb, uint8_t *__restrict__ codes,
    float *__restrict__ scales, uint8_t *__restrict__ codes_t, float *__restrict__ scales_t) {
  __shared__ uint32_t tile[TR ? 128 * 33 : 1];
  __shared__ float red[4];
  const int tid = threadIdx.x, l = tid & 15, rg = tid >> 4;
  const int64_t b = blockIdx.x;
  const int kb = (int)(b % nkb);
  const int64_t en = b / nkb;            // expert * nnb + row block
  const int64_t e = en / nnb;
  const int nb = (int)(en - e * nnb);
  const int64_t n0 = (int64_t)nb * FB, k0 = (int64_t)kb * FB;
  const T *we = w + e * N * K;
  const int64_t c = k0 + 8 * l;
  Eight<T> v[8];
  float m = 0.0f;
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const int64_t r = n0 + 16 * i + rg;
    if (r < N && c < K) v[i].load(we + r * K + c);
    else v[i].zero();
  }
#pragma unroll
  for (int i = 0; i < 8; ++i) m = fmaxf(m, eight_amax(v[i]));
  m = wave_max(m);
  if ((tid & 63) == 0) red[tid >> 6] = m;
  __syncthreads();
  m = fmaxf(fmaxf(red[0], red[1]), fmaxf(red[2], red[3]));
  float enc, dec;
  fb_scale(m, enc, dec);
  if (tid == 0) {
    scales[b] = dec;
    if (TR) scales_t[(e * nkb + kb) * nnb + nb] = dec;
  }
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const int64_t r = n0 + 16 * i + rg;
    const uint2 q = eight_codes(v[i], enc);
    if (r < N && c < K) *reinterpret_cast<uint2 *>(codes + (e * N + r) * K + c) = q;
    if constexpr (TR) {
      tile[(16 * i + rg) * 33 + 2 * l] = q.x;
      tile[(16 * i + rg) * 33 + 2 * l + 1] = q.y;
    }
  }
  if constexpr (TR) {
    __syncthreads();
    const int pr = tid & 7, c4 = tid >> 3;         // 16 rows from 16 pr on, columns 4 c4 ..
    uint32_t o[4][4];
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      uint32_t a[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) a[i] = tile[(16 * pr + 4 * q + i) * 33 + c4];
      // bytes of four rows -> four columns
      const uint32_t ab0 = __builtin_amdgcn_perm(a[1], a[0], 0x05010400u);   // a0.0 a1.0 a0.1 a1.1
      const uint32_t ab1 = __builtin_amdgcn_perm(a[1], a[0], 0x07030602u);
      const uint32_t cd0 = __builtin_amdgcn_perm(a[3], a[2], 0x05010400u);
      const uint32_t cd1 = __builtin_amdgcn_perm(a[3], a[2], 0x07030602u);
      o[0][q] = __builtin_amdgcn_perm(cd0, ab0, 0x05040100u);
      o[1][q] = __builtin_amdgcn_perm(cd0, ab0, 0x07060302u);
      o[2][q] = __builtin_amdgcn_perm(cd1, ab1, 0x05040100u);
      o[3][q] = __builtin_amdgcn_perm(cd1, ab1, 0x07060302u);
    }
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const int64_t kr = k0 + 4 * c4 + j, nc = n0 + 16 * pr;
      if (kr < K && nc < N)
        *reinterpret_cast<uint4 *>(codes_t + (e * K + kr) * N + nc) =
            make_uint4(o[j][0], o[j][1], o[j][2], o[j][3]);
    }
  }
}

template <typename T>
void launch_weight(const void *w, int64_t G, int64_t N, int64_t K, uint8_t *codes, float *scales,
                   uint8_t *codes_t, float *scales_t, hipStream_t s) {
  const int nnb = (int)((N + FB - 1) / FB), nkb = (int)((K + FB - 1) / FB);
  const dim3 grid((unsigned)(G * nnb * nkb)), block(256);
  const T *p = static_cast<const T *>(w);
  if (codes_t)
    hipLaunchKernelGGL((fp8_block_weight_kernel<T, true>), grid, block, 0, s, p, N, K, nnb, nkb,
                       codes, scales, codes_t, scales_t);
  else
    hipLaunchKernelGGL((fp8_block_weight_kernel<T, false>), grid, block, 0, s, p, N, K, nnb, nkb,
                       codes, scales, codes_t, scales_t);
}

}  // namespace

extern "C" qd_status fp8_block_quantize_act(const void *x, int32_t dtype, int64_t rows,
                                            int64_t cols, int64_t ld, uint8_t *codes,
                                            float *scales, void *stream) {
  if (dtype != QD_DTYPE_BF16 && dtype != QD_DTYPE_F32) return QD_ERR_DTYPE;
  if (rows < 0 || cols < 0 || cols % 16 != 0 || ld < cols || ld % 8 != 0) return QD_ERR_SHAPE;
  if (rows == 0 || cols == 0) return QD_OK;
  if (!x || !codes || !scales) return QD_ERR_NULL;
  if (!qdh::aligned16(x) || !qdh::aligned16(codes) || !qdh::aligned16(scales)) return QD_ERR_ALIGN;
  const int64_t gx = (rows - 1) / 16 + 1, gy = (cols - 1) / (4 * FB) + 1;
  if (!qdh::grid_fits(gx, 256) || gy > 65535) return QD_ERR_UNSUPPORTED;
  if (qdh::fault_injected()) return QD_ERR_HIP;
  hipStream_t s = qdh::S(stream);
  const dim3 grid((unsigned)gx, (unsigned)gy), block(256);
  if (dtype == QD_DTYPE_BF16)
    hipLaunchKernelGGL(fp8_block_act_kernel<uint16_t>, grid, block, 0, s,
                       static_cast<const uint16_t *>(x), rows, cols, ld, codes, scales);
  else
    hipLaunchKernelGGL(fp8_block_act_kernel<float>, grid, block, 0, s,
                       static_cast<const float *>(x), rows, cols, ld, codes, scales);
  return qdh::check_launch();
}

extern "C" qd_status fp8_block_quantize_weight(const void *w, int32_t dtype, int64_t groups,
                                               int64_t rows, int64_t cols, uint8_t *codes,
                                               float *scales, uint8_t *codes_t, float *scales_t,
                                               void *stream) {
  if (dtype != QD_DTYPE_BF16 && dtype != QD_DTYPE_F32) return QD_ERR_DTYPE;
  if (groups < 0 || rows < 0 || cols < 0 || cols % 16 != 0) return QD_ERR_SHAPE;
  if ((codes_t != nullptr) != (scales_t != nullptr)) return QD_ERR_NULL;
  if (codes_t && rows % 16 != 0) return QD_ERR_SHAPE;
  if (groups == 0 || rows == 0 || cols == 0) return QD_OK;
  if (!w || !codes || !scales) return QD_ERR_NULL;
  if (!qdh::aligned16(w) || !qdh::aligned16(codes) || !qdh::aligned16(scales) ||
      !qdh::aligned16(codes_t) || !qdh::aligned16(scales_t))
    return QD_ERR_ALIGN;
  const int64_t nnb = (rows - 1) / FB + 1, nkb = (cols - 1) / FB + 1;
  if (nnb > 0x7fffffffLL / nkb || groups > 0x7fffffffLL / (nnb * nkb) ||
      !qdh::grid_fits(groups * nnb * nkb, 256))
    return QD_ERR_UNSUPPORTED;
  if (qdh::fault_injected()) return QD_ERR_HIP;
  if (dtype == QD_DTYPE_BF16)
    launch_weight<uint16_t>(w, groups, rows, cols, codes, scales, codes_t, scales_t, qdh::S(stream));
  else
    launch_weight<float>(w, groups, rows, cols, codes, scales, codes_t, scales_t, qdh::S(stream));
  return qdh::check_launch();
}

// ---------------------------------------------------------------- layer
namespace {
struct BlockLayout {
  size_t route, ids, wts, offs, row_token, inv_row, xc, xs, hc, hs, hw, z, hw_bytes, total;
};
BlockLayout block_layer_layout(int64_t T, int64_t H, int32_t E, int32_t k, int64_t I) {
  BlockLayout L{};
  size_t o = 0;
  auto take = [&](size_t bytes) { size_t at = o; o += qdh::align_up(bytes > 0 ? bytes : 1); return at; };
  const size_t R = (size_t)T * k;
  L.route = take(moe_route_scored_workspace(T, E, k));
  L.ids = take(R * 4);
  L.wts = take(R * 4);
  L.offs = take((size_t)(E + 1) * 4);
  L.row_token = take(R * 4);
  L.inv_row = take(R * 4);
  L.xc = take((size_t)T * H);
  L.xs = take((size_t)T * ((H + FB - 1) / FB) * 4);
  L.hc = take(R * I);
  L.hs = take(R * ((I + FB - 1) / FB) * 4);
  L.hw_bytes = moe_fp8_block_grouped_gemm_workspace(T * k, 2 * I, H, E, QD_EPI_SWIGLU_FP8);
  L.hw = take(L.hw_bytes);
  L.z = take(R * H * 2);
  L.total = o;
  return L;
}
}  // namespace

extern "C" size_t qd_fp8_block_moe_layer_workspace(int64_t T, int64_t H, int32_t E, int32_t k,
                                                   int64_t I) {
  if (T < 0 || H < 0 || E < 1 || k < 1 || I < 0) return 0;
  return block_layer_layout(T, H, E, k, I).total;
}

extern "C" qd_status qd_fp8_block_moe_layer_forward(
    const void *x, const float *logits, int64_t T, int64_t H, int32_t E, int32_t k, int64_t I,
    int32_t scoring, const float *bias, int32_t groups, int32_t top_groups, int32_t group_sum,
    int32_t renorm, float scale, const uint8_t *live, const uint8_t *w13_codes,
    const float *w13_scales, const uint8_t *w2_codes, const float *w2_scales, void *y, void *ws,
    size_t ws_bytes, void *stream) {
  if (T < 0 || H <= 0 || H % 16 != 0 || I <= 0 || I % 32 != 0 || E < 1 || k < 1 || k > E)
    return QD_ERR_SHAPE;
  if (T > 0x7fffffffLL / k) return QD_ERR_SHAPE;
  if (!w13_codes || !w13_scales || !w2_codes || !w2_scales) return QD_ERR_NULL;
  if (T > 0 && (!x || !logits || !y)) return QD_ERR_NULL;
  if (!ws || ws_bytes < qd_fp8_block_moe_layer_workspace(T, H, E, k, I)) return QD_ERR_WORKSPACE;
  if (!qdh::aligned16(ws) || !qdh::aligned16(x) || !qdh::aligned16(y)) return QD_ERR_ALIGN;
  const int64_t R = T * k;
  const BlockLayout L = block_layer_layout(T, H, E, k, I);
  unsigned char *b = static_cast<unsigned char *>(ws);
  int32_t *ids = reinterpret_cast<int32_t *>(b + L.ids);
  float *wts = reinterpret_cast<float *>(b + L.wts);
  int32_t *offs = reinterpret_cast<int32_t *>(b + L.offs);
  int32_t *row_token = reinterpret_cast<int32_t *>(b + L.row_token);
  int32_t *inv_row = reinterpret_cast<int32_t *>(b + L.inv_row);
  uint8_t *xc = b + L.xc;
  float *xs = reinterpret_cast<float *>(b + L.xs);
  uint8_t *hc = b + L.hc;
  float *hs = reinterpret_cast<float *>(b + L.hs);
  // the products' refusals come before the first launch
  qd_status st = moe_fp8_block_grouped_gemm(xc, xs, T, row_token, offs, E, 0, w13_codes, w13_scales,
                                            2 * I, H, QD_EPI_SWIGLU_FP8, hc, hs, nullptr, 0, stream);
  if (st) return st;
  st = moe_fp8_block_grouped_gemm(hc, hs, R, nullptr, offs, E, 0, w2_codes, w2_scales, H, I,
                                  QD_EPI_NONE, b + L.z, nullptr, nullptr, 0, stream);
  if (st) return st;
  st = qdi::route_scored(logits, QD_DTYPE_F32, E, T, E, k, scoring, bias, groups, top_groups,
                         group_sum, renorm, scale, live, ids, wts, offs, row_token, inv_row,
                         b + L.route, moe_route_scored_workspace(T, E, k), x, H, xc, xs, stream);
  if (st || T == 0) return st;
  if (qdb::blk_few_rows(R, E, 2 * I, H, QD_EPI_SWIGLU_FP8) == 8 &&
      qdb::blk_few_rows(R, E, H, I, QD_EPI_NONE) == 8) {
    // a handful of rows: h stays in float32 and the down product quantises it (the
    // same codes): the layer of one token 29.7 -> 27.7 us
    float *h = reinterpret_cast<float *>(b + L.hw);
    const qdb::BlkArgs up{xc, xs, T, row_token, offs, E, R, w13_codes, w13_scales, (int)(2 * I), (int)H,
                     hc, hs};
    qdb::launch_blk_few(up, QD_EPI_SWIGLU_FP8, h, false, qdh::S(stream));
    const qdb::BlkArgs down{hc, hs, R, nullptr, offs, E, R, w2_codes, w2_scales, (int)H, (int)I,
                       b + L.z, nullptr};
    qdb::launch_blk_few_h(down, h, qdh::S(stream));
    st = qdh::check_launch();
    if (st) return st;
    return moe_unpermute_combine(b + L.z, inv_row, wts, T, k, H, y, stream);
  }
  st = moe_fp8_block_grouped_gemm(xc, xs, T, row_token, offs, E, R, w13_codes, w13_scales, 2 * I, H,
                                  QD_EPI_SWIGLU_FP8, hc, hs, b + L.hw, L.hw_bytes, stream);
  if (st) return st;
  st = moe_fp8_block_grouped_gemm(hc, hs, R, nullptr, offs, E, R, w2_codes, w2_scales, H, I,
                                  QD_EPI_NONE, b + L.z, nullptr, nullptr, 0, stream);
  if (st) return st;
  return moe_unpermute_combine(b + L.z, inv_row, wts, T, k, H, y, stream);
}
