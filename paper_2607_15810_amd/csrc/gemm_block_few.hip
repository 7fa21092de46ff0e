// FP8 block GEMM for a handful of rows (arithmetic: gemm_block.hip).
//
// One token's experts are a few MB in all: with tiles of 256 weight rows 48 workgroups
// would stream them.  Here a workgroup takes 32 weight rows of one expert and up to eight of
// its rows, and its four waves split K: wave w takes the blocks w, w + 4, .. of 128, each
// through a ring of three slots of its own (weights, rows and scales, direct global->LDS
// loads counted by hand, no barrier), with the operands decoded to f16 as in the large
// kernel.  The waves' float32 sums are joined in LDS in wave order.  With the quantising
// epilogue h goes to workspace in float32 and a second launch quantises it: a block of 128 of
// h spans eight workgroups.  The layer's down product takes that h instead (HIN) and each
// wave quantises the blocks it needs, a launch less.  Bound by latency: launch, tile search, row indices, the first
// block, four to eight blocks a wave, the join.
#include "gemm_block.h"
#include "lds_dma.h"
#include "tile_sched.h"
#include <algorithm>

namespace {

using namespace qdb;
using namespace qdl;

constexpr int FW_ROWS = 8;             // rows of a tile
constexpr int FW_NS = 3;               // ring slots of a wave
constexpr int FW_A = 4096, FW_S = FW_A + 1024, FW_SLOT = FW_S + 256;

__device__ __forceinline__ int fw_swz(int r) { return (r >> 1) & 7; }

// h: where h goes (QD_EPI_SWIGLU_FP8), or with HIN the rows, f32 [rows][K]
template <int EPI, bool HIN>
__global__ __launch_bounds__(256) void gemm_block_few_kernel(BlkArgs p, int nfr, float *h) {
  constexpr bool GLU = EPI != QD_EPI_NONE;
  constexpr int LPS = HIN ? 5 : 6;                 // counted loads of a block
  extern __shared__ __align__(16) unsigned char lds[];
  __shared__ int sh_w[4], sh_t[4];
  const int tid = threadIdx.x, lane = tid & 63, w = (int)uni((uint32_t)tid >> 6);
  const qdt::Tile tl = qdt::find_tile<FW_ROWS>(p.offsets, p.E, p.rows, nfr, sh_w, sh_t);
  if (tl.e < 0) return;
  const int N = p.N, K = p.K, KB = (K + FB - 1) / FB, NB = (N + FB - 1) / FB;
  const int c0 = tl.nt * (GLU ? 16 : 32);          // first output column
  const int I = GLU ? N >> 1 : N;
  const uint32_t ring = uni((uint32_t)(uintptr_t)lds + (uint32_t)(w * FW_NS * FW_SLOT));

  // ---- addresses.  A line load: 8 rows, lane l brings row l / 8's piece (l % 8) ^ swz
  const int lr = lane >> 3;
  auto row_of = [&](int r) __attribute__((always_inline)) -> int64_t {
    const int64_t i = tl.row0 + (r < tl.nrows ? r : 0);
    return p.row_token ? (int64_t)p.row_token[i] : i;
  };
  const int64_t ra = row_of(lr), rs = row_of(lane & 7);
  uint32_t pw[4];                                  // piece of the row, by load
  const uint8_t *gw[4];
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    pw[j] = 16u * (uint32_t)((lane & 7) ^ fw_swz(8 * j + lr));
    gw[j] = p.w + ((int64_t)tl.e * N + bk_wrow<GLU>(8 * j + lr, c0, N)) * K + pw[j];
  }
  const uint32_t pa = 16u * (uint32_t)((lane & 7) ^ fw_swz(lr));
  const uint8_t *ga = p.a + ra * K + pa;
  // scales: lanes 0 .. 7 the rows', lanes 8, 9 the weights' of rows 0 and 16
  const bool wsc = (lane & 8) != 0;
  const float *gs = wsc || HIN ? p.w_scales + ((int64_t)tl.e * NB + bk_wrow<GLU>(16 * (lane & 1), c0, N) / FB) * KB
                        : p.a_scales + rs;
  const int64_t sstep = wsc || HIN ? 1 : p.a_rows;
  const uint8_t *z = reinterpret_cast<const uint8_t *>(&bk_zero);
  auto issue = [&](int kb, int slot) __attribute__((always_inline)) {
    const uint32_t at = uni(ring + slot * FW_SLOT);
    const int k = kb * FB;                         // (past K: zeros; past KB: nothing is read)
#pragma unroll
    for (int j = 0; j < 4; ++j) dma16(k + (int)pw[j] < K ? gw[j] + k : z, at + j * 1024);
    if constexpr (!HIN) dma16(k + (int)pa < K ? ga + k : z, at + FW_A);
    dma4(gs + (kb < KB ? kb : KB - 1) * sstep, at + FW_S);
  };
  const int nb = (KB - w + 3) >> 2;                // blocks of this wave
  f32x16 acc;
#pragma unroll
  for (int q = 0; q < 16; ++q) acc[q] = 0.0f;
  // HIN: this wave's next two blocks of the rows, eight elements of rows lane / 16 and
  // 4 + lane / 16 each (asked for ahead of the counted loads, which their waits include)
  Eight<float> ha[2][2];
  auto load_h = [&](Eight<float> (&v)[2], int kb) __attribute__((always_inline)) {
    const int k = kb * FB + 8 * (lane & 15);
#pragma unroll
    for (int q = 0; q < 2; ++q) {
      const int rr = 4 * q + (lane >> 4);
      if (k < K) v[q].load(h + (int64_t)(tl.row0 + (rr < tl.nrows ? rr : 0)) * K + k);
      else v[q].zero();
    }
  };
  if constexpr (HIN) {
    load_h(ha[0], w);
    load_h(ha[1], w + 4);
  }
#pragma unroll
  for (int i = 0; i < FW_NS; ++i) issue(w + 4 * i, i);
  const int r = lane & 31, hh = lane >> 5, sw = fw_swz(r), sa = fw_swz(r & 7);
  int slot = 0;
  for (int i = 0; i < nb; ++i) {
    wait_vm<(FW_NS - 1) * LPS>();
    unsigned char *sl = lds + w * FW_NS * FW_SLOT + slot * FW_SLOT;
    if constexpr (HIN) {                           // codes and scales to where the loads put them
      float *ss = reinterpret_cast<float *>(sl + FW_S);
#pragma unroll
      for (int q = 0; q < 2; ++q) {
        const int rr = 4 * q + (lane >> 4), c8 = lane & 15;
        float enc, dec;
        fb_scale(row16_max(eight_amax(ha[0][q])), enc, dec);
        *reinterpret_cast<uint2 *>(sl + FW_A + rr * 128 + ((c8 >> 1 ^ fw_swz(rr)) << 4) + 8 * (c8 & 1)) =
            eight_codes(ha[0][q], enc);
        if (c8 == 0) ss[rr] = dec;
      }
      wait_lds();
      ha[0][0] = ha[1][0];
      ha[0][1] = ha[1][1];
      load_h(ha[1], w + 4 * (i + 2));
    }
    uint4 cw[4], ca[4];
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      const int pc = (k >> 1) * 4 + 2 * hh + (k & 1);
      cw[k] = *reinterpret_cast<const uint4 *>(sl + r * 128 + ((pc ^ sw) << 4));
      ca[k] = *reinterpret_cast<const uint4 *>(sl + FW_A + (r & 7) * 128 + ((pc ^ sa) << 4));
    }
    const float *ss = reinterpret_cast<const float *>(sl + FW_S);
    const float s0 = ss[r & 7] * ss[8], s1 = ss[r & 7] * ss[9];
    f32x16 part;
#pragma unroll
    for (int q = 0; q < 16; ++q) part[q] = 0.0f;
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      part = __builtin_amdgcn_mfma_f32_32x32x16_f16(dec8(cw[k].x, cw[k].y), dec8(ca[k].x, ca[k].y),
                                                    part, 0, 0, 0);
      part = __builtin_amdgcn_mfma_f32_32x32x16_f16(dec8(cw[k].z, cw[k].w), dec8(ca[k].z, ca[k].w),
                                                    part, 0, 0, 0);
    }
    // the slot is in registers
    wait_lds();
    issue(w + 4 * (i + FW_NS), slot);
    slot = slot + 1 == FW_NS ? 0 : slot + 1;
#pragma unroll
    for (int q = 0; q < 16; ++q) acc[q] = __builtin_fmaf(part[q], q < 8 ? s0 : s1, acc[q]);
  }
  wait_vm<0>();
  __syncthreads();
  // ---- the join: sums [wave][row][weight row], then one output a thread
  float *red = reinterpret_cast<float *>(lds);
  if (r < FW_ROWS) {
#pragma unroll
    for (int q = 0; q < 16; q += 4)
      *reinterpret_cast<float4 *>(red + (w * FW_ROWS + r) * 32 + 2 * q + 4 * hh) =
          make_float4(acc[q], acc[q + 1], acc[q + 2], acc[q + 3]);
  }
  __syncthreads();
  const int row = tid >> 5, m = tid & 31;
  auto sum = [&](int n) __attribute__((always_inline)) {
    float v = red[row * 32 + n];
#pragma unroll
    for (int k = 1; k < 4; ++k) v += red[(k * FW_ROWS + row) * 32 + n];
    return v;
  };
  const int64_t o = (int64_t)(tl.row0 + row) * I + c0 + m;
  const bool in = row < tl.nrows && c0 + m < I && (!GLU || m < 16);
  if (!in) return;
  if constexpr (GLU) {
    const float v = bk_swiglu(sum(m), sum(m + 16));
    if constexpr (EPI == QD_EPI_SWIGLU_FP8) h[o] = v;
    else static_cast<__bf16 *>(p.out)[o] = (__bf16)v;
  } else {
    static_cast<__bf16 *>(p.out)[o] = (__bf16)sum(m);
  }
}

// h to codes: rows below the last offset
__global__ __launch_bounds__(256) void block_few_quantize_kernel(const float *__restrict__ h,
                                                                 const int32_t *offsets, int E,
                                                                 int64_t rows, int I,
                                                                 uint8_t *__restrict__ codes,
                                                                 float *__restrict__ scales) {
  fb_quantize_act_body<float>(blockIdx.x, blockIdx.y, h, rows, offsets ? offsets[E] : rows, I, I,
                              codes, scales);
}

}  // namespace

namespace qdb {

// The 8-row tiles of the experts that the rows may reach times the large kernel's tiles
// of 256 weight rows, up to which this kernel is ahead.  Graphs of ten calls, here against
// there: K = 2048, 1536 weight rows, quantised: 8 experts of a row 13.3 us against 18.7, 16
// 18.5 against 19.3, 24 27.1 against 22.6; in bf16, 8 experts of 16 rows 14.3 against 20.2, of 32
// 23.6 against 20.4; K = 768, 2048 weight rows, bf16: 8 experts of a row 7.2 against 10.6, 16 12.1
// against 11.3; one expert, 2048 x 2048: 64 rows 11.0 against 22.5, 100 16.6 against 23.8, 256 29.2
// against 24.7; 4096 weight rows: 64 18.3 against 24.3, 100 27.4 against 24.4.
constexpr int64_t FW_TILES = 128, FW_TILES_FP8 = 96, FW_MOST = 128;
bool blk_few(int64_t rows, int E, int64_t N, int epilogue) {
  const int64_t ntn = (N + 255) / 256, mts = std::max<int64_t>((rows + 7) / 8, std::min<int64_t>(rows, E));
  return rows <= FW_MOST && mts * ntn <= (epilogue == QD_EPI_SWIGLU_FP8 ? FW_TILES_FP8 : FW_TILES);
}

template <int EPI, bool HIN>
static void launch_few_one(const BlkArgs &p, float *h, hipStream_t s) {
  const int nfr = EPI == QD_EPI_NONE ? (p.N + 31) / 32 : (p.N / 2 + 15) / 16;
  // every tile has a row
  const int64_t most = std::min<int64_t>(p.rows, (p.rows + FW_ROWS - 1) / FW_ROWS + p.E);
  const int64_t grid = (most * nfr + 7) / 8 * 8;
  constexpr int LDS = 4 * FW_NS * FW_SLOT;
  auto kern = gemm_block_few_kernel<EPI, HIN>;
  static std::atomic<uint64_t> done{0};
  blk_allow_lds(reinterpret_cast<const void *>(kern), LDS, done);
  hipLaunchKernelGGL(kern, dim3((unsigned)grid), dim3(256), LDS, s, p, nfr, h);
}

void launch_blk_few(const BlkArgs &p, int epilogue, float *h, bool codes, hipStream_t s) {
  if (epilogue == QD_EPI_NONE) {
    launch_few_one<QD_EPI_NONE, false>(p, h, s);
  } else if (epilogue == QD_EPI_SWIGLU) {
    launch_few_one<QD_EPI_SWIGLU, false>(p, h, s);
  } else {
    launch_few_one<QD_EPI_SWIGLU_FP8, false>(p, h, s);
    if (!codes) return;
    const int I = p.N / 2;
    hipLaunchKernelGGL(block_few_quantize_kernel,
                       dim3((unsigned)((p.rows + 15) / 16), (unsigned)((I + 4 * FB - 1) / (4 * FB))),
                       dim3(256), 0, s, h, p.offsets, p.E, p.rows, I,
                       static_cast<uint8_t *>(p.out), p.out_scales);
  }
}

void launch_blk_few_h(const BlkArgs &p, const float *h, hipStream_t s) {
  launch_few_one<QD_EPI_NONE, true>(p, const_cast<float *>(h), s);
}

}  // namespace qdb
