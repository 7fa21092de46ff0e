// FP8 block GEMM for a handful of rows (arithmetic: gemm_block.hip).
//
// One token's experts are a few MB in all: with tiles of 256 weight rows 48 workgroups
// would stream them, and a tile's blocks of K come one after the other, 0.9 to 1.2 us each.
// Here a workgroup takes 32 weight rows of one expert and up to 8 or 32 of its rows, and
// its four waves split K: wave w takes the blocks w, w + 4, .. of 128, each through a ring of
// its own (weights, rows and scales, direct global->LDS loads counted by hand, no barrier),
// with the operands decoded to bf16, exactly.  The waves' float32 sums are joined in LDS in
// wave order, so that a row's bits are the same in tiles of 8 and of 32 (not those of the large
// kernel, which sums in another order).  With the quantising
// epilogue h goes to workspace in float32 and a second launch quantises it: a block of 128 of
// h spans eight workgroups.  The layer's down product of one token or two takes that h
// instead (HIN) and each wave quantises the blocks it needs, a launch less.
//
// Bound by latency: launch, tile search, row indices, the first block, the join (5 to 7 us
// at one row), and then by workgroups: two on a CU, 6 us a round of 512 at K = 2048.  8 experts
// of a row, K = 2048, N = 1536: 10 us, 2.5 TB/s of weights; K = 7168, N = 4096: 50, 4.7 TB/s.
#include "gemm_block.h"
#include "lds_dma.h"
#include "tile_sched.h"
#include <algorithm>
#include <cmath>

namespace {

using namespace qdb;
using namespace qdl;

// a tile of ROWS rows: a wave's ring slots, and a slot's weights, rows and scales
template <int ROWS>
struct FwCfg {
  static constexpr int NS = ROWS > 16 ? 2 : 3;     // two workgroups on a CU either way
  static constexpr int A = 4096, S = A + ROWS * 128, SLOT = S + 256;
  static constexpr int AL = ROWS / 8;    // line loads of rows
};

__device__ __forceinline__ int fw_swz(int r) { return (r >> 1) & 7; }

// h: where h goes (QD_EPI_SWIGLU_FP8), or with HIN the rows, f32 [rows][K]
template <int EPI, int ROWS, bool HIN>
__global__ __launch_bounds__(256) void gemm_block_few_kernel(BlkArgs p, int nfr, float *h) {
  using C = FwCfg<ROWS>;
  static_assert(!HIN || ROWS == 8, "a wave's share of h");
  constexpr bool GLU = EPI != QD_EPI_NONE;
  constexpr int AL = C::AL, LPS = HIN ? 5 : 5 + AL;   // counted loads of a block
  extern __shared__ __align__(16) unsigned char lds[];
  __shared__ int sh_w[4], sh_t[4];
  const int tid = threadIdx.x, lane = tid & 63, w = (int)uni((uint32_t)tid >> 6);
  const qdt::Tile tl = qdt::find_tile<ROWS>(p.offsets, p.E, p.rows, nfr, sh_w, sh_t);
  if (tl.e < 0) return;
  const int N = p.N, K = p.K, KB = (K + FB - 1) / FB, NB = (N + FB - 1) / FB;
  const int c0 = tl.nt * (GLU ? 16 : 32);          // first output column
  const int I = GLU ? N >> 1 : N;
  const uint32_t ring = uni((uint32_t)(uintptr_t)lds + (uint32_t)(w * C::NS * C::SLOT));

  // ---- addresses.  A line load: 8 rows, lane l brings row l / 8's piece (l % 8) ^ swz
  const int lr = lane >> 3;
  auto row_of = [&](int r) __attribute__((always_inline)) -> int64_t {
    const int64_t i = tl.row0 + (r < tl.nrows ? r : 0);
    return p.row_token ? (int64_t)p.row_token[i] : i;
  };
  const int64_t rs = row_of(lane & (ROWS - 1));
  uint32_t pw[4];                                  // piece of the row, by load
  const uint8_t *gw[4];
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    pw[j] = 16u * (uint32_t)((lane & 7) ^ fw_swz(8 * j + lr));
    gw[j] = p.w + ((int64_t)tl.e * N + bk_wrow<GLU>(8 * j + lr, c0, N)) * K + pw[j];
  }
  uint32_t pa[AL];
  const uint8_t *ga[AL];
#pragma unroll
  for (int j = 0; j < AL; ++j) {
    pa[j] = 16u * (uint32_t)((lane & 7) ^ fw_swz(8 * j + lr));
    ga[j] = p.a + row_of(8 * j + lr) * K + pa[j];
  }
  // scales: lanes 0 .. ROWS - 1 the rows', the next two the weights' of rows 0 and 16
  const bool wsc = (lane & ROWS) != 0;
  const float *gs = wsc || HIN ? p.w_scales + ((int64_t)tl.e * NB + bk_wrow<GLU>(16 * (lane & 1), c0, N) / FB) * KB
                        : p.a_scales + rs;
  const int64_t sstep = wsc || HIN ? 1 : p.a_rows;
  const uint8_t *z = reinterpret_cast<const uint8_t *>(&bk_zero);
  auto issue = [&](int kb, int slot) __attribute__((always_inline)) {
    const uint32_t at = uni(ring + slot * C::SLOT);
    const int k = kb * FB;                         // (past K: zeros; past KB: nothing is read)
#pragma unroll
    for (int j = 0; j < 4; ++j) dma16(k + (int)pw[j] < K ? gw[j] + k : z, at + j * 1024);
    if constexpr (!HIN) {
#pragma unroll
      for (int j = 0; j < AL; ++j) dma16(k + (int)pa[j] < K ? ga[j] + k : z, at + C::A + j * 1024);
    }
    dma4(gs + (kb < KB ? kb : KB - 1) * sstep, at + C::S);
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
  for (int i = 0; i < C::NS; ++i) issue(w + 4 * i, i);
  const int r = lane & 31, hh = lane >> 5, sw = fw_swz(r), ar = r & (ROWS - 1), sa = fw_swz(ar);
  int slot = 0;
  for (int i = 0; i < nb; ++i) {
    wait_vm<(C::NS - 1) * LPS>();
    unsigned char *sl = lds + (w * C::NS + slot) * C::SLOT;
    if constexpr (HIN) {                           // codes and scales to where the loads put them
      float *ss = reinterpret_cast<float *>(sl + C::S);
#pragma unroll
      for (int q = 0; q < 2; ++q) {
        const int rr = 4 * q + (lane >> 4), c8 = lane & 15;
        float enc, dec;
        fb_scale(row16_max(eight_amax(ha[0][q])), enc, dec);
        *reinterpret_cast<uint2 *>(sl + C::A + rr * 128 + ((c8 >> 1 ^ fw_swz(rr)) << 4) + 8 * (c8 & 1)) =
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
      ca[k] = *reinterpret_cast<const uint4 *>(sl + C::A + ar * 128 + ((pc ^ sa) << 4));
    }
    const float *ss = reinterpret_cast<const float *>(sl + C::S);
    // the scales' exponents go into the operands, the product of their mantissas stays: no
    // product of two scales leaves float32's range where the result does not
    const float as = ss[ar], w0 = ss[ROWS], w1 = ss[ROWS + 1], wr = r & 16 ? w1 : w0;
    const float s0 = bk_mant(as) * bk_mant(w0), s1 = bk_mant(as) * bk_mant(w1);
    f32x16 part;
#pragma unroll
    for (int q = 0; q < 16; ++q) part[q] = 0.0f;
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      part = __builtin_amdgcn_mfma_f32_32x32x16_bf16(dec8b(cw[k].x, cw[k].y, wr),
                                                     dec8b(ca[k].x, ca[k].y, as), part, 0, 0, 0);
      part = __builtin_amdgcn_mfma_f32_32x32x16_bf16(dec8b(cw[k].z, cw[k].w, wr),
                                                     dec8b(ca[k].z, ca[k].w, as), part, 0, 0, 0);
    }
    // the slot is in registers
    wait_lds();
    issue(w + 4 * (i + C::NS), slot);
    slot = slot + 1 == C::NS ? 0 : slot + 1;
#pragma unroll
    for (int q = 0; q < 16; ++q) acc[q] = __builtin_fmaf(part[q], q < 8 ? s0 : s1, acc[q]);
  }
  wait_vm<0>();
  __syncthreads();
  // ---- the join: sums [wave][row][weight row], then one output a thread
  float *red = reinterpret_cast<float *>(lds);
  if (r < ROWS) {
#pragma unroll
    for (int q = 0; q < 16; q += 4)
      *reinterpret_cast<float4 *>(red + (w * ROWS + r) * 32 + 2 * q + 4 * hh) =
          make_float4(acc[q], acc[q + 1], acc[q + 2], acc[q + 3]);
  }
  __syncthreads();
#pragma unroll
  for (int j = 0; j < AL; ++j) {
    const int row = 8 * j + (tid >> 5), m = tid & 31;
    auto sum = [&](int n) __attribute__((always_inline)) {
      float v = red[row * 32 + n];
#pragma unroll
      for (int k = 1; k < 4; ++k) v += red[(k * ROWS + row) * 32 + n];
      return v;
    };
    const int64_t o = (int64_t)(tl.row0 + row) * I + c0 + m;
    if (row >= tl.nrows || c0 + m >= I || (GLU && m >= 16)) continue;
    if constexpr (GLU) {
      const float v = bk_swiglu(sum(m), sum(m + 16));
      if constexpr (EPI == QD_EPI_SWIGLU_FP8) h[o] = v;
      else static_cast<__bf16 *>(p.out)[o] = (__bf16)v;
    } else {
      static_cast<__bf16 *>(p.out)[o] = (__bf16)sum(m);
    }
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

// Tiles of h rows that rows spread at random over E experts make: of a small mean one for
// each expert that has a row, of a larger one half a tile an expert more than they fill.
static double few_tiles(double rows, int E, double h) {
  if (E == 1) return ceil(rows / h);
  const double m = rows / E, some = 1.0 - exp(-m);
  return E * std::max(some, std::min(0.5, some) + m / h);
}

// The rows of a tile, 8 or 32, or 0 where the large kernel is ahead: the least of three times
// (us), fitted to graphs of ten calls (1 to 128 experts, 1 to 1835 rows, K = 304 to 2256, 704
// to 4096 weight rows).  Here: a base, and the workgroups two to a CU, each a fixed time
// and its blocks.  There, while the tiles of 64 rows fit a round of the CUs: a stage a
// block, one or two row fragments high, and the tiles' weights.  Longer K and wider N than
// fitted, measured afterwards at N = 4096, K = 7168 and N = 7168, K = 2048 (1, 32 and 256
// experts, 1 to 256 rows): the faster kernel or one within 3% of it but once (32 rows over 32
// experts, 142 us for 118).  Measured, 8 rows | 32 rows
// | large kernel, us:
//   1 expert, K = 2048, N = 1536: 8 rows 6.5 | 7.3 | 19.6; 128 14.2 | 8.2 | 24.1; 512 39.7 |
//   15.9 | 24.3; 1000 72.4 | 25.8 | 24.7
//   8 experts, K = 768, N = 2048: 32 rows 8.4 | 9.0 | 11.6; 191 19.7 | 9.9 | 11.9; 343 29.7 | 14.5 | 13.8
//   32 experts, K = 2256, N = 768: 22 rows 11.1 | 11.6 | 23.2; 467 29.9 | 19.9 | 27.3; 1835 79.7 | 34.5 | 32.1
//   14 of 128 experts, a row each, N = 2048: K = 576 11.8 | 13.3 | 12.2, K = 1088 14.3 | 15.9 | 15.5;
//   N = 4096, K = 1024 22.7 | 25.3 | 16.8
//   8 of 256 experts, a row each: N = 4096, K = 7168, SwiGLU quantised 50.4 | 52.8 | 64.9 (235 MB of
//   weights, 48 at the copy rate); N = 7168, K = 2048 33.0 | 36.7 | 28.5
int blk_few_rows(int64_t rows, int E, int64_t N, int64_t K, int epilogue) {
  const double r = (double)rows, KB = (double)((K + FB - 1) / FB), nfr = (double)((N + 31) / 32);
  if (rows < 1) return 0;
  const double tiles = few_tiles(r, E, 64.0) * (double)((N + 255) / 256);
  if (tiles > 256.0) return 0;
  const double base = 3.5 + 0.15 * KB + (epilogue == QD_EPI_SWIGLU_FP8 ? 4.0 : 0.0);
  const double t8 = base + few_tiles(r, E, 8.0) * nfr * (0.0063 + 0.0003 * KB);
  const double t32 = base + few_tiles(r, E, 32.0) * nfr * (0.0084 + 0.0003 * KB);
  const bool low = r <= (E == 1 ? 32.0 : 24.0 * E);
  const double large = (low ? 5.9 + 0.85 * KB : 6.5 + 1.12 * KB) + 0.012 * tiles;
  if (std::min(t8, t32) > large) return 0;
  return t8 <= t32 ? 8 : 32;
}

template <int EPI, int ROWS, bool HIN>
static void launch_few_one(const BlkArgs &p, float *h, hipStream_t s) {
  const int nfr = EPI == QD_EPI_NONE ? (p.N + 31) / 32 : (p.N / 2 + 15) / 16;
  // every tile has a row
  const int64_t most = std::min<int64_t>(p.rows, (p.rows + ROWS - 1) / ROWS + p.E);
  const int64_t grid = (most * nfr + 7) / 8 * 8;
  constexpr int LDS = 4 * FwCfg<ROWS>::NS * FwCfg<ROWS>::SLOT;
  auto kern = gemm_block_few_kernel<EPI, ROWS, HIN>;
  static std::atomic<uint64_t> done{0};
  blk_allow_lds(reinterpret_cast<const void *>(kern), LDS, done);
  hipLaunchKernelGGL(kern, dim3((unsigned)grid), dim3(256), LDS, s, p, nfr, h);
}
template <int EPI>
static void launch_few(const BlkArgs &p, float *h, hipStream_t s) {
  if (blk_few_rows(p.rows, p.E, p.N, p.K, EPI) == 32) launch_few_one<EPI, 32, false>(p, h, s);
  else launch_few_one<EPI, 8, false>(p, h, s);
}

void launch_blk_few(const BlkArgs &p, int epilogue, float *h, bool codes, hipStream_t s) {
  if (epilogue == QD_EPI_NONE) {
    launch_few<QD_EPI_NONE>(p, h, s);
  } else if (epilogue == QD_EPI_SWIGLU) {
    launch_few<QD_EPI_SWIGLU>(p, h, s);
  } else {
    launch_few<QD_EPI_SWIGLU_FP8>(p, h, s);
    if (!codes) return;
    const int I = p.N / 2;
    hipLaunchKernelGGL(block_few_quantize_kernel,
                       dim3((unsigned)((p.rows + 15) / 16), (unsigned)((I + 4 * FB - 1) / (4 * FB))),
                       dim3(256), 0, s, h, p.offsets, p.E, p.rows, I,
                       static_cast<uint8_t *>(p.out), p.out_scales);
  }
}

void launch_blk_few_h(const BlkArgs &p, const float *h, hipStream_t s) {
  launch_few_one<QD_EPI_NONE, 8, true>(p, const_cast<float *>(h), s);
}

}  // namespace qdb
