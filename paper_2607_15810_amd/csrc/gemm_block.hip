// Grouped GEMM over FP8 operands with block scales:
//   v[r][n] = sum_kb sa[kb][src(r)] sw[e][n / 128][kb] sum_{k in block kb} a[src(r)][k] w[e][n][k]
// with its epilogues: bf16, SwiGLU in bf16, SwiGLU quantised to FP8 with 1 x 128 scales.
//
// Arithmetic.  The FP8 MFMAs add four products at a time and drop what lies more than
// about twelve bits below the largest of them (measured against float64, K = 128: up to
// 2^-12.5 of sum |products| from a 448 among values near 2^-4, on every fp8 and f8f6f4
// shape), so a sum on them is no 32-bit sum.  Operands are decoded to bf16 in registers
// and multiplied on v_mfma_f32_32x32x16_bf16, whose sums are (2^-22 on the same inputs),
// at half the FP8 rate.
//
// Scales.  The conversion (v_cvt_scalef32_pk_bf16_fp8) takes a power of two for nothing, so
// the exponents of both scales go into the operands, exactly.  What is left of a block is
// the product u of the two mantissas, in [1, 4): the sums stand in units of the current
// block's u and are multiplied by u_before / u once a block, one multiplication per element,
// and once by u at the end.  (Partial sums of a block folded into a total by a
// multiply-add cost the same instruction and a second set of accumulators, and those kept
// tiles at 128 rows: 4096^3 137 -> 121 us.)  The quotient of the units is corrected to its
// rounding (two instructions a fragment and block, at most 1% of a call): blocks of one unit
// are not rescaled at all, where the hardware's reciprocal alone made every block shrink what
// was summed by up to 2^-22, always to the same side (K = 7168: 2^-19.6 of a half's sum).
//
// The weights are the instruction's first operand, so a lane holds one activation row: its
// row scale is one register, and the columns of a row leave a lane together.
//
//  * Workgroup tile: up to 64 MF rows of one expert x 256 weight rows (SwiGLU: 128 gate
//    rows and the matching up rows, one block of 128 of h; a fragment of 32 holds 16 of
//    each, so that a lane has both), eight waves in a 2 x 4 grid.  A wave has two weight
//    fragments and half of the tile's row fragments; of an odd last one each half of the
//    grid takes one weight fragment, so that a tile of n row fragments costs n / 2 of
//    them whatever n is.  The schedule is the NVFP4 panel kernel's (panel_sched.h): one
//    persistent workgroup per CU, its tiles' stages one stream through an LDS ring
//    filled by direct global->LDS loads.
//  * Bound, for hundreds of rows per expert, by the matrix unit and the vector unit beside
//    it: 7 vector instructions per MFMA (decoding 3 to 4, rescaling 2), the matrix unit
//    busy 50% of the cycles at 2.1 GHz (4096^3: 1.05 to 1.13 PFLOP/s by the card; an isolated
//    loop of the same instructions on random operands, which the chip's power limits, reaches
//    1.5).  Of experts 0.73 to 0.8 PFLOP/s, busy 32 to 39%: tiles of uneven height (9 to 10
//    vector instructions per MFMA), the epilogue, weights from HBM, and a stage's loads, which
//    all eight waves issue together after the barrier with no MFMA beside them.
//    For tens of rows by HBM: 5.1 to 5.4 TB/s of weights.
//  * Calls of a few rows, whose tiles would leave most CUs idle, run on the kernel of
//    gemm_block_few.hip.
//  * A stage is one block of K: 128 bytes of every row, the tile's row scales of that
//    block and the scales of its weight fragments.  Pieces of 16 bytes past K come from a
//    zero in memory.  The pieces of a row are placed by a row-dependent XOR, so the
//    fragment reads are free of bank conflicts.  One barrier per stage.
#include "gemm_block.h"
#include "lds_dma.h"
#include "panel_sched.h"
#include "tile_sched.h"

namespace {

using namespace qdb;
using namespace qdl;
using namespace qdp;

template <int MF>
struct BkCfg {
  static constexpr int M = 64 * MF;
  static constexpr int BOFF = M * 128;                 // weight codes
  static constexpr int SOFF = BOFF + 32768;            // row scales, then fragment scales
  static constexpr int SLOT = SOFF + (MF + 1) * 256;
  static constexpr int LPS = MF + 4 + 1;               // loads per wave and stage
};

__host__ __device__ constexpr int bk_ns(int mf) { return mf > 2 ? 2 : 3; }   // stages of the ring

struct BkLayout {
  int tok, amax, dummy, offs, mpre, perm, total;
};
// after the ring: the tokens of two tiles, the waves' row maxima (quantising
// epilogue), the target of placeholder loads, the tile schedule
__host__ __device__ inline BkLayout bk_layout(int mf, int E) {
  BkLayout L{};
  int o = bk_ns(mf) * (64 * mf * 128 + 32768 + (mf + 1) * 256);
  auto take = [&](int bytes) { const int at = o; o += (bytes + 15) & ~15; return at; };
  L.tok = take(2 * 64 * mf * 4);
  L.amax = take(8 * 64 * mf * 4);
  L.dummy = take(256);
  L.offs = take((E + 1) * 4);
  L.mpre = take((E + 1) * 4);
  L.perm = take(E * 2);
  L.total = o;
  return L;
}

typedef const __attribute__((address_space(4))) BlkArgs *BkArgPtr;
__device__ __forceinline__ BkArgPtr bk_args() {
  BkArgPtr q = (BkArgPtr)__builtin_amdgcn_kernarg_segment_ptr();
  asm volatile("" : "+s"(q));
  return q;
}

// 16-byte piece c of tile row r sits at piece c ^ bk_swz(r) of the row's 128
__device__ __forceinline__ int bk_swz(int r) { return (r >> 1) & 7; }

template <int MF, int EPI>
__global__ __launch_bounds__(PN_THREADS, 2) void gemm_block_kernel(BlkArgs p, PnDeal deal) {
  using C = BkCfg<MF>;
  constexpr bool GLU = EPI != QD_EPI_NONE;
  extern __shared__ __align__(16) unsigned char lds[];
  __shared__ int sh_w[8];
  __shared__ int sh_c[8][2 * MF + 1];
  const int tid = threadIdx.x, lane = tid & 63, w = (int)uni((uint32_t)tid >> 6);
  const int N = p.N, E = p.E, K = p.K;
  const int KB = (K + FB - 1) / FB, NB = (N + FB - 1) / FB;
  constexpr int NC = GLU ? 128 : PN_N;         // output columns of a tile
  constexpr int NR = bk_ns(MF);
  const int nst = KB > 3 ? KB : 3;             // the deepest ring at least (zeros past K), at
                                               // every height, so that bits do not differ
  const BkLayout L = bk_layout(MF, E);
  const uint32_t lds0 = (uint32_t)(uintptr_t)lds;
  int32_t *offs = reinterpret_cast<int32_t *>(lds + L.offs);
  int32_t *mpre = reinterpret_cast<int32_t *>(lds + L.mpre);
  uint16_t *perm = reinterpret_cast<uint16_t *>(lds + L.perm);
  const int32_t *tokb = reinterpret_cast<const int32_t *>(lds + L.tok);
  float *amax = reinterpret_cast<float *>(lds + L.amax);
  pn_schedule<MF>(p.offsets, p.rows, E, offs, mpre, perm, sh_w, sh_c);
  __syncthreads();
  const PnSched S{offs, mpre, perm, E, deal, (int)(blockIdx.x & 7)};
  const int nsl = gridDim.x >> 3;
  const int t_end = pn_walk(S);
  // the workgroup's tiles: one of each run of nsl places of the walk, from alternate ends,
  // since the tiles' heights descend (128 experts of 256 +- 16 rows: the longest of the
  // XCD's CUs has 26 row fragments in five tiles, 29.5 from one end)
  int ct = blockIdx.x >> 3;                // the tile being multiplied
  const int odd = 2 * (nsl - ct) - 1, even = 2 * ct + 1;   // steps to runs 1, 3, .. and 2, 4, ..
  int cstep = odd, istep = odd;
  // two waves of a SIMD (w, w + 4) take different row halves
  const int wm = (w ^ (w >> 2)) & 1, wn = w >> 1;

  // ---- loads.  A line load: 8 rows, lane l brings row l / 8's piece
  // (l % 8) ^ swz (rows 8 (w + 8 j) ..: the XOR depends on w's parity only)
  const uint32_t pc = 16u * (uint32_t)((lane & 7) ^ bk_swz(8 * (w & 1) + (lane >> 3)));
  const uint32_t dummy = lds0 + (uint32_t)L.dummy;
  int it = ct, left = 0, ecur = 0, ibuf = 0;
  PnTile itl{}, nx{};
  int kb = 0;                              // the block of K of the next stage to load
  uint32_t oa[MF], ob[4], os = 0;
  const uint8_t *pa = nullptr, *wb = nullptr, *sb = nullptr;
  auto tok_dma = [&](const PnTile &tl, int buf) __attribute__((always_inline)) {
    const int32_t *rt = bk_args()->row_token;
    const int wi = pn_fresh_s(w);
    if (rt && wi < MF) {
      const int r = 64 * wi + lane;
      dma4s(uni_ptr(rt), (uint32_t)(tl.row0 + (r < tl.nrows ? r : 0)) * 4u,
            uni(lds0 + (uint32_t)(L.tok + buf * (C::M * 4) + wi * 256)));
    }
  };
  auto src = [&](const int32_t *rt, int r) __attribute__((always_inline)) -> uint32_t {
    if (rt) return (uint32_t)tokb[ibuf * C::M + r];
    return (uint32_t)(itl.row0 + (r < itl.nrows ? r : 0));
  };
  // to tile itl's first stage (its tokens are in LDS), the tokens of the tile
  // after it on their way
  auto bind = [&]() __attribute__((always_inline)) {
    const BkArgPtr q = bk_args();
    const int wi = pn_fresh_s(w), ln = pn_fresh(lane);
    // Where the tile starts in K.  Rows that lie a multiple of 4 KB apart put a block on a
    // few memory channels, and workgroups that all start at block 0 meet there: each
    // weight-row tile has a place of its own.  (Not each expert too, which would be 1 to 3%
    // faster still: within this kernel a row's bits depend on neither the batch, the schedule
    // nor the expert's number.)  128 experts of 16 rows, N = 1536: K = 4096 187 -> 154 us, K = 4224, from
    // block 0 on, 152; 256 rows, K = 768: 141 from block 0, 147 spread.
    kb = K % 4096 == 0 ? (int)uni((uint32_t)(13 * itl.nt) % (uint32_t)KB) : 0;
    wb = uni_ptr(q->w + (int64_t)itl.e * N * K + kb * FB);
    pa = uni_ptr(q->a + kb * FB);
    const int32_t *rt = q->row_token;
#pragma unroll
    for (int j = 0; j < MF; ++j)
      oa[j] = src(rt, 8 * (wi + 8 * j) + (ln >> 3)) * (uint32_t)K + pc;
#pragma unroll
    for (int j = 0; j < 4; ++j)
      ob[j] = (uint32_t)bk_wrow<GLU>(8 * (wi + 8 * j) + (ln >> 3), NC * itl.nt, N) * (uint32_t)K + pc;
    // the stage's scales: rows of the tile by waves 0 .. MF - 1, weights (lane f: the
    // tile's rows from 16 f on) by wave MF, a placeholder by the others
    if (wi < MF) {
      sb = reinterpret_cast<const uint8_t *>(uni_ptr(q->a_scales + kb * q->a_rows));
      os = src(rt, 64 * wi + ln) * 4u;
    } else {
      sb = reinterpret_cast<const uint8_t *>(uni_ptr(q->w_scales + (int64_t)itl.e * NB * KB + kb));
      os = wi == MF ? (uint32_t)(bk_wrow<GLU>(16 * (ln & 15), NC * itl.nt, N) / FB) * (uint32_t)KB * 4u : 0u;
    }
    left = nst;
    if (it + istep < t_end) {
      nx = pn_locate<MF>(S, it + istep, ecur, lane);
      tok_dma(nx, ibuf ^ 1);
    }
  };
  // a stage of loads into the slot at LDS address at, LPS per wave always
  // (placeholders past the last tile), so that the waits can count
  auto loads = [&](uint32_t at) __attribute__((always_inline)) {
    const bool none = nst - 1 - left >= KB;    // (left has been counted down) no block: zeros
    if ((kb + 1) * FB <= K && !none) {
#pragma unroll
      for (int j = 0; j < MF; ++j) dma16s(pa, oa[j], uni(at + (w + 8 * j) * 1024));
#pragma unroll
      for (int j = 0; j < 4; ++j) dma16s(wb, ob[j], uni(at + C::BOFF + (w + 8 * j) * 1024));
    } else {                                   // a short block: zeros past K
      const bool in = !none && kb * FB + (int)pc < K;
      const uint8_t *z = reinterpret_cast<const uint8_t *>(&bk_zero);
#pragma unroll
      for (int j = 0; j < MF; ++j) dma16(in ? pa + oa[j] : z, uni(at + (w + 8 * j) * 1024));
#pragma unroll
      for (int j = 0; j < 4; ++j)
        dma16(in ? wb + ob[j] : z, uni(at + C::BOFF + (w + 8 * j) * 1024));
    }
    dma4s(sb, os, uni(w <= MF ? at + C::SOFF + w * 256 : dummy));
    const int64_t step = w < MF ? bk_args()->a_rows * 4 : w == MF ? 4 : 0;
    const int d = kb + 1 < KB ? 1 : 1 - KB;    // to the next block, round to the first
    kb += d;
    pa += d * FB;
    wb += d * FB;
    sb += d * step;
  };
  auto issue = [&](uint32_t at) __attribute__((always_inline)) {
    if (left == 0) {
      it += istep;
      istep = odd + even - istep;
      if (it < t_end) {
        itl = nx;
        ibuf ^= 1;
        bind();
      } else {
        left = 0x7fffffff;
      }
    }
    --left;
    if (it < t_end) {
      loads(at);
    } else {
      const uint8_t *any = uni_ptr(bk_args()->a);
#pragma unroll
      for (int j = 0; j < C::LPS; ++j) dma4s(any, 0u, uni(dummy));
    }
  };

  if (it < t_end) {
    itl = pn_locate<MF>(S, it, ecur, lane);
    tok_dma(itl, 0);
    wait_vm<0>();
    pn_barrier();
    bind();
    for (int q = 0; q < NR; ++q) {         // stages of this tile (NR <= nst)
      --left;
      loads(uni(lds0 + q * C::SLOT));
    }
    wait_vm<(NR - 1) * C::LPS>();
    pn_barrier();
  }
  int slot = 0;
  PnTile cur = itl;
  while (ct < t_end) {
    const int nt = cur.nt, row0 = cur.row0, nrows = cur.nrows;
    const int nfr = (nrows + 31) >> 5;

    // FULL row fragments of this wave's half with both weight fragments, and HALF: the
    // tile's last one with the first of them
    auto run = [&](auto nfr_c) __attribute__((always_inline)) {
      constexpr int FULL = decltype(nfr_c)::value / 2, HALF = decltype(nfr_c)::value % 2;
      constexpr int MA = FULL + HALF, NJ = FULL > 0 ? 2 : 1;
      constexpr int ITEMS = 2 * MA;            // (half of the block, row fragment)
      constexpr int NS = GLU ? 2 : 1;          // scales of a fragment: gate and up halves
      f32x16 acc[MA][2];
      float unit[MA][NS];
      auto nj = [](int i) { return i < FULL ? 2 : 1; };
#pragma unroll
      for (int i = 0; i < MA; ++i) {
#pragma unroll
        for (int g = 0; g < NS; ++g) unit[i][g] = 1.0f;
#pragma unroll
        for (int j = 0; j < 2; ++j)
#pragma unroll
          for (int q = 0; q < 16; ++q)
            if (j < nj(i)) acc[i][j][q] = 0.0f;
      }
      const int r = lane & 31, h = lane >> 5, sw = bk_swz(r);
      struct Op {
        uint4 c[2];
      };
      // row fragment i, weight fragment j (the grid's halves take them in either order)
      auto fa = [&](int i) __attribute__((always_inline)) { return i < FULL ? wm * FULL + i : 2 * FULL; };
      auto fb = [&](int j) __attribute__((always_inline)) { return 2 * wn + (j ^ wm); };
      // half st of row fragment i, of weight fragment j
      auto rd_a = [&](const unsigned char *sl, int n) __attribute__((always_inline)) -> Op {
        Op o;
        const int st = n / MA, i = n % MA;
#pragma unroll
        for (int k = 0; k < 2; ++k)
          o.c[k] = *reinterpret_cast<const uint4 *>(sl + (32 * fa(i) + r) * 128 +
                                                    (((4 * st + 2 * h + k) ^ sw) << 4));
        return o;
      };
      auto rd_b = [&](const unsigned char *sl, int st, int j) __attribute__((always_inline)) -> Op {
        Op o;
#pragma unroll
        for (int k = 0; k < 2; ++k)
          o.c[k] = *reinterpret_cast<const uint4 *>(sl + C::BOFF + (32 * fb(j) + r) * 128 +
                                                    (((4 * st + 2 * h + k) ^ sw) << 4));
        return o;
      };
      auto step8 = [](const Op &o, int ks, float sc) __attribute__((always_inline)) -> bf16x8 {
        const uint4 q = o.c[ks >> 1];
        return (ks & 1) ? dec8b(q.z, q.w, sc) : dec8b(q.x, q.y, sc);
      };
      auto sync = [&]() __attribute__((always_inline)) -> uint32_t {
        wait_vm<(NR - 2) * C::LPS>();
        pn_barrier();
        const uint32_t at = uni(lds0 + slot * C::SLOT);
        slot = slot + 1 == NR ? 0 : slot + 1;
        return at;
      };
      struct Scales {
        float w[NS], r[MA], wl;                // wl: of this lane's weight row
      };
      auto rd_s = [&](const unsigned char *sl) __attribute__((always_inline)) -> Scales {
        const float *ss = reinterpret_cast<const float *>(sl + C::SOFF);
        Scales o;
#pragma unroll
        for (int g = 0; g < NS; ++g) o.w[g] = ss[64 * MF + 4 * wn + g];
#pragma unroll
        for (int i = 0; i < MA; ++i) o.r[i] = ss[32 * fa(i) + r];
        o.wl = ss[64 * MF + 4 * wn + (GLU ? (r >> 4) & 1 : 0)];
        return o;
      };
      // quarter e of fragment i's sums to the unit of the block whose scales are v
      float rho[NS];
      auto rescale = [&](int i, int e, const Scales &v) __attribute__((always_inline)) {
        if (e == 0) {
          const float ma = bk_mant(v.r[i]);
#pragma unroll
          for (int g = 0; g < NS; ++g) {
            const float u = ma * bk_mant(v.w[g]), rc = __builtin_amdgcn_rcpf(u);
            const float q = unit[i][g] * rc;       // and its error: the quotient rounded, 1 of equal units
            rho[g] = __builtin_fmaf(__builtin_fmaf(-q, u, unit[i][g]), rc, q);
            unit[i][g] = u;
          }
        }
        const int n = 4 * nj(i);
#pragma unroll
        for (int k = 0; k < 8; ++k) {
          const int j = (e * n + k) >> 4, q = (e * n + k) & 15;
          if (k < n) acc[i][j & 1][q] *= rho[GLU ? q >> 3 : 0];
        }
        // here and not where the compiler would sink it, past the loop's branches
#pragma unroll
        for (int j = 0; j < 2; ++j)
          if (j < nj(i))
          if (j == (e * n) >> 4 || j == (e * n + n - 1) >> 4) asm volatile("" : "+v"(acc[i][j]));
      };
      // The stream of one wave: per k-step of 16 the MFMAs of its operands, beside them
      // the decoding of the next step's and a quarter of a rescaling, held together by
      // the scheduling barriers.  Codes are read an item ahead; the workgroup's barrier
      // stands before the last item, whose codes are in registers.  Fragment i is
      // rescaled in the item before its block begins.
      Op bq[NJ];
      const unsigned char *s0 = lds + slot * C::SLOT;
      Op a = rd_a(s0, 0);
#pragma unroll
      for (int j = 0; j < NJ; ++j) bq[j] = rd_b(s0, 0, j);
      Scales sv = rd_s(s0);
      if constexpr (MA > 1) {
#pragma unroll
        for (int e = 0; e < 4; ++e) rescale(0, e, sv);
      }
      bf16x8 av = step8(a, 0, sv.r[0]), b[NJ][4];
#pragma unroll
      for (int j = 0; j < NJ; ++j) b[j][0] = step8(bq[j], 0, sv.wl);
      for (int s = 0; s < nst; ++s) {
        const unsigned char *sl = lds + slot * C::SLOT;
        Scales sn = sv;
#pragma unroll
        for (int n = 0; n < ITEMS; ++n) {
          const int st = n / MA, i = n % MA;
          const bool last = n + 1 == ITEMS, turn = i == MA - 1;   // turn: the next item is fragment 0
          Op an, bn[NJ];
          uint32_t at = 0;
          if (last) {
            at = sync();
            sl = lds + slot * C::SLOT;         // (past the last stage: the next tile's, unused)
            sn = rd_s(sl);
          }
          an = rd_a(sl, last ? 0 : n + 1);
          if (turn) {
#pragma unroll
            for (int j = 0; j < NJ; ++j) bn[j] = rd_b(sl, last ? 0 : 1, j);
          }
          if (MA == 1 && st == 0) {
#pragma unroll
            for (int e = 0; e < 4; ++e) rescale(0, e, sv);
          }
#pragma unroll
          for (int ks = 0; ks < 4; ++ks) {
            __builtin_amdgcn_sched_barrier(0);
#pragma unroll
            for (int j = 0; j < 2; ++j)
              if (j < nj(i))
              acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(b[j][ks], av, acc[i][j], 0, 0, 0);
            if (ks < 3) {
              av = step8(a, ks + 1, sv.r[i]);
              if (i == 0) {
#pragma unroll
                for (int j = 0; j < NJ; ++j) b[j][ks + 1] = step8(bq[j], ks + 1, sv.wl);
              }
            } else {
              av = step8(an, 0, last ? sn.r[0] : sv.r[turn ? 0 : i + 1]);
              if (turn) {
#pragma unroll
                for (int j = 0; j < NJ; ++j) b[j][0] = step8(bn[j], 0, last ? sn.wl : sv.wl);
              }
            }
            if (MA > 1 && last && s + 1 < nst) {   // (its scales have just been read)
              if (ks > 0) rescale(0, ks - 1, sn);
              if (ks == 3) rescale(0, 3, sn);
            }
            if (st == 0 && !turn) rescale(i + 1, ks, sv);
          }
          __builtin_amdgcn_sched_barrier(0);
          if (last) issue(at);
          a = an;
          if (turn) {
#pragma unroll
            for (int j = 0; j < NJ; ++j) bq[j] = bn[j];
          }
        }
        sv = sn;
      }
#pragma unroll
      for (int i = 0; i < MA; ++i)
#pragma unroll
        for (int j = 0; j < 2; ++j)
#pragma unroll
          for (int q = 0; q < 16; ++q)
            if (j < nj(i)) acc[i][j][q] *= unit[i][GLU ? q >> 3 : 0];
      // ---- epilogue.  Element q of a fragment: its weight row 8 (q / 4) + 4 h + q % 4, row r
      // of the rows; with SwiGLU q and q + 8 are gate and up of column 8 (q / 4) + 4 h + q % 4
      // of 16.  Four consecutive columns are a quad; the halves of the wave swap quads, so that
      // a lane stores 8 consecutive columns.
      const int ldo = pn_fresh_s(GLU ? N >> 1 : N);
      const int ln = pn_fresh(lane), rr = ln & 31, hh = ln >> 5;
      if constexpr (GLU) {
#pragma unroll
        for (int i = 0; i < MA; ++i)
#pragma unroll
          for (int j = 0; j < 2; ++j)
#pragma unroll
            for (int q = 0; q < 8; ++q)
              if (j < nj(i)) acc[i][j][q] = bk_swiglu(acc[i][j][q], acc[i][j][q + 8]);
      }
      // first column of fragment j
      auto col = [&](int j) __attribute__((always_inline)) {
        return GLU ? nt * 128 + 16 * fb(j) : nt * PN_N + 32 * fb(j);
      };
      if constexpr (EPI == QD_EPI_SWIGLU_FP8) {
        // the maximum over the block's columns, 16 of each fragment
#pragma unroll
        for (int i = 0; i < MA; ++i) {
          float m = 0.0f;
#pragma unroll
          for (int j = 0; j < 2; ++j)
#pragma unroll
            for (int q = 0; q < 8; ++q)
              if (j < nj(i)) m = fmaxf(m, fabsf(acc[i][j][q]));
          m = col(0) < ldo ? fmaxf(m, __shfl_xor(m, 32, 64)) : 0.0f;
          if (hh == 0) amax[(i < FULL ? wn : wn + 4 * wm) * C::M + 32 * fa(i) + rr] = m;
        }
        pn_barrier();
#pragma unroll
        for (int i = 0; i < MA; ++i) {
          const int rl = 32 * fa(i) + rr;
          float m = 0.0f;
#pragma unroll
          for (int k = 0; k < (i < FULL ? 4 : 8); ++k) m = fmaxf(m, amax[k * C::M + rl]);
          float enc, dec;
          fb_scale(m, enc, dec);
          const BkArgPtr g = bk_args();
          const bool in = rl < nrows;
          uint8_t *o = static_cast<uint8_t *>(g->out) + (int64_t)(row0 + rl) * ldo;
#pragma unroll
          for (int j = 0; j < 2; ++j) if (j < nj(i)) {
            const uint32_t q0 = fb_codes4(acc[i][j][0], acc[i][j][1], acc[i][j][2], acc[i][j][3], enc);
            const uint32_t q1 = fb_codes4(acc[i][j][4], acc[i][j][5], acc[i][j][6], acc[i][j][7], enc);
            const Pair32 u = swap32(q0, q1);
            if (in && col(j) < ldo)
              *reinterpret_cast<uint2 *>(o + col(j) + 8 * hh) = make_uint2(u.x, u.y);
          }
          if (in && hh == 0 && (i < FULL ? wn : w) == 0)
            g->out_scales[(int64_t)nt * g->rows + row0 + rl] = dec;
        }
      } else {
        // quads q and q + 1 of fragment j: columns 8 q .., of the wave's upper half 8 (q + 1) ..
        auto pair = [&](int i, int j, int q) __attribute__((always_inline)) {
          uint32_t lo[2], hi[2];
#pragma unroll
          for (int k = 0; k < 2; ++k) {
            const int e = 4 * q + 2 * k;
            lo[k] = bf16_pair(acc[i][j][e], acc[i][j][e + 1]);
            hi[k] = bf16_pair(acc[i][j][e + 4], acc[i][j][e + 5]);
          }
          const Pair32 u = swap32(lo[0], hi[0]), v = swap32(lo[1], hi[1]);
          return make_uint4(u.x, v.x, u.y, v.y);
        };
#pragma unroll
        for (int i = 0; i < MA; ++i)
#pragma unroll
          for (int j = 0; j < 2; ++j) if (j < nj(i)) {
            uint16_t *out = static_cast<uint16_t *>(bk_args()->out);
            auto put = [&](int rl, int c, uint4 v) __attribute__((always_inline)) {
              if (rl < nrows && c < ldo)
                *reinterpret_cast<uint4 *>(out + (int64_t)(row0 + rl) * ldo + c) = v;
            };
            if constexpr (GLU) {
              put(32 * fa(i) + rr, col(j) + 8 * hh, pair(i, j, 0));
            } else {
              // both pairs of 16 rows in one store, so that it writes 64 bytes of each
              const uint4 a = pair(i, j, 0), b = pair(i, j, 2);
              const Pair32 x = swap16(a.x, b.x), y = swap16(a.y, b.y), z = swap16(a.z, b.z),
                           w = swap16(a.w, b.w);
              const int rl = 32 * fa(i) + (ln & 15), c = col(j) + 16 * ((ln >> 4) & 1) + 8 * hh;
              put(rl, c, make_uint4(x.x, y.x, z.x, w.x));
              put(rl + 16, c, make_uint4(x.y, y.y, z.y, w.y));
            }
          }
      }
      // the stores' lane branches join here, so that they do not make the
      // scalar state of the tile loop look divergent to the compiler
      asm volatile("" ::: "memory");
    };
    auto pick = [&](auto self, auto n_c) __attribute__((always_inline)) {
      constexpr int n = decltype(n_c)::value;
      if constexpr (n == 1) {
        run(std::integral_constant<int, 1>{});
      } else {
        if (nfr == n) run(std::integral_constant<int, n>{});
        else self(self, std::integral_constant<int, n - 1>{});
      }
    };
    pick(pick, std::integral_constant<int, 2 * MF>{});
    // the issue cursor is NR (<= nst) stages ahead: at the next tile
    ct += cstep;
    cstep = odd + even - cstep;
    cur = itl;
  }
  wait_vm<0>();
}

constexpr double BK_TILE = 2.0;        // a tile's fixed time, in that of a 32-row fragment

struct BlkPlan {
  int mf, grid, lds;
  PnDeal deal;
};

inline BlkPlan blk_plan(int64_t rows, int E, int64_t N, int epilogue) {
  BlkPlan pl{};
  const int ntn = (int)((N + PN_N - 1) / PN_N);
  // the height with the least estimated time: rounds of the CUs times a tile's
  const double mean = (double)rows / E, sd = std::max(0.5, sqrt(mean));
  PnHeight h{};
  for (const int mf : {1, 2, 4}) {
    if (bk_layout(mf, E).total > PN_LDS_MAX) continue;
    double var;
    const double n = std::max(pn_tiles(mean, sd, E, 64.0 * mf, 0.0, &var), 1.0 / E);
    const double t = pn_rounds(n * E, sqrt(var * E), ntn) * (BK_TILE + (mean / 32.0 + 0.5) / n);
    if (h.mf == 0 || t < 0.995 * h.time)       // even: the lower, its ring is deeper
      h = {mf, bk_ns(mf), std::max(1, (int)std::min(8.0, n + 0.5)), n * E, t};
  }
  pl.mf = h.mf;
  pl.lds = bk_layout(h.mf, E).total;
  pl.grid = (int)std::min<int64_t>(256, qdt::tile_grid(rows, E, 64 * pl.mf, ntn));
  pl.deal = pn_deal(h, ntn, pl.grid);
  return pl;
}

template <int MF, int EPI>
void launch_blk_one(const BlkArgs &p, const BlkPlan &pl, hipStream_t s) {
  auto kern = gemm_block_kernel<MF, EPI>;
  static std::atomic<uint64_t> done{0};
  blk_allow_lds(reinterpret_cast<const void *>(kern), PN_LDS_MAX, done);
  hipLaunchKernelGGL(kern, dim3((unsigned)pl.grid), dim3(PN_THREADS), (size_t)pl.lds, s, p, pl.deal);
}
template <int EPI>
void launch_blk(const BlkArgs &p, const BlkPlan &pl, hipStream_t s) {
  if (pl.mf == 4) launch_blk_one<4, EPI>(p, pl, s);
  else if (pl.mf == 2) launch_blk_one<2, EPI>(p, pl, s);
  else launch_blk_one<1, EPI>(p, pl, s);
}

}  // namespace

extern "C" size_t moe_fp8_block_grouped_gemm_workspace(int64_t rows, int64_t N, int64_t K, int32_t E,
                                                       int32_t epilogue) {
  if (rows <= 0 || N <= 0 || K <= 0 || E < 1 || epilogue != QD_EPI_SWIGLU_FP8) return 0;
  return blk_few_rows(rows, E, N, K, epilogue) ? qdh::align_up((size_t)rows * (N / 2) * 4) : 0;
}

extern "C" qd_status moe_fp8_block_grouped_gemm(
    const uint8_t *a_codes, const float *a_scales, int64_t a_rows, const int32_t *row_token,
    const int32_t *expert_offsets, int32_t E, int64_t rows, const uint8_t *w_codes,
    const float *w_scales, int64_t N, int64_t K, int32_t epilogue, void *out, float *out_scales,
    void *ws, size_t ws_bytes, void *stream) {
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
  // (rows that are gathered: their indices' offsets are 32-bit too)
  if (E > PN_EMAX || rows > 0x3fffffffLL || a_rows > 0x3fffffffLL || N > 0x3fffffffLL ||
      K > 0x3fffffffLL || a_rows + 1 > lim / K || N > (lim - 1) / K)
    return QD_ERR_UNSUPPORTED;
  const size_t need = moe_fp8_block_grouped_gemm_workspace(rows, N, K, E, epilogue);
  if (need > 0 && (!ws || ws_bytes < need)) return QD_ERR_WORKSPACE;
  if (!qdh::aligned16(ws)) return QD_ERR_ALIGN;
  if (qdh::fault_injected()) return QD_ERR_HIP;
  if (rows == 0) return QD_OK;
  BlkArgs p{a_codes, a_scales, a_rows, row_token, expert_offsets, E, rows, w_codes, w_scales,
            (int)N, (int)K, out, out_scales};
  hipStream_t s = qdh::S(stream);
  if (blk_few_rows(rows, E, N, K, epilogue)) {
    launch_blk_few(p, epilogue, static_cast<float *>(ws), true, s);
    return qdh::check_launch();
  }
  const BlkPlan pl = blk_plan(rows, E, N, epilogue);
  if (epilogue == QD_EPI_NONE) launch_blk<QD_EPI_NONE>(p, pl, s);
  else if (epilogue == QD_EPI_SWIGLU) launch_blk<QD_EPI_SWIGLU>(p, pl, s);
  else launch_blk<QD_EPI_SWIGLU_FP8>(p, pl, s);
  return qdh::check_launch();
}
