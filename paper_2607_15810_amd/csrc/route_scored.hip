// moe_route_scored_permute and moe_route_scored_backward (the choice: route_scored_dev.h).
//
// The layer's activations are quantised in the first launch, by workgroups of their own
// behind the routing's.
//
// Up to 64 tokens the whole call is one workgroup of sixteen waves (one token, 256 experts in
// 8 groups: 6 us); up to 256 the permutation is one; above, blocks of 256 tokens are counted
// and then placed.
//
// 8192 tokens, 256 experts in 8 groups, k = 8 (8.4 MB of f32 logits, 2 us of HBM): choice
// 17.3 us, counts 4.3, placing 7.2.  The choice is bound by its vector instructions: 741 a
// token, eight tokens a SIMD one after the other at 4 cycles and more each, 11.8 of the 17.3 us
// (counters); beside them 238 scalar ones a token, the launch and the first loads.  No part
// dominates: eight of the k + 1 rounds are 2 us, the float64 weights, on k of 64 lanes, 1.5,
// the float64 choice of the doubtful 2.  The gradient, 4096 x 128 in bf16: 6.1 us, float64
// exponentials of the chosen, one wave a token.  Placing adds the counts of all blocks in
// every workgroup: the square of T / 256, which is small up to some 10^5 tokens.
#include "fp8_block_dev.h"
#include "route_scored_dev.h"

namespace {

using namespace qds;

constexpr int RS_BLK = 256;            // tokens of a ranking block

// The quantisation of x beside the routing: workgroups from `first` on, nb of them for each
// four blocks of columns (x NULL: none).
struct ActBeside {
  const uint16_t *x;
  int64_t rows, cols;
  uint8_t *codes;
  float *scales;
  int first, nb;
};
__device__ __forceinline__ bool act_beside(const ActBeside &a) {
  const int b = (int)blockIdx.x - a.first;
  if (b < 0) return false;
  const int cb = b / a.nb;
  qdb::fb_quantize_act_body<uint16_t>(b - cb * a.nb, cb, a.x, a.rows, a.rows, a.cols, a.cols, a.codes,
                                      a.scales);
  return true;
}

template <typename L, int PER>
__global__ __launch_bounds__(256) void score_topk_kernel(ScoreArgs p, ScoreLanes sl, ActBeside act) {
  extern __shared__ __align__(16) unsigned char rs_lds[];
  if (act_beside(act)) return;
  const int wid = threadIdx.x >> 6;
  const int64_t t = (int64_t)blockIdx.x * 4 + wid;
  if (t < p.T)                                   // whole waves; no barriers inside
    rs_token<L, PER>(p, sl, t, reinterpret_cast<uint64_t *>(rs_lds) + (size_t)wid * p.E,
                     nullptr);
}

// ---------------------------------------------------------------- permutation
// exclusive scan of cnt[0 .. E) into cnt by the NT threads of the workgroup; the total
// (every thread).  ws: NT / 64 ints.
template <int NT>
__device__ __forceinline__ int rs_scan(int32_t *cnt, int E, int *ws) {
  constexpr int Q = (RS_EMAX + NT - 1) / NT;
  const int tid = threadIdx.x, lane = tid & 63, wid = tid >> 6;
  int c[Q], sum = 0;
#pragma unroll
  for (int q = 0; q < Q; ++q) {
    const int e = Q * tid + q;
    c[q] = e < E ? cnt[e] : 0;
    sum += c[q];
  }
  int xs = sum;
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) {
    const int y = __shfl_up(xs, o, 64);
    if (lane >= o) xs += y;
  }
  if (lane == 63) ws[wid] = xs;
  __syncthreads();
  int ex = xs - sum, total = 0;
#pragma unroll
  for (int w = 0; w < NT / 64; ++w) {
    if (w < wid) ex += ws[w];
    total += ws[w];
  }
#pragma unroll
  for (int q = 0; q < Q; ++q) {
    const int e = Q * tid + q;
    if (e < E) cnt[e] = ex;
    ex += c[q];
  }
  __syncthreads();
  return total;
}

// The permutation of up to W * 32 tokens in one workgroup of NT threads: a bit per
// (expert, token), counts, their scan, ranks by counting bits.
template <int W, int NT>
__device__ __forceinline__ void rs_permute_one(int64_t T, int E, int k, const int32_t *ids,
                                               uint32_t *mask, int32_t *base, int *ws,
                                               int32_t *offsets, int32_t *row_token,
                                               int32_t *inv_row) {
  const int tid = threadIdx.x, n = (int)T * k;
  for (int i = tid; i < E * W; i += NT) mask[i] = 0u;
  __syncthreads();
  for (int i = tid; i < n; i += NT) {
    const int e = ids[i], t = i / k;
    if (e >= 0) atomicOr(&mask[e * W + (t >> 5)], 1u << (t & 31));
  }
  __syncthreads();
  for (int e = tid; e < E; e += NT) {
    int c = 0;
#pragma unroll
    for (int w = 0; w < W; ++w) c += __popc(mask[e * W + w]);
    base[e] = c;
  }
  __syncthreads();
  const int rows = rs_scan<NT>(base, E, ws);
  for (int e = tid; e <= E; e += NT) offsets[e] = e < E ? base[e] : rows;
  for (int i = tid; i < n; i += NT) {
    const int e = ids[i], t = i / k;
    int row = -1;
    if (e >= 0) {
      row = base[e] + __popc(mask[e * W + (t >> 5)] & ((1u << (t & 31)) - 1u));
      for (int w = 0; w < (t >> 5); ++w) row += __popc(mask[e * W + w]);
      row_token[row] = t;
    }
    inv_row[i] = row;
    if (i >= rows) row_token[i] = -1;            // rows behind the last
  }
}

constexpr int RS_ONE = 64;             // tokens of the call in one workgroup

template <typename L, int PER>
__global__ __launch_bounds__(1024) void score_small_kernel(ScoreArgs p, ScoreLanes sl,
                                                           ActBeside act, int32_t *offsets,
                                                           int32_t *row_token, int32_t *inv_row) {
  extern __shared__ __align__(16) unsigned char rs_lds[];
  __shared__ uint32_t mask[RS_EMAX * (RS_ONE / 32)];
  __shared__ int32_t base[RS_EMAX], ids[RS_ONE * RS_KMAX];
  __shared__ int ws[16];
  if (act_beside(act)) return;
  const int wid = threadIdx.x >> 6;
  for (int64_t t = wid; t < p.T; t += 16)
    rs_token<L, PER>(p, sl, t, reinterpret_cast<uint64_t *>(rs_lds) + (size_t)wid * p.E,
                     ids + t * p.k);
  __syncthreads();
  rs_permute_one<RS_ONE / 32, 1024>(p.T, p.E, p.k, ids, mask, base, ws, offsets, row_token, inv_row);
}

__global__ __launch_bounds__(1024) void score_permute_kernel(int64_t T, int E, int k,
                                                             const int32_t *__restrict__ ids,
                                                             int32_t *__restrict__ offsets,
                                                             int32_t *__restrict__ row_token,
                                                             int32_t *__restrict__ inv_row) {
  __shared__ uint32_t mask[RS_EMAX * (RS_BLK / 32)];
  __shared__ int32_t base[RS_EMAX];
  __shared__ int ws[16];
  rs_permute_one<RS_BLK / 32, 1024>(T, E, k, ids, mask, base, ws, offsets, row_token, inv_row);
}

// The rank of every (token, slot) among the block's tokens of the same expert, and
// the block's counts; slots with id -1 take no part.
__global__ __launch_bounds__(RS_BLK) void score_rank_kernel(int64_t T, int E, int k,
                                                            const int32_t *__restrict__ ids,
                                                            int32_t *__restrict__ counts,
                                                            int32_t *__restrict__ ranks) {
  __shared__ uint32_t mask[RS_EMAX][RS_BLK / 32];
  __shared__ uint8_t before[RS_EMAX][RS_BLK / 32];
  const int tl = threadIdx.x;
  const int64_t t = (int64_t)blockIdx.x * RS_BLK + tl;
  int idr[8];
#pragma unroll
  for (int s = 0; s < 8; ++s) idr[s] = t < T && s < k ? ids[t * k + s] : -1;
  for (int i = tl; i < E * (RS_BLK / 32); i += RS_BLK) (&mask[0][0])[i] = 0u;
  __syncthreads();
  if (t < T) {
#pragma unroll
    for (int s = 0; s < 8; ++s)
      if (idr[s] >= 0) atomicOr(&mask[idr[s]][tl >> 5], 1u << (tl & 31));
    for (int s = 8; s < k; ++s) {
      const int e = ids[t * k + s];
      if (e >= 0) atomicOr(&mask[e][tl >> 5], 1u << (tl & 31));
    }
  }
  __syncthreads();
  for (int e = tl; e < E; e += RS_BLK) {
    int c = 0;
#pragma unroll
    for (int w = 0; w < RS_BLK / 32; ++w) {
      before[e][w] = (uint8_t)c;
      c += __popc(mask[e][w]);
    }
    counts[(int64_t)blockIdx.x * E + e] = c;
  }
  __syncthreads();
  if (t < T) {
    const uint32_t low = (1u << (tl & 31)) - 1u;
    auto put = [&](int s, int e) __attribute__((always_inline)) {
      if (e >= 0) ranks[t * k + s] = (int)before[e][tl >> 5] + __popc(mask[e][tl >> 5] & low);
    };
#pragma unroll
    for (int s = 0; s < 8; ++s) put(s, idr[s]);
    for (int s = 8; s < k; ++s) put(s, ids[t * k + s]);
  }
}

__global__ __launch_bounds__(RS_BLK) void score_scatter_kernel(
    int64_t T, int E, int k, int nblk, const int32_t *__restrict__ ids,
    const int32_t *__restrict__ counts, const int32_t *__restrict__ ranks,
    int32_t *__restrict__ offsets, int32_t *__restrict__ row_token,
    int32_t *__restrict__ inv_row) {
  __shared__ int32_t before[RS_EMAX], base[RS_EMAX];
  __shared__ int ws[4];
  const int tid = threadIdx.x, b = blockIdx.x;
  const int64_t t = (int64_t)b * RS_BLK + tid;
  int idr[8], rkr[8];                            // in flight beside the counts
#pragma unroll
  for (int s = 0; s < 8; ++s) {
    const bool in = t < T && s < k;
    idr[s] = in ? ids[t * k + s] : -1;
    rkr[s] = in ? ranks[t * k + s] : 0;          // (unwritten, unused for id -1)
  }
  for (int e = tid; e < E; e += RS_BLK) {
    int tot = 0, pre = 0;
    for (int b0 = 0; b0 < nblk; b0 += 16) {      // sixteen blocks' counts in flight
      int c[16];
#pragma unroll
      for (int j = 0; j < 16; ++j)
        c[j] = counts[(int64_t)(b0 + j < nblk ? b0 + j : nblk - 1) * E + e];
#pragma unroll
      for (int j = 0; j < 16; ++j) {
        if (b0 + j < nblk) tot += c[j];
        if (b0 + j < b) pre += c[j];
      }
    }
    base[e] = tot;
    before[e] = pre;
  }
  __syncthreads();
  const int rows = rs_scan<RS_BLK>(base, E, ws);
  if (b == 0)
    for (int e = tid; e <= E; e += RS_BLK) offsets[e] = e < E ? base[e] : rows;
  if (t < T) {
    auto put = [&](int s, int e, int rank) __attribute__((always_inline)) {
      int row = -1;
      if (e >= 0) {
        row = base[e] + before[e] + rank;
        row_token[row] = (int32_t)t;
      }
      inv_row[t * k + s] = row;
      if (t * k + s >= rows) row_token[t * k + s] = -1;    // rows behind the last
    };
#pragma unroll
    for (int s = 0; s < 8; ++s)
      if (s < k) put(s, idr[s], rkr[s]);
    for (int s = 8; s < k; ++s) put(s, ids[t * k + s], ids[t * k + s] >= 0 ? ranks[t * k + s] : 0);
  }
}

// ---------------------------------------------------------------- gradient
struct ScoreGradArgs {
  const void *logits;
  int64_t ld;
  int64_t T;
  int E, k, scoring, renorm;
  float scale;
  const int32_t *ids;
  const float *grad_w;
  void *grad;
  int64_t ldg;
};

template <typename L>
__device__ __forceinline__ void rs_store(void *p, int64_t i, double v);
template <>
__device__ __forceinline__ void rs_store<float>(void *p, int64_t i, double v) {
  static_cast<float *>(p)[i] = (float)v;
}
// one rounding: by way of a float32 that is rounded to odd (the even neighbour of a value in
// between would hide from the second rounding on which side of a tie it lies)
template <>
__device__ __forceinline__ void rs_store<uint16_t>(void *p, int64_t i, double v) {
  const float f = (float)v;
  const double a = fabs((double)f), b = fabs(v);
  uint32_t bits = __float_as_uint(f);
  if ((a < b || a > b) && !(bits & 1u)) bits += a < b ? 1u : 0xFFFFFFFFu;
  static_cast<__bf16 *>(p)[i] = (__bf16)__uint_as_float(bits);
}

// One wavefront per token; lane j < k holds chosen expert j.
template <typename L, int PER>
__global__ __launch_bounds__(256) void score_grad_kernel(ScoreGradArgs p) {
  const int lane = threadIdx.x & 63, wid = threadIdx.x >> 6;
  const int64_t t = (int64_t)blockIdx.x * 4 + wid;
  if (t >= p.T) return;
  const int E = p.E, k = p.k;
  int id = -1;
  double g = 0.0;
  float xs = 0.0f;
  if (lane < k) {
    id = p.ids[t * k + lane];
    if (id >= 0 && id < E) {
      g = (double)p.scale * (double)p.grad_w[t * k + lane];
      xs = rs_load<L>(p.logits, t * p.ld + id);
    } else {
      id = -1;
    }
  }
  const bool on = id >= 0;
  if (__ballot(on) == 0ull) {     // a dead token, whatever its logits
    for (int e = lane; e < E; e += 64) rs_store<L>(p.grad, t * p.ldg + e, 0.0);
    return;
  }
  const bool softmax = p.scoring == QD_SCORE_SOFTMAX, full = softmax && !p.renorm;
  double d = 0.0;                 // this lane's chosen expert's gradient
  double dot = 0.0, z = 1.0;
  float m = 0.0f;
  float x[PER];
  bool broken = false;            // softmax: a NaN or +inf logit leaves no score a number
  if (softmax) {
#pragma unroll
    for (int j = 0; j < PER; ++j) {
      const int e = lane + 64 * j;
      x[j] = e < E ? rs_load<L>(p.logits, t * p.ld + e) : -INFINITY;
      broken |= !(x[j] < INFINITY);
    }
    broken = __ballot(broken) != 0ull;
  }
  const double nan = __longlong_as_double(0x7ff8000000000000ll);
  if (broken) {
    d = nan;
  } else if (full) {
    m = x[0];
#pragma unroll
    for (int j = 1; j < PER; ++j) m = fmaxf(m, x[j]);
    m = wave_max(m);
    double part = 0.0;
#pragma unroll
    for (int j = 0; j < PER; ++j)
      if (lane + 64 * j < E && m != -INFINITY) part += exp((double)x[j] - (double)m);
    z = rs_wave_sum(part);
    const double s = on && m != -INFINITY ? exp((double)xs - (double)m) / z : 0.0;
    dot = rs_wave_sum(s * g);
    d = s * (g - dot);
  } else if (softmax) {
    const float top = wave_max(on ? xs : -INFINITY);
    const double s = on && top != -INFINITY ? exp((double)xs - (double)top) : 0.0;
    const double n = rs_wave_sum(s);
    const double q = n == 0.0 ? 0.0 : s / n;
    d = q * (g - rs_wave_sum(q * g));
  } else {
    const double s = on ? rs_sigmoid(xs) : 0.0;
    // 1 - s without cancellation
    const double ns = on ? 1.0 / (1.0 + exp((double)xs)) : 0.0;
    if (p.renorm) {
      const double n = rs_wave_sum(s);
      const double q = n == 0.0 ? 0.0 : s / n;
      // dl = (g - sum g q) / n * s * (1 - s)
      d = q * (g - rs_wave_sum(q * g)) * ns;
    } else {
      d = g * s * ns;
    }
  }
#pragma unroll
  for (int j = 0; j < PER; ++j) {
    const int e = lane + 64 * j;
    double v = 0.0;
    if (full && broken) v = nan;
    else if (full && m != -INFINITY) v = -exp((double)x[j] - (double)m) / z * dot;
    for (int q = 0; q < k; ++q) {
      const int eq = __builtin_amdgcn_readlane(id, q);
      const double dq = rs_lane(d, q);
      if (eq == e) v = dq;
    }
    if (e < E) rs_store<L>(p.grad, t * p.ldg + e, v);
  }
}

qd_status check_scoring(int32_t dtype, int64_t ld, int64_t T, int32_t E, int32_t k,
                        int32_t scoring, int32_t renorm) {
  if (dtype != QD_DTYPE_BF16 && dtype != QD_DTYPE_F32) return QD_ERR_DTYPE;
  if (scoring != QD_SCORE_SOFTMAX && scoring != QD_SCORE_SIGMOID) return QD_ERR_DTYPE;
  if (T < 0 || E < 1 || E > RS_EMAX || k < 1 || k > E || k > RS_KMAX || ld < E) return QD_ERR_SHAPE;
  if (renorm != 0 && renorm != 1) return QD_ERR_SHAPE;
  if (T > 0x7fffffffLL / k || T > 0x7fffffffLL - 3) return QD_ERR_SHAPE;
  return QD_OK;
}

}  // namespace

extern "C" size_t moe_route_scored_workspace(int64_t T, int32_t E, int32_t k) {
  if (T <= RS_BLK) return 0;
  const int64_t nblk = (T + RS_BLK - 1) / RS_BLK;
  return qdh::align_up((size_t)nblk * (E > 0 ? E : 1) * 4) +
         qdh::align_up((size_t)T * (k > 0 ? k : 1) * 4);
}

namespace qdi {

qd_status route_scored(
    const void *logits, int32_t dtype, int64_t ld, int64_t T, int32_t E, int32_t k,
    int32_t scoring, const float *bias, int32_t groups, int32_t top_groups, int32_t group_sum,
    int32_t renorm, float scale, const uint8_t *live, int32_t *topk_ids, float *topk_w,
    int32_t *expert_offsets, int32_t *row_token, int32_t *inv_row, void *ws, size_t ws_bytes,
    const void *x, int64_t cols, uint8_t *x_codes, float *x_scales, void *stream) {
  const qd_status bad = check_scoring(dtype, ld, T, E, k, scoring, renorm);
  if (bad) return bad;
  if (groups < 1 || groups > RS_GMAX || E % groups != 0 || top_groups < 1 || top_groups > groups ||
      (group_sum != 1 && group_sum != 2) || (groups > 1 && group_sum > E / groups) ||
      (int64_t)top_groups * (E / groups) < k || !(scale - scale == 0.0f))
    return QD_ERR_SHAPE;
  if (!expert_offsets) return QD_ERR_NULL;
  if (T > 0 && (!logits || !topk_ids || !topk_w || !row_token || !inv_row)) return QD_ERR_NULL;
  const size_t need = moe_route_scored_workspace(T, E, k);
  if (need > 0 && (!ws || ws_bytes < need)) return QD_ERR_WORKSPACE;
  if (!qdh::aligned16(logits) || !qdh::aligned16(bias) || !qdh::aligned16(topk_ids) ||
      !qdh::aligned16(topk_w) || !qdh::aligned16(expert_offsets) || !qdh::aligned16(row_token) ||
      !qdh::aligned16(inv_row) || !qdh::aligned16(ws))
    return QD_ERR_ALIGN;   // (NULL is aligned)
  hipStream_t s = qdh::S(stream);
  if (T == 0) {
    if (qdh::fault_injected()) return QD_ERR_HIP;
    qdi::launch_fill_i32(expert_offsets, E + 1, 0, s);
    return qdh::check_launch();
  }
  ScoreArgs p{logits, ld, T, E, k, scoring, bias, groups, top_groups, group_sum,
              renorm, scale, live, topk_ids, topk_w};
  const bool bf16 = dtype == QD_DTYPE_BF16;
  const ScoreLanes sl = rs_lanes(E, groups);
  const size_t keys = sl.lq < 0 ? (size_t)E * 8 : 0;       // a wave's
  // x's workgroups: a row for each 16 threads, four blocks of columns
  const bool one = T <= RS_ONE && keys <= 2048;  // (its LDS stays below 64 KB)
  const int64_t groups_of = one ? 1 : (T + 3) / 4, arows = one ? 64 : 16;
  ActBeside act{static_cast<const uint16_t *>(x), T, cols, x_codes, x_scales, (int)groups_of,
                (int)((T + arows - 1) / arows)};
  const int64_t acts = x ? act.nb * ((cols + 4 * qdb::FB - 1) / (4 * qdb::FB)) : 0;
  if (!qdh::grid_fits(groups_of + acts, one ? 1024 : 256)) return QD_ERR_UNSUPPORTED;
  if (qdh::fault_injected()) return QD_ERR_HIP;
  const dim3 grid((unsigned)(groups_of + acts));
  if (one) {
    rs_by_width(sl.per, [&](auto w) {
      constexpr int PER = decltype(w)::value;
      hipLaunchKernelGGL((bf16 ? score_small_kernel<uint16_t, PER> : score_small_kernel<float, PER>),
                         grid, dim3(1024), 16 * keys, s, p, sl, act, expert_offsets, row_token,
                         inv_row);
    });
    return qdh::check_launch();
  }
  rs_by_width(sl.per, [&](auto w) {
    constexpr int PER = decltype(w)::value;
    hipLaunchKernelGGL((bf16 ? score_topk_kernel<uint16_t, PER> : score_topk_kernel<float, PER>),
                       grid, dim3(256), 4 * keys, s, p, sl, act);
  });
  if (T <= RS_BLK) {
    hipLaunchKernelGGL(score_permute_kernel, dim3(1), dim3(1024), 0, s, T, E, k, topk_ids,
                       expert_offsets, row_token, inv_row);
    return qdh::check_launch();
  }
  const int nblk = (int)((T + RS_BLK - 1) / RS_BLK);
  int32_t *counts = static_cast<int32_t *>(ws);
  int32_t *ranks = reinterpret_cast<int32_t *>(static_cast<char *>(ws) +
                                               qdh::align_up((size_t)nblk * E * 4));
  hipLaunchKernelGGL(score_rank_kernel, dim3(nblk), dim3(RS_BLK), 0, s, T, E, k, topk_ids, counts,
                     ranks);
  hipLaunchKernelGGL(score_scatter_kernel, dim3(nblk), dim3(RS_BLK), 0, s, T, E, k, nblk, topk_ids,
                     counts, ranks, expert_offsets, row_token, inv_row);
  return qdh::check_launch();
}

}  // namespace qdi

extern "C" qd_status moe_route_scored_permute(
    const void *logits, int32_t dtype, int64_t ld, int64_t T, int32_t E, int32_t k,
    int32_t scoring, const float *bias, int32_t groups, int32_t top_groups, int32_t group_sum,
    int32_t renorm, float scale, const uint8_t *live, int32_t *topk_ids, float *topk_w,
    int32_t *expert_offsets, int32_t *row_token, int32_t *inv_row, void *ws, size_t ws_bytes,
    void *stream) {
  return qdi::route_scored(logits, dtype, ld, T, E, k, scoring, bias, groups, top_groups, group_sum,
                           renorm, scale, live, topk_ids, topk_w, expert_offsets, row_token, inv_row,
                           ws, ws_bytes, nullptr, 0, nullptr, nullptr, stream);
}

extern "C" qd_status moe_route_scored_backward(const void *logits, int32_t dtype, int64_t ld,
                                               int64_t T, int32_t E, int32_t k, int32_t scoring,
                                               int32_t renorm, float scale,
                                               const int32_t *topk_ids, const float *grad_w,
                                               void *grad_logits, int64_t ld_grad, void *stream) {
  const qd_status bad = check_scoring(dtype, ld, T, E, k, scoring, renorm);
  if (bad) return bad;
  if (ld_grad < E || !(scale - scale == 0.0f)) return QD_ERR_SHAPE;
  if (T == 0) return QD_OK;
  if (!logits || !topk_ids || !grad_w || !grad_logits) return QD_ERR_NULL;
  if (!qdh::aligned16(logits) || !qdh::aligned16(topk_ids) || !qdh::aligned16(grad_w) ||
      !qdh::aligned16(grad_logits))
    return QD_ERR_ALIGN;
  if (!qdh::grid_fits((T + 3) / 4, 256)) return QD_ERR_UNSUPPORTED;
  if (qdh::fault_injected()) return QD_ERR_HIP;
  hipStream_t s = qdh::S(stream);
  ScoreGradArgs p{logits, ld, T, E, k, scoring, renorm, scale, topk_ids, grad_w, grad_logits, ld_grad};
  const dim3 grid((unsigned)((T + 3) / 4)), block(256);
  rs_by_width((E + 63) / 64, [&](auto per) {
    constexpr int PER = decltype(per)::value;
    if (dtype == QD_DTYPE_BF16)
      hipLaunchKernelGGL((score_grad_kernel<uint16_t, PER>), grid, block, 0, s, p);
    else
      hipLaunchKernelGGL((score_grad_kernel<float, PER>), grid, block, 0, s, p);
  });
  return qdh::check_launch();
}
