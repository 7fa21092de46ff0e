// Scored routing of the MoE layer: softmax or sigmoid scores, a bias that enters
// the choice only (balance), expert groups, renormalised and scaled weights,
// padded batches; the row permutation of moe_route_permute; the gradient of the
// logits.
//
//   s = sigmoid(l) or softmax(l), c = s + bias
//   group score = sum of the group_sum largest c of a group; the top_groups best
//   groups stay; the k largest c of their experts are chosen (ties: lower index)
//   w_j = scale s_j / sum_chosen s, or scale s_j
//
// Scores are float64: neighbouring experts differ by less than a float32 rounding
// often enough (one token in a few thousand at E = 256) that float32 scores would
// make the choice depend on the order of the arithmetic.
#include "common.h"

namespace {

using namespace qd;

constexpr int RS_EMAX = 1024;
constexpr int RS_KMAX = 32;
constexpr int RS_GMAX = 64;
constexpr int RS_BLK = 256;            // tokens of a ranking block

struct ScoreArgs {
  const void *logits;
  int64_t ld;
  int64_t T;
  int E, k;
  int scoring;
  const float *bias;
  int G, top_groups, group_sum;
  int renorm;
  float scale;
  const uint8_t *live;
  int32_t *ids;
  float *wts;
};

template <typename L>
__device__ __forceinline__ float rs_load(const void *p, int64_t i);
template <>
__device__ __forceinline__ float rs_load<float>(const void *p, int64_t i) {
  return static_cast<const float *>(p)[i];
}
template <>
__device__ __forceinline__ float rs_load<uint16_t>(const void *p, int64_t i) {
  return bf16_bits_to_f32(static_cast<const uint16_t *>(p)[i]);
}

__device__ __forceinline__ double rs_sigmoid(float x) { return 1.0 / (1.0 + exp(-(double)x)); }

// larger key: earlier slot; NaN below every number, -0 as +0, 0 is no key
__device__ __forceinline__ uint64_t rs_key(double v) {
  if (v != v) return 1ull;
  const uint64_t b = (uint64_t)__double_as_longlong(v + 0.0);
  return (b >> 63) ? ~b : (b | 0x8000000000000000ull);
}
__device__ __forceinline__ uint64_t rs_wave_max(uint64_t m) {
  for (int o = 32; o > 0; o >>= 1) {
    const uint64_t x = ((uint64_t)(uint32_t)__shfl_xor((int)(uint32_t)(m >> 32), o, 64) << 32) |
                       (uint32_t)__shfl_xor((int)(uint32_t)m, o, 64);
    m = x > m ? x : m;
  }
  return m;
}
__device__ __forceinline__ double rs_lane(double v, int lane) {
  const uint64_t b = (uint64_t)__double_as_longlong(v);
  const uint32_t lo = (uint32_t)__builtin_amdgcn_readlane((int)(uint32_t)b, lane);
  const uint32_t hi = (uint32_t)__builtin_amdgcn_readlane((int)(uint32_t)(b >> 32), lane);
  return __longlong_as_double((long long)(((uint64_t)hi << 32) | lo));
}
__device__ __forceinline__ double rs_wave_sum(double v) {
  for (int o = 32; o > 0; o >>= 1) v += __shfl_xor(v, o, 64);
  return v;
}

// One wavefront per token; lane l holds experts l, l + 64, ...
template <typename L, int PER>
__global__ __launch_bounds__(256) void score_topk_kernel(ScoreArgs p) {
  extern __shared__ __align__(16) unsigned char rs_lds[];
  const int lane = threadIdx.x & 63, wid = threadIdx.x >> 6;
  const int64_t t = (int64_t)blockIdx.x * 4 + wid;
  if (t >= p.T) return;                          // whole wave; no barriers below
  const int E = p.E, k = p.k;
  if (p.live && !p.live[t]) {
    if (lane < k) {
      p.ids[t * k + lane] = -1;
      p.wts[t * k + lane] = 0.0f;
    }
    return;
  }
  float x[PER];
  double s[PER];
  uint64_t key[PER];
#pragma unroll
  for (int j = 0; j < PER; ++j) {
    const int e = lane + 64 * j;
    x[j] = e < E ? rs_load<L>(p.logits, t * p.ld + e) : -INFINITY;
  }
  if (p.scoring == QD_SCORE_SIGMOID) {
#pragma unroll
    for (int j = 0; j < PER; ++j) s[j] = rs_sigmoid(x[j]);
  } else {
    float m = x[0];
#pragma unroll
    for (int j = 1; j < PER; ++j) m = fmaxf(m, x[j]);
    m = wave_max(m);
    double z = 0.0;
#pragma unroll
    for (int j = 0; j < PER; ++j) {
      s[j] = m == -INFINITY ? 0.0 : exp((double)x[j] - (double)m);
      if (lane + 64 * j < E) z += s[j];
    }
    z = rs_wave_sum(z);
#pragma unroll
    for (int j = 0; j < PER; ++j) s[j] = m == -INFINITY ? 0.0 : s[j] / z;
  }
  const bool by_logit = !p.bias && p.G == 1;
  double c[PER];
#pragma unroll
  for (int j = 0; j < PER; ++j) {
    const int e = lane + 64 * j;
    c[j] = by_logit ? (double)x[j] : s[j] + (p.bias && e < E ? (double)p.bias[e] : 0.0);
    key[j] = e < E ? rs_key(c[j]) : 0ull;
  }
  if (p.G > 1) {
    uint64_t *ck = reinterpret_cast<uint64_t *>(rs_lds) + (size_t)wid * E;
    const int n = E / p.G;
#pragma unroll
    for (int j = 0; j < PER; ++j)
      if (lane + 64 * j < E) ck[lane + 64 * j] = key[j];
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
    __builtin_amdgcn_wave_barrier();
    uint64_t gk = 0;
    if (lane < p.G) {
      uint64_t a = 0, b = 0;                     // the two largest
      for (int i = 0; i < n; ++i) {
        const uint64_t v = ck[lane * n + i];
        if (v > a) { b = a; a = v; }
        else if (v > b) b = v;
      }
      auto val = [](uint64_t q) -> double {
        if (q <= 1) return __longlong_as_double(0x7ff8000000000000ll);
        const uint64_t u = (q >> 63) ? q & 0x7fffffffffffffffull : ~q;
        return __longlong_as_double((long long)u);
      };
      gk = rs_key(p.group_sum == 2 ? val(a) + val(b) : val(a));
    }
    int rank = 0;
    for (int g = 0; g < p.G; ++g) {
      const uint64_t o = ((uint64_t)(uint32_t)__builtin_amdgcn_readlane((int)(uint32_t)(gk >> 32), g) << 32) |
                         (uint32_t)__builtin_amdgcn_readlane((int)(uint32_t)gk, g);
      rank += o > gk || (o == gk && g < lane) ? 1 : 0;
    }
    const uint64_t kept = __ballot(lane < p.G && rank < p.top_groups);
#pragma unroll
    for (int j = 0; j < PER; ++j) {
      const int e = lane + 64 * j;
      if (e < E && !((kept >> (e / n)) & 1ull)) key[j] = 0ull;
    }
  }
  // k rounds: the largest key, the lowest expert that has it
  int my_e = 0;
  double my_s = 0.0;
  float my_x = 0.0f;
  for (int r = 0; r < k; ++r) {
    uint64_t m = key[0];
#pragma unroll
    for (int j = 1; j < PER; ++j) m = key[j] > m ? key[j] : m;
    m = rs_wave_max(m);
    bool found = false;
#pragma unroll
    for (int j = 0; j < PER; ++j) {
      const uint64_t b = __ballot(key[j] == m);
      if (!found && b) {
        found = true;
        const int l = __ffsll((long long)b) - 1;
        const double sv = rs_lane(s[j], l);
        const float xv = __int_as_float(__builtin_amdgcn_readlane(__float_as_int(x[j]), l));
        if (lane == r) {
          my_e = l + 64 * j;
          my_s = sv;
          my_x = xv;
        }
        if (lane == l) key[j] = 0ull;
      }
    }
  }
  double w;
  if (p.renorm) {
    if (p.scoring == QD_SCORE_SOFTMAX) {         // softmax over the chosen
      const float top = wave_max(lane < k ? my_x : -INFINITY);
      my_s = top == -INFINITY ? 0.0 : exp((double)my_x - (double)top);
    }
    const double n = rs_wave_sum(lane < k ? my_s : 0.0);
    w = n == 0.0 ? 0.0 : (double)p.scale * my_s / n;
  } else {
    w = (double)p.scale * my_s;
  }
  if (lane < k) {
    p.ids[t * k + lane] = my_e;
    p.wts[t * k + lane] = (float)w;
  }
}

// ---------------------------------------------------------------- permutation
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
  for (int i = tl; i < E * (RS_BLK / 32); i += RS_BLK) (&mask[0][0])[i] = 0u;
  __syncthreads();
  if (t < T)
    for (int s = 0; s < k; ++s) {
      const int e = ids[t * k + s];
      if (e >= 0) atomicOr(&mask[e][tl >> 5], 1u << (tl & 31));
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
  if (t < T)
    for (int s = 0; s < k; ++s) {
      const int e = ids[t * k + s];
      if (e >= 0)
        ranks[t * k + s] =
            (int)before[e][tl >> 5] + __popc(mask[e][tl >> 5] & ((1u << (tl & 31)) - 1u));
    }
}

__global__ __launch_bounds__(RS_BLK) void score_scatter_kernel(
    int64_t T, int E, int k, int nblk, const int32_t *__restrict__ ids,
    const int32_t *__restrict__ counts, const int32_t *__restrict__ ranks,
    int32_t *__restrict__ offsets, int32_t *__restrict__ row_token,
    int32_t *__restrict__ inv_row) {
  __shared__ int32_t base[RS_EMAX], total[RS_EMAX];
  __shared__ int wsum[4];
  const int tid = threadIdx.x, lane = tid & 63, wid = tid >> 6, b = blockIdx.x;
  for (int e = tid; e < E; e += RS_BLK) {
    int tot = 0, pre = 0;
    for (int q = 0; q < nblk; ++q) {
      const int c = counts[(int64_t)q * E + e];
      tot += c;
      if (q < b) pre += c;
    }
    total[e] = tot;
    base[e] = pre;
  }
  __syncthreads();
  int c[4], tsum = 0;
#pragma unroll
  for (int q = 0; q < 4; ++q) {
    const int e = 4 * tid + q;
    c[q] = e < E ? total[e] : 0;
    tsum += c[q];
  }
  int xs = tsum;
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) {
    const int y = __shfl_up(xs, o, 64);
    if (lane >= o) xs += y;
  }
  if (lane == 63) wsum[wid] = xs;
  __syncthreads();
  int ex = xs - tsum;
  for (int ww = 0; ww < wid; ++ww) ex += wsum[ww];
#pragma unroll
  for (int q = 0; q < 4; ++q) {
    const int e = 4 * tid + q;
    if (e < E) {
      base[e] += ex;
      if (b == 0) offsets[e] = ex;
    }
    ex += c[q];
  }
  const int rows = wsum[0] + wsum[1] + wsum[2] + wsum[3];
  if (tid == 0 && b == 0) offsets[E] = rows;
  __syncthreads();
  const int64_t t = (int64_t)b * RS_BLK + tid;
  if (t < T)
    for (int s = 0; s < k; ++s) {
      const int e = ids[t * k + s];
      int row = -1;
      if (e >= 0) {
        row = base[e] + ranks[t * k + s];
        row_token[row] = (int32_t)t;
      }
      inv_row[t * k + s] = row;
      if (t * k + s >= rows) row_token[t * k + s] = -1;    // rows behind the last
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
template <>
__device__ __forceinline__ void rs_store<uint16_t>(void *p, int64_t i, double v) {
  static_cast<__bf16 *>(p)[i] = (__bf16)(float)v;
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
  const bool full = p.scoring == QD_SCORE_SOFTMAX && !p.renorm;
  double d = 0.0;                 // this lane's chosen expert's gradient
  double dot = 0.0, z = 1.0;
  float m = 0.0f;
  float x[PER];
  if (full) {
#pragma unroll
    for (int j = 0; j < PER; ++j) {
      const int e = lane + 64 * j;
      x[j] = e < E ? rs_load<L>(p.logits, t * p.ld + e) : -INFINITY;
    }
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
  } else if (p.scoring == QD_SCORE_SOFTMAX) {
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
    if (full && m != -INFINITY) v = -exp((double)x[j] - (double)m) / z * dot;
    for (int q = 0; q < k; ++q) {
      const int eq = __builtin_amdgcn_readlane(id, q);
      const double dq = rs_lane(d, q);
      if (eq == e) v = dq;
    }
    if (e < E) rs_store<L>(p.grad, t * p.ldg + e, v);
  }
}

template <typename F>
bool rs_by_width(int E, F f) {
  const int per = (E + 63) / 64;
  if (per <= 1) f(std::integral_constant<int, 1>{});
  else if (per == 2) f(std::integral_constant<int, 2>{});
  else if (per == 3) f(std::integral_constant<int, 3>{});
  else if (per == 4) f(std::integral_constant<int, 4>{});
  else if (per <= 8) f(std::integral_constant<int, 8>{});
  else f(std::integral_constant<int, 16>{});
  return true;
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
  const int64_t nblk = T > 0 ? (T + RS_BLK - 1) / RS_BLK : 1;
  return qdh::align_up((size_t)nblk * (E > 0 ? E : 1) * 4) +
         qdh::align_up((size_t)(T > 0 ? T : 1) * (k > 0 ? k : 1) * 4);
}

extern "C" qd_status moe_route_scored_permute(
    const void *logits, int32_t dtype, int64_t ld, int64_t T, int32_t E, int32_t k,
    int32_t scoring, const float *bias, int32_t groups, int32_t top_groups, int32_t group_sum,
    int32_t renorm, float scale, const uint8_t *live, int32_t *topk_ids, float *topk_w,
    int32_t *expert_offsets, int32_t *row_token, int32_t *inv_row, void *ws, size_t ws_bytes,
    void *stream) {
  const qd_status bad = check_scoring(dtype, ld, T, E, k, scoring, renorm);
  if (bad) return bad;
  if (groups < 1 || groups > RS_GMAX || E % groups != 0 || top_groups < 1 || top_groups > groups ||
      (group_sum != 1 && group_sum != 2) || (groups > 1 && group_sum > E / groups) ||
      (int64_t)top_groups * (E / groups) < k || !(scale - scale == 0.0f))
    return QD_ERR_SHAPE;
  if (!expert_offsets) return QD_ERR_NULL;
  if (T > 0 && (!logits || !topk_ids || !topk_w || !row_token || !inv_row)) return QD_ERR_NULL;
  if (!ws || ws_bytes < moe_route_scored_workspace(T, E, k)) return QD_ERR_WORKSPACE;
  if (!qdh::aligned16(logits) || !qdh::aligned16(bias) || !qdh::aligned16(topk_ids) ||
      !qdh::aligned16(topk_w) || !qdh::aligned16(expert_offsets) || !qdh::aligned16(row_token) ||
      !qdh::aligned16(inv_row) || !qdh::aligned16(ws))
    return QD_ERR_ALIGN;   // (NULL is aligned)
  if (qdh::fault_injected()) return QD_ERR_HIP;
  hipStream_t s = qdh::S(stream);
  if (T == 0) {
    qdi::launch_fill_i32(expert_offsets, E + 1, 0, s);
    return qdh::check_launch();
  }
  ScoreArgs p{logits, ld, T, E, k, scoring, bias, groups, top_groups, group_sum,
              renorm, scale, live, topk_ids, topk_w};
  const dim3 grid((unsigned)((T + 3) / 4)), block(256);
  const size_t lds = groups > 1 ? (size_t)4 * E * 8 : 0;
  rs_by_width(E, [&](auto per) {
    constexpr int PER = decltype(per)::value;
    if (dtype == QD_DTYPE_BF16)
      hipLaunchKernelGGL((score_topk_kernel<uint16_t, PER>), grid, block, lds, s, p);
    else
      hipLaunchKernelGGL((score_topk_kernel<float, PER>), grid, block, lds, s, p);
  });
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
  if (qdh::fault_injected()) return QD_ERR_HIP;
  hipStream_t s = qdh::S(stream);
  ScoreGradArgs p{logits, ld, T, E, k, scoring, renorm, scale, topk_ids, grad_w, grad_logits, ld_grad};
  const dim3 grid((unsigned)((T + 3) / 4)), block(256);
  rs_by_width(E, [&](auto per) {
    constexpr int PER = decltype(per)::value;
    if (dtype == QD_DTYPE_BF16)
      hipLaunchKernelGGL((score_grad_kernel<uint16_t, PER>), grid, block, 0, s, p);
    else
      hipLaunchKernelGGL((score_grad_kernel<float, PER>), grid, block, 0, s, p);
  });
  return qdh::check_launch();
}
