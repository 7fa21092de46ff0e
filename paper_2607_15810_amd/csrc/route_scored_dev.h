// Scored routing of the MoE layer: softmax or sigmoid scores, a bias that enters
// the choice only (balance), expert groups, renormalised and scaled weights,
// padded batches.
//
//   s = sigmoid(l) or softmax(l), c = s + bias
//   group score = sum of the group_sum largest c of a group; the top_groups best
//   groups stay; the k largest c of their experts are chosen (ties: lower index)
//   w_j = scale s_j / sum_chosen s, or scale s_j
//
// The choice is that of float64 scores: neighbouring experts differ by less than a
// float32 rounding often enough that float32 scores would make it depend on the order
// of the arithmetic.  One wavefront takes a token.  It first chooses with float32
// scores, whose error is bounded (rs_gap), and keeps that choice where every comparison
// that decided it has a wider gap; otherwise it chooses again in float64.  Of normal float32
// logits that is one token in 200 to 1000; in groups without a bias, bf16 logits send 20 to 30%
// there (equal ones are common, and an exact tie is no gap).  Without bias and groups the
// logits themselves are compared, exactly; a choice by scores takes two logits whose float64
// scores are equal (sigmoids from 37 on) as a tie.
#pragma once
#include <type_traits>

#include "common.h"

namespace qds {

using namespace qd;

constexpr int RS_EMAX = 1024;
constexpr int RS_KMAX = 32;
constexpr int RS_GMAX = 64;

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
__device__ __forceinline__ uint32_t rs_key(float v) {
  if (v != v) return 1u;
  const uint32_t b = __float_as_uint(v + 0.0f);
  return (b >> 31) ? ~b : (b | 0x80000000u);
}
__device__ __forceinline__ float rs_value(uint32_t key) {
  return __uint_as_float((key >> 31) ? key & 0x7fffffffu : ~key);
}

// v of the lane that DPP control C names
template <int C>
__device__ __forceinline__ uint32_t rs_dpp(uint32_t v) {
  return (uint32_t)__builtin_amdgcn_mov_dpp((int)v, C, 0xF, 0xF, false);
}
template <int C>
__device__ __forceinline__ float rs_dppf(float v) {
  return __uint_as_float(rs_dpp<C>(__float_as_uint(v)));
}
// within 16 lanes: lanes 1, 2, 4, 8 apart (the last two between values that the smaller
// sets of lanes share already)
constexpr int DPP_X1 = 0xB1, DPP_X2 = 0x4E, DPP_X4 = 0x141, DPP_X8 = 0x140;

__device__ __forceinline__ uint32_t rs_umax(uint32_t a, uint32_t b) { return a > b ? a : b; }
// the largest of 64 lanes, in every lane
__device__ __forceinline__ uint32_t rs_wave_umax(uint32_t m) {
  m = rs_umax(m, rs_dpp<DPP_X1>(m));
  m = rs_umax(m, rs_dpp<DPP_X2>(m));
  m = rs_umax(m, rs_dpp<DPP_X4>(m));
  m = rs_umax(m, rs_dpp<DPP_X8>(m));
  const uint32_t a = (uint32_t)__builtin_amdgcn_readlane((int)m, 0);
  const uint32_t b = (uint32_t)__builtin_amdgcn_readlane((int)m, 16);
  const uint32_t c = (uint32_t)__builtin_amdgcn_readlane((int)m, 32);
  const uint32_t d = (uint32_t)__builtin_amdgcn_readlane((int)m, 48);
  return rs_umax(rs_umax(a, b), rs_umax(c, d));
}
__device__ __forceinline__ float rs_lanef(float v, int lane) {
  return __int_as_float(__builtin_amdgcn_readlane(__float_as_int(v), lane));
}
__device__ __forceinline__ float rs_wave_fmax(float m) {
  m = fmaxf(m, rs_dppf<DPP_X1>(m));
  m = fmaxf(m, rs_dppf<DPP_X2>(m));
  m = fmaxf(m, rs_dppf<DPP_X4>(m));
  m = fmaxf(m, rs_dppf<DPP_X8>(m));
  return fmaxf(fmaxf(rs_lanef(m, 0), rs_lanef(m, 16)), fmaxf(rs_lanef(m, 32), rs_lanef(m, 48)));
}
__device__ __forceinline__ float rs_wave_fsum(float m) {
  m += rs_dppf<DPP_X1>(m);
  m += rs_dppf<DPP_X2>(m);
  m += rs_dppf<DPP_X4>(m);
  m += rs_dppf<DPP_X8>(m);
  return (rs_lanef(m, 0) + rs_lanef(m, 16)) + (rs_lanef(m, 32) + rs_lanef(m, 48));
}
template <int C>
__device__ __forceinline__ uint64_t rs_dpp64(uint64_t v) {
  return ((uint64_t)rs_dpp<C>((uint32_t)(v >> 32)) << 32) | rs_dpp<C>((uint32_t)v);
}
template <int C>
__device__ __forceinline__ double rs_dppd(double v) {
  return __longlong_as_double((long long)rs_dpp64<C>((uint64_t)__double_as_longlong(v)));
}
__device__ __forceinline__ double rs_lane(double v, int lane) {
  const uint64_t b = (uint64_t)__double_as_longlong(v);
  const uint32_t lo = (uint32_t)__builtin_amdgcn_readlane((int)(uint32_t)b, lane);
  const uint32_t hi = (uint32_t)__builtin_amdgcn_readlane((int)(uint32_t)(b >> 32), lane);
  return __longlong_as_double((long long)(((uint64_t)hi << 32) | lo));
}
__device__ __forceinline__ uint64_t rs_lane64(uint64_t v, int lane) {
  return (uint64_t)__double_as_longlong(rs_lane(__longlong_as_double((long long)v), lane));
}
__device__ __forceinline__ uint64_t rs_umax64(uint64_t a, uint64_t b) { return a > b ? a : b; }
__device__ __forceinline__ uint64_t rs_wave_max64(uint64_t m) {
  m = rs_umax64(m, rs_dpp64<DPP_X1>(m));
  m = rs_umax64(m, rs_dpp64<DPP_X2>(m));
  m = rs_umax64(m, rs_dpp64<DPP_X4>(m));
  m = rs_umax64(m, rs_dpp64<DPP_X8>(m));
  return rs_umax64(rs_umax64(rs_lane64(m, 0), rs_lane64(m, 16)),
                   rs_umax64(rs_lane64(m, 32), rs_lane64(m, 48)));
}
__device__ __forceinline__ double rs_wave_sum(double v) {
  v += rs_dppd<DPP_X1>(v);
  v += rs_dppd<DPP_X2>(v);
  v += rs_dppd<DPP_X4>(v);
  v += rs_dppd<DPP_X8>(v);
  return (rs_lane(v, 0) + rs_lane(v, 16)) + (rs_lane(v, 32) + rs_lane(v, 48));
}

// Experts per lane: contiguous, E / 64 rounded up, or more where that makes a group a
// power of two of whole lanes; 0 where nothing up to 8 does.
inline int rs_per(int E, int G) {
  const int n = E / G, least = (E + 63) / 64;
  if (G == 1) return least;
  for (int per = least; per <= 8; ++per) {
    const int q = n / per;
    if (n % per == 0 && (q & (q - 1)) == 0) return per;
  }
  return 0;
}

// The lanes' shares: per experts each, 2^lq lanes a group (lq < 0: groups of no whole
// lanes, whose choice is made in float64 with the groups' sums through LDS).
struct ScoreLanes {
  int per, lq;
};
inline ScoreLanes rs_lanes(int E, int G) {
  const int per = rs_per(E, G);
  if (per == 0) return {(E + 63) / 64, -1};
  int lq = 0;
  while (G > 1 && (per << lq) < E / G) ++lq;
  return {per, lq};
}

// The gap beyond which two float32 values, the larger of size v, compare as their
// float64 originals do.  In units of 2^-24: a sigmoid is off by 0.5 (exp2) + 0.4 (its
// argument) + 3 (1 + e and the reciprocal), a softmax score by its argument's rounding
// (1.1: s |ln s| < 0.37) and, of itself, by 24 (exp2, the sum with at most 20 roundings on
// the way to any term at E <= 1024, the reciprocal); the bias adds |c|.  So two sigmoids
// are off by 8 + 2 |c|, two softmax scores, 1 together at most, by 27 + 2 |c|; allowed are
// 32 (1 + |c|).  A group's sum of two scores doubles either: 64 (1 + the larger |a| + |b|).
__device__ __forceinline__ float rs_gap(float v, bool group) {
  return (1.0f + fabsf(v)) * (group ? 3.8146973e-06f : 1.9073486e-06f);   // 2^-18, 2^-19
}

// The token's choice in float64: lane r gets expert r in my_e and its logit in my_x.  ck: E
// keys of LDS, this wave's own (G > 1).
template <int PER>
__device__ __forceinline__ void rs_choose_exact(const ScoreArgs &p, ScoreLanes sl,
                                                const float (&x)[PER], const float (&bias)[PER],
                                                uint64_t *ck, int &my_e, float &my_x) {
  const int lane = threadIdx.x & 63, E = p.E, per = sl.per;
  double s[PER];
  uint64_t key[PER];
  if (p.scoring == QD_SCORE_SIGMOID) {
#pragma unroll
    for (int j = 0; j < PER; ++j) s[j] = rs_sigmoid(x[j]);
  } else {
    float m = x[0];
#pragma unroll
    for (int j = 1; j < PER; ++j) m = fmaxf(m, x[j]);
    m = rs_wave_fmax(m);
    double z = 0.0;
    // over the numbers: a NaN keeps its place, and of +inf logits each has the same share
#pragma unroll
    for (int j = 0; j < PER; ++j) {
      s[j] = x[j] == m ? 1.0 : exp((double)x[j] - (double)m);
      if (m == -INFINITY) s[j] = 0.0;
      if (x[j] != x[j]) s[j] = x[j];
      else if (j < per && lane * per + j < E) z += s[j];
    }
    z = rs_wave_sum(z);
#pragma unroll
    for (int j = 0; j < PER; ++j) s[j] = m == -INFINITY ? s[j] : s[j] / z;
  }
#pragma unroll
  for (int j = 0; j < PER; ++j) {
    const int e = lane * per + j;
    const bool in = j < per && e < E;
    key[j] = in ? rs_key(s[j] + (double)bias[j]) : 0ull;
  }
  if (p.G > 1) {
    auto val = [](uint64_t q) -> double {
      if (q <= 1) return __longlong_as_double(0x7ff8000000000000ll);
      const uint64_t u = (q >> 63) ? q & 0x7fffffffffffffffull : ~q;
      return __longlong_as_double((long long)u);
    };
    // a, b: the two largest keys of this lane's group (lq >= 0), of group `lane` (lq < 0)
    uint64_t a = 0, b = 0;
    auto add = [&](uint64_t v) __attribute__((always_inline)) {
      b = rs_umax64(b, v < a ? v : a);
      a = rs_umax64(a, v);
    };
    if (sl.lq >= 0) {
#pragma unroll
      for (int j = 0; j < PER; ++j) add(key[j]);
      auto merge = [&](uint64_t a2, uint64_t b2) __attribute__((always_inline)) {
        add(a2);
        b = rs_umax64(b, b2);
      };
      if (sl.lq > 0) merge(rs_dpp64<DPP_X1>(a), rs_dpp64<DPP_X1>(b));
      if (sl.lq > 1) merge(rs_dpp64<DPP_X2>(a), rs_dpp64<DPP_X2>(b));
      if (sl.lq > 2) merge(rs_dpp64<DPP_X4>(a), rs_dpp64<DPP_X4>(b));
      if (sl.lq > 3) merge(rs_dpp64<DPP_X8>(a), rs_dpp64<DPP_X8>(b));
      if (sl.lq > 4) merge(__shfl_xor(a, 16, 64), __shfl_xor(b, 16, 64));
    } else {
      const int n = E / p.G;
#pragma unroll
      for (int j = 0; j < PER; ++j)
        if (j < per && lane * per + j < E) ck[lane * per + j] = key[j];
      __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
      __builtin_amdgcn_wave_barrier();
      if (lane < p.G)
        for (int i = 0; i < n; ++i) add(ck[lane * n + i]);
      // the reads are done before a later token's keys are written
      __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
      __builtin_amdgcn_wave_barrier();
    }
    const int lq = sl.lq >= 0 ? sl.lq : 0, mine = lane >> lq;
    const uint64_t gk = mine < p.G ? rs_key(p.group_sum == 2 ? val(a) + val(b) : val(a)) : 0ull;
    int rank = 0;
    for (int g = 0; g < p.G; ++g) {
      const uint64_t o = rs_lane64(gk, g << lq);
      rank += o > gk || (o == gk && g < mine) ? 1 : 0;
    }
    const bool kept = rank < p.top_groups;       // this lane's group
    const uint64_t kb = __ballot(kept);
#pragma unroll
    for (int j = 0; j < PER; ++j) {
      const bool k1 = sl.lq >= 0 ? kept : (kb >> min((lane * per + j) / (E / p.G), 63)) & 1ull;
      if (!k1) key[j] = 0ull;
    }
  }
  for (int r = 0; r < p.k; ++r) {
    uint64_t m = key[0];
#pragma unroll
    for (int j = 1; j < PER; ++j) m = key[j] > m ? key[j] : m;
    const uint64_t top = rs_wave_max64(m);
    const int l = __ffsll((long long)__ballot(m == top)) - 1;
    int js = 0;
    float xv = x[0];
#pragma unroll
    for (int j = PER - 1; j >= 0; --j)
      if (key[j] == top) {
        js = j;
        xv = x[j];
      }
    const int e = l * per + __builtin_amdgcn_readlane(js, l);
    const float xs = rs_lanef(xv, l);
    if (lane == r) {
      my_e = e;
      my_x = xs;
    }
#pragma unroll
    for (int j = 0; j < PER; ++j)
      if (lane == l && j == js) key[j] = 0ull;
  }
}

// One wavefront, token t: ids and weights.  Lane l holds experts l per .. l per + per - 1;
// ids_lds: NULL, or where in LDS the ids go as well.
template <typename L, int PER>
__device__ __forceinline__ void rs_token(const ScoreArgs &p, ScoreLanes sl, int64_t t,
                                         uint64_t *ck, int32_t *ids_lds) {
  const int lane = threadIdx.x & 63, E = p.E, k = p.k, per = sl.per;
  if (p.live && !p.live[t]) {
    if (lane < k) {
      p.ids[t * k + lane] = -1;
      p.wts[t * k + lane] = 0.0f;
      if (ids_lds) ids_lds[lane] = -1;
    }
    return;
  }
  float x[PER], c[PER], bias[PER];
  uint32_t key[PER];
#pragma unroll
  for (int j = 0; j < PER; ++j) {                // loads in bounds, unpredicated
    const int e = lane * per + j;
    const bool in = j < per && e < E;
    const float v = rs_load<L>(p.logits, t * p.ld + (in ? e : 0));
    bias[j] = p.bias ? p.bias[in ? e : 0] : 0.0f;
    x[j] = in ? v : -INFINITY;
  }
  float mx = 0.0f;
  if (p.scoring == QD_SCORE_SOFTMAX) {
    mx = x[0];
#pragma unroll
    for (int j = 1; j < PER; ++j) mx = fmaxf(mx, x[j]);
    mx = rs_wave_fmax(mx);
  }
  const bool by_logit = !p.bias && p.G == 1;
  // softmax: a NaN or +inf logit, chosen or not, leaves no score of the token a number.  Its
  // weights are NaN; the choice is made over what is left (rs_choose_exact).
  bool broken = false;
  if (p.scoring == QD_SCORE_SOFTMAX) {
#pragma unroll
    for (int j = 0; j < PER; ++j) broken |= !(x[j] < INFINITY);
    broken = __ballot(broken) != 0ull;
  }
  constexpr float LOG2E = 1.4426950408889634f;
  if (by_logit) {
#pragma unroll
    for (int j = 0; j < PER; ++j) c[j] = x[j];
  } else {
    if (p.scoring == QD_SCORE_SIGMOID) {
#pragma unroll
      for (int j = 0; j < PER; ++j)
        c[j] = __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(-x[j] * LOG2E));
    } else {
      float z = 0.0f;
#pragma unroll
      for (int j = 0; j < PER; ++j) {
        c[j] = mx == -INFINITY ? 0.0f : __builtin_amdgcn_exp2f((x[j] - mx) * LOG2E);
        z += c[j];                               // 0 past the last expert
      }
      z = rs_wave_fsum(z);
      const float rz = mx == -INFINITY ? 0.0f : __builtin_amdgcn_rcpf(z);
#pragma unroll
      for (int j = 0; j < PER; ++j) c[j] *= rz;
    }
#pragma unroll
    for (int j = 0; j < PER; ++j) c[j] += bias[j];
  }
#pragma unroll
  for (int j = 0; j < PER; ++j) key[j] = j < per && lane * per + j < E ? rs_key(c[j]) : 0u;
  bool sure = sl.lq >= 0 && (by_logit || !broken);   // uniform
  if (p.G > 1 && sure) {
    float a = -INFINITY, b = -INFINITY;          // the group's two largest
    bool nan = false;
#pragma unroll
    for (int j = 0; j < PER; ++j)
      if (key[j] != 0u) {
        nan |= key[j] == 1u;
        const float v = c[j];
        b = fmaxf(b, fminf(a, v));
        a = fmaxf(a, v);
      }
    auto merge = [&](float a2, float b2) __attribute__((always_inline)) {
      b = fmaxf(fminf(a, a2), fmaxf(b, b2));
      a = fmaxf(a, a2);
    };
    if (sl.lq > 0) merge(rs_dppf<DPP_X1>(a), rs_dppf<DPP_X1>(b));
    if (sl.lq > 1) merge(rs_dppf<DPP_X2>(a), rs_dppf<DPP_X2>(b));
    if (sl.lq > 2) merge(rs_dppf<DPP_X4>(a), rs_dppf<DPP_X4>(b));
    if (sl.lq > 3) merge(rs_dppf<DPP_X8>(a), rs_dppf<DPP_X8>(b));
    if (sl.lq > 4) merge(__shfl_xor(a, 16, 64), __shfl_xor(b, 16, 64));
    const float gs = p.group_sum == 2 ? a + b : a;
    const int mine = lane >> sl.lq;
    const bool in = mine < p.G;
    const float size = p.group_sum == 2 ? fabsf(a) + fabsf(b) : fabsf(a);
    const float gap = rs_gap(rs_wave_fmax(in ? size : 0.0f), true);
    // groups surely above this one, and groups that may be
    int above = 0, maybe = 0;
    for (int g = 0; g < p.G; ++g) {
      const float o = rs_lanef(gs, g << sl.lq);
      if (g != mine) {
        above += o > gs + gap ? 1 : 0;
        maybe += o >= gs - gap ? 1 : 0;
      }
    }
    sure = __ballot(in && (nan || !(gs - gs == 0.0f) ||
                           (above < p.top_groups) != (maybe < p.top_groups))) == 0ull;
    if (in && maybe >= p.top_groups) {
#pragma unroll
      for (int j = 0; j < PER; ++j) key[j] = 0u;
    }
  }
  int my_e = 0;
  float my_x = 0.0f;
  if (sure) {
    // k rounds of the largest key (one more where values are rounded: the first expert
    // left out decides too whether the last is sure).  A lane holds its keys in
    // descending order, equal ones in that of the experts, up to four; more are
    // searched.
    int ex[PER];
#pragma unroll
    for (int j = 0; j < PER; ++j) ex[j] = lane * per + j;
    if constexpr (PER <= 4) {
#pragma unroll
      for (int i = 0; i + 1 < PER; ++i)
#pragma unroll
        for (int j = 0; j + 1 < PER - i; ++j) {
          const bool sw = key[j + 1] > key[j];
          const uint32_t kk = key[j];
          const int ee = ex[j];
          key[j] = sw ? key[j + 1] : key[j];
          key[j + 1] = sw ? kk : key[j + 1];
          ex[j] = sw ? ex[j + 1] : ex[j];
          ex[j + 1] = sw ? ee : ex[j + 1];
        }
    }
    uint32_t m = key[0], my_key = 0u;
    if constexpr (PER > 4) {
#pragma unroll
      for (int j = 1; j < PER; ++j) m = rs_umax(m, key[j]);
    }
    const int rounds = by_logit ? k : k + 1;
    for (int r = 0; r < rounds; ++r) {
      const uint32_t top = rs_wave_umax(m);
      const int l = __ffsll((long long)__ballot(m == top)) - 1;
      int js = 0;
      if constexpr (PER > 4) {
#pragma unroll
        for (int j = PER - 1; j >= 0; --j)
          if (key[j] == top) js = j;
      }
      const int e = PER > 4 ? l * per + __builtin_amdgcn_readlane(js, l)
                            : __builtin_amdgcn_readlane(ex[0], l);
      if (lane == r) {
        my_e = e;
        my_key = top;
      }
      if (lane == l) {
        if constexpr (PER > 4) {
          m = 0u;
#pragma unroll
          for (int j = 0; j < PER; ++j) {
            if (j == js) key[j] = 0u;
            m = rs_umax(m, key[j]);
          }
        } else {
#pragma unroll
          for (int j = 0; j + 1 < PER; ++j) {
            key[j] = key[j + 1];
            ex[j] = ex[j + 1];
          }
          key[PER - 1] = 0u;
          m = key[0];
        }
      }
    }
    if (!by_logit) {
      // (key 0: no expert left, nothing to mistake the last one for)
      const uint32_t nk = (uint32_t)__shfl_down((int)my_key, 1, 64);
      const float v = rs_value(my_key), n = rs_value(nk);
      sure = __ballot(lane < k && nk != 0u && !(v - n > rs_gap(v, false))) == 0ull;
    }
    if (sure && lane < k) my_x = rs_load<L>(p.logits, t * p.ld + my_e);
  }
  if (!sure) rs_choose_exact<PER>(p, sl, x, bias, ck, my_e, my_x);
  // weights, in float64 from the chosen logits
  double s = 0.0;
  if (p.scoring == QD_SCORE_SIGMOID) {
    if (lane < k) s = rs_sigmoid(my_x);
  } else if (p.renorm) {                         // softmax over the chosen
    const float top = wave_max(lane < k ? my_x : -INFINITY);
    if (lane < k && top != -INFINITY) s = exp((double)my_x - (double)top);
  } else {
    double z = 0.0;
#pragma unroll
    for (int j = 0; j < PER; ++j)
      if (j < per && lane * per + j < E && mx != -INFINITY) z += exp((double)x[j] - (double)mx);
    z = rs_wave_sum(z);
    if (lane < k && mx != -INFINITY) s = exp((double)my_x - (double)mx) / z;
  }
  double w = (double)p.scale * s;
  if (p.renorm) {
    const double n = rs_wave_sum(s);
    w = n == 0.0 ? 0.0 : w / n;
  }
  if (broken) w = __longlong_as_double(0x7ff8000000000000ll);
  if (lane < k) {
    p.ids[t * k + lane] = my_e;
    p.wts[t * k + lane] = (float)w;
    if (ids_lds) ids_lds[lane] = my_e;
  }
}

// f(PER) for a compiled width that holds `per` experts a lane
template <typename F>
inline void rs_by_width(int per, F f) {
  if (per <= 1) f(std::integral_constant<int, 1>{});
  else if (per == 2) f(std::integral_constant<int, 2>{});
  else if (per == 3) f(std::integral_constant<int, 3>{});
  else if (per == 4) f(std::integral_constant<int, 4>{});
  else if (per <= 8) f(std::integral_constant<int, 8>{});
  else f(std::integral_constant<int, 16>{});
}

}  // namespace qds
