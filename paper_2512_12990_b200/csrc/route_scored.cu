// slicemoe_route_scored: softmax or sigmoid scores, a bias for balance, groups of experts, top-k.  One warp per token.
//
// Lane l holds experts l, l + 32, ...  Without a bias experts are ordered by their logits, which is exact.  With one the key is
// score + bias, first in fp32: every key is within kNear / 2 of its value (below), so two keys further apart than kNear are in
// their true order.  Where a choice hangs on two that are nearer - about one token in a thousand for keys spread like those of 256
// experts - the warp works out the token's keys again in fp64 and chooses by those.  The same for groups' values, sums of keys.
#include "mx4.cuh"
#include "route.cuh"

namespace slicemoe {

// Error of an fp32 key.  expf is off by 2 ulp, 2^-22 relative.  Sigmoid s = 1 / (1 + t): ds = s (1 - s) dt / t <= 2^-24, the
// sum and the quotient round by 2^-24 each, s <= 1: below 2^-22.4.  Softmax p = e^-d / sum: d rounds by 2^-24 d and
// d e^-d < 0.37; expf's 2^-22 and the sum's (16 terms in a row, then 5 exchanges; at most 21 roundings of 2^-24, and expf's), the
// reciprocal and the product 2^-24 each: below (2^-22 + 2^-22 + 24 x 2^-24) p + 0.37 x 2^-24 < 2^-18.9 p.  Adding the bias rounds by
// 2^-24 |key|.  Two keys' errors, with room: 2^-20.5 for sigmoids, 2^-17.8 max p for softmax; both by kNear = 2^-20 and 2^-17,
// times max(1, |key|).  A group's value of two keys: twice that.
constexpr float kNearSigmoid = 9.5367431640625e-7f, kNearSoftmax = 7.62939453125e-6f;
constexpr int kRsWarps = 4;       // tokens of a block
constexpr int kRsMaxGroups = 32;

struct RsParams {
  const void* logits;
  int64_t ld;
  const float* bias;
  int32_t* ids;
  float* weights;
  uint8_t* prec_req;
  int T, E, k, dtype, n_group, topk_group, group_best, lanes;  // lanes: that share a group, a power of two
  int renorm, rank_high;
  float scale, tau, inv_size;
};

__device__ __forceinline__ float rs_logit(const RsParams& p, int64_t at) {
  float v;
  if (p.dtype == SLICEMOE_F32)
    v = mx_load(static_cast<const float*>(p.logits) + at);
  else if (p.dtype == SLICEMOE_BF16)
    v = mx_load(static_cast<const __nv_bfloat16*>(p.logits) + at);
  else
    v = mx_load(static_cast<const __half*>(p.logits) + at);
  return isnan(v) ? -CUDART_INF_F : v;
}

// Keys as unsigned integers of the same order; 0 stands for no key (below that of -inf).
__device__ __forceinline__ uint32_t rs_ordered(float k) {
  const uint32_t b = __float_as_uint(isnan(k) ? -CUDART_INF_F : k + 0.0f);
  return b ^ ((uint32_t)((int32_t)b >> 31) | 0x80000000u);
}
__device__ __forceinline__ float rs_value(uint32_t o) { return __uint_as_float(o & 0x80000000u ? o ^ 0x80000000u : ~o); }
__device__ __forceinline__ uint64_t rs_ordered(double k) {
  const uint64_t b = (uint64_t)__double_as_longlong(isnan(k) ? -CUDART_INF : k + 0.0);
  return b ^ ((uint64_t)((int64_t)b >> 63) | 0x8000000000000000ull);
}
__device__ __forceinline__ double rs_value(uint64_t o) {
  return __longlong_as_double((long long)(o & 0x8000000000000000ull ? o ^ 0x8000000000000000ull : ~o));
}
__device__ __forceinline__ uint32_t rs_warp_max(uint32_t v) { return __reduce_max_sync(0xffffffffu, v); }
__device__ __forceinline__ uint64_t rs_warp_max(uint64_t v) {
  const uint32_t hi = __reduce_max_sync(0xffffffffu, (uint32_t)(v >> 32));
  const uint32_t lo = __reduce_max_sync(0xffffffffu, (uint32_t)(v >> 32) == hi ? (uint32_t)v : 0u);
  return (uint64_t)hi << 32 | lo;
}
// Whether two values, a chosen before b, are too near to be told apart.
__device__ __forceinline__ bool rs_near(float a, float b, float near) {
  return !(a - b > near * fmaxf(1.0f, fmaxf(fabsf(a), fabsf(b)))) && !(isinf(a) && isinf(b));
}

// Which groups are kept, as a bit mask.  keys: the token's, in shared memory; F: their type.  `lanes` lanes scan a group each; a
// group's value is then in the first of them.
template <class F>
__device__ __forceinline__ uint32_t rs_groups(const RsParams& p, const F* keys, int lane, float near, bool* unsure) {
  const int size = p.E / p.n_group, g = lane / p.lanes;
  F b0 = (F)-CUDART_INF_F, b1 = (F)-CUDART_INF_F;
  if (g < p.n_group)
    for (int i = lane % p.lanes; i < size; i += p.lanes) {
      const F v = keys[g * size + i];
      if (v > b0) {
        b1 = b0;
        b0 = v;
      } else if (v > b1) {
        b1 = v;
      }
    }
  for (int off = 1; off < p.lanes; off <<= 1) {
    const F o0 = __shfl_xor_sync(0xffffffffu, b0, off), o1 = __shfl_xor_sync(0xffffffffu, b1, off);
    b1 = fmax(fmin(b0, o0), b0 >= o0 ? b1 : o1);
    b0 = fmax(b0, o0);
  }
  F mine = p.group_best == 2 ? b0 + b1 : b0;
  if (isnan(mine)) mine = (F)-CUDART_INF_F;
  int rank = 0;
  for (int o = 0; o < p.n_group; ++o) {
    const F v = __shfl_sync(0xffffffffu, mine, o * p.lanes);
    rank += v > mine || (v == mine && o < g);
  }
  const bool mine_counts = g < p.n_group && lane % p.lanes == 0;
  const bool kept = mine_counts && rank < p.topk_group;
  if (unsure) {
    F low = kept ? mine : (F)CUDART_INF_F, high = mine_counts && !kept ? mine : (F)-CUDART_INF_F;
#pragma unroll
    for (int off = 16; off > 0; off >>= 1) {
      low = fmin(low, __shfl_xor_sync(0xffffffffu, low, off));
      high = fmax(high, __shfl_xor_sync(0xffffffffu, high, off));
    }
    *unsure = p.topk_group < p.n_group && rs_near((float)low, (float)high, 2.0f * near);
  }
  uint32_t mask = __ballot_sync(0xffffffffu, kept);
  if (p.lanes > 1) {  // bit of group g from lane g * lanes
    uint32_t m = 0;
    for (int o = 0; o < p.n_group; ++o) m |= ((mask >> (o * p.lanes)) & 1u) << o;
    mask = m;
  }
  return mask;
}

// k rounds of the largest key, the lowest index that has it.  Lane j < k gets selection j.  `near` >= 0: *unsure is set where two
// selections in a row, or the last and the best that is left, are too near.
template <class U, int VPT>
__device__ __forceinline__ int rs_select(U (&key)[VPT], int k, int left, int lane, float near, bool* unsure) {
  int idsel = 0;
  float last = 0.0f;
  const int rounds = unsure && k < left ? k + 1 : k;
  for (int j = 0; j < rounds; ++j) {
    U best = key[0];
    int bv = 0;
#pragma unroll
    for (int v = 1; v < VPT; ++v)
      if (key[v] > best) {
        best = key[v];
        bv = v;
      }
    const U top = rs_warp_max(best);
    if (unsure) {
      const float t = (float)rs_value(top);
      if (j > 0 && rs_near(last, t, near)) *unsure = true;
      last = t;
    }
    if (j == k) break;
    const int e = (int)__reduce_min_sync(0xffffffffu, best == top ? (uint32_t)(bv * 32 + lane) : 0xffffffffu);
#pragma unroll
    for (int v = 0; v < VPT; ++v)
      if (e == v * 32 + lane) key[v] = 0;
    if (lane == j) idsel = e;
  }
  return idsel;
}

// The same choice with keys in 64 bits.
template <int VPT, bool SIGMOID>
__device__ __noinline__ int rs_exact(const RsParams& p, const float (&val)[VPT], float vmax, double* keys, int lane) {
  double s[VPT], sum = 0.0;
#pragma unroll
  for (int v = 0; v < VPT; ++v) {
    const int e = v * 32 + lane;
    if constexpr (SIGMOID) {
      s[v] = 1.0 / (1.0 + exp(-(double)val[v]));
    } else {
      s[v] = val[v] == vmax ? 1.0 : exp((double)val[v] - (double)vmax);
      if (vmax == -CUDART_INF_F || e >= p.E) s[v] = 0.0;
      sum += s[v];
    }
  }
  if constexpr (!SIGMOID) {
#pragma unroll
    for (int off = 16; off > 0; off >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, off);
  }
  uint64_t key[VPT];
#pragma unroll
  for (int v = 0; v < VPT; ++v) {
    const int e = v * 32 + lane;
    key[v] = 0;
    if (e >= p.E) continue;
    const double score = SIGMOID ? s[v] : (sum > 0.0 ? s[v] / sum : 0.0);
    const double kk = p.bias ? score + (double)__ldcg(p.bias + e) : score;
    key[v] = rs_ordered(kk);
    keys[e] = rs_value(key[v]);
  }
  if (p.n_group > 1) {
    __syncwarp();
    const uint32_t kept = rs_groups(p, (const double*)keys, lane, 0.0f, nullptr);
#pragma unroll
    for (int v = 0; v < VPT; ++v) {
      const int e = v * 32 + lane;
      if (e < p.E && !((kept >> (int)(((float)e + 0.5f) * p.inv_size)) & 1u)) key[v] = 0;
    }
  }
  if (!p.bias) {  // within the groups the logits' order is exact, and finer than that of their scores
#pragma unroll
    for (int v = 0; v < VPT; ++v)
      if (key[v]) key[v] = rs_ordered((double)val[v]);
  }
  return rs_select<uint64_t, VPT>(key, p.k, 0, lane, 0.0f, nullptr);
}

template <int VPT, bool SIGMOID>
__global__ void __launch_bounds__(32 * kRsWarps) route_scored_kernel(const RsParams p) {
  __shared__ double s_keys[kRsWarps][32 * VPT];
  mx_dep_launch();
  mx_dep_wait();
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, t = blockIdx.x * kRsWarps + warp;
  if (t >= p.T) return;
  constexpr float near = SIGMOID ? kNearSigmoid : kNearSoftmax;
  float val[VPT], vmax = -CUDART_INF_F;
#pragma unroll
  for (int v = 0; v < VPT; ++v) {
    const int e = v * 32 + lane;
    val[v] = e < p.E ? rs_logit(p, t * p.ld + e) : -CUDART_INF_F;
    vmax = fmaxf(vmax, val[v]);
  }
  float inv_sum = 0.0f;
  if constexpr (!SIGMOID) {
    asm("redux.sync.max.f32 %0, %1, 0xffffffff;" : "=f"(vmax) : "f"(vmax));
    float sum = 0.0f;
    if (vmax > -CUDART_INF_F) {
#pragma unroll
      for (int v = 0; v < VPT; ++v)
        if (v * 32 + lane < p.E) sum += val[v] == vmax ? 1.0f : expf(val[v] - vmax);
    }
#pragma unroll
    for (int off = 16; off > 0; off >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, off);
    inv_sum = sum > 0.0f ? 1.0f / sum : 0.0f;
  }
  auto score = [&](float l) -> float {
    if constexpr (SIGMOID) return 1.0f / (1.0f + expf(-l));
    return (l == vmax ? 1.0f : expf(l - vmax)) * inv_sum;
  };
  uint32_t key[VPT];
  float* keys = reinterpret_cast<float*>(s_keys[warp]);
  const bool sums = p.n_group > 1 && (p.bias || p.group_best > 1);  // groups' values are of scores, not of logits
#pragma unroll
  for (int v = 0; v < VPT; ++v) {
    const int e = v * 32 + lane;
    key[v] = 0;
    if (e >= p.E) continue;
    float kk = val[v];
    if (p.bias || sums) {
      const float s = score(val[v]);
      const float b = p.bias ? __fadd_rn(s, __ldcg(p.bias + e)) : s;
      if (p.bias) kk = b;
      if (p.n_group > 1) keys[e] = isnan(b) ? -CUDART_INF_F : b;
    } else if (p.n_group > 1) {
      keys[e] = kk;
    }
    key[v] = rs_ordered(kk);
  }
  bool unsure = false;
  if (p.n_group > 1) {
    __syncwarp();
    const uint32_t kept = rs_groups(p, (const float*)keys, lane, near, sums ? &unsure : nullptr);
#pragma unroll
    for (int v = 0; v < VPT; ++v) {
      const int e = v * 32 + lane;
      if (e < p.E && !((kept >> (int)(((float)e + 0.5f) * p.inv_size)) & 1u)) key[v] = 0;
    }
  }
  int id = rs_select<uint32_t, VPT>(key, p.k, p.topk_group * (p.E / p.n_group), lane, near, p.bias ? &unsure : nullptr);
  if (unsure) {  // the same in all lanes
    __syncwarp();
    id = rs_exact<VPT, SIGMOID>(p, val, vmax, s_keys[warp], lane);
  }
  float l = 0.0f;  // the selection's logit, from the lane that holds it
#pragma unroll
  for (int v = 0; v < VPT; ++v) {
    const float got = __shfl_sync(0xffffffffu, val[v], id & 31);
    if ((id >> 5) == v) l = got;
  }
  const float s = lane < p.k ? score(l) : 0.0f;
  float w = s;
  if (p.renorm) {
    float total = 0.0f;
    for (int j = 0; j < p.k; ++j) total += __shfl_sync(0xffffffffu, s, j);
    w = total > 0.0f ? s / total : 0.0f;
  }
  if (lane < p.k) {
    const int64_t o = (int64_t)t * p.k + lane;
    p.ids[o] = id;
    p.weights[o] = w * p.scale;
    if (p.prec_req) p.prec_req[o] = (uint8_t)(s >= p.tau || lane < p.rank_high);
  }
}

template <bool SIGMOID>
static int rs_launch(const RsParams& p, cudaStream_t st) {
  void (*kernel)(RsParams) = p.E <= 64    ? route_scored_kernel<2, SIGMOID>
                             : p.E <= 128 ? route_scored_kernel<4, SIGMOID>
                             : p.E <= 256 ? route_scored_kernel<8, SIGMOID>
                                          : route_scored_kernel<16, SIGMOID>;
  return mx_launch(kernel, dim3((p.T + kRsWarps - 1) / kRsWarps), 32 * kRsWarps, 0, st, RsParams(p));
}

}  // namespace slicemoe

using namespace slicemoe;

extern "C" int slicemoe_route_scored(const void* logits, int dtype, int T, int E, int64_t ld, int score, const float* bias, int n_group,
                                     int topk_group, int group_best, int k, int renorm, float scale, float tau, int rank_high, int32_t* ids,
                                     float* weights, uint8_t* prec_req, void* stream) {
  if (!logits || !ids || !weights || T <= 0 || E <= 0 || ld < E) return SLICEMOE_E_INVALID_ARG;
  if (k < 1 || k > SLICEMOE_MAX_TOP_K || n_group < 1 || E % n_group || topk_group < 1 || topk_group > n_group) return SLICEMOE_E_INVALID_ARG;
  if (E > 512 || n_group > kRsMaxGroups || group_best < 1 || group_best > 2 || !mx_dtype(dtype)) return SLICEMOE_E_UNSUPPORTED;
  if (score != SLICEMOE_SCORE_SOFTMAX && score != SLICEMOE_SCORE_SIGMOID) return SLICEMOE_E_UNSUPPORTED;
  if (group_best > E / n_group || k > topk_group * (E / n_group)) return SLICEMOE_E_INVALID_ARG;
  if (!mx_aligned(logits, mx_elem(dtype))) return SLICEMOE_E_INVALID_ARG;
  RsParams p;
  p.logits = logits;
  p.ld = ld;
  p.bias = bias;
  p.ids = ids;
  p.weights = weights;
  p.prec_req = prec_req;
  p.T = T;
  p.E = E;
  p.k = k;
  p.dtype = dtype;
  p.n_group = n_group;
  p.topk_group = topk_group;
  p.group_best = group_best;
  p.lanes = 1;
  while (p.lanes * 2 * n_group <= 32) p.lanes *= 2;
  p.renorm = renorm;
  p.rank_high = rank_high;
  p.scale = scale;
  p.tau = tau;
  p.inv_size = (float)n_group / (float)E;
  return score == SLICEMOE_SCORE_SIGMOID ? rs_launch<true>(p, (cudaStream_t)stream) : rs_launch<false>(p, (cudaStream_t)stream);
}
