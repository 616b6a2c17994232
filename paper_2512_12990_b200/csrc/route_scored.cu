// slicemoe_route_scored: softmax or sigmoid scores, a bias for balance, groups of experts, top-k.  One warp per token.
//
// Lane l holds the VPT consecutive experts from l VPT on.  Without a bias experts are ordered by their logits, which is exact.  With
// one the key is score + bias, first in fp32: keys further apart than kNear are in their true order.  Where a choice hangs on two
// that are nearer - about one token in a thousand for keys spread like those of 256 experts - the warp works out the token's keys again
// in fp64 and chooses by those.  The same for groups' values, sums of keys.
//
// What counts is the number of instructions (8,192 tokens of 256 experts are 8 MB, 1.3 us of reading).  A lane sorts its keys once; a round
// of the selection is then a warp maximum of the lanes' first keys, a ballot for the lowest lane that has it, and a shift in that
// lane.  Which expert a selected key belongs to is looked up at the end, for all selections side by side.  A group that is made of
// whole lanes has its two largest keys from the sorted ones by exchanges, and is kept or dropped by lanes.  (Rounds that look through
// all of a lane's keys, and groups scanned in shared memory, took 1,930 instructions a token and 30 us; now 1,070 and 15.9 us in a graph, half of the
// issue slots.)
#include "mx4.cuh"
#include "route.cuh"

namespace slicemoe {

// Error of an fp32 key.  Sigmoid s = 1 / (1 + t), t = __expf(-l), off by (2 + 1.2 |l|) 2^-23 relative, which enters s with s (1 - s):
// below 0.64 x 2^-23 for every l; 1 + t rounds by 2^-24 s, __fdividef by 2 ulp, 2^-22 s; adding the bias by 2^-24 |key|: below
// 2^-21.1 max(1, |key|), two keys 2^-20.1.  Softmax p = e^-d / sum: d rounds by 2^-24 d and d e^-d < 0.37; expf's 2 ulp and the sum's (16 terms
// in a row, then 5 exchanges: at most 21 roundings of 2^-24, and expf's), the reciprocal and the product 2^-24 each: below 2^-18.9 p +
// 0.37 x 2^-24, two keys 2^-17.8.
constexpr float kNearSigmoid = 9.5367431640625e-7f, kNearSoftmax = 7.62939453125e-6f;  // 2^-20, 2^-17; times max(1, |key|)
// A group's value: one key is off by less than half of that, 8 x 2^-24 max(1, |key|) and 64 x 2^-24, and a sum by its keys' errors and its own
// rounding, both of which go with the keys and not with the sum: keys of opposite sign cancel, their errors do not.  kGroup holds them
// and the rounding of the value's bounds.
constexpr float kGroup = 0.625f, kRsMaxFinite = 3.402823466e38f, kRsLeast = 1.17549435e-38f;
constexpr int kRsWarps = 4;
constexpr int kRsMaxGroups = 32;

struct RsParams {
  const void* logits;
  int64_t ld;
  const float* bias;
  int32_t* ids;
  float* weights;
  uint8_t* prec_req;
  int T, E, k, dtype, n_group, topk_group, group_best;
  int lanes;    // that share a group: of whole lanes, a power of two; 0: groups are scanned in shared memory
  int wide;     // a lane's logits are loaded 16 bytes at a time
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
  return v;
}
// A lane's logits as they are in memory; those of experts that do not exist are -inf.
template <int VPT>
__device__ __forceinline__ void rs_load(const RsParams& p, int t, int lane, float (&val)[VPT]) {
  const int64_t at = t * p.ld + lane * VPT;
  if (VPT >= 8 && p.wide) {
#pragma unroll
    for (int v = 0; v < VPT; v += 8) {
      float f[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) f[i] = -CUDART_INF_F;
      if (lane * VPT + v < p.E) {
        if (p.dtype == SLICEMOE_F32)
          mx_load8<float, true>(static_cast<const float*>(p.logits) + at + v, f);
        else if (p.dtype == SLICEMOE_BF16)
          mx_load8<__nv_bfloat16, true>(static_cast<const __nv_bfloat16*>(p.logits) + at + v, f);
        else
          mx_load8<__half, true>(static_cast<const __half*>(p.logits) + at + v, f);
      }
#pragma unroll
      for (int i = 0; i < 8 && v + i < VPT; ++i) val[v + i] = f[i];
    }
  } else {
#pragma unroll
    for (int v = 0; v < VPT; ++v) val[v] = lane * VPT + v < p.E ? rs_logit(p, at + v) : -CUDART_INF_F;
  }
}

// Keys as unsigned integers of the same order; 0 stands for no key (below that of -inf).
__device__ __forceinline__ uint32_t rs_ordered(float k) {
  const uint32_t b = __float_as_uint(k + 0.0f);
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
__device__ __forceinline__ uint64_t rs_warp_max(uint64_t v) {
  const uint32_t hi = __reduce_max_sync(0xffffffffu, (uint32_t)(v >> 32));
  const uint32_t lo = __reduce_max_sync(0xffffffffu, (uint32_t)(v >> 32) == hi ? (uint32_t)v : 0u);
  return (uint64_t)hi << 32 | lo;
}
// Whether two values, a chosen before b, are too near to be told apart.
__device__ __forceinline__ bool rs_near(float a, float b, float near) {
  return !(a - b > near * fmaxf(1.0f, fmaxf(fabsf(a), fabsf(b)))) && !(isinf(a) && isinf(b));
}

// A group's value in 32 bits: its largest key, or half the sum of its two largest, which stays within the range of a float.
__device__ __forceinline__ float rs_group_value(float b0, float b1, bool two) {
  const float v = two ? 0.5f * b0 + 0.5f * b1 : b0;
  return isnan(v) ? -CUDART_INF_F : v;
}
__device__ __forceinline__ double rs_group_value(double b0, double b1, bool two) {
  const double v = two ? b0 + b1 : b0;
  return isnan(v) ? -CUDART_INF : v;
}
// The least and the most that it may be worth.  An infinite one is taken as it is: a key is infinite, which no rounding has made it.  The
// bounds of another are no infinities, even where they leave the range of a float.
__device__ __forceinline__ void rs_group_bounds(float v, float b0, float b1, bool two, float near, float& least, float& most) {
  const float far = kGroup * near, m0 = fmaxf(1.0f, fabsf(b0)), m1 = fmaxf(1.0f, fabsf(b1));
  const float err = isinf(v) ? 0.0f : two ? 0.5f * far * m0 + 0.5f * far * m1 : far * m0, most_finite = isinf(v) ? CUDART_INF_F : kRsMaxFinite;
  least = fmaxf(v - err, -most_finite);
  most = fminf(v + err, most_finite);
}
// Whether the least that a kept group may be worth is above the most that a dropped one may be, or both are the same infinity.
__device__ __forceinline__ bool rs_apart(float least, float most) { return least > most || (least == most && isinf(least)); }

// Which groups are kept, as a bit mask, from the token's keys (of type F) in shared memory: `share` lanes scan a group each.
template <class F>
__device__ __forceinline__ uint32_t rs_groups(const RsParams& p, const F* keys, int lane, float near, bool* unsure) {
  int share = 1;
  while (share * 2 * p.n_group <= 32) share *= 2;
  const int size = p.E / p.n_group, g = lane / share;
  F b0 = (F)-CUDART_INF_F, b1 = (F)-CUDART_INF_F;
  if (g < p.n_group)
    for (int i = lane % share; i < size; i += share) {
      const F v = keys[g * size + i];
      if (v > b0) {
        b1 = b0;
        b0 = v;
      } else if (v > b1) {
        b1 = v;
      }
    }
  for (int off = 1; off < share; off <<= 1) {
    const F o0 = __shfl_xor_sync(0xffffffffu, b0, off), o1 = __shfl_xor_sync(0xffffffffu, b1, off);
    b1 = fmax(fmin(b0, o0), b0 >= o0 ? b1 : o1);
    b0 = fmax(b0, o0);
  }
  const F mine = rs_group_value(b0, b1, p.group_best == 2);
  int rank = 0;
  for (int o = 0; o < p.n_group; ++o) {
    const F v = __shfl_sync(0xffffffffu, mine, o * share);
    rank += v > mine || (v == mine && o < g);
  }
  const bool counts = g < p.n_group && lane % share == 0, kept = counts && rank < p.topk_group;
  if (unsure) {
    float low, high;
    rs_group_bounds((float)mine, (float)b0, (float)b1, p.group_best == 2, near, low, high);
    if (!kept) low = CUDART_INF_F;
    if (!counts || kept) high = -CUDART_INF_F;
#pragma unroll
    for (int off = 16; off > 0; off >>= 1) {
      const float l = __shfl_xor_sync(0xffffffffu, low, off), h = __shfl_xor_sync(0xffffffffu, high, off);
      low = fminf(low, l);
      high = fmaxf(high, h);
    }
    *unsure = p.topk_group < p.n_group && !rs_apart(low, high);
  }
  const uint32_t lanes = __ballot_sync(0xffffffffu, kept);  // bit of group g from lane g * share
  uint32_t mask = 0;
  for (int o = 0; o < p.n_group; ++o) mask |= ((lanes >> (o * share)) & 1u) << o;
  return mask;
}
__device__ __forceinline__ bool rs_kept(const RsParams& p, uint32_t kept, int e) {
  return (kept >> (int)(((float)e + 0.5f) * p.inv_size)) & 1u;
}

// A score in 64 bits; total: the sum that a softmax divides by.
template <bool SIGMOID>
__device__ __forceinline__ double rs_score(float l, float vmax, double total) {
  if constexpr (SIGMOID) return 1.0 / (1.0 + exp(-(double)l));
  return total > 0.0 ? (l == vmax ? 1.0 : exp((double)l - (double)vmax)) / total : 0.0;
}
template <bool SIGMOID>
__device__ __forceinline__ double rs_total(const RsParams& p, const float* logits, float vmax, int lane) {
  double total = 0.0;
  if constexpr (!SIGMOID) {
    if (vmax > -CUDART_INF_F) {
#pragma unroll 1
      for (int e = lane; e < p.E; e += 32) total += logits[e] == vmax ? 1.0 : exp((double)logits[e] - (double)vmax);
    }
#pragma unroll
    for (int off = 16; off > 0; off >>= 1) total += __shfl_xor_sync(0xffffffffu, total, off);
  }
  return total;
}

// Both of the following are made of small loops: they run for few tokens, and instructions that have to be fetched first are what they
// would otherwise wait for (with everything unrolled one such token took 10 us).

// The order of the first `n` candidates (lane j holds one, id) by their keys in 64 bits; lane j gets the j-th of them.
template <bool SIGMOID>
__device__ __noinline__ int rs_reorder(const RsParams& p, const float* logits, const float* bias, float vmax, int id, int n, int lane) {
  const double total = rs_total<SIGMOID>(p, logits, vmax, lane);
  double key = -CUDART_INF;
  if (lane < n) key = rs_score<SIGMOID>(logits[id], vmax, total) + (double)bias[id];
  if (isnan(key)) key = -CUDART_INF;
  int rank = 0;
#pragma unroll 1
  for (int j = 0; j < n; ++j) {
    const double k = __shfl_sync(0xffffffffu, key, j);
    const int i = __shfl_sync(0xffffffffu, id, j);
    rank += k > key || (k == key && i < id);
  }
  int mine = 0;
#pragma unroll 1
  for (int j = 0; j < n; ++j) {  // the candidate of rank `lane`
    const int r = __shfl_sync(0xffffffffu, rank, j), i = __shfl_sync(0xffffffffu, id, j);
    if (r == lane) mine = i;
  }
  return mine;
}

// The share of the first k lanes' logits' scores in their sum, in 64 bits; a score that those do not hold either is 0.
template <bool SIGMOID>
__device__ __noinline__ float rs_share(const RsParams& p, const float* logits, float vmax, float l, int lane) {
  const double total = rs_total<SIGMOID>(p, logits, vmax, lane), s = lane < p.k ? rs_score<SIGMOID>(l, vmax, total) : 0.0;
  double sum = s;
#pragma unroll 1
  for (int off = 8; off > 0; off >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, off);
  return sum > 0.0 ? (float)(s / sum) : 0.0f;
}

// A token's keys in 64 bits, and which groups are kept by them, as a bit mask.
template <bool SIGMOID>
__device__ __noinline__ uint32_t rs_exact_keys(const RsParams& p, const float* logits, const float* bias, double* keys, float vmax, int lane) {
  const double total = rs_total<SIGMOID>(p, logits, vmax, lane);
  // four at a time: an exponential and a quotient in fp64 are a thousand clocks one after the other
  for (int e0 = lane; e0 < p.E; e0 += 128) {
    double key[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) key[i] = rs_score<SIGMOID>(logits[min(e0 + 32 * i, p.E - 1)], vmax, total);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int e = e0 + 32 * i;
      if (e >= p.E) break;
      if (p.bias) key[i] += (double)bias[e];
      keys[e] = isnan(key[i]) ? -CUDART_INF : key[i];
    }
  }
  __syncwarp();
  const uint32_t kept = p.n_group > 1 ? rs_groups(p, (const double*)keys, lane, 0.0f, nullptr) : 0xffffffffu;
  __syncwarp();
  return kept;
}

// The choice with keys in 64 bits where more than 32 of them are near one another: k rounds of the largest key, the lowest index that has
// it.  Lane j < k gets selection j.
__device__ __noinline__ int rs_exact_choice(const RsParams& p, double* keys, uint32_t kept, int lane) {
  if (p.n_group > 1) {
#pragma unroll 1
    for (int e = lane; e < p.E; e += 32)
      if (!rs_kept(p, kept, e)) keys[e] = CUDART_NAN;  // out of the choice
  }
  int id = 0;
#pragma unroll 1
  for (int j = 0; j < p.k; ++j) {
    uint64_t best = 0;
    int at = 0;
#pragma unroll 1
    for (int e = lane; e < p.E; e += 32) {
      const double v = keys[e];
      const uint64_t o = isnan(v) ? 0ull : rs_ordered(v);
      if (o > best) best = o, at = e;
    }
    const uint64_t top = rs_warp_max(best);
    const int e = (int)__reduce_min_sync(0xffffffffu, best == top ? (uint32_t)at : 0xffffffffu);
    if ((e & 31) == lane) keys[e] = CUDART_NAN;
    if (lane == j) id = e;
  }
  return id;
}

// Descending, by an odd-even merge network.
template <int N>
__device__ __forceinline__ void rs_sort(uint32_t (&a)[N]) {
#pragma unroll
  for (int p = 1; p < N; p <<= 1)
#pragma unroll
    for (int k = p; k >= 1; k >>= 1)
#pragma unroll
      for (int j = k % p; j + k < N; j += 2 * k)
#pragma unroll
        for (int i = 0; i < k; ++i)
          if (i + j + k < N && (i + j) / (2 * p) == (i + j + k) / (2 * p)) {
            const uint32_t x = a[i + j], y = a[i + j + k];
            a[i + j] = max(x, y);
            a[i + j + k] = min(x, y);
          }
}

template <int VPT, bool SIGMOID>
__global__ void __launch_bounds__(32 * kRsWarps, VPT <= 8 ? 8 : 4) route_scored_kernel(const RsParams p) {
  __shared__ __align__(16) uint32_t s_keys[kRsWarps][32 * VPT];
  __shared__ double s_exact[kRsWarps][32 * VPT];
  __shared__ __align__(16) float s_logits[kRsWarps][32 * VPT];
  __shared__ float s_bias[32 * VPT];
  mx_dep_launch();
  mx_dep_wait();
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  constexpr float near = SIGMOID ? kNearSigmoid : kNearSoftmax;
  uint32_t* keys = s_keys[warp];
  float* logits = s_logits[warp];
  const int stride = gridDim.x * kRsWarps;
  int t = blockIdx.x * kRsWarps + warp;
  float bias[VPT], ahead[VPT];
  if (t < p.T) rs_load<VPT>(p, t, lane, ahead);
  if (p.bias) {
    // read once a block, in whole lines: the same kilobyte read by every warp for itself, eight values apart, kept a few L2 slices busy
    // for 19 of 28 us (8,192 tokens of 256 experts)
    for (int e = threadIdx.x; e < 32 * VPT; e += 32 * kRsWarps) s_bias[e] = e < p.E ? __ldcg(p.bias + e) : 0.0f;
    __syncthreads();
#pragma unroll
    for (int v = 0; v < VPT; ++v) bias[v] = s_bias[lane * VPT + v];
  }
  if (t >= p.T) return;
  for (; t < p.T; t += stride) {
    float val[VPT], vmax = -CUDART_INF_F;
#pragma unroll
    for (int v = 0; v < VPT; ++v) val[v] = isnan(ahead[v]) ? -CUDART_INF_F : ahead[v];
    if (t + stride < p.T) rs_load<VPT>(p, t + stride, lane, ahead);  // the next token's are on their way meanwhile
    float inv_sum = 0.0f;
    if constexpr (!SIGMOID) {
#pragma unroll
      for (int v = 0; v < VPT; ++v) vmax = fmaxf(vmax, val[v]);
      asm("redux.sync.max.f32 %0, %1, 0xffffffff;" : "=f"(vmax) : "f"(vmax));
      float sum = 0.0f;
      if (vmax > -CUDART_INF_F) {
#pragma unroll
        for (int v = 0; v < VPT; ++v) sum += val[v] == vmax ? 1.0f : expf(val[v] - vmax);  // 0 for an expert that does not exist
      }
#pragma unroll
      for (int off = 16; off > 0; off >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, off);
      inv_sum = sum > 0.0f ? 1.0f / sum : 0.0f;
    }
    auto score = [&](float l) -> float {
      if constexpr (SIGMOID) return __fdividef(1.0f, 1.0f + __expf(-l));
      return (l == vmax ? 1.0f : expf(l - vmax)) * inv_sum;
    };
    uint32_t key[VPT];
#pragma unroll
    for (int v = 0; v < VPT; ++v) {
      float kk = val[v];
      if (p.bias) {
        kk = __fadd_rn(score(val[v]), bias[v]);
        if (isnan(kk)) kk = -CUDART_INF_F;
      }
      key[v] = lane * VPT + v < p.E ? rs_ordered(kk) : 0u;
    }
    __syncwarp();  // the token before is done with the arrays
#pragma unroll
    for (int v = 0; v < VPT; v += 2) {
      *reinterpret_cast<uint2*>(keys + lane * VPT + v) = make_uint2(key[v], key[v + 1]);
      *reinterpret_cast<float2*>(logits + lane * VPT + v) = make_float2(val[v], val[v + 1]);
    }
    uint32_t (&a)[VPT] = key;
    bool unsure = false;
    if (p.n_group > 1 && p.lanes == 0) {
      __syncwarp();
      // values of groups as floats, in the logits' place
      const bool sums = p.bias || p.group_best > 1;  // of scores, not of logits
#pragma unroll
      for (int v = 0; v < VPT; ++v)
        logits[lane * VPT + v] = p.bias ? rs_value(key[v]) : (sums ? score(val[v]) : val[v]);
      __syncwarp();
      uint32_t kept = rs_groups(p, (const float*)logits, lane, near, sums ? &unsure : nullptr);
      __syncwarp();
#pragma unroll
      for (int v = 0; v < VPT; ++v) logits[lane * VPT + v] = val[v];
      __syncwarp();
      if (unsure) kept = rs_exact_keys<SIGMOID>(p, logits, s_bias, s_exact[warp], vmax, lane);
      unsure = false;
#pragma unroll
      for (int v = 0; v < VPT; ++v)
        if (lane * VPT + v < p.E && !rs_kept(p, kept, lane * VPT + v)) a[v] = keys[lane * VPT + v] = 0u;
    }
    rs_sort<VPT>(a);
    if (p.n_group > 1 && p.lanes > 0) {
      // a group's two largest keys, in all of its lanes
      uint32_t b0 = a[0], b1 = VPT > 1 ? a[VPT > 1 ? 1 : 0] : 0u;
      for (int off = 1; off < p.lanes; off <<= 1) {
        const uint32_t o0 = __shfl_xor_sync(0xffffffffu, b0, off), o1 = __shfl_xor_sync(0xffffffffu, b1, off);
        b1 = max(min(b0, o0), max(b1, o1));
        b0 = max(b0, o0);
      }
      float first = rs_value(b0), second = 0.0f;
      const bool sums = p.bias || p.group_best > 1, two = p.group_best > 1;
      if (two) {
        second = rs_value(b1);
        if (!p.bias) first = score(first), second = score(second);
      }
      const float mine = rs_group_value(first, second, two);
      const int size = p.lanes, groups = p.n_group;
      const bool real = lane < groups * size;
      const uint32_t order = real ? rs_ordered(mine) : 0u;
      int rank = 0;
      const int me = lane / size;
      for (int o = 0; o < groups; ++o) {
        const uint32_t v = __shfl_sync(0xffffffffu, order, o * size);
        rank += v > order || (v == order && o < me);
      }
      bool kept = real && rank < p.topk_group;
      if (sums && p.topk_group < groups) {
        float least, most;
        rs_group_bounds(mine, first, second, two, near, least, most);
        const uint32_t low = __reduce_min_sync(0xffffffffu, kept ? rs_ordered(least) : 0xffffffffu);
        const uint32_t high = __reduce_max_sync(0xffffffffu, real && !kept ? rs_ordered(most) : 0u);
        if (!rs_apart(rs_value(low), rs_value(high))) {  // the same in all lanes
          __syncwarp();
          // by all lanes, those without experts too: they exchange values in there
          const uint32_t mask = rs_exact_keys<SIGMOID>(p, logits, s_bias, s_exact[warp], vmax, lane);
          kept = real && ((mask >> me) & 1u);
        }
      }
      if (!kept) {
#pragma unroll
        for (int v = 0; v < VPT; ++v) a[v] = 0u;
      }
    }
    // k rounds, and with a bias one more, to see how near the best that is left is
    uint32_t my_top = 0u;
    int my_owner = 0;
    auto choose = [&](int j) {
      const uint32_t top = __reduce_max_sync(0xffffffffu, a[0]);
      const int owner = __ffs(__ballot_sync(0xffffffffu, a[0] == top)) - 1;
      if (lane == j) my_top = top, my_owner = owner;
      if (lane == owner) {
#pragma unroll
        for (int v = 0; v + 1 < VPT; ++v) a[v] = a[v + 1];
        a[VPT - 1] = 0u;
      }
    };
    int chosen = p.k + (p.bias != nullptr);
    for (int j = 0; j < chosen; ++j) choose(j);
    uint32_t next = __shfl_down_sync(0xffffffffu, my_top, 1);
    bool close = false, all = false;  // whether selections have to be put in order, or the whole choice made again, in 64 bits
    if (p.bias) {
      close = __any_sync(0xffffffffu, lane < p.k && next != 0u && rs_near(rs_value(my_top), rs_value(next), near));
      if (close) {  // more candidates, until the last is clearly behind the k-th
        const float kth = rs_value(__shfl_sync(0xffffffffu, my_top, p.k - 1));
        for (;;) {
          const uint32_t last = __shfl_sync(0xffffffffu, my_top, chosen - 1);
          if (last == 0u || !rs_near(kth, rs_value(last), near)) break;
          if (chosen == 32) {
            all = true;
            break;
          }
          choose(chosen++);
        }
        next = __shfl_down_sync(0xffffffffu, my_top, 1);
      }
    }
    int id;
    if (all) {  // the same in all lanes
      __syncwarp();
      const uint32_t kept = rs_exact_keys<SIGMOID>(p, logits, s_bias, s_exact[warp], vmax, lane);
      id = rs_exact_choice(p, s_exact[warp], kept, lane);
    } else {
      const bool tied = __any_sync(0xffffffffu, lane + 1 < chosen && next == my_top);
      int skip = 0;  // of equal keys in one lane, which one
      if (tied) {
        const unsigned same = __match_any_sync(0xffffffffu, my_top), lanes = __match_any_sync(0xffffffffu, my_owner);
        skip = __popc(same & lanes & ((1u << lane) - 1u));
      }
      __syncwarp();
      id = my_owner * VPT;
#pragma unroll
      for (int v = VPT - 1; v >= 0; --v)
        if (keys[my_owner * VPT + v] == my_top) id = my_owner * VPT + v;
      if (tied) {
        for (int v = 0; v < VPT; ++v)
          if (keys[my_owner * VPT + v] == my_top && skip-- == 0) id = my_owner * VPT + v;
      }
      if (close) {
        const int n = __popc(__ballot_sync(0xffffffffu, lane < chosen && my_top != 0u));
        id = rs_reorder<SIGMOID>(p, logits, s_bias, vmax, id, n, lane);
      }
    }
    __syncwarp();
    const float l = logits[min(id, p.E - 1)];
    float s = 0.0f;
    if (lane < p.k) {
      if constexpr (SIGMOID)
        s = 1.0f / (1.0f + expf(-l));
      else
        s = score(l);
    }
    float w = s;
    if (p.renorm) {
      float total = s;
#pragma unroll
      for (int off = 8; off > 0; off >>= 1) total += __shfl_xor_sync(0xffffffffu, total, off);
      w = total > 0.0f ? s / total : 0.0f;
      // a score that fp32 does not hold, in a sum that does not outweigh it: the quotients in 64 bits
      if (__any_sync(0xffffffffu, lane < p.k && s < kRsLeast && total < 0.25f && l > -CUDART_INF_F)) w = rs_share<SIGMOID>(p, logits, vmax, l, lane);
    }
    if (lane < p.k) {
      const int64_t o = (int64_t)t * p.k + lane;
      p.ids[o] = id;
      p.weights[o] = w * p.scale;
      if (p.prec_req) p.prec_req[o] = (uint8_t)(s >= p.tau || lane < p.rank_high);
    }
  }
}

template <bool SIGMOID>
static int rs_launch(RsParams p, cudaStream_t st) {
  void (*kernel)(RsParams) = p.E <= 64    ? route_scored_kernel<2, SIGMOID>
                             : p.E <= 128 ? route_scored_kernel<4, SIGMOID>
                             : p.E <= 256 ? route_scored_kernel<8, SIGMOID>
                                          : route_scored_kernel<16, SIGMOID>;
  const int vpt = p.E <= 64 ? 2 : p.E <= 128 ? 4 : p.E <= 256 ? 8 : 16, size = p.E / p.n_group;
  const size_t elem = mx_elem(p.dtype);
  p.wide = vpt >= 8 && p.E % 8 == 0 && mx_aligned(p.logits, 16) && p.ld * elem % 16 == 0;
  p.lanes = 0;
  if (size % vpt == 0 && ((size / vpt) & (size / vpt - 1)) == 0) p.lanes = size / vpt;
  const int blocks = (p.T + kRsWarps - 1) / kRsWarps, most = 148 * (vpt <= 8 ? 8 : 4);  // as many as are resident together
  const int rounds = (blocks + most - 1) / most;  // of tokens to a warp: the same for all
  return mx_launch(kernel, dim3((blocks + rounds - 1) / rounds), 32 * kRsWarps, 0, st, RsParams(p));
}

}  // namespace slicemoe

using namespace slicemoe;

extern "C" int slicemoe_route_scored(const void* logits, int dtype, int T, int E, int64_t ld, int score, const float* bias, int n_group,
                                     int topk_group, int group_best, int k, int renorm, float scale, float tau, int rank_high, int32_t* ids,
                                     float* weights, uint8_t* prec_req, void* stream) {
  if (!logits || !ids || !weights || T <= 0 || E <= 0 || ld < E) return SLICEMOE_E_INVALID_ARG;
  if (k < 1 || k > SLICEMOE_MAX_TOP_K || n_group < 1 || E % n_group || topk_group < 1 || topk_group > n_group) return SLICEMOE_E_INVALID_ARG;
  if (T > kMxMaxRow || E > 512 || n_group > kRsMaxGroups || group_best < 1 || group_best > 2 || !mx_dtype(dtype)) return SLICEMOE_E_UNSUPPORTED;
  if (score != SLICEMOE_SCORE_SOFTMAX && score != SLICEMOE_SCORE_SIGMOID) return SLICEMOE_E_UNSUPPORTED;
  if (group_best > E / n_group || k > topk_group * (E / n_group)) return SLICEMOE_E_INVALID_ARG;
  if (!mx_aligned(logits, mx_elem(dtype)) || !mx_aligned(bias, 4) || !mx_aligned(ids, 4) || !mx_aligned(weights, 4)) return SLICEMOE_E_INVALID_ARG;
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
  p.renorm = renorm;
  p.rank_high = rank_high;
  p.scale = scale;
  p.tau = tau;
  p.inv_size = (float)n_group / (float)E;
  return score == SLICEMOE_SCORE_SIGMOID ? rs_launch<true>(p, (cudaStream_t)stream) : rs_launch<false>(p, (cudaStream_t)stream);
}
