// slicemoe_combine: out[t] = base[t] + sum_j weights[t, j] rows[t, j].
#include <type_traits>

#include "mx4.cuh"

namespace slicemoe {

struct CbParams {
  const void* rows;
  const float* weights;
  const int32_t* ids;
  const void* base;
  void* out;
  int T, k, N, n_experts;
};
constexpr int kCbThreads = 256;

// A warp takes runs of 256 columns of a token, eight a lane, and asks for the rows of up to kCbAhead experts at a time before it uses the
// first.  Bound: the rows read.  (One row after the other, with a 64-bit division for each run: 60 us for 8,192 tokens x 6 of 2,048.)
constexpr int kCbAhead = 8;
template <class R, class O, bool WIDE>
__global__ void __launch_bounds__(kCbThreads) combine_kernel(const CbParams p) {
  mx_dep_launch();
  mx_dep_wait();
  const int per_row = (p.N + 255) >> 8, lane = threadIdx.x & 31;
  const int64_t run = ((int64_t)blockIdx.x * kCbThreads + threadIdx.x) >> 5;
  const int64_t t = (run >> 31) ? run / per_row : (int64_t)((uint32_t)run / (uint32_t)per_row);
  const int c = (int)(run - t * per_row) * 256 + lane * 8, here = min(8, p.N - c);
  if (t >= p.T || here <= 0) return;
  float acc[8];
#pragma unroll
  for (int q = 0; q < 8; ++q) acc[q] = 0.0f;
  const O* b = static_cast<const O*>(p.base) + t * p.N + c;
  if (p.base) {
    if constexpr (WIDE) {
      mx_load8<O, true>(b, acc);
    } else {
      for (int q = 0; q < here; ++q) acc[q] = mx_load(b + q);
    }
  }
  for (int j0 = 0; j0 < p.k; j0 += kCbAhead) {
    const R* first = static_cast<const R*>(p.rows) + (t * p.k + j0) * p.N + c;
    float w[kCbAhead];
    using Raw = typename std::conditional<sizeof(R) == 4, float4, uint2>::type;  // four elements
    Raw raw[kCbAhead][2];
    bool in[kCbAhead];
#pragma unroll
    for (int j = 0; j < kCbAhead; ++j) {
      in[j] = j0 + j < p.k;
      if (in[j] && p.ids) in[j] = (unsigned)__ldcg(p.ids + t * p.k + j0 + j) < (unsigned)p.n_experts;
      w[j] = in[j] ? __ldcg(p.weights + t * p.k + j0 + j) : 0.0f;
      if (!in[j]) continue;
      const R* r = first + (int64_t)j * p.N;
      if constexpr (!WIDE) {
        R e[8] = {};
#pragma unroll
        for (int q = 0; q < 8; ++q)
          if (q < here) e[q] = mx_from_float<R>(mx_load(r + q));
        memcpy(raw[j], e, sizeof(e));
      } else if constexpr (sizeof(R) == 4) {
        raw[j][0] = __ldcg(reinterpret_cast<const float4*>(r));
        raw[j][1] = __ldcg(reinterpret_cast<const float4*>(r) + 1);
      } else {
        const uint4 v = __ldcg(reinterpret_cast<const uint4*>(r));
        raw[j][0] = make_uint2(v.x, v.y);
        raw[j][1] = make_uint2(v.z, v.w);
      }
    }
#pragma unroll
    for (int j = 0; j < kCbAhead; ++j) {
      if (!in[j]) continue;
      R e[8];
      memcpy(e, raw[j], sizeof(e));
#pragma unroll
      for (int q = 0; q < 8; ++q) acc[q] = fmaf(w[j], mx_to_float<R>(e[q]), acc[q]);
    }
  }
  O* o = static_cast<O*>(p.out) + t * p.N + c;
  if constexpr (WIDE) {
    mx_store8<O, true>(o, acc);
  } else {
#pragma unroll
    for (int q = 0; q < 8; ++q)
      if (q < here) o[q] = mx_from_float<O>(acc[q]);
  }
}

template <class R, class O>
static int combine_as(const CbParams& p, cudaStream_t st) {
  const bool wide = p.N % 8 == 0 && mx_aligned(p.rows, 16) && mx_aligned(p.base, 16) && mx_aligned(p.out, 16);
  const int64_t blocks = ((int64_t)p.T * ((p.N + 255) >> 8) + kCbThreads / 32 - 1) / (kCbThreads / 32);
  if (blocks > INT32_MAX) return SLICEMOE_E_UNSUPPORTED;
  return mx_launch(wide ? combine_kernel<R, O, true> : combine_kernel<R, O, false>, dim3((unsigned)blocks), kCbThreads, 0, st, CbParams(p));
}
template <class R>
static int combine_to(const CbParams& p, int out_dtype, cudaStream_t st) {
  if (out_dtype == SLICEMOE_F32) return combine_as<R, float>(p, st);
  if (out_dtype == SLICEMOE_BF16) return combine_as<R, __nv_bfloat16>(p, st);
  return combine_as<R, __half>(p, st);
}

}  // namespace slicemoe

using namespace slicemoe;

extern "C" int slicemoe_combine(const void* rows, int rows_dtype, int T, int k, int N, const float* weights, const int32_t* ids, int n_experts,
                                const void* base, void* out, int out_dtype, void* stream) {
  if (!rows || !weights || !out || T <= 0 || k < 1 || N <= 0 || (ids && n_experts <= 0)) return SLICEMOE_E_INVALID_ARG;
  if (k > SLICEMOE_MAX_TOP_K || !mx_dtype(rows_dtype) || !mx_dtype(out_dtype)) return SLICEMOE_E_UNSUPPORTED;
  if (!mx_aligned(rows, mx_elem(rows_dtype)) || !mx_aligned(out, mx_elem(out_dtype)) || !mx_aligned(base, mx_elem(out_dtype)))
    return SLICEMOE_E_INVALID_ARG;
  const CbParams p = {rows, weights, ids, base, out, T, k, N, n_experts};
  cudaStream_t st = (cudaStream_t)stream;
  if (rows_dtype == SLICEMOE_F32) return combine_to<float>(p, out_dtype, st);
  if (rows_dtype == SLICEMOE_BF16) return combine_to<__nv_bfloat16>(p, out_dtype, st);
  return combine_to<__half>(p, out_dtype, st);
}
