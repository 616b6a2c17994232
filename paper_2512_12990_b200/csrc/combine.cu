// slicemoe_combine: out[t] = base[t] + sum_j weights[t, j] rows[t, j].
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

// A thread per eight columns of a token; the rows' loads of a thread do not depend on one another.  Bound: the rows read.
template <class R, class O, bool WIDE>
__global__ void __launch_bounds__(kCbThreads) combine_kernel(const CbParams p) {
  mx_dep_launch();
  mx_dep_wait();
  const int per_row = (p.N + 7) >> 3;
  const int64_t n = (int64_t)p.T * per_row, step = (int64_t)gridDim.x * kCbThreads;
  for (int64_t i = (int64_t)blockIdx.x * kCbThreads + threadIdx.x; i < n; i += step) {
    const int64_t t = i / per_row;
    const int c = (int)(i - t * per_row) * 8, here = min(8, p.N - c);
    float acc[8];
#pragma unroll
    for (int q = 0; q < 8; ++q) acc[q] = 0.0f;
    if (p.base) {
      const O* b = static_cast<const O*>(p.base) + t * p.N + c;
      if constexpr (WIDE) {
        mx_load8<O, true>(b, acc);
      } else {
        for (int q = 0; q < here; ++q) acc[q] = mx_load(b + q);
      }
    }
    for (int j = 0; j < p.k; ++j) {
      if (p.ids && (unsigned)__ldcg(p.ids + t * p.k + j) >= (unsigned)p.n_experts) continue;
      const float w = __ldcg(p.weights + t * p.k + j);
      const R* r = static_cast<const R*>(p.rows) + (t * p.k + j) * p.N + c;
      float v[8];
      if constexpr (WIDE) {
        mx_load8<R, true>(r, v);
      } else {
#pragma unroll
        for (int q = 0; q < 8; ++q) v[q] = q < here ? mx_load(r + q) : 0.0f;
      }
#pragma unroll
      for (int q = 0; q < 8; ++q) acc[q] = fmaf(w, v[q], acc[q]);
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
}

template <class R, class O>
static int combine_as(const CbParams& p, cudaStream_t st) {
  const bool wide = p.N % 8 == 0 && mx_aligned(p.rows, 16) && mx_aligned(p.base, 16) && mx_aligned(p.out, 16);
  const int64_t blocks = ((int64_t)p.T * ((p.N + 7) / 8) + kCbThreads - 1) / kCbThreads;
  return mx_launch(wide ? combine_kernel<R, O, true> : combine_kernel<R, O, false>, dim3((unsigned)(blocks < 148 * 64 ? blocks : 148 * 64)), kCbThreads, 0,
                   st, CbParams(p));
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
