// slicemoe_mx4_product: rows of microscaled 4-bit activations times the matrices of the experts that a routing list names.
#include "mx4.cuh"

namespace slicemoe {

// The head of a workspace: as far as slicemoe_get_status and slicemoe_workspace_set_wait go it is that of the layer calls.
struct MpHeader {
  unsigned unused0, unused1;
  unsigned status;
  unsigned extra_arrivals;
  unsigned long long wait_cycles;
};
constexpr size_t kMpHeaderBytes = 256;
constexpr int kMpMaxExperts = 1024;
constexpr int64_t kMpMaxPairs = 1 << 24;

struct MpParams {
  const slicemoe_mx4_mat* mats;
  const uint8_t* codes;
  const uint8_t* scale;
  const int32_t* ids;
  void* out;
  MpHeader* head;
  int n_experts, N, K, gated, T, k, x_per_pair, dtype;
};

__device__ __forceinline__ void mp_store(const MpParams& p, int64_t at, float v) {
  if (p.dtype == SLICEMOE_F32)
    static_cast<float*>(p.out)[at] = v;
  else if (p.dtype == SLICEMOE_BF16)
    static_cast<__nv_bfloat16*>(p.out)[at] = __float2bfloat16_rn(v);
  else
    static_cast<__half*>(p.out)[at] = __float2half_rn(v);
}

__device__ __forceinline__ float mp_dot(const MpParams& p, const slicemoe_mx4_mat& m, int row, const uint8_t* xc, const uint8_t* xs) {
  float acc = 0.0f;
  for (int kb = 0; kb < p.K / kMxBlock; ++kb) {
    const uint4 a = *reinterpret_cast<const uint4*>(m.codes + mx_code_offset(p.K, row, kb));
    const uint4 b = __ldcg(reinterpret_cast<const uint4*>(xc) + kb);
    const uint32_t wa[4] = {a.x, a.y, a.z, a.w}, wb[4] = {b.x, b.y, b.z, b.w};
    float s = 0.0f;
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const float2 f = __half22float2(mx_decode2(wa[i] >> (8 * j))), g = __half22float2(mx_decode2(wb[i] >> (8 * j)));
        s = fmaf(f.x, g.x, fmaf(f.y, g.y, s));
      }
    acc = fmaf(s * mx_scale_value(m.scale[mx_scale_offset(p.K, row, kb)]), mx_scale_value(__ldcg(xs + kb)), acc);
  }
  return acc;
}

// A thread per value of the result.
__global__ void __launch_bounds__(128) mp_simple_kernel(const MpParams p) {
  mx_dep_launch();
  mx_dep_wait();
  const int n = blockIdx.x * 128 + threadIdx.x;
  for (int64_t pair = blockIdx.y; pair < (int64_t)p.T * p.k; pair += gridDim.y) {
    const int e = p.ids ? __ldcg(p.ids + pair) : 0;
    slicemoe_mx4_mat m = {};
    if ((unsigned)e < (unsigned)p.n_experts) m = p.mats[e];
    if (!m.codes || !m.scale || m.N != p.N || m.K != p.K || (m.gated != 0) != (p.gated != 0)) {
      if (n == 0) atomicOr(&p.head->status, (unsigned)SLICEMOE_STATUS_BAD_EXPERT_ID);
      continue;
    }
    if (n >= p.N) continue;
    const int64_t r = p.x_per_pair ? pair : pair / p.k;
    const uint8_t *xc = p.codes + r * (p.K / 2), *xs = p.scale + r * mx_pitch(p.K);
    float v;
    if (p.gated) {
      const int row = (n >> 4) * 32 + (n & 15);
      const float g = mp_dot(p, m, row, xc, xs), u = mp_dot(p, m, row + 16, xc, xs);
      v = g / (1.0f + expf(-g)) * u;
    } else {
      v = mp_dot(p, m, n, xc, xs);
    }
    mp_store(p, pair * p.N + n, v);
  }
}

}  // namespace slicemoe

using namespace slicemoe;

extern "C" size_t slicemoe_mx4_workspace_bytes(int T, int k, int n_experts) {
  if (T <= 0 || k < 1 || k > SLICEMOE_MAX_TOP_K || n_experts <= 0 || n_experts > kMpMaxExperts || (int64_t)T * k > kMpMaxPairs) return 0;
  return kMpHeaderBytes;
}

extern "C" int slicemoe_mx4_workspace_init(void* workspace, size_t workspace_bytes, void* stream) {
  if (!workspace || workspace_bytes < kMpHeaderBytes || !mx_aligned(workspace, 256)) return SLICEMOE_E_INVALID_ARG;
  SM_CUDA_TRY(cudaMemsetAsync(workspace, 0, kMpHeaderBytes, (cudaStream_t)stream));
  return SLICEMOE_OK;
}

extern "C" int slicemoe_mx4_product(const slicemoe_mx4_mat* mats, int n_experts, int N, int K, int gated, const uint8_t* codes,
                                    const uint8_t* scale, int T, int k, int x_per_pair, const int32_t* ids, void* out, int dtype, void* workspace,
                                    size_t workspace_bytes, void* stream) {
  if (!mats || !codes || !scale || !out || !workspace) return SLICEMOE_E_INVALID_ARG;
  if (n_experts <= 0 || N <= 0 || K <= 0 || K % kMxBlock || T <= 0 || k < 1 || (!ids && k != 1)) return SLICEMOE_E_INVALID_ARG;
  if (n_experts > kMpMaxExperts || N > kMxMaxN || K > kMxMaxK || k > SLICEMOE_MAX_TOP_K || (int64_t)T * k > kMpMaxPairs || !mx_dtype(dtype))
    return SLICEMOE_E_UNSUPPORTED;
  if (!mx_aligned(mats, 8) || !mx_aligned(codes, 16) || !mx_aligned(scale, 4) || !mx_aligned(out, 16) || !mx_aligned(ids, 4) ||
      !mx_aligned(workspace, 256) || workspace_bytes < slicemoe_mx4_workspace_bytes(T, k, n_experts))
    return SLICEMOE_E_INVALID_ARG;
  MpParams p = {mats, codes, scale, ids, out, static_cast<MpHeader*>(workspace), n_experts, N, K, gated, T, k, x_per_pair, dtype};
  const int64_t pairs = (int64_t)T * k;
  return mx_launch(mp_simple_kernel, dim3((N + 127) / 128, (unsigned)(pairs < 65535 ? pairs : 65535)), 128u, 0, (cudaStream_t)stream, MpParams(p));
}
