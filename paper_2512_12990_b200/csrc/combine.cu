// slicemoe_combine: out[t] = base[t] + sum_j weights[t, j] rows[t, j].
#include <type_traits>

#include "decode_common.cuh"
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

// Eight values of a row as pairs of floats.
__device__ __forceinline__ void cb_pairs(const float4 (&raw)[2], float2 (&v)[4]) {
  v[0] = make_float2(raw[0].x, raw[0].y), v[1] = make_float2(raw[0].z, raw[0].w), v[2] = make_float2(raw[1].x, raw[1].y), v[3] = make_float2(raw[1].z, raw[1].w);
}
template <class R>
__device__ __forceinline__ void cb_pairs(const uint4 (&raw)[1], float2 (&v)[4]) {
  const uint32_t w[4] = {raw[0].x, raw[0].y, raw[0].z, raw[0].w};
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    R e[2];
    memcpy(e, &w[i], 4);
    v[i] = make_float2(mx_to_float<R>(e[0]), mx_to_float<R>(e[1]));
  }
}
// acc += w v, two at a time in one instruction
__device__ __forceinline__ void cb_fma2(float2& acc, float w, float2 v) {
  asm("{\n .reg .b64 a, b, c;\n mov.b64 a, {%0, %1};\n mov.b64 b, {%2, %2};\n mov.b64 c, {%3, %4};\n fma.rn.f32x2 a, b, c, a;\n mov.b64 {%0, %1}, a;\n}"
      : "+f"(acc.x), "+f"(acc.y)
      : "f"(w), "f"(v.x), "f"(v.y));
}

// A warp takes a run of 256 columns of a token, eight a lane (next to one another where rows begin on 16 bytes, else 32 apart, so that a
// warp's loads are whole lines either way), and asks for the rows of up to eight (of fp32, four) experts at a time before it uses the
// first.  Bound: the rows read.  (One row after the other, with a 64-bit division for each run: 60 us for 8,192 tokens x 6 of 2,048.)
template <class R, class O, bool WIDE>
__global__ void __launch_bounds__(kCbThreads, 3) combine_kernel(const CbParams p) {
  mx_dep_launch();
  mx_dep_wait();
  const int per_row = (p.N + 255) >> 8, lane = threadIdx.x & 31;
  const int64_t runs = (int64_t)p.T * per_row, step = (int64_t)gridDim.x * (kCbThreads / 32);
  constexpr int kCbAhead = sizeof(R) == 4 ? 4 : 8;
  for (int64_t run = ((int64_t)blockIdx.x * kCbThreads + threadIdx.x) >> 5; run < runs; run += step) {
    const int64_t t = (run >> 31) ? run / per_row : (int64_t)((uint32_t)run / (uint32_t)per_row);
    const int c0 = (int)(run - t * per_row) * 256, c = c0 + (WIDE ? lane * 8 : lane);
    if (c >= p.N) continue;
    const int here = WIDE ? 8 : (p.N - c + 31) >> 5;  // of the lane's columns
    const R* row = static_cast<const R*>(p.rows) + t * p.k * p.N + c;
    const float* weights = p.weights + t * p.k;
    const int32_t* ids = p.ids ? p.ids + t * p.k : nullptr;
    float2 acc[4];
    {
      float base[8];
#pragma unroll
      for (int q = 0; q < 8; ++q) base[q] = 0.0f;
      if (p.base) {
        const O* b = static_cast<const O*>(p.base) + t * p.N + c;
        if constexpr (WIDE) {
          mx_load8<O, true>(b, base);
        } else {
#pragma unroll
          for (int q = 0; q < 8; ++q)
            if (q < here) base[q] = mx_load(b + 32 * q);
        }
      }
#pragma unroll
      for (int q = 0; q < 4; ++q) acc[q] = make_float2(base[2 * q], base[2 * q + 1]);
    }
    if constexpr (WIDE) {
      constexpr int kPieces = sizeof(R) == 4 ? 2 : 1;
      using Raw = typename std::conditional<sizeof(R) == 4, float4, uint4>::type;
      for (int j0 = 0; j0 < p.k; j0 += kCbAhead) {
        Raw raw[kCbAhead][kPieces];
        float w[kCbAhead];
        uint32_t in = 0;
#pragma unroll
        for (int j = 0; j < kCbAhead; ++j) {
          if (j0 + j >= p.k) break;
          if (!ids || (unsigned)__ldcg(ids + j0 + j) < (unsigned)p.n_experts) {
            in |= 1u << j;
            w[j] = __ldcg(weights + j0 + j);
#pragma unroll
            for (int h = 0; h < kPieces; ++h) raw[j][h] = __ldcg(reinterpret_cast<const Raw*>(row) + h);
          }
          row += p.N;
        }
#pragma unroll
        for (int j = 0; j < kCbAhead; ++j) {
          if (j0 + j >= p.k) break;
          if (!((in >> j) & 1u)) continue;
          float2 v[4];
          if constexpr (sizeof(R) == 4) cb_pairs(raw[j], v);
          else cb_pairs<R>(raw[j], v);
#pragma unroll
          for (int q = 0; q < 4; ++q) cb_fma2(acc[q], w[j], v[q]);
        }
      }
    } else {
      // two rows at a time
      for (int j = 0; j < p.k; j += 2, row += 2 * (int64_t)p.N) {
        float v[2][8], w[2];
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          const bool in = j + h < p.k && (!ids || (unsigned)__ldcg(ids + j + h) < (unsigned)p.n_experts);
          w[h] = in ? __ldcg(weights + j + h) : 0.0f;
#pragma unroll
          for (int q = 0; q < 8; ++q) v[h][q] = in && q < here ? mx_load(row + (int64_t)h * p.N + 32 * q) : 0.0f;
        }
#pragma unroll
        for (int h = 0; h < 2; ++h)
#pragma unroll
          for (int q = 0; q < 4; ++q) cb_fma2(acc[q], w[h], make_float2(v[h][2 * q], v[h][2 * q + 1]));
      }
    }
    const float y[8] = {acc[0].x, acc[0].y, acc[1].x, acc[1].y, acc[2].x, acc[2].y, acc[3].x, acc[3].y};
    O* o = static_cast<O*>(p.out) + t * p.N + c;
    if constexpr (WIDE) {
      mx_store8<O, true>(o, y);
    } else {
#pragma unroll
      for (int q = 0; q < 8; ++q)
        if (q < here) o[32 * q] = mx_from_float<O>(y[q]);
    }
  }
}

// The same for 16-bit rows that come from HBM: what a lane needs of the next two runs is on its way into shared memory (its own 16 bytes of every
// row and of the base, so that no lane waits for another) while one is added up: 48 us for 8,192 tokens x 6 of 2,048, 5.6 TB/s.  (The kernel
// above takes 53: its registers hold one run's rows at most, 74 KB an SM, and a block that ends takes its place with it.)
constexpr int kCbDepth = 3, kCbMostRows = 8, kCbSmem = 113 * 1024;
constexpr int64_t kCbStreamBytes = 112 << 20;
__host__ __device__ constexpr int cb_slot(int k, int base_bytes) { return k * 16 + base_bytes; }  // of a lane and a run
template <class R, class O>
__global__ void __launch_bounds__(kCbThreads) combine_stream_kernel(const CbParams p) {
  extern __shared__ __align__(16) uint8_t cb_smem[];
  mx_dep_launch();
  mx_dep_wait();
  const int per_row = (p.N + 255) >> 8, lane = threadIdx.x & 31;
  const int64_t runs = (int64_t)p.T * per_row, step = (int64_t)gridDim.x * (kCbThreads / 32);
  int64_t run = ((int64_t)blockIdx.x * kCbThreads + threadIdx.x) >> 5;
  // pieces of 16 bytes: [stage][piece][thread]; a base of fp32 has two
  constexpr int kBase = sizeof(O) == 4 ? 2 : 1;
  const int pieces = p.k + (p.base ? kBase : 0);
  const uint32_t mine = smem_u32(cb_smem) + threadIdx.x * 16, stage_bytes = pieces * kCbThreads * 16;
  float w[kCbDepth];     // lane j: the weight of row j,
  bool in[kCbDepth];     // and whether it counts
  auto place = [&](int64_t r, int64_t& t, int& c) {
    t = (r >> 31) ? r / per_row : (int64_t)((uint32_t)r / (uint32_t)per_row);
    c = (int)(r - t * per_row) * 256 + lane * 8;
  };
  auto ask = [&](int64_t r, int stage, float& weight, bool& counts) {
    weight = 0.0f;
    counts = false;
    if (r < runs) {
      int64_t t;
      int c;
      place(r, t, c);
      if (lane < p.k) {
        weight = __ldcg(p.weights + t * p.k + lane);
        counts = !p.ids || (unsigned)__ldcg(p.ids + t * p.k + lane) < (unsigned)p.n_experts;
      }
      if (c < p.N) {
        const uint32_t at = mine + stage * stage_bytes;
        const R* row = static_cast<const R*>(p.rows) + t * p.k * p.N + c;
        for (int j = 0; j < p.k; ++j)
          asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(at + j * (kCbThreads * 16)), "l"(row + (int64_t)j * p.N) : "memory");
        if (p.base) {
          const O* b = static_cast<const O*>(p.base) + t * p.N + c;
#pragma unroll
          for (int h = 0; h < kBase; ++h)
            asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(at + (p.k + h) * (kCbThreads * 16)), "l"(b + h * (16 / (int)sizeof(O))) : "memory");
        }
      }
    }
    asm volatile("cp.async.commit_group;" ::: "memory");
  };
#pragma unroll
  for (int d = 0; d < kCbDepth; ++d) ask(run + d * step, d, w[d], in[d]);
  while (run < runs) {
#pragma unroll
    for (int d = 0; d < kCbDepth; ++d) {
      if (run >= runs) break;
      asm volatile("cp.async.wait_group %0;" ::"n"(kCbDepth - 1) : "memory");  // all but the newest: this run's
      int64_t t;
      int c;
      place(run, t, c);
      const uint32_t counts = __ballot_sync(0xffffffffu, in[d]);
      const uint8_t* at = cb_smem + threadIdx.x * 16 + d * stage_bytes;
      float2 acc[4] = {};
      if (p.base && c < p.N) {
        float base[8];
        if constexpr (sizeof(O) == 4) {
          memcpy(base, __builtin_assume_aligned(at + p.k * (kCbThreads * 16), 16), 16);
          memcpy(base + 4, __builtin_assume_aligned(at + (p.k + 1) * (kCbThreads * 16), 16), 16);
        } else {
          O e[8];
          memcpy(e, __builtin_assume_aligned(at + p.k * (kCbThreads * 16), 16), 16);
#pragma unroll
          for (int q = 0; q < 8; ++q) base[q] = mx_to_float<O>(e[q]);
        }
#pragma unroll
        for (int q = 0; q < 4; ++q) acc[q] = make_float2(base[2 * q], base[2 * q + 1]);
      }
      for (int j = 0; j < p.k; ++j) {
        const float weight = __shfl_sync(0xffffffffu, w[d], j);
        if (!((counts >> j) & 1u) || c >= p.N) continue;
        uint4 raw[1];
        memcpy(raw, __builtin_assume_aligned(at + j * (kCbThreads * 16), 16), 16);
        float2 v[4];
        cb_pairs<R>(raw, v);
#pragma unroll
        for (int q = 0; q < 4; ++q) cb_fma2(acc[q], weight, v[q]);
      }
      if (c < p.N) {
        const float y[8] = {acc[0].x, acc[0].y, acc[1].x, acc[1].y, acc[2].x, acc[2].y, acc[3].x, acc[3].y};
        mx_store8<O, true>(static_cast<O*>(p.out) + t * p.N + c, y);
      }
      ask(run + kCbDepth * step, d, w[d], in[d]);
      run += step;
    }
  }
  asm volatile("cp.async.wait_all;" ::: "memory");
}

template <class R, class O>
static int combine_as(const CbParams& p, cudaStream_t st) {
  const bool wide = p.N % 8 == 0 && mx_aligned(p.rows, 16) && mx_aligned(p.base, 16) && mx_aligned(p.out, 16);
  if constexpr (sizeof(R) == 2) {
    // where the rows do not fit L2: 8,192 x 6 x 2,048 in bf16 53 us without, 48 so; rows that L2 still holds are read faster by many warps
    // than by copies that wait for one another (4,096 x 6 x 1,000: 9.0 and 11.8)
    const int slot = cb_slot(p.k, p.base ? 8 * (int)sizeof(O) : 0), smem = slot * kCbThreads * kCbDepth;
    if (wide && p.k <= kCbMostRows && smem <= kCbSmem && (int64_t)p.T * p.k * p.N * (int)sizeof(R) >= kCbStreamBytes) {
      static bool attr_set[64];
      int dev = 0;
      SM_CUDA_TRY(cudaGetDevice(&dev));
      if (dev < 0 || dev >= 64) return SLICEMOE_E_UNSUPPORTED;
      if (!attr_set[dev]) {
        SM_CUDA_TRY(cudaFuncSetAttribute(combine_stream_kernel<R, O>, cudaFuncAttributeMaxDynamicSharedMemorySize, kCbSmem));
        attr_set[dev] = true;
      }
      const int per_sm = (226 * 1024) / (smem + 1024);
      return mx_launch(combine_stream_kernel<R, O>, dim3(148u * (per_sm < 8 ? per_sm : 8)), kCbThreads, (size_t)smem, st, CbParams(p));
    }
  }
  const int64_t blocks = ((int64_t)p.T * ((p.N + 255) >> 8) + kCbThreads / 32 - 1) / (kCbThreads / 32);
  return mx_launch(wide ? combine_kernel<R, O, true> : combine_kernel<R, O, false>, dim3((unsigned)(blocks < (1 << 20) ? blocks : 1 << 20)), kCbThreads, 0, st,
                   CbParams(p));
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
  if (k > SLICEMOE_MAX_TOP_K || N > kMxMaxRow || !mx_dtype(rows_dtype) || !mx_dtype(out_dtype)) return SLICEMOE_E_UNSUPPORTED;
  if (!mx_aligned(rows, mx_elem(rows_dtype)) || !mx_aligned(out, mx_elem(out_dtype)) || !mx_aligned(base, mx_elem(out_dtype)) || !mx_aligned(weights, 4) ||
      !mx_aligned(ids, 4))
    return SLICEMOE_E_INVALID_ARG;
  const CbParams p = {rows, weights, ids, base, out, T, k, N, n_experts};
  cudaStream_t st = (cudaStream_t)stream;
  if (rows_dtype == SLICEMOE_F32) return combine_to<float>(p, out_dtype, st);
  if (rows_dtype == SLICEMOE_BF16) return combine_to<__nv_bfloat16>(p, out_dtype, st);
  return combine_to<__half>(p, out_dtype, st);
}
