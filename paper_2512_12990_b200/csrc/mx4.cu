// slicemoe_mx4_quantize / _dequantize / _pack / _unpack: values to microscaled 4-bit floats and back.
#include "mx4.cuh"

namespace slicemoe {

constexpr int kMxThreads = 256;

// Both ways a warp takes runs of 256 values of a row (eight a lane), kMxAhead of them one after the other, and asks for all before it uses
// the first.  Where a run begins is divided out once for all of them.  (One run at a time, with a 64-bit division for each: 15.6 us
// for 8,192 rows of 2,048 bf16 values, and 14.8 back; now 16.5 for both.)
constexpr int kMxAhead = 4;
struct MxRun {
  int64_t row;
  int c;  // first of the lane's eight values; K or above: none
  bool live;
};
__device__ __forceinline__ void mx_runs(int64_t first, int64_t rows, int per_row, int K, int lane, MxRun (&run)[kMxAhead]) {
  int64_t row = (first >> 31) ? first / per_row : (int64_t)((uint32_t)first / (uint32_t)per_row);
  int seg = (int)(first - row * per_row);
#pragma unroll
  for (int i = 0; i < kMxAhead; ++i) {
    run[i].row = row;
    run[i].c = seg * 256 + lane * 8;
    run[i].live = row < rows && run[i].c < K;
    if (++seg == per_row) seg = 0, ++row;
  }
}

// Eight values as they are loaded; the bits of the largest magnitude among them, as fp32; the values.
template <class T>
struct MxRaw;
template <>
struct MxRaw<float> {
  float4 a, b;
  __device__ __forceinline__ void load(const float* p) { a = __ldcg(reinterpret_cast<const float4*>(p)), b = __ldcg(reinterpret_cast<const float4*>(p) + 1); }
  __device__ __forceinline__ void values(float (&v)[8]) const { v[0] = a.x, v[1] = a.y, v[2] = a.z, v[3] = a.w, v[4] = b.x, v[5] = b.y, v[6] = b.z, v[7] = b.w; }
  __device__ __forceinline__ uint32_t largest() const {
    float v[8];
    values(v);
    uint32_t m = 0;
#pragma unroll
    for (int j = 0; j < 8; ++j) m = max(m, __float_as_uint(v[j]) & 0x7fffffffu);
    return m;
  }
};
template <class T>
struct MxRaw {  // 16 bits: two to a word
  uint4 a;
  __device__ __forceinline__ void load(const T* p) { a = __ldcg(reinterpret_cast<const uint4*>(p)); }
  __device__ __forceinline__ void values(float (&v)[8]) const {
    const uint32_t w[4] = {a.x, a.y, a.z, a.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      T e[2];
      memcpy(e, &w[i], 4);
      v[2 * i] = mx_to_float<T>(e[0]), v[2 * i + 1] = mx_to_float<T>(e[1]);
    }
  }
  __device__ __forceinline__ uint32_t largest() const {  // magnitudes order like their bits, infinities and NaN above all
    constexpr uint32_t kMag = 0x7fff7fffu;
    const uint32_t m = __vmaxu2(__vmaxu2(a.x & kMag, a.y & kMag), __vmaxu2(a.z & kMag, a.w & kMag));
    const unsigned short h = (unsigned short)max(m >> 16, m & 0xffffu);
    T e;
    memcpy(&e, &h, 2);
    return __float_as_uint(mx_to_float<T>(e)) & 0x7fffffffu;
  }
};

// A run whose row does not begin on 16 bytes: the warp loads it 32 neighbouring values at a time and swaps them about in shared memory.
template <class T>
struct MxScattered {
  T v[8];
  __device__ __forceinline__ void load(const T* run, int lane, int n) {  // n: values of the run that there are
#pragma unroll
    for (int q = 0; q < 8; ++q) {
      if (32 * q + lane >= n) continue;
      if constexpr (sizeof(T) == 4) {
        v[q] = __ldcg(run + 32 * q + lane);
      } else {
        const unsigned short h = __ldcg(reinterpret_cast<const unsigned short*>(run) + 32 * q + lane);
        memcpy(&v[q], &h, 2);
      }
    }
  }
  __device__ __forceinline__ MxRaw<T> gather(T* room, int lane, int n) const {
    MxRaw<T> raw;
    __syncwarp();
#pragma unroll
    for (int q = 0; q < 8; ++q)
      if (32 * q + lane < n) room[32 * q + lane] = v[q];
    __syncwarp();
    memcpy(&raw, __builtin_assume_aligned(room + 8 * lane, 16), sizeof(raw));
    return raw;
  }
};

// Four lanes hold a block of 32 values, eight each: the largest magnitude by two exchanges, then each lane writes the four bytes
// of its eight codes (a warp's stores are 128 consecutive bytes) and the first the scale.  LINEAR: the rows are one behind the other
// and whole runs, so that a place is a shift of a counter.  Bound: the values read.
template <class T, bool WIDE, bool LINEAR>
__global__ void __launch_bounds__(kMxThreads) mx_quantize_kernel(const T* __restrict__ x, int rows, int K, int64_t ld, uint8_t* __restrict__ codes,
                                                                 uint8_t* __restrict__ scale) {
  mx_dep_launch();
  mx_dep_wait();
  const int pitch = mx_pitch(K), blocks = K / kMxBlock, per_row = (K + 255) >> 8, lane = threadIdx.x & 31;
  const int64_t runs = (int64_t)rows * per_row, step = (int64_t)gridDim.x * (kMxThreads / 32) * kMxAhead;
  for (int64_t first = (((int64_t)blockIdx.x * kMxThreads + threadIdx.x) >> 5) * kMxAhead; first < runs; first += step) {
    MxRun run[kMxAhead];
    if constexpr (!LINEAR) mx_runs(first, rows, per_row, K, lane, run);
    const int64_t at = first * 256 + lane * 8;
    MxRaw<T> raw[kMxAhead];
    if constexpr (WIDE) {
#pragma unroll
      for (int i = 0; i < kMxAhead; ++i) {
        if constexpr (LINEAR) {
          if (first + i < runs) raw[i].load(x + at + 256 * i);
        } else if (run[i].live) {
          raw[i].load(x + run[i].row * ld + run[i].c);
        }
      }
    } else {
      __shared__ __align__(16) T room[kMxThreads / 32][256];
      MxScattered<T> loose[kMxAhead];
      int n[kMxAhead];
#pragma unroll
      for (int i = 0; i < kMxAhead; ++i) {  // the same row and run in all lanes
        const int c0 = run[i].c - lane * 8;
        n[i] = run[i].row < rows ? min(256, K - c0) : 0;
        loose[i].load(x + (n[i] > 0 ? run[i].row * ld + c0 : 0), lane, n[i]);
      }
#pragma unroll
      for (int i = 0; i < kMxAhead; ++i) raw[i] = loose[i].gather(room[threadIdx.x >> 5], lane, n[i]);
    }
#pragma unroll
    for (int i = 0; i < kMxAhead; ++i) {
      const bool live = LINEAR ? first + i < runs : run[i].live;
      uint32_t m = live ? raw[i].largest() : 0u;
      m = max(m, __shfl_xor_sync(0xffffffffu, m, 1));
      m = max(m, __shfl_xor_sync(0xffffffffu, m, 2));
      if (!live) continue;
      const uint32_t b = mx_scale_byte(m);
      float v[8];
      raw[i].values(v);
      const uint32_t w = b == 255u ? 0u : mx_encode8(v, mx_inverse(b));
      if constexpr (LINEAR) {
        *reinterpret_cast<uint32_t*>(codes + (at >> 1) + 128 * i) = w;
        if ((lane & 3) == 0) scale[(at >> 5) + 8 * i] = (uint8_t)b;
      } else {
        *reinterpret_cast<uint32_t*>(codes + run[i].row * (K >> 1) + (run[i].c >> 1)) = w;
        if ((lane & 3) == 0) {
          const int kb = run[i].c / kMxBlock;
          uint8_t* s = scale + run[i].row * pitch;
          s[kb] = (uint8_t)b;
          if (kb == blocks - 1)
            for (int p = blocks; p < pitch; ++p) s[p] = 0;
        }
      }
    }
  }
}

// The other way: a lane's eight codes are four bytes, what it writes 16 or 32.  LINEAR as above.  Bound: the values written.
template <class T, bool WIDE, bool LINEAR>
__global__ void __launch_bounds__(kMxThreads) mx_dequantize_kernel(const uint8_t* __restrict__ codes, const uint8_t* __restrict__ scale,
                                                                   int rows, int K, T* __restrict__ out, int64_t ld) {
  mx_dep_launch();
  mx_dep_wait();
  const int pitch = mx_pitch(K), per_row = (K + 255) >> 8, lane = threadIdx.x & 31;
  const int64_t runs = (int64_t)rows * per_row, step = (int64_t)gridDim.x * (kMxThreads / 32) * kMxAhead;
  for (int64_t first = (((int64_t)blockIdx.x * kMxThreads + threadIdx.x) >> 5) * kMxAhead; first < runs; first += step) {
    MxRun run[kMxAhead];
    if constexpr (!LINEAR) mx_runs(first, rows, per_row, K, lane, run);
    const int64_t at = first * 256 + lane * 8;
    uint32_t w[kMxAhead], b[kMxAhead];
#pragma unroll
    for (int i = 0; i < kMxAhead; ++i) {
      w[i] = b[i] = 0;
      if constexpr (LINEAR) {
        if (first + i < runs) {
          w[i] = __ldcg(reinterpret_cast<const uint32_t*>(codes + (at >> 1) + 128 * i));
          b[i] = __ldcg(scale + (at >> 5) + 8 * i);
        }
      } else if (run[i].live) {
        w[i] = __ldcg(reinterpret_cast<const uint32_t*>(codes + run[i].row * (K >> 1) + (run[i].c >> 1)));
        b[i] = __ldcg(scale + run[i].row * pitch + run[i].c / kMxBlock);
      }
    }
#pragma unroll
    for (int i = 0; i < kMxAhead; ++i) {
      if (LINEAR ? first + i >= runs : !run[i].live) continue;
      const float s = mx_scale_value(b[i]);
      float v[8];
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const float2 f = __half22float2(mx_decode2(w[i] >> (8 * j)));
        v[2 * j] = f.x * s;
        v[2 * j + 1] = f.y * s;
      }
      if constexpr (LINEAR) mx_store8<T, WIDE>(out + at + 256 * i, v);
      else mx_store8<T, WIDE>(out + run[i].row * ld + run[i].c, v);
    }
  }
}

// Pack: a thread per block of 32 values of a physical row, eight rows x four blocks a warp, so that reads are whole sectors and
// writes 128 consecutive bytes.  Rows and blocks beyond the matrix are written as zeros.
template <class T>
__global__ void __launch_bounds__(kMxThreads) mx_pack_kernel(const T* __restrict__ W, const T* __restrict__ up, int N, int K, int64_t ld,
                                                             uint8_t* __restrict__ codes, uint8_t* __restrict__ scale) {
  const int gated = up != nullptr;
  const int row = blockIdx.y * kMxRows + (threadIdx.x >> 5) * 8 + (threadIdx.x & 7);  // 8 warps: 64 rows; twice
  const int kb = blockIdx.x * 4 + ((threadIdx.x & 31) >> 3);
#pragma unroll 1
  for (int half = 0; half < 2; ++half) {
    const int r = row + half * 64;
    const T* src = W;
    int n = r;
    if (gated) {
      n = (r >> 5) * 16 + (r & 15);
      if (r & 16) src = up;
    }
    uint32_t w[4] = {0, 0, 0, 0}, b = 0;
    if (n < N && kb * kMxBlock < K) {
      const T* p = src + n * ld + (int64_t)kb * kMxBlock;
      float v[32];
#pragma unroll
      for (int j = 0; j < 32; ++j) v[j] = mx_to_float<T>(p[j]);
      uint32_t m = 0;
#pragma unroll
      for (int j = 0; j < 32; ++j) m = max(m, __float_as_uint(v[j]) & 0x7fffffffu);
      b = mx_scale_byte(m);
      const float inv = mx_inverse(b);
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        float e[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) e[j] = b == 255u ? 0.0f : v[8 * q + j];
        w[q] = mx_encode8(e, inv);
      }
    }
    if ((kb >> 1) < mx_chunks(K)) *reinterpret_cast<uint4*>(codes + mx_code_offset(K, r, kb)) = make_uint4(w[0], w[1], w[2], w[3]);
    scale[mx_scale_offset(K, r, kb)] = (uint8_t)b;
  }
}

__global__ void __launch_bounds__(kMxThreads) mx_unpack_kernel(const uint8_t* __restrict__ codes, const uint8_t* __restrict__ scale, int N, int K,
                                                               int gated, int part, uint8_t* __restrict__ codes_rm, uint8_t* __restrict__ scale_rm) {
  const int blocks = K / kMxBlock, pitch = mx_pitch(K);
  const int64_t n = (int64_t)N * pitch;
  for (int64_t i = (int64_t)blockIdx.x * kMxThreads + threadIdx.x; i < n; i += (int64_t)gridDim.x * kMxThreads) {
    const int row = (int)(i / pitch), kb = (int)(i % pitch);
    const int r = gated ? (row >> 4) * 32 + (row & 15) + 16 * part : row;
    uint8_t b = 0;
    if (kb < blocks) {
      b = scale[mx_scale_offset(K, r, kb)];
      *reinterpret_cast<uint4*>(codes_rm + (int64_t)row * (K >> 1) + 16 * kb) = *reinterpret_cast<const uint4*>(codes + mx_code_offset(K, r, kb));
    }
    scale_rm[i] = b;
  }
}

static int mx_grid(int64_t threads) {
  const int64_t b = (threads + kMxThreads - 1) / kMxThreads;
  return (int)(b < 148 * 64 ? b : 148 * 64);
}

// Blocks for all runs of a matrix; 0: more than a grid holds.
static unsigned mx_run_blocks(int rows, int K) {
  constexpr int kRuns = kMxThreads / 32 * kMxAhead;
  const int64_t b = ((int64_t)rows * ((K + 255) >> 8) + kRuns - 1) / kRuns;
  return b <= INT32_MAX ? (unsigned)b : 0u;
}

template <class T>
static int quantize_as(const void* x, int rows, int K, int64_t ld, uint8_t* codes, uint8_t* scale, cudaStream_t st) {
  const bool wide = mx_aligned(x, 16) && (ld * sizeof(T)) % 16 == 0;
  const unsigned blocks = mx_run_blocks(rows, K);
  if (!blocks) return SLICEMOE_E_UNSUPPORTED;
  const auto kernel = wide && ld == K && K % 256 == 0 ? mx_quantize_kernel<T, true, true> : wide ? mx_quantize_kernel<T, true, false> : mx_quantize_kernel<T, false, false>;
  return mx_launch(kernel, dim3(blocks < 148 * 8 ? blocks : 148 * 8), kMxThreads, 0, st, static_cast<const T*>(x), rows, K, ld, codes, scale);
}
template <class T>
static int dequantize_as(const uint8_t* codes, const uint8_t* scale, int rows, int K, void* out, int64_t ld, cudaStream_t st) {
  const bool wide = mx_aligned(out, 16) && (ld * sizeof(T)) % 16 == 0;
  const unsigned blocks = mx_run_blocks(rows, K);
  if (!blocks) return SLICEMOE_E_UNSUPPORTED;
  const auto kernel = wide && ld == K && K % 256 == 0 ? mx_dequantize_kernel<T, true, true> : wide ? mx_dequantize_kernel<T, true, false> : mx_dequantize_kernel<T, false, false>;
  return mx_launch(kernel, dim3(blocks < 148 * 8 ? blocks : 148 * 8), kMxThreads, 0, st, codes, scale, rows, K, static_cast<T*>(out), ld);
}

static int mx_check(const void* x, int dtype, int rows, int K, int64_t ld, const void* codes, const void* scale) {
  if (!x || !codes || !scale || rows <= 0 || K <= 0 || K % kMxBlock || ld < K) return SLICEMOE_E_INVALID_ARG;
  if (K > kMxMaxRow || !mx_dtype(dtype)) return SLICEMOE_E_UNSUPPORTED;
  if (!mx_aligned(x, mx_elem(dtype)) || !mx_aligned(codes, 16) || !mx_aligned(scale, 4)) return SLICEMOE_E_INVALID_ARG;
  return SLICEMOE_OK;
}

}  // namespace slicemoe

using namespace slicemoe;

extern "C" size_t slicemoe_mx4_scale_pitch(int K) { return K > 0 && K <= kMxMaxRow ? (size_t)mx_pitch(K) : 0; }

extern "C" int slicemoe_mx4_quantize(const void* x, int dtype, int rows, int K, int64_t ld, uint8_t* codes, uint8_t* scale, void* stream) {
  const int rc = mx_check(x, dtype, rows, K, ld, codes, scale);
  if (rc != SLICEMOE_OK) return rc;
  cudaStream_t st = (cudaStream_t)stream;
  if (dtype == SLICEMOE_F32) return quantize_as<float>(x, rows, K, ld, codes, scale, st);
  if (dtype == SLICEMOE_BF16) return quantize_as<__nv_bfloat16>(x, rows, K, ld, codes, scale, st);
  return quantize_as<__half>(x, rows, K, ld, codes, scale, st);
}

extern "C" int slicemoe_mx4_dequantize(const uint8_t* codes, const uint8_t* scale, int rows, int K, void* out, int dtype, int64_t ld, void* stream) {
  const int rc = mx_check(out, dtype, rows, K, ld, codes, scale);
  if (rc != SLICEMOE_OK) return rc;
  cudaStream_t st = (cudaStream_t)stream;
  if (dtype == SLICEMOE_F32) return dequantize_as<float>(codes, scale, rows, K, out, ld, st);
  if (dtype == SLICEMOE_BF16) return dequantize_as<__nv_bfloat16>(codes, scale, rows, K, out, ld, st);
  return dequantize_as<__half>(codes, scale, rows, K, out, ld, st);
}

static bool mx_sizes(int N, int K) { return N > 0 && K > 0 && K % kMxBlock == 0 && N <= kMxMaxN && K <= kMxMaxK; }

extern "C" size_t slicemoe_mx4_codes_bytes(int N, int K, int gated) {
  return mx_sizes(N, K) ? (size_t)mx_row_blocks(N, gated) * mx_chunks(K) * kMxChunkBytes : 0;
}
extern "C" size_t slicemoe_mx4_scale_bytes(int N, int K, int gated) {
  return mx_sizes(N, K) ? (size_t)mx_row_blocks(N, gated) * mx_atoms(K) * kMxAtomBytes : 0;
}

extern "C" int slicemoe_mx4_pack(const void* W, const void* up, int dtype, int N, int K, int64_t ld, uint8_t* codes, uint8_t* scale, void* stream) {
  const int rc = mx_check(W, dtype, N, K, ld, codes, scale);
  if (rc != SLICEMOE_OK) return rc;
  if (up && !mx_aligned(up, mx_elem(dtype))) return SLICEMOE_E_INVALID_ARG;
  if (!mx_aligned(scale, 16)) return SLICEMOE_E_INVALID_ARG;
  if (!mx_sizes(N, K)) return SLICEMOE_E_UNSUPPORTED;
  const dim3 grid(mx_atoms(K), mx_row_blocks(N, up != nullptr));
  static_assert(2ll * kMxMaxN / kMxRows + 1 <= 65535, "row blocks in a grid's second dimension");
  cudaStream_t st = (cudaStream_t)stream;
  if (dtype == SLICEMOE_F32)
    mx_pack_kernel<float><<<grid, kMxThreads, 0, st>>>(static_cast<const float*>(W), static_cast<const float*>(up), N, K, ld, codes, scale);
  else if (dtype == SLICEMOE_BF16)
    mx_pack_kernel<__nv_bfloat16><<<grid, kMxThreads, 0, st>>>(static_cast<const __nv_bfloat16*>(W), static_cast<const __nv_bfloat16*>(up), N, K, ld,
                                                               codes, scale);
  else
    mx_pack_kernel<__half><<<grid, kMxThreads, 0, st>>>(static_cast<const __half*>(W), static_cast<const __half*>(up), N, K, ld, codes, scale);
  SM_LAUNCH_CHECK();
  return SLICEMOE_OK;
}

extern "C" int slicemoe_mx4_unpack(const uint8_t* codes, const uint8_t* scale, int N, int K, int gated, int part, uint8_t* codes_rm,
                                   uint8_t* scale_rm, void* stream) {
  if (!codes || !scale || !codes_rm || !scale_rm || N <= 0 || K <= 0 || K % kMxBlock || part < 0 || part > (gated ? 1 : 0)) return SLICEMOE_E_INVALID_ARG;
  if (!mx_aligned(codes, 16) || !mx_aligned(codes_rm, 16)) return SLICEMOE_E_INVALID_ARG;
  if (!mx_sizes(N, K)) return SLICEMOE_E_UNSUPPORTED;
  mx_unpack_kernel<<<mx_grid((int64_t)N * mx_pitch(K)), kMxThreads, 0, (cudaStream_t)stream>>>(codes, scale, N, K, gated, part, codes_rm, scale_rm);
  SM_LAUNCH_CHECK();
  return SLICEMOE_OK;
}
